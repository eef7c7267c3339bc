"""Every form of the 8-bit products, with every type and epilogue, against 64 bits, element by element with the bounds of operators_bounds.py (which
test_product_bounds_cpu.py holds against planted mistakes)."""
import ctypes as C
import math

import pytest
import torch

import operators_bounds as ob
import paper_2009_08065_amd as bsp

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TAG = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
D = torch.float64
U = ob.U


def rand(seed, *shape, std=1.0, dt=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dt)


def inside(got, want, bound, what=""):
    assert got.shape == want.shape, what
    err = (got.to(want) - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float((err / bound).nan_to_num(0, 0, 0).max()):.3g} of what is allowed"


def held(q):
    """The matrix that codes and scales stand for, in 64 bits."""
    s = torch.pow(torch.tensor(2.0, dtype=D, device="cuda"), q.scales.to(D) - 127)
    if q.layout == bsp.FP8_BLOCK:
        s = s.repeat_interleave(128, 0)[:q.rows]
    return (q.codes.to(torch.float32).to(D) * s.repeat_interleave(128, 1))[:, :q.cols].contiguous()


# ---- forms of the products ----------------------------------------------------------------------------------------------------
def form(T, M, K, dt, act):
    v = [C.c_int32() for _ in range(3)]
    assert bsp.lib().bsp_matmul_fp8_form(T, M, K, TAG[dt], act, *(C.byref(x) for x in v)) == 0
    return tuple(x.value for x in v)


FORMS = {"256": (256, 2), "128": (128, 2), "128 three deep": (128, 3), "64": (64, 2), "64 four deep": (64, 4)}


def sizes(name, dt, act, steps, odd):
    """Sizes whose product takes the form, no multiples of its tile, the fewest outputs first: they are looked for, so that an estimate that is fitted again
    moves the test and does not empty it."""
    found = []
    for T in (int(37 * 1.19 ** i) | 1 for i in range(36)):
        for m in (int(5 * 1.16 ** i) * 8 for i in range(34)):
            M = m + 1 if odd else m + 8 * (m % 64 == 0)
            if T * M <= 24e6 and form(T, M, 128 * steps - 50, dt, act)[:2] == FORMS[name]:
                found.append((T * M, T, M))
    return min(found)[1:] if found else None


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("name", FORMS)
def test_every_form_of_the_products(name, gelu, dtype):
    """From the fewest steps that take the form (its ring of steps is not full then) to many; odd widths and whole vectors; a scale per block and per row;
    results between other data, beside a bias, in the residual's place, at an address of the element only."""
    dt, act = DT[dtype], bsp.ACT_GELU if gelu else bsp.ACT_NONE
    cases = []
    for odd in (True, False):
        for steps in (1, 2, 3, 4, 5, 6, 7, 9, 12, 17, 24):
            at = sizes(name, dt, act, steps, odd)
            if at:
                cases.append((odd, steps, *at))
    assert any(c[0] for c in cases) and any(not c[0] for c in cases), "no size takes this form"
    few = [next(c for c in cases if c[0] == odd) for odd in (True, False)]
    for odd, steps, T, M in few + [c for c in cases if c[1] in (3, 6, 17) and (c[1], c[0]) in ((3, True), (6, False), (17, True)) and c not in few]:
        K = 128 * steps - 50
        what = f"{name} {dtype} T={T} M={M} K={K} gelu={gelu}"
        assert form(T, M, K, dt, act)[:2] == FORMS[name]
        a, b = rand(T + K, T, K), rand(M + K, M, K, std=1 / math.sqrt(K))
        a[:, : K // 7] *= 8.0                           # segments of different scales
        b[M // 2] *= 1e-2
        layout = bsp.FP8_BLOCK if odd else bsp.FP8_ROW
        A, B = bsp.bsp_fp8_quant(a)[0], bsp.bsp_fp8_quant(b, layout)[0]
        av, bv = held(A), held(B)
        s, bias, res = av @ bv.t(), rand(5, M, dt=dt), rand(6, T, M, dt=dt)
        for bi, re, shift in ((None, None, 0), (bias, None, 0), (bias, res, 0), (None, res, 1)):
            want, bound = ob.layer(s, ob.product(av, bv, dt), dt, bi, act, re)
            room = torch.full((T * M + 64,), 7.0, dtype=dt, device="cuda")
            y = room[16 + shift:16 + shift + T * M].view(T, M)
            if re is not None:
                y.copy_(re)                             # the residual's place is the result's
            bsp.bsp_matmul_fp8(A, B, bi, act=act, residual=None if re is None else y, Y=y)
            inside(y, want, bound, what)
            assert (room[:16 + shift] == 7).all() and (room[16 + shift + T * M:] == 7).all(), what
            if re is None:
                assert torch.equal(y, bsp.bsp_matmul_fp8(A, B, bi, act=act, out_dtype=dt)), what
        lost = torch.linalg.vector_norm(bsp.bsp_matmul_fp8(A, B, out_dtype=dt).to(D) - s) / torch.linalg.vector_norm(s) if not gelu else 0.0
        # N(0, 1) operands: the type's rounding, and 1.3e-5 of the result where the instruction on codes is used (2^-16 is 1.5e-5)
        assert float(lost) <= (2.0 ** -21 if dt == torch.float32 else ob.half(dt) + 2.0 ** -16), what


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("K", [1000, 8192])
def test_forms_that_split_the_columns(K, dtype):
    """The runs' sums are joined with bias, activation and residual."""
    dt, seen = DT[dtype], set()
    for T in (34, 70, 130, 260):
        for M in (33, 136, 1040):
            for act in (bsp.ACT_NONE, bsp.ACT_GELU):
                splits = form(T, M, K, dt, act)[2]
                if splits == 1:
                    continue
                seen.add(splits)
                A, B = bsp.bsp_fp8_quant(rand(T, T, K))[0], bsp.bsp_fp8_quant(rand(M, M, K, std=1 / math.sqrt(K)))[0]
                av, bv = held(A), held(B)
                bias, res = rand(5, M, dt=dt), rand(6, T, M, dt=dt)
                want, bound = ob.layer(av @ bv.t(), ob.product(av, bv, dt), dt, bias, act, res)
                y = res.clone()
                inside(bsp.bsp_matmul_fp8(A, B, bias, act=act, residual=y, Y=y), want, bound, f"T={T} M={M} splits={splits}")
    assert seen or K < 4096


# ---- the ends of the range ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 16, 32, 40, 300])
def test_a_mask_of_the_types_lowest_value_stays_finite(T, dtype):
    """The least finite values as inputs: their codes stand for numbers of fp32, so that beside weights of 0 (pruned ones, or gradients of masked tokens) a product
    is what the other columns give."""
    dt, M, N = DT[dtype], 48, 300
    x, w = rand(1, T, N, dt=dt), rand(2, M, N, std=0.05, dt=dt)
    low = torch.finfo(dt).min
    x[:, 7], x[:, 8], x[0, 130] = low, -low, low
    x[:, 9], x[:, 10] = 1.9374 * 2.0 ** 127, 1.9376 * 2.0 ** 127   # to the two sides of 248 of the scale (bf16: 1.9375 itself, a tie)
    w[:, 7:11], w[:, 130] = 0, 0
    for layout in (bsp.FP8_ROW, bsp.FP8_BLOCK):
        X, Xt = bsp.bsp_fp8_quant(x, layout, want=("plain", "transposed"))
        W = bsp.bsp_fp8_quant(w, layout)[0]
        for q, cols in ((X, slice(7, 11)), (Xt, None)):
            c = (q.codes.view(torch.uint8)[:, cols] if cols else q.codes.view(torch.uint8)[7:11].t()[:T]) & 127
            assert (c == 0x77).all() and q.codes.float().isfinite().all()
            codes, scales = ob.quant((x if cols else x.t()).cpu().to(D), layout == bsp.FP8_BLOCK)
            assert torch.equal(q.codes.view(torch.uint8).cpu(), codes) and torch.equal(q.scales.cpu(), scales)
        assert (X.scales.max() == 247) and held(X).abs().max() == 240 * 2.0 ** 120
        if layout == bsp.FP8_ROW:
            xv, wv = held(X), held(W)
            want = xv @ wv.t()
            assert want.abs().max() < 1e3
            y = bsp.bsp_matmul_fp8(X, W, out_dtype=torch.float32)
            assert y.isfinite().all() and torch.equal(bsp.bsp_linear_fp8(x, W), bsp.bsp_matmul_fp8(X, W, out_dtype=dt))
            inside(y, want, (N + 8) * U * (xv.abs() * (xv.abs() < 1e30)) @ wv.abs().t() + 1e-30)
            # the gradient of the weights, where the masked tokens' gradients are zero
            dy = rand(3, T, M, dt=dt)
            dy[0] = 0
            only = rand(4, T, N, dt=dt)
            only[0] = low
            D8, O8 = (bsp.bsp_fp8_quant(t, want=("transposed",))[1] for t in (dy, only))
            assert bsp.bsp_matmul_fp8(D8, O8, out_dtype=torch.float32).isfinite().all()


@pytest.mark.parametrize("T", [1, 40])
def test_values_of_fp32_results_far_below(T):
    """fp32 results have their operands as bfloat16: exact while they are whole multiples of 2^-133, and of those below it what is whole."""
    M, K = 24, 128
    for e in (-100, -118, -124, -130):
        a, b = torch.zeros(T, K, device="cuda"), torch.zeros(M, K, device="cuda")
        a[:, 0], a[:, 1] = 1.75 * 2.0 ** e, 1.5 * 2.0 ** (e - 1)
        b[:, 0], b[:, 1] = 2.0 ** 60, 2.0 ** 62
        y = bsp.bsp_matmul_fp8(bsp.bsp_fp8_quant(a)[0], bsp.bsp_fp8_quant(b)[0], out_dtype=torch.float32)
        assert torch.equal(y, torch.full_like(y, 1.75 * 2.0 ** (e + 60) + 1.5 * 2.0 ** (e + 61))), e


# ---- products that cancel -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [1, 20, 40, 300])
def test_products_that_cancel(T, dtype):
    """Columns in pairs of opposite sign, one small product left in each output, away from the pairs and among them: fp32 results have it to the last bits
    of the sum's magnitude; of 16-bit results what is off goes by the largest products of eight columns, not by the result."""
    dt, M, K = DT[dtype], 72, 520
    a, b = torch.zeros(T, K, device="cuda"), torch.zeros(M, K, device="cuda")
    big, w = rand(1, T, 250), rand(2, M, 250)
    a[:, 0:500:2], a[:, 1:500:2] = big, -big
    b[:, 0:500:2], b[:, 1:500:2] = w, w
    a[:, 510], b[:, 510] = 2.0 ** -5, 2.0 ** -4     # codes under the segments' scales; columns 504 to 511 hold nothing else
    A, B = bsp.bsp_fp8_quant(a)[0], bsp.bsp_fp8_quant(b)[0]
    av, bv = held(A), held(B)
    want = av @ bv.t()
    assert torch.equal(want, torch.full_like(want, 2.0 ** -9))
    y = bsp.bsp_matmul_fp8(A, B, out_dtype=dt)
    inside(y, want, ob.rounded_to(dt, want, ob.product(av, bv, dt)))
    a[:, 510] = 0.0
    a[:, 3], b[:, 3] = a[:, 3] + 2.0 ** -3, b[:, 3]  # now the rest of a pair
    A, B = bsp.bsp_fp8_quant(a)[0], bsp.bsp_fp8_quant(b)[0]
    av, bv = held(A), held(B)
    want = av @ bv.t()
    inside(bsp.bsp_matmul_fp8(A, B, out_dtype=dt), want, ob.rounded_to(dt, want, ob.product(av, bv, dt)))


@pytest.mark.parametrize("T,M,K", [(100, 64, 8192), (200, 130, 4096), (300, 1000, 300), (5, 64, 1024)])
def test_products_in_scratch_of_the_callers_own(T, M, K):
    """The bits of the call that allocates, whatever the scratch holds before; without any bytes the columns are not split; too few are refused."""
    A, B = bsp.bsp_fp8_quant(rand(1, T, K))[0], bsp.bsp_fp8_quant(rand(2, M, K))[0]
    need = bsp.lib().bsp_matmul_fp8_workspace_bytes(T, M, K)
    for dt in DT.values():
        want = bsp.bsp_matmul_fp8(A, B, out_dtype=dt)
        ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
        for _ in range(2):
            assert torch.equal(bsp.bsp_matmul_fp8(A, B, out_dtype=dt, ws=ws[:need] if need else ws), want)
        assert (ws[need:] == 255).all()
        av, bv = held(A), held(B)
        s = av @ bv.t()
        inside(bsp.bsp_matmul_fp8(A, B, out_dtype=dt, ws=ws[:0]), s, ob.rounded_to(dt, s, ob.product(av, bv, dt)))
    if need:
        with pytest.raises(bsp.BspError):
            bsp.bsp_matmul_fp8(A, B, ws=ws[:need - 1])
    for bad in (ws.cpu(), ws[::2], 3):
        with pytest.raises((ValueError, TypeError)):
            bsp.bsp_matmul_fp8(A, B, ws=bad)
