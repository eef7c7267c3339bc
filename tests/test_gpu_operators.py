"""8-bit products, the norms round a block and AdamW over many tensors on the GPU, against the plain implementations in 64 bits.

Tolerances: a rounding is off by half a step at most, eps / 2 of the value for a type's eps; an fp32 sum of n terms in any order by
(n - 1) 2^-24 times the sum of their magnitudes.  What a test allows is the sum of these for what its kernel computes, and is written
beside it."""
import math

import pytest
import torch

import operators_oracle as orc
import paper_2009_08065_amd as bsp

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
D = torch.float64
U = 2.0 ** -24


def half(dt):
    return torch.finfo(dt).eps / 2


def rand(seed, *shape, std=1.0, dt=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dt)


def off_by_one(t):
    """The same values at an address that is a multiple of the element only."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
    view = flat[1:].view(t.shape)
    view.copy_(t)
    return view


def inside(got, want, bound):
    assert got.shape == want.shape
    err = (got.detach().cpu().to(D) - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside, worst {float((err / bound).nan_to_num(0, 0, 0).max()):.3g} of what is allowed"


# ---- 8-bit floating point -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 130), (128, 256), (129, 127), (77, 690), (260, 520)])
@pytest.mark.parametrize("aligned", [True, False])
def test_quant(dtype, rows, cols, aligned):
    """Codes and scales are those of the definition, in either orientation: nothing in them is off by a rounding."""
    x = rand(rows + cols, rows, cols, dt=DT[dtype])
    x[0] *= 100.0
    x[-1] = 0.0                                     # a row without a value
    x[:, cols // 2] *= 2.0 ** -12                   # far below its neighbours: subnormal codes and zeros
    if cols > 20:
        x[0, 1], x[0, 2], x[0, 3], x[0, 4] = math.nan, math.inf, -math.inf, -0.0
        x[1 % rows, 5:14] = torch.tensor([448.0, 26.0, 27.0, 25.0, 17.0, 19.0, -21.0, 2.0 ** -9, 1.5 * 2.0 ** -9]).to(x.dtype)   # ties
    if dtype == "f32" and rows > 2:
        x[1, :] = 2.0 ** -140                       # the least scale
        x[2, 0] = 3e38                              # the greatest
    xd = x.cuda() if aligned else off_by_one(x.cuda())
    for layout, block in ((bsp.FP8_ROW, False), (bsp.FP8_BLOCK, True)):
        p, t = bsp.bsp_fp8_quant(xd, layout, want=("plain", "transposed"))
        only, none = bsp.bsp_fp8_quant(xd, layout)
        assert none is None
        for q, ref in ((p, x), (only, x), (t, x.t())):
            codes, scales = orc.quant(ref.to(D), block)
            got = q.codes.view(torch.uint8).cpu()
            nan = (codes & 127) == 127
            assert torch.equal((got & 127) == 127, nan) and torch.equal(got[~nan], codes[~nan])
            assert torch.equal(q.scales.cpu(), scales)
    # no row behind the last one is written
    alone, none = bsp.bsp_fp8_quant(xd, bsp.FP8_ROW, want=("transposed",))
    assert alone is None and torch.equal(none.codes.view(torch.uint8), bsp.bsp_fp8_quant(x.cuda().t().contiguous())[0].codes.view(torch.uint8))


def fp8_bound(a, b, dt, more=0.0):
    """Allowed for a product of quantised matrices.  fp32: K exact products in chains of fp32 additions.  16 bits: what the
    instruction drops, 2^-13 of the largest product it adds at once (13 binades below it are kept), for each product at most,
    and the rounding of the result."""
    K = a.shape[1]
    sums = a.abs() @ b.abs().t()
    if dt == torch.float32:
        return (K + 8) * U * (sums + more) + 1e-40
    worst = torch.zeros_like(sums)
    for k in range(0, K, 128):
        worst += 128 * 2.0 ** -13 * a[:, k:k + 128].abs().amax(1)[:, None] * b[:, k:k + 128].abs().amax(1)[None, :]
    return worst + (K + 8) * U * (sums + more)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,M,K", [(1, 1, 1), (1, 16, 128), (1, 300, 1000), (5, 7, 130), (16, 100, 700), (17, 129, 257), (33, 64, 256), (64, 65, 1000), (129, 257, 384),
                                   (300, 700, 1100), (1030, 520, 640), (2000, 1100, 130), (64, 64, 8192), (40, 200, 5000)])
def test_matmul(dtype, T, M, K):
    dt = DT[dtype]
    a, b = rand(T + K, T, K), rand(M + K + 1, M, K, std=0.05)
    a[:, : (K + 9) // 10] *= 30.0                   # segments of different scales
    b[M // 2] *= 1e-3
    for layout, block in ((bsp.FP8_ROW, False), (bsp.FP8_BLOCK, True)):
        A, B = bsp.bsp_fp8_quant(a.cuda())[0], bsp.bsp_fp8_quant(b.cuda(), layout)[0]
        av, bv = orc.value(*orc.quant(a.to(D), False), K, False), orc.value(*orc.quant(b.to(D), block), K, block)
        want = av @ bv.t()
        y = bsp.bsp_matmul_fp8(A, B, out_dtype=dt)
        bound = fp8_bound(av, bv, dt)
        inside(y, want, half(dt) * (want.abs() + bound) + bound)
        # in the 2-norm: the rounding to the type, and 2^-13 where the 8-bit instruction is used (1.3e-5 was seen of one)
        rel = float((y.cpu().to(D) - want).norm() / want.norm())
        assert rel <= (2.0 ** -20 if dt == torch.float32 else half(dt) + 2.0 ** -13), rel
        assert torch.equal(y, bsp.bsp_matmul_fp8(A, B, out_dtype=dt))


@pytest.mark.parametrize("T,M,K", [(70, 2900, 300), (450, 2000, 640), (2000, 66, 500), (65, 65, 70), (1100, 1300, 200)])
def test_matmul_tiles_that_no_eight_share_evenly(T, M, K):
    a, b = rand(T + K, T, K), rand(M + K + 1, M, K, std=0.05)
    A, B = bsp.bsp_fp8_quant(a.cuda())[0], bsp.bsp_fp8_quant(b.cuda(), bsp.FP8_BLOCK)[0]
    av, bv = orc.value(*orc.quant(a.to(D), False), K, False), orc.value(*orc.quant(b.to(D), True), K, True)
    want = av @ bv.t()
    for dt in (torch.bfloat16, torch.float32):
        bound = fp8_bound(av, bv, dt)
        y = torch.full((T, M), math.nan, dtype=dt, device="cuda")
        inside(bsp.bsp_matmul_fp8(A, B, Y=y), want, half(dt) * (want.abs() + bound) + bound)
        r = rand(7, T, M, dt=dt).cuda()
        both = want + r.cpu().to(D)
        mine = r.clone()                             # the residual's place is the result's
        inside(bsp.bsp_matmul_fp8(A, B, residual=mine, Y=mine), both, half(dt) * (both.abs() + bound) + bound + U * want.abs())


@pytest.mark.parametrize("T,M", [(3500, 3600), (4100, 2900)])
def test_matmul_large_tiles(T, M):
    """Sizes of the largest tile, ragged in both directions; rows and columns at the borders of tiles among those compared."""
    K = 300
    a, b = rand(1, T, K), rand(2, M, K)
    A, B = bsp.bsp_fp8_quant(a.cuda())[0], bsp.bsp_fp8_quant(b.cuda(), bsp.FP8_BLOCK)[0]
    rows = torch.tensor([0, 31, 32, 63, 127, 128, 255, 256, 1023, 2047, T - 300, T - 1])
    av, bv = orc.value(*orc.quant(a[rows].to(D), False), K, False), orc.value(*orc.quant(b.to(D), True), K, True)
    want = av @ bv.t()
    for dt in (torch.float32, torch.bfloat16):
        y = bsp.bsp_matmul_fp8(A, B, out_dtype=dt)
        bound = fp8_bound(av, bv, dt)
        inside(y.cpu()[rows], want, half(dt) * (want.abs() + bound) + bound)
        # every other row against the product of single precision
        full = torch.from_numpy(orc.value(A.codes.view(torch.uint8).cpu(), A.scales.cpu(), K, False).numpy()).float().cuda() @ bv.float().t().cuda()
        assert float((y.float() - full).norm() / full.norm()) <= half(dt) + 2.0 ** -13


def test_matmul_rows_behind_the_last_and_padding():
    """Nothing is written outside [T, M], and a K that ends inside a segment adds nothing beyond it."""
    T, M, K = 37, 45, 200
    a, b = rand(5, T, K), rand(6, M, K)
    A, B = bsp.bsp_fp8_quant(a.cuda())[0], bsp.bsp_fp8_quant(b.cuda())[0]
    for dt in DT.values():
        buf = torch.full((T * M + 512,), 7.0, dtype=dt, device="cuda")
        y = buf[256:256 + T * M].view(T, M)
        bsp.bsp_matmul_fp8(A, B, Y=y)
        assert (buf[:256] == 7).all() and (buf[256 + T * M:] == 7).all()
        assert torch.equal(y, bsp.bsp_matmul_fp8(A, B, out_dtype=dt))


@pytest.mark.parametrize("T,M,K", [(100, 64, 8192), (200, 130, 4096), (70, 64, 16384)])
def test_matmul_split(T, M, K):
    """Products of few outputs and many columns, with the scratch (the columns split) and without."""
    a, b = rand(7, T, K), rand(8, M, K)
    A, B = bsp.bsp_fp8_quant(a.cuda())[0], bsp.bsp_fp8_quant(b.cuda())[0]
    av, bv = orc.value(*orc.quant(a.to(D), False), K, False), orc.value(*orc.quant(b.to(D), False), K, False)
    want = av @ bv.t()
    bound = fp8_bound(av, bv, torch.float32)
    y = torch.empty(T, M, device="cuda")
    st = bsp.lib().bsp_matmul_fp8(A.codes.data_ptr(), A.scales.data_ptr(), B.codes.data_ptr(), B.scales.data_ptr(), 0, T, M, K, None, 0, None,
                                  y.data_ptr(), 0, None, 0, torch.cuda.current_stream().cuda_stream)
    assert st == 0
    inside(y, want, bound)
    inside(bsp.bsp_matmul_fp8(A, B, out_dtype=torch.float32), want, bound)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,M,N", [(1, 256, 512), (3, 77, 690), (16, 1024, 256), (31, 130, 128), (333, 1111, 690), (1500, 520, 300)])
@pytest.mark.parametrize("aligned", [True, False])
def test_layer_with_its_epilogue(dtype, T, M, N, aligned):
    dt = DT[dtype]
    x, w = rand(T, T, N, dt=dt), rand(M, M, N, std=0.05, dt=dt)
    bias, res = rand(3, M, std=0.5, dt=dt), rand(4, T, M, dt=dt)
    place = (lambda t: t.cuda()) if aligned else (lambda t: off_by_one(t.cuda()))
    W = bsp.bsp_fp8_quant(w.cuda(), bsp.FP8_BLOCK)[0]
    xd, bd, rd = place(x), place(bias), place(res)
    xv, wv = orc.value(*orc.quant(x.to(D), False), N, False), orc.value(*orc.quant(w.to(D), True), N, True)
    s = xv @ wv.t()
    for b, act, r in ((None, bsp.ACT_NONE, None), (bd, bsp.ACT_NONE, None), (bd, bsp.ACT_GELU, None), (bd, bsp.ACT_GELU, rd), (None, bsp.ACT_NONE, rd)):
        want = s + (bias.to(D) if b is not None else 0)
        bound = fp8_bound(xv, wv, dt, want.abs())
        if act:
            # GELU's slope is at most 1.13; its fit is off by 3e-8 of N(0, 1) values in the 2-norm, 2e-7 at most absolutely
            want, bound = orc.gelu(want), 1.13 * bound + 2e-7 + 4 * U * want.abs()
        want = want + (res.to(D) if r is not None else 0)
        y = bsp.bsp_linear_fp8(xd, W, b, act=act, residual=r)
        inside(y, want, half(dt) * (want.abs() + bound) + bound + U * want.abs())
        two = bsp.bsp_matmul_fp8(bsp.bsp_fp8_quant(xd)[0], W, b, act=act, residual=r, out_dtype=dt)
        assert torch.equal(y, two)
    buf = off_by_one(torch.zeros(T, M, dtype=dt, device="cuda"))
    assert bsp.bsp_linear_fp8(xd, W, bd, Y=buf) is buf and torch.equal(buf, bsp.bsp_linear_fp8(xd, W, bd))


def test_layer_of_pruned_weights_and_what_is_not_finite():
    """The masked matrix: pruned positions are code 0.  A NaN reaches its row's outputs and no other row."""
    T, M, N, R = 70, 256, 512, 16
    x, w = rand(1, T, N, dt=torch.bfloat16).cuda(), rand(2, M, N, std=0.05, dt=torch.bfloat16).cuda()
    sumsq, _, _ = bsp.bsp_group_norms(w, R, want=("sumsq",))
    keep, _ = bsp.bsp_prune_mask(sumsq, n_keep=sumsq.numel() // 3, scope=bsp.SCOPE_MATRIX)
    bsp.bsp_mask_weights(w, R, keep)
    W = bsp.bsp_fp8_quant(w, bsp.FP8_BLOCK)[0]
    assert not W.codes.view(torch.uint8)[(w == 0)].logical_and(torch.tensor(127, device="cuda", dtype=torch.uint8)).any()
    y = bsp.bsp_linear_fp8(x, W)
    dense = x.float() @ w.float().t()
    assert float((y.float() - dense).norm() / dense.norm()) < 2.0 ** -4      # two operands rounded by at most 2^-4 each, independently
    x[5, 7] = math.nan
    z = bsp.bsp_linear_fp8(x, W)
    assert torch.isnan(z[5]).all() and torch.equal(z[:5], y[:5]) and torch.equal(z[6:], y[6:])


# ---- the norms round a block --------------------------------------------------------------------------------------------------
def norm_inputs(seed, T, H, dt, gate_rows, aligned=True):
    place = (lambda t: t.cuda()) if aligned else (lambda t: off_by_one(t.cuda()))
    c = dict(x=rand(seed, T, H, dt=dt), f=rand(seed + 1, T, H, std=0.5, dt=dt), gate=rand(seed + 2, gate_rows, H, std=0.5, dt=dt) if gate_rows else None,
             w_post=1 + rand(seed + 3, H, std=0.1), b_post=rand(seed + 4, H, std=0.1), w_pre=1 + rand(seed + 5, H, std=0.1), b_pre=rand(seed + 6, H, std=0.1),
             dz=rand(seed + 7, T, H, dt=dt), dh=rand(seed + 8, T, H, dt=dt))
    c = {k: None if v is None else v.to(dt) for k, v in c.items()}
    return c, {k: None if v is None else place(v) for k, v in c.items()}


WIDTHS = [1, 7, 64, 130, 512, 513, 770, 1024, 1500, 2048, 2056, 4096, 5000, 8192]


def check_norm(T, H, dt, rms, post, pre, gate_rows, x_scale=0.8, weights=True, aligned=True, offset=0.0):
    c, g = norm_inputs(T + H, T, H, dt, gate_rows, aligned)
    if offset:
        for k in "xf":
            c[k] = (c[k].float() + offset).to(dt)
            g[k].copy_(c[k])
    if not weights:
        for k in ("w_post", "b_post", "w_pre", "b_pre"):
            c[k] = g[k] = None
    norms = (bsp.NORM_POST if post else 0) | (bsp.NORM_PRE if pre else 0)
    kind = bsp.NORM_RMS if rms else bsp.NORM_LAYER
    eps = 1e-5
    wants = {k: None if v is None else v.to(D) for k, v in c.items()}
    w = lambda k, there: wants[k] if there else None  # noqa: E731
    Z, Hn, sp, sq = bsp.bsp_block_norm(g["x"], g["f"], norms, kind=kind, eps=eps, x_scale=x_scale, gate=g["gate"], w_post=g["w_post"] if post else None,
                                       b_post=g["b_post"] if post else None, w_pre=g["w_pre"] if pre else None, b_pre=g["b_pre"] if pre else None)
    args = dict(post=post, pre=pre, rms=rms)
    z, h, rp, rq = orc.block_norm(wants["x"], wants["f"], eps=eps, x_scale=x_scale, gate=wants["gate"], w_post=w("w_post", post), b_post=w("b_post", post),
                                  w_pre=w("w_pre", pre), b_pre=w("b_pre", pre), round_z=lambda v: Z.cpu().to(D), **args)
    # fp32: a mean of H values errs by (H / lanes + log lanes) u of their mean magnitude, and by as many u the variance; 64 lanes or more add
    # H / 64 + 7 values in a row.  The difference from the mean loses (that + 1) u of the magnitude, and is divided by the deviation.
    n = H / 64 + 16
    # (the largest magnitude over the deviation is what a difference from the mean can lose)
    spread = lambda v, st: (v.abs().amax(1, keepdim=True) + 1e-6) * st[:, 1:]  # noqa: E731
    zb = 4 * U * ((x_scale * wants["x"]).abs() + 1)
    if post:
        k = n * U * (1 + spread(wants["f"], rp)) * (1 + spread(wants["f"], rp).clamp(max=1e3) * n * U)
        inside(sp[:, 1:].contiguous(), rp[:, 1:], 2 * k * rp[:, 1:])
        zb = zb + (k * (4 + ((wants["f"] - rp[:, :1]) * rp[:, 1:]).abs())) * (1.5 if wants["gate"] is None else 1.5 * orc.rows_of(wants["gate"], T).abs())
    if wants["gate"] is not None:
        zb = zb + 4 * U * (z - x_scale * wants["x"]).abs()
    inside(Z, z, half(dt) * (z.abs() + zb) + zb)
    if pre:
        v = Z.cpu().to(D)
        k = n * U * (1 + spread(v, rq))
        hb = k * (4 + ((v - rq[:, :1]) * rq[:, 1:]).abs()) * 1.5
        inside(sq[:, 1:].contiguous(), rq[:, 1:], 2 * k * rq[:, 1:])
        inside(Hn, h, half(dt) * (h.abs() + hb) + hb)
    else:
        assert Hn is None and sq is None
    if offset:
        return
    # backward, from what the forward pass kept
    out = bsp.bsp_block_norm_backward(g["dz"], g["dh"] if pre else None, Z if pre else None, g["f"], norms, kind=kind, x_scale=x_scale, gate=g["gate"],
                                      w_post=g["w_post"] if post else None, b_post=g["b_post"] if post else None, w_pre=g["w_pre"] if pre else None,
                                      b_pre=g["b_pre"] if pre else None, stats_post=sp, stats_pre=sq)
    ref = orc.block_norm_backward(wants["dz"], w("dh", pre), Z.cpu().to(D) if pre else None, wants["f"], x_scale=x_scale, gate=wants["gate"],
                                  w_post=w("w_post", post), b_post=w("b_post", post), w_pre=w("w_pre", pre),
                                  stats_post=None if sp is None else sp.cpu().to(D), stats_pre=None if sq is None else sq.cpu().to(D), **args)
    # a gradient element: some 20 roundings of terms no larger than these, and two means of H
    big = 1 + wants["dz"].abs().amax() + (wants["dh"].abs().amax() * 1.6 if pre else 0)
    dev = max(1.0, float(rq[:, 1].max()) if pre else 1.0) * (max(1.0, float(rp[:, 1].max())) if post else 1.0)
    hats = 1 + (float(((Z.cpu().to(D) - rq[:, :1]) * rq[:, 1:]).abs().max()) if pre else 0) + (float(((wants["f"] - rp[:, :1]) * rp[:, 1:]).abs().max()) if post else 0)
    gmax = 1 + (float(wants["gate"].abs().max()) if wants["gate"] is not None else 0)
    each = (n + 24) * U * float(big) * dev * hats ** 2 * gmax ** 2
    for name in ("dx", "df"):
        inside(out[name], ref[name], half(dt) * (ref[name].abs() + each) + each)
    for name in ("dw_post", "db_post", "dw_pre", "db_pre", "dgate"):
        there = {"dgate": wants["gate"] is not None, "w": weights}.get(name if name == "dgate" else "w") and name in ref
        assert (out[name] is not None) == bool(there), name
        if there:  # sums over the rows: each term's error, and the additions'
            rows = T // gate_rows if name == "dgate" else T
            inside(out[name], ref[name], rows * (each * hats + (rows / 64 + 40) * U * float(big) * dev * hats ** 2 * gmax))
    again = bsp.bsp_block_norm_backward(g["dz"], g["dh"] if pre else None, Z if pre else None, g["f"], norms, kind=kind, x_scale=x_scale, gate=g["gate"],
                                        w_post=g["w_post"] if post else None, b_post=g["b_post"] if post else None, w_pre=g["w_pre"] if pre else None,
                                        b_pre=g["b_pre"] if pre else None, stats_post=sp, stats_pre=sq)
    for name, t in out.items():
        assert t is None or torch.equal(t, again[name])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("H", WIDTHS)
def test_block_norm_widths(dtype, H):
    for T in (1, 5, 67):
        check_norm(T, H, DT[dtype], False, True, True, 1)
    check_norm(6, H, DT[dtype], True, False, True, 0, x_scale=1.0)


@pytest.mark.parametrize("H", [1, 5, 8, 79, 96, 128, 129, 200, 248, 256, 257])
def test_block_norm_narrow_rows(H):
    """Several rows in a wavefront: the last ones missing, gate rows of one token and of many, rows at any address."""
    for dt in (torch.float32, torch.bfloat16):
        check_norm(1, H, dt, False, True, True, 1)
        check_norm(15, H, dt, True, True, False, 5, aligned=False)
        check_norm(1030, H, dt, False, True, True, 515)
        check_norm(3 * 700, H, dt, False, False, True, 3)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H", [2, 10, 266, 514, 1030, 2054, 4102, 8190])
def test_block_norm_rows_of_whole_words(dtype, H):
    """Even widths that are no multiple of 8: pieces that end with the row, at addresses of words and (unaligned) of half ones."""
    for aligned in (True, False):
        check_norm(37, H, DT[dtype], False, True, True, 37, aligned=aligned)
        check_norm(300, H, DT[dtype], True, False, True, 0, aligned=aligned)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("T,gate_rows", [(120, 0), (120, 1), (120, 8), (120, 120), (1200, 3), (1200, 600), (2500, 0)])
def test_block_norm_forms(rms, post, pre, T, gate_rows):
    check_norm(T, 136, torch.bfloat16, rms, post, pre, gate_rows)
    check_norm(T, 136, torch.float32, rms, post, pre, gate_rows, weights=False)


@pytest.mark.parametrize("T,H", [(40, 2056), (4, 4104), (600, 1536)])
@pytest.mark.parametrize("gate_rows", [1, 2, 4])
def test_block_norm_gates_of_wide_rows(T, H, gate_rows):
    check_norm(T, H, torch.float16, False, True, True, gate_rows)


@pytest.mark.parametrize("H", [64, 770, 1024, 3000])
def test_block_norm_unaligned(H):
    for dtype in DT.values():
        check_norm(9, H, dtype, False, True, True, 3, aligned=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_block_norm_large_means(dtype):
    """Means far above the deviation: the difference is taken before it is squared."""
    check_norm(33, 1024, DT[dtype], False, True, True, 0, offset=1000.0)


def test_block_norm_rows_of_one_value_zeros_and_nan():
    T, H = 5, 256
    x = torch.zeros(T, H, device="cuda")
    x[1] = 3.0
    x[2, 4] = math.nan
    x[3, 5] = math.inf
    x[4] = torch.arange(H, device="cuda")
    Z, Hn, _, st = bsp.bsp_block_norm(x, eps=1e-6)
    assert torch.equal(Hn[0], torch.zeros(H, device="cuda")) and torch.equal(Hn[1], torch.zeros(H, device="cuda"))
    assert torch.isnan(Hn[2]).all() and torch.isnan(Hn[3]).any() and torch.isfinite(Hn[4]).all()
    assert float(st[0, 1]) == pytest.approx(1000.0, rel=1e-6)


def test_block_norm_in_place_and_partial_outputs():
    c, g = norm_inputs(1, 40, 200, torch.bfloat16, 1)
    kw = dict(eps=1e-5, gate=g["gate"], w_post=g["w_post"], b_post=g["b_post"], w_pre=g["w_pre"], b_pre=g["b_pre"])
    Z, Hn, sp, sq = bsp.bsp_block_norm(g["x"], g["f"], 3, **kw)
    z0, h0, a, b = bsp.bsp_block_norm(g["x"], g["f"], 3, want=(), **kw)
    assert z0 is None and a is None and b is None and torch.equal(h0, Hn)
    x, f = g["x"].clone(), g["f"].clone()
    assert bsp.bsp_block_norm(x, f, 3, Z=x, H=f, **kw)[0] is x and torch.equal(x, Z) and torch.equal(f, Hn)
    back = dict(gate=g["gate"], w_post=g["w_post"], b_post=g["b_post"], w_pre=g["w_pre"], b_pre=g["b_pre"], stats_post=sp, stats_pre=sq)
    out = bsp.bsp_block_norm_backward(g["dz"], g["dh"], Z, g["f"], 3, **back)
    dz, dh = g["dz"].clone(), g["dh"].clone()
    inplace = bsp.bsp_block_norm_backward(dz, dh, Z, g["f"], 3, dX=dz, dF=dh, **back)
    assert all(torch.equal(inplace[k], out[k]) for k in out) and inplace["dx"] is dz
    part = bsp.bsp_block_norm_backward(g["dz"], g["dh"], Z, g["f"], 3, want=("dw_pre",), **back)
    assert torch.equal(part["dw_pre"], out["dw_pre"]) and all(v is None for k, v in part.items() if k != "dw_pre")
    # without a gradient from the stream, and the norm before the first block
    zero = bsp.bsp_block_norm_backward(torch.zeros_like(g["dz"]), g["dh"], Z, g["f"], 3, **back)
    none = bsp.bsp_block_norm_backward(None, g["dh"], Z, g["f"], 3, **back)
    assert all(torch.equal(zero[k], none[k]) for k in zero)
    first = bsp.bsp_block_norm(g["x"], eps=1e-5, w_pre=g["w_pre"])
    assert torch.equal(first[0], g["x"])
    for T in (0,):
        e = torch.empty(T, 200, dtype=torch.bfloat16, device="cuda")
        st = torch.empty(T, 2, device="cuda")
        assert bsp.bsp_block_norm(e, e, 3, **kw)[1].shape == (0, 200)
        got = bsp.bsp_block_norm_backward(e, e, e, e, 3, **{**back, "stats_post": st, "stats_pre": st})
        assert not got["dw_pre"].any() and not got["dgate"].any()


# ---- AdamW --------------------------------------------------------------------------------------------------------------------
SHAPES = [(1, 1), (1, 255), (1, 256), (1, 257), (16, 130), (32, 64), (0, 5), (1, 2049), (48, 300), (64, 1000), (1, 4097), (80, 256)]
HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8)


def adamw_inputs(seed, gdt, shapes, masked):
    W = [rand(seed + i, M, N, std=0.05) for i, (M, N) in enumerate(shapes)]
    G = [rand(seed + 500 + i, M, N, std=1e-3, dt=gdt) for i, (M, N) in enumerate(shapes)]
    groups = lambda M: masked and M >= 16  # noqa: E731
    g = torch.Generator().manual_seed(seed)
    keep = [(torch.rand(M // 16, N, generator=g) < 0.4).to(torch.uint8) if groups(M) else None for M, N in shapes]
    alpha = [torch.rand(M // 16, N, generator=g) if groups(M) and i % 2 else None for i, (M, N) in enumerate(shapes)]
    return W, G, keep, alpha


def on_gpu(ts, unaligned=False):
    return [None if t is None else (off_by_one(t.cuda()) if unaligned else t.cuda()) for t in ts]


@pytest.mark.parametrize("gdtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("unaligned", [False, True])
def test_adamw_is_adam_over_many_tensors(gdtype, unaligned):
    """Without decay the weights and moments have the bits of bsp_adam_step of each tensor, over steps (with betas whose complements are numbers of
    fp32, which that call forms in fp32); 60 tensors are two launches."""
    shapes = SHAPES * 5
    hyper = dict(beta1=0.875, beta2=1 - 2.0 ** -10, eps=2.0 ** -27)
    W, G, keep, alpha = adamw_inputs(1, DT[gdtype], shapes, True)
    Wd, kd, ad = on_gpu(W, unaligned), on_gpu(keep), on_gpu(alpha)
    m, v = [torch.zeros_like(w) for w in Wd], [torch.zeros_like(w) for w in Wd]
    copies = [torch.empty_like(w, dtype=torch.bfloat16) if i % 3 else None for i, w in enumerate(Wd)]
    Wr, mr, vr = on_gpu(W), [torch.zeros_like(w) for w in Wd], [torch.zeros_like(w) for w in Wd]
    for t in (1, 2, 1000):
        Gd = on_gpu([g * (1 + t % 3) for g in G], unaligned)
        bsp.bsp_adamw_step(Wd, Gd, m, v, 3e-5, t=t, keep=kd, alpha=ad, lam=1e-3, copies=copies, **hyper)
        for i, (M, N) in enumerate(shapes):
            if M:
                grouped = keep[i] is not None
                bsp.bsp_adam_step(Wr[i], Gd[i].clone(), mr[i], vr[i], 16 if grouped else 1, 3e-5, t=t, alpha=ad[i], lam=1e-3, keep=kd[i], **hyper)
            assert torch.equal(Wd[i], Wr[i]) and torch.equal(m[i], mr[i]) and torch.equal(v[i], vr[i]), (t, i)
            assert copies[i] is None or torch.equal(copies[i], Wr[i].bfloat16())


@pytest.mark.parametrize("gdtype,cdtype", [("f32", "bf16"), ("bf16", "f16")])
def test_adamw_decay_against_64_bits(gdtype, cdtype):
    W, G, keep, alpha = adamw_inputs(7, DT[gdtype], SHAPES, True)
    decay = [0.1 if i % 2 else 0.0 for i in range(len(W))]
    Wd, Gd, kd = on_gpu(W), on_gpu(G), on_gpu(keep)
    m, v = [rand(i, *w.shape, std=1e-3).cuda() for i, w in enumerate(W)], [rand(i, *w.shape, std=1e-3).square().cuda() for i, w in enumerate(W)]
    m0, v0 = [t.cpu().to(D) for t in m], [t.cpu().to(D) for t in v]
    copies = [torch.empty_like(w, dtype=DT[cdtype]) for w in Wd]
    scale = torch.tensor([0.25], device="cuda")
    bsp.bsp_adamw_step(Wd, Gd, m, v, 1e-2, t=5, weight_decay=decay, keep=kd, R=16, copies=copies, grad_scale=scale, **HYPER)
    for i in range(len(W)):
        w1, m1, v1 = orc.adamw(W[i].to(D), G[i].to(D), m0[i], v0[i], 1e-2, 0.9, 0.999, 1e-8, decay[i], 5, None if keep[i] is None else keep[i].to(D), None, 0, 16, 0.25)
        # four roundings of m, six of v; the update has 12 more, half of v's and all of m's.  eps adds nothing.
        mb = (m0[i].abs() + G[i].to(D).abs()) * 4 * U
        vb = v1 * 6 * U
        inside(m[i], m1, mb + 1e-30)
        inside(v[i], v1, vb + 1e-30)
        den = torch.sqrt(v1 / (1 - 0.999 ** 5)) + 1e-8
        wb = 4 * U * W[i].to(D).abs() + 1e-2 / (1 - 0.9 ** 5) * (m1.abs() * 20 * U + mb) / den
        inside(Wd[i], w1, wb + 1e-30)
        assert torch.equal(copies[i], Wd[i].to(DT[cdtype]))


def test_adamw_step_size_from_the_device_and_a_skipped_step():
    W, G, keep, _ = adamw_inputs(9, torch.float32, SHAPES, True)
    for bits in (32, 8):
        a, b = on_gpu(W), on_gpu(W)
        sa, sb = bsp.bsp_adamw_state(a, bits), bsp.bsp_adamw_state(b, bits)
        Gd, kd = on_gpu(G), on_gpu(keep)
        for t in (1, 2, 7):
            bsp.bsp_adamw_step(a, Gd, sa[0], sa[1], 1e-3, t=t, scales=sa[2], keep=kd, weight_decay=0.1, seed=5, **HYPER)
            bsp.bsp_adamw_step(b, Gd, sb[0], sb[1], 0.0, t=99, scales=sb[2], keep=kd, weight_decay=0.1, seed=5,
                               lr_t=torch.tensor([1e-3, t], device="cuda"), **HYPER)
        # 1 - beta^t and lr * decay in fp32 two ways: up to 16 roundings of each update, |update| <= lr; and a step ends with two roundings of
        # numbers of w's size, w less decay and less update, each of which may then fall to the neighbour, 2 U of w: 4 U a step, three steps
        for x, y in zip(a, b):
            assert float((x - y).abs().max() if x.numel() else 0) <= 3 * 1e-3 * 16 * U + 12 * U * float(x.abs().max() if x.numel() else 0)
        before = [t.clone() for s in sb if s for t in s] + [t.clone() for t in b]
        for bad in (math.nan, math.inf, -math.inf):
            bsp.bsp_adamw_step(b, Gd, sb[0], sb[1], 1e-3, t=8, scales=sb[2], keep=kd, seed=5, grad_scale=torch.tensor([bad], device="cuda"), **HYPER)
        after = [t for s in sb if s for t in s] + b
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(before, after))


@pytest.mark.parametrize("gdtype", ["f32", "bf16"])
@pytest.mark.parametrize("unaligned", [False, True])
def test_adamw_8bit(gdtype, unaligned):
    """One step from given codes.  A code differs from the 64-bit one only where the place is within what fp32 can tell of the
    next rounding decision: a value is at most 16 steps, so 30 roundings are 30 16 2^-24 of one."""
    W, G, keep, alpha = adamw_inputs(21, DT[gdtype], SHAPES, True)
    t, seed, lr, decay = 3, 77, 1e-3, 0.02
    Wd, Gd, kd, ad = on_gpu(W, unaligned), on_gpu(G, unaligned), on_gpu(keep), on_gpu(alpha)
    codes = lambda s, w, pos: orc.to_codes((rand(s, *w.shape, std=100.0).clamp(-448, 448).abs() if pos else rand(s, *w.shape, std=100.0).clamp(-448, 448)).to(D))  # noqa: E731
    mc, vc = [codes(i, w, False) for i, w in enumerate(W)], [codes(i + 90, w, True) for i, w in enumerate(W)]
    sc = [(rand(i + 40, 2, -(-w.numel() // 256)).abs() + 0.5) * 1e-6 for i, w in enumerate(W)]
    m = [x.cuda().view(torch.float8_e4m3fn) for x in mc]
    v = [x.cuda().view(torch.float8_e4m3fn) for x in vc]
    if unaligned:
        m, v = ([off_by_one(x.view(torch.uint8)).view(torch.float8_e4m3fn) for x in s] for s in (m, v))
    scales, copies = on_gpu(sc), [torch.empty_like(w, dtype=torch.float16) for w in Wd]
    bsp.bsp_adamw_step(Wd, Gd, m, v, lr, t=t, weight_decay=decay, scales=scales, keep=kd, alpha=ad, lam=1e-3, R=16, copies=copies, seed=seed, **HYPER)
    for i, w in enumerate(W):
        n = w.numel()
        if not n:
            continue
        each = sc[i].to(D).repeat_interleave(256, 1)[:, :n].view(2, *w.shape)
        w1, m1, v1 = orc.adamw(w.to(D), G[i].to(D), orc.from_codes(mc[i]) * each[0], (orc.from_codes(vc[i]) * each[1]) ** 2, lr, 0.9, 0.999, 1e-8, decay, t,
                               None if keep[i] is None else keep[i].to(D), None if alpha[i] is None else alpha[i].to(D), 1e-3, 16)
        # about 20 roundings of the update's terms, m's two largest among them (which may cancel)
        big = (orc.from_codes(mc[i]) * each[0]).abs() + G[i].to(D).abs() + (1e-3 * alpha[i].to(D).repeat_interleave(16, 0) * w.to(D) if alpha[i] is not None else 0)
        inside(Wd[i], w1, 4 * U * w.to(D).abs() + 24 * U * lr / (1 - 0.9 ** t) * (m1.abs() + big) / (torch.sqrt(v1 / (1 - 0.999 ** t)) + 1e-8))
        bits_m, bits_r = orc.random_bits(n, t, seed)
        for got, x, bits, row, up in ((m[i], m1, bits_m, 0, False), (v[i], torch.sqrt(v1), bits_r, 1, True)):
            q, s, near = orc.stored(x.reshape(-1), bits, up)
            gs = scales[i][row].cpu().to(D)
            assert ((gs - s).abs() <= 12 * U * s + 4 * U * (big.max() if row == 0 else 0) / 448).all()
            gq = orc.from_codes(got.view(torch.uint8).cpu().reshape(-1))
            differ = gq != q
            assert not (differ & (near > 1e-4)).any()
            if up:
                assert (gq[x.reshape(-1) > 0] > 0).all()
        assert torch.equal(copies[i], Wd[i].half())


@pytest.mark.parametrize("N", [1, 2, 3, 5, 142, 147, 766])
def test_adamw_8bit_masks_of_any_width(N):
    """The mask zeroes weights and leaves moments alone, the factors are an addition to the gradient (one rounding): bit for bit what the step without
    them gives on that gradient, where rows end anywhere among four elements."""
    M, R, lam = 48, 16, 1e-3
    w, g = rand(N, M, N, std=0.05), rand(N + 1, M, N, std=1e-3)
    gen = torch.Generator().manual_seed(N)
    keep, alpha = (torch.rand(M // R, N, generator=gen) < 0.5).to(torch.uint8), torch.rand(M // R, N, generator=gen)
    factor = (torch.tensor(lam) * alpha).repeat_interleave(R, 0)
    added = (factor.to(D) * w.to(D) + g.to(D)).float()
    runs = []
    for grad, more in ((g, dict(keep=[keep.cuda()], alpha=[alpha.cuda()], lam=lam, R=R)), (added, {})):
        W, copies = [w.cuda()], [torch.empty(M, N, dtype=torch.bfloat16, device="cuda")]
        m, v, s = bsp.bsp_adamw_state(W, 8)
        bsp.bsp_adamw_step(W, [grad.cuda()], m, v, 1e-3, t=1, scales=s, weight_decay=0.01, seed=3, copies=copies, **more, **HYPER)
        runs.append((W[0].cpu(), m[0].view(torch.uint8).cpu(), v[0].view(torch.uint8).cpu(), s[0].cpu(), copies[0].cpu()))
    kept = keep.repeat_interleave(R, 0).bool()
    assert torch.equal(runs[0][0], torch.where(kept, runs[1][0], torch.zeros(()))) and torch.equal(runs[0][4], runs[0][0].bfloat16())
    assert all(torch.equal(a, b) for a, b in zip(runs[0][1:4], runs[1][1:4]))


def test_adamw_8bit_moments_follow_over_steps():
    """200 steps of gradients of one size and then a tenth of it: the 8-bit moments stay unbiased, so the mean of sqrt(v) and of m over many
    elements follows the exact recursion.  A code is off by at most 2^-3 of its value at random, 2^-3 / sqrt(3) / sqrt(steps it lives)
    each; over 65536 elements the mean by 1e-3."""
    n = 65536
    w = [torch.zeros(n, device="cuda")]
    m, v, s = bsp.bsp_adamw_state(w, 8)
    em = ev = 0.0
    for t in range(1, 401):
        size = 1e-3 if t <= 200 else 1e-4
        bsp.bsp_adamw_step(w, [torch.full((n,), size, device="cuda") * torch.where(torch.arange(n, device="cuda") % 256 == 0, 4.0, 1.0)], m, v, 1e-4, t=t,
                           scales=s, seed=1, beta1=0.9, beta2=0.99, eps=1e-8)
        em, ev = 0.9 * em + 0.1 * size, 0.99 * ev + 0.01 * size * size
    small = torch.arange(n, device="cuda") % 256 != 0
    mean = lambda c, row: float((c[0].float() * s[0][row].repeat_interleave(256))[small].double().mean())  # noqa: E731
    assert mean(m, 0) == pytest.approx(em, rel=0.01)
    # (r = sqrt(v) is what keeps its mean; v = r^2 gains its variance, at most (step / 2)^2 of r in a step, decayed by 1 - beta2: 2^-8 / 4 / 0.02 of v)
    assert math.sqrt(ev) * 0.97 <= mean(v, 1) <= math.sqrt(ev) * 1.06


def test_adamw_flushes_what_has_no_scale_and_starts_fresh():
    w = [torch.ones(300, device="cuda")]
    m, v, s = bsp.bsp_adamw_state(w, 8)
    g = torch.zeros(300, device="cuda")
    g[256:] = 1e-3
    bsp.bsp_adamw_step(w, [g], m, v, 1e-2, t=1, scales=s, **HYPER)
    assert (w[0][:256] == 1).all() and torch.allclose(w[0][256:], torch.tensor(0.99, device="cuda"), rtol=1e-5)
    assert not s[0][:, 0].any() and (s[0][:, 1] > 0).all() and not m[0].view(torch.uint8)[:256].any()


def test_adamw_8bit_block_with_a_moment_that_is_not_finite_starts_afresh():
    """One gradient of infinity, NaN or more than the root of fp32's range leaves the other weights of its block finite, then and later; a
    step from fresh moments at t = 3 is lr (0.1 / 0.271) / sqrt(0.001 / 0.002997) = 0.639 lr."""
    n, lr = 1024, 1e-2
    w = [torch.ones(n, device="cuda")]
    m, v, s = bsp.bsp_adamw_state(w, 8)
    g = torch.linspace(0.5, 1.5, n, device="cuda")
    bsp.bsp_adamw_step(w, [g], m, v, lr, t=1, scales=s, **HYPER)
    bad = g.clone()
    bad[10], bad[300], bad[700] = 1e30, float("inf"), float("nan")
    bsp.bsp_adamw_step(w, [bad], m, v, lr, t=2, scales=s, **HYPER)
    lost = torch.zeros(n, dtype=torch.bool, device="cuda")
    lost[300] = lost[700] = True
    assert torch.equal(w[0].isnan(), lost) and w[0].isfinite().sum() == n - 2
    assert (s[0][:, :3] == 0).all() and (s[0][:, 3] > 0).all()
    before = w[0].clone()
    bsp.bsp_adamw_step(w, [g], m, v, lr, t=3, scales=s, **HYPER)
    moved = (w[0] - before)[~lost].abs()
    assert torch.equal(w[0].isnan(), lost) and float((moved[:766] / (0.639 * lr) - 1).abs().max()) < 1e-2 and (s[0] > 0).all()


def test_adamw_refuses_what_does_not_fit():
    w = torch.zeros(32, 16, device="cuda")
    ok = lambda **k: bsp.bsp_adamw_step(**{**dict(W=[w], G=[w.clone()], m=[w.clone()], v=[w.clone()], lr=1e-3), **k})  # noqa: E731
    e4 = torch.zeros(32, 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    for bad in (dict(W=[w.half()]), dict(G=[w[:16]]), dict(G=[w.double()]), dict(m=[w.half()]), dict(v=[w[:, :8]]), dict(W=[w.t()]),
                dict(scales=[torch.zeros(2, 2, device="cuda")]), dict(m=[e4], v=[e4]), dict(m=[e4], v=[e4], scales=[torch.zeros(2, 3, device="cuda")]),
                dict(keep=[torch.zeros(2, 15, dtype=torch.uint8, device="cuda")]), dict(keep=[torch.zeros(2, 16, device="cuda")]),
                dict(keep=[torch.zeros(2, 16, dtype=torch.uint8, device="cuda")], R=5), dict(alpha=[torch.zeros(2, 16, device="cuda")], R=0),
                dict(copies=[w.clone()]), dict(copies=[w.bfloat16()[:1]]), dict(weight_decay=[0.1, 0.2]), dict(lr_t=torch.zeros(1, device="cuda")),
                dict(grad_scale=torch.zeros(0, device="cuda")), dict(W=[w, w], G=[w, w], m=[w, w], v=[w])):
        with pytest.raises(ValueError):
            ok(**bad)
    with pytest.raises(bsp.BspError):
        ok(t=0)
    with pytest.raises(bsp.BspError):
        bsp.bsp_adamw_step([w, w], [w.clone()] * 2, [w.clone(), w.clone()], [w.clone(), w.clone()], 1e-3)   # a tied tensor twice
    assert not w.any()


def test_products_and_norms_refuse_what_does_not_fit():
    x = torch.zeros(40, 128, dtype=torch.bfloat16, device="cuda")
    W = bsp.bsp_fp8_quant(torch.zeros(64, 128, device="cuda"), bsp.FP8_BLOCK)[0]
    A = bsp.bsp_fp8_quant(x)[0]
    row = lambda **k: bsp.Fp8(**{**dict(codes=W.codes, scales=W.scales, rows=64, cols=128, layout=bsp.FP8_BLOCK), **k})  # noqa: E731
    half, one = torch.zeros(64, dtype=torch.float16, device="cuda"), torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: bsp.bsp_linear_fp8(x[:, :64].contiguous(), W), lambda: bsp.bsp_linear_fp8(x.cpu(), W), lambda: bsp.bsp_linear_fp8(x.t(), W),
                 lambda: bsp.bsp_linear_fp8(x.double(), W), lambda: bsp.bsp_linear_fp8(x, row(rows=65)), lambda: bsp.bsp_linear_fp8(x, row(layout=bsp.FP8_ROW)),
                 lambda: bsp.bsp_linear_fp8(x, row(codes=W.codes.view(torch.uint8))), lambda: bsp.bsp_linear_fp8(x, row(scales=W.scales.float())),
                 lambda: bsp.bsp_linear_fp8(x, W, half), lambda: bsp.bsp_linear_fp8(x, W, one[:63]), lambda: bsp.bsp_linear_fp8(x, W, residual=x),
                 lambda: bsp.bsp_linear_fp8(x, W, Y=x), lambda: bsp.bsp_matmul_fp8(row(), row()), lambda: bsp.bsp_matmul_fp8(A, row(cols=256)),
                 lambda: bsp.bsp_matmul_fp8(A, W, half), lambda: bsp.bsp_matmul_fp8(A, W, residual=x), lambda: bsp.bsp_matmul_fp8(A, W, Y=x),
                 lambda: bsp.bsp_fp8_quant(x.t()), lambda: bsp.bsp_fp8_quant(x.cpu()),
                 lambda: bsp.bsp_block_norm(x, x[:20]), lambda: bsp.bsp_block_norm(x, x.float()), lambda: bsp.bsp_block_norm(x, w_pre=one),
                 lambda: bsp.bsp_block_norm(x, x, gate=half.view(1, 64)), lambda: bsp.bsp_block_norm(x.cpu()), lambda: bsp.bsp_block_norm(x.double()),
                 lambda: bsp.bsp_block_norm(x[0]), lambda: bsp.bsp_block_norm_backward(None, None, x), lambda: bsp.bsp_block_norm_backward(x, x[:20], x),
                 lambda: bsp.bsp_block_norm_backward(x, x, x, stats_pre=torch.zeros(40, device="cuda")), lambda: bsp.bsp_block_norm(x, x, dX=x)):
        with pytest.raises((ValueError, TypeError)):
            call()
    for call in (lambda: bsp.bsp_block_norm(x, x, norms=0), lambda: bsp.bsp_block_norm(x, norms=bsp.NORM_POST), lambda: bsp.bsp_block_norm(x, kind=3),
                 lambda: bsp.bsp_block_norm(x, x, gate=torch.zeros(3, 128, dtype=x.dtype, device="cuda")), lambda: bsp.bsp_block_norm_backward(x, x, x),
                 lambda: bsp.bsp_linear_fp8(x, W, act=5), lambda: bsp.bsp_block_norm(torch.zeros(2, 8200, device="cuda")),
                 lambda: bsp.bsp_linear_fp8(x, W, ws=torch.zeros(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(bsp.BspError):
            call()


# ---- sizes past 32 bits -------------------------------------------------------------------------------------------------------
def test_products_past_32_bits():
    """More than 2^31 elements of X: the last rows are those of a call of their own."""
    T, M, N = (1 << 21) + 37, 80, 1100
    x = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
    x[-300:] = rand(1, 300, N, dt=torch.bfloat16).cuda()
    W = bsp.bsp_fp8_quant(rand(2, M, N).cuda(), bsp.FP8_BLOCK)[0]
    y = bsp.bsp_linear_fp8(x, W)
    assert not y[:-300].any()
    tail = bsp.bsp_matmul_fp8(bsp.bsp_fp8_quant(x[-300:].clone())[0], W, out_dtype=torch.float32)
    assert float((y[-300:].float() - tail).norm() / tail.norm()) <= 2.0 ** -8 + 2.0 ** -13


def test_norms_past_32_bits_and_past_one_row_of_workgroups():
    T, H = (1 << 18) + 5, 8192
    x = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    x[-9:] = rand(1, 9, H, dt=torch.bfloat16).cuda()
    h = bsp.bsp_block_norm(x, want=())[1]
    assert torch.equal(h[-9:], bsp.bsp_block_norm(x[-9:].clone(), want=())[1]) and not h[:-9].any()
    del h
    st = bsp.bsp_block_norm(x, want=("stats_pre",))[3]
    out = bsp.bsp_block_norm_backward(None, x, x, stats_pre=st, want=("dx",))
    small = bsp.bsp_block_norm_backward(None, x[-9:].clone(), x[-9:].clone(), stats_pre=st[-9:].clone(), want=("dx",))
    assert torch.equal(out["dx"][-9:], small["dx"])
    del x, out
    T = (1 << 22) + 4099                                # more than 2^20 workgroups
    x = rand(2, T, 8).cuda()
    h = bsp.bsp_block_norm(x, eps=1e-5)[1]
    for part in (slice(0, 5000), slice(T - 5000, T)):
        assert torch.equal(h[part], bsp.bsp_block_norm(x[part].clone(), eps=1e-5)[1])


def test_adamw_past_32_bits():
    M, N = (1 << 21) + 32, 1024
    w = torch.zeros(M, N, device="cuda")
    g = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    keep = torch.ones(M // 16, N, dtype=torch.uint8, device="cuda")
    w[-48:], g[-48:] = rand(1, 48, N).cuda(), rand(2, 48, N, dt=torch.bfloat16).cuda()
    keep[-3:] = (rand(3, 3, N) > 0).to(torch.uint8).cuda()
    tail = [t[-48:].clone() for t in (w, g)]
    m, v, _ = bsp.bsp_adamw_state([w])
    bsp.bsp_adamw_step([w], [g], m, v, 1e-2, keep=[keep], **HYPER)
    m1, v1, _ = bsp.bsp_adamw_state([tail[0]])
    bsp.bsp_adamw_step([tail[0]], [tail[1]], m1, v1, 1e-2, keep=[keep[-3:].clone()], **HYPER)
    assert torch.equal(w[-48:], tail[0]) and torch.equal(m[0][-48:], m1[0]) and torch.equal(v[0][-48:], v1[0])
    del m, v
    w[-48:] = rand(1, 48, N).cuda()
    m, v, s = bsp.bsp_adamw_state([w], 8)
    bsp.bsp_adamw_step([w], [g], m, v, 1e-2, keep=[keep], scales=s, seed=4, **HYPER)
    assert float((w[-48:] - tail[0]).abs().max()) <= 1e-2 * 24 * U + 4 * U * 5   # as above, |update| <= lr, |w| < 5
    x = 0.1 * g[-1].cpu().to(D)                          # m of the last row, whose places are past 2^31
    place = (M - 1) * N
    bits = orc.random_bits(N, 1, 4, first=place)[0]
    q, scale, near = orc.stored(x, bits, False)
    got = orc.from_codes(m[0][-1].view(torch.uint8).cpu())
    assert not ((got != q) & (near > 1e-4)).any() and float((s[0][0, -4:].cpu().to(D) / scale - 1).abs().max()) <= 12 * U


# ---- together -----------------------------------------------------------------------------------------------------------------
def encoder_block(x, w, b, gate, w_pre, b_pre, w_post, dz, state=None):
    """Norm, 8-bit layer, norm, gate and addition; gradients; an AdamW step of all its parameters (fp32 masters with 16-bit copies)."""
    W, Wt = bsp.bsp_fp8_quant(w[1], bsp.FP8_BLOCK, want=("plain", "transposed"))
    _, h, _, s0 = bsp.bsp_block_norm(x, w_pre=w_pre[1], b_pre=b_pre[1], eps=1e-5)
    h8, h8t = bsp.bsp_fp8_quant(h, want=("plain", "transposed"))
    f = bsp.bsp_matmul_fp8(h8, W, b[1], out_dtype=x.dtype)
    z, _, sp, _ = bsp.bsp_block_norm(x, f, bsp.NORM_POST, kind=bsp.NORM_RMS, eps=1e-5, gate=gate[1], w_post=w_post[1])
    g = bsp.bsp_block_norm_backward(dz, None, None, f, bsp.NORM_POST, kind=bsp.NORM_RMS, gate=gate[1], w_post=w_post[1], stats_post=sp)
    d8, d8t = bsp.bsp_fp8_quant(g["df"], want=("plain", "transposed"))
    dh = bsp.bsp_matmul_fp8(d8, Wt, out_dtype=x.dtype)
    dw = bsp.bsp_matmul_fp8(d8t, h8t, out_dtype=torch.float32)
    db = g["df"].float().sum(0)
    k = bsp.bsp_block_norm_backward(g["dx"], dh, x, norms=bsp.NORM_PRE, w_pre=w_pre[1], b_pre=b_pre[1], stats_pre=s0, want=("dx", "dw_pre", "db_pre"))
    grads = [dw, db, g["dgate"], k["dw_pre"], k["db_pre"], g["dw_post"]]
    if state:
        masters, copies, m, v, s, lr_t = state
        bsp.bsp_adamw_step(masters, grads, m, v, 0.0, scales=s, copies=copies, weight_decay=[0.1, 0, 0, 0, 0, 0], lr_t=lr_t, seed=3, **HYPER)
    return z, k["dx"], grads


def block_state(seed, T, N, dt):
    p = [rand(seed, N, N, std=0.05), rand(seed + 1, N, std=0.1), rand(seed + 2, 1, N), 1 + rand(seed + 3, N, std=0.1), rand(seed + 4, N, std=0.1), 1 + rand(seed + 5, N, std=0.1)]
    masters = [t.cuda() for t in p]
    copies = [t.to(dt) for t in masters]
    pairs = list(zip(masters, copies))
    return rand(seed + 6, T, N, dt=dt).cuda(), rand(seed + 7, T, N, dt=dt).cuda(), masters, copies, pairs


def test_a_training_step_of_a_block():
    """The operators as they are used together, against automatic differentiation in 64 bits through the same quantised operands.
    Every 16-bit tensor on the way is rounded (2^-8 of it in bf16, 2^-11 in fp16); the comparison is in the 2-norm, where these
    roundings add up: eight of them at most on any path, and e4m3's of a rounded operand may fall the other way: 2^-4 of an element where
    2^-7 or more of them flip, 2^-4 sqrt(2^-6)."""
    dt = torch.float16
    x, dz, masters, copies, (w, b, gate, w_pre, b_pre, w_post) = block_state(50, 300, 256, dt)
    z, dx, grads = encoder_block(x, w, b, gate, w_pre, b_pre, w_post, dz)
    leaf = lambda t: t.detach().cpu().to(D).requires_grad_()  # noqa: E731
    X, Wl, Bl, Gl, A, Bp, P = (leaf(t) for t in (x, *copies))
    quant = lambda t, block: orc.value(*orc.quant(t.detach(), block), t.shape[1], block)  # noqa: E731
    through = lambda t, block=False: t + (quant(t, block) - t).detach()  # noqa: E731
    h = torch.nn.functional.layer_norm(X, (256,), A, Bp, 1e-5)
    h = h + (h.detach().half().to(D) - h.detach())
    f = through(h) @ through(Wl, True).t() + Bl
    n = f / torch.sqrt((f * f).mean(1, keepdim=True) + 1e-5) * P
    Z = X + Gl * n
    (Z * dz.cpu().to(D)).sum().backward()
    allowed = 8 * 2.0 ** -11 + 2.0 ** -4 * 2.0 ** -3
    close = lambda got, want: float((got.cpu().to(D) - want).norm() / want.norm())  # noqa: E731
    assert close(z, Z.detach()) <= 8 * 2.0 ** -11 + 2.0 ** -7
    # gradients: dY is quantised as well, 2^-4 of an element at most, 2^-4 / sqrt(3) in the 2-norm, and so are h and W's other operand
    for got, want in zip([dx] + grads, [X.grad, Wl.grad, Bl.grad, Gl.grad, A.grad, Bp.grad, P.grad]):
        assert close(got.view(want.shape), want) <= allowed + 2 * 2.0 ** -4 / math.sqrt(3)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_training_step(bits):
    """The whole step in a graph, replayed with other inputs and step sizes and eager work in between, gives the bits of eager steps."""
    dt = torch.bfloat16

    def fresh():
        x, dz, masters, copies, pairs = block_state(80, 200, 384, dt)
        m, v, s = bsp.bsp_adamw_state(masters, bits)
        return x, dz, masters, copies, pairs, [masters, copies, m, v, s, torch.tensor([1e-3, 1.0], device="cuda")]
    x, dz, masters, copies, pairs, state = fresh()
    inputs = [(rand(200 + i, 200, 384, dt=dt).cuda(), rand(300 + i, 200, 384, dt=dt).cuda()) for i in range(4)]
    want = []
    for i, (a, d) in enumerate(inputs):
        state[5].copy_(torch.tensor([1e-3 / (i + 1), i + 1.0]))
        z, dx, grads = encoder_block(a, *pairs, d, state)
        want.append([t.clone() for t in (z, dx, *grads, *masters, *copies, *(u.view(torch.uint8) for u in state[2] + state[3]))])
    x, dz, masters, copies, pairs, state = fresh()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):                     # another stream than the tensors' own
        encoder_block(x, *pairs, dz)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z, dx, grads = encoder_block(x, *pairs, dz, state)
    for i, (a, d) in enumerate(inputs):
        x.copy_(a)
        dz.copy_(d)
        state[5].copy_(torch.tensor([1e-3 / (i + 1), i + 1.0]))
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip((z, dx, *grads, *masters, *copies, *(u.view(torch.uint8) for u in state[2] + state[3])), want[i]):
            assert torch.equal(got, ref), i
        encoder_block(x, *pairs, dz)                    # eager work between the replays
        torch.cuda.synchronize()


def test_the_layer_captured_with_its_workspace():
    """A server's layer in a graph with a workspace of its own, replayed."""
    for T in (1, 40, 700):
        x, w = rand(1, T, 640, dt=torch.bfloat16).cuda(), rand(2, 512, 640, std=0.05, dt=torch.bfloat16).cuda()
        W = bsp.bsp_fp8_quant(w, bsp.FP8_BLOCK)[0]
        ws = torch.empty(max(256, bsp.lib().bsp_linear_fp8_workspace_bytes(T, 512, 640)), dtype=torch.uint8, device="cuda")
        y = torch.empty(T, 512, dtype=torch.bfloat16, device="cuda")
        bsp.bsp_linear_fp8(x, W, Y=y, ws=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            bsp.bsp_linear_fp8(x, W, Y=y, ws=ws)
        for i in range(3):
            x.copy_(rand(10 + i, T, 640, dt=torch.bfloat16))
            ws.random_(0, 256)
            y.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, bsp.bsp_linear_fp8(x, W))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_results_side_by_side_in_one_buffer(bits):
    """Neighbours that touch are not taken for an overlap, in any order; a copy, a moment or scales listed twice are refused and nothing is written."""
    shapes = [(16, 16), (1, 300), (3, 171), (48, 16)]
    W, G, _, _ = adamw_inputs(31, torch.float32, shapes, False)
    G = on_gpu(G)
    runs = []
    for order in (1, -1, 0):                            # one buffer, ascending and descending; tensors of their own
        w, c, (m, v, s) = on_gpu(W), [torch.zeros_like(x, dtype=torch.bfloat16, device="cuda") for x in W], bsp.bsp_adamw_state(on_gpu(W), bits)
        if order:
            lists = [w, m, v, c] + ([s] if s else [])
            flat = [t for of in zip(*lists) for t in of][::order]
            buf = torch.empty(sum(-(-t.nbytes // 4) * 4 for t in flat), dtype=torch.uint8, device="cuda")
            at, new = 0, {}
            for t in flat:
                new[id(t)] = buf[at:at + t.nbytes].view(t.dtype).view(t.shape)
                new[id(t)].copy_(t)
                at += -(-t.nbytes // 4) * 4
            w, m, v, c = ([new[id(t)] for t in of] for of in (w, m, v, c))
            s = [new[id(t)] for t in s] if s else None
        for t in (1, 2):
            bsp.bsp_adamw_step(w, G, m, v, 1e-3, t=t, scales=s, copies=c, weight_decay=0.1, seed=2, **HYPER)
        runs.append([t.view(torch.uint8).cpu() for of in (w, m, v, c, s or []) for t in of])
        before = [t.clone() for t in runs[-1]]
        for k in range(5 if s else 4):
            two = [[of[0], of[0].clone()] for of in (w, m, v, c, s or [torch.zeros(1)])]
            two[k][1] = two[k][0]
            with pytest.raises(bsp.BspError):
                bsp.bsp_adamw_step(two[0], [G[0], G[0]], two[1], two[2], 1e-3, scales=two[4] if s else None, copies=two[3], **HYPER)
        with pytest.raises(bsp.BspError):
            bsp.bsp_adamw_step([w[0]], [G[0]], [m[0]], [m[0]], 1e-3, scales=[s[0]] if s else None, **HYPER)   # both moments one tensor
        assert all(torch.equal(a, t.view(torch.uint8).cpu()) for a, t in zip(before, [t for of in (w, m, v, c, s or []) for t in of]))
    assert all(torch.equal(a, b) for a, b in zip(runs[0], runs[1])) and all(torch.equal(a, b) for a, b in zip(runs[0], runs[2]))


def test_adamw_8bit_update_from_equal_moments():
    """The 8-bit form groups the update in its own way and divides with the hardware's reciprocal.  Its moments have the bits of the 32-bit step from the same
    ones; then, in roundings of the update: 32 bits m / c1, the product with lr, half of v / c2, the root, the addition and the division, 5.5; 8 bits lr / c1,
    r, 1 / sqrt(c2) (two), the fma, the reciprocal (1 ulp: two) and two products, 9: 15 together.  A step ends with one rounding of the weight's size in either."""
    n = 4096
    mc, vc = (orc.to_codes(rand(i, n, std=100.0).clamp(-448, 448).to(D)) for i in (1, 2))
    vc = vc & 127
    sc = (rand(3, 2, n // 256).abs() + 0.5) * 1e-6
    each = sc.repeat_interleave(256, 1)
    m32 = orc.from_codes(mc).float() * each[0]
    r32 = orc.from_codes(vc).float() * each[1]
    for t, lr, eps, decay in ((1, 1e-3, 1e-8, 0.0), (7, 2e-2, 1e-6, 0.01), (20000, 0.3, 1e-12, 0.0)):
        hyper = dict(beta1=0.9, beta2=0.999, eps=eps, t=t, weight_decay=decay)
        w0, g = rand(4, n, std=0.02), rand(5, n, std=1e-4)
        a, b, none = w0.cuda(), w0.cuda(), torch.zeros(n, device="cuda")
        bsp.bsp_adamw_step([a], [g.cuda()], [m32.cuda()], [(r32 * r32).cuda()], lr, **hyper)
        bsp.bsp_adamw_step([none], [g.cuda()], [m32.cuda()], [(r32 * r32).cuda()], lr, **{**hyper, "weight_decay": 0.0})   # the update alone
        bsp.bsp_adamw_step([b], [g.cuda()], [mc.cuda().view(torch.float8_e4m3fn)], [vc.cuda().view(torch.float8_e4m3fn)], lr, scales=[sc.cuda()], **hyper)
        inside(b, a.cpu().to(D), 15 * U * none.cpu().to(D).abs() + 2 * U * a.cpu().to(D).abs() + 1e-38)
