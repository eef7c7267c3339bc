"""The operators round the layer without a GPU: their refusals (made on the host, before anything is launched), and the plain
implementations that the GPU tests compare with, held against closed forms and differences."""
import ctypes as C
import math

import pytest
import torch

import operators_oracle as orc
import paper_2009_08065_amd as bsp

OK, NULL, SHAPE, DTYPE, CAP = 0, 1, 2, 3, 4
P = C.c_void_p(4096)    # never dereferenced
ODD = C.c_void_p(4097)


# ---- refusals -----------------------------------------------------------------------------------------------------------------
def test_fp8_refusals():
    L = bsp.lib()
    q = L.bsp_fp8_quant
    assert q(None, 1, 4, 8, 0, P, P, None, None, None) == NULL
    assert q(P, 1, 4, 8, 0, P, None, None, None, None) == NULL
    assert q(P, 1, 4, 8, 0, None, None, P, None, None) == NULL
    assert q(P, 5, 4, 8, 0, P, P, None, None, None) == DTYPE
    assert q(P, 1, 4, 8, 2, P, P, None, None, None) == DTYPE
    assert q(P, 1, -1, 8, 0, P, P, None, None, None) == SHAPE and q(P, 1, 4, 0, 0, P, P, None, None, None) == SHAPE
    assert q(ODD, 1, 4, 8, 0, P, P, None, None, None) == SHAPE and q(P, 1, 4, 8, 0, C.c_void_p(4104), P, None, None, None) == SHAPE
    assert q(P, 1, 1 << 31, 8, 0, P, P, None, None, None) == SHAPE
    assert q(P, 1, 0, 8, 0, P, P, P, P, None) == OK and q(P, 1, 4, 8, 0, None, None, None, None, None) == OK   # nothing to do

    def mm(A=P, SA=P, B=P, SB=P, lay=1, T=4, M=8, K=128, bias=None, act=0, res=None, Y=P, ydt=1, ws=None, n=0):
        return L.bsp_matmul_fp8(A, SA, B, SB, lay, T, M, K, bias, act, res, Y, ydt, ws, n, None)
    assert mm(A=None) == NULL and mm(SA=None) == NULL and mm(B=None) == NULL and mm(SB=None) == NULL and mm(Y=None) == NULL
    assert mm(lay=3) == DTYPE and mm(act=7) == DTYPE and mm(ydt=4) == DTYPE
    assert mm(T=-1) == SHAPE and mm(M=0) == SHAPE and mm(K=0) == SHAPE and mm(K=(1 << 23) + 1) == SHAPE
    assert mm(A=C.c_void_p(4104)) == SHAPE and mm(B=C.c_void_p(4104)) == SHAPE and mm(Y=ODD) == SHAPE and mm(bias=ODD) == SHAPE
    assert mm(res=ODD) == SHAPE and mm(ws=C.c_void_p(4100), n=64) == SHAPE and mm(Y=C.c_void_p(4098), ydt=0) == SHAPE
    assert mm(T=0) == OK
    need = L.bsp_matmul_fp8_workspace_bytes(100, 64, 8192)
    assert need > 0 and mm(T=100, M=64, K=8192, ws=P, n=need - 1) == CAP
    assert L.bsp_matmul_fp8_workspace_bytes(0, 64, 64) == 0 and L.bsp_matmul_fp8_workspace_bytes(4, 0, 64) == 0

    def lin(X=P, xdt=1, T=40, M=8, N=128, W=P, SW=P, lay=1, bias=None, act=0, res=None, Y=P, ws=P, n=1 << 20):
        return L.bsp_linear_fp8(X, xdt, T, M, N, W, SW, lay, bias, act, res, Y, ws, n, None)
    assert lin(X=None) == NULL and lin(W=None) == NULL and lin(SW=None) == NULL and lin(Y=None) == NULL and lin(ws=None) == NULL
    assert lin(xdt=9) == DTYPE and lin(lay=-1) == DTYPE and lin(N=0) == SHAPE and lin(X=ODD) == SHAPE and lin(ws=C.c_void_p(4100)) == SHAPE
    assert lin(n=L.bsp_linear_fp8_workspace_bytes(40, 8, 128) - 1) == CAP and lin(T=0) == OK


def test_block_norm_refusals():
    L = bsp.lib()

    def fwd(X=P, F=P, dt=1, T=4, H=64, norms=3, kind=0, gate=None, rows=0, w=None, Z=P, Hn=P, st=None):
        return L.bsp_block_norm(X, F, dt, T, H, norms, kind, 1e-6, 1.0, gate, rows, w, None, None, None, Z, Hn, st, None, None)
    assert fwd(X=None) == NULL and fwd(F=None) == NULL and fwd(Hn=None) == NULL and fwd(norms=1, Z=None) == NULL
    assert fwd(F=None, norms=2, gate=P, rows=1) == NULL
    assert fwd(dt=8) == DTYPE and fwd(norms=0) == DTYPE and fwd(norms=4) == DTYPE and fwd(kind=2) == DTYPE
    assert fwd(H=0) == SHAPE and fwd(H=8193) == SHAPE and fwd(T=-1) == SHAPE and fwd(T=1 << 31) == SHAPE
    assert fwd(gate=P, rows=0) == SHAPE and fwd(gate=P, rows=3) == SHAPE and fwd(gate=P, rows=8) == SHAPE
    assert fwd(X=ODD) == SHAPE and fwd(w=ODD) == SHAPE and fwd(st=C.c_void_p(4100)) == SHAPE
    assert fwd(T=0) == OK

    def bwd(dZ=P, dH=P, Z=P, F=P, dt=1, T=4, H=64, norms=3, kind=0, gate=None, rows=0, sp=P, sq=P, dX=P, dF=P, dwp=None, dbq=None, dg=None,
            ws=None, n=0):
        return L.bsp_block_norm_backward(dZ, dH, Z, F, dt, T, H, norms, kind, 1.0, gate, rows, None, None, None, sp, sq, dX, dF, dwp, None,
                                         None, dbq, dg, ws, n, None)
    assert bwd(dH=None) == NULL and bwd(Z=None) == NULL and bwd(F=None) == NULL and bwd(sp=None) == NULL and bwd(sq=None) == NULL
    assert bwd(norms=1, dZ=None) == NULL and bwd(norms=2, F=None, gate=P, rows=1, dg=P, ws=P, n=1 << 20) == NULL
    assert bwd(dwp=P) == NULL and bwd(dwp=P, ws=P, n=16) == CAP and bwd(dwp=P, ws=C.c_void_p(4100), n=1 << 20) == SHAPE
    assert bwd(norms=2, dwp=P, ws=P, n=1 << 20) == SHAPE and bwd(norms=1, dbq=P, ws=P, n=1 << 20) == SHAPE and bwd(dg=P, ws=P, n=1 << 20) == SHAPE
    assert bwd(dt=3) == DTYPE and bwd(norms=0) == DTYPE and bwd(H=9000) == SHAPE and bwd(gate=P, rows=3) == SHAPE and bwd(sq=C.c_void_p(4100)) == SHAPE
    assert bwd(T=0) == OK
    q = L.bsp_block_norm_backward_workspace_bytes
    assert q(0, 64, 0) == 0 and q(4, 9000, 0) == 0 and q(4, 64, 3) == 0 and q(4, 64, 4) > 0 and q(100000, 1024, 0) > q(10, 1024, 0)


def test_what_no_launch_can_hold_is_refused():
    """2^32 threads or more, or more lines of workgroups than a grid has."""
    L = bsp.lib()
    assert L.bsp_fp8_quant(P, 1, 1 << 30, 1, 0, P, P, None, None, None) == SHAPE
    assert L.bsp_fp8_quant(P, 1, (1 << 31) - 1, 4096, 0, P, P, None, None, None) == SHAPE
    mm = lambda T, M, K: L.bsp_matmul_fp8(P, P, P, P, 0, T, M, K, None, 0, None, P, 1, None, 0, None)  # noqa: E731
    assert mm((1 << 31) - 1, 1, 128) == SHAPE and mm(1, 1 << 28, 1024) == SHAPE
    assert L.bsp_linear_fp8(P, 1, 1, 1 << 28, 1024, P, P, 0, None, 0, None, P, P, 0, None) == SHAPE
    assert L.bsp_block_norm_backward(P, P, P, P, 1, 0, 64, 3, 0, 1.0, P, 1 << 16, None, None, None, P, P, P, P, None, None, None, None, P, P, 1 << 20,
                                     None) == SHAPE


class _Tensor(C.Structure):
    _fields_ = [("w", C.c_void_p), ("g", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p), ("scales", C.c_void_p), ("copy", C.c_void_p),
                ("keep", C.c_void_p), ("alpha", C.c_void_p), ("M", C.c_int64), ("N", C.c_int64), ("R", C.c_int32), ("weight_decay", C.c_float)]


def test_adamw_refusals():
    L = bsp.lib()

    def step(*changes, count=None, gdt=0, cdt=1, bits=32, t=1, lr_t=None):
        each = [_Tensor(**dict(dict(w=4096 * (2 + i), g=4096, m=4096, v=4096, M=4, N=8, R=2), **c)) for i, c in enumerate(changes or ({},))]
        return L.bsp_adamw_step((_Tensor * len(each))(*each), len(each) if count is None else count, gdt, cdt, bits, 0.0, 1e-3, 0.9, 0.999,
                                1e-8, t, 0, lr_t, None, None)
    assert step(dict(w=None)) == NULL and step(dict(g=None)) == NULL and step(dict(m=None)) == NULL and step(dict(v=None)) == NULL
    assert step(bits=8) == NULL and step(bits=16) == SHAPE and step(count=-1) == SHAPE
    assert step(gdt=3) == DTYPE and step(cdt=0) == DTYPE
    assert step(t=0) == SHAPE and step(dict(M=-1)) == SHAPE and step(dict(N=1 << 31)) == SHAPE and step(dict(M=1 << 40, N=1 << 30)) == SHAPE
    assert step(dict(keep=4096, R=3)) == SHAPE and step(dict(alpha=4096, R=0)) == SHAPE
    assert step(dict(w=8194)) == SHAPE and step(dict(m=4098)) == SHAPE and step(dict(copy=4097)) == SHAPE
    assert step({}, dict(w=None)) == NULL                                         # a bad one behind a good one: nothing is launched
    assert step({}, {}, dict(w=8192 + 4)) == SHAPE and step(dict(w=65536), dict(w=65536)) == SHAPE    # shared memory, a tied tensor twice
    assert step(dict(w=65536), dict(w=65536 - 64)) == SHAPE and step(dict(M=0, w=None)) == OK and step(count=0) == OK
    assert L.bsp_adamw_step(None, 0, 0, 1, 32, 0.0, 1e-3, 0.9, 0.999, 1e-8, 1, 0, None, None, None) == OK
    assert L.bsp_adamw_step(None, 1, 0, 1, 32, 0.0, 1e-3, 0.9, 0.999, 1e-8, 1, 0, None, None, None) == NULL


def test_bindings_refuse_what_does_not_fit():
    """Wrong places, shapes and types end in an error of the binding; nothing reaches the library."""
    x = torch.zeros(4, 128)
    for call in (lambda: bsp.bsp_fp8_quant(x), lambda: bsp.bsp_block_norm(x), lambda: bsp.bsp_block_norm_backward(x, x, x)):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            call()
    native = bsp.bsp._native()
    rest = (16, 0.0, 32, 0.0, 1e-3, 0.9, 0.999, 1e-8, 1, 0, None, None, 0, 0)
    none = (None,) * 4
    with pytest.raises(ValueError, match="contiguous tensors on the current device"):
        native.bsp_adamw_step([x], [x], [x], [x], *none, *rest)
    with pytest.raises(ValueError, match="one length"):
        native.bsp_adamw_step([x], [], [x], [x], *none, *rest)
    with pytest.raises(ValueError, match="one length"):
        native.bsp_adamw_step([], [], [], [], *none, [16], *rest[1:])
    with pytest.raises(TypeError, match="must hold tensors"):
        native.bsp_adamw_step([3], [x], [x], [x], *none, *rest)
    with pytest.raises(TypeError):
        native.bsp_adamw_step(5, [x], [x], [x], *none, *rest)
    with pytest.raises(TypeError):
        native.bsp_adamw_step([], [], [], [])
    assert native.bsp_adamw_step([], [], [], [], *none, *rest) == 0
    with pytest.raises(ValueError):
        bsp.bsp_adamw_state([x], bits=4)
    m, v, s = bsp.bsp_adamw_state([x, torch.zeros(300)], bits=8)
    assert m[0].dtype == torch.float8_e4m3fn and s[1].shape == (2, 2) and v[1].shape == (300,)


# ---- the plain implementations ------------------------------------------------------------------------------------------------
def test_codes_are_those_of_the_type():
    v = torch.cat([orc.e4m3_values(), -orc.e4m3_values()])
    assert torch.equal(orc.from_codes(orc.to_codes(v)), v)
    x = torch.randn(20000, dtype=torch.float64, generator=torch.Generator().manual_seed(1)) * 60
    ties = (orc.e4m3_values()[1:] + orc.e4m3_values()[:-1]) / 2
    x = torch.cat([x.clamp(-448, 448), ties, -ties]).float()
    assert torch.equal(orc.to_codes(x.double()), x.to(torch.float8_e4m3fn).view(torch.uint8))


@pytest.mark.parametrize("largest,e", [(448.0, 127), (448.0001, 128), (0.0, 127), (224.0, 126), (1.75, 119), (1.76, 120), (2.0 ** -149, 0), (3e38, 247)])
def test_exponents(largest, e):
    assert orc.exponent(largest) == e
    if 0 < e < 254 and largest:
        assert largest / 2.0 ** (e - 127) <= 448 < largest / 2.0 ** (e - 128)


@pytest.mark.parametrize("rms", [False, True])
def test_gradients_of_the_norms_against_differences(rms):
    """Central differences in 64 bits: their error is h^2 of the third derivative plus 2^-52 / h, about 1e-9 at h = 1e-5 here."""
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, dtype=torch.float64, generator=g)  # noqa: E731
    T, H = 6, 5
    a = dict(x=r(T, H), f=r(T, H), gate=r(2, H), w_post=1 + 0.1 * r(H), b_post=r(H), w_pre=1 + 0.1 * r(H), b_pre=r(H))
    dz, dh = r(T, H), r(T, H)

    def loss(**k):
        z, h, _, _ = orc.block_norm(k["x"], k["f"], True, True, rms, 1e-3, 0.8, k["gate"], k["w_post"], k["b_post"], k["w_pre"], k["b_pre"])
        return float((z * dz).sum() + (h * dh).sum())
    z, _, sp, sq = orc.block_norm(a["x"], a["f"], True, True, rms, 1e-3, 0.8, a["gate"], a["w_post"], a["b_post"], a["w_pre"], a["b_pre"])
    out = orc.block_norm_backward(dz, dh, z, a["f"], True, True, rms, 0.8, a["gate"], a["w_post"], a["b_post"], a["w_pre"], sp, sq)
    for name, t in a.items():
        got = out["d" + name]
        for i in range(t.numel()):
            step = torch.zeros_like(t).view(-1)
            step[i] = 1e-5
            up, down = loss(**{**a, name: t + step.view(t.shape)}), loss(**{**a, name: t - step.view(t.shape)})
            assert abs((up - down) / 2e-5 - float(got.reshape(-1)[i])) < 1e-7, (name, i)


def test_random_rounding_keeps_the_mean():
    """Equal values over many elements: the mean of what is stored is the value, within five standard deviations of a step."""
    n = 1 << 16
    x = torch.full((n,), 0.3, dtype=torch.float64)
    x[::256] = 1.0
    bits, bits2 = orc.random_bits(n, 3, 11)
    for b in (bits, bits2):
        q, s, _ = orc.stored(x, b, False)
        got = (q * s.repeat_interleave(256))[x == 0.3]
        step = 8 / 448   # the code's unit at 0.3 * 448
        assert abs(float(got.mean()) - 0.3) < 5 * step / 2 / math.sqrt(got.numel())
        assert got.unique().numel() == 2
    # neighbouring steps and seeds give other bits, the two halves are not alike
    assert float((bits == bits2).double().mean()) < 1e-3
    for other in (orc.random_bits(n, 4, 11)[0], orc.random_bits(n, 3, 12)[0]):
        assert float((bits == other).double().mean()) < 1e-3
    assert abs(float(bits.double().mean()) / 65535 - 0.5) < 5 * 0.29 / math.sqrt(n)


def test_quantisation_of_a_few_very_long_rows_is_refused():
    """Tiles of 128 x 128 are launched with 512 threads each: 2^23 of them side by side are 2^32 threads, however few the rows; by rows alone a line of up
    to 32 rows and 128 columns has 256."""
    q = bsp.lib().bsp_fp8_quant
    for rows in (1, 32, 64):
        for cols in (1 << 30, (1 << 30) + 1, (1 << 31) - 1):
            assert q(P, 1, rows, cols, bsp.FP8_BLOCK, P, P, None, None, None) == SHAPE
            assert q(P, 1, rows, cols, bsp.FP8_BLOCK, P, P, P, P, None) == SHAPE
            assert q(P, 1, rows, cols, bsp.FP8_ROW, None, None, P, P, None) == SHAPE
    assert q(P, 1, 33, 1 << 30, bsp.FP8_ROW, P, P, None, None, None) == SHAPE and q(P, 1, 1, (1 << 31) - 1, bsp.FP8_ROW, P, P, None, None, None) == SHAPE


def test_adamw_refuses_results_that_share_memory():
    """Whatever the step writes (weights, moments, scales, copies), of one tensor or of two: another workgroup would write the same place at the same time.
    The calls that are refused for it are good ones with one address moved; gradients, masks and factors may be shared."""
    L = bsp.lib()
    n, kinds = 4 * 512, ("w", "m", "v", "scales", "copy")
    size = {32: dict(w=4 * n, m=4 * n, v=4 * n, copy=2 * n), 8: dict(w=4 * n, m=n, v=n, scales=2 * (n // 256) * 4, copy=2 * n)}

    def step(bits, places, **more):
        each = [_Tensor(**dict(dict(g=1 << 30, keep=1 << 31, alpha=1 << 32, M=4, N=512, R=2), **p)) for p in places]
        args = dict(dict(gdt=0, cdt=1, t=1), **more)
        return L.bsp_adamw_step((_Tensor * len(each))(*each), len(each), args["gdt"], args["cdt"], bits, 0.0, 1e-3, 0.9, 0.999, 1e-8, args["t"], 0, None, None,
                                None)
    for bits in (32, 8):
        for order in (1, -1):                    # in ascending order of their addresses and not
            base = [{k: 1 << 20 | i << 16 | j << 22 for j, k in enumerate(kinds) if k in size[bits]} for i in range(3)][::order]
            for i, a in ((i, a) for i in range(3) for a in size[bits]):
                for o, b in ((o, b) for o in range(3) for b in size[bits] if (o, b) != (i, a)):
                    for shift in (0, 4 - size[bits][a], size[bits][b] - 4):
                        moved = [dict(p) for p in base]
                        moved[i][a] = base[o][b] + shift
                        assert step(bits, moved) == SHAPE, (bits, order, a, b, shift)


def test_form_of_a_product():
    """The query knows what the call would refuse, and that few tokens have no tiles and few outputs of many columns are split where there is scratch."""
    form = bsp.lib().bsp_matmul_fp8_form
    v = [C.c_int32(-1) for _ in range(3)]
    at = [C.byref(x) for x in v]
    assert form(4, 8, 128, 5, 0, *at) == DTYPE and form(4, 8, 128, 1, 2, *at) == DTYPE and form(4, 0, 128, 1, 0, *at) == SHAPE and form(-1, 8, 128, 1, 0, *at) == SHAPE
    assert form(4, 8, 128, 1, 0, None, at[1], at[2]) == NULL and form(4, 8, 128, 1, 0, at[0], at[1], None) == NULL and all(x.value == -1 for x in v)
    for T in (0, 1, 32):
        assert form(T, 4096, 1024, 1, 0, *at) == OK and [x.value for x in v] == [0, 0, 1]
    assert form(100, 64, 8192, 0, 0, *at) == OK and v[0].value in (64, 128, 256) and v[1].value >= 2 and v[2].value > 1
