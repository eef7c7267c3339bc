"""The norms' results, statistics and gradients against 64 bits, element by element with the bounds of operators_bounds.py (which test_norm_bounds_cpu.py
holds against planted mistakes)."""
import pytest
import torch

import operators_bounds as ob
import operators_oracle as orc
import paper_2009_08065_amd as bsp

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
D = torch.float64


def rand(seed, *shape, std=1.0, dt=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dt)


def inside(got, want, bound, what=""):
    assert got.shape == want.shape, what
    err = (got.to(want) - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float((err / bound).nan_to_num(0, 0, 0).max()):.3g} of what is allowed"


# ---- norms --------------------------------------------------------------------------------------------------------------------
def norm_case(seed, T, H, dt, gate_rows, weights, aligned, offset=0.0):
    def place(t):
        if aligned:
            return t
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        flat[1:].copy_(t.reshape(-1))
        return flat[1:].view(t.shape)
    c = dict(x=rand(seed, T, H) + offset, f=rand(seed + 1, T, H, std=0.5) + offset, gate=rand(seed + 2, gate_rows, H, std=0.5) if gate_rows else None,
             dz=rand(seed + 3, T, H), dh=rand(seed + 4, T, H))
    for i, k in enumerate(("w_post", "b_post", "w_pre", "b_pre")):
        c[k] = (k[0] == "w") + rand(seed + 5 + i, H, std=0.2) if weights else None
    return {k: None if v is None else place(v.to(dt)) for k, v in c.items()}


def check(T, H, dt, rms, post, pre, gate_rows, x_scale=0.8125, weights=True, aligned=True, offset=0.0):
    c = norm_case(T + H, T, H, dt, gate_rows, weights, aligned, offset)
    eps = 2.0 ** -17
    e = {k: None if v is None else v.to(D) for k, v in c.items()}
    norms, kind = (bsp.NORM_POST if post else 0) | (bsp.NORM_PRE if pre else 0), bsp.NORM_RMS if rms else bsp.NORM_LAYER
    on = dict(w_post=c["w_post"] if post else None, b_post=c["b_post"] if post else None, w_pre=c["w_pre"] if pre else None, b_pre=c["b_pre"] if pre else None)
    en = {k: None if v is None else v.to(D) for k, v in on.items()}
    what = f"T={T} H={H} {dt} rms={rms} post={post} pre={pre} gate={gate_rows} weights={weights} aligned={aligned}"
    Z, Hn, sp, sq = bsp.bsp_block_norm(c["x"], c["f"], norms, kind=kind, eps=eps, x_scale=x_scale, gate=c["gate"], **on)
    z, zb, st, sb = ob.forward_z(e["x"], e["f"], post, rms, eps, x_scale, e["gate"], en["w_post"], en["b_post"], dt)
    inside(Z, z, zb, "Z " + what)
    if post:
        inside(sp, st, sb, "stats_post " + what)
    if pre:
        v = Z.to(D)
        rq, rb = ob.stats(v, rms, eps)
        inside(sq, rq, rb, "stats_pre " + what)
        h, hb = ob.normed(v, rq, rb, en["w_pre"], en["b_pre"])
        inside(Hn, h, ob.rounded_to(dt, h, hb), "H " + what)
    if rms:
        assert all(s is None or not s[:, 0].any() for s in (sp, sq)), what
    # backward from statistics of its own (rounded once, and exact from there on), not from those of the forward kernel
    kept = {"stats_post": orc.statistics(e["f"], rms, eps).float() if post else None, "stats_pre": orc.statistics(Z.to(D), rms, eps).float() if pre else None}
    args = dict(norms=norms, kind=kind, x_scale=x_scale, gate=c["gate"], **on, **kept)
    got = bsp.bsp_block_norm_backward(c["dz"], c["dh"] if pre else None, Z if pre else None, c["f"], **args)
    ref = ob.backward(e["dz"], e["dh"] if pre else None, Z.to(D) if pre else None, e["f"], post, pre, rms, x_scale, e["gate"], en["w_post"], en["b_post"],
                      en["w_pre"], *(None if s is None else s.to(D) for s in kept.values()), dt)
    for name, there in (("dx", True), ("df", True), ("dw_post", post and weights), ("db_post", post and weights), ("dw_pre", pre and weights),
                        ("db_pre", pre and weights), ("dgate", gate_rows > 0)):
        assert (got[name] is not None) == bool(there), (name, what)
        if there:
            want, bound = ref[name]
            inside(got[name], want, bound, name + " " + what)
            # and as a whole: fp32 a few 1e-6 of the sums' own magnitudes, 16 bits their rounding
            scale = 1e-6 if got[name].dtype == torch.float32 else ob.half(dt)
            assert float((got[name].to(D) - want).norm()) <= scale * float(want.norm()) + float(bound.norm()) * 0.5, (name, what)


WIDTHS = [1, 5, 8, 64, 79, 128, 130, 200, 256, 257, 512, 513, 770, 1024, 1030, 1500, 2048, 2056, 4096, 4102, 5000, 8190, 8192]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("H", WIDTHS)
def test_norms_element_by_element(H, dtype):
    dt = DT[dtype]
    check(67, H, dt, False, True, True, 1)
    check(5, H, dt, False, True, True, 5, aligned=False)
    check(130, H, dt, True, True, True, 2)
    check(1, H, dt, False, False, True, 0, x_scale=1.0)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("T,gate_rows", [(120, 0), (120, 8), (120, 120), (1200, 3), (1200, 600), (2500, 0)])
def test_norms_in_every_form_element_by_element(rms, post, pre, T, gate_rows):
    check(T, 136, torch.float32, rms, post, pre, gate_rows)
    check(T, 770, torch.float32, rms, post, pre, gate_rows)
    check(T, 1536, torch.bfloat16, rms, post, pre, gate_rows, weights=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H", [96, 1024, 4096])
def test_statistics_of_rows_with_large_means(H, dtype):
    """The mean as it is kept, far above the deviation: what its rounding adds to the deviation is part of the bound."""
    check(33, H, DT[dtype], False, True, True, 0, offset=100.0)
