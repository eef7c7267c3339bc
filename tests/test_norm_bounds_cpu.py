"""The bounds of operators_bounds.py for norms without a GPU: results of the 64-bit formulas, rounded to their type, are inside; the same formulas with a
mistake planted in them are not, at any of the sizes that the GPU tests use."""
import pytest
import torch

import operators_bounds as ob
import operators_oracle as orc

D = torch.float64
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def rand(seed, *shape, std=1.0):
    return torch.randn(*shape, dtype=D, generator=torch.Generator().manual_seed(seed)) * std


def outside(got, want, bound, dt):
    return int((~((got.to(dt).to(D) - want).abs() <= bound)).sum())


# ---- norms --------------------------------------------------------------------------------------------------------------------
WIDTHS = [5, 8, 64, 79, 128, 130, 200, 256, 257, 512, 513, 770, 1024, 1030, 1500, 2048, 2056, 4096, 4102, 5000, 8190, 8192]


def planted(dz, dh, z, f, post, pre, rms, x_scale, gate, w_post, b_post, w_pre, sp, sq, mistake=""):
    """The gradients by their formulas, with one mistake."""
    T, out = dz.shape[0], {}

    def sums(t):
        if mistake == "sums of zero":
            return torch.zeros_like(t[0])
        return t[:-1].sum(0) if mistake == "a row is lost" else t.sum(0)

    def back(d, v, st, w):
        if mistake == "mean and deviation change places":
            st = st.flip(1)
        hat = (v - st[:, :1]) * st[:, 1:]
        g = d if w is None or mistake == "no weight" else d * w
        c1, c2 = (g * hat).mean(1, keepdim=True), g.mean(1, keepdim=True)
        if mistake == "no mean of g hat":
            c1 = c1 * 0
        if mistake == "no mean of g" or rms:
            c2 = c2 * 0
        return st[:, 1:] * (g - hat * c1 - c2), sums(d * hat), sums(d)
    d = dz
    if pre:
        g, out["dw_pre"], out["db_pre"] = back(dh, z, sq, w_pre)
        d = g if mistake == "no dZ" else d + g
    out["dx"] = d if mistake == "no scale of the residual" else x_scale * d
    n = f
    if post:
        n = orc.normed(f, sp, w_post, None if mistake == "no bias" else b_post)
    if gate is not None:
        rows = orc.rows_of(gate.roll(1, 0) if mistake == "another gate row" else gate, T)
        out["dgate"] = torch.stack([sums(p) for p in (d * n).view(gate.shape[0], -1, d.shape[1])])
        d = d if mistake == "no gate" else d * rows
    if post:
        d, out["dw_post"], out["db_post"] = back(d, f, sp, w_post)
    out["df"] = d
    return out


def seen(T, H, dt, rms, post, pre, gate_rows, mistakes):
    """{mistake: the results that show it}"""
    eps, x_scale = 2.0 ** -17, 0.8125
    c = {k: (1.0 * (k[0] == "w") + rand(T + H + i, *s, std=t)).to(dt).to(D) for i, (k, s, t) in enumerate(
        (("x", (T, H), 1.0), ("f", (T, H), 0.5), ("dz", (T, H), 1.0), ("dh", (T, H), 1.0), ("gate", (max(gate_rows, 1), H), 0.5), ("w_post", (H,), 0.2),
         ("b_post", (H,), 0.2), ("w_pre", (H,), 0.2)))}
    gate = c["gate"] if gate_rows else None
    z, zb, sp, _ = ob.forward_z(c["x"], c["f"], post, rms, eps, x_scale, gate, c["w_post"] if post else None, c["b_post"] if post else None, dt)
    assert outside(z, z, zb, dt) == 0
    z = z.to(dt).to(D)
    sp = sp.float().to(D) if post else None
    sq = orc.statistics(z, rms, eps).float().to(D) if pre else None
    args = (c["dz"], c["dh"], z, c["f"], post, pre, rms, x_scale, gate, c["w_post"] if post else None, c["b_post"] if post else None, c["w_pre"] if pre else None,
            sp, sq)
    ref = ob.backward(*args, dt)
    types = {k: dt if k in ("dx", "df") else torch.float32 for k in ref}
    right = planted(*args)
    assert set(right) == set(ref)
    for k, (want, bound) in ref.items():
        assert torch.allclose(right[k], want, rtol=1e-9, atol=1e-9) and outside(right[k], want, bound, types[k]) == 0, k
    out = {}
    for m in mistakes:
        wrong = planted(*args, mistake=m)
        out[m] = {k for k, (want, bound) in ref.items() if outside(wrong[k], want, bound, types[k])}
    return out


SUMS = {"dw_pre", "db_pre", "dw_post", "db_post", "dgate"}


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("H", WIDTHS)
def test_a_mistake_in_a_gradient_of_the_norms_is_seen(H, dtype):
    """Every result that a mistake touches leaves its bound, at every width and at the row counts of the GPU tests."""
    for T, gate_rows in ((67, 1), (5, 5), (130, 2)):
        got = seen(T, H, DT[dtype], False, True, True, gate_rows, ("sums of zero", "a row is lost", "no mean of g", "no mean of g hat", "no weight", "no dZ", "no gate",
                                                                  "no bias", "no scale of the residual", "mean and deviation change places"))
        assert got["sums of zero"] == SUMS and got["a row is lost"] == SUMS
        for m in ("no mean of g", "no mean of g hat", "no weight", "mean and deviation change places"):
            assert {"dx", "df"} <= got[m], (m, T)
        assert "dx" in got["no scale of the residual"] and {"df", "dw_post"} <= got["no gate"] and "dgate" in got["no bias"]
        assert {"dx", "df", "dgate", "dw_post", "db_post"} <= got["no dZ"]
    assert {"df", "dw_post", "db_post"} <= seen(130, H, DT[dtype], True, True, True, 2, ("another gate row",))["another gate row"]


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("T,gate_rows", [(120, 0), (120, 8), (120, 120), (1200, 3), (1200, 600), (2500, 0)])
def test_a_mistake_in_many_rows_is_seen(rms, T, gate_rows):
    """One row of up to 2500 that a sum has lost."""
    for H, dt in ((136, torch.float32), (770, torch.float32), (1536, torch.bfloat16)):
        got = seen(T, H, dt, rms, True, True, gate_rows, ("sums of zero", "a row is lost"))
        want = SUMS if gate_rows else SUMS - {"dgate"}
        assert got["sums of zero"] == want and got["a row is lost"] == want


def test_a_mistake_in_the_statistics_is_seen():
    for H in WIDTHS:
        v = rand(H, 20, H)
        for rms in (False, True):
            want, bound = ob.stats(v, rms, 2.0 ** -17)
            assert outside(want, want, bound, torch.float32) == 0
            for wrong in (orc.statistics(v, not rms, 2.0 ** -17), orc.statistics(v, rms, 2.0 ** -10), orc.statistics(torch.cat([v, v[:, :1] * 0], 1), rms, 2.0 ** -17)):
                assert outside(wrong, want, bound, torch.float32) >= 20
