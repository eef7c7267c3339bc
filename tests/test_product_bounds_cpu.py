"""The bounds of operators_bounds.py for products without a GPU: results of the 64-bit formulas, rounded to their type, are inside; the same formulas with a
mistake planted in them are not, at any of the sizes that the GPU tests use."""
import math

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


# ---- products -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,M,K", [(3, 40, 78), (37, 41, 334), (40, 72, 718), (20, 33, 2126), (34, 40, 8192)])
def test_a_mistake_in_a_product_is_seen(T, M, K, dtype):
    dt = DT[dtype]
    of = lambda x, block: orc.quant(x, block)  # noqa: E731
    a, b = rand(T + K, T, K), rand(M + K, M, K, std=1 / math.sqrt(K))
    (ac, ae), (bc, be) = of(a, False), of(b, False)
    av, bv = orc.value(ac, ae, K, False), orc.value(bc, be, K, False)
    s, bias, res = av @ bv.t(), rand(5, M).to(dt).to(D), rand(6, T, M).to(dt).to(D)
    want, bound = ob.layer(s, ob.product(av, bv, dt), dt, bias, True, res)
    assert outside(want, want, bound, dt) == 0
    finish = lambda x, bi=bias, act=True, re=res: (orc.gelu(x + bi) if act else x + bi) + re  # noqa: E731
    part = lambda lo, hi: av[:, lo:hi] @ bv[:, lo:hi].t()  # noqa: E731
    doubled = be.clone()
    doubled[:, -1] += 1
    shifted = torch.roll(av, 1, 0)
    wrong = {"the last step is lost": finish(s - part((K - 1) // 128 * 128, K)), "a step twice": finish(s + part(0, min(K, 128))),
             "sixteen columns are lost": finish(s - part(32, 48)), "a scale is one off": finish(av @ orc.value(bc, doubled, K, False).t()),
             "the tokens are shifted": finish(shifted @ bv.t()), "no bias": finish(s, 0.0), "no activation": finish(s, act=False),
             "no residual": finish(s, re=0.0)}
    # (the least of them, sixteen of 8192 columns, are 0.044 of a result's deviation before GELU halves it; of 16-bit results about 0.07 may be off there, which
    # N(0, 0.044) passes for a few in a hundred)
    for name, y in wrong.items():
        assert outside(y, want, bound, dt) >= T * M // 64, name
    # one column lost: from some outputs it takes more than they may be off by (of 16 bits in short sums; all of fp32)
    one = s - part(K // 2, K // 2 + 1)
    if dt == torch.float32 or K <= 1000:
        assert outside(finish(one), want, bound, dt) >= T * M // 64
