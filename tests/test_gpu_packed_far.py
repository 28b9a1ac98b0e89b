"""Packed attention where the scaled scores are far from zero: forward up to the largest scale that a call takes, backward as far as lse determines the weights."""
import math

import numpy as np
import pytest
import test_gpu_packed as packed
import torch
from test_gpu_packed import F, H8, Case

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu


def far_scores(lens, Hq, Hkv, D, causal, scale, lift, seed):
    """Scores that fp32 holds exactly: products of small whole numbers, and `lift` (a power of four) more for all keys of a row, so that weights are neither 0 nor 1 however far the scores are."""
    c = Case(lens, Hq, Hkv, D, causal, scale=scale, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in (c.q, c.k):
        t[:] = torch.randint(-3, 4, t.shape, generator=g, device="cuda").bfloat16()
        t[..., 0] = math.sqrt(lift)
    return c


@pytest.mark.parametrize("lens,Hq,Hkv", [([40, 1, 128], 2, 1), ([200, 129, 256], 2, 2), ([900], 1, 1), ([700, 300, 60, 390], 6, 2)])
@pytest.mark.parametrize("causal,D", [(0, 64), (1, 64), (1, 32)])
@pytest.mark.parametrize("scale,lift", [(1.0, 0), (1.0, 4.0 ** 8), (0.01, 4.0 ** 9), (40.0, 4.0 ** 7), (1e4, 0), (1e8, 0), (1e8, 4.0 ** 6), (1e12, 4.0 ** 9), (1e30, 0), (1e30, 4.0 ** 9)])
def test_scores_far_from_zero(lens, Hq, Hkv, causal, D, scale, lift):
    """Up to the largest scale that a call takes the weights of a row are those of its scores' differences.  The products of the scores and their sums are exact; scaled, a score is off by
    its factor's rounding and one more, 2^-23 of itself, and so is lse; a difference of scores by 2^-22 of itself, whose exponential is 0 in bf16 and in fp32 where that is a step (2^-8)."""
    c = far_scores(lens, Hq, Hkv, D, causal, scale, lift, seed=len(lens) + Hq)
    out = c.new()
    vd.vardrop_packed_plan(c.cu, c.cfg, c.plan)
    vd.vardrop_attn_packed_fwd(c.q, c.k, c.v, c.plan, c.cfg, out["o"], out["lse"], out["ws"])
    assert vd.ws_status(out["ws"]) == vd.OK
    scale = float(np.float32(scale))
    for a, b in c.spans:
        for h in range(Hq):
            Q, K, V = (t.double() for t in (c.q[a:b, h], c.k[a:b, h * Hkv // Hq], c.v[a:b, h * Hkv // Hq]))
            S = Q @ K.T
            assert torch.equal(S, S.float().double()) and float(S.abs().max()) < 2 ** 24
            S = S * scale
            if causal:
                S = S.masked_fill(torch.ones_like(S, dtype=torch.bool).triu(1), -math.inf)
            P = torch.softmax(S, 1)
            O, lse = P @ V, torch.logsumexp(S, 1)
            rel = H8 + 2 * F                 # of a rounded P; exponentials and sums
            bound = (rel * P) @ V.abs() + H8 * O.abs() + 1e-6
            assert bool(((out["o"][a:b, h].double() - O).abs() <= bound).all()), (a, h)
            assert bool(((out["lse"][h, a:b].double() - lse).abs() <= 2.0 ** -22 * lse.abs() + F).all()), (a, h)


@pytest.mark.parametrize("lens,Hq,Hkv", [([40, 5], 2, 1), ([40, 5], 2, 2), ([300, 131], 2, 1)])
@pytest.mark.parametrize("scale,lift", [(0.0, 4.0 ** 8), (0.9, 4.0 ** 8), (7.0, 4.0 ** 6)])
def test_gradients_of_scores_far_from_zero(lens, Hq, Hkv, scale, lift, monkeypatch):
    """lse comes with 24 bits, itself off by 2^-22; divided by the scale it sees two roundings and a split into three bf16 terms, and five sums with the scores of half a step of fp32 each: 4.5 2^-22
    of lse and of the scores' magnitudes together, in the exponents."""
    c = far_scores(lens, Hq, Hkv, 64, 1, scale, lift, seed=5)
    out = c.run()
    monkeypatch.setattr(packed, "F", 2.0 ** -19)
    val, off, live = packed.reference(c.q, c.k, c.v, c.d_o, c.spans, 1, c.scale)
    for n in ("dq", "dk", "dv"):
        err = (out[n].double() - val[n]).abs()[live]
        assert bool((err <= off[n][live] + 1e-6 * c.scale * 64).all()), (n, float(err.max()))


@pytest.mark.parametrize("lens,Hq,Hkv", [([40, 5], 2, 1), ([40, 5], 2, 2), ([300, 131], 2, 1)])
@pytest.mark.parametrize("scale", [1.1, 1e8, 1e30])
def test_gradients_that_lse_does_not_determine_are_reported(lens, Hq, Hkv, scale):
    """|lse| above 2^16: the bits that fp32 has for it leave the weights of a row open."""
    c = far_scores(lens, Hq, Hkv, 64, 1, scale, 4.0 ** 8, seed=6)
    out = c.new()
    c.call(out)
    assert vd.ws_status(out["ws"]) == vd.ERR_UNSUPPORTED
