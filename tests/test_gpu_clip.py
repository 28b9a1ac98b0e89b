"""vardrop_grad_clip against the formula in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def clip(grads, max_norm, outs=None, eps=1e-6):
    norm = torch.full((1,), -1.0, device="cuda")
    ws = vd.alloc_ws(vd.vardrop_grad_clip_workspace_bytes())
    ws[256:] = 0xFF
    vd.vardrop_grad_clip(grads, vd.ClipCfg(max_norm, eps), outs, norm, ws)
    torch.cuda.synchronize()
    return float(norm.item()), vd.ws_status(ws)


def wanted(grads, max_norm, eps=1e-6):
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    return norm, min(1.0, max_norm / (norm + eps))


def check(grads, max_norm, in_place):
    """A factor rounded to fp32 and a product rounded to fp32 and then to the type: 2^-24 twice, and half a step.  Below the type's least normal value half a step is
    half its least value."""
    norm, factor = wanted(grads, max_norm)
    before = [g.clone() for g in grads]
    outs = None if in_place else [torch.full_like(g, 3.0) for g in grads]
    got, status = clip(grads, max_norm, outs)
    assert status == vd.OK and abs(got - norm) <= 2.0 ** -23 * norm
    for b, g, o in zip(before, grads, outs or grads):
        if not in_place:
            assert torch.equal(b, g)
        want = b.double() * factor
        info = torch.finfo(b.dtype)
        assert bool(((o.double() - want).abs() <= want.abs() * (info.eps / 2 + 3 * 2.0 ** -24) + info.smallest_normal * info.eps / 2).all())
        if factor == 1.0:
            assert torch.equal(o, b)


def tensors(sizes, seed, types=TYPES, std=0.01):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * std).to(types[i % len(types)]) for i, n in enumerate(sizes)]


SIZES = [[1], [7], [0, 5, 0], [4095, 4096, 4097], [8191, 8192, 8193, 16384, 16385], [512 * 512, 512, 96 * 512, 96, 3], [1 << 22, 33], list(range(1, 64)), list(range(1, 70)),
         [13] * 1023 + [4], [13] * 1024, [13] * 1025, [37] * 2500]


@pytest.mark.parametrize("sizes", SIZES, ids=[f"{len(s)}x{max(s)}" for s in SIZES])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("share", [0.3, 5.0])
def test_sizes(sizes, in_place, share):
    grads = tensors(sizes, len(sizes))
    check(grads, share * max(wanted(grads, 1.0)[0], 1e-3), in_place)


@pytest.mark.parametrize("types", [[torch.bfloat16], [torch.float16], [torch.float32], TYPES])
@pytest.mark.parametrize("shift", [0, 1, 3, 5])
def test_views_at_odd_offsets(types, shift):
    """Gradients as views of buckets: not one of them on a 16-byte boundary, neighbours left as they are."""
    n = [1, 2, 9, 4099, 31, 20000]
    flat = {t: (torch.randn(40000, device="cuda") * 0.1).to(t) for t in types}
    for out_shift in (shift, shift + 2):
        outs = {t: torch.full((40100,), 9.0, dtype=t, device="cuda") for t in types}
        grads, views, used = [], [], {t: shift for t in types}
        for i, m in enumerate(n):
            t = types[i % len(types)]
            grads.append(flat[t][used[t]:used[t] + m])
            views.append(outs[t][used[t] - shift + out_shift:used[t] - shift + out_shift + m])
            used[t] += m + 1                    # a gap of one between neighbours
        norm, factor = wanted(grads, 1.0)
        got, status = clip(grads, 1.0, views)
        assert status == vd.OK and abs(got - norm) <= 2.0 ** -23 * norm
        total = 0
        for g, v in zip(grads, views):
            assert bool(((v.double() - g.double() * factor).abs() <= g.double().abs() * factor * (torch.finfo(g.dtype).eps / 2 + 3 * 2.0 ** -24)
                         + torch.finfo(g.dtype).smallest_normal * torch.finfo(g.dtype).eps / 2).all())
            total += v.numel()
        assert sum(int((o == 9.0).sum()) for o in outs.values()) >= 40100 * len(types) - total


def test_norm_alone():
    grads = tensors([1000, 333], 1)
    before = [g.clone() for g in grads]
    norm, status = clip(grads, 0.0)
    assert status == vd.OK and abs(norm - wanted(grads, 1.0)[0]) <= 2.0 ** -23 * norm
    assert all(torch.equal(a, b) for a, b in zip(before, grads))
    assert clip([], 0.0) == (0.0, vd.OK) and clip([], 1.0) == (0.0, vd.OK)
    zeros = [torch.zeros(100, device="cuda")]
    check(zeros, 1.0, True)


@pytest.mark.parametrize("size", [1e-30, 1e-22, 1e18, 1e25])
def test_squares_beyond_the_range_of_fp32(size):
    check([torch.full((1000,), size, device="cuda"), torch.full((77,), -size, device="cuda")], 1.0, False)


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite(value):
    grads = tensors([5000, 77], 2)
    grads[1][40] = value
    before = [g.clone() for g in grads]
    norm, status = clip(grads, 0.1)
    assert status == vd.ERR_NONFINITE and (math.isnan(norm) if math.isnan(value) else norm == math.inf)
    assert all(torch.equal(a.nan_to_num(1.0), b.nan_to_num(1.0)) for a, b in zip(before, grads))
    outs = [torch.zeros_like(g) for g in grads]
    clip(grads, 0.1, outs)
    assert all(torch.equal(a.nan_to_num(1.0), b.nan_to_num(1.0)) for a, b in zip(outs, grads))


def test_runs_repeat_bit_for_bit_and_replay():
    grads = tensors([1 << 20, 4097, 5], 3)
    ref = [torch.empty_like(g) for g in grads]
    first = clip(grads, 0.5, ref)
    assert clip(grads, 0.5, [torch.empty_like(g) for g in grads]) == first
    outs, norm, ws = [torch.empty_like(g) for g in grads], torch.zeros(1, device="cuda"), vd.alloc_ws(vd.vardrop_grad_clip_workspace_bytes())
    cfg = vd.ClipCfg(0.5, 1e-6)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        vd.vardrop_grad_clip(grads, cfg, outs, norm, ws)
    graph.replay()
    torch.cuda.synchronize()
    assert float(norm.item()) == first[0] and all(torch.equal(a, b) for a, b in zip(outs, ref))
    for g in grads:
        g.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert abs(float(norm.item()) - 2 * first[0]) <= 2.0 ** -22 * first[0]


def test_transposed_gradients():
    g = torch.randn(33, 65, device="cuda")
    check([g.t()], 1.0, True)
    with pytest.raises(ValueError):
        clip([g[:, :64]], 1.0)


def test_offsets_beyond_32_bits():
    """2.2e9 values of one tensor, zeros but for some behind the 2^31st."""
    n = 2_200_000_007
    big = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([5, 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 12345, n - 1], device="cuda")
    big[at] = 2.0
    norm, status = clip([big], 1.0)
    assert status == vd.OK and abs(norm - math.sqrt(20)) < 1e-5
    want = (2.0 * torch.tensor(1 / (math.sqrt(20) + 1e-6))).bfloat16().cuda()
    assert bool((big[at] == want).all()) and int(torch.count_nonzero(big)) == 5


def test_refusals():
    g = torch.randn(64, device="cuda")
    for grads, outs in (([g.double()], None), ([g.cpu()], None), ([1.0], None), ([g], [g.bfloat16()]), ([g], [g[:63]]), ([g], []), ([g.view(8, 8)], [g.view(8, 8).t()])):
        with pytest.raises(ValueError):
            clip(grads, 1.0, outs)
    with pytest.raises(TypeError):
        clip(g, 1.0)
    for max_norm, eps in ((-1.0, 0.0), (float("nan"), 0.0), (1.0, -1.0)):
        with pytest.raises(vd.VardropError):
            clip([g], max_norm, eps=eps)
    with pytest.raises(vd.VardropError):
        clip([g[:32]], 1.0, [g[16:48]])
    assert np.isfinite(clip([g], 1.0)[0])
