"""vardrop_loss_bwd where the tokens' d_loss lie far apart and the vocabulary is large: what an entry of G loses on its way through 16 bits, token by token."""
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

U = 2.0 ** -24          # half a step of fp32


@pytest.mark.parametrize("V", [1000, 131072])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_each_token_has_the_bound_of_its_own_entries(V, dtype):
    """G goes to 16 bits times what takes the largest |d_loss| to 16320.  bf16 has the range for every token.  In fp16 an entry is off by half a step of its own or of the least number, 2^-25 / 16320 of the
    largest |d_loss|: so entries d_loss p below 2^-28 of that have fewer bits, below 2^-39 none, however large the token's label's entry is."""
    T, C, scale = 96, 64, 0.5
    g = torch.Generator(device="cuda").manual_seed(V)
    h, w = (torch.randn(*s, generator=g, device="cuda").to(dtype) for s in ((T, C), (V, C)))
    labels = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    d_loss = torch.exp2(-(torch.arange(T, device="cuda") % 25).float()) * 1024
    cfg = vd.LossCfg(T, V, C, vd.DTYPES[dtype], scale)
    ws = vd.alloc_ws(vd.vardrop_loss_workspace_bytes(cfg))
    loss, lse, d_h = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(h)
    vd.vardrop_loss_fwd(h, w, labels, cfg, loss, lse, ws)
    vd.vardrop_loss_bwd(h, w, labels, lse, d_loss, cfg, d_h, None, ws)
    assert vd.ws_status(ws) == vd.OK
    half = torch.finfo(dtype).eps / 2
    least = 2.0 ** -25 / 16320 * 1024 * scale if dtype == torch.float16 else 0.0
    w = w.double()
    logits = scale * (h.double() @ w.T)
    exact = torch.logsumexp(logits, 1, keepdim=True)
    p = torch.exp(logits - exact)
    G = p.scatter_add(1, labels.long()[:, None], torch.full((T, 1), -1.0, dtype=torch.float64, device="cuda")) * (scale * d_loss.double()[:, None])
    # the logits: two roundings of the running sum for each 16 of their products; lse: as many of its sum of exponentials
    err = scale * (h.double().abs() @ w.abs().T).amax(1, keepdim=True) * (C / 8 + 8) * U
    size = G.abs() * (half + 4 * U) + p * (scale * d_loss.double()[:, None]) * (3 * err + (V / 128 + 64) * U + 2.0 ** -20)
    size = size + (size + G.abs()).clamp_max(least * (1 + 2.0 ** -10))
    want, bound = G @ w, size @ w.abs() + (G.abs() @ w.abs()) * (V / 8 + 40) * U
    # d_h itself is fp16 too: half a step, of its least number at least
    tiny = torch.finfo(dtype).smallest_normal * half
    assert bool(((d_h.double() - want).abs() <= bound + (want.abs() + bound) * half + tiny).all())
