"""Both halves of one projection as the branches of a gated activation: widths whose second half begins on 16 bytes give what tensors of their own give, others are refused."""
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu


def halves(B, N, C, dtype, seed=0):
    both = torch.randn((B, N, 2 * C), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)
    return both, both[..., :C], both[..., C:]


@pytest.mark.parametrize("dtype,C", [(torch.float32, 4), (torch.float32, 12), (torch.float32, 260), (torch.bfloat16, 8), (torch.float16, 40)])
@pytest.mark.parametrize("kind", [vd.ACT_GELU, vd.ACT_SILU])
def test_the_same_as_tensors_of_their_own(dtype, C, kind):
    B, N = 3, 21
    both, a, b = halves(B, N, C, dtype)
    d_y = halves(B, N, C, dtype, 1)[1].contiguous()
    n_sel = torch.tensor([N, 4, 0], dtype=torch.int32, device="cuda")
    got = []
    for stride, x, z, grads in ((2 * C, a, b, torch.full_like(both, 7.0).split(C, 2)), (0, a.contiguous(), b.contiguous(), [torch.full_like(d_y, 7.0) for _ in range(2)])):
        cfg = vd.ActCfg(B, N, C, vd.DTYPES[dtype], kind, 1, B, stride)
        ckpt, y, again = vd.alloc_act_ckpt(cfg), torch.full_like(d_y, 7.0), torch.full_like(d_y, 7.0)
        vd.vardrop_act_fwd(x, z, n_sel, cfg, y, ckpt)
        vd.vardrop_act_bwd(d_y, ckpt, n_sel, cfg, *grads, again)
        got.append((y, *grads, again))
    assert all(torch.equal(p, q) for p, q in zip(*got))


@pytest.mark.parametrize("dtype,C", [(torch.bfloat16, 12), (torch.float16, 4)])
def test_halves_off_sixteen_bytes_are_refused(dtype, C):
    both, a, b = halves(2, 5, C, dtype)
    cfg = vd.ActCfg(2, 5, C, vd.DTYPES[dtype], vd.ACT_SILU, 1, 0, 2 * C)
    y = torch.full((2, 5, C), 7.0, dtype=dtype, device="cuda")
    with pytest.raises(vd.VardropError, match="16-byte"):
        vd.vardrop_act_fwd(a, b, None, cfg, y, None)
    assert bool((y == 7.0).all())
