"""The operators of a model's ends and middle on two streams at once: every call of both is queued before the host waits for any, each stream with buffers and a workspace of its own."""
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
ROUNDS = 8


def rng(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(shape, dtype, g):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


class Loss:
    def __init__(self, T, V, C, gaps, seed):
        g = rng(seed)
        self.cfg = vd.LossCfg(T, V, C, 0, C ** -0.5)
        self.h, self.w = normal((T, C), BF, g), normal((V, C), BF, g)
        self.labels = torch.randint(0, V, (T,), generator=g, device="cuda").int()
        self.labels[torch.rand(T, generator=g, device="cuda") < gaps] = -1
        self.d_loss = torch.rand(T, generator=g, device="cuda")
        self.ws = vd.alloc_ws(vd.vardrop_loss_workspace_bytes(self.cfg))
        self.out = [torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty_like(self.h), torch.empty_like(self.w)]

    def call(self):
        loss, lse, d_h, d_w = self.out
        vd.vardrop_loss_fwd(self.h, self.w, self.labels, self.cfg, loss, lse, self.ws)
        vd.vardrop_loss_bwd(self.h, self.w, self.labels, lse, self.d_loss, self.cfg, d_h, d_w, self.ws)


class Embed:
    def __init__(self, T, V, C, seed):
        g = rng(seed)
        self.cfg = vd.EmbedCfg(T, V, C, vd.DTYPES[FP], vd.DTYPES[BF], 0, 1.5)
        self.table, self.d_x = normal((V, C), FP, g), normal((T, C), BF, g)
        self.idx = (torch.rand(T, generator=g, device="cuda") ** 4 * V).int().clamp(0, V - 1)
        self.ws = vd.alloc_ws(vd.vardrop_embed_workspace_bytes(self.cfg))
        self.out = [torch.empty_like(self.d_x), torch.empty_like(self.table)]

    def call(self):
        vd.vardrop_embed_fwd(self.table, self.idx, self.cfg, self.out[0], self.ws)
        vd.vardrop_embed_bwd(self.d_x, self.idx, self.cfg, self.out[1], self.ws)


class Act:
    ws = None

    def __init__(self, B, N, C, kept, seed):
        g = rng(seed)
        self.cfg = vd.ActCfg(B, N, C, 0, vd.ACT_SILU, 1, 1, 2 * C)
        self.ab, self.d_y = normal((B, N, 2 * C), BF, g), normal((B, N, C), BF, g)
        self.n_sel = torch.tensor([kept], dtype=torch.int32, device="cuda")
        self.ckpt = vd.alloc_act_ckpt(self.cfg)
        self.out = [torch.zeros_like(self.d_y), torch.zeros_like(self.d_y), torch.zeros_like(self.ab)]

    def call(self):
        C, (y, again, d_ab) = self.cfg.C, self.out
        vd.vardrop_act_fwd(self.ab[..., :C], self.ab[..., C:], self.n_sel, self.cfg, y, self.ckpt)
        vd.vardrop_act_bwd(self.d_y, self.ckpt, self.n_sel, self.cfg, d_ab[..., :C], d_ab[..., C:], again)


PAIRS = {"loss": lambda: [Loss(900, 1200, 64, 0.0, 1), Loss(900, 1200, 64, 0.4, 2)],
         "loss of one row of tiles and a long one": lambda: [Loss(200, 30000, 128, 0.1, 3), Loss(5000, 2000, 256, 0.5, 4)],
         "embeddings, sorted": lambda: [Embed(20000, 5000, 136, 5), Embed(20000, 5000, 136, 6)],
         "embeddings, placed and looked through": lambda: [Embed(4000, 30000, 64, 7), Embed(9000, 300, 512, 8)],
         "activation": lambda: [Act(4, 700, 520, 700, 9), Act(4, 700, 520, 233, 10)],
         "different operators": lambda: [Loss(2000, 3000, 136, 0.3, 11), Embed(9000, 700, 256, 12)]}


@pytest.mark.parametrize("pair", PAIRS)
def test_two_streams_at_once(pair):
    cases = PAIRS[pair]()
    want = []
    for case in cases:
        case.call()
        torch.cuda.synchronize()
        want.append([t.clone() for t in case.out])
        for t in case.out:
            t.zero_()
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for i in range(ROUNDS):
        for case, stream in zip(cases, streams) if i % 2 else zip(reversed(cases), reversed(streams)):
            with torch.cuda.stream(stream):
                case.call()
    torch.cuda.synchronize()
    for case, w in zip(cases, want):
        assert all(torch.equal(a, b) for a, b in zip(case.out, w))
        assert case.ws is None or vd.ws_status(case.ws) == vd.OK
