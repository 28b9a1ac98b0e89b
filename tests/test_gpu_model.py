"""The operators of a model's ends and middle as a training step calls them, with the norms and the clipping between and behind them: embeddings of tokens, a gated feed-forward block on the normed stream with
its activation held in 8 bits, a norm, the loss over a vocabulary, and the way back to every weight.  Padding tokens have neither index nor label.  Against the same model in 64 bits, whose activation's
derivative is taken where the checkpoint says.

Tolerance: a tensor of 16 bits is off by at most 2^-8 of its values from being rounded, products with weights of random sign pass a relative error on as it is, errors of different roundings add up at most
linearly.  The longest way (to the embeddings) rounds x, u, a | b, y, z, h2, u2, G, then d_u2, dz, dy, d_a | d_b, du, dx1, dx2 and dx: 16 tensors."""
import math

import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

BOUND = 16 * 2.0 ** -8
EPS = 1e-5
BLOCK = 32


def rms(t, w):
    return t / torch.sqrt((t * t).mean(-1, keepdim=True) + EPS) * w


class HeldAct(torch.autograd.Function):
    """silu(a) o b, differentiated at the values of a checkpoint."""
    @staticmethod
    def forward(ctx, a, b, ha, hb):
        ctx.save_for_backward(ha, hb)
        return a * torch.sigmoid(a) * b

    @staticmethod
    def backward(ctx, d):
        ha, hb = ctx.saved_tensors
        p = torch.sigmoid(ha)
        return d * hb * (p + ha * p * (1 - p)), d * ha * p, None, None


class Step:
    def __init__(self, T, V, C, F, classes, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, std=1.0: torch.randn(*s, generator=g, device="cuda") * std  # noqa: E731
        new = lambda *s, dt=torch.bfloat16: torch.full(s, float("nan"), dtype=dt, device="cuda")  # noqa: E731
        self.T, self.V, self.C, self.F, self.classes = T, V, C, F, classes
        self.idx = torch.randint(0, V, (T,), generator=g, device="cuda").int()
        self.labels = torch.randint(0, classes, (T,), generator=g, device="cuda").int()
        self.labels[torch.rand(T, generator=g, device="cuda") < 0.3] = -1           # tokens that nothing is asked of
        self.idx[-T // 5:], self.labels[-T // 5:] = -1, -1                          # padding
        self.p = dict(E=rand(V, C), w1=1 + 0.1 * rand(C), W1=rand(C, 2 * F, std=C ** -0.5).bfloat16(), W2=rand(F, C, std=F ** -0.5).bfloat16(), w2=1 + 0.1 * rand(C),
                      Wo=rand(classes, C, std=1.5 * C ** -0.5).bfloat16())
        bf, f32 = vd.DTYPES[torch.bfloat16], vd.DTYPES[torch.float32]
        self.ecfg = vd.EmbedCfg(T, V, C, f32, bf, 0, 1.0)
        self.n1 = vd.NormCfg(1, T, C, bf, vd.NORM_RMS, 0, 0, 0, 1.0, EPS)
        self.acfg = vd.ActCfg(1, T, F, bf, vd.ACT_SILU, 1, 0, 2 * F)
        self.n2 = vd.NormCfg(1, T, C, bf, vd.NORM_RMS, 0, 0, 0, 1.0, EPS)
        self.lcfg = vd.LossCfg(T, classes, C, bf, 1.0)
        self.ws = vd.alloc_ws(max(vd.vardrop_embed_workspace_bytes(self.ecfg), vd.vardrop_norm_workspace_bytes(self.n1), vd.vardrop_loss_workspace_bytes(self.lcfg),
                                  vd.vardrop_grad_clip_workspace_bytes()))
        self.ckpt = vd.alloc_act_ckpt(self.acfg)
        self.x, self.u, self.h2, self.u2, self.d_u2, self.dz, self.dx1, self.dx2 = (new(T, C) for _ in range(8))
        self.st1, self.st2 = new(T, 4, dt=torch.float32), new(T, 4, dt=torch.float32)
        self.y, self.again, self.d_ab = new(1, T, F), new(1, T, F), new(1, T, 2 * F)
        self.loss, self.lse, self.norm = new(T, dt=torch.float32), new(T, dt=torch.float32), new(1, dt=torch.float32)
        self.grads = {n: new(*t.shape, dt=t.dtype) for n, t in self.p.items()}

    def run(self):
        p, T, C, F, g = self.p, self.T, self.C, self.F, self.grads
        vd.vardrop_embed_fwd(p["E"], self.idx, self.ecfg, self.x, self.ws)
        vd.vardrop_norm_fwd(self.x, None, None, None, None, p["w1"], None, None, None, self.n1, None, self.u, self.st1)
        ab = (self.u @ p["W1"]).view(1, T, 2 * F)
        vd.vardrop_act_fwd(ab[..., :F], ab[..., F:], None, self.acfg, self.y, self.ckpt)
        z = self.y[0] @ p["W2"]
        vd.vardrop_norm_fwd(self.x, z, None, None, None, p["w2"], None, None, None, self.n2, self.h2, self.u2, self.st2)
        vd.vardrop_loss_fwd(self.u2, p["Wo"], self.labels, self.lcfg, self.loss, self.lse, self.ws)
        self.d_loss = (self.labels >= 0).float() / (self.labels >= 0).sum()          # the mean's
        vd.vardrop_loss_bwd(self.u2, p["Wo"], self.labels, self.lse, self.d_loss, self.lcfg, self.d_u2, g["Wo"], self.ws)
        vd.vardrop_norm_bwd(self.x, z, None, None, None, p["w2"], None, None, None, self.st2, None, self.d_u2, self.n2, self.dx2, self.dz, None, None, None, g["w2"], None, self.ws)
        vd.vardrop_act_bwd((self.dz @ p["W2"].t()).view(1, T, F), self.ckpt, None, self.acfg, self.d_ab[..., :F], self.d_ab[..., F:], self.again)
        g["W2"].copy_(self.again[0].t() @ self.dz)
        d_ab = self.d_ab[0]
        g["W1"].copy_(self.u.t() @ d_ab)
        vd.vardrop_norm_bwd(self.x, None, None, None, None, p["w1"], None, None, None, self.st1, None, d_ab @ p["W1"].t(), self.n1, self.dx1, None, None, None, None, g["w1"], None, self.ws)
        vd.vardrop_embed_bwd(self.dx1 + self.dx2, self.idx, self.ecfg, g["E"], self.ws)

    def clip(self):
        vd.vardrop_grad_clip(list(self.grads.values()), vd.ClipCfg(0.5, 1e-6), None, self.norm, self.ws)

    def held(self):
        """What the checkpoint stands for."""
        rows, blocks = self.T, -(-self.F // BLOCK)
        at = -(-2 * rows * self.F // 256) * 256
        codes = self.ckpt[:2 * rows * self.F].view(torch.float8_e4m3fn).view(2, rows, self.F).double()
        return codes * torch.exp2(self.ckpt[at:at + 2 * rows * blocks].view(2, rows, blocks).double() - 127).repeat_interleave(BLOCK, -1)[..., :self.F]

    def exact(self):
        leaf = {n: t.double().clone().requires_grad_(True) for n, t in self.p.items()}
        live = self.idx >= 0
        x = torch.where(live[:, None], leaf["E"][self.idx.long().clamp_min(0)], 0.0)
        a, b = (rms(x, leaf["w1"]) @ leaf["W1"]).split(self.F, 1)
        u2 = rms(x + HeldAct.apply(a, b, *self.held()) @ leaf["W2"], leaf["w2"])
        asked = self.labels >= 0
        loss = torch.nn.functional.cross_entropy(u2[asked] @ leaf["Wo"].T, self.labels[asked].long(), reduction="none")
        return loss.detach(), dict(zip(leaf, torch.autograd.grad(loss.mean(), list(leaf.values()))))


def near(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("T,V,C,F,classes", [(700, 90, 64, 96, 333), (300, 2000, 136, 200, 1000)])
def test_a_training_step_of_a_small_model(T, V, C, F, classes):
    s = Step(T, V, C, F, classes, T)
    s.run()
    torch.cuda.synchronize()
    assert vd.ws_status(s.ws) == vd.OK
    loss, grads = s.exact()
    asked = s.labels >= 0
    assert near(s.loss[asked], loss) <= BOUND and not s.loss[~asked].any()
    for n, t in grads.items():
        assert near(s.grads[n], t) <= BOUND, n
    before = {n: t.clone() for n, t in s.grads.items()}
    s.clip()
    total = math.sqrt(sum(float((t.double() ** 2).sum()) for t in before.values()))
    assert abs(float(s.norm.item()) - total) <= 2.0 ** -23 * total
    for n, t in s.grads.items():
        assert near(t, before[n].double() * min(1.0, 0.5 / (total + 1e-6))) <= 2.0 ** -8, n
    # the same step captured, replayed with other tokens
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
        s.clip()
    other = Step(T, V, C, F, classes, T + 1)
    s.idx.copy_(other.idx)
    s.labels.copy_(other.labels)
    graph.replay()
    torch.cuda.synchronize()
    got = {n: t.clone() for n, t in s.grads.items()}, s.loss.clone()
    s.run()
    s.clip()
    torch.cuda.synchronize()
    assert torch.equal(got[1], s.loss) and all(torch.equal(got[0][n], t) for n, t in s.grads.items()) and vd.ws_status(s.ws) == vd.OK


def test_tied_weights():
    """One table at both ends: the loss writes its gradient, the embeddings' is added to it."""
    T, V, C = 500, 300, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    E = (torch.randn(V, C, generator=g, device="cuda") * 0.2).bfloat16()
    idx, labels = (torch.randint(0, V, (T,), generator=g, device="cuda").int() for _ in range(2))
    ecfg, lcfg = vd.EmbedCfg(T, V, C, 0, 0, 1, 8.0), vd.LossCfg(T, V, C, 0, 1.0)
    ws = vd.alloc_ws(max(vd.vardrop_embed_workspace_bytes(ecfg), vd.vardrop_loss_workspace_bytes(lcfg)))
    x, d_x, d_E = torch.empty((T, C), dtype=torch.bfloat16, device="cuda"), torch.empty((T, C), dtype=torch.bfloat16, device="cuda"), torch.empty_like(E)
    loss, lse, d_loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.full((T,), 1.0 / T, device="cuda")
    vd.vardrop_embed_fwd(E, idx, ecfg, x, ws)
    vd.vardrop_loss_fwd(x, E, labels, lcfg, loss, lse, ws)
    vd.vardrop_loss_bwd(x, E, labels, lse, d_loss, lcfg, d_x, d_E, ws)
    vd.vardrop_embed_bwd(d_x, idx, ecfg, d_E, ws)
    assert vd.ws_status(ws) == vd.OK
    leaf = E.double().requires_grad_(True)
    want, = torch.autograd.grad(torch.nn.functional.cross_entropy(8.0 * leaf[idx.long()] @ leaf.T, labels.long()), leaf)
    assert near(d_E, want) <= 5 * 2.0 ** -8         # x, G, d_x, the loss's part and the sum are rounded
