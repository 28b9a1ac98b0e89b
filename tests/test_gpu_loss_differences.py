"""Gradients of vardrop_loss_bwd against differences of vardrop_loss_fwd, each with the bound of its own token or class, at entries that stand out far enough for a gradient of zeros or of the other sign to
fail."""
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

U = 2.0 ** -24          # half a step of fp32
STEP = 2.0 ** -4        # what an entry is moved by; entries are multiples of it, so either side is exact
THIRD = 0.0963          # 1 / (6 sqrt 3): the largest third central moment of a variable in an interval of one, and of p (1 - p) (1 - 2 p)


class Setting:
    def __init__(self, T, V, C, dtype, scale, seed, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        grid = lambda *s: (torch.randn(*s, generator=g, device=device) / STEP).round().clamp(-60, 60).mul(STEP).to(dtype)  # noqa: E731
        self.h, self.w, self.scale, self.dtype = grid(T, C), grid(V, C), scale, dtype
        self.labels = torch.randint(0, V, (T,), generator=g, device=device).int()
        self.labels[::5] = -1
        self.d_loss = (0.5 + torch.rand(T, generator=g, device=device)) / T
        self.live = self.labels >= 0

    def run(self):
        """The library's loss and gradients."""
        cfg = vd.LossCfg(*self.h.shape[:1], *self.w.shape, vd.DTYPES[self.dtype], self.scale)
        ws = vd.alloc_ws(vd.vardrop_loss_workspace_bytes(cfg))
        loss, lse = (torch.empty(self.h.shape[0], device="cuda") for _ in range(2))
        d_h, d_w = torch.empty_like(self.h), torch.empty_like(self.w)
        vd.vardrop_loss_fwd(self.h, self.w, self.labels, cfg, loss, lse, ws)
        vd.vardrop_loss_bwd(self.h, self.w, self.labels, lse, self.d_loss, cfg, d_h, d_w, ws)
        assert vd.ws_status(ws) == vd.OK
        return loss.double(), d_h.double(), d_w.double()

    def bounds(self):
        """What a difference and a gradient may be apart by: [T, C] of h and [V, C] of w."""
        (T, C), V, s = self.h.shape, self.w.shape[0], self.scale
        h, w, g = self.h.double(), self.w.double(), (self.d_loss.double() * self.live)[:, None]
        logits = s * (h @ w.T)
        p = torch.softmax(logits, 1)
        G = p.clone()
        G[torch.arange(T, device=h.device), self.labels.long().clamp_min(0)] -= 1
        G *= g * s
        # loss: sums of products in fp32, two roundings of the running sum for each 16; sums of exponentials; a few steps of lse and of the label's logit.  (An entry that has moved: one step more of each factor.)
        size = s * ((h.abs() + STEP) @ (w.abs() + STEP).T).amax(1, keepdim=True)
        err = size * (C / 4 + 16) * U + (V / 128 + 64) * U + 2.0 ** -20 + 8 * U * size
        # G and the gradient rounded to 16 bits, fp16's least step of G
        half = torch.finfo(self.dtype).eps / 2
        spread = w.amax(0) - w.amin(0)
        off = G.abs() * (half + 8 * U) + p * g * s * (3 * err + 2.0 ** -20) + 2.0 ** -38 * s * g.amax()
        off *= self.live[:, None]
        of_h = (STEP * STEP / 6) * THIRD * g * (s * spread) ** 3 + g * err / STEP + off @ w.abs() + half * (G @ w).abs()
        of_w = (STEP * STEP / 6) * THIRD * s ** 3 * (g * h.abs() ** 3).sum(0) + (g * err).sum() / STEP + off.T @ h.abs() + half * (G.T @ h).abs()
        return of_h, of_w

    def entries(self, grad, bound, count):
        """The entries that stand out most, no two of a row."""
        ratio, col = (grad.abs() / bound.clamp_min(1e-300)).max(1)
        rows = ratio.topk(count).indices
        return [(int(r), int(col[r])) for r in rows]


def compare(setting, run, count=6):
    """None, or what is wrong."""
    loss, d_h, d_w = run()
    f = lambda: float((setting.d_loss.double() * run()[0]).sum())  # noqa: E731
    for tensor, grad, bound in zip((setting.h, setting.w), (d_h, d_w), setting.bounds()):
        for at in setting.entries(grad, bound, count):
            old = tensor[at].item()
            tensor[at] = old + STEP
            up = f()
            tensor[at] = old - STEP
            down = f()
            tensor[at] = old
            slope = (up - down) / (2 * STEP)
            if abs(slope) <= 3 * float(bound[at]):
                return f"{at}: a difference of {slope} does not stand out from its bound {float(bound[at])}"
            if abs(grad[at].item() - slope) > float(bound[at]):
                return f"{at}: gradient {grad[at].item()}, difference {slope}, bound {float(bound[at])}"
    return None


SETTINGS = [(20, 90, 16, torch.bfloat16, 1.0), (40, 30, 24, torch.float16, 0.5), (300, 17, 64, torch.bfloat16, 0.25), (9, 300, 8, torch.float16, 1.0)]


@pytest.mark.parametrize("T,V,C,dtype,scale", SETTINGS)
def test_against_differences(T, V, C, dtype, scale):
    setting = Setting(T, V, C, dtype, scale, T)
    assert compare(setting, setting.run) is None
