"""vardrop_loss_fwd / vardrop_loss_bwd with classes that are switched off: logits of -inf for groups of classes of any place and length, against the formulas in 64 bits over the other classes."""
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
U = 2.0 ** -24          # half a step of fp32


class Masked:
    """A channel of h is one; `off` holds a weight there that takes the logits of the classes in `off` to -inf, the others have zero.  mask: -inf itself, or the type's lowest value in `times` channels."""

    def __init__(self, T, V, C, off, dtype=BF, mask=float("-inf"), times=1, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T, self.V, self.C, self.dtype, self.times = T, V, C, dtype, times
        self.off = torch.zeros(V, dtype=torch.bool, device="cuda")
        for a, b in off:
            self.off[a:b] = True
        on = torch.nonzero(~self.off)[:, 0]
        self.h, self.w = (torch.randn(*s, generator=g, device="cuda").to(dtype) for s in ((T, C), (V, C)))
        self.w *= 1.5 / C ** 0.5
        self.h[:, :times] = 1.0
        self.w[:, :times] = 0.0
        self.w[self.off, :times] = mask
        self.labels = on[torch.randint(0, len(on), (T,), generator=g, device="cuda")].int()
        self.d_loss = (0.5 + torch.rand(T, generator=g, device="cuda")) / T
        self.cfg = vd.LossCfg(T, V, C, vd.DTYPES[dtype], 1.0)
        self.ws = vd.alloc_ws(vd.vardrop_loss_workspace_bytes(self.cfg))
        self.ws[256:] = 0xFF

    def check(self):
        T, V, C, skip = self.T, self.V, self.C, self.times
        loss, lse = (torch.full((T,), 7.0, device="cuda") for _ in range(2))
        d_h, d_w = torch.full_like(self.h, 7.0), torch.full_like(self.w, 7.0)
        vd.vardrop_loss_fwd(self.h, self.w, self.labels, self.cfg, loss, lse, self.ws)
        vd.vardrop_loss_bwd(self.h, self.w, self.labels, lse, self.d_loss, self.cfg, d_h, d_w, self.ws)
        assert vd.ws_status(self.ws) == vd.OK
        on = ~self.off
        h, w, label, g = self.h.double(), self.w.double()[on], (on.cumsum(0) - 1)[self.labels.long()][:, None], self.d_loss.double()[:, None]
        logits = h @ w.T
        exact = torch.logsumexp(logits, 1, keepdim=True)
        target = logits.gather(1, label)
        # fp32 sums of exact products, at most two roundings of the running sum for each 16; sums of exponentials, each good to 2^-21
        off = (h.abs() @ w.abs().T).amax(1, keepdim=True) * (C / 8 + 8) * U
        err = off + (V / 128 + 64) * U + 2.0 ** -21 + 4 * U * exact.abs()
        assert bool(((lse.double()[:, None] - exact).abs() <= err).all())
        assert bool(((loss.double()[:, None] - (exact - target)).abs() <= err + off + 4 * U * target.abs()).all())
        # G is off by what the logits and lse are, by half a step of its 16 bits or of the least that fp16 holds
        half = torch.finfo(self.dtype).eps / 2
        tiny = torch.finfo(self.dtype).smallest_normal * half
        p = torch.exp(logits - exact)
        G = p.scatter_add(1, label, torch.full_like(target, -1.0)) * g
        size = G.abs() * (half + 4 * U) + p * g * (2 * err + off + 2.0 ** -20)
        most = float(self.d_loss.max())
        want, bound = G @ w, size @ w.abs() + (G.abs() @ w.abs()) * (V / 8 + 40) * U + most * 2.0 ** -38 * w.abs().sum(0)
        near = lambda got, want, bound: (got.double() - want).abs() <= bound + (want.abs() + bound) * half + tiny  # noqa: E731
        # (the channels of the mask: zero times -inf, by the formula)
        assert bool(near(d_h, want, bound)[:, skip:].all())
        want, bound = G.T @ h, size.T @ h.abs() + (G.abs().T @ h.abs()) * (T / 8 + 40) * U + most * 2.0 ** -38 * h.abs().sum(0)
        assert bool(near(d_w[on], want, bound).all()) and not d_w[self.off].any()
        return d_h[:, :skip]


GROUPS = [[(0, 32)], [(0, 128)], [(0, 256)], [(0, 600)], [(32, 64)], [(128, 160)], [(128, 256), (512, 640)], [(640, 660)], [(256, 660)], [(0, 33)], [(1, 660)], [(0, 659)], [(0, 31), (128, 159), (256, 300)]]


@pytest.mark.parametrize("off", GROUPS)
@pytest.mark.parametrize("T", [5, 300])
def test_groups_of_classes(off, T):
    Masked(T, 660, 64, off, seed=T).check()
    Masked(T, 660, 72, off, HF, seed=T + 1).check()


@pytest.mark.parametrize("V", [129, 160, 257, 384, 1000, 50304])
def test_a_vocabulary_padded_at_its_end(V):
    for pad in (1, 32, 100, 128):
        if pad < V:
            Masked(70, V, 64, [(V - pad, V)], seed=V).check()


def test_the_lowest_value_of_the_type():
    """One channel of it is finite, the sum of two is beyond fp32: the gradient is finite either way."""
    for times in (1, 2):
        for off in ([(0, 128)], [(0, 32), (200, 300)], [(512, 660)]):
            assert bool(Masked(300, 660, 64, off, mask=torch.finfo(BF).min, times=times).check().isfinite().all())


def test_no_class_left():
    """The sum of no exponentials: lse is -inf, the loss of any label is not a number."""
    for T, V in ((40, 300), (300, 40), (300, 129)):
        case = Masked(T, V, 64, [(0, 32)])
        case.w[:, 0] = float("-inf")
        loss, lse = (torch.full((T,), 7.0, device="cuda") for _ in range(2))
        vd.vardrop_loss_fwd(case.h, case.w, case.labels, case.cfg, loss, lse, case.ws)
        assert bool((lse == float("-inf")).all()) and bool(loss.isnan().all())
