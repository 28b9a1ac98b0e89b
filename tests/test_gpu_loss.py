"""vardrop_loss_fwd / vardrop_loss_bwd against the formulas in 64 bits."""
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
U = 2.0 ** -24          # half a step of fp32


class Case:
    def __init__(self, T, V, C, dtype=BF, gaps=0.0, scale=1.0, std=1.0, seed=0, shift=0.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.T, self.V, self.C, self.dtype, self.scale = T, V, C, dtype, scale
        self.h, self.w = (rand(T, C) * std + shift).to(dtype), (rand(V, C) * (1.5 / C ** 0.5) + shift).to(dtype)
        self.labels = (torch.rand(T, generator=g, device="cuda") ** 3 * V).int().clamp(0, V - 1)
        self.labels[torch.rand(T, generator=g, device="cuda") < gaps] = -1
        self.d_loss = (0.5 + torch.rand(T, generator=g, device="cuda")) * (1 - 2 * (torch.rand(T, generator=g, device="cuda") < 0.2).float()) / T
        self.cfg = vd.LossCfg(T, V, C, vd.DTYPES[dtype], scale)
        self.ws = vd.alloc_ws(vd.vardrop_loss_workspace_bytes(self.cfg))
        self.ws[256:] = 0xFF                    # NaN, wherever it is read before it is written

    def run(self, d_h=True, d_w=True):
        bad = self.labels < 0                   # what lies there does not matter
        h, d_loss = self.h.clone(), self.d_loss.clone()
        h[bad], d_loss[bad] = float("nan"), float("nan")
        loss, lse = (torch.full((self.T,), 7.0, device="cuda") for _ in range(2))
        vd.vardrop_loss_fwd(h, self.w, self.labels, self.cfg, loss, lse, self.ws)
        self.lse = lse
        seen = torch.where(bad, float("nan"), lse)
        d_h = torch.full_like(self.h, 7.0) if d_h else None
        d_w = torch.full_like(self.w, 7.0) if d_w else None
        vd.vardrop_loss_bwd(h, self.w, self.labels, seen, d_loss, self.cfg, d_h, d_w, self.ws)
        self.far = bool((lse.abs() > 65536).any())          # gradients that lse does not determine are reported
        assert vd.ws_status(self.ws) == (vd.ERR_UNSUPPORTED if self.far else vd.OK)
        return loss, lse, d_h, d_w

    def check(self):
        loss, lse, d_h, d_w = self.run()
        T, V, C = self.T, self.V, self.C
        live, scale = self.labels >= 0, self.scale or 1.0
        assert not loss[~live].any() and not lse[~live].any() and not d_h[~live].any()
        half = torch.finfo(self.dtype).eps / 2
        tiny = torch.finfo(self.dtype).smallest_normal * half
        w = self.w.double()
        want_w, size_w = (torch.zeros((V, C), dtype=torch.float64, device="cuda") for _ in range(2))
        sum_h = torch.zeros(C, dtype=torch.float64, device="cuda")
        most = float(self.d_loss[live].abs().max()) * scale if bool(live.any()) else 0.0
        for rows in torch.split(torch.nonzero(live)[:, 0], 2048):
            h, label, g = self.h[rows].double(), self.labels[rows].long()[:, None], self.d_loss[rows].double()[:, None]
            logits = scale * (h @ w.T)
            # fp32 sums of exact products, at most two roundings of the running sum for each 16 of them
            off = scale * (h.abs() @ w.abs().T).amax(1, keepdim=True) * (C / 8 + 8) * U
            exact = torch.logsumexp(logits, 1, keepdim=True)
            # sums of exponentials: 8 values in a chain of a thread, chunks of 32, then half tiles; an exponential is good to 2^-21
            err = off + (V / 128 + 64) * U + 2.0 ** -21 + 4 * U * exact.abs()
            target = logits.gather(1, label)
            assert bool(((lse[rows].double()[:, None] - exact).abs() <= err).all())
            assert bool(((loss[rows].double()[:, None] - (exact - target)).abs() <= err + off + 4 * U * target.abs()).all())
            if self.far:
                continue
            p = torch.exp(logits - exact)
            G = p.clone()
            G.scatter_add_(1, label, torch.full_like(target, -1.0))
            G *= g * scale
            # p is off by what the logits and lse are, G by half a step of its 16 bits or of the least that fp16 holds
            size = G.abs() * (half + 4 * U) + (p * g.abs() * scale) * (2 * err + off + 2.0 ** -20)
            want, bound = G @ w, size @ w.abs() + (G.abs() @ w.abs()) * (V / 8 + 40) * U + most * 2.0 ** -37 * w.abs().sum(0)
            assert bool(((d_h[rows].double() - want).abs() <= bound + (want.abs() + bound) * half + tiny).all())
            want_w += G.T @ h
            size_w += size.T @ h.abs() + (G.abs().T @ h.abs()) * (T / 8 + 40) * U
            sum_h += h.abs().sum(0)
        if self.far:
            return
        bound = size_w + most * 2.0 ** -37 * sum_h
        assert bool(((d_w.double() - want_w).abs() <= bound + (want_w.abs() + bound) * half + tiny).all())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T", [1, 2, 64, 65, 255, 256, 257, 700])
@pytest.mark.parametrize("V", [1, 2, 127, 129, 256, 257, 1000, 4099])
def test_tokens_and_classes(T, V, dtype):
    Case(T, V, 64, dtype, seed=T + V).check()
    Case(T, V, 72, dtype, gaps=0.5, seed=T + V, scale=0.5).check()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("C", [8, 16, 56, 128, 248, 264, 512, 1032, 4096])
def test_channels(C, dtype):
    Case(300, 520, C, dtype, gaps=0.3, seed=C).check()
    Case(33, 3000, C, dtype, seed=C).check()


def test_no_labels_at_all_and_a_single_one():
    for T in (1, 63, 300, 1100):
        case = Case(T, 300, 64, gaps=1.1)
        case.check()
        assert not case.run()[3].any()
        case.labels[T // 2] = 299
        case.check()


def test_labels_everywhere_in_the_vocabulary():
    case = Case(1500, 1500, 40)
    case.labels.copy_(torch.randperm(1500, device="cuda").int())
    case.check()
    case.labels.fill_(1499)
    case.check()


@pytest.mark.parametrize("T,V,C", [(16384, 20001, 64), (40000, 7000, 32), (9000, 30000, 264), (5000, 300, 64), (100, 50000, 64), (20000, 128, 512)])
def test_pieces_and_splits(T, V, C):
    """More classes than a piece of G has, few tiles with a long axis to split."""
    Case(T, V, C, seed=1, gaps=0.1).check()
    Case(T, V, C, HF, seed=2).check()


def test_more_tokens_than_any_row_of_tiles_and_the_widest_channels():
    Case(300000, 40, 8, gaps=0.9, seed=1).check()
    Case(3, 5, 65536, seed=2).check()
    for V, T in ((1000, 1000), (1100, 900), (900, 1100), (1030, 1030)):          # around where the gradients' products are split
        Case(T, V, 64, gaps=0.1, seed=3).check()


@pytest.mark.parametrize("scale,std", [(1.0, 30.0), (100.0, 3.0), (1e-6, 1.0), (1e4, 1.0), (0.0, 1.0)])
def test_logits_near_and_far(scale, std):
    Case(200, 700, 64, scale=scale, std=std, gaps=0.2).check()


def test_logits_far_from_zero():
    """All logits of a row near a value of thousands: sums of exponentials go by their differences."""
    Case(200, 700, 64, shift=6.0).check()


def test_gradients_of_different_magnitudes():
    for dtype in (BF, HF):
        for size in (1e-12, 1.0, 65536.0 * 512):
            case = Case(150, 300, 64, dtype)
            case.d_loss *= size * 150
            if dtype == HF and size != 1.0:
                continue                        # gradients that fp16 does not hold
            case.check()
        case = Case(150, 300, 64, dtype)
        case.d_loss[::2] = 0.0
        case.check()
        case.d_loss.zero_()
        assert not case.run()[2].any() and not case.run()[3].any()


def test_against_differences():
    case = Case(20, 90, 16, seed=3)
    *_, d_h, d_w = case.run()
    f = lambda: float((case.d_loss.double() * Case.run(case, d_w=False)[0].double()).sum())  # noqa: E731
    for tensor, grad in ((case.h, d_h), (case.w, d_w)):
        for at in ((3, 5), (11, 0), (19, 15)):
            old = tensor[at].item()
            hi, lo = torch.tensor(old + 2.0 ** -4).to(BF).item(), torch.tensor(old - 2.0 ** -4).to(BF).item()
            tensor[at] = hi
            up = f()
            tensor[at] = lo
            down = f()
            tensor[at] = old
            # third derivatives of a loss along one logit are below 1/10, a channel's step moves a logit by |w| or |h| of it; the loss is good to 2^-20 of its size
            reach = max(float(case.w.abs().max()), float(case.h.abs().max()))
            bound = (2.0 ** -4) * reach ** 2 * float(case.d_loss.abs().sum()) * 0.25 + 2.0 ** -18 + abs(grad[at].item()) * 2.0 ** -6
            assert abs(grad[at].item() - (up - down) / (hi - lo)) <= bound


def test_the_same_bits_every_time_and_one_gradient_alone():
    case = Case(2000, 3000, 136, gaps=0.3)
    first = case.run()
    case.ws[256:] = 0x7F
    for d_h, d_w in ((True, True), (True, False), (False, True)):
        again = case.run(d_h, d_w)
        assert all(b is None or torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("C", [64, 72])
def test_buffers_on_any_sixteen_bytes(C):
    """Tensors and workspace that begin on 16 bytes, not on 32."""
    case = Case(300, 700, C, gaps=0.2)
    first = case.run()

    def shifted(t):
        flat = torch.zeros(t.numel() + 64, dtype=t.dtype, device="cuda")
        at = 16 // t.element_size() + (-flat.data_ptr() // t.element_size()) % (512 // t.element_size())
        view = flat[at:at + t.numel()].view(t.shape)
        assert view.data_ptr() % 32 == 16
        return view.copy_(t)

    case.h, case.w, case.labels, case.d_loss = (shifted(t) for t in (case.h, case.w, case.labels, case.d_loss))
    case.ws = shifted(torch.zeros(vd.vardrop_loss_workspace_bytes(case.cfg), dtype=torch.uint8, device="cuda"))
    loss, lse, d_h, d_w = (shifted(torch.full_like(t, 7.0)) for t in first)
    vd.vardrop_loss_fwd(case.h, case.w, case.labels, case.cfg, loss, lse, case.ws)
    vd.vardrop_loss_bwd(case.h, case.w, case.labels, lse, case.d_loss, case.cfg, d_h, d_w, case.ws)
    assert vd.ws_status(case.ws) == vd.OK and all(torch.equal(a, b) for a, b in zip(first, (loss, lse, d_h, d_w)))


def test_labels_behind_the_classes_are_none_and_reported():
    case = Case(50, 30, 16)
    want = case.run()
    case.labels[[4, 49]] = torch.tensor([30, 1 << 30], dtype=torch.int32, device="cuda")
    loss, lse = torch.empty(50, device="cuda"), torch.empty(50, device="cuda")
    vd.vardrop_loss_fwd(case.h, case.w, case.labels, case.cfg, loss, lse, case.ws)
    assert vd.ws_status(case.ws) == vd.ERR_INVALID_ARG and not loss[[4, 49]].any()
    keep = [i for i in range(50) if i not in (4, 49)]
    assert torch.equal(loss[keep], want[0][keep])


def test_lse_that_does_not_determine_the_weights_is_reported():
    case = Case(50, 30, 16)
    loss, lse, d_h, d_w = case.run()
    lse[7] = 70000.0
    vd.vardrop_loss_bwd(case.h, case.w, case.labels, lse, case.d_loss, case.cfg, d_h, d_w, case.ws)
    assert vd.ws_status(case.ws) == vd.ERR_UNSUPPORTED


def test_a_row_that_is_not_finite():
    case = Case(300, 500, 64)
    want = case.run()
    case.h[17, 3] = float("inf")
    case.h[200, 9] = float("nan")
    loss, lse, d_h, d_w = case.run()
    fine = [i for i in range(300) if i not in (17, 200)]
    assert bool(loss[[17, 200]].isnan().all()) and torch.equal(loss[fine], want[0][fine]) and torch.equal(d_h[fine], want[2][fine]) and bool(d_h[[17, 200]].isnan().any(1).all())


def test_captured_and_replayed_with_other_labels():
    case = Case(700, 900, 64)
    loss, lse, d_h, d_w = case.run()

    def call():
        vd.vardrop_loss_fwd(case.h, case.w, case.labels, case.cfg, loss, lse, case.ws)
        vd.vardrop_loss_bwd(case.h, case.w, case.labels, lse, case.d_loss, case.cfg, d_h, d_w, case.ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for gaps in (0.6, 0.0, 1.1):
        other = Case(700, 900, 64, gaps=gaps, seed=9)
        for name in ("h", "w", "labels", "d_loss"):
            getattr(case, name).copy_(getattr(other, name))
        for t in (loss, lse, d_h, d_w):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (loss, lse, d_h, d_w)]
        want = other.run()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and vd.ws_status(case.ws) == vd.OK


def test_on_two_streams_at_once():
    cases = [Case(900, 1200, 64, seed=s, gaps=0.2 * s) for s in range(2)]
    want = [c.run() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            got.append(c.run())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))


def test_binding_refuses_other_tensors():
    case = Case(8, 20, 16)
    loss, lse = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    for bad in ((case.h.float(), case.w, case.labels, loss), (case.h, case.w.half(), case.labels, loss), (case.h, case.w, case.labels.long(), loss), (case.h[:7], case.w, case.labels, loss),
                (case.h, case.w.t(), case.labels, loss), (case.h, case.w, case.labels, loss.double()), (case.h.cpu(), case.w, case.labels, loss)):
        with pytest.raises(ValueError):
            vd.vardrop_loss_fwd(*bad[:3], case.cfg, bad[3], lse, case.ws)
