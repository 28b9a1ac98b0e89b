"""vardrop_norm_fwd / vardrop_norm_bwd against the formulas in 64 bits, and the backward against differences of the forward's formula."""
import numpy as np
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

EPS = 1e-5
U = 2.0 ** -24          # half a step of fp32
# A sum over C <= 8192 elements takes at most 8 roundings in a thread, 5 in a warp and 32 over warps; with the mean, the square root and a few products around it
# an element has seen fewer than 64.
DEPTH = 64


def normed(t, kind, w, b):
    if kind == 0:
        return t, t, torch.ones_like(t[:, :1])
    c = t - t.mean(1, keepdim=True) if kind == 2 else t
    r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    return c * r * w + b, c * r, r


def normed_back(d, z, r, kind, w):
    """Gradient of t, and the sum of the magnitudes that it is made of."""
    if kind == 0:
        return d, d.abs()
    e = d * w
    m0, m1 = (e * z).mean(1, keepdim=True), e.mean(1, keepdim=True) if kind == 2 else 0.0
    size = r * (e.abs() + z.abs() * (e * z).abs().mean(1, keepdim=True) + (e.abs().mean(1, keepdim=True) if kind == 2 else 0.0))
    return r * (e - z * m0 - m1), size


class Case:
    def __init__(self, B, N, C, dtype, pre, post, gate_rows, kept=None, scale=1.0, offset=0.0, seed=0, with_y=True, std=1.0):
        g = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
        self.B, self.N, self.C, self.dtype, self.pre, self.post, self.gate_rows, self.scale = B, N, C, dtype, pre, post, gate_rows, scale
        dev = lambda t, ty=dtype: t.to(ty).cuda()  # noqa: E731
        self.x, self.y = dev(std * rand(B, N, C) + offset), dev(0.5 * rand(B, N, C)) if with_y else None
        self.d_h, self.d_u = dev(rand(B, N, C)), dev(rand(B, N, C)) if pre else None
        f = lambda t, on: t.float().cuda() if on else None  # noqa: E731
        self.gate = f(rand(max(1, gate_rows), C), gate_rows)
        self.w_post, self.b_post = f(1 + 0.2 * rand(C), post), f(0.2 * rand(C), post == 2)
        self.w_pre, self.b_pre = f(1 + 0.2 * rand(C), pre), f(0.2 * rand(C), pre == 2)
        self.sel = self.n_sel = self.inv = None
        self.kept = [N] * B
        if kept is not None:
            S = len(kept)
            self.kept = [kept[b if S > 1 else 0] for b in range(B)]
            sel, inv = np.full((S, N), -1, np.int32), np.full((S, N), -1, np.int32)
            rng = np.random.default_rng(seed)
            for s, m in enumerate(kept):
                sel[s, :m] = np.sort(rng.choice(N, m, replace=False))
                inv[s, sel[s, :m]] = np.arange(m)
            self.sel, self.inv, self.n_sel = (torch.from_numpy(a).cuda() for a in (sel, inv, np.array(kept, np.int32)))
        self.cfg = vd.NormCfg(B, N, C, vd.DTYPES[dtype], pre, post, gate_rows, 0 if kept is None else len(kept), scale, EPS)

    def run(self, want=("gate", "w_post", "b_post", "w_pre", "b_pre"), fill=7.0):
        new = lambda: torch.full((self.B, self.N, self.C), fill, dtype=self.dtype, device="cuda")  # noqa: E731
        out = {"h": new(), "u": new() if self.pre else None, "stats": torch.full((self.B, self.N, 4), fill, device="cuda")}
        vd.vardrop_norm_fwd(self.x, self.y, self.gate, self.w_post, self.b_post, self.w_pre, self.b_pre, self.sel, self.n_sel, self.cfg, out["h"], out["u"], out["stats"])
        out["dx"], out["dy"] = new(), new() if self.y is not None else None
        grads = {n: torch.full_like(getattr(self, n), fill) if getattr(self, n) is not None and n in want else None for n in ("gate", "w_post", "b_post", "w_pre", "b_pre")}
        ws = vd.alloc_ws(vd.vardrop_norm_workspace_bytes(self.cfg))
        ws[256:] = 0xFF
        vd.vardrop_norm_bwd(self.x, self.y, self.gate, self.w_post, self.b_post, self.w_pre, self.sel, self.n_sel, self.inv, out["stats"], self.d_h, self.d_u, self.cfg,
                            out["dx"], out["dy"], *grads.values(), ws)
        torch.cuda.synchronize()
        return {**out, **{"d_" + n: t for n, t in grads.items()}}

    def check(self, **kw):
        got = self.run(**kw)
        C, half = self.C, torch.finfo(self.dtype).eps / 2
        d = lambda t: t.double().cpu()  # noqa: E731
        par = {n: d(getattr(self, n)) if getattr(self, n) is not None else None for n in ("gate", "w_post", "b_post", "w_pre", "b_pre")}
        w_post, w_pre = (torch.ones(C, dtype=torch.float64) if par[n] is None else par[n] for n in ("w_post", "w_pre"))
        b_post, b_pre = (torch.zeros(C, dtype=torch.float64) if par[n] is None else par[n] for n in ("b_post", "b_pre"))
        want = {n: torch.zeros(self.gate_rows if n == "gate" else 1, C, dtype=torch.float64) for n in par}
        size = {n: torch.zeros_like(t) for n, t in want.items()}

        # Below the type's least normal value its step no longer shrinks: half of it is half of smallest_normal eps (2^-25 for fp16), whatever the value.
        least = torch.finfo(self.dtype).smallest_normal * torch.finfo(self.dtype).eps / 2

        def near(name, b, rows, value, bound):
            a = d(got[name])[b, rows]
            if not value.numel():
                return
            assert bool(torch.isfinite(a).all()), name
            worst = ((a - value).abs() - half * value.abs() - bound).max() - least
            assert worst <= 0, (name, b, float((a - value).abs().max()), float(worst))

        for b in range(self.B):
            m, s = self.kept[b], 0 if self.sel is None or self.sel.shape[0] == 1 else b
            rows = self.sel[s, :m].long().cpu() if self.sel is not None else torch.arange(m)
            rest = [r for r in range(self.N) if r not in set(rows.tolist())]
            x, y = d(self.x)[b, rows], d(self.y)[b, :m] if self.y is not None else torch.zeros(m, C, dtype=torch.float64)
            g = par["gate"][b if self.gate_rows > 1 else 0] if self.gate_rows else torch.ones(C, dtype=torch.float64)
            yn, zy, ry = normed(y, self.post, w_post, b_post)
            h = self.scale * x + g * yn
            u, zh, rh = normed(h, self.pre, w_pre, b_pre)
            top = lambda t: t.abs().amax(1, keepdim=True) if m else t[:, :1]  # noqa: E731
            # an element of N(t) carries the rounding of the t around it, scaled as it is
            off_yn = DEPTH * U * (w_post.abs() * (zy.abs() + ry * top(y)) + b_post.abs()) if self.post else U * yn.abs()
            off_h = g.abs() * off_yn + 4 * U * ((self.scale * x).abs() + (g * yn).abs())
            off_zh = rh * (off_h + top(off_h) + DEPTH * U * (h.abs() + top(h)))
            near("h", b, slice(0, m), h, off_h)
            if self.pre:
                near("u", b, slice(0, m), u, w_pre.abs() * (off_zh + zh.abs() * top(off_zh)) + DEPTH * U * (zh * w_pre).abs() + 4 * U * b_pre.abs())
            dh, du = d(self.d_h)[b, :m], d(self.d_u)[b, :m] if self.pre else torch.zeros_like(h)
            back, mag = normed_back(du, zh, rh, self.pre, w_pre) if self.pre else (torch.zeros_like(h), torch.zeros_like(h))
            t = dh + back
            # the gradient is linear in z with factors of the size of its terms
            off_t = DEPTH * U * (dh.abs() + mag) + mag * 4 * top(off_zh)
            near("dx", b, rows, self.scale * t, abs(self.scale) * off_t)
            if rest:
                assert not got["dx"][b, rest].any(), "rows of dropped tokens"
            if self.y is not None:
                off_zy = DEPTH * U * (zy.abs() + ry * top(y)) if self.post else 0 * zy
                dy, mag_y = normed_back(g * t, zy, ry, self.post, w_post)
                off_dy = DEPTH * U * mag_y + (ry * ((g * w_post).abs() * off_t + top((g * w_post).abs() * off_t) * (1 + zy.abs())) + mag_y * 4 * top(off_zy) if self.post else g.abs() * off_t)
                near("dy", b, slice(0, m), dy, off_dy)
                assert bool((got["dy"][b, m:] == kw.get("fill", 7.0)).all())
                terms = {"gate": (t * yn, off_t * yn.abs() + t.abs() * off_yn), "w_post": (g * t * zy, g.abs() * (off_t * zy.abs() + t.abs() * off_zy)), "b_post": (g * t, g.abs() * off_t)}
            else:
                terms = {}
            terms |= {"w_pre": (du * zh, du.abs() * off_zh), "b_pre": (du, 0 * du)}
            for n, (v, off) in terms.items():
                at = b if n == "gate" and self.gate_rows > 1 else 0
                if want[n].shape[0] > at:
                    want[n][at] += v.sum(0)
                    # fewer than 64 roundings a term behind the ones of a thread's own rows, of which there are fewer than B N
                    size[n][at] += (off + (DEPTH + min(self.B * self.N, 256)) * U * v.abs()).sum(0)
            for n in ("h", "u"):
                if got[n] is not None:
                    assert bool((got[n][b, m:] == kw.get("fill", 7.0)).all()), "rows behind the kept ones"
        for n in want:
            if got["d_" + n] is not None:
                a = d(got["d_" + n]).view(want[n].shape)
                # d_gate and d_w_post come as products of sums: w A + b T, with their cancellation
                slack = size[n] * (4 if n != "gate" or par["b_post"] is None else 64) + 1e-30
                assert bool(((a - want[n]).abs() <= slack).all()), (n, float(((a - want[n]).abs() / slack).max()))
        return got


TYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pre,post,gate_rows", [(1, 0, 0), (2, 0, 0), (0, 1, 1), (1, 1, 1), (2, 2, 1), (2, 1, 3), (1, 2, 3), (0, 0, 3), (0, 0, 0), (0, 2, 3)])
def test_kinds_and_gates(dtype, pre, post, gate_rows):
    Case(3, 37, 136, dtype, pre, post, gate_rows, scale=0.75, seed=1).check()


@pytest.mark.parametrize("C", [1, 2, 7, 8, 31, 96, 256, 257, 264, 512, 515, 1000, 1024, 1031, 2048, 2056, 4095, 4096, 5000, 8191, 8192])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_widths(C, dtype):
    Case(2, 5, C, dtype, 1 if C < 4 else 2, 1, 2, seed=C).check()


@pytest.mark.parametrize("B,N", [(1, 1), (1, 700), (700, 1), (5, 65), (64, 9)])
@pytest.mark.parametrize("gate_rows", [0, 1, -1])
def test_shapes(B, N, gate_rows):
    Case(B, N, 72, torch.float32, 2, 2, B if gate_rows < 0 else gate_rows, seed=B).check()


@pytest.mark.parametrize("kept", [[1], [0], [41], [17], [3, 0, 41, 20], [1, 1, 1, 1]])
@pytest.mark.parametrize("dtype,C", [(torch.bfloat16, 512), (torch.float32, 77)])
@pytest.mark.parametrize("gate_rows", [1, 4])
def test_selections(kept, dtype, C, gate_rows):
    Case(4, 41, C, dtype, 2, 1, gate_rows, kept=kept, seed=3).check()


def test_without_a_block():
    got = Case(2, 9, 512, torch.bfloat16, 2, 0, 0, with_y=False, seed=4).check()
    assert got["dy"] is None


def test_tokens_far_from_zero_and_tiny_ones():
    Case(2, 9, 512, torch.float32, 2, 2, 1, offset=300.0, seed=5).check()
    Case(2, 9, 512, torch.float32, 2, 1, 1, std=1e-6, seed=6).check()      # eps decides


def test_a_constant_row_has_no_gradient():
    """Layer norm of a row of one value: z = 0, and what comes back is r (e - mean(e))."""
    c = Case(1, 4, 64, torch.float32, 2, 0, 0, with_y=False, seed=7)
    c.x[:] = 3.0
    got = c.check()
    assert bool((got["u"] == c.b_pre).all())


def test_only_some_parameters_gradients_and_no_stream_gradient():
    c = Case(2, 33, 96, torch.bfloat16, 2, 2, 2, seed=8)
    all_of = c.check()
    some = c.run(want=("w_post", "b_pre"))
    for n in ("d_w_post", "d_b_pre", "dx", "dy"):
        assert torch.equal(some[n], all_of[n])
    none = c.run(want=())
    assert torch.equal(none["dx"], all_of["dx"])
    zero = torch.zeros_like(c.d_h)
    c.d_h = zero
    with_zeros = c.run()
    c.d_h = None
    without = c.run()
    for n, t in with_zeros.items():
        assert torch.equal(t, without[n]), n


def test_in_place_and_runs_repeat_bit_for_bit():
    c = Case(3, 70, 512, torch.bfloat16, 1, 2, 3, seed=9)
    a, b = c.run(), c.run()
    for n, t in a.items():
        assert t is None or torch.equal(t, b[n]), n
    x, y, d_h, d_u = c.x.clone(), c.y.clone(), c.d_h.clone(), c.d_u.clone()
    stats = torch.empty_like(a["stats"])
    vd.vardrop_norm_fwd(x, y, c.gate, c.w_post, c.b_post, c.w_pre, c.b_pre, None, None, c.cfg, x, y, stats)
    assert torch.equal(x, a["h"]) and torch.equal(y, a["u"]) and torch.equal(stats, a["stats"])
    ws = vd.alloc_ws(vd.vardrop_norm_workspace_bytes(c.cfg))
    vd.vardrop_norm_bwd(c.x, c.y, c.gate, c.w_post, c.b_post, c.w_pre, None, None, None, stats, d_h, d_u, c.cfg, d_h, d_u, None, None, None, None, None, ws)
    assert torch.equal(d_h, a["dx"]) and torch.equal(d_u, a["dy"])


def test_rows_that_are_not_finite_stay_alone():
    c = Case(2, 12, 256, torch.bfloat16, 2, 1, 1, seed=10)
    clean = c.run()
    c.x[0, 3, 5], c.y[1, 7, 9] = float("nan"), float("inf")
    got = c.run()
    for n in ("h", "u", "dx", "dy"):
        bad = torch.zeros(2, 12, dtype=torch.bool)
        bad[0, 3] = bad[1, 7] = True
        assert torch.equal(got[n][~bad], clean[n][~bad]), n
    assert bool(torch.isnan(got["u"][0, 3]).all()) and bool(torch.isnan(got["u"][1, 7]).all())


def test_gradients_against_differences():
    """Of the 64-bit formula: a loss linear in h and u, moved along random directions."""
    c = Case(2, 6, 40, torch.float32, 2, 1, 2, scale=1.25, seed=11)
    got = c.run()
    names = ["x", "y", "gate", "w_post", "w_pre", "b_pre"]
    base = {n: getattr(c, n).double().cpu() for n in names}

    def loss(v):
        total = 0.0
        for b in range(2):
            h = c.scale * v["x"][b] + v["gate"][b] * normed(v["y"][b], 1, v["w_post"], 0.0)[0]
            u = normed(h, 2, v["w_pre"], v["b_pre"])[0]
            total += float((h * c.d_h[b].double().cpu()).sum() + (u * c.d_u[b].double().cpu()).sum())
        return total

    g = torch.Generator().manual_seed(12)
    for n in names:
        e = torch.randn(base[n].shape, generator=g, dtype=torch.float64)
        step = 1e-5
        diff = (loss({**base, n: base[n] + step * e}) - loss({**base, n: base[n] - step * e})) / (2 * step)
        grad = {"x": "dx", "y": "dy"}.get(n, "d_" + n)
        mine = float((got[grad].double().cpu().view(e.shape) * e).sum())
        assert abs(mine - diff) <= 1e-4 * (abs(diff) + float((got[grad].double().cpu().view(e.shape) * e).abs().sum()) * 0.1), (n, mine, diff)


def test_captured_and_replayed_and_on_another_stream():
    c = Case(2, 50, 512, torch.bfloat16, 1, 1, 2, kept=[20, 31], seed=13)
    want = c.run()
    out = {n: torch.full_like(t, 7.0) if t is not None else None for n, t in want.items()}
    ws = vd.alloc_ws(vd.vardrop_norm_workspace_bytes(c.cfg))

    def both():
        vd.vardrop_norm_fwd(c.x, c.y, c.gate, c.w_post, c.b_post, c.w_pre, c.b_pre, c.sel, c.n_sel, c.cfg, out["h"], out["u"], out["stats"])
        vd.vardrop_norm_bwd(c.x, c.y, c.gate, c.w_post, c.b_post, c.w_pre, c.sel, c.n_sel, c.inv, out["stats"], c.d_h, c.d_u, c.cfg, out["dx"], out["dy"], out["d_gate"],
                            out["d_w_post"], out["d_b_post"], out["d_w_pre"], out["d_b_pre"], ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    for n, t in want.items():
        assert t is None or torch.equal(t, out[n]), n
        if t is not None:
            out[n].fill_(7.0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        both()
    c.x.neg_()
    graph.replay()
    torch.cuda.synchronize()
    moved = c.run()
    for n, t in moved.items():
        assert t is None or torch.equal(t, out[n]), n


def test_offsets_beyond_32_bits():
    """270000 rows of 8192: what the last ones give is what they give alone, bit for bit."""
    N, C, last = 270000, 8192, 33
    small = Case(1, last, C, torch.bfloat16, 1, 0, 0, with_y=False, seed=4)
    want = small.run()
    big = lambda: torch.empty((1, N, C), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    x, u, d_u, dx = big(), big(), big(), big()
    x.fill_(1.0)
    d_u.zero_()
    x[0, N - last:], d_u[0, N - last:] = small.x[0], small.d_u[0]
    cfg = vd.NormCfg(1, N, C, 0, 1, 0, 0, 0, 1.0, EPS)
    stats = torch.empty((1, N, 4), device="cuda")
    vd.vardrop_norm_fwd(x, None, None, None, None, small.w_pre, None, None, None, cfg, None, u, stats)
    d_h = torch.zeros_like(x)
    d_h[0, N - last:] = small.d_h[0]
    ws = vd.alloc_ws(vd.vardrop_norm_workspace_bytes(cfg))
    vd.vardrop_norm_bwd(x, None, None, None, None, small.w_pre, None, None, None, stats, d_h, d_u, cfg, dx, None, None, None, None, None, None, ws)
    assert vd.ws_status(ws) == vd.OK
    for t, n in ((u, "u"), (dx, "dx")):
        assert torch.equal(t[0, N - last:], want[n][0]), n
    assert torch.equal(stats[0, N - last:, 3], want["stats"][0, :, 3])


@pytest.mark.parametrize("selected", [False, True])
def test_as_many_rows_as_a_call_may_have(selected):
    """2^31 - 1 tokens of one channel: the walk over them looks ahead past what 32 bits with a sign hold.  h = x / 2 and dx = d_h / 2 are exact."""
    N = 2 ** 31 - 1
    cfg = vd.NormCfg(1, N, 1, vd.DTYPES[torch.bfloat16], 0, 0, 0, 1 if selected else 0, 0.5, EPS)
    x, d_h = (torch.empty((1, N, 1), dtype=torch.bfloat16, device="cuda").normal_() for _ in range(2))
    h, dx = (torch.zeros_like(x) for _ in range(2))
    every = torch.arange(N, dtype=torch.int32, device="cuda")[None] if selected else None
    n_sel = torch.tensor([N], dtype=torch.int32, device="cuda") if selected else None
    vd.vardrop_norm_fwd(x, None, None, None, None, None, None, every, n_sel, cfg, h, None, None)
    stats, ws = torch.empty((1, N, 4), device="cuda"), vd.alloc_ws(vd.vardrop_norm_workspace_bytes(cfg))
    vd.vardrop_norm_bwd(x, None, None, None, None, None, every, n_sel, every, stats, d_h, None, cfg, dx, None, None, None, None, None, None, ws)
    for part in range(0, N, 1 << 28):
        at = slice(part, part + (1 << 28))
        assert torch.equal(h[:, at], x[:, at] / 2) and torch.equal(dx[:, at], d_h[:, at] / 2), part


def test_counts_outside_the_rows_are_taken_as_none_or_all():
    """A count that no selection gives: nothing is written behind the rows that there are."""
    for n, kept in ((-3, 0), (9, 9), (1 << 30, 9)):
        c = Case(2, 9, 64, torch.float32, 1, 1, 1, kept=[9], seed=6)
        c.n_sel.fill_(n)
        c.kept = [kept] * 2
        got = c.run()
        assert bool((got["h"] == 7.0).all()) == (kept == 0) and bool(torch.isfinite(got["d_w_pre"]).all())


def test_refusals():
    c = Case(2, 6, 40, torch.float32, 1, 1, 1, seed=14)
    h, u, st = torch.empty_like(c.x), torch.empty_like(c.x), torch.empty(2, 6, 4, device="cuda")
    fwd = lambda x=c.x, y=c.y, gate=c.gate, cfg=c.cfg, b_pre=None: vd.vardrop_norm_fwd(x, y, gate, c.w_post, None, c.w_pre, b_pre, None, None, cfg, h, u, st)  # noqa: E731
    fwd()
    for bad in (dict(x=c.x.bfloat16()), dict(x=c.x.cpu()), dict(x=c.x[:, :5]), dict(x=c.x.transpose(0, 1)), dict(gate=c.gate[:, :39]), dict(y=c.y.reshape(-1)[:-1])):
        with pytest.raises(ValueError):
            fwd(**bad)
    for bad in (dict(gate=None), dict(y=None), dict(b_pre=c.w_pre), dict(x=None)):
        with pytest.raises(vd.VardropError):
            fwd(**bad)
    with pytest.raises((TypeError, ValueError)):
        fwd(cfg=vd.ClipCfg(1.0, 0.0))
    torch.cuda.synchronize()
