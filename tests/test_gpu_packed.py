"""vardrop_packed_plan and vardrop_attn_packed_fwd / _bwd against the formulas in 64 bits, element by element.

Tolerances, from half a step of bf16 (2^-8 of a value): P is rounded once ahead of P V and P^T dO, dS once ahead of its products, o, dq, dk, dv once at the end, and Delta is
taken from the rounded o.  fp32 scores, exponentials and sums add less than 2^-16 of the magnitudes that they are made of at the sizes here."""
import math

import numpy as np
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

H8, F = 2.0 ** -8, 2.0 ** -16
NAN = float("nan")


def reference(q, k, v, d_o, spans, causal, scale):
    """Values and bounds {name: (value, bound)} over the packed rows; rows of no sequence are None by the mask."""
    T, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    z = lambda H, *m: torch.zeros(T, H, *m, dtype=torch.float64, device=q.device)  # noqa: E731
    val = dict(o=z(Hq, D), lse=z(Hq), dq=z(Hq, D), dk=z(Hkv, D), dv=z(Hkv, D))
    off = {n: torch.zeros_like(t) for n, t in val.items()}
    live = torch.zeros(T, dtype=torch.bool, device=q.device)
    for a, b in spans:
        if a == b:
            continue
        live[a:b] = True
        mask = torch.ones(b - a, b - a, dtype=torch.bool, device=q.device).triu(1) if causal else None
        for h in range(Hq):
            Q, K, V, dO = (t.double() for t in (q[a:b, h], k[a:b, h // G], v[a:b, h // G], d_o[a:b, h]))
            S, size = Q @ K.T * scale, Q.abs() @ K.abs().T * scale
            if causal:
                S = S.masked_fill(mask, -math.inf)
            lse = torch.logsumexp(S, 1)
            P = torch.exp(S - lse[:, None])
            rel = H8 + F * (1 + size.amax(1, keepdim=True))                  # of a rounded P
            O = P @ V
            o_off = (rel * P) @ V.abs() + H8 * O.abs()
            dP, delta = dO @ V.T, (dO * O).sum(1, keepdim=True)
            dS = P * (dP - delta)
            ds_off = H8 * dS.abs() + P * ((dO.abs() * o_off).sum(1, keepdim=True) + F * (1 + size.amax(1, keepdim=True)) * (dO.abs() @ V.abs().T + (dO * O).abs().sum(1, keepdim=True)))
            dq, dk, dv = scale * dS @ K, scale * dS.T @ Q, P.T @ dO
            val["o"][a:b, h], off["o"][a:b, h] = O, o_off
            val["lse"][a:b, h], off["lse"][a:b, h] = lse, F * (1 + size.amax(1))
            val["dq"][a:b, h], off["dq"][a:b, h] = dq, scale * ds_off @ K.abs() + H8 * dq.abs()
            val["dk"][a:b, h // G] += dk
            off["dk"][a:b, h // G] += scale * ds_off.T @ Q.abs()
            val["dv"][a:b, h // G] += dv
            off["dv"][a:b, h // G] += (rel * P).T @ dO.abs()
    for n in ("dk", "dv"):
        off[n] += H8 * val[n].abs()
    return val, off, live


class Case:
    def __init__(self, lens, Hq, Hkv, D, causal, fused=False, front=0, tail=0, scale=0.0, std=1.0, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T, self.Hq, self.Hkv, self.D, self.causal = front + sum(lens) + tail, Hq, Hkv, D, causal
        T = self.T
        rand = lambda *s: (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()  # noqa: E731
        if fused:
            x = rand(T, Hq + 2 * Hkv, D)
            self.q, self.k, self.v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
            strides = [(Hq + 2 * Hkv) * D, D] * 2
        else:
            self.q, self.k, self.v, strides = rand(T, Hq, D), rand(T, Hkv, D), rand(T, Hkv, D), [0] * 4
        self.d_o = rand(T, Hq, D)
        at = np.cumsum([front] + list(lens))
        self.spans = list(zip(at[:-1].tolist(), at[1:].tolist()))
        self.cu = torch.from_numpy(at.astype(np.int32)).cuda()
        self.scale = scale or 1 / math.sqrt(D)
        self.cfg = vd.PackedCfg(len(lens), T, Hq, Hkv, D, scale, causal, *strides)
        self.plan = vd.alloc_packed_plan(self.cfg)
        live = torch.zeros(T, dtype=torch.bool, device="cuda")
        for a, b in self.spans:
            live[a:b] = True
        self.live = live
        for t in (self.q, self.k, self.v, self.d_o):       # rows of no sequence may hold anything
            t[~live] = NAN

    def new(self, fill=5.0):
        T, Hq, Hkv, D = self.T, self.Hq, self.Hkv, self.D
        b = lambda H: torch.full((T, H, D), fill, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        ws = vd.alloc_ws(vd.vardrop_attn_packed_workspace_bytes(self.cfg))
        ws.view(torch.int16).fill_(0x7FC1)
        ws[:4] = 0
        return dict(o=b(Hq), lse=torch.full((Hq, T), fill, device="cuda"), dq=b(Hq), dk=b(Hkv), dv=b(Hkv), ws=ws)

    def call(self, out, plan=True):
        if plan:
            vd.vardrop_packed_plan(self.cu, self.cfg, self.plan)
        vd.vardrop_attn_packed_fwd(self.q, self.k, self.v, self.plan, self.cfg, out["o"], out["lse"], out["ws"])
        vd.vardrop_attn_packed_bwd(self.q, self.k, self.v, out["o"], out["lse"], self.d_o, self.plan, self.cfg, out["dq"], out["dk"], out["dv"], out["ws"])

    def run(self):
        out = self.new()
        self.call(out)
        torch.cuda.synchronize()
        assert vd.ws_status(self.plan) == vd.OK and vd.ws_status(out["ws"]) == vd.OK
        return out

    def check(self, out=None):
        out = out or self.run()
        val, off, live = reference(self.q, self.k, self.v, self.d_o, self.spans, self.causal, self.scale)
        for n in ("o", "lse", "dq", "dk", "dv"):
            got = (out[n].t() if n == "lse" else out[n]).double()
            assert bool((got[~live] == 5.0).all()), f"{n}: rows of no sequence"
            err = (got - val[n]).abs()[live]
            assert bool(torch.isfinite(err).all()), n
            worst = (err - off[n][live]).max() if err.numel() else torch.tensor(-1.0)
            assert worst <= 1e-6 * self.scale * self.D, (n, float(err.max()), float(worst))
            norm = val[n].norm()
            if n not in ("lse",) and norm > 1e-2 and max(b - a for a, b in self.spans) > 8:
                assert err.norm() <= 3 * H8 * norm, (n, float(err.norm() / norm))
        return out


LENS = [[1], [2], [5], [64], [65], [127, 128, 129], [0, 5, 0, 300, 0], [1] * 40, [257, 1, 384, 33], [511, 700], [1025], [130, 17, 260, 128, 3, 256, 1, 400]]


@pytest.mark.parametrize("lens", LENS, ids=lambda x: "-".join(map(str, x[:6])))
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("Hq,Hkv,D", [(2, 2, 64), (4, 2, 32), (3, 1, 64)])
def test_lengths(lens, causal, Hq, Hkv, D):
    Case(lens, Hq, Hkv, D, causal, seed=sum(lens)).check()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (2, 1), (5, 5), (6, 2), (8, 1), (15, 3), (16, 4), (7, 7)])
@pytest.mark.parametrize("causal,fused,front,tail", [(1, True, 0, 0), (0, False, 3, 200), (1, False, 131, 1)])
def test_heads_and_layouts(Hq, Hkv, causal, fused, front, tail):
    Case([200, 1, 131, 0, 390, 64], Hq, Hkv, 64 if Hq % 2 else 32, causal, fused=fused, front=front, tail=tail, seed=Hq).check()


@pytest.mark.parametrize("n", [148, 300, 1024, 1025, 2500])
@pytest.mark.parametrize("causal", [0, 1])
def test_many_sequences(n, causal):
    rng = np.random.default_rng(n)
    Case(rng.integers(0, 60 if n > 1000 else 200, n).tolist(), 2, 1, 32, causal, seed=n).check()


@pytest.mark.parametrize("lens,Hq,Hkv,causal", [([4000, 131], 2, 1, 1), ([2300, 900], 3, 3, 0), ([2049, 1, 2047, 700], 8, 2, 1)])
def test_long_sequences(lens, Hq, Hkv, causal):
    Case(lens, Hq, Hkv, 64, causal, seed=1).check()


@pytest.mark.parametrize("lens,Hq,Hkv,D", [([1300], 1, 1, 64), ([900, 1500, 400], 1, 1, 32), ([385, 513, 641, 769, 897], 3, 3, 64), ([640, 1281], 4, 2, 32), ([384, 385, 512], 5, 1, 64), ([3333], 2, 2, 64),
                                           ([300, 20, 1000, 257], 8, 2, 64), ([1100] * 16, 2, 1, 64), ([1100] * 17, 2, 1, 64)])
@pytest.mark.parametrize("causal", [0, 1])
def test_few_long_items(lens, Hq, Hkv, D, causal):
    """Calls in which the query tiles of two heads are fewer than the SMs, with odd and even numbers of key tiles, and those around the line."""
    Case(lens, Hq, Hkv, D, causal, seed=len(lens)).check()


@pytest.mark.parametrize("more", [-1, 0, 1])
@pytest.mark.parametrize("D,causal", [(64, 0), (32, 0), (64, 1)])
def test_one_head_with_a_long_tile_for_every_sm(more, D, causal):
    """One head, and as many tiles with more than two key tiles as SMs, one fewer and one more, beside sequences of one and two tiles."""
    tiles = torch.cuda.get_device_properties(0).multi_processor_count + more
    if causal:                       # four tiles of a sequence of six have more than two key tiles
        lens = [768] * (tiles // 4) + ([256 + 128 * (tiles % 4)] if tiles % 4 else [])
    else:
        lens = [384] * (tiles // 3 - 1) + [384 + 128 * (tiles % 3)]
    Case(lens + [100, 1, 0, 130, 256], 1, 1, D, causal, seed=tiles).check()


@pytest.mark.parametrize("late", [0, 1])
def test_parts_of_far_apart_sizes(late):
    """The keys of one of every two tiles have scores far above the others': one part of a row outweighs the other by more than fp32 holds."""
    c = Case([900], 1, 1, 64, 0, seed=8)
    for tile in range(8):
        c.k[128 * tile:128 * (tile + 1)] *= 4.0 if tile % 2 == late else 0.01
    c.check()


@pytest.mark.parametrize("scale", [0.01, 0.3, 1.0])
def test_scales(scale):
    Case([300, 77, 129], 2, 2, 64, 1, scale=scale, seed=2).check()


@pytest.mark.parametrize("scale", [1e-40, 1e-30, 1e-6, 2.0])
@pytest.mark.parametrize("lens", [[40], [300, 131]])
def test_scales_far_from_one(scale, lens):
    """Where the scores are next to nothing the exponents' -lse / scale has to stay finite.  A gradient below the least normal bf16 value has half of that value's step (2^-134)."""
    c = Case(lens, 2, 1, 64, 1, scale=scale, seed=3)
    if scale > 1e-38:
        c.check()
        return
    out = c.run()
    val, off, live = reference(c.q, c.k, c.v, c.d_o, c.spans, 1, scale)
    for n in ("o", "lse", "dv"):
        got = (out[n].t() if n == "lse" else out[n]).double()[live]
        assert bool(((got - val[n][live]).abs() <= off[n][live] + 1e-6).all()), n
    for n in ("dq", "dk"):
        assert bool(torch.isfinite(out[n].double()[live]).all()) and float(out[n].double()[live].abs().max()) <= 1e-35, n


def test_forward_with_a_header_for_a_workspace():
    c = Case([300, 131, 1], 3, 1, 64, 1, seed=4)
    want, out = c.run(), c.new()
    ws = torch.full((512,), 0x7F, dtype=torch.uint8, device="cuda")
    ws[:4] = 0
    vd.vardrop_attn_packed_fwd(c.q, c.k, c.v, c.plan, c.cfg, out["o"], out["lse"], ws[:256])
    assert vd.ws_status(ws) == vd.OK and torch.equal(out["o"], want["o"]) and torch.equal(out["lse"], want["lse"]) and bool((ws[256:] == 0x7F).all())


def test_large_scores():
    """Scores in the hundreds: rows in which one key has all the weight, references that move by far more than a step."""
    Case([300, 77, 129, 600], 2, 1, 64, 1, std=5.0, seed=3).check()
    Case([300, 600], 2, 1, 64, 0, std=5.0, seed=4).check()


def test_one_key_takes_everything_late():
    """The reference maximum grows behind the first key tiles: what has been summed up is scaled down."""
    c = Case([700], 2, 2, 64, 1, seed=5)
    c.k[500:, :, :] *= 6
    c.q[:, :, :] *= 2
    c.check()


def expected_plan(lens, front, causal):
    at, base, out = front, 0, []
    for n in lens:
        t = (n + 127) // 128
        out += [(i + 1 if causal else t, (at, n, i, base)) for i in range(t)]
        at += n
        base += t
    return out


@pytest.mark.parametrize("lens,front", [([5], 0), ([0, 0, 1], 4), ([1000, 30, 0, 129, 128, 5000], 7), (list(range(0, 300)), 0), ([3] * 5000, 2), ([700000], 0)])
@pytest.mark.parametrize("causal", [0, 1])
def test_plan(lens, front, causal):
    T = front + sum(lens) + 11
    cfg = vd.PackedCfg(len(lens), T, 1, 1, 32, 0.0, causal, 0, 0, 0, 0)
    plan = vd.alloc_packed_plan(cfg)
    cu = torch.from_numpy(np.cumsum([front] + lens).astype(np.int32)).cuda()
    vd.vardrop_packed_plan(cu, cfg, plan)
    words = plan.cpu().numpy().view(np.int32)
    want = expected_plan(lens, front, causal)
    assert words[0] == vd.OK and words[2] == len(want)
    got = [tuple(e) for e in words[64:64 + 4 * len(want)].reshape(-1, 4).tolist()]
    work = {e: w for w, e in want}
    assert sorted(got) == sorted(work)
    order = [min(work[e], 4096) for e in got]
    assert order == sorted(order, reverse=True)


@pytest.mark.parametrize("cu", [[0, 5, 3, 9], [-1, 2, 3, 9], [0, 4, 8, 101], [0, 2 ** 31 - 1, 3, 9], [9, 8, 7, 6]])
def test_offsets_that_are_none(cu):
    """The plan says so, and calls with it write nothing and say so too."""
    c = Case([30, 30, 40], 2, 1, 32, 1)
    c.cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    out = c.new()
    c.call(out)
    torch.cuda.synchronize()
    assert vd.ws_status(c.plan) == vd.ERR_INVALID_ARG and vd.ws_status(out["ws"]) == vd.ERR_INVALID_ARG
    for n in ("o", "lse", "dq", "dk", "dv"):
        assert bool((out[n] == 5.0).all()), n
    many = vd.PackedCfg(40000, 1 << 20, 1, 1, 32, 0.0, 0, 0, 0, 0, 0)           # bad from the first sequence on, tiles without end if they were counted
    plan = vd.alloc_packed_plan(many)
    vd.vardrop_packed_plan(torch.tensor([0, 1 << 20] * 20001, dtype=torch.int32, device="cuda"), many, plan)
    assert vd.ws_status(plan) == vd.ERR_INVALID_ARG


def test_a_plan_of_another_kind():
    c = Case([30, 30, 40], 2, 1, 32, 1)
    vd.vardrop_packed_plan(c.cu, c.cfg, c.plan)
    for change in (dict(causal=0), dict(n_seqs=2), dict(T=99)):
        cfg = vd.PackedCfg(*[change.get(n, getattr(c.cfg, n)) for n, _ in vd.PackedCfg._fields_])
        out = c.new()
        vd.vardrop_attn_packed_fwd(c.q, c.k, c.v, c.plan, cfg, out["o"], out["lse"], out["ws"])
        assert vd.ws_status(out["ws"]) == vd.ERR_INVALID_ARG and bool((out["o"] == 5.0).all())
    blank = torch.zeros_like(c.plan)
    out = c.new()
    vd.vardrop_attn_packed_fwd(c.q, c.k, c.v, blank, c.cfg, out["o"], out["lse"], out["ws"])
    assert vd.ws_status(out["ws"]) == vd.ERR_INVALID_ARG and bool((out["o"] == 5.0).all())


@pytest.mark.parametrize("bad", [NAN, float("inf")])
@pytest.mark.parametrize("causal", [0, 1])
def test_values_that_are_not_finite_stay_in_their_sequence(bad, causal):
    lens = [100, 77, 300, 5, 128, 40]
    c = Case(lens, 4, 2, 64, causal, seed=6)
    clean = c.run()
    a, b = c.spans[2]
    for t in (c.q, c.k, c.v, c.d_o):
        t[a + 2:a + 4] = bad
        t[b - 1] = bad
    got = c.run()
    other = torch.ones(c.T, dtype=torch.bool, device="cuda")
    other[a:b] = False
    for n in ("o", "dk", "dv", "dq"):
        assert torch.equal(got[n][other], clean[n][other]), n
    assert torch.equal(got["lse"][:, other], clean["lse"][:, other])


def test_runs_repeat_bit_for_bit():
    c = Case([1500, 300, 20, 777], 6, 2, 64, 1, seed=7)
    a, b = c.run(), c.run()
    for n in ("o", "lse", "dk", "dv"):
        assert torch.equal(a[n], b[n]), n
    near = (a["dq"].double() - b["dq"].double()).norm() / a["dq"].double().norm()
    assert near < H8
    c = Case([256, 100, 20, 129], 6, 2, 64, 1, seed=7)           # at most two terms: their order does not matter
    assert torch.equal(c.run()["dq"], c.run()["dq"])


def test_captured_replayed_and_two_streams_at_once():
    c = Case([700, 33, 129, 260], 4, 2, 64, 1, seed=8)
    want = c.run()
    out = c.new()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.call(out)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for n in ("o", "lse", "dk", "dv"):
        assert torch.equal(out[n], want[n]), n
    c.q[:] = -c.q
    graph.replay()
    torch.cuda.synchronize()
    c.check(out)
    c.q[:] = -c.q
    outs, streams = [c.new() for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    vd.vardrop_packed_plan(c.cu, c.cfg, c.plan)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                c.call(o, plan=False)
    torch.cuda.synchronize()
    for o in outs:
        assert vd.ws_status(o["ws"]) == vd.OK
        for n in ("o", "lse", "dk", "dv"):
            assert torch.equal(o[n], want[n]), n


def test_offsets_beyond_32_bits():
    """2^20 rows of 34 heads of 64: the last sequences' elements lie behind 2^31."""
    T, Hq, Hkv, D = 1 << 20, 34, 2, 64
    lens = [200, 131]
    small = Case(lens, Hq, Hkv, D, 1, seed=9)
    got = small.new()
    big = lambda H: torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q, k, v, d_o, o, dq, dk, dv = big(Hq), big(Hkv), big(Hkv), big(Hq), big(Hq), big(Hq), big(Hkv), big(Hkv)
    rows = slice(T - sum(lens), T)
    for a, b in ((q, small.q), (k, small.k), (v, small.v), (d_o, small.d_o)):
        a[rows] = b
    cfg = vd.PackedCfg(2, T, Hq, Hkv, D, 0.0, 1, 0, 0, 0, 0)
    plan, lse = vd.alloc_packed_plan(cfg), torch.empty((Hq, T), device="cuda")
    cu = torch.tensor([T - 331, T - 131, T], dtype=torch.int32, device="cuda")
    ws = vd.alloc_ws(vd.vardrop_attn_packed_workspace_bytes(cfg))
    vd.vardrop_packed_plan(cu, cfg, plan)
    vd.vardrop_attn_packed_fwd(q, k, v, plan, cfg, o, lse, ws)
    vd.vardrop_attn_packed_bwd(q, k, v, o, lse, d_o, plan, cfg, dq, dk, dv, ws)
    assert vd.ws_status(ws) == vd.OK
    for t, n in ((o, "o"), (dq, "dq"), (dk, "dk"), (dv, "dv")):
        got[n][:] = t[rows]
    got["lse"][:] = lse[:, rows]
    small.check(got)


def test_refusals():
    c = Case([30, 30, 40], 4, 2, 32, 1)
    out = c.new()
    vd.vardrop_packed_plan(c.cu, c.cfg, c.plan)
    fwd = lambda q=c.q, k=c.k, plan=c.plan, cfg=c.cfg, lse=out["lse"], ws=out["ws"]: vd.vardrop_attn_packed_fwd(q, k, c.v, plan, cfg, out["o"], lse, ws)  # noqa: E731
    fwd()
    for bad in (dict(q=c.q.float()), dict(q=c.q[:99]), dict(k=c.k.cpu()), dict(q=c.q.transpose(0, 1)), dict(lse=out["lse"].half()), dict(plan=c.plan.view(torch.int32))):
        with pytest.raises(ValueError):
            fwd(**bad)
    strided = vd.PackedCfg(3, 100, 4, 2, 32, 0.0, 1, 256, 32, 0, 0)
    with pytest.raises(ValueError):
        fwd(cfg=strided)
    for bad in (dict(q=None), dict(plan=c.plan[:256]), dict(ws=out["ws"][:128]), dict(plan=None)):
        with pytest.raises(vd.VardropError):
            fwd(**bad)
    with pytest.raises(ValueError):
        vd.vardrop_packed_plan(c.cu[:3], c.cfg, c.plan)
    with pytest.raises(vd.VardropError):
        vd.vardrop_attn_packed_bwd(c.q, c.k, c.v, out["o"], out["lse"], c.d_o, c.plan, c.cfg, out["dq"], out["dk"], out["dv"], out["ws"][:1024])
