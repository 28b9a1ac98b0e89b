"""The work of the operators around the token reduction: what a layer on kept tokens, and the end of its training step, have this library do.

Kinds of a case (`kind`), each one pass through the public entry points of paper_2501_14183_b200.binding:

  prompt   attention over packed sequences, forward alone: vardrop_packed_plan -> vardrop_attn_packed_fwd
  train    the same with its backward pass: vardrop_packed_plan -> vardrop_attn_packed_fwd -> vardrop_attn_packed_bwd
  norm     h = res_scale x + gate o N_post(y), u = N_pre(h), forward alone: vardrop_norm_fwd
  layer    the same with its backward pass: vardrop_norm_fwd -> vardrop_norm_bwd
  clip     the 2-norm over all gradients of a step and the gradients scaled to it: vardrop_grad_clip

Ranges: 1 to 64 sequences of 1 to 8192 tokens, 1 to 32 query heads in groups of 1 to 8 a key head, heads of 32 or 64, causal or not, q / k / v as tensors of
their own or as views of one fused projection, rows behind the last sequence; norms over 8 to 4096 channels, odd ones among them, 1 to 64 instances of 1 to
8192 tokens, bf16, fp16 or fp32, with or without a selection of the tokens; 1 to 400 gradients of 1 to 2^25 values.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
KINDS = {"none": 0, "rms": 1, "layer": 2}
EPS = 1e-5


def _attn(name, kind, lens, Hq, Hkv, D, causal, fused=False, tail=0):
    return dict(name=name, kind=kind, lens=",".join(str(n) for n in lens), Hq=Hq, Hkv=Hkv, D=D, causal=causal, fused=fused, tail=tail)


def _norm(name, kind, B, N, C, dtype, pre, post, gate, kept="", scale=1.0):
    return dict(name=name, kind=kind, B=B, N=N, C=C, dtype=dtype, pre=pre, post=post, gate=gate, kept=kept, scale=scale)


def _clip(name, sizes, dtypes, share):
    return dict(name=name, kind="clip", sizes=",".join(str(n) for n in sizes), dtypes=",".join(dtypes), share=share)


def _layer_sizes(d, f, layers):
    """An encoder's parameters: four projections, two of the feed-forward block, their biases and two norms a layer."""
    return [n for _ in range(layers) for n in (d * d, d, d * d, d, d * d, d, d * d, d, d * f, f, f * d, d, d, d, d, d)]


def listed():
    encoder = _layer_sizes(512, 512, 3) + [96 * 512, 512, 512 * 96, 96]
    wide = [n for _ in range(24) for n in (2048 * 2048, 2048 * 512, 2048 * 512, 2048 * 2048, 2048 * 5632, 2048 * 5632, 5632 * 2048, 2048, 2048)]
    return [
        # a handful of short series, causal along their steps: latency and launches are all there is
        _attn("few short prompts", "prompt", [21, 9, 1, 17], 4, 2, 32, True),
        # prompts of very different lengths in one call, grouped heads
        _attn("ragged prompts", "prompt", [1423, 96, 720, 1, 1999, 336, 862, 55, 1200, 301, 1777, 640, 128, 1025, 90, 411], 16, 4, 64, True),
        # two long prompts, grouped heads: the most products in one forward call
        _attn("long prompts", "prompt", [8192, 5001], 16, 4, 64, True),
        # kept sets of electricity-consumption windows, every instance with a selection of its own, packed without padding: views of a fused projection
        _attn("kept sets", "train", [119, 104, 131, 97, 121, 88, 140, 117, 109, 126, 92, 133, 115, 120, 101, 99, 124, 137, 111, 95, 118, 129, 106, 122, 113, 90, 136, 108,
                                     116, 127, 103, 110], 8, 8, 64, False, fused=True, tail=500),
        # training on windows of different lookbacks, causal along the steps, grouped heads
        _attn("ragged windows", "train", [1423, 96, 720, 1, 1999, 336, 862, 55, 1200, 301, 1777, 640], 8, 2, 64, True),
        # two long sequences: the largest training pass
        _attn("long sequences", "train", [8192, 5001], 16, 4, 64, True),
        # inference of a layer on a small batch: one instance's variates, layer norms as iTransformer-like encoders have them
        _norm("norms of one instance", "norm", 1, 321, 512, "bf16", "layer", "none", 0),
        # the residual stream of kept tokens: gathered by the selection, a gate per instance on the normed branch, road-traffic sensors
        _norm("gated norms of kept tokens", "layer", 32, 862, 512, "bf16", "rms", "rms", 32, kept="172"),
        # fp32 training with a channel count that no vector width divides
        _norm("fp32 norms, odd width", "layer", 16, 321, 515, "fp32", "layer", "layer", 1, scale=1.41),
        # thousands of tokens, every one kept: larger than L2
        _norm("norms of all tokens", "layer", 8, 8192, 1024, "bf16", "rms", "rms", 1),
        # gradients of a three-layer encoder, fp32, norm above the limit
        _clip("encoder gradients", encoder, ["fp32"], 0.5),
        # gradients of a wide model: bf16 weights with fp32 norms, larger than L2
        _clip("wide gradients", wide, ["bf16", "bf16", "bf16", "bf16", "bf16", "bf16", "bf16", "fp32", "fp32"], 0.5),
    ]


MOST_SCORES = 2 * 16 * 8192 * 8192          # padded scores of the largest listed attention
MOST_PAIRS = 16 * (8192 * 8193 + 5001 * 5002) // 2


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "train", "train", "norm", "layer", "layer", "clip"])
    if kind in ("prompt", "train"):
        G = rng.choice([1, 1, 2, 3, 4, 5, 8])
        Hkv = rng.choice([1, 2, 3, 4, 8])
        Hq = min(32, G * Hkv) // Hkv * Hkv
        top, causal = _log(rng, 2, 8192), rng.random() < 0.7
        n = _log(rng, 1, 64)
        lens = [rng.choice([_log(rng, 1, top), rng.randint(1, top)]) for _ in range(n)]
        while n * Hq * max(lens) ** 2 > MOST_SCORES or sum(Hq * m * m for m in lens) > MOST_PAIRS:
            lens = [(m + 1) // 2 for m in lens]
        if rng.random() < 0.2:
            lens[rng.randrange(n)] = 0
        if max(lens) < 2:       # one key a query alone has gradients of zero, which no relative error says anything about
            lens[0] = 2
        return _attn("", kind, lens, Hq, Hkv, rng.choice([32, 64, 64]), causal, rng.random() < 0.5, rng.choice([0, 0, rng.randint(1, 300)]))
    if kind in ("norm", "layer"):
        B, C = _log(rng, 1, 64), rng.choice([_log(rng, 8, 4096), 8 * _log(rng, 1, 512)])      # (two channels' layer norm has no gradient but rounding)
        N = max(1, min(_log(rng, 1, 8192), 8 * 8192 * 1024 // (B * C)))
        sel = rng.choice([0, 1, B])
        kept = ",".join(str(rng.randint(1, N)) for _ in range(sel))
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        if dtype == "fp32":
            N = max(1, N // 2)
            kept = ",".join(str(rng.randint(1, N)) for _ in range(sel))
        pre, post = rng.choice(["rms", "layer"]), rng.choice(["none", "rms", "layer"])
        return _norm("", kind, B, N, C, dtype, pre, post, rng.choice([0, 1, B]), kept, rng.choice([1.0, 0.7, 1.5]))
    n = _log(rng, 1, 400)
    sizes = [_log(rng, 1, 1 << rng.choice([8, 14, 20, 25])) for _ in range(n)]
    while sum(sizes) > 1000000000:
        sizes = [(m + 1) // 2 for m in sizes]
    return _clip("", sizes, [rng.choice(["bf16", "fp16", "fp32"]) for _ in range(rng.randint(1, 5))], rng.choice([0.1, 0.5, 2.0]))


def _ints(text):
    return [int(t) for t in text.split(",")] if text else []


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    if case["kind"] in ("prompt", "train"):
        lens, Hq, Hkv, D = _ints(case["lens"]), case["Hq"], case["Hkv"], case["D"]
        T = sum(lens) + case["tail"]
        offsets = [0]
        for n in lens:
            offsets.append(offsets[-1] + n)
        s["T"], s["n"], s["longest"] = T, len(lens), max(lens)
        s["cu_seqlens"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        if case["fused"]:
            all3 = _normal(g, (T, Hq + 2 * Hkv, D), 1.0, torch.bfloat16)
            s["q"], s["k"], s["v"] = all3[:, :Hq], all3[:, Hq:Hq + Hkv], all3[:, Hq + Hkv:]
        else:
            s["q"], s["k"], s["v"] = (_normal(g, (T, H, D), 1.0, torch.bfloat16) for H in (Hq, Hkv, Hkv))
        s["d_o"] = _normal(g, (T, Hq, D), 1.0, torch.bfloat16) if case["kind"] == "train" else None
        return s
    if case["kind"] in ("norm", "layer"):
        B, N, C, dt = case["B"], case["N"], case["C"], TYPES[case["dtype"]]
        kept = _ints(case["kept"])
        s["x"], s["y"] = _normal(g, (B, N, C), 1.0, dt), _normal(g, (B, N, C), 0.5, dt)
        s["gate"] = _normal(g, (case["gate"], C), 0.5, torch.float32) if case["gate"] else None
        s["w_post"] = 1 + _normal(g, (C,), 0.1, torch.float32) if case["post"] != "none" else None
        s["b_post"] = _normal(g, (C,), 0.1, torch.float32) if case["post"] == "layer" else None
        s["w_pre"] = 1 + _normal(g, (C,), 0.1, torch.float32)
        s["b_pre"] = _normal(g, (C,), 0.1, torch.float32) if case["pre"] == "layer" else None
        s["sel_idx"] = s["inv_idx"] = s["n_sel"] = None
        if kept:            # as vardrop_select gives them: kept tokens ascending, -1 behind them, and every token's place
            S = len(kept)
            order = torch.argsort(torch.rand((S, N), generator=g, device="cuda"), dim=1)
            n_sel = torch.tensor(kept, dtype=torch.int32, device="cuda")
            drawn = torch.where(torch.arange(N, device="cuda") < n_sel[:, None], order, N)
            sel = torch.sort(drawn, dim=1).values
            inv = torch.full((S, N + 1), -1, dtype=torch.int32, device="cuda")
            inv.scatter_(1, sel, torch.arange(N, dtype=torch.int32, device="cuda").expand(S, N).contiguous())
            s["n_sel"], s["sel_idx"] = n_sel, torch.where(sel < N, sel, -1).to(torch.int32)
            s["inv_idx"] = inv[:, :N].contiguous()
        if case["kind"] == "layer":
            s["d_h"], s["d_u"] = _normal(g, (B, N, C), 1.0, dt), _normal(g, (B, N, C), 1.0, dt)
        return s
    sizes, dtypes = _ints(case["sizes"]), case["dtypes"].split(",")
    types = [TYPES[dtypes[i % len(dtypes)]] for i in range(len(sizes))]
    s["flat"] = {dt: _normal(g, (sum(n for n, d in zip(sizes, types) if d == dt),), 0.01, dt) for dt in sorted(set(types), key=str)}
    s["grads"], s["at"], used = [], [], {dt: 0 for dt in s["flat"]}
    for n, dt in zip(sizes, types):         # views of one buffer a type, one behind the other, as buckets for a reduction over ranks have them
        s["at"].append((dt, used[dt], n))
        s["grads"].append(s["flat"][dt][used[dt]:used[dt] + n])
        used[dt] += n
    s["max_norm"] = case["share"] * 0.01 * math.sqrt(sum(sizes))
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------------
def _attn_plain(s):
    """Sequences padded to the longest, masked scores, every step in 32 bits."""
    Hq, Hkv, D, n, m, T = s["Hq"], s["Hkv"], s["D"], s["n"], s["longest"], s["T"]
    G, scale = Hq // Hkv, 1.0 / math.sqrt(D)
    cu = s["cu_seqlens"].long()
    lens = cu[1:] - cu[:-1]
    at = torch.arange(m, device="cuda")
    there = at < lens[:, None]                                              # [n, m]
    rows = torch.where(there, cu[:-1, None] + at, T)                        # row T: a row of zeros

    def padded(t, heads):                                                   # [T, H, D] -> [n, Hkv, heads, m, D]
        z = torch.cat([t.float(), torch.zeros((1, *t.shape[1:]), device="cuda")])[rows]
        return z.view(n, m, Hkv, heads, D).permute(0, 2, 3, 1, 4)

    def unpadded(t, H):                                                     # [n, H, m, X] -> [T, H, X], zeros behind the last sequence
        out = torch.zeros((T + 1, H, t.shape[-1]), device="cuda")
        out[rows] = t.permute(0, 2, 1, 3)
        out[T] = 0
        return out[:T]

    q, k, v = padded(s["q"], G), padded(s["k"], 1), padded(s["v"], 1)
    seen = there[:, None, :] & (at[:, None] >= at[None, :]) if s["causal"] else there[:, None, :].expand(n, m, m)
    seen = seen[:, None, None]
    p = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True).clamp_min(-3e38)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = top + total.log()
    p = p.div_(total.clamp_min(1e-38))
    o = torch.matmul(p, v)
    res = {"o": unpadded(o.reshape(n, Hq, m, D), Hq).to(torch.bfloat16), "lse": unpadded(lse.reshape(n, Hq, m, 1), Hq)[..., 0].t().contiguous()}
    if s["kind"] == "prompt":
        return res
    d_o = padded(s["d_o"], G)
    delta = (d_o * o).sum(-1, keepdim=True)
    dv = torch.matmul(p.transpose(-1, -2), d_o).sum(2)
    ds = torch.matmul(d_o, v.transpose(-1, -2)).sub_(delta).mul_(p).mul_(scale)
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q).sum(2)
    return {**res, "dq": unpadded(dq.reshape(n, Hq, m, D), Hq).to(torch.bfloat16), "dk": unpadded(dk, Hkv).to(torch.bfloat16), "dv": unpadded(dv, Hkv).to(torch.bfloat16)}


def _normed(t, kind, w, b):
    """N(t), t without its mean and scaled, and the scale."""
    if kind == "none":
        return t, t, None
    c = t - t.mean(-1, keepdim=True) if kind == "layer" else t
    r = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
    z = c * r
    return z * w + (b if b is not None else 0), z, r


def _normed_back(d, z, r, kind, w):
    """Gradient of t from the gradient d of N(t)."""
    if kind == "none":
        return d
    e = d * w
    e = e - z * (e * z).mean(-1, keepdim=True)
    return r * (e - (d * w).mean(-1, keepdim=True) if kind == "layer" else e)


def _norm_plain(s):
    B, N, C, dt = s["B"], s["N"], s["C"], TYPES[s["dtype"]]
    live, x = torch.ones((B, N, 1), dtype=torch.bool, device="cuda"), s["x"].float()
    if s["kept"]:
        sel = s["sel_idx"].long().clamp_min(0).expand(B, N)
        live = (torch.arange(N, device="cuda") < s["n_sel"][:, None]).expand(B, N)[..., None]
        x = torch.gather(x, 1, sel[..., None].expand(B, N, C))
    gate = s["gate"][:, None] if s["gate"] is not None else torch.ones((1, 1, 1), device="cuda")
    yn, zy, ry = _normed(s["y"].float(), s["post"], s["w_post"], s["b_post"])
    h = s["scale"] * x + gate * yn
    u, zh, rh = _normed(h, s["pre"], s["w_pre"], s["b_pre"])
    res = {"h": torch.where(live, h, 0).to(dt), "u": torch.where(live, u, 0).to(dt)}
    if s["kind"] == "norm":
        return res
    d_u, d_h = torch.where(live, s["d_u"].float(), 0), torch.where(live, s["d_h"].float(), 0)
    t = d_h + _normed_back(d_u, zh, rh, s["pre"], s["w_pre"])
    dx = s["scale"] * t
    if s["kept"]:
        inv = s["inv_idx"].long().expand(B, N)[..., None]
        dx = torch.where(inv >= 0, torch.gather(dx, 1, inv.clamp_min(0).expand(B, N, C)), 0)
    d_yn = gate * t
    res["dx"], res["dy"] = dx.to(dt), torch.where(live, _normed_back(d_yn, zy, ry, s["post"], s["w_post"]), 0).to(dt)
    if s["gate"] is not None:       # 64 bits for sums over tens of thousands of tokens
        res["d_gate"] = (t * yn).sum((0, 1) if s["gate"].shape[0] == 1 else 1, dtype=torch.float64).view(s["gate"].shape).float()
    if s["post"] != "none":
        res["d_w_post"] = (d_yn * zy).sum((0, 1), dtype=torch.float64).float()
    if s["post"] == "layer":
        res["d_b_post"] = d_yn.sum((0, 1), dtype=torch.float64).float()
    res["d_w_pre"] = (d_u * zh).sum((0, 1), dtype=torch.float64).float()
    if s["pre"] == "layer":
        res["d_b_pre"] = d_u.sum((0, 1), dtype=torch.float64).float()
    return res


def _clip_plain(s):
    squares = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]])
    norm = squares.sum().sqrt()
    factor = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0).float()
    return {"norm": norm.float().view(1), "grads": [(g.float() * factor).to(g.dtype) for g in s["flat"].values()]}


# ---- the framework's calls -------------------------------------------------------------------------------------------------
def _attn_own(s):
    from paper_2501_14183_b200 import binding as vd
    if "cfg" not in s:              # what a training program sets up once: configuration, plan, outputs, workspace
        Hq, Hkv, D, T = s["Hq"], s["Hkv"], s["D"], s["T"]
        strides = [(Hq + 2 * Hkv) * D, D, (Hq + 2 * Hkv) * D, D] if s["fused"] else [0, 0, 0, 0]
        s["cfg"] = cfg = vd.PackedCfg(s["n"], T, Hq, Hkv, D, 0.0, 1 if s["causal"] else 0, *strides)
        s["plan"] = vd.alloc_packed_plan(cfg)
        s["o"] = torch.zeros((T, Hq, D), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((Hq, T), device="cuda")
        s["ws"] = vd.alloc_ws(vd.vardrop_attn_packed_workspace_bytes(cfg))
        if s["kind"] == "train":
            s["dq"] = torch.zeros_like(s["o"])
            s["dk"], s["dv"] = (torch.zeros((T, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    vd.vardrop_packed_plan(s["cu_seqlens"], s["cfg"], s["plan"])
    vd.vardrop_attn_packed_fwd(s["q"], s["k"], s["v"], s["plan"], s["cfg"], s["o"], s["lse"], s["ws"])
    if s["kind"] == "prompt":
        return {"o": s["o"], "lse": s["lse"]}
    vd.vardrop_attn_packed_bwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["d_o"], s["plan"], s["cfg"], s["dq"], s["dk"], s["dv"], s["ws"])
    return {"o": s["o"], "lse": s["lse"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _norm_own(s):
    from paper_2501_14183_b200 import binding as vd
    if "cfg" not in s:
        B, N, C = s["B"], s["N"], s["C"]
        s["cfg"] = cfg = vd.NormCfg(B, N, C, vd.DTYPES[TYPES[s["dtype"]]], KINDS[s["pre"]], KINDS[s["post"]], s["gate"].shape[0] if s["gate"] is not None else 0,
                                    s["n_sel"].shape[0] if s["kept"] else 0, s["scale"], EPS)
        s["h"], s["u"] = torch.zeros_like(s["x"]), torch.zeros_like(s["x"])
        s["stats"] = torch.empty((B, N, 4), device="cuda")
        if s["kind"] == "layer":
            s["dx"], s["dy"] = torch.zeros_like(s["x"]), torch.zeros_like(s["x"])
            s["out"] = {"d_" + k: torch.empty_like(s[k]) if s[k] is not None else None for k in ("gate", "w_post", "b_post", "w_pre", "b_pre")}
            s["ws"] = vd.alloc_ws(vd.vardrop_norm_workspace_bytes(cfg))
    vd.vardrop_norm_fwd(s["x"], s["y"], s["gate"], s["w_post"], s["b_post"], s["w_pre"], s["b_pre"], s["sel_idx"], s["n_sel"], s["cfg"], s["h"], s["u"], s["stats"])
    if s["kind"] == "norm":
        return {"h": s["h"], "u": s["u"]}
    out = s["out"]
    vd.vardrop_norm_bwd(s["x"], s["y"], s["gate"], s["w_post"], s["b_post"], s["w_pre"], s["sel_idx"], s["n_sel"], s["inv_idx"], s["stats"], s["d_h"], s["d_u"], s["cfg"],
                        s["dx"], s["dy"], out["d_gate"], out["d_w_post"], out["d_b_post"], out["d_w_pre"], out["d_b_pre"], s["ws"])
    return {"h": s["h"], "u": s["u"], "dx": s["dx"], "dy": s["dy"], **{k: t for k, t in out.items() if t is not None}}


def _clip_own(s):
    from paper_2501_14183_b200 import binding as vd
    if "cfg" not in s:
        s["cfg"] = vd.ClipCfg(s["max_norm"], 1e-6)
        s["norm"], s["out"] = torch.zeros(1, device="cuda"), {dt: torch.empty_like(f) for dt, f in s["flat"].items()}
        s["clipped"] = [s["out"][dt][at:at + n] for dt, at, n in s["at"]]
        s["ws"] = vd.alloc_ws(vd.vardrop_grad_clip_workspace_bytes())
    vd.vardrop_grad_clip(s["grads"], s["cfg"], s["clipped"], s["norm"], s["ws"])
    return {"norm": s["norm"], "grads": list(s["out"].values())}


def run(state):
    if state["kind"] in ("prompt", "train"):
        return _attn_own(state) if own else _attn_plain(state)
    if state["kind"] in ("norm", "layer"):
        return _norm_own(state) if own else _norm_plain(state)
    return _clip_own(state) if own else _clip_plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------
def work(case):
    if case["kind"] in ("prompt", "train"):
        lens, Hq, Hkv, D = _ints(case["lens"]), case["Hq"], case["Hkv"], case["D"]
        pairs = Hq * sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lens)
        rows_q, rows_kv, lse = 2 * sum(lens) * Hq * D, 2 * sum(lens) * Hkv * D, 4 * sum(lens) * Hq
        if case["kind"] == "prompt":
            return {"bytes": 2 * rows_q + 2 * rows_kv + lse, "flops": 4 * D * pairs}
        return {"bytes": 4 * rows_q + 4 * rows_kv + lse, "flops": 14 * D * pairs}
    if case["kind"] in ("norm", "layer"):
        B, N, C, size = case["B"], case["N"], case["C"], 4 if case["dtype"] == "fp32" else 2
        kept = _ints(case["kept"])
        rows = B * N if not kept else B * kept[0] if len(kept) == 1 else sum(kept)
        params = 4 * C * (case["gate"] + 3)
        if case["kind"] == "norm":
            return {"bytes": 4 * rows * C * size + params, "flops": 12 * rows * C}
        return {"bytes": (7 * rows + B * N) * C * size + 2 * params, "flops": 40 * rows * C}
    sizes, dtypes = _ints(case["sizes"]), case["dtypes"].split(",")
    held = sum(n * (4 if dtypes[i % len(dtypes)] == "fp32" else 2) for i, n in enumerate(sizes))
    return {"bytes": 2 * held + 4, "flops": 3 * sum(sizes)}


# ---- the definitions in 64 bits, gradients by differentiating them ---------------------------------------------------------------
def _exact_attn(case, s):
    Hq, Hkv, D, T, train = case["Hq"], case["Hkv"], case["D"], s["T"], case["kind"] == "train"
    G, new = Hq // Hkv, lambda H, *more: torch.zeros((T, H, *more), dtype=torch.float64, device="cuda")  # noqa: E731
    o, lse, dq, dk, dv = new(Hq, D), new(Hq), new(Hq, D), new(Hkv, D), new(Hkv, D)
    begin = 0
    for n in _ints(case["lens"]):
        rows = slice(begin, begin + n)
        begin += n
        if n == 0:
            continue
        future = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1) if case["causal"] else None
        for h in range(Hq):
            q, k, v = (t[rows, i].double().requires_grad_(train) for t, i in ((s["q"], h), (s["k"], h // G), (s["v"], h // G)))
            scores = q @ k.T / D ** 0.5
            if future is not None:
                scores = scores.masked_fill(future, -math.inf)
            lse[rows, h] = torch.logsumexp(scores, 1).detach()
            out = torch.softmax(scores, 1) @ v
            o[rows, h] = out.detach()
            if train:
                gq, gk, gv = torch.autograd.grad(out, (q, k, v), s["d_o"][rows, h].double())
                dq[rows, h] = gq
                dk[rows, h // G] += gk
                dv[rows, h // G] += gv
    res = {"o": o, "lse": lse.T.contiguous()}
    return {**res, "dq": dq, "dk": dk, "dv": dv} if train else res


def _exact_norm(case, s):
    B, N, C, train = case["B"], case["N"], case["C"], case["kind"] == "layer"
    names = [n for n in ("x", "y", "gate", "w_post", "b_post", "w_pre", "b_pre") if s[n] is not None]
    leaf = {n: s[n].double().requires_grad_(train) for n in names}

    def norm(t, kind, w, b):
        if kind == "none":
            return t
        if kind == "layer":
            return (t - t.mean(-1, keepdim=True)) / torch.sqrt(t.var(-1, unbiased=False, keepdim=True) + EPS) * w + b
        return t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + EPS) * w

    zero = torch.zeros((B, N, C), dtype=torch.float64, device="cuda")
    out = {"h": zero.clone(), "u": zero.clone()}
    grads = {n: torch.zeros_like(t) for n, t in leaf.items()}
    kept = _ints(case["kept"])
    for b in range(B):
        m = kept[b if len(kept) > 1 else 0] if kept else N
        x = leaf["x"][b]
        if kept:
            x = x[s["sel_idx"][b if len(kept) > 1 else 0, :m].long()]
        h = case["scale"] * x
        branch = norm(leaf["y"][b, :m], case["post"], leaf.get("w_post"), leaf.get("b_post"))
        h = h + (leaf["gate"][b if case["gate"] > 1 else 0] * branch if case["gate"] else branch)
        u = norm(h, case["pre"], leaf["w_pre"], leaf.get("b_pre"))
        out["h"][b, :m], out["u"][b, :m] = h.detach(), u.detach()
        if train:
            for n, t in zip(names, torch.autograd.grad((h, u), list(leaf.values()), (s["d_h"][b, :m].double(), s["d_u"][b, :m].double()))):
                grads[n] += t
    if train:
        out |= {"dx": grads["x"], "dy": grads["y"], **{"d_" + n: grads[n] for n in names if n not in ("x", "y")}}
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("prompt", "train"):
        return _exact_attn(case, s)
    if case["kind"] in ("norm", "layer"):
        return _exact_norm(case, s)
    total = 0.0
    for g in s["grads"]:
        total += float((g.double() ** 2).sum())
    norm = math.sqrt(total)
    factor = min(1.0, s["max_norm"] / (norm + 1e-6))
    return {"norm": torch.tensor([norm], dtype=torch.float64, device="cuda"), "grads": [g.double() * factor for g in s["flat"].values()]}
