"""The work of the operators at the ends and in the middle of a model on token sets: embeddings of token indices, the feed-forward's activation with an 8-bit checkpoint, and the loss over
a vocabulary, with their gradients.

Kinds of a case (`kind`), each one pass through the public entry points of paper_2501_14183_b200.binding:

  lookup   out[t] = scale table[idx[t]], zeros where idx[t] < 0: vardrop_embed_fwd
  embed    the same with its backward pass, d_table[v] = scale sum of d_out[t] over idx[t] = v: vardrop_embed_fwd -> vardrop_embed_bwd
  batches  the backward pass of two micro-batches, the second added to the first: vardrop_embed_bwd twice
  act      y = f(a) or f(a) o b, forward alone: vardrop_act_fwd
  ffn      the same in training: the forward pass leaves a (and b) in 8 bits, the backward pass works from these: vardrop_act_fwd -> vardrop_act_bwd
  loss     loss[t] = logsumexp_v(scale h[t] . w[v]) - scale h[t] . w[label[t]], 0 where label[t] < 0, forward alone: vardrop_loss_fwd
  step     the same with the gradients of h and w: vardrop_loss_fwd -> vardrop_loss_bwd

Ranges: 1 to 2^17 tokens, tables of 1 to 2^17 rows of 1 to 4096 channels, bf16, fp16 or fp32 and mixed, indices even, skewed or with gaps; activations of 1 to 64 instances of 1 to 8192 tokens of
1 to 8192 channels, odd ones among them, with or without a selection of the tokens, as tensors of their own or as halves of one; losses of 1 to 16384 tokens over 2 to 2^17 classes with 8 to
4096 channels, with or without tokens that have no label.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ACTS = {"relu": 0, "gelu": 1, "silu": 2}
BLOCK = 32          # values of a row that share a scale in 8 bits


def _embed(name, kind, T, V, C, table_type, out_type, spread, gaps=0.0, scale=1.0):
    return dict(name=name, kind=kind, T=T, V=V, C=C, table_type=table_type, out_type=out_type, spread=spread, gaps=gaps, scale=scale)


def _act(name, kind, B, N, C, dtype, act, gated, fused=False, kept=""):
    return dict(name=name, kind=kind, B=B, N=N, C=C, dtype=dtype, act=act, gated=gated, fused=fused, kept=kept)


def _loss(name, kind, T, V, C, dtype, gaps=0.0, scale=1.0):
    return dict(name=name, kind=kind, T=T, V=V, C=C, dtype=dtype, gaps=gaps, scale=scale)


def listed():
    return [
        # the tokens of a few requests on their way into a model: latency is all there is
        _embed("few tokens", "lookup", 16, 32768, 2048, "bf16", "bf16", "skewed", 0.0, math.sqrt(2048.0)),
        # an embedding of its own for each variate, added to the kept tokens of every instance: indices as the selections give them, -1 behind the last kept one
        _embed("variates of kept tokens", "embed", 32 * 321, 321, 512, "fp32", "bf16", "even", 0.63),
        # a long batch over a vocabulary of odd size, a few tokens everywhere and most of them rare
        _embed("skewed tokens", "embed", 65536, 50001, 1024, "bf16", "bf16", "skewed", 0.0, 32.0),
        # gradients of two micro-batches in one table, fp32 weights under a 16-bit stream
        _embed("two micro-batches", "batches", 16384, 131072, 512, "fp32", "bf16", "skewed", 0.05),
        # inference of a gated feed-forward block on one instance's variates, both branches from one projection
        _act("one instance", "act", 1, 321, 2048, "bf16", "silu", True, fused=True),
        # training on the kept tokens of road-traffic sensors, one selection for the batch
        _act("kept tokens", "ffn", 32, 862, 2048, "bf16", "gelu", False, kept="172"),
        # fp32 training with a channel count that no vector width divides
        _act("fp32, odd width", "ffn", 16, 321, 2051, "fp32", "gelu", False),
        # the widest activations of a training step: larger than L2
        _act("wide gated block", "ffn", 8, 8192, 5632, "bf16", "silu", True, fused=True),
        # classes of one small batch: latency
        _loss("few classes", "loss", 32, 1000, 512, "bf16"),
        # values cut into bins, a label for the kept variates alone
        _loss("bins of kept tokens", "step", 32 * 321, 4096, 512, "bf16", 0.63),
        # an odd vocabulary in fp16, ragged batch, a third of it without labels
        _loss("odd vocabulary", "step", 3001, 50001, 1024, "fp16", 0.33),
        # the largest: a long batch over a large vocabulary
        _loss("large vocabulary", "step", 8192, 131072, 2048, "bf16", 0.0, 1.0),
    ]


MOST_PRODUCTS = 8192 * 131072 * 2048         # of the largest listed loss
MOST_ROWS = 65536 * 5632                     # elements of the widest activation
MOST_TABLE = 131072 * 1024


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lookup", "embed", "embed", "batches", "act", "ffn", "ffn", "loss", "step", "step", "step"])
    if kind in ("lookup", "embed", "batches"):
        V, C = _log(rng, 2, 1 << 17), rng.choice([_log(rng, 2, 4096), 8 * _log(rng, 1, 512)])
        V = max(1, min(V, MOST_TABLE // C))
        T = max(1, min(_log(rng, 2, 1 << 17), MOST_TABLE // C))
        table = rng.choice(["bf16", "fp16", "fp32", "fp32"])
        return _embed("", kind, T, V, C, table, rng.choice([table, table, "bf16"]), rng.choice(["even", "skewed", "skewed"]), rng.choice([0.0, 0.0, 0.1, 0.6]), rng.choice([1.0, math.sqrt(C)]))
    if kind in ("act", "ffn"):
        B, C = _log(rng, 1, 64), rng.choice([_log(rng, 2, 8192), 8 * _log(rng, 1, 1024)])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        N = max(1, min(_log(rng, 1, 8192), MOST_ROWS // (B * C) // (2 if dtype == "fp32" else 1)))
        kept = ",".join(str(rng.randint(1, N)) for _ in range(rng.choice([0, 1, B])))
        return _act("", kind, B, N, C, dtype, rng.choice(["relu", "gelu", "silu"]), rng.random() < 0.5, rng.random() < 0.5 and C % 8 == 0, kept)
    C = 8 * _log(rng, 1, 512)
    V, T = _log(rng, 2, 1 << 17), _log(rng, 1, 16384)
    while T * V * C > MOST_PRODUCTS or T * V > 8192 * 131072:
        T = (T + 1) // 2
    return _loss("", kind, T, V, C, rng.choice(["bf16", "bf16", "fp16"]), rng.choice([0.0, 0.0, 0.2, 0.7]), rng.choice([1.0, 1.0, 0.5]))


def _ints(text):
    return [int(t) for t in text.split(",")] if text else []


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _tokens(g, T, V, spread, gaps):
    """Indices of T tokens in [0, V), evenly spread or with frequencies that fall like one over the rank; a share of them -1. One token at least has an index."""
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    idx = (u * V if spread == "even" else torch.exp(u * math.log(V + 1)) - 1).long().clamp(0, V - 1)
    if gaps:
        idx = torch.where(torch.rand(T, generator=g, device="cuda") < gaps, -1, idx)
        idx[0] = idx[0].clamp_min(0)
    return idx.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    if case["kind"] in ("lookup", "embed", "batches"):
        T, V, C = case["T"], case["V"], case["C"]
        if case["kind"] != "batches":
            s["table"] = _normal(g, (V, C), 1 / case["scale"], TYPES[case["table_type"]])
        s["idx"] = [_tokens(g, T, V, case["spread"], case["gaps"]) for _ in range(2 if case["kind"] == "batches" else 1)]
        if case["kind"] != "lookup":
            s["d_out"] = [_normal(g, (T, C), 1.0, TYPES[case["out_type"]]) for _ in s["idx"]]
        return s
    if case["kind"] in ("act", "ffn"):
        B, N, C, dt = case["B"], case["N"], case["C"], TYPES[case["dtype"]]
        kept = _ints(case["kept"])
        s["n_sel"] = torch.tensor(kept, dtype=torch.int32, device="cuda") if kept else None
        if case["gated"] and case["fused"]:
            both = _normal(g, (B, N, 2 * C), 1.5, dt)
            s["a"], s["b"] = both[..., :C], both[..., C:]
        else:
            s["a"], s["b"] = _normal(g, (B, N, C), 1.5, dt), _normal(g, (B, N, C), 1.0, dt) if case["gated"] else None
        s["d_y"] = _normal(g, (B, N, C), 1.0, dt) if case["kind"] == "ffn" else None
        return s
    T, V, C, dt = case["T"], case["V"], case["C"], TYPES[case["dtype"]]
    s["h"], s["w"] = _normal(g, (T, C), 1.0, dt), _normal(g, (V, C), 1.5 / math.sqrt(C), dt)
    s["labels"] = _tokens(g, T, V, "skewed", case["gaps"])
    weight = 0.5 + torch.rand(T, generator=g, device="cuda")            # the mean over labelled tokens, some of them weighted higher
    s["d_loss"] = weight / (s["labels"] >= 0).sum() if case["kind"] == "step" else None
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------------
def _embed_plain(s):
    V, C, table = s["V"], s["C"], TYPES[s["table_type"]]
    res = {}
    if s["kind"] != "batches":
        idx = s["idx"][0].long()
        rows = s["table"][idx.clamp_min(0)].float() * s["scale"]
        res["out"] = torch.where(idx[:, None] >= 0, rows, 0).to(TYPES[s["out_type"]])
    if s["kind"] != "lookup":
        d_table = None
        for idx, d_out in zip(s["idx"], s["d_out"]):
            total = torch.zeros((V + 1, C), dtype=torch.float64, device="cuda")         # row V: tokens without an index
            total.index_add_(0, torch.where(idx < 0, V, idx).long(), d_out.double())
            total = total[:V] * s["scale"]
            d_table = (total if d_table is None else d_table.double() + total).float().to(table)
        res["d_table"] = d_table
    return res


def _eight_bits(x):
    """x [..., C] in 32 bits as it comes back from 8: blocks of a row share a power of two that takes the largest of them to 448 at most, each value is an e4m3 of that scale."""
    C = x.shape[-1]
    blocks = torch.nn.functional.pad(x, (0, -C % BLOCK)).unflatten(-1, (-1, BLOCK))
    part, power = torch.frexp(blocks.abs().amax(-1, keepdim=True))
    power = (power - torch.where(part > 0.875, 8, 9)).clamp(-127, 127)
    stored = torch.ldexp(blocks, -power).to(torch.float8_e4m3fn)
    return torch.ldexp(stored.float(), power).flatten(-2)[..., :C]


def _act_of(a, act):
    if act == "relu":
        return a.clamp_min(0)
    return a / (1 + torch.exp(-a)) if act == "silu" else a * 0.5 * torch.erfc(a * -math.sqrt(0.5))


def _act_slope(a, act):
    if act == "relu":
        return (a > 0).float()
    if act == "silu":
        p = 1 / (1 + torch.exp(-a))
        return p * (1 + a * (1 - p))
    return 0.5 * torch.erfc(a * -math.sqrt(0.5)) + a * torch.exp(a * a * -0.5) * (1 / math.sqrt(2 * math.pi))


def _act_plain(s):
    B, N, dt, act = s["B"], s["N"], TYPES[s["dtype"]], s["act"]
    live = torch.ones((B, N, 1), dtype=torch.bool, device="cuda")
    if s["kept"]:
        live = (torch.arange(N, device="cuda") < s["n_sel"][:, None]).expand(B, N)[..., None]
    a, b = s["a"].float(), s["b"].float() if s["gated"] else None
    y = _act_of(a, act)
    res = {"y": torch.where(live, y * b if s["gated"] else y, 0).to(dt)}
    if s["kind"] == "act":
        return res
    del y
    a, b = _eight_bits(a), _eight_bits(b) if s["gated"] else None
    d_y, f = s["d_y"].float(), _act_of(a, act)
    res["d_a"] = torch.where(live, d_y * (b if s["gated"] else 1) * _act_slope(a, act), 0).to(dt)
    if s["gated"]:
        res["d_b"] = torch.where(live, d_y * f, 0).to(dt)
    res["y_again"] = torch.where(live, f * b if s["gated"] else f, 0).to(dt)
    return res


def _loss_plain(s):
    T, scale = s["T"], s["scale"]
    at, labelled = s["labels"].long().clamp_min(0), s["labels"] >= 0
    h, w = torch.where(labelled[:, None], s["h"].float(), 0), s["w"].float()
    logits = torch.matmul(h, w.t()).mul_(scale)
    top = logits.amax(1, keepdim=True)
    target = logits.gather(1, at[:, None])
    p = logits.sub_(top).exp_()
    total = p.sum(1, keepdim=True)
    lse = top + total.log()
    res = {"loss": torch.where(labelled, (lse - target)[:, 0], 0), "lse": torch.where(labelled, lse[:, 0], 0)}
    if s["kind"] == "loss":
        return res
    p.div_(total)
    p[torch.arange(T, device="cuda"), at] -= 1
    p.mul_(torch.where(labelled, s["d_loss"] * scale, 0)[:, None])
    return {**res, "d_h": torch.matmul(p, w).to(s["h"].dtype), "d_w": torch.matmul(p.t(), h).to(s["w"].dtype)}


# ---- the framework's calls -------------------------------------------------------------------------------------------------
def _embed_own(s):
    from paper_2501_14183_b200 import binding as vd
    T, V, C, kind = s["T"], s["V"], s["C"], s["kind"]
    if "cfg" not in s:              # what a training program sets up once: configurations, outputs, workspace
        types = vd.DTYPES[TYPES[s["table_type"]]], vd.DTYPES[TYPES[s["out_type"]]]
        s["cfg"], s["more"] = (vd.EmbedCfg(T, V, C, *types, accumulate, s["scale"]) for accumulate in (0, 1))
        s["ws"] = vd.alloc_ws(vd.vardrop_embed_workspace_bytes(s["cfg"]))
        if kind != "batches":
            s["rows"] = torch.empty((T, C), dtype=TYPES[s["out_type"]], device="cuda")
        if kind != "lookup":
            s["d_table"] = torch.empty((V, C), dtype=TYPES[s["table_type"]], device="cuda")
    res = {}
    if kind != "batches":
        vd.vardrop_embed_fwd(s["table"], s["idx"][0], s["cfg"], s["rows"], s["ws"])
        res["out"] = s["rows"]
    if kind != "lookup":
        vd.vardrop_embed_bwd(s["d_out"][0], s["idx"][0], s["cfg"], s["d_table"], s["ws"])
        res["d_table"] = s["d_table"]
    if kind == "batches":
        vd.vardrop_embed_bwd(s["d_out"][1], s["idx"][1], s["more"], s["d_table"], s["ws"])
    return res


def _act_own(s):
    from paper_2501_14183_b200 import binding as vd
    train = s["kind"] == "ffn"
    if "cfg" not in s:
        B, N, C, dt = s["B"], s["N"], s["C"], TYPES[s["dtype"]]
        fused = s["gated"] and s["fused"]
        s["cfg"] = vd.ActCfg(B, N, C, vd.DTYPES[dt], ACTS[s["act"]], 1 if s["gated"] else 0, s["n_sel"].shape[0] if s["kept"] else 0, 2 * C if fused else 0)
        s["y"] = torch.zeros((B, N, C), dtype=dt, device="cuda")
        s["ckpt"] = None
        if train:
            s["ckpt"] = vd.alloc_act_ckpt(s["cfg"])
            s["y_again"] = torch.zeros_like(s["y"])
            if fused:
                both = torch.zeros((B, N, 2 * C), dtype=dt, device="cuda")
                s["d_a"], s["d_b"] = both[..., :C], both[..., C:]
            else:
                s["d_a"], s["d_b"] = torch.zeros_like(s["y"]), torch.zeros_like(s["y"]) if s["gated"] else None
    vd.vardrop_act_fwd(s["a"], s["b"], s["n_sel"], s["cfg"], s["y"], s["ckpt"])
    if not train:
        return {"y": s["y"]}
    vd.vardrop_act_bwd(s["d_y"], s["ckpt"], s["n_sel"], s["cfg"], s["d_a"], s["d_b"], s["y_again"])
    res = {"y": s["y"], "d_a": s["d_a"], "d_b": s["d_b"], "y_again": s["y_again"]}
    return {k: t for k, t in res.items() if t is not None}


def _loss_own(s):
    from paper_2501_14183_b200 import binding as vd
    train = s["kind"] == "step"
    if "cfg" not in s:
        T, V, C = s["T"], s["V"], s["C"]
        s["cfg"] = vd.LossCfg(T, V, C, vd.DTYPES[TYPES[s["dtype"]]], s["scale"])
        s["loss"], s["lse"] = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        s["ws"] = vd.alloc_ws(vd.vardrop_loss_workspace_bytes(s["cfg"]))
        if train:
            s["d_h"], s["d_w"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
    vd.vardrop_loss_fwd(s["h"], s["w"], s["labels"], s["cfg"], s["loss"], s["lse"], s["ws"])
    if not train:
        return {"loss": s["loss"], "lse": s["lse"]}
    vd.vardrop_loss_bwd(s["h"], s["w"], s["labels"], s["lse"], s["d_loss"], s["cfg"], s["d_h"], s["d_w"], s["ws"])
    return {"loss": s["loss"], "lse": s["lse"], "d_h": s["d_h"], "d_w": s["d_w"]}


def run(state):
    if state["kind"] in ("lookup", "embed", "batches"):
        return _embed_own(state) if own else _embed_plain(state)
    if state["kind"] in ("act", "ffn"):
        return _act_own(state) if own else _act_plain(state)
    return _loss_own(state) if own else _loss_plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------
def _size(dtype):
    return 4 if dtype == "fp32" else 2


def work(case):
    if case["kind"] in ("lookup", "embed", "batches"):
        T, V, C = case["T"], case["V"], case["C"]
        live = T * (1 - case["gaps"])
        found = V * (1 - (1 - 1 / V) ** live) if case["spread"] == "even" else min(V, live) / max(1.0, math.log(V + 1))        # rows that some token has, about
        rows, table, of_table = T * C * _size(case["out_type"]), found * C * _size(case["table_type"]), V * C * _size(case["table_type"])
        forward = rows + table + 4 * T
        back = live * C * _size(case["out_type"]) + of_table + 4 * T
        if case["kind"] == "batches":       # the second one reads and writes the rows that it has
            return {"bytes": back + live * C * _size(case["out_type"]) + 4 * T + 2 * table, "flops": 2 * live * C}
        return {"bytes": forward, "flops": T * C} if case["kind"] == "lookup" else {"bytes": forward + back, "flops": 2 * T * C}
    if case["kind"] in ("act", "ffn"):
        kept = _ints(case["kept"])
        rows = case["B"] * case["N"] if not kept else case["B"] * kept[0] if len(kept) == 1 else sum(kept)
        n, size, of = rows * case["C"], _size(case["dtype"]), 2 if case["gated"] else 1
        if case["kind"] == "act":
            return {"bytes": (of + 1) * n * size, "flops": 12 * n}
        held = of * (n + rows * -(-case["C"] // BLOCK))
        return {"bytes": (2 * of + 3) * n * size + 2 * held, "flops": 50 * n}
    T, V, C = case["T"] * (1 - case["gaps"]), case["V"], case["C"]
    rows, table = 2 * T * C, 2 * V * C
    if case["kind"] == "loss":
        return {"bytes": rows + table + 12 * case["T"], "flops": 2 * T * V * C}
    return {"bytes": 2 * (rows + table) + 2 * case["T"] * C - rows + 16 * case["T"], "flops": 6 * T * V * C}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def _exact_embed(case, s):
    V, C = case["V"], case["C"]
    res = {}
    if case["kind"] != "batches":
        weight = s["table"].double().requires_grad_(case["kind"] == "embed")
        live = torch.nonzero(s["idx"][0] >= 0)[:, 0]
        picked = weight.index_select(0, s["idx"][0][live].long()) * case["scale"]
        out = torch.zeros((case["T"], C), dtype=torch.float64, device="cuda")
        out[live] = picked.detach()
        res["out"] = out
        if case["kind"] == "embed":
            res["d_table"] = torch.autograd.grad(picked, weight, s["d_out"][0][live].double())[0]
        return res
    order = torch.cat(s["idx"]).long()
    live = order >= 0
    rows = torch.cat(s["d_out"]).double()[live] * case["scale"]
    return {"d_table": torch.zeros((V, C), dtype=torch.float64, device="cuda").scatter_add_(0, order[live][:, None].expand(-1, C), rows)}


def _held(x):
    """What 8 bits stand for, by steps: of a block's scale the smallest power of two 2^e with max <= 448 2^e, of a value the multiple of its own step that is nearest."""
    C = x.shape[-1]
    full = torch.zeros((*x.shape[:-1], -(-C // BLOCK) * BLOCK), dtype=torch.float64, device=x.device)
    full[..., :C] = x
    full = full.view(*x.shape[:-1], -1, BLOCK)
    top = full.abs().max(-1, keepdim=True).values
    e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 448))
    e = torch.where(top > 448 * torch.exp2(e), e + 1, torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e)).clamp(-127, 127)      # (the logarithm's last bit)
    v = full / torch.exp2(e)
    k = torch.floor(torch.log2(v.abs().clamp_min(1e-300)))
    k = torch.where(v.abs() >= torch.exp2(k + 1), k + 1, torch.where(v.abs() < torch.exp2(k), k - 1, k))
    step = torch.exp2(k.clamp_min(-6) - 3)
    return (torch.round(v / step) * step * torch.exp2(e)).flatten(-2)[..., :C]


def _exact_act(case, s):
    B, N, C, train = case["B"], case["N"], case["C"], case["kind"] == "ffn"
    f = {"relu": torch.nn.functional.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[case["act"]]
    kept = _ints(case["kept"])
    names = ["y"] + (["d_a"] + (["d_b"] if case["gated"] else []) + ["y_again"] if train else [])
    out = {n: torch.zeros((B, N, C), dtype=torch.float64, device="cuda") for n in names}
    for i in range(B):
        m = kept[i if len(kept) > 1 else 0] if kept else N
        a, b = s["a"][i, :m].double(), s["b"][i, :m].double() if case["gated"] else None
        out["y"][i, :m] = f(a) * b if case["gated"] else f(a)
        if not train:
            continue
        leaf = [_held(t).requires_grad_(True) for t in (a, b) if t is not None]
        again = f(leaf[0]) * leaf[1] if case["gated"] else f(leaf[0])
        out["y_again"][i, :m] = again.detach()
        for n, t in zip(("d_a", "d_b"), torch.autograd.grad(again, leaf, s["d_y"][i, :m].double())):
            out[n][i, :m] = t
    return out


def _exact_loss(case, s):
    T, V, C, train = case["T"], case["V"], case["C"], case["kind"] == "step"
    if 6.0 * T * V * C > 3e14:
        return None
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out = {"loss": new(T), "lse": new(T)}
    if train:
        out |= {"d_h": new(T, C), "d_w": new(V, C)}
    w = s["w"].double()
    for rows in torch.split(torch.nonzero(s["labels"] >= 0)[:, 0], 1024):
        h, label = s["h"][rows].double(), s["labels"][rows].long()
        logits = case["scale"] * (h @ w.T)
        out["lse"][rows] = torch.logsumexp(logits, 1)
        out["loss"][rows] = torch.nn.functional.cross_entropy(logits, label, reduction="none")
        if train:
            g = torch.softmax(logits, 1) - torch.nn.functional.one_hot(label, V)
            g *= (case["scale"] * s["d_loss"][rows].double())[:, None]
            out["d_h"][rows] = g @ w
            out["d_w"] += g.T @ h
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("lookup", "embed", "batches"):
        return _exact_embed(case, s)
    return _exact_act(case, s) if case["kind"] in ("act", "ffn") else _exact_loss(case, s)
