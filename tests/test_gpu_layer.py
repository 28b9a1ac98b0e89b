"""The operators around the attention as a training step calls them: hash and selection of every instance on its own, the residual stream of the kept tokens gathered and normed,
projections, attention over the kept sets packed one behind the other, the branch normed, gated and added, the way back, and the gradients clipped.  Against the same layer in 64 bits.

Tolerance: a tensor of 16 bits is off by at most 2^-8 of its values from being rounded, products with weights of random sign pass a relative error on as it is, and errors of different
roundings add up at most linearly.  The longest way (to dx) rounds u, q | k | v, P, o, y, h2's inputs, then dy, d_o, dS, dq | dk | dv, du, dx: at most 14 tensors."""
import math

import pytest
import torch

from paper_2501_14183_b200 import binding as vd
from paper_2501_14183_b200 import inputs

pytestmark = pytest.mark.gpu

BOUND = 14 * 2.0 ** -8
EPS = 1e-5


def rms(t, w):
    return t / torch.sqrt((t * t).mean(-1, keepdim=True) + EPS) * w


def exact_layer(x, sels, p, d_out, H, Hkv, D, causal):
    """Loss sum(out * d_out) of the layer in 64 bits, kept rows one behind the other; gradients by differentiation."""
    leaf = {n: t.double().clone().requires_grad_(True) for n, t in {**p, "x": x}.items()}
    outs = []
    for b, sel in enumerate(sels):
        xs = leaf["x"][b, sel]
        u = rms(xs, leaf["w1"])
        qkv = u @ leaf["W"]
        n = len(sel)
        q, k, v = (t.reshape(n, -1, D) for t in qkv.split([H * D, Hkv * D, Hkv * D], 1))
        k, v = (t.repeat_interleave(H // Hkv, 1) for t in (k, v))
        s = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(D)
        if causal:
            s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=s.device).triu(1), -math.inf)
        o = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v)
        outs.append(rms(xs + leaf["gate"][b] * rms(o.reshape(n, -1) @ leaf["Wo"], leaf["w2"]), leaf["w3"]))
    out = torch.cat(outs)
    grads = torch.autograd.grad(out, list(leaf.values()), d_out.double())
    return out.detach(), dict(zip(leaf, grads))


@pytest.mark.parametrize("causal,Hkv", [(0, 8), (1, 2)])
def test_a_training_step_of_a_layer_on_kept_tokens(causal, Hkv):
    B, L, H, D = 6, 96, 8, 64
    C = H * D
    w = inputs.WORKLOADS["elec"]
    windows = torch.from_numpy(inputs.make_windows(w)[:B, :321]).cuda().contiguous()
    N = windows.shape[1]
    hcfg, scfg = vd.HashCfg(B, N, L, 3, 0, 0, 1), vd.SelectCfg(B, N, 0, 0.3, 5, 1)
    keys, freqs, _ = vd.alloc_hash_outputs(hcfg)
    vd.vardrop_hash(windows, hcfg, keys, freqs, None, vd.alloc_ws(vd.vardrop_hash_workspace_bytes(hcfg)))
    sel = vd.alloc_select_outputs(scfg)
    vd.vardrop_select(keys, scfg, *(sel[n] for n in ("group_id", "group_offsets", "members", "n_groups", "sel_idx", "n_sel", "inv_idx")), vd.alloc_ws(vd.vardrop_select_workspace_bytes(scfg)))
    counts = sel["n_sel"].tolist()
    T = sum(counts)
    sels = [sel["sel_idx"][b, :m].long() for b, m in enumerate(counts)]
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    cu[1:] = torch.cumsum(sel["n_sel"], 0)
    pack = torch.cat([b * N + torch.arange(m, device="cuda") for b, m in enumerate(counts)])        # rows of [B, N] that hold kept tokens

    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda") * std)  # noqa: E731
    x = rand(B, N, C).bfloat16()
    p = dict(W=rand(C, (H + 2 * Hkv) * D, std=C ** -0.5).bfloat16(), Wo=rand(C, C, std=C ** -0.5).bfloat16(), w1=1 + 0.1 * rand(C), w2=1 + 0.1 * rand(C), w3=1 + 0.1 * rand(C), gate=rand(B, C))
    d_out = rand(T, C).bfloat16()

    def padded(rows):                                       # [T, C] -> [B, N, C], anything behind the kept rows
        out = torch.full((B * N, rows.shape[1]), float("nan"), dtype=rows.dtype, device="cuda")
        out[pack] = rows
        return out.view(B, N, -1)

    new = lambda *s: torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    # ---- forward
    n1 = vd.NormCfg(B, N, C, 0, vd.NORM_RMS, 0, 0, B, 1.0, EPS)
    xs, u1, st1 = new(B, N, C), new(B, N, C), torch.empty(B, N, 4, device="cuda")
    vd.vardrop_norm_fwd(x, None, None, None, None, p["w1"], None, sel["sel_idx"], sel["n_sel"], n1, xs, u1, st1)
    u1p = u1.view(B * N, C)[pack]
    qkv = (u1p @ p["W"]).view(T, H + 2 * Hkv, D)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    sT = (H + 2 * Hkv) * D
    pc = vd.PackedCfg(B, T, H, Hkv, D, 0.0, causal, sT, D, sT, D)
    plan, ws = vd.alloc_packed_plan(pc), vd.alloc_ws(vd.vardrop_attn_packed_workspace_bytes(pc))
    o, lse = new(T, H, D), torch.empty(H, T, device="cuda")
    vd.vardrop_packed_plan(cu, pc, plan)
    vd.vardrop_attn_packed_fwd(q, k, v, plan, pc, o, lse, ws)
    y = padded(o.view(T, C) @ p["Wo"])
    n2 = vd.NormCfg(B, N, C, 0, vd.NORM_RMS, vd.NORM_RMS, B, B, 1.0, EPS)
    h2, u2, st2 = new(B, N, C), new(B, N, C), torch.empty(B, N, 4, device="cuda")
    vd.vardrop_norm_fwd(x, y, p["gate"], p["w2"], None, p["w3"], None, sel["sel_idx"], sel["n_sel"], n2, h2, u2, st2)
    out = u2.view(B * N, C)[pack]
    # ---- backward
    grads = {n: torch.empty_like(p[n]) for n in ("w1", "w2", "w3", "gate")}
    nws = vd.alloc_ws(max(vd.vardrop_norm_workspace_bytes(n1), vd.vardrop_norm_workspace_bytes(n2)))
    dx2, dy = new(B, N, C), new(B, N, C)
    vd.vardrop_norm_bwd(x, y, p["gate"], p["w2"], None, p["w3"], sel["sel_idx"], sel["n_sel"], sel["inv_idx"], st2, None, padded(d_out), n2, dx2, dy, grads["gate"], grads["w2"], None,
                        grads["w3"], None, nws)
    dyp = dy.view(B * N, C)[pack]
    d_o = (dyp @ p["Wo"].t()).view(T, H, D).contiguous()
    grads["Wo"] = o.view(T, C).t() @ dyp
    dq, dk, dv = new(T, H, D), new(T, Hkv, D), new(T, Hkv, D)
    vd.vardrop_attn_packed_bwd(q, k, v, o, lse, d_o, plan, pc, dq, dk, dv, ws)
    dqkv = torch.cat([dq, dk, dv], 1).view(T, -1)
    grads["W"] = u1p.t() @ dqkv
    dx1 = new(B, N, C)
    vd.vardrop_norm_bwd(x, None, None, None, None, p["w1"], sel["sel_idx"], sel["n_sel"], sel["inv_idx"], st1, None, padded(dqkv @ p["W"].t()), n1, dx1, None, None, None, None, grads["w1"], None,
                        nws)
    grads["x"] = dx1.float() + dx2.float()
    # ---- the step's end
    names = ["W", "Wo", "w1", "w2", "w3", "gate"]
    before = {n: grads[n].clone() for n in names}
    norm, cws = torch.empty(1, device="cuda"), vd.alloc_ws(vd.vardrop_grad_clip_workspace_bytes())
    vd.vardrop_grad_clip([grads[n] for n in names], vd.ClipCfg(1.0, 1e-6), None, norm, cws)
    torch.cuda.synchronize()
    for t in (plan, ws, nws, cws):
        assert vd.ws_status(t) == vd.OK

    want, exact = exact_layer(x, sels, p, d_out, H, Hkv, D, causal)
    near = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert near(out, want) <= BOUND
    for n in names:
        assert near(before[n], exact[n]) <= BOUND, n
    assert near(grads["x"], exact["x"]) <= BOUND
    dropped = sel["inv_idx"] < 0
    assert not grads["x"][dropped].any()
    total = math.sqrt(sum(float((t.double() ** 2).sum()) for t in before.values()))
    assert abs(float(norm.item()) - total) <= 2.0 ** -23 * total and total > 1.0
    for n in names:
        assert near(grads[n], before[n].double() / (total + 1e-6)) <= (2.0 ** -8 if grads[n].dtype == torch.bfloat16 else 1e-6), n
