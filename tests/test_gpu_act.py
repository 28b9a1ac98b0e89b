"""vardrop_act_fwd / vardrop_act_bwd against the formulas in 64 bits, the checkpoint against its definition."""
import math

import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

BF, HF, FP = torch.bfloat16, torch.float16, torch.float32
BLOCK = 32
RELU, GELU, SILU = vd.ACT_RELU, vd.ACT_GELU, vd.ACT_SILU


def held(x, dtype=FP):
    """Scales' exponents and the values that 8 bits stand for, by the definition, in 64 bits.  2^16 and 2^128 are no values of their types: 15/16 of them stands for what rounds there."""
    C = x.shape[-1]
    most = 15 * 2.0 ** (12 if dtype == HF else 124)
    full = torch.zeros((*x.shape[:-1], -(-C // BLOCK) * BLOCK), dtype=torch.float64, device=x.device)
    full[..., :C] = x
    full = full.unflatten(-1, (-1, BLOCK))
    fine = full.isfinite()
    top = torch.where(fine, full, 0).abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -127.0)
    for k in range(-126, 129):                  # the smallest power of two that takes the largest value to 448 at most
        e = torch.where(top > 448 * 2.0 ** (k - 1), float(k), e)
    v = torch.where(fine, full, 0).clamp(-most, most) / torch.exp2(e)
    power = torch.full_like(v, -6.0)
    for k in range(-5, 9):
        power = torch.where(v.abs() >= 2.0 ** k, float(k), power)
    step = torch.exp2(power - 3)
    out = torch.where(fine, torch.round(v / step) * step * torch.exp2(e), float("nan"))
    return e[..., 0], out.flatten(-2)[..., :C]


def formulas(a, kind):
    """f(a), f'(a), and the errors that fp32 arithmetic may leave in them: exp to (2 + 1.2 |x|) steps, a quotient to 2, erfc to 4 and through its rounded argument by |a| times the density."""
    u = 2.0 ** -23
    if kind == RELU:
        return a.clamp_min(0), (a > 0).double(), 0 * a, 0 * a
    if kind == SILU:
        p = 1 / (1 + torch.exp(-a))
        f = a * p
        return f, p + f * (1 - p), f.abs() * (8 + 1.2 * a.abs()) * u, (p + f.abs()) * (12 + 2.4 * a.abs()) * u
    p, density = 0.5 * torch.erfc(-a / math.sqrt(2)), torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    ep = (12 * p + 2 * (a * density).abs()) * u
    return a * p, p + a * density, a.abs() * ep + (a * p).abs() * u, ep + (a * density).abs() * (12 + a * a) * u


def near(got, want, error, dtype):
    info = torch.finfo(dtype)
    bound = error + (want.abs() + error) * info.eps / 2 + info.smallest_normal * info.eps / 2
    # the least normal value of fp32 is where its products end
    bad = (got.double() - want).abs() > bound + 2.0 ** -126
    assert not bool((bad | (got.isnan() != want.isnan())).any()), float(((got.double() - want).abs() / bound).nan_to_num().max())


def make(B, N, C, dtype, gated, fused=False, std=1.5, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: (torch.randn(*s, generator=g, device="cuda") * std).to(dtype)  # noqa: E731
    if fused:
        both = rand(B, N, 2 * C)
        return both[..., :C], both[..., C:]
    return rand(B, N, C), rand(B, N, C) if gated else None


def check(B, N, C, dtype, kind, gated, fused=False, kept=None, std=1.5, inputs=None, seed=0):
    a, b = inputs or make(B, N, C, dtype, gated, fused, std, seed)
    d_y = make(B, N, C, dtype, False, seed=seed + 1, std=1.0)[0]
    n_sel = None if kept is None else torch.tensor(kept, dtype=torch.int32, device="cuda")
    cfg = vd.ActCfg(B, N, C, vd.DTYPES[dtype], kind, int(gated), 0 if kept is None else len(kept), 2 * C if fused else 0)
    live = torch.ones((B, N), dtype=torch.bool, device="cuda")
    if kept is not None:
        live = (torch.arange(N, device="cuda") < n_sel[:, None]).expand(B, N)
    new = lambda: torch.full((B, N, C), 7.0, dtype=dtype, device="cuda")  # noqa: E731
    y, plain, again, ckpt = new(), new(), new(), vd.alloc_act_ckpt(cfg)
    ckpt.fill_(0xA5)
    if fused:
        both = torch.full((B, N, 2 * C), 7.0, dtype=dtype, device="cuda")
        d_a, d_b = both[..., :C], both[..., C:]
    else:
        d_a, d_b = new(), new() if gated else None
    vd.vardrop_act_fwd(a, b, n_sel, cfg, y, ckpt)
    vd.vardrop_act_fwd(a, b, n_sel, cfg, plain, None)
    vd.vardrop_act_bwd(d_y, ckpt, n_sel, cfg, d_a, d_b, again)
    without = new()
    vd.vardrop_act_bwd(d_y, ckpt, n_sel, cfg, without, new() if gated else None, None) if not fused else None
    torch.cuda.synchronize()
    assert torch.equal(y.nan_to_num(1e4), plain.nan_to_num(1e4)) and (fused or torch.equal(without.nan_to_num(1e4), d_a.nan_to_num(1e4)))
    for t in (y, again, d_a) + ((d_b,) if gated else ()):                     # rows that are not kept stay as they were
        assert bool((t[~live] == 7.0).all())
    # the checkpoint
    blocks, rows, halves = -(-C // BLOCK), B * N, 2 if gated else 1
    at = -(-halves * rows * C // 256) * 256
    codes = ckpt[:halves * rows * C].view(halves, B, N, C)
    scales = ckpt[at:at + halves * rows * blocks].view(halves, B, N, blocks)
    kept_values = []
    for h, t in enumerate((a, b)[:halves]):
        e, want = held(t.double(), dtype)
        assert torch.equal(scales[h][live].double() - 127, e[live])
        got = codes[h].view(torch.float8_e4m3fn).double() * torch.exp2(scales[h].double() - 127).repeat_interleave(BLOCK, -1)[..., :C]
        assert torch.equal(got[live].nan_to_num(12345.0), want[live].nan_to_num(12345.0))
        size = torch.exp2(scales[h].double() - 127).repeat_interleave(BLOCK, -1)[..., :C]
        bound = torch.maximum(t.double().abs() * 2.0 ** -4, size * 2.0 ** -10)
        assert bool(((got - t.double()).abs() <= bound)[live & t.isfinite().all(-1)].all())
        kept_values.append(want)
    # the results
    va, vb = a.double(), b.double() if gated else torch.ones_like(a, dtype=torch.float64)
    f, _, ef, _ = formulas(va, kind)
    u = 2.0 ** -23
    near(y[live], (f * vb)[live], (ef * vb.abs() + (f * vb).abs() * u)[live], dtype)
    ha, hb = kept_values[0], kept_values[1] if gated else torch.ones_like(va)
    f, slope, ef, es = formulas(ha, kind)
    dy = d_y.double()
    near(again[live], (f * hb)[live], (ef * hb.abs() + (f * hb).abs() * u)[live], dtype)
    near(d_a[live], (dy * hb * slope)[live], ((dy * hb).abs() * (es + slope.abs() * 2 * u))[live], dtype)
    if gated:
        near(d_b[live], (dy * f)[live], (dy.abs() * (ef + f.abs() * u))[live], dtype)


@pytest.mark.parametrize("dtype", [BF, HF, FP])
@pytest.mark.parametrize("kind", [RELU, GELU, SILU])
@pytest.mark.parametrize("gated,fused", [(False, False), (True, False), (True, True)])
def test_types_kinds_and_gates(dtype, kind, gated, fused):
    check(3, 37, 264, dtype, kind, gated, fused)
    if not fused:
        check(3, 7, 45, dtype, kind, gated)


@pytest.mark.parametrize("C", [1, 7, 8, 31, 32, 33, 40, 63, 64, 248, 255, 256, 257, 2048, 2051, 5632])
@pytest.mark.parametrize("N", [1, 3, 130])
def test_widths(C, N):
    check(2, N, C, BF, SILU, True)
    check(2, N, C, FP, GELU, False)


def test_more_instances_than_a_grid_has_rows():
    B = 70001
    kept = torch.randint(0, 3, (B,)).tolist()
    check(B, 2, 8, BF, SILU, True, kept=kept)
    check(B, 1, 3, FP, RELU, False)


@pytest.mark.parametrize("C,stride", [(45, 48), (45, 104), (40, 48), (264, 512)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_with_gaps(C, stride, dtype):
    """Rows further apart than they are long, in tensors of their own and in one for both branches."""
    B, N = 3, 20
    both = torch.full((B, N, 2 * stride), 5.0, dtype=dtype, device="cuda")
    a, b = make(B, N, C, dtype, True)
    d_y = make(B, N, C, dtype, False, seed=9)[0]
    wide = vd.ActCfg(B, N, C, vd.DTYPES[dtype], SILU, 1, 0, 2 * stride)
    va, vb = both[..., :C], both[..., stride:stride + C]
    va.copy_(a)
    vb.copy_(b)
    grads = torch.full_like(both, 6.0)
    y, again, ckpt = torch.empty_like(a), torch.empty_like(a), vd.alloc_act_ckpt(wide)
    vd.vardrop_act_fwd(va, vb, None, wide, y, ckpt)
    vd.vardrop_act_bwd(d_y, ckpt, None, wide, grads[..., :C], grads[..., stride:stride + C], again)
    plain = vd.ActCfg(B, N, C, vd.DTYPES[dtype], SILU, 1, 0, 0)
    want = [torch.empty_like(a) for _ in range(4)]
    other = vd.alloc_act_ckpt(plain)
    vd.vardrop_act_fwd(a, b, None, plain, want[0], other)
    vd.vardrop_act_bwd(d_y, other, None, plain, want[1], want[2], want[3])
    assert all(torch.equal(x, z) for x, z in zip((y, grads[..., :C], grads[..., stride:stride + C], again), want))
    assert bool((grads[..., C:stride] == 6.0).all()) and bool((grads[..., stride + C:] == 6.0).all())


@pytest.mark.parametrize("kept", [[0], [1], [29], [40], [0, 40, 7, 1, 39], [0, 0, 0, 0, 0]])
def test_kept_rows(kept):
    check(5, 40, 72, BF, GELU, True, kept=kept)
    check(5, 40, 35, HF, RELU, False, kept=kept)


def test_rows_enough_for_several_pieces_a_warp():
    check(4, 1500, 2304, BF, SILU, True, fused=True, kept=[700])
    check(40, 300, 515, BF, GELU, False)


@pytest.mark.parametrize("dtype,std", [(BF, 1e-30), (BF, 1e30), (FP, 1e-36), (FP, 3e37), (HF, 1e-6), (HF, 2e4), (BF, 30.0), (FP, 30.0)])
def test_magnitudes(dtype, std):
    """Scales at both ends of their range, values far out on both sides of the function."""
    for kind in (RELU, GELU, SILU):
        a = make(2, 50, 96, dtype, False, std=std)[0].clamp(-torch.finfo(dtype).max, torch.finfo(dtype).max)
        check(2, 50, 96, dtype, kind, False, inputs=(a, None))


def test_borders_between_codes():
    """Values half way between two codes, the largest of a block at and next to where its scale changes, zeros and blocks of nothing else."""
    codes = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).float()
    ties = torch.cat([codes, (codes[1:] + codes[:-1]) / 2, -(codes[1:] + codes[:-1]) / 2, torch.zeros(3, device="cuda")])
    row = torch.zeros((len(ties) // 31 + 1, BLOCK), device="cuda")
    flat = torch.zeros(row.shape[0] * 31, device="cuda")
    flat[:len(ties)] = ties
    row[:, 1:] = flat.view(-1, 31)
    row[:, 0] = 448.0                           # holds the scale at one
    edge = torch.tensor([448.0, 449.0, 447.9999, 224.0, 224.0001, 512.0, 256.0, 1.0, 0.0], device="cuda")
    other = torch.zeros((len(edge), BLOCK), device="cuda")
    other[:, 5] = edge
    other[:, 9] = 1.0
    other[-1] = 0.0
    x = torch.cat([row, other]).view(1, -1, BLOCK)
    for scale in (1.0, 2.0 ** -60, 2.0 ** 90):
        check(1, x.shape[1], BLOCK, FP, RELU, False, inputs=(x * scale, None))


def test_values_that_are_not_finite_stay_where_they_are():
    a, b = make(1, 6, 70, FP, True)
    a[0, 1, 3], a[0, 1, 40], a[0, 2, 69] = float("nan"), float("inf"), float("-inf")
    b[0, 4, 0] = float("nan")
    a[0, 5] = float("nan")
    cfg = vd.ActCfg(1, 6, 70, vd.DTYPES[FP], RELU, 1, 0, 0)
    y, ckpt, d_a, d_b = torch.empty_like(a), vd.alloc_act_ckpt(cfg), torch.empty_like(a), torch.empty_like(a)
    vd.vardrop_act_fwd(a, b, None, cfg, y, ckpt)
    vd.vardrop_act_bwd(torch.ones_like(a), ckpt, None, cfg, d_a, d_b, None)
    assert torch.equal(d_a.isnan(), ~(a.isfinite() & b.isfinite())) and torch.equal(d_b.isnan(), ~a.isfinite())
    ea, wa = held(a.double())
    assert torch.equal(d_b.double().nan_to_num(9.0), torch.where(wa.isnan(), wa, wa.clamp_min(0)).nan_to_num(9.0))


def test_in_place():
    for dtype, C in ((BF, 264), (FP, 45)):
        a, b = make(3, 50, C, dtype, True)
        d_y = make(3, 50, C, dtype, False, seed=5)[0]
        cfg = vd.ActCfg(3, 50, C, vd.DTYPES[dtype], SILU, 1, 0, 0)
        ckpt = vd.alloc_act_ckpt(cfg)
        y, d_a, d_b, again = (torch.empty_like(a) for _ in range(4))
        vd.vardrop_act_fwd(a, b, None, cfg, y, ckpt)
        vd.vardrop_act_bwd(d_y, ckpt, None, cfg, d_a, d_b, again)
        kept = ckpt.clone()
        vd.vardrop_act_fwd(a, b, None, cfg, a, ckpt)
        vd.vardrop_act_bwd(d_y, ckpt, None, cfg, d_y, b, a.clone())
        torch.cuda.synchronize()
        assert torch.equal(a, y) and torch.equal(kept, ckpt) and torch.equal(d_y, d_a) and torch.equal(b, d_b)


def test_gradient_against_differences():
    """Along the values that the checkpoint stands for: they are what the backward pass differentiates at."""
    for kind in (GELU, SILU):
        a, b = make(1, 8, 64, FP, True)
        a, b = held(a.double())[1].float(), held(b.double())[1].float()
        cfg = vd.ActCfg(1, 8, 64, vd.DTYPES[FP], kind, 1, 0, 0)
        ckpt, d_a, d_b, y, lo, hi = vd.alloc_act_ckpt(cfg), *(torch.empty_like(a) for _ in range(5))
        vd.vardrop_act_fwd(a, b, None, cfg, y, ckpt)
        vd.vardrop_act_bwd(torch.ones_like(a), ckpt, None, cfg, d_a, d_b, None)
        h = 2.0 ** -7                           # third derivatives of both functions stay below 1.2: off by h^2 / 6 of that, and by roundings of y over 2 h
        for t, d, other in ((a, d_a, b), (b, d_b, a)):
            near_ = (a + h, b) if t is a else (a, b + h)
            far = (a - h, b) if t is a else (a, b - h)
            vd.vardrop_act_fwd(*near_, None, cfg, hi, None)
            vd.vardrop_act_fwd(*far, None, cfg, lo, None)
            step = (hi.double() - lo.double()) / (2 * h)
            bound = (1.2 * h * h / 6) * (b.double().abs() + 1e-3) + 2.0 ** -20 * (y.double().abs() + b.double().abs() + 1) / h
            assert bool(((d.double() - step).abs() <= bound).all())


def test_captured_and_replayed():
    a, b = make(2, 64, 96, BF, True)
    d_y = make(2, 64, 96, BF, False, seed=3)[0]
    n_sel = torch.tensor([10], dtype=torch.int32, device="cuda")
    cfg = vd.ActCfg(2, 64, 96, 0, SILU, 1, 1, 0)
    ckpt, y, d_a, d_b = vd.alloc_act_ckpt(cfg), *(torch.zeros_like(a) for _ in range(3))

    def call():
        vd.vardrop_act_fwd(a, b, n_sel, cfg, y, ckpt)
        vd.vardrop_act_bwd(d_y, ckpt, n_sel, cfg, d_a, d_b, None)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    n_sel.fill_(64)
    a.mul_(0.5)
    graph.replay()
    got = [t.clone() for t in (y, d_a, d_b)]
    call()
    torch.cuda.synchronize()
    assert all(torch.equal(g, t) for g, t in zip(got, (y, d_a, d_b))) and bool(y[:, 63].any())


def test_offsets_behind_32_bits():
    B, N, C = 1, (1 << 20) + 3, 2056            # 2.16e9 elements
    n_sel = torch.tensor([N], dtype=torch.int32, device="cuda")
    a = torch.zeros((B, N, C), dtype=BF, device="cuda")
    tail, _ = make(1, 5, C, BF, False)
    a[:, -5:] = tail
    cfg = vd.ActCfg(B, N, C, 0, GELU, 0, 1, 0)
    ckpt, y = vd.alloc_act_ckpt(cfg), torch.empty_like(a)
    vd.vardrop_act_fwd(a, None, n_sel, cfg, y, ckpt)
    small = vd.ActCfg(1, 5, C, 0, GELU, 0, 0, 0)
    sc, sy, sd = vd.alloc_act_ckpt(small), torch.empty_like(tail), torch.empty_like(tail)
    vd.vardrop_act_fwd(tail, None, None, small, sy, sc)
    vd.vardrop_act_bwd(tail, sc, None, small, sd, None, None)
    assert torch.equal(y[:, -5:], sy)
    vd.vardrop_act_bwd(a, ckpt, n_sel, cfg, y, None, None)
    assert torch.equal(y[:, -5:], sd)


def test_binding_refuses_other_tensors():
    a, b = make(2, 8, 32, BF, True, fused=True)
    cfg = vd.ActCfg(2, 8, 32, 0, SILU, 1, 0, 64)
    y, ckpt = torch.empty((2, 8, 32), dtype=BF, device="cuda"), vd.alloc_act_ckpt(cfg)
    vd.vardrop_act_fwd(a, b, None, cfg, y, ckpt)
    for bad in ((a.contiguous(), b, y), (a, b.float(), y), (a, b, y.half()), (a, b, y[:1]), (a[:, ::2], b, y), (a.cpu(), b, y)):
        with pytest.raises(ValueError):
            vd.vardrop_act_fwd(bad[0], bad[1], None, cfg, bad[2], ckpt)
    with pytest.raises(ValueError):
        vd.vardrop_act_fwd(a, b, torch.tensor([8], device="cuda"), cfg, y, ckpt)
    with pytest.raises(vd.VardropError):
        vd.vardrop_act_fwd(a, b, None, cfg, y, ckpt[:256])
