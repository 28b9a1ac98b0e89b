"""vardrop_embed_fwd / vardrop_embed_bwd against the formulas in 64 bits."""
import pytest
import torch

from paper_2501_14183_b200 import binding as vd

pytestmark = pytest.mark.gpu

BF, HF, FP = torch.bfloat16, torch.float16, torch.float32
U = 2.0 ** -24          # half a step of fp32


def tokens(T, V, seed, spread="even", gaps=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    idx = (u * V if spread == "even" else u ** 8 * V if spread == "skewed" else torch.zeros_like(u)).long().clamp(0, V - 1)
    return torch.where(torch.rand(T, generator=g, device="cuda") < gaps, -1 - idx, idx).to(torch.int32)


def normal(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def config(T, V, C, table=BF, out=BF, accumulate=0, scale=1.0):
    cfg = vd.EmbedCfg(T, V, C, vd.DTYPES[table], vd.DTYPES[out], accumulate, scale)
    ws = vd.alloc_ws(vd.vardrop_embed_workspace_bytes(cfg))
    ws[256:] = 0xFF
    return cfg, ws


def check_forward(T, V, C, table=BF, out=BF, scale=1.0, spread="even", gaps=0.0):
    cfg, ws = config(T, V, C, table, out, 0, scale)
    w, idx = normal((V, C), table, 1), tokens(T, V, 2, spread, gaps)
    got = torch.full((T, C), 7.0, dtype=out, device="cuda")
    vd.vardrop_embed_fwd(w, idx, cfg, got, ws)
    assert vd.ws_status(ws) == vd.OK
    want = torch.where((idx >= 0)[:, None], w.double()[idx.long().clamp_min(0)] * cfg.scale, 0)
    info = torch.finfo(out)                     # a product rounded to fp32 and to the type
    assert bool(((got.double() - want).abs() <= want.abs() * (info.eps / 2 + U) + info.smallest_normal * info.eps / 2).all())


def wanted_rows(d_out, idx, V, scale):
    """The gradient, the magnitudes that it is made of, and the tokens of each row."""
    live = idx >= 0
    at, d = idx[live].long(), d_out[live].double() * scale
    zero = torch.zeros((V, d_out.shape[1]), dtype=torch.float64, device="cuda")
    return zero.index_add(0, at, d), zero.index_add(0, at, d.abs()), torch.bincount(at, minlength=V)[:, None]


def near(got, want, size, count, old=0.0):
    """fp32 sums of `count` values (and what was there), times the scale, rounded once."""
    info = torch.finfo(got.dtype)
    bound = (size + abs(old)) * (count + 3) * U + want.abs() * info.eps / 2 + info.smallest_normal * info.eps / 2
    assert bool(((got.double() - want).abs() <= bound).all()), float(((got.double() - want).abs() / bound.clamp_min(1e-300)).max())


def check_backward(T, V, C, table=BF, out=BF, scale=1.0, spread="even", gaps=0.0, idx=None):
    idx = tokens(T, V, 3, spread, gaps) if idx is None else idx
    d = normal((T, C), out, 4)
    d[idx < 0] = float("nan")                   # not read
    cfg, ws = config(T, V, C, table, out, 0, scale)
    got = torch.full((V, C), float("nan"), dtype=table, device="cuda")
    vd.vardrop_embed_bwd(d, idx, cfg, got, ws)
    assert vd.ws_status(ws) == vd.OK
    want, size, count = wanted_rows(d, idx, V, cfg.scale)
    near(got, want, size, count)
    # the same order whatever ran before, and added to what is there
    again = torch.full_like(got, 3.0)
    vd.vardrop_embed_bwd(d, idx, cfg, again, ws)
    assert torch.equal(got, again)
    cfg, ws = config(T, V, C, table, out, 1, scale)
    old = normal((V, C), table, 5)
    more = old.clone()
    vd.vardrop_embed_bwd(d, idx, cfg, more, ws)
    assert vd.ws_status(ws) == vd.OK
    near(more, want + old.double(), size, count, old.double())
    assert torch.equal(more[count[:, 0] == 0], old[count[:, 0] == 0])


@pytest.mark.parametrize("table", [BF, HF, FP])
@pytest.mark.parametrize("out", [BF, HF, FP])
@pytest.mark.parametrize("C", [1, 6, 36, 520, 4104])
def test_types_and_widths(table, out, C):
    check_forward(77, 50, C, table, out, 3.25, gaps=0.2)
    check_backward(300, 50, C, table, out, 3.25, gaps=0.2)


@pytest.mark.parametrize("T", [1, 2, 31, 33, 4095, 4096, 4097, 8193, 30000])
@pytest.mark.parametrize("V", [1, 2, 511, 512, 513, 70000])
def test_tokens_and_rows(T, V):
    check_forward(T, V, 24, scale=0.5)
    check_backward(T, V, 24, FP, BF, 0.5)
    check_backward(T, V, 24, BF, BF, 1.0, "skewed", 0.4)


@pytest.mark.parametrize("T", [5, 700, 50000])
def test_all_tokens_of_one_row_and_none_at_all(T):
    check_backward(T, 300, 65, FP, BF, 1.0, "one")
    check_backward(T, 300, 65, FP, BF, 1.0, idx=torch.full((T,), 299, dtype=torch.int32, device="cuda"))
    check_backward(T, 300, 65, FP, BF, 1.0, idx=torch.full((T,), -1, dtype=torch.int32, device="cuda"))
    check_backward(T, 300, 64, FP, BF, 1.0, idx=torch.arange(T, dtype=torch.int32, device="cuda").flip(0) % 300)


@pytest.mark.parametrize("T", [200, 6000])
@pytest.mark.parametrize("V,C", [(1, 1), (1, 3), (2, 3), (3, 7), (5, 9)])
def test_tables_that_are_no_whole_words(T, V, C):
    """Tens of tokens a row and more, tables that end inside sixteen bytes, with rows that no token has."""
    for table in (BF, FP):
        check_backward(T, V, C, table, BF)
        check_backward(T, V, C, table, BF, idx=torch.full((T,), -1, dtype=torch.int32, device="cuda"))
        check_backward(T, V, C, table, BF, idx=torch.full((T,), V - 1, dtype=torch.int32, device="cuda"))


def test_neighbours_of_the_table_are_left_alone():
    T, V, C = 6000, 5, 9
    idx, d = tokens(T, V, 3), normal((T, C), BF, 4)
    cfg, ws = config(T, V, C, BF, BF)
    flat = torch.full((V * C + 64,), 5.0, dtype=BF, device="cuda")
    vd.vardrop_embed_bwd(d, idx, cfg, flat[:V * C].view(V, C), ws)
    near(flat[:V * C].view(V, C), *wanted_rows(d, idx, V, 1.0))
    assert bool((flat[V * C:] == 5.0).all())


def test_more_digits_and_tiles_than_one():
    check_backward((1 << 20) + 4097, 7, 3, FP, FP, 1.0, "skewed", 0.1)           # several tiles to a CTA
    check_backward(5000, (1 << 18) + 1, 2, FP, FP, 1.0, "skewed", 0.1)           # three passes
    check_backward((1 << 20) + 5, 600, 2, FP, FP, 1.0, "even")


def test_selected_variates():
    """Indices as a selection gives them: kept variates ascending, -1 behind the last one, for several instances."""
    N, kept = 321, [119, 1, 321, 40]
    idx = torch.full((len(kept), N), -1, dtype=torch.int32, device="cuda")
    for s, m in enumerate(kept):
        idx[s, :m] = torch.randperm(N, device="cuda")[:m].sort().values.int()
    check_backward(len(kept) * N, N, 512, FP, BF, 1.0, idx=idx.view(-1))


def test_indices_behind_the_table_are_none_and_reported():
    cfg, ws = config(40, 10, 8)
    w, d = normal((10, 8), BF, 1), normal((40, 8), BF, 2)
    idx = tokens(40, 10, 3)
    idx[[5, 39]] = torch.tensor([10, 1 << 30], dtype=torch.int32, device="cuda")
    out = torch.empty((40, 8), dtype=BF, device="cuda")
    vd.vardrop_embed_fwd(w, idx, cfg, out, ws)
    assert vd.ws_status(ws) == vd.ERR_INVALID_ARG and not out[[5, 39]].any()
    cfg, ws = config(40, 10, 8, FP)
    got = torch.empty((10, 8), device="cuda")
    vd.vardrop_embed_bwd(d, idx, cfg, got, ws)
    assert vd.ws_status(ws) == vd.ERR_INVALID_ARG
    near(got, *wanted_rows(d, torch.where(idx < 10, idx, -1), 10, 1.0))


@pytest.mark.parametrize("T,V", [(300, 20), (3000, 5000), (9000, 5000)])
def test_indices_behind_the_table_in_every_form_of_the_sums(T, V):
    idx, d = tokens(T, V, 3), normal((T, 16), BF, 2)
    idx[::7] += V
    cfg, ws = config(T, V, 16, FP)
    got = torch.full((V, 16), float("nan"), device="cuda")
    vd.vardrop_embed_bwd(d, idx, cfg, got, ws)
    assert vd.ws_status(ws) == vd.ERR_INVALID_ARG
    near(got, *wanted_rows(d, torch.where(idx < V, idx, -1), V, 1.0))


@pytest.mark.parametrize("C", [255, 256, 257, 258, 260, 2050, 4097])
def test_rows_of_several_accesses(C):
    check_forward(200, 60, C, FP, BF, 1.5)
    check_backward(9000, 700, C, FP, BF, 1.5, "skewed", 0.1)           # sorted
    check_backward(3000, 4000, C, BF, BF, 1.5, "skewed", 0.1)          # placed
    check_backward(500, 60, C, HF, HF, 1.0, "skewed", 0.1)             # looked through


def test_a_table_behind_32_bit_offsets():
    V, C = (1 << 21) + 3, 1040                  # 2.2e9 elements
    w = torch.zeros((V, C), dtype=BF, device="cuda")
    idx = torch.tensor([V - 1, 0, V - 2, V - 1], dtype=torch.int32, device="cuda")
    w[idx.long()] = normal((4, C), BF, 1)
    cfg, ws = config(4, V, C, accumulate=1)
    out = torch.empty((4, C), dtype=BF, device="cuda")
    vd.vardrop_embed_fwd(w, idx, cfg, out, ws)
    assert torch.equal(out, w[idx.long()])
    before, d = w[[0, V - 2, V - 1]].double(), normal((4, C), BF, 2)
    vd.vardrop_embed_bwd(d, idx, cfg, w, ws)
    want = torch.stack([d[1], d[2], d[0].double() + d[3].double()]) + before
    near(w[[0, V - 2, V - 1]], want, want.abs(), 2, before)
    assert not w[1:V - 2].any()


def test_captured_and_replayed_with_other_tokens():
    T, V, C = 9000, 700, 40
    cfg, ws = config(T, V, C, FP, BF, 0, 2.0)
    w, d, idx = normal((V, C), FP, 1), normal((T, C), BF, 2), tokens(T, V, 3)
    out, got = torch.empty((T, C), dtype=BF, device="cuda"), torch.empty((V, C), device="cuda")

    def call():
        vd.vardrop_embed_fwd(w, idx, cfg, out, ws)
        vd.vardrop_embed_bwd(d, idx, cfg, got, ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (8, 9):
        idx.copy_(tokens(T, V, seed, "skewed", 0.3))
        out.fill_(float("nan"))
        got.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        again, rows = got.clone(), out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(again, got) and torch.equal(rows, out) and vd.ws_status(ws) == vd.OK
        near(got, *wanted_rows(d, idx, V, 2.0))


def test_on_a_stream_of_its_own():
    T, V, C = 5000, 300, 64
    cfg, ws = config(T, V, C, FP, BF)
    d, idx = normal((T, C), BF, 2), tokens(T, V, 3)
    got = torch.full((V, C), float("nan"), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        vd.vardrop_embed_bwd(d, idx, cfg, got, ws)
    torch.cuda.synchronize()
    near(got, *wanted_rows(d, idx, V, 1.0))


@pytest.mark.parametrize("T", [1, 3, 4, 5, 4094, 4099, 11262, 11264, 11265, 12290])
@pytest.mark.parametrize("spread", ["even", "skewed"])
def test_the_last_tokens_of_a_short_call(T, spread):
    """Numbers of tokens that are and are no multiple of four, up to both ends of the form that looks through all of them; the last one behind the table."""
    V, C = 300, 48
    check_backward(T, V, C, FP, BF, 1.5, spread, 0.3)
    idx, d = tokens(T, V, 3, spread), normal((T, C), BF, 4)
    idx[-1] = V
    cfg, ws = config(T, V, C, FP, BF)
    got = torch.full((V, C), float("nan"), device="cuda")
    vd.vardrop_embed_bwd(d, idx, cfg, got, ws)
    assert vd.ws_status(ws) == vd.ERR_INVALID_ARG
    idx[-1] = -1
    near(got, *wanted_rows(d, idx, V, 1.0))


def test_binding_refuses_other_tensors():
    cfg, ws = config(8, 5, 16)
    w, idx, out = normal((5, 16), BF, 1), tokens(8, 5, 2), torch.empty((8, 16), dtype=BF, device="cuda")
    for bad in ((w.float(), idx, out), (w, idx.long(), out), (w, idx, out.half()), (w.t(), idx, out), (w[:4], idx, out), (w, idx[:7], out), (w, idx, out[:, ::2]), (w.cpu(), idx, out)):
        with pytest.raises(ValueError):
            vd.vardrop_embed_fwd(*bad[:2], cfg, bad[2], ws)
