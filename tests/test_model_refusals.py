"""Argument checks of the embeddings, the activations and the loss: they run ahead of any CUDA call, on a machine without a GPU too."""
import ctypes as C

import pytest

from paper_2501_14183_b200 import binding as vd
from paper_2501_14183_b200 import build as lib_build


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return vd.load()


def spots(n, apart=1 << 24):
    """Aligned addresses of buffers that do not overlap; nothing is launched in these tests."""
    return [(i + 1) * apart for i in range(n)]


def make(struct, usual, **kw):
    return struct(*[{**usual, **kw}[n] for n, _ in struct._fields_])


def embed_cfg(**kw):
    return make(vd.EmbedCfg, dict(T=100, V=50, C=64, dtype=2, out_dtype=0, accumulate=0, scale=1.0), **kw)


@pytest.mark.parametrize("kw,status", [(dict(T=0), 1), (dict(V=0), 1), (dict(C=0), 1), (dict(T=-5), 1), (dict(dtype=3), 1), (dict(out_dtype=-1), 1), (dict(accumulate=2), 1), (dict(scale=float("nan")), 1),
                                       (dict(scale=float("inf")), 1), (dict(T=(1 << 28) + 1), 2), (dict(V=(1 << 30) + 1), 2), (dict(C=65537), 2)])
def test_embed_configurations(lib, kw, status):
    cfg = embed_cfg(**kw)
    table, idx, out, ws = spots(4, 1 << 40)
    assert lib.vardrop_embed_fwd(table, idx, C.byref(cfg), out, ws, 1 << 36, None) == status
    assert lib.vardrop_last_error().startswith(b"embed")
    assert lib.vardrop_embed_bwd(out, idx, C.byref(cfg), table, ws, 1 << 36, None) == status
    assert vd.vardrop_embed_workspace_bytes(cfg) == 0


def test_embed_arguments(lib):
    cfg = C.byref(embed_cfg())
    need = vd.vardrop_embed_workspace_bytes(embed_cfg())
    assert need >= 256 + 4 * 100 * 4
    for call, nb in ((lib.vardrop_embed_fwd, 256), (lib.vardrop_embed_bwd, need)):
        good = spots(4)
        for at in range(4):
            for bad in (None, good[at] + 8):
                a = list(good)
                a[at] = bad
                assert call(a[0], a[1], cfg, a[2], a[3], nb, None) == vd.ERR_INVALID_ARG, at
        assert call(good[0], good[1], None, good[2], good[3], nb, None) == vd.ERR_INVALID_ARG
        assert call(good[0], good[1], cfg, good[2], good[3], nb - 1, None) == vd.ERR_WORKSPACE
        for at in (0, 1, 3):            # the output on something else
            a = list(good)
            a[at] = a[2] + 16
            assert call(a[0], a[1], cfg, a[2], a[3], nb, None) == vd.ERR_INVALID_ARG and b"overlap" in lib.vardrop_last_error(), at


def act_cfg(**kw):
    return make(vd.ActCfg, dict(B=4, N=10, C=64, dtype=0, kind=1, gated=1, S=0, stride=0), **kw)


@pytest.mark.parametrize("kw,status", [(dict(B=0), 1), (dict(N=0), 1), (dict(C=0), 1), (dict(dtype=3), 1), (dict(kind=3), 1), (dict(kind=-1), 1), (dict(gated=2), 1), (dict(S=3), 1), (dict(S=-1), 1),
                                       (dict(stride=56), 1), (dict(stride=68), 1), (dict(stride=-64), 1), (dict(B=1 << 16, N=1 << 15), 2), (dict(C=(1 << 20) + 1), 2), (dict(stride=1 << 33), 2),
                                       (dict(B=1, N=1 << 20, C=1 << 20), 2)])
def test_act_configurations(lib, kw, status):
    cfg = act_cfg(**kw)
    a, b, y, ckpt = spots(4, 1 << 44)
    assert lib.vardrop_act_fwd(a, b, None, C.byref(cfg), y, ckpt, 1 << 43, None) == status
    assert lib.vardrop_last_error().startswith(b"act")
    assert lib.vardrop_act_bwd(y, ckpt, 1 << 43, None, C.byref(cfg), a, b, None, None) == status
    assert vd.vardrop_act_ckpt_bytes(cfg) == 0


def test_act_arguments(lib):
    cfg = act_cfg()
    by, need = C.byref(cfg), vd.vardrop_act_ckpt_bytes(cfg)
    assert need == 2 * 40 * 64 + 256            # 160 scales take a multiple of 256
    a, b, y, ckpt, n_sel, d_y = spots(6)
    fwd = lambda a=a, b=b, n=n_sel, by=by, y=y, k=ckpt, nb=need: lib.vardrop_act_fwd(a, b, n, by, y, k, nb, None)  # noqa: E731
    bwd = lambda d=d_y, k=ckpt, nb=need, n=n_sel, by=by, da=a, db=b, y=y: lib.vardrop_act_bwd(d, k, nb, n, by, da, db, y, None)  # noqa: E731
    bad = [fwd(a=None), fwd(b=None), fwd(y=None), fwd(by=None), fwd(a=a + 8), fwd(b=b + 8), fwd(y=y + 4), fwd(k=ckpt + 8), fwd(n=n_sel + 4),
           bwd(d=None), bwd(k=None), bwd(da=None), bwd(db=None), bwd(by=None), bwd(d=d_y + 8), bwd(k=ckpt + 8), bwd(da=a + 8), bwd(db=b + 2), bwd(y=y + 8), bwd(n=n_sel + 4)]
    assert bad == [vd.ERR_INVALID_ARG] * len(bad)
    assert fwd(nb=need - 1) == bwd(nb=need - 1) == vd.ERR_WORKSPACE
    overlaps = [fwd(y=a + 16), fwd(y=n_sel), fwd(k=a), fwd(y=ckpt), bwd(da=ckpt), bwd(db=a), bwd(y=a), bwd(y=b + 16), bwd(da=d_y + 16), bwd(y=n_sel)]
    assert overlaps == [vd.ERR_INVALID_ARG] * len(overlaps) and b"overlap" in lib.vardrop_last_error()
    plain = C.byref(act_cfg(gated=0))           # a branch that the configuration does not have
    assert fwd(by=plain) == bwd(by=plain) == vd.ERR_INVALID_ARG
    wide = C.byref(act_cfg(stride=128))         # both halves of one projection, but not rows that reach into each other
    assert fwd(by=wide, b=a + 64, y=a) == bwd(by=wide, db=a + 64) == vd.ERR_INVALID_ARG


def loss_cfg(**kw):
    return make(vd.LossCfg, dict(T=100, V=50, C=64, dtype=0, scale=1.0), **kw)


@pytest.mark.parametrize("kw,status", [(dict(T=0), 1), (dict(V=0), 1), (dict(C=0), 1), (dict(dtype=3), 1), (dict(dtype=-1), 1), (dict(dtype=2), 2), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1),
                                       (dict(scale=2e30), 1), (dict(C=65), 2), (dict(C=4), 2), (dict(C=65544), 2), (dict(T=(1 << 24) + 1), 2), (dict(V=(1 << 24) + 1), 2), (dict(T=1 << 24, V=1 << 24), 2)])
def test_loss_configurations(lib, kw, status):
    cfg = loss_cfg(**kw)
    h, w, labels, loss, lse, ws, d_h, d_w = spots(8, 1 << 44)
    assert lib.vardrop_loss_fwd(h, w, labels, C.byref(cfg), loss, lse, ws, 1 << 43, None) == status
    assert lib.vardrop_last_error().startswith(b"loss")
    assert lib.vardrop_loss_bwd(h, w, labels, lse, loss, C.byref(cfg), d_h, d_w, ws, 1 << 43, None) == status
    assert vd.vardrop_loss_workspace_bytes(cfg) == 0


def test_loss_arguments(lib):
    cfg = C.byref(loss_cfg())
    need = vd.vardrop_loss_workspace_bytes(loss_cfg())
    good = spots(6)                             # h, w, labels, loss, lse, ws
    fwd = lambda a, nb=need, by=cfg: lib.vardrop_loss_fwd(*a[:3], by, *a[3:], nb, None)  # noqa: E731
    for at in range(6):
        for bad in (None, good[at] + 8):
            assert fwd(good[:at] + [bad] + good[at + 1:]) == vd.ERR_INVALID_ARG, at
    assert fwd(good, by=None) == vd.ERR_INVALID_ARG and fwd(good, need - 1) == vd.ERR_WORKSPACE
    for out in (3, 4, 5):
        for other in range(6):
            if other != out:
                a = list(good)
                a[out] = a[other] + (16 if other < 3 else 0)
                assert fwd(a) == vd.ERR_INVALID_ARG and b"overlap" in lib.vardrop_last_error(), (out, other)
    good = spots(8)                             # h, w, labels, lse, d_loss, d_h, d_w, ws
    bwd = lambda a, nb=need, by=cfg: lib.vardrop_loss_bwd(*a[:5], by, *a[5:], nb, None)  # noqa: E731
    for at in range(8):
        for bad in (None, good[at] + 8):
            if bad is None and at in (5, 6):    # one gradient alone is fine, none at all is not
                continue
            assert bwd(good[:at] + [bad] + good[at + 1:]) == vd.ERR_INVALID_ARG, at
    assert bwd(good[:5] + [None, None] + good[7:]) == bwd(good, by=None) == vd.ERR_INVALID_ARG and bwd(good, need - 1) == vd.ERR_WORKSPACE
    for out in (5, 6, 7):
        for other in range(8):
            if other != out:
                a = list(good)
                a[out] = a[other]
                assert bwd(a) == vd.ERR_INVALID_ARG and b"overlap" in lib.vardrop_last_error(), (out, other)


def test_struct_layouts_match_header():
    assert C.sizeof(vd.EmbedCfg) == 28 and vd.EmbedCfg.scale.offset == 24
    assert C.sizeof(vd.ActCfg) == 40 and vd.ActCfg.stride.offset == 32
    assert C.sizeof(vd.LossCfg) == 20
