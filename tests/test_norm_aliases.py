"""Which buffers of the norms may be the same: what would be read after it has been overwritten is refused, ahead of any CUDA call."""
import ctypes as C

import pytest

from paper_2501_14183_b200 import binding as vd
from paper_2501_14183_b200 import build as lib_build

B, N, CH = 2, 8, 64
ROWS = B * N * CH * 2                # bytes of a bf16 tensor


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return vd.load()


def far_apart(names):
    return {n: (i + 1) << 20 for i, n in enumerate(names)}


def run(lib, fwd, selected, change):
    """Status of a call whose buffers lie far apart but for those in `change`; on a machine without a GPU a call that passes the checks fails at its launch."""
    cfg = vd.NormCfg(B, N, CH, 0, 1, 1, 1, 0, 1.0, 1e-5)
    ins = ["x", "y", "gate", "w_post", "b_post", "w_pre"] + (["b_pre", "sel_idx", "n_sel"] if fwd else ["sel_idx", "n_sel", "inv_idx", "stats", "d_h", "d_u"])
    outs = ["h", "u", "stats"] if fwd else ["dx", "dy", "d_gate", "d_w_post", "d_b_post", "d_w_pre", "d_b_pre"]
    a = far_apart(dict.fromkeys(ins + outs))
    a.update(dict.fromkeys(["b_post", "b_pre", "d_b_post", "d_b_pre"]))
    if not selected:
        a.update(dict.fromkeys(["sel_idx", "n_sel", "inv_idx"]))
    a.update({n: a[of] + off for n, (of, off) in change.items()})
    tail = [] if fwd else [1 << 30, vd.vardrop_norm_workspace_bytes(cfg)]
    return (lib.vardrop_norm_fwd if fwd else lib.vardrop_norm_bwd)(*[a[n] for n in ins], C.byref(cfg), *[a[n] for n in outs], *tail, None)


FWD_BAD = [dict(h=("u", 0)), dict(h=("x", 16)), dict(u=("y", -16)), dict(u=("x", ROWS - 16)), dict(stats=("h", 0)), dict(stats=("y", 0)), dict(h=("gate", 0)), dict(u=("w_pre", 0)), dict(stats=("x", ROWS - 16))]
FWD_SELECTED = [dict(h=("x", 0)), dict(u=("x", 0)), dict(h=("sel_idx", 0)), dict(stats=("n_sel", 0))]
BWD_BAD = [dict(dx=("dy", 0)), dict(dx=("d_h", 16)), dict(dy=("d_u", -16)), dict(dx=("stats", 0)), dict(dy=("gate", 0)), dict(d_gate=("gate", 0)), dict(d_w_post=("w_post", 0)), dict(d_w_pre=("d_w_post", 0)),
           dict(d_w_pre=("d_u", 64)), dict(d_gate=("dx", 0))]
BWD_SELECTED = [dict(dx=("d_h", 0)), dict(dx=("x", 16)), dict(dx=("y", 0)), dict(dx=("d_u", 0)), dict(dy=("x", 0)), dict(dx=("inv_idx", 0)), dict(dy=("sel_idx", 0))]


@pytest.mark.parametrize("fwd,selected,change", [(True, s, c) for s in (False, True) for c in FWD_BAD] + [(True, True, c) for c in FWD_SELECTED] +
                         [(False, s, c) for s in (False, True) for c in BWD_BAD] + [(False, True, c) for c in BWD_SELECTED])
def test_buffers_that_may_not_overlap(lib, fwd, selected, change):
    assert run(lib, fwd, selected, change) == vd.ERR_INVALID_ARG, change
    assert b"overlap" in lib.vardrop_last_error(), lib.vardrop_last_error()
