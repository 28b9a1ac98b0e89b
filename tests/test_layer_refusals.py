"""Argument checks of the operators around the attention: they run ahead of any CUDA call, on a machine without a GPU too."""
import ctypes as C
import os
import re
import subprocess

import pytest

from paper_2501_14183_b200 import binding as vd
from paper_2501_14183_b200 import build as lib_build


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return vd.load()


GOOD = 4096         # an address that is aligned; nothing is launched in these tests


def norm_cfg(**kw):
    return vd.NormCfg(*[{**dict(B=2, N=8, C=64, dtype=0, pre=1, post=1, gate_rows=1, S=0, res_scale=1.0, eps=1e-5), **kw}[n] for n, _ in vd.NormCfg._fields_])


@pytest.mark.parametrize("kw,status", [(dict(B=0), 1), (dict(N=0), 1), (dict(C=0), 1), (dict(C=8193), 2), (dict(B=1 << 16, N=1 << 15, gate_rows=0), 2), (dict(dtype=3), 1), (dict(pre=3), 1),
                                       (dict(post=-1), 1), (dict(gate_rows=3), 1), (dict(S=3), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1),
                                       (dict(res_scale=float("inf")), 1), (dict(B=65535, gate_rows=65535), 2)])
def test_norm_configurations(lib, kw, status):
    cfg = norm_cfg(**kw)
    assert lib.vardrop_norm_fwd(*[GOOD] * 6, None, None, None, C.byref(cfg), GOOD, GOOD, GOOD, None) == status
    assert lib.vardrop_last_error().startswith(b"norm")
    assert vd.vardrop_norm_workspace_bytes(cfg) == 0


def test_norm_arguments(lib):
    cfg = C.byref(norm_cfg())
    names = ["x", "y", "gate", "w_post", "b_post", "w_pre", "b_pre", "sel_idx", "n_sel"]
    outs = ["h", "u", "stats"]
    usual = dict(x=GOOD, y=GOOD, gate=GOOD, w_post=GOOD, b_post=None, w_pre=GOOD, b_pre=None, sel_idx=None, n_sel=None, h=GOOD, u=GOOD, stats=GOOD)
    for change in (dict(x=None), dict(y=None), dict(gate=None), dict(b_post=GOOD), dict(b_pre=GOOD), dict(u=None), dict(sel_idx=GOOD), dict(x=GOOD + 8), dict(w_pre=GOOD + 4), dict(h=GOOD + 2),
                   dict(stats=GOOD + 4)):
        a = {**usual, **change}
        assert lib.vardrop_norm_fwd(*[a[n] for n in names], cfg, *[a[n] for n in outs], None) == vd.ERR_INVALID_ARG, change
    assert lib.vardrop_norm_fwd(*[GOOD] * 9, None, *[GOOD] * 3, None) == vd.ERR_INVALID_ARG
    need = vd.vardrop_norm_workspace_bytes(norm_cfg())
    names = ["x", "y", "gate", "w_post", "b_post", "w_pre", "sel_idx", "n_sel", "inv_idx", "stats", "d_h", "d_u"]
    outs = ["dx", "dy", "d_gate", "d_w_post", "d_b_post", "d_w_pre", "d_b_pre"]
    usual = dict.fromkeys(names + outs, GOOD) | dict(b_post=None, sel_idx=None, n_sel=None, inv_idx=None, d_b_post=None, d_b_pre=None)
    for change in (dict(x=None), dict(stats=None), dict(d_u=None), dict(dx=None), dict(dy=None), dict(y=None), dict(sel_idx=GOOD, n_sel=GOOD), dict(d_b_post=GOOD), dict(d_b_pre=GOOD),
                   dict(d_gate=GOOD + 4), dict(gate=None)):
        a = {**usual, **change}
        assert lib.vardrop_norm_bwd(*[a[n] for n in names], cfg, *[a[n] for n in outs], GOOD, need, None) == vd.ERR_INVALID_ARG, change
    a = usual
    assert lib.vardrop_norm_bwd(*[a[n] for n in names], cfg, *[a[n] for n in outs], GOOD, need - 1, None) == vd.ERR_WORKSPACE
    assert lib.vardrop_norm_bwd(*[a[n] for n in names], cfg, *[a[n] for n in outs], None, need, None) == vd.ERR_INVALID_ARG


class Tensor(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("n", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32)]


def test_clip_arguments(lib):
    need = vd.vardrop_grad_clip_workspace_bytes()

    def call(*tensors, count=None, max_norm=1.0, eps=0.0, norm=GOOD, nb=need):
        table = (Tensor * max(1, len(tensors)))(*[Tensor(*t, 0) for t in tensors])
        return lib.vardrop_grad_clip(table, len(tensors) if count is None else count, C.byref(vd.ClipCfg(max_norm, eps)), norm, GOOD, nb, None)

    ok = (GOOD, GOOD, 10, 2)
    assert call((GOOD, GOOD, 10, 3)) == call((GOOD, GOOD, -1, 2)) == call((None, GOOD, 10, 2)) == call((GOOD, None, 10, 2)) == vd.ERR_INVALID_ARG
    assert call((GOOD + 2, GOOD, 10, 2)) == call((GOOD, GOOD + 2, 10, 2)) == call((GOOD + 1, GOOD + 1, 10, 0)) == vd.ERR_INVALID_ARG
    assert call((GOOD, GOOD + 4, 10, 2)) == call((GOOD + 4, GOOD, 10, 2)) == vd.ERR_INVALID_ARG and b"overlaps" in lib.vardrop_last_error()
    assert call(ok, max_norm=-1.0) == call(ok, max_norm=float("nan")) == call(ok, eps=-1.0) == call(ok, norm=None) == call(ok, count=-1) == vd.ERR_INVALID_ARG
    assert call(*[ok] * 16385) == vd.ERR_UNSUPPORTED
    apart = [(GOOD + 64 * i, GOOD + 64 * i, 16, 2) for i in range(40)]
    assert call(*apart, ok) == call(*apart[::-1], (GOOD + 60, GOOD + 60, 2, 0)) == call(ok, ok) == vd.ERR_INVALID_ARG and b"overlaps another" in lib.vardrop_last_error()
    far = 1 << 20                       # one tensor's output on another's input; inputs may be the same
    assert call((GOOD, far, 16, 2), (far + 64, GOOD + 60, 16, 2)) == vd.ERR_INVALID_ARG and b"another tensor's input" in lib.vardrop_last_error()
    assert call((GOOD, far, 16, 2), (GOOD, far, 16, 2)) == vd.ERR_INVALID_ARG
    assert call(ok, nb=need - 1) == vd.ERR_WORKSPACE


def packed_cfg(**kw):
    return vd.PackedCfg(*[{**dict(n_seqs=3, T=100, Hq=4, Hkv=2, D=64, sm_scale=0.0, causal=1, sTq=0, sHq=0, sTkv=0, sHkv=0), **kw}[n] for n, _ in vd.PackedCfg._fields_])


@pytest.mark.parametrize("kw,status", [(dict(n_seqs=0), 1), (dict(T=0), 1), (dict(Hq=0), 1), (dict(Hkv=0), 1), (dict(Hq=5), 1), (dict(D=128), 2), (dict(D=48), 2), (dict(T=(1 << 24) + 1), 2),
                                       (dict(n_seqs=(1 << 24) + 1), 2), (dict(Hq=8192), 2), (dict(T=1 << 24, n_seqs=1 << 24), 2), (dict(causal=2), 1), (dict(sm_scale=-1.0), 1),
                                       (dict(sm_scale=float("nan")), 1), (dict(sm_scale=float("inf")), 1), (dict(sm_scale=2e30), 1), (dict(sTq=256), 1), (dict(sTq=260, sHq=64), 1), (dict(sTkv=32, sHkv=64), 1),
                                       (dict(sTq=256, sHq=60), 1), (dict(sTq=-256, sHq=64), 1), (dict(sTkv=1 << 40, sHkv=64), 2)])
def test_packed_configurations(lib, kw, status):
    cfg = packed_cfg(**kw)
    assert lib.vardrop_packed_plan(GOOD, C.byref(cfg), GOOD, 1 << 30, None) == status
    assert lib.vardrop_attn_packed_fwd(*[GOOD] * 4, 1 << 30, C.byref(cfg), GOOD, GOOD, GOOD, 1 << 30, None) == status
    assert lib.vardrop_attn_packed_bwd(*[GOOD] * 7, 1 << 30, C.byref(cfg), *[GOOD] * 4, 1 << 40, None) == status
    assert lib.vardrop_last_error().startswith(b"packed attention")
    assert vd.vardrop_packed_plan_bytes(cfg) == 0 and vd.vardrop_attn_packed_workspace_bytes(cfg) == 0


def test_packed_arguments(lib):
    cfg = packed_cfg()
    plan, ws, by = vd.vardrop_packed_plan_bytes(cfg), vd.vardrop_attn_packed_workspace_bytes(cfg), C.byref(cfg)
    assert plan == 256 + 3 * 16 and ws >= 3 * 128 * 4 * (64 + 1) * 4
    assert lib.vardrop_packed_plan(None, by, GOOD, plan, None) == lib.vardrop_packed_plan(GOOD, by, None, plan, None) == lib.vardrop_packed_plan(GOOD + 4, by, GOOD, plan, None) == 1
    assert lib.vardrop_packed_plan(GOOD, by, GOOD, plan - 1, None) == vd.ERR_WORKSPACE and lib.vardrop_packed_plan(GOOD, None, GOOD, plan, None) == 1
    for at in range(7):                 # q, k, v, plan, o, lse, ws
        for bad in (None, GOOD + 8):
            a = [GOOD] * 7
            a[at] = bad
            assert lib.vardrop_attn_packed_fwd(*a[:4], plan, by, *a[4:], 256, None) == 1, at
    assert lib.vardrop_attn_packed_fwd(*[GOOD] * 4, plan - 1, by, *[GOOD] * 3, 256, None) == vd.ERR_WORKSPACE
    assert lib.vardrop_attn_packed_fwd(*[GOOD] * 4, plan, by, *[GOOD] * 3, 255, None) == vd.ERR_WORKSPACE
    for at in range(11):                # q, k, v, o, lse, d_o, plan, dq, dk, dv, ws
        for bad in (None, GOOD + 8):
            a = [GOOD] * 11
            a[at] = bad
            assert lib.vardrop_attn_packed_bwd(*a[:7], plan, by, *a[7:], ws, None) == 1, at
    assert lib.vardrop_attn_packed_bwd(*[GOOD] * 7, plan, by, *[GOOD] * 4, ws - 1, None) == vd.ERR_WORKSPACE


def test_struct_layouts_match_header():
    assert C.sizeof(vd.PackedCfg) == 64 and vd.PackedCfg.sTq.offset == 32
    assert C.sizeof(vd.NormCfg) == 40 and vd.NormCfg.res_scale.offset == 32
    assert C.sizeof(vd.ClipCfg) == 8 and C.sizeof(Tensor) == 32


# What the branch of attn_packed_bwd_kernel that takes results out needs around it to run on the host, a thread a warp: waits that succeed but for one, and a named barrier that says when
# not all four come.
HOST_WARPGROUP = r"""
#include <chrono>
#include <condition_variable>
#include <cstdint>
#include <mutex>
#include <thread>
struct uint4 { uint32_t x, y, z, w; };
struct float4 { float x, y, z, w; };
typedef uint16_t __nv_bfloat16;
struct Item { int start, len, jt, kvh, base, steps, per, s0; };
struct Params { __nv_bfloat16 *dk, *dv; int T, Hq, Hkv, group, D; float scale; } P;
const int kTile = 128, kRowBytes = 128, kTileBytes = 16384, kMostParts = 4;
const uint32_t kColDq = 0, kColDv = 0, kColDk = 0;
alignas(16) unsigned char sOut[2 * 16384];
int map_acc, map_parts;
Item items[6];
std::mutex m;
std::condition_variable cv;
int arrived, gone, phase, waits[4], fail_warp, fail_at;
bool all_ok, result, hung;
thread_local int me;
bool group_sync_and(int, bool ok) {
    std::unique_lock<std::mutex> l(m);
    if (arrived == 0) all_ok = true;
    all_ok = all_ok && ok;
    const int p = phase;
    if (++arrived == 4) { arrived = 0; result = all_ok; ++phase; cv.notify_all(); return result; }
    if (!cv.wait_for(l, std::chrono::seconds(5), [&] { return phase != p || gone > 0; }) || phase == p) { hung = true; return false; }
    return result;
}
bool warp_wait_relaxed(uint64_t*, uint32_t) { return !(me == fail_warp && waits[me]++ == fail_at); }
int small_div(int a, int d) { return a / d; }
uint32_t pack2(float, float) { return 0; }
uint4 make_uint4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return {a, b, c, d}; }
float4 make_float4(float a, float b, float c, float d) { return {a, b, c, d}; }
template <class... A> void nothing(A&&...) {}
#define bulk_wait_group_read0 nothing
#define bulk_wait_group0 nothing
#define bulk_commit_group nothing
#define tma_reduce_add_3d nothing
#define tma_store_3d nothing
#define tc_fence_after nothing
#define tc_fence_before nothing
#define tmem_ld32(at, v) for (float& e : v) e = 0.f
#define tmem_ld_wait nothing
#define fence_proxy_async_smem nothing
void role(int warp, bool& left_ok) {
    const int lane = 0, tid = warp * 32;
    uint32_t tmem = 0;
    bool ok = true;
    uint64_t bars[64];
    uint64_t *bar_dv_done = bars, *bar_dv_free = bars, *bar_dk_done = bars, *bar_dk_free = bars, *bar_g = bars, *bar_gfree = bars;
    auto begin = [] {};
    auto item_wait = [&](uint32_t) { ok &= warp_wait_relaxed(bars, 0); };
    auto item_read = [&](uint32_t i) { return items[i]; };
    auto warp_arrive = [](uint64_t*) {};
    me = warp & 3;
BODY
    left_ok = ok;
    std::lock_guard<std::mutex> l(m);
    ++gone;
    cv.notify_all();
}
// number of waits of the warp; -1: a barrier that not all four reach, -2: a warp that leaves without having learnt of the wait that gave up
extern "C" int run(int group, int failing, int at) {
    static __nv_bfloat16 data[512 * 2 * 64];
    P = Params{data, data, 512, 4, 2, 2, 64, 1.f};
    const Item list[6] = {{0, 300, 0, 0, 0, 6, 3, 0}, {0, 300, 1, 1, 0, 4, 2, 0}, {0, 300, 0, 4096, 0, 3, 3, 0}, {0, 300, 0, 8192, 0, 3, 3, 3}, {0, -1, 0, 0, 0, 0, 0, 0}, {0, -1, 0, 0, 0, 0, 0, 0}};
    for (int i = 0; i < 6; ++i) items[i] = list[i];
    arrived = gone = phase = 0; hung = false; fail_warp = failing; fail_at = at;
    for (int& w : waits) w = 0;
    bool ok[4];
    std::thread t[4];
    for (int w = 0; w < 4; ++w) t[w] = std::thread([=, &ok] { role(4 + 4 * group + w, ok[w]); });
    for (auto& x : t) x.join();
    if (hung) return -1;
    const bool gave_up = waits[failing] > at;
    for (bool o : ok) if (o == gave_up) return -2;
    return waits[failing];
}
"""


def test_warps_that_share_a_named_barrier_leave_together(tmp_path):
    """Nothing bounds a named barrier.  Whichever wait of whichever warp gives up, whole items and parts of them among what is under way, all four warps learn of it and leave behind the same
    barrier.  The text of their branch, run on the host with every wait failing in turn."""
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_14183_b200", "csrc", "attn_packed_bwd.cu")
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(path).read(), flags=re.S)
    body = text[text.index("attn_packed_bwd_kernel("):]
    start = body.index("{", body.index("else if (warp < 12)")) + 1
    depth, end = 1, start
    while depth:
        depth += {"{": 1, "}": -1}.get(body[end], 0)
        end += 1
    branch = re.sub(r"asm volatile[^\n]*", "", body[start:end - 1])
    assert "setmaxnreg" not in branch and branch.count("group_sync_and") >= 3
    (tmp_path / "role.cpp").write_text(HOST_WARPGROUP.replace("BODY", branch))
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-w", "-shared", "-fPIC", "-pthread", "-o", str(tmp_path / "role.so"), str(tmp_path / "role.cpp")])
    lib = C.CDLL(str(tmp_path / "role.so"))
    for group in (0, 1):
        for warp in range(4):
            waits = lib.run(group, warp, 1 << 30)
            assert waits >= 5 + 16 + 4, "items, query tiles, finished items"
            got = [lib.run(group, warp, at) for at in range(waits)]
            assert min(got) > 0, (group, warp, got)
