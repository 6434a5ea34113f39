"""CPU checks of the decoding-time calls: exports, workspace sizes, refusals before anything reaches a GPU, the split's plan."""
import ctypes
import os
import random
import re

import pytest
import torch  # noqa: F401  (loaded first so that the library binds to the same HIP runtime)

from tests.host_plan import host_library

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "metok_decode.h")


@pytest.fixture(scope="module")
def B():
    from paper_2506_02850_amd import build
    if not os.path.exists(build.LIB):
        build.build(verbose=False)
    from paper_2506_02850_amd import binding
    return binding


def test_every_declared_symbol_is_exported_and_bound(B):
    names = re.findall(r"METOK_API\s+[\w\s\*]+?\b(metok_\w+)\s*\(", open(HEADER).read())
    assert len(set(names)) == len(names) and sorted(names) == sorted(B.DECODE_EXPORTS)
    for name in names:
        assert hasattr(B.lib(), name) and callable(getattr(B, name)), name


def test_header_is_plain_c(tmp_path):
    import subprocess
    src = tmp_path / "x.c"
    src.write_text('#include "metok_decode.h"\nint main(void) { return METOK_MAX_DECODE_BATCH == 4096 ? 0 : 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "x.o")], check=True)


FAKE = [0x10000000 * (i + 1) for i in range(16)]        # aligned, far apart, never dereferenced: validation fails first


def attention_args(**kw):
    a = dict(q=FAKE[0], B=2, Hq=8, Hkv=2, dh=64, dtype=1, k=FAKE[1], v=FAKE[2], S_cap=128, len=FAKE[3], k_new=FAKE[4], v_new=FAKE[5], scale=0.125,
             cap=0.0, out=FAKE[6], lse=FAKE[7], weight=FAKE[8], stride=128, ws=FAKE[9], bytes=0, stream=None)
    a.update(kw)
    return list(a.values())


def test_refused_attention_calls(B):
    f = B.lib().metok_decode_attention

    def refused(code, text, **kw):
        assert f(*attention_args(**kw)) == code, kw
        assert text in B.metok_last_error(), (kw, B.metok_last_error())

    refused(-3, "workspace")
    refused(-3, "workspace", ws=None, bytes=1 << 30)
    refused(-3, "workspace", ws=FAKE[9] + 8, bytes=1 << 30)
    for name in ("q", "k", "v", "len", "out"):
        refused(-1, "NULL", **{name: None})
    refused(-1, "go together", k_new=None)
    refused(-1, "go together", v_new=None)
    for name in ("q", "k", "v", "k_new", "v_new", "out"):
        refused(-1, "aligned", **{name: FAKE[10] + 8})
    for name in ("len", "lse", "weight"):
        refused(-1, "aligned", **{name: FAKE[10] + 2})
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        refused(-1, "scale", scale=scale)
    for cap in (-1.0, float("nan"), float("inf")):
        refused(-1, "logit_cap", cap=cap)
    refused(-1, "weight_stride", stride=127)
    refused(-1, "dtype", dtype=2)
    for n in (0, -1, 4097):
        refused(-1, "B must", B=n)
    for hq, hkv in ((8, 3), (0, 2), (8, 0), (7, 2), (1025, 1), (-8, -2)):
        refused(-1, "Hq must", Hq=hq, Hkv=hkv)
    for dh in (0, 16, 96, 512):
        refused(-1, "dh must", dh=dh)
    refused(-1, "dh must", dh=256, dtype=0)
    for s in (0, -5, 2 ** 31 - 64, 2 ** 40):
        refused(-1, "capacity", S_cap=s, stride=2 ** 41)
    refused(-1, "too many rows", B=4096, S_cap=2 ** 30, stride=2 ** 41)
    refused(-1, "too many rows", B=64, Hq=1024, Hkv=64, S_cap=2 ** 24, stride=2 ** 41)
    big = 1 << 40
    refused(-1, "overlaps", out=FAKE[0], bytes=big)
    refused(-1, "overlaps", lse=FAKE[6], bytes=big)
    refused(-1, "overlaps", v=FAKE[1], bytes=big)
    refused(-1, "overlaps", v=FAKE[1] + 16, bytes=big)
    refused(-1, "overlaps", k_new=FAKE[1] + 64, bytes=big)
    refused(-1, "overlaps", weight=FAKE[3], bytes=big)
    refused(-1, "overlaps", ws=FAKE[2], bytes=big)


def test_scales_that_fp32_does_not_hold_are_refused(B):
    """1e-40 would lose its bits, 1e-50 be 0: as a cap it would mean none, as a scale 0 times -inf where a row is not there."""
    def refused(text, **kw):
        assert B.lib().metok_decode_attention(*attention_args(**kw)) == -1, kw
        assert text in B.metok_last_error(), (kw, B.metok_last_error())

    for x in (1e-40, 1e-50, 5e-324, 1e30):
        refused("scale must", scale=x)
        refused("logit_cap must", cap=x)
    refused("scale / logit_cap", scale=1e10, cap=1e-25)


def test_quotients_of_scale_and_cap_that_fp32_does_not_hold_are_refused(B):
    """The kernels take tanh of q . k times scale / logit_cap: below fp32's range that factor would lose its bits or be 0, and all scores with it."""
    for scale, cap in ((1e-25, 1e25), (1e-30, 1.1), (1e-10, 1.1e20), (1e-9, 9e29), (1.01, 1e-30), (1e25, 1e-5)):
        assert B.lib().metok_decode_attention(*attention_args(scale=scale, cap=cap)) == -1, (scale, cap)
        assert "scale / logit_cap must" in B.metok_last_error(), B.metok_last_error()
    for scale, cap in ((1e-30, 1.0), (1e-10, 1e20), (0.125, 9e28), (1e25, 1.1e-5)):         # taken: the workspace is what is missing
        assert B.lib().metok_decode_attention(*attention_args(scale=scale, cap=cap)) == -3, (scale, cap, B.metok_last_error())


def test_one_cache_for_keys_and_values_is_not_appended_to(B):
    f = B.lib().metok_decode_attention
    for v in (FAKE[1], FAKE[1] + 16):
        assert f(*attention_args(v=v, bytes=1 << 40)) == -1 and "overlaps" in B.metok_last_error()
    for name in ("out", "lse", "weight", "q", "len", "ws"):                                # and nothing else lies in it when it is only read
        assert f(*attention_args(v=FAKE[1], k_new=None, v_new=None, bytes=1 << 40, **{name: FAKE[1]})) == -1 and "overlaps" in B.metok_last_error(), name


def test_refused_paged_attention_calls(B):
    f = B.lib().metok_decode_attention_paged

    def refused(code, text, **kw):
        a = dict(q=FAKE[0], B=2, Hq=8, Hkv=2, dh=64, dtype=1, k=FAKE[1], v=FAKE[2], n_pages=20, page=16, table=FAKE[11], pps=8, len=FAKE[3], k_new=None, v_new=None,
                 scale=0.125, cap=0.0, out=FAKE[6], lse=None, weight=None, stride=0, ws=FAKE[9], bytes=0, stream=None)
        a.update(kw)
        assert f(*a.values()) == code, kw
        assert text in B.metok_last_error(), (kw, B.metok_last_error())

    refused(-3, "workspace", pps=80)
    refused(-1, "page_table", table=None)
    refused(-1, "page_table", table=FAKE[11] + 1)
    for name in ("n_pages", "page", "pps"):
        refused(-1, "positive", **{name: 0})
    refused(-1, "capacity", page=2 ** 20, pps=2 ** 20)
    refused(-2, "below 2^31", n_pages=2 ** 40, pps=80)
    refused(-2, "below 2^31", n_pages=2 ** 31 // 32 + 1, pps=80)
    refused(-1, "overlaps", table=FAKE[1], bytes=1 << 40)


def test_workspace_sizes(B):
    f = B.metok_decode_attention_workspace_bytes
    assert f(1, 28, 4, 31, 128, B.BF16) == 0                            # one tile per kv head: nothing to join
    small, big = f(8, 28, 4, 36992, 128, B.BF16), f(8, 28, 4, 36992, 128, B.BF16, True)
    assert 0 < small < 24 << 20
    assert big - small >= 8 * 28 * 36993 * 4                            # the logits
    assert f(8, 28, 4, 36992, 128, B.F32) > 0
    for bad in ((0, 28, 4, 100, 128, 1), (1, 28, 5, 100, 128, 1), (1, 28, 4, 0, 128, 1), (1, 28, 4, 100, 48, 1), (1, 28, 4, 100, 256, 0), (1, 28, 4, 100, 128, 7)):
        assert f(*bad) == 0


def test_the_workspace_of_partial_results(B):
    """Two of a maximum, a sum and an output in fp32 for each of 1024 waves (2048 where a tile of K and V is 4 KB) and each query head that it takes at a
    time, whatever the batch and the capacity: 67.6 MB at most; and 8 bytes per (video, kv head, turn of its query heads)."""
    f, most = B.metok_decode_attention_workspace_bytes, 0
    for dtype, dh in ((B.BF16, 32), (B.BF16, 64), (B.BF16, 128), (B.BF16, 256), (B.F32, 32), (B.F32, 64), (B.F32, 128)):
        waves = 2048 if dh == 32 else 1024
        for group in (1, 7, 16, 17, 31, 32, 33, 40, 64, 65, 128, 1000, 1024):
            turn = 16 if group <= 16 else 64 if dh <= 64 and group > 32 else 32
            parts = 2 * waves * min(group, turn) * (dh + 2) * 4
            most = max(most, parts)
            for videos, capacity in ((1, 5000), (8, 100000), (64, 5000)):
                pairs = videos * -(-group // turn)
                assert f(videos, group, 1, capacity, dh, dtype) == parts + -(-8 * pairs // 256) * 256, (dtype, dh, group)
    assert most == 2 * 1024 * 32 * 258 * 4 == 67633152


PLAN = r"""
#include <initializer_list>
#include "decode_plan.h"
using namespace metok;
extern "C" void attend_plan(int B, int Hq, int Hkv, int64_t cap, int dh, int esize, int w, int64_t* o) {
    const AttendPlan p = plan_attend(B, Hq, Hkv, cap, dh, esize, w != 0);
    for (int64_t v : {int64_t(p.tile), int64_t(p.row_blocks), int64_t(p.block_rows), int64_t(p.rows), p.pairs, p.grid, p.workers, int64_t(p.joined), p.logit_stride, int64_t(p.pair_workers),
                      int64_t(p.part_ml), int64_t(p.part_o), int64_t(p.lse2), int64_t(p.logits), int64_t(p.bytes), int64_t(attend_groups(esize, dh)), int64_t(p.whole)}) *o++ = v;
}
extern "C" int64_t workers(int groups, int64_t units) { return groups == 512 ? Deal<512>::workers(units) : Deal<256>::workers(units); }
extern "C" int64_t first(int groups, int64_t w, int64_t units) { return groups == 512 ? Deal<512>::first(w, units) : Deal<256>::first(w, units); }
extern "C" int pair_cost() { return kAttendPairCost; }
"""


def plan_library():
    lib = host_library(PLAN)
    i, q = ctypes.c_int, ctypes.c_int64
    lib.workers.restype, lib.workers.argtypes = q, [i, q]
    lib.first.restype, lib.first.argtypes = q, [i, q, q]
    return lib


@pytest.mark.parametrize("groups", [256, 512])
def test_units_are_dealt_out_evenly(groups):
    """Every unit has one worker, no worker is without a unit, and none has more than the even share rounded up (the few that there
    are in a small call: two)."""
    lib = plan_library()
    rng = random.Random(groups)
    for total in [1, 2, 3, 255, 1023, 1024, 1025, 2047, 2048, 4095, 4096, 4097, 2 ** 31 - 1] + [rng.randint(1, 20000) for _ in range(40)]:
        n = lib.workers(groups, total)
        assert 1 <= n <= min(total, 4 * groups)
        firsts = [lib.first(groups, w, total) for w in range(n + 1)]
        sizes = [b - a for a, b in zip(firsts, firsts[1:])]
        assert firsts[0] == 0 and firsts[-1] == total and min(sizes) >= 1 and max(sizes) <= max(2, -(-total // (4 * groups)))
        assert lib.first(groups, n, total) == lib.first(groups, 4 * groups, total) == total


@pytest.mark.parametrize("seed", range(4))
def test_partial_results_have_slots_of_their_own(seed):
    """Whatever the lengths, as the kernel goes through them: every tile has one worker, two parts of results never share a slot, all slots
    are in the workspace, calls that are not joined have no parts, and the regions of the workspace lie one behind the other."""
    lib = plan_library()
    cost = lib.pair_cost()
    rng = random.Random(seed)
    for _ in range(60):
        Hq, Hkv = rng.choice([(28, 4), (40, 40), (71, 1), (17, 1), (8, 8), (1, 1), (1024, 2)])
        Bn = rng.choice([1, 2, 8, 64, 65, 300])
        esize, dh = rng.choice([(2, 128), (4, 64), (2, 256), (2, 32), (4, 32)])
        cap = int(2 ** rng.uniform(0, 13))
        w = rng.randint(0, 1)
        o = (ctypes.c_int64 * 17)()
        lib.attend_plan(Bn, Hq, Hkv, ctypes.c_int64(cap), dh, esize, w, o)
        tile, row_blocks, block_rows, rows, pairs, grid, most_workers, joined, stride, table, ml, part, lse2, logits, total, groups, whole = list(o)
        heads = Hkv * row_blocks
        if whole:                                                        # a workgroup to a pair: nothing is left for another one
            assert not w and Hq // Hkv <= 16 and total == 0 and not joined
            assert -(-(cap + 1) // tile) <= 32 and pairs == Bn * Hkv
            continue
        assert pairs == Bn * heads and block_rows * row_blocks >= Hq // Hkv > (row_blocks - 1) * block_rows and rows == min(block_rows, Hq // Hkv) and most_workers == 4 * groups
        slots = (part - ml) // (rows * 2 * 4)
        for kind in range(4):
            fresh = rng.randint(0, 1)
            lens = [cap if kind == 0 else (0 if kind == 1 else rng.randint(0, cap) if kind == 2 or rng.random() < 0.02 else min(cap, 3)) for _ in range(Bn)]
            tiles = [max(1, -(-(n + fresh) // tile)) for n in lens]
            units = sum(t + cost for t in tiles) * heads
            n = lib.workers(groups, units)
            # workers are spread over the workgroups first: worker = wave * grid + workgroup
            assert n <= 4 * grid and (grid == groups or n <= grid)
            firsts = [lib.first(groups, x, units) for x in range(n + 1)]
            used, at, x = set(), 0, 0
            for t in tiles:
                for _ in range(heads):
                    mine = set()
                    for unit in range(at, at + t):
                        while firsts[x + 1] <= unit:
                            x += 1
                        mine.add(x)
                    mine = sorted(mine)
                    assert mine == list(range(mine[0], mine[-1] + 1))
                    if len(mine) > 1:
                        assert joined
                        mine = [2 * v + (v == mine[0]) for v in mine]
                        assert not used & set(mine) and max(mine) < slots
                        used |= set(mine)
                    at += t + cost
        if joined or w:
            assert ml - table >= pairs * 8
        if joined:
            assert lse2 - part >= slots * rows * dh * 4
        if w:
            assert stride >= cap + 1 and stride % 32 == 0 and logits - lse2 >= Bn * Hq * 4 and total - logits == -(-Bn * Hq * stride * 4 // 256) * 256
        else:
            assert logits == total


def evict_args(**kw):
    vp, i32 = ctypes.c_void_p, ctypes.c_int32
    a = dict(k=(vp * 2)(FAKE[0], FAKE[1]), v=(vp * 2)(FAKE[2], FAKE[3]), L=2, B=2, Hkv=2, S_cap=128, dh=64, dtype=1,
             weight=(vp * 2)(FAKE[4], FAKE[5]), weight_out=(vp * 2)(FAKE[6], FAKE[7]), stride=128, len=FAKE[8], budget=(i32 * 2)(64, 64), first=4, last=8,
             idx=(vp * 2)(FAKE[9], FAKE[10]), new_len=FAKE[11], ws=FAKE[12], bytes=0, stream=None)
    a.update(kw)
    return a


def test_refused_evictions(B):
    vp, i32 = ctypes.c_void_p, ctypes.c_int32

    def refused(code, text, **kw):
        a = evict_args(**kw)
        assert B.lib().metok_kv_evict(*a.values()) == code, kw
        assert text in B.metok_last_error(), (kw, B.metok_last_error())
        if code == -1 and not {"k", "v", "dtype", "dh", "Hkv"} & set(kw):
            b = [a[n] for n in ("weight", "weight_out", "stride", "L", "B", "S_cap", "len", "budget", "first", "last", "idx", "new_len", "stream")]
            assert B.lib().metok_kv_evict_select(*b) == code and text in B.metok_last_error()

    refused(-3, "workspace")
    refused(-3, "workspace", ws=None, bytes=1 << 30)
    for n in (0, -1, 129):
        refused(-1, "L must", L=n)
    for n in (0, 4097):
        refused(-1, "B must", B=n)
    for n in (0, 2 ** 31):
        refused(-1, "capacity", S_cap=n, stride=2 ** 40)
    for name in ("weight", "weight_out", "len", "budget", "idx", "new_len"):
        refused(-1, "NULL", **{name: None})
    refused(-1, "aligned", len=FAKE[8] + 1)
    refused(-1, "misaligned", weight=(vp * 2)(FAKE[4], FAKE[5] + 2))
    refused(-1, "NULL or misaligned", weight_out=(vp * 2)(FAKE[6], None))
    refused(-1, "NULL or misaligned", idx=(vp * 2)(FAKE[9], FAKE[10] + 1))
    refused(-1, "overlaps", weight_out=(vp * 2)(FAKE[4] + 64, FAKE[5]))
    refused(-1, "overlaps", new_len=FAKE[8] + 8)
    refused(-1, "weight_stride", stride=127)
    refused(-1, "budget", budget=(i32 * 2)(64, 0))
    refused(-1, "budget", budget=(i32 * 2)(129, 64))
    refused(-1, "more than budget", first=60)
    refused(-1, "more than budget", first=2 ** 31 - 1, last=2 ** 31 - 1)
    refused(-1, "negative", last=-1)
    refused(-1, "dtype", dtype=5)
    refused(-1, "multiple of 16", dh=4)
    refused(-1, "layer 1", k=(vp * 2)(FAKE[0], None))
    refused(-1, "layer 0", v=(vp * 2)(FAKE[2] + 8, FAKE[3]))

    def paged(code, text, **kw):
        a = evict_args(**kw)
        args = [a[n] for n in ("k", "v", "L", "B", "Hkv")] + [kw.get("pages", 40), kw.get("page", 16), a["dh"], a["dtype"], kw.get("table", FAKE[13]), kw.get("pps", 8)]
        args += [a[n] for n in ("weight", "weight_out", "stride", "len", "budget", "first", "last", "idx", "new_len", "ws", "bytes", "stream")]
        assert B.lib().metok_kv_evict_paged(*args) == code and text in B.metok_last_error(), (kw, B.metok_last_error())

    paged(-3, "workspace")
    paged(-1, "page_table", table=None)
    paged(-1, "positive", page=0)
    paged(-1, "positive", pps=0)
    paged(-1, "positive", pages=0)
    paged(-1, "capacity", page=2 ** 20, pps=2 ** 20)


def test_evictions_whose_buffers_overlap_are_refused(B):
    vp, i32 = ctypes.c_void_p, ctypes.c_int32
    names = ("weight", "weight_out", "stride", "L", "B", "S_cap", "len", "budget", "first", "last", "idx", "new_len", "stream")

    def refused(**kw):
        a = evict_args(**kw)
        assert B.lib().metok_kv_evict_select(*[a[n] for n in names]) == -1, kw
        assert "overlaps" in B.metok_last_error(), (kw, B.metok_last_error())
        assert B.lib().metok_kv_evict(*a.values()) == -1 and "overlaps" in B.metok_last_error()

    same = (vp * 2)(FAKE[4], FAKE[4])
    refused(weight=same, weight_out=same)                                # one buffer for two layers, in place
    refused(weight_out=(vp * 2)(FAKE[6], FAKE[6] + 4 * 255))             # the second layer's from the last word of the first's
    refused(weight_out=(vp * 2)(FAKE[5], FAKE[7]))                       # the first layer's onto the second's weights
    refused(idx=(vp * 2)(FAKE[9], FAKE[9]))
    refused(idx=(vp * 2)(FAKE[9], FAKE[9] + 4 * 127))
    refused(idx=(vp * 2)(FAKE[4], FAKE[10]))
    refused(idx=(vp * 2)(FAKE[9], FAKE[7] + 4))
    refused(idx=(vp * 2)(FAKE[9], FAKE[8]))
    refused(new_len=FAKE[10] + 4)
    # neighbours, weights that two layers share, and layers without weights: no overlap; the workspace is what is missing
    for kw in (dict(weight_out=(vp * 2)(FAKE[6], FAKE[6] + 4 * 256)), dict(idx=(vp * 2)(FAKE[9], FAKE[9] + 4 * 128)), dict(weight=same),
               dict(weight=(vp * 2)(FAKE[4], None), weight_out=(vp * 2)(FAKE[6], FAKE[6]), idx=(vp * 2)(FAKE[9], FAKE[9])),
               dict(weight_out=(vp * 2)(FAKE[4], FAKE[5])), dict(new_len=FAKE[8])):
        a = evict_args(**kw)
        assert B.lib().metok_kv_evict(*a.values()) == -3, (kw, B.metok_last_error())


def test_eviction_workspace(B):
    f = B.metok_kv_evict_workspace_bytes
    assert f(28, 8, 4, 36992, 128, B.BF16) == B.metok_kv_compact_workspace_bytes(28, 8, 4, 36992, 128, B.BF16) + 28 * 8 * 8
    assert f(28, 4097, 4, 128, 128, B.BF16) == 0 and f(28, 8, 4, 36992, 12, B.BF16) == 0


def test_the_oracles_eviction_by_hand():
    from oracle import decode_oracle as D
    w = [5.0, 1.0, 3.0, 3.0, 0.0, 3.0, 2.0, 9.0]
    assert D.evict(w, 8, 8, 0, 0) == list(range(8))
    assert D.evict(w, 8, 4, 0, 0) == [0, 2, 3, 7]                # of the three 3s the first two
    assert D.evict(w, 8, 4, 2, 1) == [0, 1, 2, 7]
    assert D.evict(w, 8, 3, 1, 2) == [0, 6, 7]
    assert D.evict(w, 3, 4, 0, 0) == [0, 1, 2]
    assert D.index_list([0, 1], 4).tolist() == [0, 1, 2, 3]


def test_the_oracles_attention_by_hand():
    import numpy as np
    from oracle import decode_oracle as D
    out, lse, p = D.attend([1.0, 0.0], [[0.0, 5.0], [np.log(3.0), 1.0]], [[1.0, 0.0], [0.0, 1.0]], 1.0)
    np.testing.assert_allclose(p, [0.25, 0.75])
    np.testing.assert_allclose(out, [0.25, 0.75])
    assert abs(lse - np.log(4.0)) < 1e-12
    _, lse, p = D.attend([1.0, 0.0], [[1e9, 0.0], [-1e9, 0.0]], [[1.0, 0.0], [0.0, 1.0]], 1.0, cap=2.0)
    np.testing.assert_allclose(p, [1 / (1 + np.exp(-4.0)), 1 / (1 + np.exp(4.0))])
    out, lse, p = D.attend([1.0, 0.0], np.zeros((0, 2)), np.zeros((0, 2)), 1.0)
    assert not out.any() and lse == -np.inf
    q = np.random.default_rng(0).standard_normal((1, 4, 8))
    k = np.random.default_rng(1).standard_normal((200, 2, 8))
    out, lse, mean = D.decode_attention(q, [k], [k], 0.3)
    t = torch.from_numpy(np.repeat(k.transpose(1, 0, 2), 2, axis=0))[None]
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q)[:, :, None], t, t, scale=0.3)[:, :, 0]
    np.testing.assert_allclose(out, want.numpy(), rtol=1e-12, atol=1e-14)
    assert abs(mean[0].sum() - 1) < 1e-12
