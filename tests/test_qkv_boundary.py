"""CPU checks of the calls around queries, keys and values: exports, sizes, refusals before anything reaches a GPU, the split over a 4-bit cache, and the
oracle by hand."""
import ctypes
import math
import os
import random
import re
import subprocess

import numpy as np
import pytest
import torch  # noqa: F401  (loaded first so that the library binds to the same HIP runtime)

from oracle import qkv_oracle as Q
from tests import kv4_large as large
from tests.host_plan import host_library

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "metok_qkv.h")


@pytest.fixture(scope="module")
def B():
    from paper_2506_02850_amd import build
    if not os.path.exists(build.LIB):
        build.build(verbose=False)
    from paper_2506_02850_amd import binding
    return binding


def test_every_declared_symbol_is_exported_and_bound(B):
    names = re.findall(r"METOK_API\s+[\w\s\*]+?\b(metok_\w+)\s*\(", open(HEADER).read())
    assert len(set(names)) == len(names) and sorted(names) == sorted(B.QKV_EXPORTS)
    for name in names:
        assert hasattr(B.lib(), name) and callable(getattr(B, name)), name


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "x.c"
    src.write_text('#include "metok_qkv.h"\nint main(void) { return METOK_MAX_POSITION_AXES == 4 ? METOK_PAIRS_HALVES : 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "x.o")], check=True)


FAKE = [0x10000000 * (i + 1) for i in range(24)]        # aligned, far apart, never dereferenced: validation fails first


class Refused:
    """Calls one entry point with one argument after the other wrong."""

    def __init__(self, B, name, defaults):
        self.B, self.f, self.defaults = B, getattr(B.lib(), name), defaults

    def __call__(self, code, text, **kw):
        assert not set(kw) - set(self.defaults), kw
        assert self.f(*{**self.defaults, **kw}.values()) == code, (kw, self.B.metok_last_error())
        assert text in self.B.metok_last_error(), (kw, self.B.metok_last_error())


ROTATE = dict(q=FAKE[0], k=FAKE[1], v=FAKE[2], qs=512, ks=128, vs=128, B=2, n=5, Hq=8, Hkv=2, dh=64, dtype=1, count=FAKE[3], qw=FAKE[4], kw=FAKE[5], eps=1e-6,
              pos=FAKE[6], axes=3, freq=FAKE[7], axis=bytes([0, 1, 2] * 10 + [0, 1]), rot=64, pairs=0, q_out=FAKE[8], kc=FAKE[9], vc=FAKE[10])
DENSE, PAGED = dict(S_cap=128, start=FAKE[11], stream=None), dict(n_pages=20, page=16, table=FAKE[12], pps=8, start=FAKE[11], stream=None)


@pytest.mark.parametrize("paged", [False, True])
def test_refused_rotations(B, paged):
    refused = Refused(B, "metok_rotate_qk_paged" if paged else "metok_rotate_qk", {**ROTATE, **(PAGED if paged else DENSE)})
    refused(-1, "dtype", dtype=2)
    for dh in (0, 16, 96, 512):
        refused(-1, "dh must", dh=dh)
    refused(-1, "dh must", dh=256, dtype=0)
    for n in (0, -1, 4097):
        refused(-1, "B must", B=n)
    for n in (0, -1, 2 ** 26 + 1, 2 ** 62):
        refused(-1, "n must", n=n)
    for kw in (dict(Hq=0), dict(Hkv=0), dict(Hq=-1), dict(Hkv=-3), dict(Hq=4093), dict(Hkv=2045), dict(Hq=2 ** 31 - 1), dict(Hkv=2 ** 31 - 1)):
        if not (paged and kw.get("Hkv", 1) > 10 ** 6):
            refused(-1, "Hq and Hkv must", **kw)
    for name in ("q", "k", "v", "pos", "freq", "q_out", "kc", "vc"):
        refused(-1, "NULL", **{name: None})
    refused(-1, "go together", qw=None)
    refused(-1, "go together", kw=None)
    for name in ("q", "k", "v", "qw", "kw", "freq", "q_out", "kc", "vc"):
        refused(-1, "16-byte aligned", **{name: FAKE[20] + 8})
    for name in ("pos", "count", "start"):
        refused(-1, "4-byte aligned", **{name: FAKE[20] + 2})
    for eps in (-1e-9, float("nan"), 1.5, float("inf")):
        refused(-1, "eps", eps=eps)
    for n in (0, 5, -1):
        refused(-1, "n_axes", axes=n)
    for rot in (0, -16, 8, 24, 80):
        refused(-1, "rot must", rot=rot)
    refused(-1, "pairs", pairs=2)
    refused(-1, "pair_axis[2]", axes=2)
    refused(-1, "pair_axis[31]", axis=bytes(31) + b"\x03")
    for name, least in (("qs", 512), ("ks", 128), ("vs", 128)):
        long = {"qs": "q", "ks": "k", "vs": "v"}[name] + "_stride"
        for s in (least - 8, least + 4, 0, -512, 2 ** 40):
            refused(-1, long, **{name: s})
    for kw in (dict(q_out=FAKE[0]), dict(q_out=FAKE[0] + 16 * 100), dict(kc=FAKE[8]), dict(vc=FAKE[9]), dict(vc=FAKE[9] + 64), dict(kc=FAKE[1]), dict(vc=FAKE[2]), dict(q_out=FAKE[3]),
               dict(kc=FAKE[4]), dict(kc=FAKE[5]), dict(vc=FAKE[6]), dict(q_out=FAKE[7]), dict(vc=FAKE[11])):
        refused(-1, "overlaps", **kw)
    if paged:
        refused(-1, "page_table", table=None)
        refused(-1, "page_table", table=FAKE[12] + 1)
        for name in ("n_pages", "page", "pps"):
            refused(-1, "positive", **{name: 0})
        refused(-1, "capacity", page=2 ** 20, pps=2 ** 20)
        refused(-2, "below 2^31", n_pages=2 ** 40)
        refused(-1, "overlaps", table=FAKE[9])
    else:
        for s in (0, -5, 2 ** 31 - 64, 2 ** 40):
            refused(-1, "capacity", S_cap=s)


PACK = dict(k=FAKE[0], v=FAKE[1], B=2, Hkv=2, S_src=100, dh=64, dtype=1, idx=FAKE[2], n=50, count=FAKE[3], kc=FAKE[4], vc=FAKE[5])


@pytest.mark.parametrize("paged", [False, True])
def test_refused_packing(B, paged):
    refused = Refused(B, "metok_kv4_pack_paged" if paged else "metok_kv4_pack", {**PACK, **(PAGED if paged else DENSE)})
    refused(-1, "dtype", dtype=-1)
    for n in (0, 4097):
        refused(-1, "B must", B=n)
    for n in (0, -2, 1025):
        refused(-1, "Hkv must", Hkv=n)
    for dh in (0, 16, 96, 512):
        refused(-1, "dh must", dh=dh)
    for s in (0, -1, 2 ** 31 - 64):
        refused(-1, "rows of a video", S_src=s)
    for n in (0, -1, 2 ** 29 + 1):
        refused(-1, "n must", n=n)
    refused(-1, "at most S_src", idx=None, n=101)
    for name in ("k", "v", "kc", "vc"):
        refused(-1, "NULL", **{name: None})
        refused(-1, "16-byte aligned", **{name: FAKE[20] + 8})
    for name in ("idx", "count", "start"):
        refused(-1, "4-byte aligned", **{name: FAKE[20] + 2})
    for kw in (dict(vc=FAKE[4]), dict(vc=FAKE[4] + 32), dict(kc=FAKE[0]), dict(kc=FAKE[1]), dict(vc=FAKE[2]), dict(vc=FAKE[3]), dict(kc=FAKE[11])):
        refused(-1, "overlaps", **kw)
    check_pages_or_capacity(refused, paged, FAKE[4])


UNPACK_HEAD = dict(kc=FAKE[0], vc=FAKE[1], B=2, Hkv=2)
UNPACK_TAIL = dict(len=FAKE[2], first=FAKE[3], idx=None, n=50, k=FAKE[4], v=FAKE[5], S_out=60, dtype=1, stream=None)


@pytest.mark.parametrize("paged", [False, True])
def test_refused_unpacking(B, paged):
    middle = dict(n_pages=20, page=16, dh=64, table=FAKE[12], pps=8) if paged else dict(S_cap=128, dh=64)
    refused = Refused(B, "metok_kv4_unpack_paged" if paged else "metok_kv4_unpack", {**UNPACK_HEAD, **middle, **UNPACK_TAIL})
    refused(-1, "dtype", dtype=2)
    for n in (0, 4097):
        refused(-1, "B must", B=n)
    refused(-1, "Hkv must", Hkv=0)
    refused(-1, "dh must", dh=48)
    refused(-1, "rows of a video", S_out=0)
    refused(-1, "n must", n=0)
    refused(-4, "S_out", n=61)
    refused(-1, "do not go together", idx=FAKE[6])
    for name in ("kc", "vc", "len", "k", "v"):
        refused(-1, "NULL", **{name: None})
    for name in ("kc", "vc", "k", "v"):
        refused(-1, "16-byte aligned", **{name: FAKE[20] + 8})
    for name in ("len", "first"):
        refused(-1, "4-byte aligned", **{name: FAKE[20] + 2})
    for kw in (dict(v=FAKE[4]), dict(k=FAKE[0]), dict(v=FAKE[1] + 16), dict(k=FAKE[2]), dict(v=FAKE[3]), dict(k=FAKE[6], idx=FAKE[6], first=None)):
        refused(-1, "overlaps", **kw)
    check_pages_or_capacity(refused, paged, FAKE[4])


def check_pages_or_capacity(refused, paged, written, **more):
    if paged:
        refused(-1, "page_table", table=None)
        refused(-1, "page_table", table=FAKE[12] + 2)
        for name in ("n_pages", "page", "pps"):
            refused(-1, "positive", **{name: 0})
        for page in (1, 8, 24, 1000):
            refused(-1, "multiple of 16", page=page)
        refused(-1, "capacity", page=2 ** 20, pps=2 ** 20)
        refused(-2, "below 2^31", n_pages=2 ** 40)
        refused(-1, "overlaps", table=written, **more)
    else:
        for s in (0, -16, 8, 24, 2 ** 31 - 64, 2 ** 40):
            refused(-1, "capacity", S_cap=s)


ATTEND_HEAD = dict(q=FAKE[0], B=2, Hq=8, Hkv=2, dh=64, dtype=1, k=FAKE[1], v=FAKE[2])
ATTEND_TAIL = dict(len=FAKE[3], k_new=FAKE[4], v_new=FAKE[5], scale=0.125, cap=0.0, out=FAKE[6], lse=FAKE[7], weight=FAKE[8], stride=1 << 20, ws=FAKE[9], bytes=0, stream=None)


@pytest.mark.parametrize("paged", [False, True])
def test_refused_attention(B, paged):
    middle = dict(n_pages=20, page=16, table=FAKE[12], pps=8) if paged else dict(S_cap=128)
    refused = Refused(B, "metok_kv4_attention_paged" if paged else "metok_kv4_attention", {**ATTEND_HEAD, **middle, **ATTEND_TAIL})
    big = dict(bytes=1 << 40)
    refused(-3, "workspace")
    refused(-3, "workspace", ws=None, **big)
    refused(-3, "workspace", ws=FAKE[9] + 8, **big)
    for name in ("q", "k", "v", "len", "out"):
        refused(-1, "NULL", **{name: None})
    refused(-1, "go together", k_new=None)
    for name in ("q", "k", "v", "k_new", "v_new", "out"):
        refused(-1, "aligned", **{name: FAKE[20] + 8})
    for name in ("len", "lse", "weight"):
        refused(-1, "aligned", **{name: FAKE[20] + 2})
    for x in (0.0, -1.0, float("nan"), float("inf"), 1e-40):
        refused(-1, "scale", scale=x)
    for x in (-1.0, float("nan"), float("inf"), 1e-40):
        refused(-1, "logit_cap", cap=x)
    refused(-1, "scale / logit_cap", scale=1e-25, cap=1e25)
    refused(-1, "weight_stride", stride=127)
    refused(-1, "dtype", dtype=2)
    refused(-1, "B must", B=0)
    refused(-1, "Hq must", Hq=7)
    refused(-1, "Hq must", Hq=1026)
    refused(-1, "dh must", dh=96)
    refused(-1, "dh must", dh=256, dtype=0)
    for kw in (dict(out=FAKE[0]), dict(lse=FAKE[6]), dict(v=FAKE[1]), dict(k_new=FAKE[1] + 64), dict(weight=FAKE[3]), dict(ws=FAKE[2]), dict(out=FAKE[2] + 16)):
        refused(-1, "overlaps", **kw, **big)
    check_pages_or_capacity(refused, paged, FAKE[1], **big)
    if not paged:
        refused(-1, "too many rows", B=4096, S_cap=2 ** 30, stride=2 ** 41)


def test_sizes(B):
    for dh in (32, 64, 128, 256):
        assert B.metok_kv4_cache_bytes(3, 5, 48, dh) == 3 * 5 * 3 * Q.block_bytes(dh) == 3 * 5 * 48 * dh * 17 // 32
    for bad in ((0, 1, 16, 64), (1, 0, 16, 64), (1, 1, 0, 64), (1, 1, 24, 64), (1, 1, 16, 48), (2 ** 31, 1, 16, 64)):
        assert B.metok_kv4_cache_bytes(*bad) == 0
    f = B.metok_kv4_attention_workspace_bytes
    assert f(1, 28, 4, 48, 128, B.BF16) == 0                            # one tile per kv head, and one launch
    assert 0 < f(8, 28, 4, 36992, 128, B.BF16) < 24 << 20
    assert f(8, 28, 4, 36992, 128, B.BF16, True) - f(8, 28, 4, 36992, 128, B.BF16) >= 8 * 28 * 36993 * 4
    for bad in ((0, 28, 4, 96, 128, 1), (1, 28, 5, 96, 128, 1), (1, 28, 4, 100, 128, 1), (1, 28, 4, 96, 48, 1), (1, 28, 4, 96, 256, 0), (1, 28, 4, 96, 128, 7)):
        assert f(*bad) == 0


PLAN = r"""
#include <initializer_list>
#include "decode_plan.h"
using namespace metok;
extern "C" void attend_plan(int B, int Hq, int Hkv, int64_t cap, int dh, int w, int64_t* o) {
    const AttendPlan p = plan_attend4(B, Hq, Hkv, cap, dh, w != 0);
    for (int64_t v : {int64_t(p.tile), int64_t(p.row_blocks), int64_t(p.block_rows), int64_t(p.rows), p.pairs, p.grid, p.workers, int64_t(p.joined), p.logit_stride, int64_t(p.pair_workers),
                      int64_t(p.part_ml), int64_t(p.part_o), int64_t(p.lse2), int64_t(p.logits), int64_t(p.bytes), int64_t(p.whole)}) *o++ = v;
}
typedef Deal4 D;
extern "C" int64_t workers(int64_t units) { return D::workers(units); }
extern "C" int64_t first(int64_t w, int64_t units) { return D::first(w, units); }
extern "C" int pair_cost() { return kAttend4PairCost; }
extern "C" int most_whole() { return kAttend4Whole; }
extern "C" int middle(int64_t w, int64_t units, int64_t t, int64_t tiles) { return D::in_the_middle(w, units, t, tiles); }
extern "C" int parts(int first, int last, int* slots) {
    const PairParts p = pair_parts(first, last, true);
    for (int i = 0; i < p.n; ++i) slots[i] = p.slot(i);
    return p.n;
}
"""


@pytest.mark.parametrize("seed", range(4))
def test_partial_results_have_slots_of_their_own(seed):
    """Every tile has one worker, two parts of results never share a slot, all slots are in the workspace, calls that are not joined have no parts, whole
    tiles of logits fit, and the workspace's regions lie one behind the other."""
    lib = host_library(PLAN)
    q = ctypes.c_int64
    lib.workers.restype, lib.workers.argtypes, lib.first.restype, lib.first.argtypes = q, [q], q, [q, q]
    cost, rng = lib.pair_cost(), random.Random(seed)
    for _ in range(50):
        Hq, Hkv = rng.choice([(28, 4), (40, 40), (71, 1), (17, 1), (8, 8), (1, 1), (1024, 2)])
        Bn, dh = rng.choice([1, 2, 8, 64, 65, 300]), rng.choice([32, 64, 128, 256])
        cap, w = 16 * int(2 ** rng.uniform(0, 10)), rng.randint(0, 1)
        o = (q * 16)()
        lib.attend_plan(Bn, Hq, Hkv, q(cap), dh, w, o)
        tile, row_blocks, block_rows, rows, pairs, grid, most_workers, joined, stride, table, ml, part, lse2, logits, total, whole = list(o)
        assert tile % 32 == 0
        if whole:
            assert not w and Hq // Hkv <= 16 and total == 0 and not joined and -(-(cap + 1) // tile) <= lib.most_whole() and pairs == Bn * Hkv
            continue
        heads = Hkv * row_blocks
        assert pairs == Bn * heads and block_rows * row_blocks >= Hq // Hkv > (row_blocks - 1) * block_rows and rows == min(block_rows, Hq // Hkv)
        slots = (part - ml) // (rows * 2 * 4)
        for kind in range(4):
            fresh = rng.randint(0, 1)
            lens = [cap if kind == 0 else (0 if kind == 1 else rng.randint(0, cap) if kind == 2 or rng.random() < 0.02 else min(cap, 3)) for _ in range(Bn)]
            tiles = [max(1, -(-(n + fresh) // tile)) for n in lens]
            units = sum(t + cost for t in tiles) * heads
            n = lib.workers(units)
            assert n <= 4 * grid
            firsts = [lib.first(x, units) for x in range(n + 1)]
            assert firsts[0] == 0 and firsts[-1] == units
            used, at, x = set(), 0, 0
            for t in tiles:
                for _ in range(heads):
                    mine = set()
                    for unit in range(at, at + t):
                        while firsts[x + 1] <= unit:
                            x += 1
                        mine.add(x)
                    mine = sorted(mine)
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
            assert stride >= -(-(cap + 1) // tile) * tile and stride % 4 == 0 and logits - lse2 >= Bn * Hq * 4 and total - logits == -(-Bn * Hq * stride * 4 // 256) * 256
        else:
            assert logits == total


@pytest.mark.parametrize("seed", range(4))
def test_the_join_finds_what_workgroups_in_the_middle_of_a_pair_leave(seed):
    """The kernel's loop over tiles, with a set of tiles for a result: all workers of a workgroup agree whether it is in the middle, every part is written once,
    and the parts that the join reads are the pair's tiles, each once."""
    lib = host_library(PLAN)
    q = ctypes.c_int64
    lib.first.restype, lib.first.argtypes, lib.middle.argtypes = q, [q, q], [q, q, q, q]
    cost, rng, waves, most = lib.pair_cost(), random.Random(seed), 4, 2048
    for kind in range(6):
        longest, n = [(60000, 3), (9000, 1), (300, 40), (40, 200), (3, 2000), (5000, 16)][kind]
        tiles = [rng.choice([1, rng.randint(1, longest), rng.randint(1, longest), longest]) for _ in range(n)]
        begin = [0]
        for t in tiles:
            begin.append(begin[-1] + t + cost)
        units, written, workers, pair = begin[-1], {}, [[None, None] for _ in tiles], 0
        for group in range(0, most, waves):
            teams, left_over = set(), []
            for w in range(group, group + waves):
                at, end = lib.first(w, units), lib.first(w + 1, units)
                if at >= end:
                    teams.add(False)
                    continue
                while begin[pair + 1] <= at:
                    pair += 1
                i, t = pair, at - begin[pair]
                team = bool(lib.middle(w, units, t, tiles[i]))
                teams.add(team)
                if t >= tiles[i]:
                    at, i, t = begin[i + 1], i + 1, 0
                while at < end:                            # a pair, or the worker's part of it
                    stop = min(end - begin[i], tiles[i])
                    have = range(t, stop)
                    if team:
                        left_over.append((i, have))
                    else:
                        if t == 0:
                            workers[i][0] = w
                        if stop == tiles[i]:
                            workers[i][1] = w
                        if len(have) < tiles[i]:
                            assert 2 * w + (t == 0) not in written
                            written[2 * w + (t == 0)] = (i, [have])
                    at, i, t = begin[i + 1], i + 1, 0
            assert len(teams) == 1
            if teams == {True}:
                assert len({i for i, _ in left_over}) == 1 and len(left_over) == waves and 2 * group not in written
                written[2 * group] = (left_over[0][0], [have for _, have in left_over])
        slots = (ctypes.c_int * (2 * most))()
        for i, (a, b) in enumerate(workers):
            if a == b:
                continue
            found = []
            for p in range(lib.parts(a, b, slots)):
                of, ranges = written.pop(slots[p])
                assert of == i
                found += [x for r in ranges for x in r]
            assert sorted(found) == list(range(tiles[i]))
        assert not written


def test_the_oracles_rows_by_hand():
    row = np.zeros(32)
    row[:12] = [7.0, 5.0, -5.1, 2.5, -2.6, 0.25, 0.26, -0.75, 1.25, 1.75, 3.5, -0.1]
    codes, e = Q.quantise(row)
    assert e.tolist() == [0] and codes[:12].tolist() == [7, 6, 15, 4, 13, 0, 1, 10, 2, 4, 6, 8] and not codes[12:].any()
    assert Q.values(codes, e)[:6].tolist() == [6.0, 4.0, -6.0, 2.0, -3.0, 0.0]
    for m, want in ((7.0, 0), (7.0001, 1), (3.5, -1), (3.6, 0), (0.0, -100), (2.0 ** 120, 100), (7 * 2.0 ** -50, -50)):
        assert Q.scale_exponent(m) == want == Q.quantise(np.array([-m] + [0.0] * 31))[1][0]
    # a row's error is at most its scale, and a row that came out of 4 bits goes back unchanged
    rng = np.random.default_rng(0)
    x = rng.standard_normal((500, 64)) * np.exp2(rng.integers(-9, 9, (500, 1)))
    y = Q.values(*Q.quantise(x))
    assert (np.abs(x - y) <= np.repeat(np.exp2(Q.quantise(x)[1].astype(float)), 32, -1)).all() and np.array_equal(Q.values(*Q.quantise(y)), y)


@pytest.mark.parametrize("dh", [32, 64, 128, 256])
def test_a_block_has_a_place_for_everything(dh):
    for which in range(2):
        at = {Q.code_byte(which, r, x, dh) for r in range(16) for x in range(dh)}
        scales = {Q.scale_place(r, g, dh) for r in range(16) for g in range(dh // 32)}
        assert len(at) == 16 * dh and {b for b, _ in at} == set(range(8 * dh)) and scales == set(range(8 * dh, Q.block_bytes(dh)))
    blocks = np.zeros((2, Q.block_bytes(dh)), dtype=np.uint8)
    x = np.random.default_rng(dh).standard_normal((3, dh))
    codes, e = Q.quantise(x)
    Q.store(blocks, 1, [3, 17, 31], codes.astype(np.uint8), e)
    assert np.array_equal(Q.load(blocks, 1, [31, 3], dh), Q.values(codes, e)[[2, 0]])


def test_the_oracles_rotation_by_hand():
    x = np.arange(1.0, 9.0)
    y = Q.rotate_head(x, None, 0.0, [2, 3], [math.pi / 4, math.pi / 3], [0, 1], Q.HALVES)       # quarter and half a turn of (1, 3) and (2, 4)
    np.testing.assert_allclose(y, [-3, -2, 1, -4, 5, 6, 7, 8], atol=1e-14)
    y = Q.rotate_head(x, None, 0.0, [2, 3], [math.pi / 4, math.pi / 3], [0, 1], Q.ADJACENT)
    np.testing.assert_allclose(y, [-2, 1, -3, -4, 5, 6, 7, 8], atol=1e-14)
    y = Q.rotate_head([3.0, 4.0], [1.0, 2.0], 0.0, [0], [1.0], [0], Q.HALVES)
    np.testing.assert_allclose(y, [3 / math.sqrt(12.5), 8 / math.sqrt(12.5)])
    rng = np.random.default_rng(1)
    x, pos, freq = rng.standard_normal((5, 3, 32)), rng.integers(0, 99, (3, 5)), rng.random(8)
    for pairs in (Q.HALVES, Q.ADJACENT):
        got = Q.rotate(x, np.ones(32), 1e-6, pos, freq, [0, 1, 2, 0, 1, 2, 0, 1], pairs)
        for i in range(5):
            for h in range(3):
                np.testing.assert_allclose(got[i, h], Q.rotate_head(x[i, h], np.ones(32), 1e-6, pos[:, i], freq, [0, 1, 2, 0, 1, 2, 0, 1], pairs), atol=1e-13)
    # what a query and a key have in common depends on the distance of their positions alone
    q, k = rng.standard_normal((2, 1, 1, 32))
    dots = [float((Q.rotate(q, None, 0, [[p]], freq, [0] * 8, 0) * Q.rotate(k, None, 0, [[p + 7]], freq, [0] * 8, 0)).sum()) for p in (0, 5, 1000)]
    np.testing.assert_allclose(dots, dots[0], rtol=1e-10)


def walk(lib, tiles):
    """The kernel's loop for pairs of so many tiles: of every worker, its pieces (pair, tiles) and whether its workgroup is in the middle of a pair."""
    cost, begin = lib.pair_cost(), [0]
    for t in tiles:
        begin.append(begin[-1] + t + cost)
    units, pair, found = begin[-1], 0, []
    for w in range(lib.workers(units)):
        at, end, pieces = lib.first(w, units), lib.first(w + 1, units), []
        while begin[pair + 1] <= at:
            pair += 1
        i, team = pair, bool(lib.middle(w, units, at - begin[pair], tiles[pair]))
        while at < end:
            have = range(at - begin[i], min(end - begin[i], tiles[i]))
            if have:
                pieces.append((i, have))
            i += 1
            at = begin[i]
        found.append((pieces, team))
    return units, found


@pytest.mark.parametrize("name", sorted(large.CASES))
def test_the_large_cases_give_a_worker_several_tiles(name):
    """What tests/test_gpu_kv4_large.py is for: several tiles of a pair to a worker, several pairs and videos, teams of several tiles, rows that are appended before the
    last tile of a worker.  A split that is tuned anew must not empty it."""
    lib = host_library(PLAN)
    q = ctypes.c_int64
    lib.workers.restype, lib.workers.argtypes, lib.first.restype, lib.first.argtypes, lib.middle.argtypes = q, [q], q, [q, q], [q, q, q, q]
    dtype, lens, Hq, Hkv, dh, capacity, kw = large.CASES[name]
    o = (q * 16)()
    lib.attend_plan(len(lens), Hq, Hkv, q(capacity), dh, int(kw.get("weights", False)), o)
    tile, row_blocks, whole, most = o[0], o[1], o[15], o[6]
    fresh = int(kw.get("append", True))
    tiles = [max(1, -(-(min(n, capacity) + fresh) // tile)) for n in lens for _ in range(Hkv * row_blocks)]
    units, workers = walk(lib, tiles)
    assert not whole and units > 2 * most and len(workers) == most
    assert max(len(have) for pieces, _ in workers for _, have in pieces) > 1
    crossing = [pieces for pieces, _ in workers if len(pieces) > 1]
    assert crossing
    if "short" in name or "ragged" in name:
        assert any(len({i // (Hkv * row_blocks) for i, _ in pieces}) > 1 for pieces in crossing) and len(lens) > 64
    if name == "short_pairs":
        assert any(len(pieces) > 2 for pieces in crossing)
    if "long" in name or "three" in name:
        assert any(team and len(pieces[0][1]) > 1 for pieces, team in workers)
    if "three" in name:
        assert row_blocks == 3
    if fresh:                                              # the new row's tile, and tiles of the same worker behind it
        assert any(have[-1] + 1 == tiles[i] and (i, have) != pieces[-1] for pieces, _ in workers for i, have in pieces)
    if "streamed" in name:
        assert dh >= 128 and len(lens) * Hkv * capacity * dh * 17 // 16 > 128 << 20
