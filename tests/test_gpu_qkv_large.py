"""What the operators around queries, keys and values do in large calls alone: workers with several tiles and several pairs, several heads to a workgroup of the
rotation, rows that are read and written with the streaming hint."""
import os
import re

import numpy as np
import pytest
import torch

from oracle import qkv_oracle as Q
from tests import kv4_cases as K
from tests import kv4_large as large
from tests.kv4_cases import TORCH, rotate_tolerance, same
from tests.test_gpu_kv4_attention import go
from tests.test_gpu_rotate import i32, make, run

pytestmark = pytest.mark.gpu
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_02850_amd", "csrc")


@pytest.fixture(scope="module")
def B():
    from paper_2506_02850_amd import binding
    return binding


def constant(source, name):
    """The value of a constant of the kernels."""
    value, shift = re.search(rf"\b{name} = (\d+)(?: << (\d+))?\b", open(os.path.join(CSRC, source)).read()).groups()
    return int(value) << int(shift or 0)


@pytest.mark.parametrize("name", sorted(large.CASES))
def test_attention_of_workers_with_several_tiles(B, name):
    """tests/test_qkv_boundary.py shows that they have them."""
    c = large.make(name)
    start = None if c["weight"] is None else c["weight"].clone()
    first = go(B, c)
    again = K.call(B, c if start is None else dict(c, weight=start))         # a row that is appended twice is the same row
    assert same(first["out"], again["out"]) and same(first["lse"], again["lse"]) and (start is None or same(start, c["weight"]))


ROTATIONS = [
    # dtype, B, n, Hq, Hkv, dh, rot, pairs, norm, page, with the streaming hint: 0 not, 1 writes, 2 reads too
    ("bf16", 2, 2500, 11, 2, 128, 128, Q.HALVES, True, 0, 0),
    ("bf16", 3, 3001, 11, 2, 128, 96, Q.ADJACENT, True, 16, 1),
    ("bf16", 1, 35001, 11, 2, 128, 128, Q.HALVES, True, 0, 2),
    ("f32", 2, 4100, 6, 1, 64, 32, Q.HALVES, True, 0, 0),
    ("f32", 2, 9000, 6, 1, 64, 64, Q.ADJACENT, False, 7, 1),
    ("f32", 1, 66001, 6, 1, 64, 48, Q.HALVES, True, 0, 2),
    ("bf16", 2, 9001, 5, 1, 256, 256, Q.HALVES, False, 64, 1),
    ("bf16", 1, 20001, 11, 2, 256, 240, Q.ADJACENT, True, 0, 2),
    ("f32", 1, 17001, 6, 1, 128, 128, Q.HALVES, True, 0, 1),
    ("f32", 2, 17000, 6, 1, 128, 64, Q.ADJACENT, True, 16, 2),
    ("bf16", 1, 40001, 9, 2, 64, 32, Q.ADJACENT, True, 0, 1),
    ("bf16", 1, 50001, 17, 4, 32, 32, Q.HALVES, True, 0, 1),
    ("f32", 1, 50001, 7, 2, 32, 16, Q.ADJACENT, True, 0, 1),
]


@pytest.mark.parametrize("dtype,Bn,n,Hq,Hkv,dh,rot,pairs,norm,page,hint", ROTATIONS)
def test_rotations_of_several_heads_to_a_workgroup(B, dtype, Bn, n, Hq, Hkv, dh, rot, pairs, norm, page, hint):
    """A workgroup's heads are queries, keys and values: the call is bit for bit what calls of a few tokens are, and what the oracle says of some of them."""
    esize, heads = 2 if dtype == "bf16" else 4, Hq + 2 * Hkv
    small, threads = 250, constant("rotate.hip", "kRotateThreads")
    groups = [-(-tokens * dh * esize // 16 // threads) * heads for tokens in (Bn * n, small)]
    assert groups[0] >= constant("rotate.hip", "kRotateSpread") > groups[1]
    size = Bn * n * heads * dh * esize
    assert (size > constant("rotate.hip", "kStreamOut")) + (size > constant("rotate.hip", "kStreamIn")) == hint
    count = [n - 777 * b for b in range(Bn)]
    capacity = n + 20 if page == 0 else -(-(n + 20) // page) * page
    c = make(dtype, Bn, n, Hq, Hkv, dh, rot, 3, pairs, norm, capacity=capacity, page=page, start=[3 + 5 * b for b in range(Bn)], count=count, far=10 ** 5, seed=n)
    got, kv = run(B, c), c["kv"]
    want, want_kv = torch.full_like(got, 7.0), torch.full_like(kv, 7.0)
    kw = dict(pair_axis=bytes(c["axis"]), pairs=pairs, q_weight=c["weights"][0][0], k_weight=c["weights"][1][0])
    pos, freq, table = i32(c["pos"]), torch.from_numpy(c["freq"]).cuda(), i32(c["table"]) if page else None
    for b in range(Bn):
        for i in range(0, count[b], small):
            m = min(small, count[b] - i)
            rows, start = [t[b:b + 1, i:i + m] for t in c["rows"]], i32([c["start"][b] + i])
            args = (*rows, pos[:, b:b + 1, i:i + m].contiguous(), freq)
            if page:
                want[b:b + 1, :, i:i + m] = B.metok_rotate_qk_paged(*args, want_kv[0], want_kv[1], table[b:b + 1], start=start, **kw)["q"]
            else:
                want[b:b + 1, :, i:i + m] = B.metok_rotate_qk(*args, want_kv[0, b:b + 1], want_kv[1, b:b + 1], start=start, **kw)["q"]
    assert same(got, want) and same(kv, want_kv)
    for b in range(Bn):
        some = np.r_[0:20, count[b] - 20:count[b]]
        for which in range(2):
            weight, x = c["weights"][which][1], c["x64"][which][b, some]
            exact = Q.rotate(x, weight, 1e-6, c["pos"][:, b, some], c["freq"], c["axis"], pairs)
            limit = rotate_tolerance(x, weight, 1e-6, exact, dtype, dh, c["half"], pairs)
            if which == 0:
                there = got[b][:, some]
            else:
                row = some + c["start"][b]
                there = kv[0, b][:, row] if page == 0 else kv[0][c["table"][b][row // page], :, row % page].transpose(0, 1)
            assert (np.abs(there.double().cpu().numpy().transpose(1, 0, 2) - exact) <= limit).all(), (b, which)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [32, 64, 128, 256])
@pytest.mark.parametrize("listed,page", [(False, 0), (True, 64)])
def test_rows_that_pass_by_the_caches(B, dtype, dh, listed, page):
    """Packing and unpacking with the streaming hint, bit for bit what calls of a few rows are, and what the oracle says of some of them."""
    Bn, Hkv, esize, few, least = 2, 2, 2 if dtype == "bf16" else 4, 1000, [7, 30]
    each = 2 * Bn * Hkv * dh * esize
    n = constant("kv4.hip", "kStreamPack") // each + 3
    assert n * each > constant("kv4.hip", "kStreamPack") > constant("kv4.hip", "kStreamUnpack") > few * each
    g = torch.Generator(device="cuda").manual_seed(dh)
    k, v = (torch.randn((Bn, Hkv, n, dh), generator=g, device="cuda").to(TORCH[dtype]) for _ in range(2))
    idx = torch.randint(-2, n + 2, (Bn, n), generator=g, device="cuda", dtype=torch.int32) if listed else None
    capacity = -(-(n + 40) // 64) * 64
    table = torch.randperm(Bn * capacity // page, generator=g, device="cuda").int().view(Bn, -1) if page else None
    shape = (Bn * capacity // page, Hkv, page, dh) if page else (Bn, Hkv, capacity, dh)
    one, many = ([t.fill_(130) for t in B.metok_kv4_cache(*shape, "cuda")] for _ in range(2))
    start, lens = i32(least), i32([x + n for x in least])
    paged = (table,) if page else ()
    pack, unpack = (B.metok_kv4_pack_paged, B.metok_kv4_unpack_paged) if page else (B.metok_kv4_pack, B.metok_kv4_unpack)
    out, want = ({x: torch.full((Bn, Hkv, n, dh), 7.0, dtype=TORCH[dtype], device="cuda") for x in "kv"} for _ in range(2))
    pack(k, v, *one, *paged, start=start, idx=idx)
    unpack(*one, *paged, lens, n, first=start, out=out)
    for i in range(0, n, few):
        m = min(few, n - i)
        if listed:
            pack(k, v, *many, *paged, start=start + i, idx=idx[:, i:i + m].contiguous())
        else:
            pack(k[:, :, i:i + m].contiguous(), v[:, :, i:i + m].contiguous(), *many, *paged, start=start + i)
        rows = unpack(*many, *paged, lens, m, first=start + i, dtype=TORCH[dtype])
        for x in "kv":
            want[x][:, :, i:i + m] = rows[x]
    assert all(torch.equal(x, y) for x, y in zip(one, many)) and all(same(out[x], want[x]) for x in "kv")
    some = np.r_[0:30, n - 30:n]
    for name, x in (("k", k), ("v", v)):
        for b in range(Bn):
            src = idx[b].cpu().numpy()[some] if listed else some
            ok = (src >= 0) & (src < n)
            exact = Q.values(*Q.quantise(x[b][:, src[ok]].double().cpu().numpy()))
            assert np.array_equal(out[name][b][:, some[ok]].double().cpu().numpy(), exact)
