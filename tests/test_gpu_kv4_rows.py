"""Rows into a 4-bit cache and back on the GPU, bit for bit against the oracle."""
import numpy as np
import pytest
import torch

from oracle import qkv_oracle as Q
from tests.kv4_cases import Cache4, TORCH, typed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2506_02850_amd import binding
    return binding


def i32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def pack(B, c, k, v, start=None, count=None, idx=None):
    """The call on a copy of c's bytes, and what they are to be."""
    kd, vd, table = c.device()
    kw = dict(start=i32(start), count=i32(count), idx=i32(idx))
    if c.page:
        B.metok_kv4_pack_paged(k, v, kd, vd, table, **kw)
    else:
        B.metok_kv4_pack(k, v, kd, vd, **kw)
    torch.cuda.synchronize()
    return kd, vd, table


def expect(c, sources, start, count, idx, n):
    for b in range(c.B):
        first = max(start[b], 0) if start is not None else 0
        i = np.arange(min(max(count[b], 0), n) if count is not None else n)
        src = idx[b, i] if idx is not None else i
        ok = (src >= 0) & (src < sources[0].shape[2]) & (first + i < c.capacity)
        for which in range(2):
            c.put(which, b, first + i[ok], sources[which][b][:, src[ok]].transpose(1, 0, 2))


CASES = [
    # dtype, B, Hkv, S_src, dh, capacity, page, start, count, listed
    ("bf16", 1, 1, 16, 128, 16, 0, None, None, 0),
    ("bf16", 2, 3, 37, 128, 64, 0, [5, 30], [37, 20], 0),
    ("bf16", 1, 1, 1, 32, 16, 0, [15], None, 0),
    ("bf16", 2, 2, 70, 64, 64, 16, [3, 0], [70, 0], 0),
    ("bf16", 1, 2, 33, 256, 48, 0, [-4], [100], 0),
    ("f32", 2, 2, 37, 128, 96, 32, [16, 61], None, 0),
    ("f32", 1, 3, 50, 64, 64, 0, [1], None, 30),
    ("f32", 2, 1, 21, 32, 32, 16, [2, 9], [21, -3], 25),
    ("f32", 1, 2, 19, 256, 32, 0, None, None, 19),
    ("bf16", 3, 1, 130, 128, 112, 16, [0, 7, 111], [112, 105, 4], 90),
]


@pytest.mark.parametrize("dtype,Bn,Hkv,S,dh,capacity,page,start,count,listed", CASES)
def test_rows_go_in_and_come_out(B, dtype, Bn, Hkv, S, dh, capacity, page, start, count, listed):
    rng = np.random.default_rng(S * dh)
    x = rng.standard_normal((2, Bn, Hkv, S, dh)) * np.exp2(rng.integers(-3, 4, (2, Bn, Hkv, S, 1)))
    k, k64 = typed(x[0], dtype)
    v, v64 = typed(x[1], dtype)
    idx = rng.integers(-2, S + 2, (Bn, listed)).astype(np.int32) if listed else None
    n = listed or S
    c = Cache4(Bn, Hkv, capacity, dh, page, seed=S, scaled=True)
    kd, vd, table = pack(B, c, k, v, start, count, idx)
    expect(c, (k64, v64), start, count, idx, n)
    for which, t in ((0, kd), (1, vd)):
        assert np.array_equal(t.cpu().numpy(), c.data[which])

    lens = [max(capacity - 3 - 5 * b, 0) for b in range(Bn)]
    for kw, rows in ((dict(), lambda b, i: i), (dict(first=[3] * Bn), lambda b, i: 3 + i),
                     (dict(idx=rng.integers(-1, capacity + 1, (Bn, 24)).astype(np.int32)), None)):
        m = 24
        out = {name: torch.full((Bn, Hkv, m + 2, dh), 7.0, dtype=TORCH[dtype], device="cuda") for name in ("k", "v")}
        args = {name: i32(val) for name, val in kw.items()}
        if page:
            B.metok_kv4_unpack_paged(kd, vd, table, i32(lens), m, out=out, **args)
        else:
            B.metok_kv4_unpack(kd, vd, i32(lens), m, out=out, **args)
        for which, name in ((0, "k"), (1, "v")):
            got = out[name].to(torch.float64).cpu().numpy()
            for b in range(Bn):
                for i in range(m + 2):
                    row = -1 if i >= m else rows(b, i) if rows else int(kw["idx"][b, i])
                    want = c.get(which, b, row) if 0 <= row < lens[b] else np.full((Hkv, dh), 7.0)
                    assert np.array_equal(got[b, :, i], want), (name, b, i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_borders_and_extremes(B, dtype):
    """Every border of the eight values and of the scale, at ordinary, tiny and huge sizes: 0, the ties, 7 s and what follows it, sizes beyond the scales."""
    step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    rows = []
    for e in (-120, -101, -100, -99, -20, -1, 0, 3, 60, 99, 100, 101, 110):
        ties = [0.0, -0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.0 * (1 + step)]
        for top in (4.0, 6.0, 7.0, 7.0 * (1 + step), 7.5, 8.0 * (1 - step)):
            for way in (-1, 0, 1):                         # at the borders and a step to each side of them
                g = [t * (1 + way * step) * s for t in ties[:10] for s in (1.0, -1.0)] + [top]
                g = g + [0.0] * (32 - len(g))
                rows.append(np.ldexp(np.asarray(g[:32]), e))
    rows.append(np.zeros(32))
    rows = np.stack(rows + [np.zeros(32)] * (-len(rows) % 4)).reshape(1, 1, -1, 128)
    k, k64 = typed(rows, dtype)
    v, v64 = typed(-rows, dtype)
    c = Cache4(1, 1, (rows.shape[2] + 15) // 16 * 16, 128)
    kd, vd, _ = pack(B, c, k, v)
    expect(c, (k64, v64), None, None, None, rows.shape[2])
    assert np.array_equal(kd.cpu().numpy(), c.data[0]) and np.array_equal(vd.cpu().numpy(), c.data[1])
    got = B.metok_kv4_unpack(kd, vd, i32([rows.shape[2]]), rows.shape[2], dtype=torch.float32)
    for which, name in ((0, "k"), (1, "v")):
        codes, e = Q.quantise((k64, v64)[which])
        assert np.array_equal(got[name].to(torch.float64).cpu().numpy(), Q.values(codes, e))


@pytest.mark.parametrize("dh", [32, 64, 128, 256])
def test_rows_of_a_cache_go_back_unchanged(B, dh):
    rng = np.random.default_rng(dh)
    k, _ = typed(rng.standard_normal((2, 2, 64, dh)), "bf16")
    v, _ = typed(rng.standard_normal((2, 2, 64, dh)), "bf16")
    a, b = B.metok_kv4_cache(2, 2, 64, dh, "cuda"), B.metok_kv4_cache(2, 2, 64, dh, "cuda")
    B.metok_kv4_pack(k, v, *a)
    one = B.metok_kv4_unpack(*a, i32([64, 64]), 64)
    B.metok_kv4_pack(one["k"], one["v"], *b)
    two = B.metok_kv4_unpack(*b, i32([64, 64]), 64)
    assert torch.equal(one["k"], two["k"]) and torch.equal(one["v"], two["v"])


def test_pages_that_are_none_and_tables_of_other_videos(B):
    """Entries outside the pool: nothing is stored, nothing comes out; the neighbours' rows are theirs."""
    rng = np.random.default_rng(9)
    c = Cache4(2, 2, 96, 64, 16, seed=4, scaled=True)
    c.table[0, 1], c.table[1, 0], c.table[1, 4] = -1, c.data.shape[1], 2 ** 31 - 1
    k, k64 = typed(rng.standard_normal((2, 2, 90, 64)), "bf16")
    v, v64 = typed(rng.standard_normal((2, 2, 90, 64)), "bf16")
    kd, vd, table = pack(B, c, k, v, [3, 0])
    expect(c, (k64, v64), [3, 0], None, None, 90)
    assert np.array_equal(kd.cpu().numpy(), c.data[0]) and np.array_equal(vd.cpu().numpy(), c.data[1])
    out = {x: torch.full((2, 2, 96, 64), 7.0, dtype=torch.bfloat16, device="cuda") for x in "kv"}
    B.metok_kv4_unpack_paged(kd, vd, table, i32([93, 90]), 96, out=out)
    for b, n in ((0, 93), (1, 90)):
        for j in range(3 if b == 0 else 0, 96):
            want = c.get(0, b, j) if j < n else None
            want = np.full((2, 64), 7.0) if want is None else want
            assert np.array_equal(out["k"][b, :, j].to(torch.float64).cpu().numpy(), want), (b, j)


def test_a_chunk_at_a_time_is_the_whole(B):
    """Appended in pieces of odd sizes, at starts inside blocks, the cache is what one call makes of it, and replays of a captured call are, too."""
    rng = np.random.default_rng(2)
    k, _ = typed(rng.standard_normal((1, 2, 100, 128)), "bf16")
    v, _ = typed(rng.standard_normal((1, 2, 100, 128)), "bf16")
    whole, parts = B.metok_kv4_cache(1, 2, 112, 128, "cuda"), B.metok_kv4_cache(1, 2, 112, 128, "cuda")
    for t in whole + parts:
        t.zero_()
    B.metok_kv4_pack(k, v, *whole)
    at, sizes = 0, [1, 2, 13, 16, 5, 31, 32]
    for n in sizes:
        B.metok_kv4_pack(k[:, :, at:at + n].contiguous(), v[:, :, at:at + n].contiguous(), *parts, start=i32([at]))
        at += n
    assert at == 100 and all(torch.equal(x, y) for x, y in zip(whole, parts))

    start, rows = i32([0]), torch.zeros((2, 1, 2, 1, 128), dtype=torch.bfloat16, device="cuda")
    again = B.metok_kv4_cache(1, 2, 112, 128, "cuda")
    for t in again:
        t.zero_()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            B.metok_kv4_pack(rows[0], rows[1], *again, start=start)
            start += 1
    start.zero_()
    for t in again:
        t.zero_()
    for j in range(100):
        rows[0].copy_(k[:, :, j:j + 1])
        rows[1].copy_(v[:, :, j:j + 1])
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(whole, again))
