"""Calls of the operators around queries, keys and values that are allowed and unusual: large batches, padded ones, offsets beyond 32 bits, other streams, two calls at
once, a workspace that graphs share."""
import numpy as np
import pytest
import torch

from oracle import qkv_oracle as Q
from tests import kv4_cases as K
from tests.kv4_cases import same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2506_02850_amd import binding
    return binding


def go(B, c, **kw):
    before = c["weight"].clone() if c["weight"] is not None else None
    res = K.call(B, c, **kw)
    K.check(c, res, before, kw.get("scale"))
    K.check_cache(c)
    return res


def workspace(B, c):
    code = B.BF16 if c["dtype"] == "bf16" else B.F32
    return torch.full((max(256, B.metok_kv4_attention_workspace_bytes(len(c["lens"]), c["Hq"], c["Hkv"], c["capacity"], c["dh"], code, c["weight"] is not None)),), 255,
                      dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("capacity,page", [(48, 0), (1040, 16)])
def test_many_videos(B, capacity, page):
    """More than 64, so that a worker looks for its place in several turns; most are short, and some hold nothing."""
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 49, 300)]
    lens[17], lens[255], lens[299] = capacity - 1, capacity, 0
    go(B, K.make("bf16", lens, 4, 1, 32, capacity, page, seed=1))
    go(B, K.make("f32", lens[:70], 2, 2, 32, capacity, page, append=False, weights=True, seed=2))


@pytest.mark.parametrize("dtype,dh,rows", [("bf16", 128, 20011), ("f32", 64, 9003), ("bf16", 256, 6000)])
def test_long_videos(B, dtype, dh, rows):
    """Workgroups in the middle of a pair, many to a pair, with ends of pairs in others."""
    capacity = -(-rows // 16) * 16
    go(B, K.make(dtype, [rows, rows // 3, 0], 4, 1, dh, capacity, seed=rows))
    go(B, K.make(dtype, [rows // 2, rows], 4, 2, dh, capacity, 16, append=False, weights=True, cap=30.0, seed=rows))


@pytest.mark.parametrize("capacity", [64, 2048])
def test_padded_batches(B, capacity):
    """Videos that are not there: no rows, and a table without pages; their results are those of no row (without a new one)."""
    lens = [0, capacity - 9, 0, 33]
    broken = [(b, p, -1) for b in (0, 2) for p in range(capacity // 16)]
    c = K.make("bf16", lens, 8, 2, 64, capacity, 16, append=False, broken=broken, seed=capacity)
    res = go(B, c)
    assert (res["out"][[0, 2]] == 0).all() and torch.isneginf(res["lse"][[0, 2]]).all()
    # with a new one: it is attended to and stored nowhere
    go(B, K.make("bf16", lens, 8, 2, 64, capacity, 16, broken=broken, seed=capacity))


def test_other_streams_and_two_calls_at_once(B):
    cases = [K.make("bf16", [3000 + 40 * s, 7], 28, 4, 128, 3200, weights=True, append=False, seed=s) for s in range(2)]
    work = [workspace(B, c) for c in cases]
    before = [c["weight"].clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    results = [[], []]
    for turn in range(10):
        for s, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                w = before[s].clone()
                results[s].append((K.call(B, dict(cases[s], weight=w), workspace=work[s]), w))
    torch.cuda.synchronize()
    for s in range(2):
        first, weight = results[s][0]
        K.check(dict(cases[s], weight=weight), first, before[s])
        for res, w in results[s][1:]:
            assert same(res["out"], first["out"]) and same(res["lse"], first["lse"]) and same(w, weight)


def test_graphs_that_share_a_workspace(B):
    """Calls of different shapes, captured over one workspace and replayed one behind the other."""
    cases = [K.make("bf16", [2000, 90], 28, 4, 128, 2048, append=False, seed=1), K.make("f32", [1500, 1, 400], 4, 2, 64, 1504, 16, weights=True, append=False, seed=2)]
    work = max((workspace(B, c) for c in cases), key=lambda t: t.numel())
    want, outs, graphs = [], [], []
    for c in cases:
        w = None if c["weight"] is None else c["weight"].clone()
        want.append((K.call(B, dict(c, weight=w)), w))
        outs.append({x: torch.empty_like(t) for x, t in want[-1][0].items()})
    torch.cuda.synchronize()
    start = [None if c["weight"] is None else c["weight"].clone() for c in cases]
    for c, out in zip(cases, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            K.call(B, c, out=out, workspace=work)
        graphs.append(graph)
    for turn in range(5):
        for c, s in zip(cases, start):
            if s is not None:
                c["weight"].copy_(s)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for c, out, (res, w) in zip(cases, outs, want):
            assert same(out["out"], res["out"]) and same(out["lse"], res["lse"]) and (w is None or same(c["weight"], w)), turn


def test_offsets_beyond_32_bits_of_a_cache_in_4_bits(B):
    """Four videos, 2.9 GB each of K and of V, the last of which has rows: packing, attention with a new row and unpacking there do what they do in a small cache."""
    Hkv, dh, big, small, n = 40, 128, 2 ** 20, 2048, 50
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn((4, Hkv, n, dh), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    q, kn, vn = (torch.randn((4, Hkv, dh), generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    count = torch.tensor([0, 0, 0, n], dtype=torch.int32, device="cuda")
    got = []
    for capacity in (big, small):
        k4, v4 = B.metok_kv4_cache(4, Hkv, capacity, dh, "cuda")
        B.metok_kv4_pack(k, v, k4, v4, count=count)
        res = B.metok_kv4_attention(q, k4, v4, count, k_new=kn, v_new=vn)
        rows = B.metok_kv4_unpack(k4, v4, count + torch.tensor([0, 0, 0, 1], dtype=torch.int32, device="cuda"), n + 1)
        got.append((res["out"][3], res["lse"][3], rows["k"][3], rows["v"][3]))
        # the last rows of the last head
        end = torch.full((4,), capacity - n, dtype=torch.int32, device="cuda")
        B.metok_kv4_pack(k, v, k4, v4, start=end)
        last = B.metok_kv4_unpack(k4, v4, end + n, n, first=end)
        got[-1] += (last["k"], last["v"])
        del k4, v4
    assert all(same(x, y) for x, y in zip(*got))
    want = Q.values(*Q.quantise(k[3].double().cpu().numpy().transpose(1, 0, 2))).transpose(1, 0, 2)
    assert np.array_equal(got[0][2][:, :n].double().cpu().numpy(), want) and np.array_equal(got[0][4][3].double().cpu().numpy(), want)


def test_offsets_beyond_32_bits_of_rotated_keys(B):
    """The last rows of a cache of 10.7 GB, and of a pool as large."""
    Hkv, dh, n = 40, 64, 5
    g = torch.Generator().manual_seed(6)
    x = torch.randn((2, n, 3 * Hkv, dh), generator=g).to(torch.bfloat16).cuda()
    pos = torch.randint(0, 100000, (1, 2, n), generator=g).to(torch.int32).cuda()
    freq = torch.rand(dh // 2, generator=g).cuda()
    got = []
    for capacity in (2 ** 20, 64):
        end = torch.full((2,), capacity - n, dtype=torch.int32, device="cuda")
        k, v = (torch.empty((2, Hkv, capacity, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        out = B.metok_rotate_qk(x[:, :, :Hkv], x[:, :, Hkv:2 * Hkv], x[:, :, 2 * Hkv:], pos, freq, k, v, start=end)["q"]
        got.append((out, k[:, :, -n:].clone(), v[:, :, -n:].clone()))
        # the last page of a pool is the videos' page for their rows
        pages = capacity // 32
        table = torch.tensor([[2 * pages - 1], [2 * pages - 2]], dtype=torch.int32, device="cuda")
        k, v = (t.view(2 * pages, Hkv, 32, dh) for t in (k, v))
        B.metok_rotate_qk_paged(x[:, :, :Hkv], x[:, :, Hkv:2 * Hkv], x[:, :, 2 * Hkv:], pos, freq, k, v, table)
        got[-1] += (k[-2:, :, :n].clone(), v[-2:, :, :n].clone())
        del k, v
    assert all(same(x, y) for x, y in zip(*got))
    assert same(got[0][2], x[:, :, 2 * Hkv:].transpose(1, 2).contiguous()) and same(got[0][1], got[0][3].flip(0))


def test_many_videos_of_a_token_each(B):
    """A decoding step of a large batch: rows of their own, some behind the cache's end, some in pages that are none, into a cache of one row as well."""
    Bn, Hq, Hkv, dh, page, per_seq = 700, 6, 2, 64, 16, 3
    rng = np.random.default_rng(8)
    g = torch.Generator().manual_seed(8)
    x = torch.randn((Bn, 1, Hq + 2 * Hkv, dh), generator=g).to(torch.bfloat16).cuda()
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    pos = torch.from_numpy(rng.integers(0, 10 ** 6, (1, Bn, 1)).astype(np.int32)).cuda()
    freq = torch.rand(dh // 2, generator=g).cuda()
    one = [torch.empty((Bn, Hkv, 1, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    out = B.metok_rotate_qk(q, k, v, pos, freq, *one)["q"]
    assert same(one[1][:, :, 0], v[:, 0].contiguous())
    table = rng.permutation(Bn * per_seq).reshape(Bn, per_seq).astype(np.int32)
    table[::7, 1] = -1
    table[3::11, 0] = 2 ** 31 - 1
    start = rng.integers(0, per_seq * page + 9, Bn).astype(np.int32)
    pool = [torch.full((Bn * per_seq, Hkv, page, dh), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    paged = B.metok_rotate_qk_paged(q, k, v, pos, freq, *pool, torch.from_numpy(table).cuda(), start=torch.from_numpy(start).cuda())["q"]
    assert same(paged, out)
    for which in range(2):
        want = torch.full_like(pool[which], 5.0).cpu()
        rows = one[which][:, :, 0].cpu()
        for b in range(Bn):
            if start[b] < per_seq * page and 0 <= table[b, start[b] // page] < len(want):
                want[table[b, start[b] // page], :, start[b] % page] = rows[b]
        assert same(pool[which].cpu(), want)


def test_what_is_no_number_stays_in_its_head(B):
    """A NaN among a normed head's elements makes the whole head NaN, and nothing else; in 4 bits an infinity is the largest value of the largest scale."""
    x = torch.randn((2, 3, 6, 64), generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).cuda()
    x[1, 2, 1, 40] = float("nan")
    pos = torch.ones((1, 2, 3), dtype=torch.int32, device="cuda")
    weight = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros((2, 1, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = B.metok_rotate_qk(x[:, :, :4], x[:, :, 4:5], x[:, :, 5:], pos, torch.rand(16, device="cuda"), k, v, q_weight=weight, k_weight=weight)["q"]
    want = torch.zeros_like(q, dtype=torch.bool)
    want[1, 1, 2] = True
    assert torch.equal(q.isnan(), want) and not k.isnan().any() and not v.isnan().any()
    k[0, 0, 0, 5], k[1, 0, 3, 60] = float("inf"), float("-inf")
    k4, v4 = B.metok_kv4_cache(2, 1, 16, 64, "cuda")
    B.metok_kv4_pack(k, v, k4, v4)
    back = B.metok_kv4_unpack(k4, v4, torch.full((2,), 16, dtype=torch.int32, device="cuda"), 16)["k"]
    assert back[0, 0, 0, 5] == 6 * 2.0 ** 100 and back[1, 0, 3, 60] == -6 * 2.0 ** 100 and back.isfinite().all()
    assert (back[0, 0, 0, :32].count_nonzero(), back[1, 0, 3, 32:].count_nonzero()) == (1, 1) and back[0, 0, 0, 32:].any()


def test_long_videos_of_many_heads_and_of_pages_that_are_none(B):
    """Several blocks of query heads to a kv head, each split over many workgroups; and whole workgroups that find no row."""
    go(B, K.make("bf16", [9000, 70], 33, 1, 64, 9008, seed=1))
    go(B, K.make("f32", [5000], 40, 2, 32, 5008, 16, append=False, weights=True, seed=2))
    broken = [(0, p, -1 - p) for p in range(10, 110)] + [(1, p, -1) for p in range(128)]
    go(B, K.make("bf16", [8191, 8000], 8, 2, 128, 8192, 64, broken=broken, seed=3))
    res = go(B, K.make("bf16", [8192, 8000], 8, 2, 128, 8192, 64, append=False, broken=broken, seed=4))
    assert (res["out"][1] == 0).all() and torch.isneginf(res["lse"][1]).all()
