"""GPU tests of metok_decode_attention and metok_decode_attention_paged against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from tests import decode_cases as C

pytestmark = pytest.mark.gpu


def mk():
    from paper_2506_02850_amd import binding as B
    return B


def run(c, scale=None):
    B = mk()
    before = dict(k=c["k"].clone(), v=c["v"].clone())
    weight = None if c["weight"] is None else c["weight"].clone()
    res = C.call(B, c) if scale is None else C.call(B, c, scale=scale)
    torch.cuda.synchronize()
    C.check(c, res, weight, scale)
    C.check_caches(c, before)
    return res


HEADS = [(28, 4), (4, 4), (14, 2), (17, 1), (40, 1), (32, 8), (1, 1)]


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("page", [0, 16, 7])
@pytest.mark.parametrize("weights", [False, True])
def test_every_kernel(dtype, dh, page, weights):
    """Each dtype, head size, cache form and with or without weights: lengths around the tiles, an empty video among them."""
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 129, 300]
    capacity = 350 if page == 0 else page * (-(-350 // page))
    Hq, Hkv = HEADS[(dh // 32 + page) % len(HEADS)]
    run(C.make(dtype, lens, Hq, Hkv, dh, capacity, page, append=True, weights=weights, seed=dh + page))
    run(C.make(dtype, lens, Hq, Hkv, dh, capacity, page, append=False, weights=weights, seed=dh + page + 1))


@pytest.mark.parametrize("Hq,Hkv", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_layouts(Hq, Hkv, dtype):
    run(C.make(dtype, [700, 33], Hq, Hkv, 64, 701, weights=True, seed=Hq))
    run(C.make(dtype, [90, 640], Hq, Hkv, 64, 640, 16, append=False, seed=Hq + 1))


@pytest.mark.parametrize("page", [0, 1, 2, 5, 32, 64, 128])
def test_long_caches_are_split_and_joined(page):
    capacity = 5120 if page != 5 else 5125
    run(C.make("bf16", [5000], 28, 4, 128, capacity, page, weights=True, seed=page))
    run(C.make("bf16", [4999, 3, 0, 2048], 14, 2, 64, capacity, page, append=page % 2 == 0, seed=page + 1))


def test_a_very_long_cache():
    run(C.make("bf16", [70001], 4, 1, 64, 70100, weights=True, seed=5))
    run(C.make("f32", [40000], 2, 2, 32, 40000, 16, append=False, seed=6))


@pytest.mark.parametrize("B", [1, 63, 64, 65, 130, 300])
def test_many_videos(B):
    rng = np.random.default_rng(B)
    run(C.make("bf16", rng.integers(0, 90, B), 4, 2, 32, 96, 16, weights=True, seed=B))
    lens = rng.integers(0, 20, B)
    lens[B // 2] = 2500
    run(C.make("bf16", lens, 4, 2, 32, 2600, append=False, seed=B + 1))


@pytest.mark.parametrize("page", [0, 16])
def test_lengths_beyond_the_ends(page):
    """A full cache attends to the new row without storing it; lengths below 0 and above the capacity count as the ends."""
    run(C.make("bf16", [64, 63, 65, 1000, -1, -2 ** 31, 2 ** 31 - 1], 8, 2, 64, 64, page, append=True, weights=True, seed=3))
    run(C.make("f32", [64, 63, 65, 1000, -1, -2 ** 31, 2 ** 31 - 1], 8, 2, 64, 64, page, append=False, weights=True, seed=4))


@pytest.mark.parametrize("cap", [5.0, 30.0, 1000.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_capped_scores(cap, dtype):
    run(C.make(dtype, [333, 40], 8, 2, 128, 400, cap=cap, spread=8.0, weights=True, seed=int(cap)))


@pytest.mark.parametrize("spread", [0.0, 1e-3, 30.0, 1000.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_flat_and_peaked_scores(spread, dtype):
    """Equal logits, and logits so far apart that all but one row underflow."""
    run(C.make(dtype, [1, 500, 77], 8, 2, 64, 512, spread=spread, weights=True, seed=9))


def test_scale():
    run(C.make("f32", [200, 3], 4, 4, 64, 256, weights=True, seed=2), scale=0.01)
    run(C.make("bf16", [200, 3], 4, 4, 64, 256, 16, seed=2), scale=1.0)


def test_masked_places_may_hold_anything():
    """Infinities in rows behind the last one and in pages of nobody change nothing (the other tests have NaNs there)."""
    B = mk()
    for page in (0, 16):
        got = []
        for poison in (float("nan"), float("inf"), 0.0):
            c = C.make("bf16", [45, 0, 130], 8, 2, 64, 160, page, append=False, poison=poison, seed=8)
            got.append(C.call(B, c))
        for other in got[1:]:
            assert C.same(got[0]["out"], other["out"]) and C.same(got[0]["lse"], other["lse"])


def test_pages_that_are_none_take_no_part():
    B = mk()
    c = C.make("bf16", [100, 100, 96], 8, 2, 64, 112, 16, append=True, weights=True, seed=11)
    bad = c["table_dev"].clone()
    bad[0, 1] = -1                                   # rows 16 .. 31 of video 0
    bad[1, 6] = c["k"].shape[0]                      # the page of video 1's last rows and of its new row
    bad[2] = 2 ** 31 - 1                             # all of video 2 but its new row
    gone = [set(range(16, 32)), set(range(96, 100)), set(range(96))]
    before, weight = dict(k=c["k"].clone(), v=c["v"].clone()), c["weight"].clone()
    res = B.metok_decode_attention_paged(c["q"], c["k"], c["v"], bad, c["lens_dev"], k_new=c["k_new"], v_new=c["v_new"], weight=c["weight"])
    torch.cuda.synchronize()
    want = dict(k=before["k"].clone(), v=before["v"].clone())
    for w in ("k", "v"):
        want[w][int(c["table"][0, 6]), :, 4] = c[w + "_new"][0]
        assert C.same(c[w], want[w])
    full = [len(x) for x in c["rows64"][0]]
    left = [[j for j in range(n) if j not in gone[b]] for b, n in enumerate(full)]
    grown = c["weight"].clone()
    for b in range(3):
        for j in gone[b]:
            assert grown[b, j] == weight[b, j]
    c["rows64"] = [[x[left[b]] for b, x in enumerate(c["rows64"][w])] for w in range(2)]
    small = dict(c, weight=None)
    C.check(small, res)


def test_a_prefix_of_pages_may_be_shared():
    c = C.make("bf16", [60, 60, 70], 8, 2, 64, 80, 16, append=True, seed=12)
    for b in (1, 2):
        c["table"][b, :2] = c["table"][0, :2]
        for w in range(2):
            c["rows64"][w][b] = np.concatenate([c["rows64"][w][0][:32], c["rows64"][w][b][32:]])
    c["table_dev"] = torch.from_numpy(c["table"]).cuda()
    run(c)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("capacity", [320, 2048])
def test_keys_may_be_the_values(page, capacity):
    """One cache for both, only read: as with a copy of it."""
    B = mk()
    c = C.make("bf16", [300, 7], 8, 2, 64, capacity, page, append=False, weights=True, seed=20)
    for w in (None, c["weight"]):
        want = C.call(B, c, weight=None if w is None else w.clone()), C.call(B, dict(c, v=c["k"].clone()), weight=None if w is None else w.clone())
        got = C.call(B, dict(c, v=c["k"]), weight=w)
        torch.cuda.synchronize()
        assert C.same(got["out"], want[1]["out"]) and C.same(got["lse"], want[0]["lse"])


def test_same_result_every_time_and_on_another_stream():
    B = mk()
    c = C.make("bf16", [3000, 17, 900], 28, 4, 128, 3104, 16, append=True, weights=True, seed=13)
    w0 = c["weight"].clone()
    first = C.call(B, c)
    w1 = c["weight"].clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        c["weight"].copy_(w0)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = C.call(B, c)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert C.same(first["out"], again["out"]) and C.same(first["lse"], again["lse"]) and C.same(w1, c["weight"])


def test_results_do_not_depend_on_what_the_workspace_held():
    B = mk()
    c = C.make("bf16", [2000, 300], 8, 2, 64, 2048, append=False, weights=True, seed=14)
    w0 = c["weight"].clone()
    need = B.metok_decode_attention_workspace_bytes(2, 8, 2, 2048, 64, B.BF16, True)
    got = []
    for fill in (0, 255, 127):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        c["weight"].copy_(w0)
        got.append((C.call(B, c, workspace=ws), c["weight"].clone()))
    for res, w in got[1:]:
        assert C.same(res["out"], got[0][0]["out"]) and C.same(res["lse"], got[0][0]["lse"]) and C.same(w, got[0][1])


def test_graphs_replay_while_the_caches_grow_and_share_a_workspace():
    """Two captured calls (other shapes, one workspace) replayed in turn: lengths, queries and new rows change between the replays;
    every replay equals the eager call."""
    B = mk()
    big = C.make("bf16", [500, 20], 8, 2, 64, 1600, 16, append=True, weights=True, poison=0.0, seed=15)
    small = C.make("f32", [100], 4, 4, 32, 300, append=True, weights=True, poison=0.0, seed=16)
    cases = [big, small]
    need = max(B.metok_decode_attention_workspace_bytes(len(c["lens"]), c["Hq"], c["Hkv"], c["capacity"], c["dh"], B.BF16 if c["dtype"] == "bf16" else B.F32, True)
               for c in cases)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs = [dict(out=torch.empty_like(c["q"]), lse=torch.empty(c["q"].shape[:2], device="cuda")) for c in cases]
    graphs = []
    for c, o in zip(cases, outs):
        keep = {n: c[n].clone() for n in ("k", "v", "weight")}
        C.call(B, c, workspace=ws, out=o)
        for n, t in keep.items():
            c[n].copy_(t)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            C.call(B, c, workspace=ws, out=o)
        graphs.append(g)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for step in range(6):
        for c, o, g in zip(cases, outs, graphs):
            for n in ("q", "k_new", "v_new"):
                c[n].copy_(torch.randn(c[n].shape, generator=gen, device="cuda"))
            eager = dict(c, **{n: c[n].clone() for n in ("k", "v", "weight")})
            want = C.call(B, eager)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert C.same(o["out"], want["out"]) and C.same(o["lse"], want["lse"])
            for n in ("k", "v", "weight"):
                assert C.same(c[n], eager[n]), (step, n)
            c["lens_dev"] += 1 if step % 2 else 37


def test_offsets_beyond_32_bits():
    """Pools and slabs whose byte offsets pass 2^32: the rows lie in the last pages of 5 GB pools, and in the last of the dense slabs."""
    B = mk()
    c = C.make("bf16", [300], 8, 2, 256, 320, 16, append=True, weights=True, seed=17)
    n_big = 320000                                   # 320000 x 2 x 16 rows of 512 bytes
    assert n_big * 2 * 16 * 512 > 2 ** 32
    shift = n_big - c["k"].shape[0]
    small = (c["k"], c["v"])
    for name in ("k", "v"):
        pool = torch.empty((n_big,) + tuple(c[name].shape[1:]), dtype=torch.bfloat16, device="cuda")
        pool[shift:] = c[name]
        c[name] = pool
    c["table_dev"] = c["table_dev"] + shift
    w0 = c["weight"].clone()
    res = C.call(B, c)
    torch.cuda.synchronize()
    C.check(c, res, w0)
    page, slot = int(c["table"][0, 300 // 16]), 300 % 16
    assert C.same(c["k"][shift + page, :, slot], c["k_new"][0]) and C.same(c["v"][shift + page, :, slot], c["v_new"][0])
    del small
    c["k"] = c["v"] = None
    torch.cuda.empty_cache()
    # two dense slabs of 2.2 GB each: all of the second one lies behind 2^31 bytes, its last rows behind 2^32
    cap = 4300000
    d = C.make("bf16", [4, 40], 1, 1, 256, 64, append=True, seed=18)
    d["capacity"] = cap
    for name in ("k", "v"):
        cache = torch.empty((2, 1, cap, 256), dtype=torch.bfloat16, device="cuda")
        cache[:, :, :64] = d[name]
        d[name] = cache
    res = C.call(B, d)
    torch.cuda.synchronize()
    C.check(d, res)
    assert C.same(d["k"][1, :, 40], d["k_new"][1])


def test_refusals():
    B = mk()
    c = C.make("bf16", [10, 20], 8, 2, 64, 64, append=True, weights=True, seed=19)
    q, k, v, lens, w = c["q"], c["k"], c["v"], c["lens_dev"], c["weight"]
    with pytest.raises(ValueError):
        B.metok_decode_attention(q, k, v, lens.long())
    with pytest.raises(ValueError):
        B.metok_decode_attention(q, k, v, lens[:1])
    with pytest.raises(ValueError):
        B.metok_decode_attention(q, k, v.float(), lens)
    with pytest.raises(ValueError):
        B.metok_decode_attention(q, k, v, lens, k_new=c["k_new"])
    with pytest.raises(ValueError):
        B.metok_decode_attention(q, k.transpose(1, 2).contiguous().transpose(1, 2), v, lens)
    with pytest.raises(ValueError):
        B.metok_decode_attention(q.cpu(), k, v, lens)
    with pytest.raises(ValueError):
        B.metok_decode_attention(q, k, v, lens, weight=w.double())
    with pytest.raises(B.MetokError):
        B.metok_decode_attention(q, k, v, lens, weight=w[:, :63].contiguous())
    with pytest.raises(B.MetokError):
        B.metok_decode_attention(q, k, v, lens, scale=0.0)
    with pytest.raises(B.MetokError):
        B.metok_decode_attention(q, k, v, lens, logit_cap=-1.0)
    with pytest.raises(B.MetokError):
        B.metok_decode_attention(q, k, k, lens, k_new=c["k_new"], v_new=c["v_new"])
    with pytest.raises(B.MetokError):
        B.metok_decode_attention(q, k, v, lens, out=dict(out=q))
    with pytest.raises(B.MetokError):
        B.metok_decode_attention(q, k, v, lens, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"), weight=w)
    with pytest.raises(B.MetokError):
        B.metok_decode_attention(q[:, :7].contiguous(), k, v, lens)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("page", [0, 16, 7])
@pytest.mark.parametrize("weights", [False, True])
def test_every_kernel_of_many_query_heads(dtype, dh, page, weights):
    """More than 16 query heads to a kv head: whole and part blocks, one and several turns of them."""
    lens = [0, 1, 16, 31, 33, 260]
    capacity = 350 if page == 0 else page * (-(-350 // page))
    heads = [(71, 1), (64, 2), (65, 1), (34, 2), (128, 1), (48, 1), (66, 2)]
    Hq, Hkv = heads[(dh // 32 + page + 3 * weights) % len(heads)]
    run(C.make(dtype, lens, Hq, Hkv, dh, capacity, page, append=True, weights=weights, seed=dh + page))
    run(C.make(dtype, lens, Hq, Hkv, dh, capacity, page, append=False, weights=weights, cap=20.0, seed=dh + page + 1))


@pytest.mark.parametrize("Hq,Hkv", [(32, 1), (33, 1), (64, 1), (71, 1), (1024, 1), (1024, 8), (512, 4)])
def test_many_query_heads_split_and_joined(Hq, Hkv):
    run(C.make("bf16", [2100 if Hq < 100 else 300, 5], Hq, Hkv, 64, 2112, 16, weights=True, seed=Hq))
    run(C.make("f32", [40, 301], Hq, Hkv, 32, 320, append=False, seed=Hq + 1))


def test_the_largest_batch():
    """4096 videos, most of them short, in one call: 64 steps of the search for a worker's first video."""
    rng = np.random.default_rng(12)
    lens = rng.integers(0, 3, 4096)
    lens[[0, 63, 64, 2000, 4095]] = [40, 0, 33, 40, 17]
    run(C.make("f32", lens, 2, 1, 32, 40, weights=True, seed=12))


@pytest.mark.parametrize("page", [1, 7, 8, 48])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (71, 1)])
def test_rows_of_no_page_between_others(page, Hq, Hkv):
    """Every third entry of the table is no page: its rows take no part, in blocks and row by row."""
    B = mk()
    capacity = page * (-(-200 // page))
    c = C.make("bf16", [200, 0, 97], Hq, Hkv, 64, capacity, page, append=False, weights=True, seed=page)
    bad = c["table_dev"].clone()
    pages = bad.shape[1]
    gone_pages = [i for i in range(pages) if i % 3 == 1]
    bad[:, gone_pages] = torch.tensor([-1, c["k"].shape[0], -2 ** 31] * len(gone_pages), dtype=torch.int32, device="cuda")[:len(gone_pages)]
    weight = c["weight"].clone()
    res = B.metok_decode_attention_paged(c["q"], c["k"], c["v"], bad, c["lens_dev"], weight=c["weight"])
    torch.cuda.synchronize()
    left = [[j for j in range(len(x)) if (j // page) % 3 != 1] for x in c["rows64"][0]]
    for b, x in enumerate(c["rows64"][0]):
        for j in set(range(len(x))) - set(left[b]):
            assert c["weight"][b, j] == weight[b, j]
        if left[b]:
            grown = (c["weight"][b] - weight[b]).double().sum().item()
            assert abs(grown - 1) < 4 * 2.0 ** -24 * 2 * len(x) * float(weight.abs().max() + 1)       # the sums' and the differences' roundings
    c["rows64"] = [[x[left[b]] for b, x in enumerate(c["rows64"][w])] for w in range(2)]
    C.check(dict(c, weight=None), res)


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("page", [0, 16, 7])
def test_every_kernel_of_long_capacities(dtype, dh, page):
    """Caches that could be long are split over all workgroups even while they are short."""
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 129, 300]
    capacity = 1100 if page == 0 else page * (-(-1100 // page))
    Hq, Hkv = [(28, 4), (4, 4), (14, 2), (16, 1), (8, 2), (32, 8), (1, 1)][(dh // 32 + page) % 7]
    run(C.make(dtype, lens, Hq, Hkv, dh, capacity, page, append=True, seed=dh + page))
    run(C.make(dtype, lens, Hq, Hkv, dh, capacity, page, append=False, cap=20.0, seed=dh + page + 1))


@pytest.mark.parametrize("capacity", [31, 32, 255, 256, 510, 511, 512, 1022, 1023, 1024])
@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("f32", 64), ("bf16", 256)])
def test_capacities_where_the_form_changes(capacity, dtype, dh):
    """On both sides of the number of tiles that one workgroup takes, full caches and nearly full ones."""
    run(C.make(dtype, [capacity, capacity - 1, capacity // 2, 0], 8, 2, dh, capacity, append=True, seed=capacity))
    run(C.make(dtype, [capacity, 1], 16, 1, dh, capacity, append=False, cap=5.0, seed=capacity + 1))


def test_short_caches_need_no_workspace():
    B = mk()
    c = C.make("bf16", [100, 0, 511], 28, 4, 128, 511, 7, append=True, seed=2)
    assert B.metok_decode_attention_workspace_bytes(3, 28, 4, 511, 128, B.BF16) == 0
    first = C.call(B, c)
    torch.cuda.synchronize()
    C.check(c, first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        C.call(B, c, out=first)
    for _ in range(3):
        first["out"].fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        C.check(c, first)


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("page", [0, 16, 7])
def test_every_kernel_of_large_caches(dtype, dh, page):
    """Caches beyond the 128 MB from which on they are read past the caches of the chip, with few rows in them, and many in one."""
    row = 2 * 2 * dh * (2 if dtype == "bf16" else 4)
    unit = page or 1
    capacity = ((140 << 20) // (row * 4) // unit + 1) * unit
    run(C.make(dtype, [0, 33, 1500, 100], 8, 2, dh, capacity, page, append=True, seed=dh + page))
    run(C.make(dtype, [0, 33, 1500, 100], 8, 2, dh, capacity, page, append=page == 0, weights=True, seed=dh + page + 1))


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("page", [0, 16, 7])
@pytest.mark.parametrize("Hq", [24, 64])
def test_every_kernel_of_many_query_heads_and_large_caches(dtype, dh, page, Hq):
    """The same beyond 128 MB, with two blocks of query heads at a time and, where they fit, four; and caches below that."""
    row = 2 * dh * (2 if dtype == "bf16" else 4)
    unit = page or 1
    capacity = ((140 << 20) // (row * 3) // unit + 1) * unit
    run(C.make(dtype, [0, 700, 45], Hq, 1, dh, capacity, page, append=True, weights=Hq == 24, seed=dh + page))
    run(C.make(dtype, [0, 700, 45], Hq, 1, dh, 200 * max(unit, 4), page, append=False, cap=10.0, weights=Hq == 64, seed=dh + page + 1))
