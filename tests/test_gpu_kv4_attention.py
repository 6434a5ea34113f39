"""Attention of one new token over a 4-bit cache on the GPU, against the oracle over the values that the cache stands for."""
import pytest
import torch

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


KINDS = [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64), ("f32", 128)]


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("page", [0, 16])
def test_short_caches(B, dtype, dh, page):
    """One launch; single rows, none, ends of blocks and tiles."""
    for lens in ([0, 1, 15], [16, 17, 31], [63, 64, 65], [127, 100, 0]):
        go(B, K.make(dtype, lens, 6, 2, dh, 128, page, seed=sum(lens)))
        go(B, K.make(dtype, lens, 6, 2, dh, 128, page, append=False, seed=sum(lens)))


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("page", [0, 32])
def test_split_caches(B, dtype, dh, page):
    """Two launches: parts of several waves are joined."""
    go(B, K.make(dtype, [1500, 3, 0, 1187], 4, 2, dh, 2048 if dh > 128 else 4096, page, seed=dh))
    go(B, K.make(dtype, [1500, 64], 4, 2, dh, 2048 if dh > 128 else 4096, page, weights=True, cap=20.0, append=False, seed=dh))


@pytest.mark.parametrize("dtype,dh", KINDS)
def test_weights(B, dtype, dh):
    for capacity, lens in ((64, [0, 1, 63, 64]), (336, [200, 335, 7, 336])):
        go(B, K.make(dtype, lens, 4, 2, dh, capacity, weights=True, seed=capacity))
        go(B, K.make(dtype, lens, 4, 2, dh, capacity, 16, weights=True, append=False, cap=5.0, seed=capacity))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (28, 4), (16, 1), (17, 1), (40, 40), (71, 1), (64, 2), (33, 3)])
def test_heads(B, Hq, Hkv):
    for weights in (False, True):
        go(B, K.make("bf16", [200, 90], Hq, Hkv, 64, 256, weights=weights, seed=Hq))
    go(B, K.make("f32", [77], Hq, Hkv, 32, 112, 16, seed=Hq))


def test_full_caches_and_lengths_out_of_range(B):
    """A full video's new row is attended to, but not stored; lengths are clamped."""
    for page in (0, 16):
        go(B, K.make("bf16", [48, 47, 60, -5], 4, 2, 128, 48, page, seed=1))
        go(B, K.make("bf16", [48, 47, 60, -5], 4, 2, 128, 48, page, weights=True, seed=1))
        go(B, K.make("f32", [48, 47, 60, -5], 4, 2, 64, 48, page, append=False, seed=1))


def test_pages_that_are_none(B):
    """Rows behind them take no part, a new row there is not stored; pages of one block and of several, in the middle of a tile."""
    for page in (16, 48):
        for weights in (False, True):
            broken = [(0, 0, -1), (0, 96 // page, 10 ** 6), (1, 144 // page, -7), (2, 0, -1), (2, 1, -1)]
            c = K.make("bf16", [144, 150, 20], 4, 2, 128, 192, page, weights=False, broken=broken, seed=page)
            before = None
            if weights:                                    # the weights of rows that take no part grow by nothing
                c["weight"] = torch.zeros((3, 192), device="cuda")
                before = c["weight"].clone()
            res = K.call(B, c)
            w, c["weight"] = c["weight"], None
            K.check(c, res)
            K.check_cache(c)
            if weights:
                gone = torch.zeros((3, 192), dtype=torch.bool)
                for b, p, _ in broken:
                    gone[b, p * page:(p + 1) * page] = True
                n = torch.tensor([144, 150, 20])[:, None]
                at = torch.arange(192)[None]
                assert (w.cpu()[gone & (at < n)] == 0).all()
                assert torch.allclose(w.sum(1).cpu(), torch.ones(3), atol=1e-5)


def test_scales_and_caps(B):
    for scale, cap in ((1.0, 0.0), (1e-3, 0.0), (30.0, 0.0), (0.125, 1.0), (2.0, 50.0)):
        go(B, K.make("bf16", [100, 500], 4, 2, 64, 512, cap=cap, seed=3), scale=scale)
        go(B, K.make("f32", [100, 500], 4, 2, 64, 512, cap=cap, seed=3), scale=scale)


def test_large_scores(B):
    """Scores whose exponentials no type holds, in fp32 with all their bits."""
    for dtype in ("bf16", "f32"):
        go(B, K.make(dtype, [300, 2000], 2, 1, 64, 2048, spread=300.0, seed=11), scale=1.0)


def test_one_row_is_its_value(B):
    """One row: the probability is 1, and the result is the row as 4 bits have it."""
    for dtype, dh in KINDS:
        c = K.make(dtype, [0], 3, 1, dh, 16, seed=dh)
        res = K.call(B, c)
        want = torch.from_numpy(K.attended(c)[1][0][0]).to(K.TORCH[dtype])
        assert torch.equal(res["out"][0].cpu(), want.expand(3, dh))          # a sum that is 0 has no sign


def test_results_do_not_depend_on_what_lies_behind_the_rows_or_in_the_workspace(B):
    outs = []
    for fill in (0, 255):
        c = K.make("bf16", [1000, 70], 28, 4, 128, 2048, weights=True, append=False, seed=5)
        need = B.metok_kv4_attention_workspace_bytes(2, 28, 4, 2048, 128, B.BF16, True)
        for t in (c["k"], c["v"]):
            t[0, :, 63:] = fill                            # rows from 1008 on
            t[1, :, 5:] = fill
        res = K.call(B, c, workspace=torch.full((need,), fill, dtype=torch.uint8, device="cuda"))
        outs.append((res["out"], res["lse"], c["weight"]))
    assert all(same(x, y) for x, y in zip(*outs))


def test_repeated_calls_are_equal_bit_for_bit(B):
    c = K.make("bf16", [3000, 1, 700, 2047], 28, 4, 128, 3008, 16, append=False, seed=6)
    first = K.call(B, c)
    for _ in range(5):
        again = K.call(B, c)
        assert same(first["out"], again["out"]) and same(first["lse"], again["lse"])


def test_a_captured_loop_is_the_eager_one(B):
    """Twenty tokens, lengths on the device: replays of one captured call against eager calls on a copy of the cache."""
    for capacity, page in ((128, 0), (4096, 32)):
        c = K.make("bf16", [40, 100], 8, 2, 64, capacity, page, weights=True, seed=7)
        eager = {x: c[x].clone() for x in ("k", "v", "weight", "lens_dev")}
        out = {x: torch.zeros_like(t) for x, t in K.call(B, dict(c, **{x: t.clone() for x, t in eager.items()})).items()}
        ws = torch.empty(max(B.metok_kv4_attention_workspace_bytes(2, 8, 2, capacity, 64, B.BF16, True), 256), dtype=torch.uint8, device="cuda")
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            K.call(B, c, out=out, workspace=ws)
            c["lens_dev"] += 1
        for step in range(20):
            for x in ("q", "k_new", "v_new"):
                c[x].normal_()
            graph.replay()
            want = K.call(B, dict(c, **eager))
            eager["lens_dev"] += 1
            torch.cuda.synchronize()
            assert same(out["out"], want["out"]) and same(out["lse"], want["lse"]), step
        assert same(c["k"], eager["k"]) and same(c["v"], eager["v"]) and same(c["weight"], eager["weight"])


@pytest.mark.parametrize("dtype,dh", KINDS)
@pytest.mark.parametrize("rows,page", [(700, 0), (3000, 32)])
def test_the_largest_scores_and_values(B, dtype, dh, rows, page):
    """Queries and values at the end of the documented range: rows that agree with the query in every sign, all alike, have the whole weight, the others, which disagree,
    none.  Equal rows have equal scores, so the result is these rows' value: off by its rounding, by that of the sums of up to two (fp32: three) products for 32 rows
    and by some 64 roundings on the way; the scores are sums of dh (fp32: 3 dh) products of one sign."""
    big, capacity = 6 * 2.0 ** 100, -(-rows // 32) * 32 + 32
    g = torch.Generator().manual_seed(dh)
    sign = torch.randint(0, 2, (2, dh), generator=g) * 2.0 - 1.0
    q = (sign[0] * (2.0 ** 25 / dh * (1 - 2 * K.HALF[dtype]))).to(K.TORCH[dtype]).expand(1, 4, dh).contiguous().cuda()
    assert 2.0 ** 102 * dh * float(q.abs().max()) < 2.0 ** 127 and float(q.abs().max()) >= 2.0 ** 25 / dh * (1 - 2.0 ** -6)
    with_it = torch.randint(0, 2, (rows,), generator=g).bool()
    k = torch.where(with_it[:, None], big * sign[0], -big * sign[0]).to(K.TORCH[dtype])
    v = torch.where(with_it[:, None], big * sign[1], -big).to(K.TORCH[dtype])
    k, v = (x.expand(1, 2, rows, dh).contiguous().cuda() for x in (k, v))
    lens = torch.tensor([rows], dtype=torch.int32, device="cuda")
    if page:
        table = torch.randperm(capacity // page, generator=g).int().view(1, -1).cuda()
        four = [t.fill_(130) for t in B.metok_kv4_cache(capacity // page, 2, page, dh, "cuda")]
        B.metok_kv4_pack_paged(k, v, *four, table)
        res = B.metok_kv4_attention_paged(q, *four, table, lens)
    else:
        four = [t.fill_(130) for t in B.metok_kv4_cache(1, 2, capacity, dh, "cuda")]
        B.metok_kv4_pack(k, v, *four)
        res = B.metok_kv4_attention(q, *four, lens)
    want = (big * sign[1]).double()
    parts = (1, 2) if dtype == "bf16" else (3, 3)
    tol = K.HALF[dtype] + (parts[1] * rows / 32 + 64) * K.U
    assert (res["out"].double().cpu() - want).abs().max() <= tol * big
    score = float(q.double().abs()[0, 0].sum()) * big * dh ** -0.5
    assert (res["lse"].double().cpu() - score - float(with_it.sum().double().log())).abs().max() <= (parts[0] * dh + 8) * K.U * score


def test_sums_of_the_largest_values_over_a_long_cache(B):
    """160000 rows of the largest value, whose scores grow by almost 2^8 within the tiles' runs: the sums stay finite, and the result is the value,
    off by its rounding and by at most one rounding for each of the two products of 32 rows and 64 more; the sum of the probabilities likewise."""
    rows, dh, big = 160000, 32, 6 * 2.0 ** 100
    at = torch.arange(rows, device="cuda")
    for run in (32, 96, 80000):
        high = (at // run) % 2 == 1
        k = torch.where(high[:, None], 1.0, 0.0).expand(rows, dh).to(torch.bfloat16).expand(1, 1, rows, dh).contiguous()
        v = torch.full((1, 1, rows, dh), big, dtype=torch.bfloat16, device="cuda")
        q = torch.full((1, 2, dh), 1.0, dtype=torch.bfloat16, device="cuda")
        four = B.metok_kv4_cache(1, 1, rows, dh, "cuda")
        B.metok_kv4_pack(k, v, *four)
        res = B.metok_kv4_attention(q, *four, torch.tensor([rows], dtype=torch.int32, device="cuda"), scale=7.99 / 1.4426950408889634 / dh)
        assert (res["out"].double() - big).abs().max() <= (2.0 ** -8 + (2 * rows / 32 + 64) * K.U) * big
        want = torch.log(high.sum().double() * 2 ** 7.99 + (~high).sum().double())
        assert (res["lse"].double() - want).abs().max() <= (2 * rows / 32 + 64) * K.U
