"""Norm, rotation and storage of new tokens' queries, keys and values on the GPU, against the oracle."""
import numpy as np
import pytest
import torch

from oracle import qkv_oracle as Q
from tests.kv4_cases import TORCH, rotate_tolerance, same, typed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2506_02850_amd import binding
    return binding


def i32(x):
    return None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def make(dtype, Bn, n, Hq, Hkv, dh, rot, axes, pairs=Q.HALVES, norm=True, capacity=64, page=0, start=None, count=None, far=1000, packed=True, axis=None, seed=0, scale=1.0):
    rng = np.random.default_rng(seed)
    H = Hq + 2 * Hkv
    x, x64 = typed(scale * rng.standard_normal((Bn, n, H, dh)), dtype)
    parts = (slice(0, Hq), slice(Hq, Hq + Hkv), slice(Hq + Hkv, H))
    rows = [x[:, :, p] if packed else x[:, :, p].contiguous() for p in parts]
    half = rot // 2
    axis = [i % axes for i in range(half)] if axis is None else axis
    freq = np.float32(10000.0) ** (-np.arange(half, dtype=np.float32) * 2 / rot)
    pos = rng.integers(-5 if far < 10 ** 6 else -far, far, (axes, Bn, n)).astype(np.int32)
    weights = [typed(1 + 0.3 * rng.standard_normal(dh), dtype) for _ in range(2)] if norm else [(None, None)] * 2
    if page:
        per_seq = capacity // page
        table = rng.permutation(Bn * per_seq + 2)[:Bn * per_seq].reshape(Bn, per_seq).astype(np.int32)
        shape = (Bn * per_seq + 2, Hkv, page, dh)
    else:
        table, shape = None, (Bn, Hkv, capacity, dh)
    kv = torch.full((2, *shape), 7.0, dtype=TORCH[dtype], device="cuda")
    return dict(dtype=dtype, B=Bn, n=n, Hq=Hq, Hkv=Hkv, dh=dh, half=half, pairs=pairs, rows=rows, x64=[x64[:, :, p] for p in parts], pos=pos, freq=freq, axis=axis,
                weights=weights, kv=kv, table=table, start=start, count=count, capacity=capacity, page=page)


def run(B, c, eps=1e-6, **more):
    kw = dict(start=i32(c["start"]), count=i32(c["count"]), pair_axis=bytes(c["axis"]), pairs=c["pairs"], eps=eps, q_weight=c["weights"][0][0], k_weight=c["weights"][1][0],
              out={"q": torch.full((c["B"], c["Hq"], c["n"], c["dh"]), 7.0, dtype=TORCH[c["dtype"]], device="cuda")})
    kw.update(more)
    args = (*c["rows"], i32(c["pos"]), torch.from_numpy(c["freq"]).cuda(), c["kv"][0], c["kv"][1])
    return (B.metok_rotate_qk_paged(*args, i32(c["table"]), **kw) if c["page"] else B.metok_rotate_qk(*args, **kw))["q"]


def check(c, q, eps=1e-6):
    """Everything that the call wrote is within its tolerance, and everything else is as it was."""
    want_kv = torch.full_like(c["kv"], 7.0)
    q64, kv64 = q.to(torch.float64).cpu().numpy(), c["kv"].to(torch.float64).cpu().numpy()
    for b in range(c["B"]):
        n = min(max(c["count"][b], 0), c["n"]) if c["count"] is not None else c["n"]
        first = max(c["start"][b], 0) if c["start"] is not None else 0
        for which in range(2):
            weight, x = c["weights"][which][1], c["x64"][which][b, :n]
            want = Q.rotate(x, weight, eps, c["pos"][:, b, :n], c["freq"], c["axis"], c["pairs"])
            limit = rotate_tolerance(x, weight, eps, want, c["dtype"], c["dh"], c["half"], c["pairs"])
            if which == 0:
                assert (np.abs(q64[b, :, :n] - want.transpose(1, 0, 2)) <= limit.transpose(1, 0, 2)).all(), f"queries of video {b}"
                assert (q64[b, :, n:] == 7.0).all()
                continue
            for i in range(n):
                j = first + i
                slab, row = b, j
                if j >= c["capacity"]:
                    continue
                if c["page"]:
                    slab, row = int(c["table"][b, j // c["page"]]), j % c["page"]
                    if not 0 <= slab < c["kv"].shape[1]:
                        continue
                assert (np.abs(kv64[0, slab, :, row] - want[i]) <= limit[i]).all(), f"key {i} of video {b}"
                want_kv[0, slab, :, row] = c["kv"][0, slab, :, row]
                want_kv[1, slab, :, row] = c["rows"][2][b, i]
    assert same(c["kv"], want_kv), "the cache is not what it was with the new rows"


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("pairs", [Q.HALVES, Q.ADJACENT])
def test_heads_and_pairs(B, dtype, dh, pairs):
    for rot in sorted({16, dh // 32 * 16, dh, max(16, dh - 16)}):
        for norm in (True, False):
            c = make(dtype, 2, 9, 5, 2, dh, rot, 3, pairs, norm, capacity=40, start=[3, 0], seed=rot)
            check(c, run(B, c))


@pytest.mark.parametrize("Bn,n", [(1, 1), (1, 2), (64, 1), (3, 33), (1, 700), (2, 257), (300, 1)])
def test_tokens(B, Bn, n):
    c = make("bf16", Bn, n, 7, 1, 128, 128, 3, capacity=n + 20, start=[b % 17 for b in range(Bn)], seed=n)
    check(c, run(B, c))


def test_one_axis_four_axes_and_runs_of_axes(B):
    for axes, axis in ((1, None), (2, [0] * 20 + [1] * 12), (4, None), (3, [0] * 8 + [1] * 12 + [2] * 12), (4, [3] * 32)):
        c = make("f32", 2, 5, 4, 2, 64, 64, axes, axis=axis, seed=axes)
        check(c, run(B, c))
    c = make("f32", 2, 5, 4, 2, 64, 64, 1)
    q = run(B, c)
    want, kv = q.clone(), c["kv"].clone()
    c["kv"].fill_(7.0)
    assert same(run(B, c, pair_axis=None), want) and same(c["kv"], kv)
    half = dict(c, pos=c["pos"][0])
    c["kv"].fill_(7.0)
    assert same(run(B, half, pair_axis=None), want)


def test_positions_of_any_size(B):
    """Up to the ends of int32: a fraction of a revolution is the same to 2^-22 there."""
    c = make("f32", 2, 64, 2, 1, 64, 64, 3, far=10 ** 6, norm=False, seed=5)
    check(c, run(B, c))
    c = make("f32", 1, 64, 2, 1, 64, 64, 1, far=2 ** 31 - 1, norm=False, seed=6)
    q = run(B, c).to(torch.float64).cpu().numpy()
    want = Q.rotate(c["x64"][0][0], None, 0.0, c["pos"][:, 0], c["freq"], c["axis"], c["pairs"]).transpose(1, 0, 2)
    # pos * freq has 55 bits of which float64 keeps 53, here and in the oracle, and so do the revolutions: 2^31 * 3 * 2^-53 radians
    size = np.abs(c["x64"][0][0]).transpose(1, 0, 2)
    limit = rotate_tolerance(c["x64"][0][0], None, 0.0, want.transpose(1, 0, 2), "f32", 64, 32, c["pairs"]).transpose(1, 0, 2) + 2.0 ** -19 * (size + np.roll(size, 32, -1))
    assert (np.abs(q[0] - want) <= limit).all()


def test_counts_starts_and_full_caches(B):
    c = make("bf16", 5, 20, 4, 2, 64, 32, 2, capacity=30, start=[0, 25, 30, -7, 2 ** 31 - 1], count=[20, 19, 20, 3, 25], seed=1)
    check(c, run(B, c))
    c = make("bf16", 3, 20, 4, 2, 64, 32, 2, capacity=30, count=[0, -5, 1], seed=2)
    check(c, run(B, c))


@pytest.mark.parametrize("page", [1, 7, 16, 64])
def test_pages(B, page):
    c = make("bf16", 3, 50, 6, 2, 128, 64, 3, capacity=-(-80 // page) * page, page=page, start=[0, 13, 40], count=[50, 49, 50], seed=page)
    c["table"][1, 20 // page], c["table"][2, 50 // page] = -1, c["kv"].shape[1]
    check(c, run(B, c))


def test_strided_rows_and_rows_of_their_own(B):
    packed, apart = (make("f32", 3, 11, 4, 2, 32, 32, 2, packed=p, seed=3) for p in (True, False))
    assert not packed["rows"][0].is_contiguous() and apart["rows"][0].is_contiguous()
    a, b = run(B, packed), run(B, apart)
    assert same(a, b) and same(packed["kv"], apart["kv"])
    check(packed, a)


def test_norms_of_any_size(B):
    """Heads of zeros, tiny and large ones; the sums of squares are fp32 ones."""
    for scale in (1e-15, 1e-4, 1e4, 1e15):
        c = make("f32", 1, 6, 3, 1, 64, 64, 1, scale=scale, seed=8)
        check(c, run(B, c, eps=0.0), eps=0.0)
    c = make("bf16", 1, 4, 2, 1, 128, 128, 1, seed=8)
    for t in c["rows"]:
        t[0, 1] = 0
    for x in c["x64"]:
        x[0, 1] = 0
    check(c, run(B, c, eps=0.0), eps=0.0)
    c["kv"].fill_(7.0)
    check(c, run(B, c, eps=1.0), eps=1.0)


def test_a_captured_step_follows_its_positions(B):
    """The step of a decoding loop in a graph: positions and starts are on the device and grow; every replay is the eager call."""
    c = make("bf16", 2, 1, 4, 2, 64, 64, 3, capacity=16, start=[0, 3], seed=4)
    pos, start, freq = i32(c["pos"]), i32(c["start"]), torch.from_numpy(c["freq"]).cuda()
    out = {"q": torch.zeros((2, 4, 1, 64), dtype=torch.bfloat16, device="cuda")}
    kw = dict(start=start, pair_axis=bytes(c["axis"]), q_weight=c["weights"][0][0], k_weight=c["weights"][1][0], out=out)
    B.metok_rotate_qk(*c["rows"], pos, freq, c["kv"][0], c["kv"][1], **kw)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        B.metok_rotate_qk(*c["rows"], pos, freq, c["kv"][0], c["kv"][1], **kw)
    for step in range(5):
        graph.replay()
        torch.cuda.synchronize()
        got, kv = out["q"].clone(), c["kv"].clone()
        want = B.metok_rotate_qk(*c["rows"], pos, freq, c["kv"][0], c["kv"][1], **dict(kw, out=None))["q"]
        assert same(got, want) and same(kv, c["kv"])
        pos += 1
        start += 1


def specials(dtype, shape, rng):
    """Infinities, NaN, zeros of both signs, the smallest and the largest numbers among ordinary ones."""
    x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TORCH[dtype])
    odd = torch.tensor([np.inf, -np.inf, np.nan, 0.0, -0.0, 1e-40, -1e-40, 3e38, -3e38], dtype=torch.float32).to(TORCH[dtype])
    at = torch.from_numpy(rng.random(shape) < 0.4)
    x[at] = odd[torch.from_numpy(rng.integers(0, len(odd), int(at.sum())))]
    return x.cuda()


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("pairs", [Q.HALVES, Q.ADJACENT])
@pytest.mark.parametrize("page", [0, 16])
def test_what_is_not_rotated_is_copied(B, dtype, dh, pairs, page):
    """Without a norm, the elements behind the rotated ones stay what they are, whatever they are, and touch nothing else."""
    for rot in sorted({16, dh // 32 * 16, max(16, dh - 16)}):
        c = make(dtype, 2, 9, 5, 2, dh, rot, 3, pairs, norm=False, capacity=48, page=page, start=[3, 0], seed=rot)
        plain = run(B, c)
        want = [plain, c["kv"].clone()]
        rest = specials(dtype, (2, 9, 9, dh - rot), np.random.default_rng(rot))          # 5 + 2 + 2 heads
        c["rows"][0]._base[..., rot:] = rest
        c["kv"].fill_(7.0)
        got = [run(B, c), c["kv"]]
        want[0][..., rot:] = rest[:, :, :5].transpose(1, 2)
        for b in range(2):
            for i in range(9):
                j = (c["start"][b]) + i
                slab, row = (int(c["table"][b, j // page]), j % page) if page else (b, j)
                want[1][0, slab, :, row, rot:], want[1][1, slab, :, row, rot:] = rest[b, i, 5:7], rest[b, i, 7:]
        for x, y in zip(got, want):
            assert torch.equal(x.isnan(), y.isnan()) and torch.equal(x.masked_fill(x.isnan(), 0.5), y.masked_fill(y.isnan(), 0.5))
            assert torch.equal(x.signbit() & ~x.isnan(), y.signbit() & ~y.isnan())
