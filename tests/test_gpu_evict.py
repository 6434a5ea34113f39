"""GPU tests of metok_kv_evict, metok_kv_evict_paged and metok_kv_evict_select: index lists, lengths and moved weights equal to the
oracle's, rows of the caches bit for bit."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from tests import decode_cases as C

pytestmark = pytest.mark.gpu


def mk():
    from paper_2506_02850_amd import binding as B
    return B


def weights_of(kind, rng, shape):
    if kind == "attention":                          # heavy tailed, as accumulated probabilities are
        return np.exp(2.0 * rng.standard_normal(shape)).astype(np.float32) / shape[-1]
    if kind == "zeros":                              # rows that were never attended to among others
        return (rng.random(shape) * (rng.random(shape) < 0.3)).astype(np.float32)
    if kind == "equal":
        return np.full(shape, 0.25, dtype=np.float32)
    if kind == "few":                                # few values: ties at the border, across waves
        return rng.integers(0, 4, shape).astype(np.float32)
    if kind == "near":                               # neighbouring floats
        return (np.float32(1.0).view(np.uint32) + rng.integers(0, 50, shape).astype(np.uint32)).view(np.float32)
    if kind == "any":                                # both signs, tiny, huge, infinite
        w = rng.standard_normal(shape).astype(np.float32) * np.exp2(rng.integers(-140, 120, shape)).astype(np.float32)
        w[rng.random(shape) < 0.05] = np.float32(np.inf)
        w[rng.random(shape) < 0.05] = np.float32(-np.inf)
        w[rng.random(shape) < 0.05] = np.float32(-0.0)
        return w
    raise KeyError(kind)


def expected(w, lens, budget, first, last, capacity):
    """Per layer [B, budget] lists and [L, B] lengths."""
    L, B = lens.shape
    lists, new = [], np.zeros((L, B), dtype=np.int32)
    for l in range(L):
        rows = []
        for b in range(B):
            n = min(max(int(lens[l, b]), 0), capacity)
            kept = D.evict(w[l][b], n, budget[l], first, last)
            new[l, b] = len(kept)
            rows.append(D.index_list(kept, budget[l]))
        lists.append(np.stack(rows))
    return lists, new


def check_selection(res, w, lists, new, before=None):
    np.testing.assert_array_equal(res["new_len"].cpu().numpy(), new)
    for l, ix in enumerate(lists):
        np.testing.assert_array_equal(res["idx"][l].cpu().numpy(), ix)
        got = res["weight"][l].cpu().numpy()
        for b in range(ix.shape[0]):
            n = new[l, b]
            np.testing.assert_array_equal(got[b, :n], w[l][b][ix[b, :n]])
            if before is not None:
                np.testing.assert_array_equal(got[b, n:].view(np.uint32), before[l][b, n:].view(np.uint32), err_msg="behind the last row")


@pytest.mark.parametrize("kind", ["attention", "zeros", "equal", "few", "near", "any"])
@pytest.mark.parametrize("n,budget,first,last", [(1, 1, 0, 0), (2, 1, 0, 0), (2, 1, 1, 0), (2, 1, 0, 1), (65, 64, 3, 3), (777, 500, 1, 33), (1024, 1023, 0, 0),
                                                 (1025, 512, 4, 508), (4224, 4096, 4, 128), (5000, 10, 0, 0), (40960, 20000, 4, 64), (41000, 40000, 7, 9),
                                                 (70001, 513, 0, 100), (300, 300, 10, 10), (4096, 1, 0, 0)])
def test_selection(kind, n, budget, first, last):
    B = mk()
    rng = np.random.default_rng(n * 7 + budget)
    S = n + 5
    w = [weights_of(kind, rng, (2, S + 3)) for _ in range(2)]
    lens = np.array([[n, min(n, budget)], [max(1, n - 1), n]], dtype=np.int32)
    lists, new = expected(w, lens, [budget] * 2, first, last, S)
    dev = [torch.from_numpy(x).cuda() for x in w]
    # to buffers of their own, then in place
    to = [torch.full_like(x, -7.0) for x in dev]
    res = B.metok_kv_evict_select(dev, torch.from_numpy(lens).cuda(), S, budget, first, last, weight_out=to)
    torch.cuda.synchronize()
    check_selection(res, w, lists, new, [np.full_like(x, -7.0) for x in w])
    for x, y in zip(dev, w):
        np.testing.assert_array_equal(x.cpu().numpy().view(np.uint32), y.view(np.uint32))
    held = torch.from_numpy(lens).cuda()
    res = B.metok_kv_evict_select(dev, held, S, budget, first, last, new_len=held)
    torch.cuda.synchronize()
    assert res["new_len"] is held
    check_selection(res, w, lists, new, w)


def test_many_layers_and_budgets():
    B = mk()
    rng = np.random.default_rng(4)
    L, videos, S = 128, 3, 333
    w = [weights_of("attention", rng, (videos, S)) for _ in range(L)]
    lens = rng.integers(0, S + 1, (L, videos)).astype(np.int32)
    budget = [int(x) for x in rng.integers(40, S + 1, L)]
    lists, new = expected(w, lens, budget, 3, 30, S)
    res = B.metok_kv_evict_select([torch.from_numpy(x).cuda() for x in w], torch.from_numpy(lens).cuda(), S, budget, 3, 30)
    torch.cuda.synchronize()
    check_selection(res, w, lists, new, w)


def test_lengths_beyond_the_ends():
    B = mk()
    rng = np.random.default_rng(5)
    w = [weights_of("attention", rng, (5, 64))]
    lens = np.array([[-1, -2 ** 31, 65, 2 ** 31 - 1, 64]], dtype=np.int32)
    lists, new = expected(w, lens, [32], 0, 0, 64)
    res = B.metok_kv_evict_select([torch.from_numpy(x).cuda() for x in w], torch.from_numpy(lens).cuda(), 64, 32)
    torch.cuda.synchronize()
    check_selection(res, w, lists, new, w)


def test_nan_weights_stay_in_bounds_and_are_ordered_by_sign():
    """Positive NaNs come above infinity, negative ones below minus infinity; the lists stay ascending and full."""
    B = mk()
    w = np.linspace(1.0, 2.0, 200, dtype=np.float32)
    w[[10, 50]] = np.float32(np.nan)
    w[[20, 60]] = np.array([0xffc00000], dtype=np.uint32).view(np.float32)
    res = B.metok_kv_evict_select([torch.from_numpy(w[None]).cuda()], torch.tensor([[200]], dtype=torch.int32, device="cuda"), 200, 50)
    kept = set(res["idx"][0][0].tolist())
    assert {10, 50} <= kept and not {20, 60} & kept and len(kept) == 50


def caches(rng, L, shape, dtype):
    kind = torch.int16 if dtype == "bf16" else torch.int32
    k, v = ([torch.randint(-2 ** 15, 2 ** 15, shape, dtype=kind, device="cuda").view(C.TORCH[dtype]) for _ in range(L)] for _ in range(2))
    return k, v


def bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32).cpu().numpy()


@pytest.mark.parametrize("dtype,Hkv,dh,page", [("bf16", 4, 128, 0), ("f32", 2, 64, 0), ("bf16", 2, 32, 16), ("bf16", 1, 128, 7), ("f32", 3, 32, 1), ("bf16", 2, 64, 64)])
def test_caches_follow_the_selection(dtype, Hkv, dh, page):
    B = mk()
    rng = np.random.default_rng(page + dh)
    torch.manual_seed(page + dh)
    L, videos = 4, 3
    S = 1300 if page == 0 else page * -(-1300 // page)
    lens = rng.integers(1000, S + 1, (L, videos)).astype(np.int32)
    lens[0, 0], lens[1, 1], lens[2, 2] = S, 600, 0
    budget = [700, 900, 700, 512]
    first, last = 4, 100
    w = [weights_of("attention", rng, (videos, S)) for _ in range(L)]
    lists, new = expected(w, lens, budget, first, last, S)
    if page == 0:
        table, shape = None, (videos, Hkv, S, dh)
    else:
        per_seq = S // page
        table = rng.permutation(videos * per_seq + 3)[:videos * per_seq].reshape(videos, per_seq).astype(np.int32)
        shape = (videos * per_seq + 3, Hkv, page, dh)
    k, v = caches(rng, L, shape, dtype)
    before = [[bits(t) for t in x] for x in (k, v)]
    dev_w = [torch.from_numpy(x).cuda() if l != 3 else None for l, x in enumerate(w)]
    args = (dev_w, torch.from_numpy(lens).cuda(), budget, first, last)
    need = B.metok_kv_evict_workspace_bytes(L, videos, Hkv, S, dh, B.BF16 if dtype == "bf16" else B.F32)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    res = B.metok_kv_evict(k, v, *args, workspace=ws) if page == 0 else B.metok_kv_evict_paged(k, v, torch.from_numpy(table).cuda(), *args, workspace=ws)
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)[0]) == 0
    new[3] = lens[3]                                 # the layer that was left alone
    np.testing.assert_array_equal(res["new_len"].cpu().numpy(), new)
    assert res["idx"][3] is None
    for l in range(L):
        for old, now in ((before[0][l], bits(k[l])), (before[1][l], bits(v[l]))):
            if l == 3:
                np.testing.assert_array_equal(now, old)
                continue
            np.testing.assert_array_equal(res["idx"][l].cpu().numpy(), lists[l])
            want = old.copy()
            for b in range(videos):
                for i in range(new[l, b]):
                    j = lists[l][b, i]
                    if page == 0:
                        want[b, :, i] = old[b, :, j]
                    else:
                        want[table[b, i // page], :, i % page] = old[table[b, j // page], :, j % page]
            np.testing.assert_array_equal(now, want)


def test_selection_feeds_page_relinking():
    """metok_kv_evict_select's lists go into metok_kv_relink_paged as they are."""
    B = mk()
    rng = np.random.default_rng(9)
    torch.manual_seed(9)
    L, videos, Hkv, page, dh, per_seq = 2, 2, 2, 16, 64, 40
    S = page * per_seq
    table = rng.permutation(videos * per_seq)[:videos * per_seq].reshape(videos, per_seq).astype(np.int32)
    k, v = caches(rng, L, (videos * per_seq, Hkv, page, dh), "bf16")
    before = [bits(t) for t in k]
    w = [weights_of("attention", rng, (videos, S)) for _ in range(L)]
    lens = np.full((L, videos), S, dtype=np.int32)
    sel = B.metok_kv_evict_select([torch.from_numpy(x).cuda() for x in w], torch.from_numpy(lens).cuda(), S, 300, 32, 64)
    out = B.metok_kv_relink_paged(k, v, torch.from_numpy(table).cuda(), sel["idx"], len_in=[S] * L)
    torch.cuda.synchronize()
    lists, _ = expected(w, lens, [300] * L, 32, 64, S)
    tables = out["page_table_out"].cpu().numpy()
    for l in range(L):
        now = bits(k[l])
        for b in range(videos):
            for i in (0, 31, 32, 150, 299):
                j = lists[l][b, i]
                np.testing.assert_array_equal(now[tables[l, b, i // page], :, i % page], before[l][table[b, j // page], :, j % page])


def test_captured_eviction_replays():
    B = mk()
    rng = np.random.default_rng(10)
    torch.manual_seed(10)
    L, videos, Hkv, S, dh = 3, 2, 2, 900, 64
    k, v = caches(rng, L, (videos, Hkv, S, dh), "bf16")
    w = [torch.rand((videos, S), device="cuda") for _ in range(L)]
    lens = torch.full((L, videos), 800, dtype=torch.int32, device="cuda")
    need = B.metok_kv_evict_workspace_bytes(L, videos, Hkv, S, dh, B.BF16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    idx = [torch.empty((videos, 500), dtype=torch.int32, device="cuda") for _ in range(L)]
    out = [torch.zeros_like(x) for x in w]
    new_len = torch.zeros_like(lens)

    def step():
        return B.metok_kv_evict(k, v, w, lens, 500, 2, 40, weight_out=out, idx=idx, new_len=new_len, workspace=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for it in range(4):
        for t in k + v:
            t.copy_(torch.randn(t.shape, device="cuda"))
        for t in w:
            t.copy_(torch.rand(t.shape, device="cuda"))
        lens.copy_(torch.randint(300, 901, lens.shape, dtype=torch.int32, device="cuda"))
        keep = [[t.clone() for t in x] for x in (k, v)]
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in x] for x in (k, v, idx, out)] + [new_len.clone()]
        for x, y in zip((k, v), keep):
            for t, old in zip(x, y):
                t.copy_(old)
        for t in out:
            t.zero_()
        step()
        torch.cuda.synchronize()
        for x, y in zip((k, v, idx), got):
            for t, old in zip(x, y):
                assert C.same(t, old)
        assert torch.equal(new_len, got[4])
        for l in range(L):
            for b in range(videos):
                n = int(new_len[l, b])
                assert torch.equal(out[l][b, :n], got[3][l][b, :n])


def test_refusals():
    B = mk()
    k = [torch.zeros((2, 2, 64, 64), dtype=torch.bfloat16, device="cuda")]
    v = [torch.zeros_like(k[0])]
    w = [torch.zeros((2, 64), device="cuda")]
    lens = torch.full((1, 2), 60, dtype=torch.int32, device="cuda")
    for bad in (dict(budget=0), dict(budget=65), dict(budget=10, n_first=6, n_last=5), dict(budget=10, n_first=-1)):
        with pytest.raises(B.MetokError):
            B.metok_kv_evict(k, v, w, lens, **bad)
    with pytest.raises(ValueError):
        B.metok_kv_evict(k, v, w, lens.long(), 10)
    with pytest.raises(ValueError):
        B.metok_kv_evict(k, v, w, lens[0], 10)
    with pytest.raises(ValueError):
        B.metok_kv_evict(k, v, [w[0].double()], lens, 10)
    with pytest.raises(ValueError):
        B.metok_kv_evict(k, v, [None], lens, 10)
    with pytest.raises(ValueError):
        B.metok_kv_evict(k + k, v, w, lens, 10)
    with pytest.raises(ValueError):
        B.metok_kv_evict(k, v, w, lens, [10, 10])
    with pytest.raises(ValueError):
        B.metok_kv_evict(k, v, w, lens, 10, idx=[torch.zeros((2, 9), dtype=torch.int32, device="cuda")])
    with pytest.raises(ValueError):
        B.metok_kv_evict([k[0].cpu()], v, w, lens, 10)
    with pytest.raises(B.MetokError):
        B.metok_kv_evict(k, v, [w[0][:, :63].contiguous()], lens, 10)
    with pytest.raises(B.MetokError):
        B.metok_kv_evict(k, v, w, lens, 10, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert not w[0].any()


@pytest.mark.parametrize("S", [96, 9000, 41000])
def test_lengths_in_place_of_many_videos(S):
    """new_len may be len: every wave of a video's workgroup has to see the old length."""
    B = mk()
    L, videos = (4, 1024) if S == 96 else (3, 40)
    rng = np.random.default_rng(S)
    w = [weights_of("attention", rng, (videos, S)) for _ in range(L)]
    lens = rng.integers(S // 3, S + 1, (L, videos)).astype(np.int32)
    budget = [S // 2 - 5 * l for l in range(L)]
    lists, new = expected(w, lens, budget, 3, 11, S)
    held = torch.from_numpy(lens).cuda()
    res = B.metok_kv_evict_select([torch.from_numpy(x).cuda() for x in w], held, S, budget, 3, 11, new_len=held)
    torch.cuda.synchronize()
    check_selection(res, w, lists, new)


@pytest.mark.parametrize("page", [0, 4])
def test_caches_of_many_videos(page):
    """More (layer, video) pairs than a workgroup of the row mover has threads; every third video is within the budget, some are empty."""
    B = mk()
    L, videos, Hkv, dh, S = 2, 1500, 2, 8, 40
    rng = np.random.default_rng(page)
    lens = rng.integers(21, S + 1, (L, videos)).astype(np.int32)
    lens[:, ::3] = rng.integers(0, 21, lens[:, ::3].shape)
    lens[:, 1000:1400] = 20                          # a long run in which nothing moves
    w = [weights_of("attention", rng, (videos, S)) for _ in range(L)]
    lists, new = expected(w, lens, [20] * L, 1, 3, S)
    per_seq = S // page if page else 0
    table = rng.permutation(videos * per_seq).reshape(videos, per_seq).astype(np.int32) if page else None
    shape = (videos * per_seq, Hkv, page, dh) if page else (videos, Hkv, S, dh)
    k, v = caches(rng, L, shape, "f32")
    before = [[bits(t) for t in x] for x in (k, v)]
    args = ([torch.from_numpy(x).cuda() for x in w], torch.from_numpy(lens).cuda(), 20, 1, 3)
    res = B.metok_kv_evict_paged(k, v, torch.from_numpy(table).cuda(), *args) if page else B.metok_kv_evict(k, v, *args)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(res["new_len"].cpu().numpy(), new)
    for l in range(L):
        np.testing.assert_array_equal(res["idx"][l].cpu().numpy(), lists[l])
        for old, now in ((before[0][l], bits(k[l])), (before[1][l], bits(v[l]))):
            want = old.copy()
            for b in range(videos):
                n = new[l, b]
                i, j = np.arange(n), lists[l][b, :n]
                if page:
                    want[table[b, i // page], :, i % page] = old[table[b, j // page], :, j % page]
                else:
                    want[b][:, i] = old[b][:, j]
            np.testing.assert_array_equal(now, want)


def test_pages_shared_among_the_first_rows():
    """Two videos share the pages of their first 32 rows, which stay: nothing there moves."""
    B = mk()
    rng = np.random.default_rng(4)
    videos, Hkv, page, dh, S = 2, 2, 16, 32, 320
    lens = np.array([[300, 277]], dtype=np.int32)
    w = [weights_of("attention", rng, (videos, S))]
    lists, new = expected(w, lens, [150], 32, 20, S)
    table = rng.permutation(videos * 20).reshape(videos, 20).astype(np.int32)
    table[1, :2] = table[0, :2]
    k, v = caches(rng, 1, (videos * 20, Hkv, page, dh), "bf16")
    before = [bits(k[0]), bits(v[0])]
    res = B.metok_kv_evict_paged(k, v, torch.from_numpy(table).cuda(), [torch.from_numpy(w[0]).cuda()], torch.from_numpy(lens).cuda(), 150, 32, 20)
    torch.cuda.synchronize()
    check_selection(res, w, lists, new)
    for old, now in zip(before, (bits(k[0]), bits(v[0]))):
        want = old.copy()
        for b in range(videos):
            i, j = np.arange(150), lists[0][b]
            want[table[b, i // page], :, i % page] = old[table[b, j // page], :, j % page]
        np.testing.assert_array_equal(now, want)


@pytest.mark.parametrize("page", [0, 8])
@pytest.mark.parametrize("L", [41, 128])
def test_more_layers_than_a_launch_of_the_row_mover_takes(L, page):
    """Budgets and lengths of their own, several tiles a layer, of the 128 every ninth left alone: caches, lists, weights and lengths of all."""
    B = mk()
    videos, Hkv, dh, S = 2, 1, 16, 4800
    rng = np.random.default_rng(L + page)
    torch.manual_seed(L + page)
    lens = rng.integers(2000, S + 1, (L, videos)).astype(np.int32)
    budget = [int(x) for x in rng.integers(200, 4500, L)]
    alone = set(range(4, L, 9)) if L > 41 else set()
    w = [weights_of("attention", rng, (videos, S)) for _ in range(L)]
    lists, new = expected(w, lens, budget, 3, 40, S)
    for l in alone:
        new[l] = lens[l]
    per_seq = S // page if page else 0
    table = rng.permutation(videos * per_seq).reshape(videos, per_seq).astype(np.int32) if page else None
    shape = (videos * per_seq, Hkv, page, dh) if page else (videos, Hkv, S, dh)
    k, v = caches(rng, L, shape, "f32")
    before = [[bits(t) for t in x] for x in (k, v)]
    need = B.metok_kv_evict_workspace_bytes(L, videos, Hkv, S, dh, B.F32)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    args = ([None if l in alone else torch.from_numpy(x).cuda() for l, x in enumerate(w)], torch.from_numpy(lens).cuda(), budget, 3, 40)
    res = B.metok_kv_evict_paged(k, v, torch.from_numpy(table).cuda(), *args, workspace=ws) if page else B.metok_kv_evict(k, v, *args, workspace=ws)
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)[0]) == 0
    np.testing.assert_array_equal(res["new_len"].cpu().numpy(), new)
    for l in range(L):
        if l not in alone:
            np.testing.assert_array_equal(res["idx"][l].cpu().numpy(), lists[l])
        for old, now in ((before[0][l], bits(k[l])), (before[1][l], bits(v[l]))):
            want = old.copy()
            for b in range(videos):
                if l in alone:
                    continue
                i, j = np.arange(new[l, b]), lists[l][b, :new[l, b]]
                if page:
                    want[table[b, i // page], :, i % page] = old[table[b, j // page], :, j % page]
                else:
                    want[b][:, i] = old[b][:, j]
                    got = res["weight"][l].cpu().numpy()
                    np.testing.assert_array_equal(got[b, i], w[l][b][j])
            np.testing.assert_array_equal(now, want)


@pytest.mark.parametrize("page", [0, 16])
def test_waits_that_expire_are_reported(page):
    """Every tile waits for the one before; without polls a wait may be given up: the call ends, says so in the workspace's first word and has replaced
    lengths and weights.  The next call is whole."""
    B = mk()
    Hkv, S, dh, layers = 2, 24000, 128, 2
    torch.manual_seed(page)
    weight = torch.rand((1, S), generator=torch.Generator().manual_seed(1)) + 1
    weight[0, 0] = 0.5                               # the first row leaves, all others move up by one
    shape = (S // page, Hkv, page, dh) if page else (1, Hkv, S, dh)
    table = torch.arange(S // page, dtype=torch.int32, device="cuda")[None] if page else None
    need = B.metok_kv_evict_workspace_bytes(layers, 1, Hkv, S, dh, B.BF16)

    def evict():
        k, v = caches(None, layers, shape, "bf16")
        old = [t.clone() for t in k + v]
        w = [weight.cuda() for _ in range(layers)]
        lens = torch.full((layers, 1), S, dtype=torch.int32, device="cuda")
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        args = (w, lens, S - 1)
        res = (B.metok_kv_evict_paged(k, v, table, *args, new_len=lens, workspace=ws) if page else B.metok_kv_evict(k, v, *args, new_len=lens, workspace=ws))
        torch.cuda.synchronize()
        assert lens.tolist() == [[S - 1]] * layers
        for l in range(layers):
            assert torch.equal(res["idx"][l][0].cpu(), torch.arange(1, S, dtype=torch.int32)) and torch.equal(w[l][0, :S - 1].cpu(), weight[0, 1:])
        rows = lambda t: t.transpose(0, 1).reshape(Hkv, S, dh) if page else t[0]
        moved = all(C.same(rows(t)[:, :S - 1], rows(o)[:, 1:]) and C.same(rows(t)[:, S - 1:], rows(o)[:, S - 1:]) for t, o in zip(k + v, old))
        return int(ws[:4].view(torch.int32)[0]), moved

    try:
        B.metok_debug_set_move_spin_limit(0)
        error, moved = evict()
        print(f"poll limit 0: error word {error}")
        assert error == 1 or (error == 0 and moved)
    finally:
        B.metok_debug_set_move_spin_limit(1 << 24)
    assert evict() == (0, True)
