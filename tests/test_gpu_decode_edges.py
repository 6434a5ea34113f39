"""GPU tests of the decoding-time calls at the ends of what they take: single rows, padded batches, two calls at once, a whole step in one graph."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from tests import decode_cases as C

pytestmark = pytest.mark.gpu


def mk():
    from paper_2506_02850_amd import binding as B
    return B


def run(c):
    B = mk()
    before = dict(k=c["k"].clone(), v=c["v"].clone())
    weight = None if c["weight"] is None else c["weight"].clone()
    res = C.call(B, c)
    torch.cuda.synchronize()
    C.check(c, res, weight)
    C.check_caches(c, before)


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 256), ("f32", 32), ("f32", 128)])
@pytest.mark.parametrize("capacity,page", [(1, 0), (2, 0), (1, 1), (2, 1), (3, 3)])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (17, 1)])
def test_caches_of_a_row_or_two(dtype, dh, capacity, page, Hq, Hkv):
    for length in range(capacity + 1):
        for weights in (False, True):
            for append in (False, True):
                run(C.make(dtype, [length], Hq, Hkv, dh, capacity, page, append=append, weights=weights, seed=length))


@pytest.mark.parametrize("capacity", [96, 4096])
def test_padded_batches(capacity):
    """Videos that are not there: no rows and a table without pages.  They attend to their new row, nothing of it is stored, and no other video
    changes; the weight of that row is set, as for every row that has a place in the table."""
    B = mk()
    c = C.make("bf16", [50, 0, 33, 0], 8, 2, 64, capacity, 16, append=True, weights=True, seed=3)
    table = c["table_dev"].clone()
    table[1], table[3] = -1, -1
    before, weight = dict(k=c["k"].clone(), v=c["v"].clone()), c["weight"].clone()
    for w in (c["weight"], None):
        for n in ("k", "v"):
            c[n].copy_(before[n])
        res = B.metok_decode_attention_paged(c["q"], c["k"], c["v"], table, c["lens_dev"], k_new=c["k_new"], v_new=c["v_new"], weight=w)
        torch.cuda.synchronize()
        C.check(dict(c, weight=w), res, weight)
        for n, new in (("k", c["k_new"]), ("v", c["v_new"])):
            want = before[n].clone()
            for b, at in ((0, 50), (2, 33)):
                want[int(c["table"][b, at // 16]), :, at % 16] = new[b]
            assert C.same(c[n], want)


def test_two_calls_at_once_have_workspaces_of_their_own():
    """Calls on two streams, with the workspaces that the binding makes: the results of one after the other."""
    B = mk()
    cases = [C.make("bf16", [20000, 300], 28, 4, 128, 20032, 16, append=False, weights=True, seed=1), C.make("f32", [9000], 14, 2, 64, 9008, append=False, weights=True, seed=2)]
    want = []
    for c in cases:
        w = c["weight"].clone()
        for _ in range(5):
            res = C.call(B, c, weight=w)
        want.append((res, w))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [None, None]
    for _ in range(5):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                got[i] = C.call(B, c)
    torch.cuda.synchronize()
    for res, c, (first, w) in zip(got, cases, want):
        assert C.same(res["out"], first["out"]) and C.same(res["lse"], first["lse"]) and C.same(c["weight"], w)


@pytest.mark.parametrize("page", [0, 16])
def test_a_step_of_all_layers_and_an_eviction_in_one_graph(page):
    """Attention of three layers, the lengths' increment and an eviction in one captured graph and one workspace, replayed while the caches grow and
    shrink; every replay equals the eager calls."""
    B = mk()
    L, videos, Hq, Hkv, dh, S, budget = 3, 2, 8, 2, 64, 320, 200
    gen = torch.Generator(device="cuda").manual_seed(page)
    shape = (videos * S // 16, Hkv, 16, dh) if page else (videos, Hkv, S, dh)
    table = torch.randperm(shape[0], generator=gen, device="cuda").int().view(videos, -1) if page else None
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)
    need = max(B.metok_decode_attention_workspace_bytes(videos, Hq, Hkv, S, dh, B.BF16, True), B.metok_kv_evict_workspace_bytes(L, videos, Hkv, S, dh, B.BF16))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def state():
        return dict(k=[rand(*shape) for _ in range(L)], v=[rand(*shape) for _ in range(L)], w=[torch.rand((videos, S), generator=gen, device="cuda") for _ in range(L)],
                    lens=torch.tensor([[198, 150]] * L, dtype=torch.int32, device="cuda"), q=rand(L, videos, Hq, dh), new=rand(L, 2, videos, Hkv, dh),
                    out=[dict(out=torch.empty((videos, Hq, dh), dtype=torch.bfloat16, device="cuda"), lse=torch.empty((videos, Hq), device="cuda")) for _ in range(L)],
                    idx=[torch.empty((videos, budget), dtype=torch.int32, device="cuda") for _ in range(L)])

    def step(s):
        for l in range(L):
            kw = dict(k_new=s["new"][l, 0], v_new=s["new"][l, 1], weight=s["w"][l], workspace=ws, out=s["out"][l])
            if page:
                B.metok_decode_attention_paged(s["q"][l], s["k"][l], s["v"][l], table, s["lens"][l], **kw)
            else:
                B.metok_decode_attention(s["q"][l], s["k"][l], s["v"][l], s["lens"][l], **kw)
        s["lens"] += 1
        kw = dict(n_first=4, n_last=20, idx=s["idx"], new_len=s["lens"], workspace=ws)
        if page:
            B.metok_kv_evict_paged(s["k"], s["v"], table, s["w"], s["lens"], budget, **kw)
        else:
            B.metok_kv_evict(s["k"], s["v"], s["w"], s["lens"], budget, **kw)

    def copy(to, of):
        for n in of:
            for a, b in ([(to[n], of[n])] if isinstance(of[n], torch.Tensor) else zip(to[n], of[n])):
                for x, y in ([(a, b)] if isinstance(a, torch.Tensor) else [(a[m], b[m]) for m in b]):
                    x.copy_(y)

    def tensors(s):
        return s["k"] + s["v"] + s["w"] + [s["lens"]] + [t for o in s["out"] for t in o.values()] + s["idx"]

    a, b = state(), state()
    start = state()
    copy(a, start)
    step(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    copy(a, start)
    copy(b, start)
    torch.cuda.synchronize()
    for it in range(6):
        q, new = rand(*a["q"].shape), rand(*a["new"].shape)
        for s in (a, b):
            s["q"].copy_(q)
            s["new"].copy_(new)
        step(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(C.same(x, y) for x, y in zip(tensors(a), tensors(b))), it
        assert a["lens"].tolist() == [[min(199 + it, budget), 151 + it]] * L


def test_weights_of_equal_rows_are_equal():
    """A cache whose rows are all the same: every weight is 1 / n, and the eviction keeps the first ones."""
    B = mk()
    n, S = 1000, 1200
    k = torch.ones((1, 2, S, 64), dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    w = torch.zeros((1, S), device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    B.metok_decode_attention(torch.ones((1, 8, 64), dtype=torch.bfloat16, device="cuda"), k, v, lens, weight=w)
    assert w[0, :n].unique().numel() == 1 and not w[0, n:].any()
    assert abs(w[0, 0].item() * n - 1) < 4 * 2.0 ** -24
    res = B.metok_kv_evict([k], [v], [w], lens[None], 300, n_first=2, n_last=10)
    assert res["idx"][0][0].tolist() == D.evict(w[0].cpu().numpy(), n, 300, 2, 10) == list(range(290)) + list(range(990, 1000))
