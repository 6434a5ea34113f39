"""The native marshalling of the decoding-time calls against the step-by-step path: the same outputs bit for bit, what is not of the
ordinary form is declined before anything happens, and nothing that can fail follows the launch."""
import gc

import pytest
import torch

from tests.test_native_binding import both

B = pytest.importorskip("paper_2506_02850_amd.binding")


def leaves(x, path=""):
    if isinstance(x, dict):
        for n, v in x.items():
            yield from leaves(v, f"{path}.{n}")
    elif isinstance(x, (list, tuple)):
        for i, v in enumerate(x):
            yield from leaves(v, f"{path}[{i}]")
    else:
        yield path, x


def check_same(native, plain):
    a, b = list(leaves(native)), list(leaves(plain))
    assert [p for p, _ in a] == [p for p, _ in b]
    for (path, x), (_, y) in zip(a, b):
        if isinstance(x, torch.Tensor):
            assert x.dtype == y.dtype and torch.equal(x, y), path
        else:
            assert x is y is None, path


def test_calls_off_the_gpu_are_declined():
    q, kv, lens = torch.zeros(1, 4, 64), torch.zeros(1, 2, 32, 64), torch.zeros(1, dtype=torch.int32)
    asked = []
    assert B._host.decode_attention(q, kv, kv, None, lens, None, None, None, 0.0, None, None, None, asked.append) is None
    w = torch.zeros(1, 32)
    assert B._host.kv_evict([w], lens[None], 16, 0, 0, None, None, None, [kv], [kv], None, None, asked.append) is None
    assert B._host.kv_evict_select([w], lens[None], 16, 0, 0, None, None, None, 32, asked.append) is None
    assert not asked
    with pytest.raises(TypeError):
        B._host.decode_attention(q, kv, kv)
    with pytest.raises(ValueError, match="GPU"):
        B.metok_decode_attention(q, kv, kv, lens)
    with pytest.raises(ValueError, match="GPU"):
        B.metok_kv_evict([kv], [kv], [w], lens[None], 16)
    with pytest.raises(ValueError, match="GPU"):
        B.metok_kv_evict_select([w], lens[None], 32, 16)


def test_budgets_are_numbers_of_any_kind_or_one_per_layer():
    import numpy as np
    w, lens = [torch.zeros(1, 32)] * 2, torch.zeros(2, 1, dtype=torch.int32)
    for budget in (16, np.int64(16), np.array(16), torch.tensor(16), [16, 8], (np.int32(16), 8), np.array([16, 8]), torch.tensor([16, 8])):
        with pytest.raises(ValueError, match="GPU"):             # taken: what is wrong is the tensors' place
            B.metok_kv_evict_select(w, lens, 32, budget)
    for budget in (16.5, [16, 8.5], "16", None):
        with pytest.raises(TypeError):
            B.metok_kv_evict_select(w, lens, 32, budget)
    for budget in ([16], np.array([16, 8, 4])):
        with pytest.raises(ValueError, match="budget"):
            B.metok_kv_evict_select(w, lens, 32, budget)


def attention_inputs(paged, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(3)
    shape = (2, 2, 96, 64) if not paged else (12, 2, 16, 64)
    kv = torch.randn((2,) + shape, generator=g, device="cuda").to(dtype)
    return dict(q=torch.randn((2, 8, 64), generator=g, device="cuda").to(dtype), kv=kv, table=torch.randperm(12, generator=g, device="cuda").int().view(2, 6),
                lens=torch.tensor([90, 33], dtype=torch.int32, device="cuda"), new=torch.randn((2, 2, 2, 64), generator=g, device="cuda").to(dtype),
                weight=torch.rand((2, 100), generator=g, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["plain", "paged", "f32", "new", "weight", "scale", "scale_int", "given", "workspace", "numpy_scale", "view"])
def test_attention_calls(monkeypatch, form):
    paged = form == "paged"
    x = attention_inputs(paged, torch.float32 if form == "f32" else torch.bfloat16)

    def run():
        kv, w = x["kv"].clone(), x["weight"].clone()
        q = x["q"]
        if form == "view":
            q = torch.stack([q, q], 1)[:, 0]                 # not contiguous: refused step by step
        kw = {}
        if form in ("new", "paged"):
            kw.update(k_new=x["new"][0], v_new=x["new"][1])
        if form in ("weight", "paged"):
            kw.update(weight=w)
        if form == "scale":
            kw.update(scale=0.2, logit_cap=20.0)
        if form == "scale_int":
            kw.update(scale=1, logit_cap=20)
        if form == "numpy_scale":
            import numpy as np
            kw.update(scale=np.float32(0.125))
        if form == "given":
            kw.update(out=dict(out=torch.empty_like(q), lse=torch.empty((2, 8), device="cuda")))
        if form == "workspace":
            kw.update(workspace=torch.empty(1 << 20, dtype=torch.int32, device="cuda"))
        if paged:
            res = B.metok_decode_attention_paged(q, kv[0], kv[1], x["table"], x["lens"], **kw)
        else:
            res = B.metok_decode_attention(q, kv[0], kv[1], x["lens"], **kw)
        if form == "given":
            assert res["out"].data_ptr() == kw["out"]["out"].data_ptr()
        torch.cuda.synchronize()
        return dict(res, kv=kv, weight=w)

    if form == "view":
        with pytest.raises(ValueError, match="contiguous"):
            run()
        return
    check_same(*both(monkeypatch, run, [form != "numpy_scale"]))


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["dense", "paged", "select", "per_layer", "tuple", "given", "in_place", "some", "numpy_budget"])
def test_eviction_calls(monkeypatch, form):
    g = torch.Generator(device="cuda").manual_seed(4)
    L, shape = 3, ((12, 2, 16, 64) if form == "paged" else (2, 2, 96, 64))
    kv = torch.randn((L, 2) + shape, generator=g, device="cuda").to(torch.bfloat16)
    table = torch.randperm(12, generator=g, device="cuda").int().view(2, 6)
    weight = torch.rand((L, 2, 96), generator=g, device="cuda")
    lens = torch.tensor([[96, 40], [80, 96], [10, 70]], dtype=torch.int32, device="cuda")

    def run():
        x, w = kv.clone(), weight.clone()
        k, v, ws = [x[i, 0] for i in range(L)], [x[i, 1] for i in range(L)], [w[i] for i in range(L)]
        budget, kw = 50, {}
        if form == "per_layer":
            budget = [50, 60, 30]
        if form == "numpy_budget":
            import numpy as np
            budget = [int(b) for b in np.array([50, 60, 30])]
            kw.update(n_first=np.int64(2))
        if form == "tuple":
            k, v, ws = tuple(k), tuple(v), tuple(ws)
        if form == "some":
            ws[1] = None
        if form != "in_place":
            kw.update(weight_out=[torch.zeros_like(t) if t is not None else None for t in ws])
        if form == "given":
            kw.update(idx=[torch.empty((2, 50), dtype=torch.int32, device="cuda") for _ in range(L)], new_len=torch.empty_like(lens),
                      workspace=torch.empty(1 << 16, dtype=torch.uint8, device="cuda"))
        if form == "select":
            res = B.metok_kv_evict_select(ws, lens, 96, budget, 2, 10, **kw)
        elif form == "paged":
            res = B.metok_kv_evict_paged(k, v, table, ws, lens, budget, 2, 10, **kw)
        elif form == "numpy_budget":
            res = B.metok_kv_evict(k, v, ws, lens, budget, **kw)
        else:
            res = B.metok_kv_evict(k, v, ws, lens, budget, 2, 10, **kw)
        assert type(res["idx"]) is list and type(res["weight"]) is list
        if form == "given":
            assert res["new_len"] is kw["new_len"] and all(a is b for a, b in zip(res["idx"], kw["idx"]))
        torch.cuda.synchronize()
        return dict(idx=res["idx"], new_len=res["new_len"], weight=res["weight"], kv=x)

    check_same(*both(monkeypatch, run, [form != "numpy_budget"]))


def native_calls():
    x, p = attention_inputs(False), attention_inputs(True)
    kv = [t.contiguous() for t in x["kv"]]
    pool = [t.contiguous() for t in p["kv"]]
    lens = x["lens"][None].contiguous()
    H = B._host
    return {
        "decode_attention": lambda s: H.decode_attention(x["q"], kv[0], kv[1], None, x["lens"], None, None, None, 0.0, x["weight"], None, None, s),
        "decode_attention paged": lambda s: H.decode_attention(p["q"], pool[0], pool[1], p["table"], p["lens"], p["new"][0], p["new"][1], 0.1, 0.0, None, None, None, s),
        "kv_evict": lambda s: H.kv_evict([x["weight"]], lens, 32, 0, 0, None, None, None, kv[:1], kv[1:], None, None, s),
        "kv_evict paged": lambda s: H.kv_evict([x["weight"]], lens, 32, 0, 0, None, None, None, pool[:1], pool[1:], p["table"], None, s),
        "kv_evict_select": lambda s: H.kv_evict_select([x["weight"]], lens, 32, 0, 0, None, None, None, 96, s),
    }


NATIVE_CALLS = ["decode_attention", "decode_attention paged", "kv_evict", "kv_evict paged", "kv_evict_select"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", NATIVE_CALLS)
def test_nothing_that_can_fail_follows_the_launch(name):
    call, handles, late = native_calls()[name], [B._stream()], []

    def watch(phase, info):
        if not handles:
            late.append(phase)

    before = gc.get_threshold()
    gc.collect()
    gc.callbacks.append(watch)
    gc.set_threshold(1)
    try:
        res = call(lambda index: handles.pop())
        gc.disable()
    finally:
        gc.callbacks.remove(watch)
        gc.set_threshold(*before)
        gc.enable()
    torch.cuda.synchronize()
    assert res is not None and type(res) is dict and not handles and not late


@pytest.mark.gpu
@pytest.mark.parametrize("name", NATIVE_CALLS)
def test_errors_of_the_stream_function_are_raised(name):
    def interrupted(index):
        raise KeyboardInterrupt
    with pytest.raises(KeyboardInterrupt):
        native_calls()[name](interrupted)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NATIVE_CALLS)
def test_a_tensor_of_another_device_is_not_launched(name):
    """The stream function knows no stream for a device that is not the current one: the native call declines, and the step-by-step
    path says which tensor it is."""
    indices = []
    assert native_calls()[name](indices.append) is None
    assert indices == [torch.cuda.current_device()]


@pytest.mark.gpu
def test_the_current_device_is_checked(monkeypatch):
    x = attention_inputs(False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 5)
    with pytest.raises(ValueError, match="current device"):
        B.metok_decode_attention(x["q"], x["kv"][0], x["kv"][1], x["lens"])
    with pytest.raises(ValueError, match="current device"):
        B.metok_kv_evict([x["kv"][0]], [x["kv"][1]], [x["weight"]], x["lens"][None], 32)
    with pytest.raises(ValueError, match="current device"):
        B.metok_kv_evict_select([x["weight"]], x["lens"][None], 96, 32)
