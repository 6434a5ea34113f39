"""The native marshalling of the calls around queries, keys and values against the step-by-step path: the same outputs bit for bit, and what is not of the
ordinary form is declined before anything happens."""
import pytest
import torch

from tests.test_native_binding import both
from tests.test_native_decode_binding import check_same

B = pytest.importorskip("paper_2506_02850_amd.binding")


def test_calls_off_the_gpu_are_declined():
    rows, kv, pos, freq = torch.zeros(1, 1, 2, 64), torch.zeros(1, 2, 16, 64), torch.zeros(1, 1, 1, dtype=torch.int32), torch.zeros(32)
    four, lens, q, asked = torch.zeros(1, 2, 1, 544, dtype=torch.uint8), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, 64), []
    assert B._host.rotate_qk(rows, rows, rows, pos, freq, kv, kv, None, None, None, None, None, None, 1e-6, 0, None, asked.append) is None
    assert B._host.kv4_pack(kv, kv, four, four, None, None, None, None, asked.append) is None
    assert B._host.kv4_unpack(four, four, None, lens, 16, None, None, None, asked.append) is None
    assert B._host.kv4_attention(q, four, four, None, lens, None, None, None, 0.0, None, None, None, asked.append) is None
    assert not asked
    for name in ("rotate_qk", "kv4_pack", "kv4_unpack", "kv4_attention"):
        with pytest.raises(TypeError):
            getattr(B._host, name)(rows)
    for call in (lambda: B.metok_rotate_qk(rows, rows, rows, pos, freq, kv, kv), lambda: B.metok_kv4_pack(kv, kv, four, four),
                 lambda: B.metok_kv4_unpack(four, four, lens, 16), lambda: B.metok_kv4_attention(q, four, four, lens)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call in (B.metok_rotate_qk_paged, B.metok_kv4_pack_paged, B.metok_kv4_unpack_paged, B.metok_kv4_attention_paged):
        args = {B.metok_rotate_qk_paged: (rows, rows, rows, pos, freq, kv, kv), B.metok_kv4_pack_paged: (kv, kv, four, four)}.get(call, (four, four))
        with pytest.raises((ValueError, TypeError), match="page_table|missing"):
            call(*args, None, *([lens, 4] if call is B.metok_kv4_unpack_paged else [lens] if call is B.metok_kv4_attention_paged else []))


def cuda(*shape, g, dtype=torch.bfloat16):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["plain", "paged", "f32", "norm", "one_token", "given", "two_dim_pos", "list_axis", "numpy_eps", "wrong_heads", "gap"])
def test_rotation_calls(monkeypatch, form):
    g = torch.Generator(device="cuda").manual_seed(1)
    dtype, n = torch.float32 if form == "f32" else torch.bfloat16, 1 if form == "one_token" else 5
    qkv = cuda(2, n, 10, 64, g=g, dtype=dtype)
    pos, freq = ints([[[7 * b + i + a for i in range(n)] for b in range(2)] for a in range(2)]), torch.rand(32, generator=g, device="cuda")
    weights = cuda(2, 64, g=g, dtype=dtype)

    def run():
        kv = torch.zeros((2, 8, 2, 16, 64) if form == "paged" else (2, 2, 2, 16, 64), dtype=dtype, device="cuda")
        kw = dict(start=ints([1, 3]), count=ints([n, n - 1]), out={"q": torch.zeros((2, 6, n, 64), dtype=dtype, device="cuda")})
        if form in ("paged", "norm"):
            kw.update(q_weight=weights[0], k_weight=weights[1], eps=1e-5, pair_axis=bytes([0, 1] * 16), pairs=B.PAIRS_ADJACENT)
        if form == "list_axis":
            kw.update(pair_axis=[0, 1] * 16)
        if form == "numpy_eps":
            import numpy as np
            kw.update(eps=np.float64(1e-5))
        if form == "given":
            kw.update(start=None, count=None)
        v = qkv[:, :, 8:9] if form == "wrong_heads" else qkv[:, :, 8:]
        q = torch.stack([qkv, qkv], 2)[:, :, 0, :6, :] if form != "gap" else torch.stack([qkv, qkv], 3)[:, :, :6, 0]
        args = (q, qkv[:, :, 6:8], v, pos[0] if form == "two_dim_pos" else pos, freq, kv[0], kv[1])
        res = B.metok_rotate_qk_paged(*args, ints([[3, 0], [6, 1]]), **kw) if form == "paged" else B.metok_rotate_qk(*args, **kw)
        assert res["q"].data_ptr() == kw["out"]["q"].data_ptr()
        torch.cuda.synchronize()
        return dict(res, kv=kv)

    if form in ("wrong_heads", "gap"):
        with pytest.raises(ValueError, match="heads"):
            run()
        return
    check_same(*both(monkeypatch, run, [form not in ("list_axis", "numpy_eps")]))


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["plain", "paged", "f32", "listed", "fresh", "more_rows", "wrong_dh"])
def test_row_calls(monkeypatch, form):
    g = torch.Generator(device="cuda").manual_seed(2)
    dtype = torch.float32 if form == "f32" else torch.bfloat16
    kv = cuda(2, 2, 2, 40, 64, g=g, dtype=dtype)

    def run():
        four = [t.zero_() for t in (B.metok_kv4_cache(9, 2, 16, 64, "cuda") if form == "paged" else B.metok_kv4_cache(2, 2, 48, 64, "cuda"))]
        if form == "wrong_dh":
            four = [t.zero_() for t in B.metok_kv4_cache(2, 2, 48, 128, "cuda")]
        table = (ints([[5, 0, 8], [2, 7, 1]]),) if form == "paged" else ()
        pack, unpack = (B.metok_kv4_pack_paged, B.metok_kv4_unpack_paged) if form == "paged" else (B.metok_kv4_pack, B.metok_kv4_unpack)
        pack(kv[0], kv[1], *four, *table, start=ints([0, 7]), count=ints([40, 11]), idx=ints([[3, 9, 1, 1], [39, 0, -1, 40]]) if form == "listed" else None)
        kw = {}
        if form != "fresh":
            rows = 50 if form == "more_rows" else 41
            kw.update(out={x: torch.full((2, 2, rows, 64), 3.0, dtype=dtype, device="cuda") for x in "kv"})
        if form == "listed":
            kw.update(idx=ints([[i % 3 for i in range(41)], list(range(41))]))
        elif form != "plain":
            kw.update(first=ints([0, 7]))
        res = unpack(*four, *table, ints([40, 18]), 41, **kw)
        torch.cuda.synchronize()
        if form == "fresh":                                  # rows that are not there hold anything
            return dict(four=four, k=res["k"][0, :, :40], v=res["v"][1, :, :11])
        return dict(res, four=four)

    if form == "wrong_dh":
        with pytest.raises(ValueError, match="4-bit"):
            run()
        return
    check_same(*both(monkeypatch, run, [True, form != "fresh"]))


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["plain", "paged", "f32", "new", "weight", "given", "workspace", "numpy_scale", "wrong_type"])
def test_attention_calls(monkeypatch, form):
    g = torch.Generator(device="cuda").manual_seed(3)
    dtype = torch.float32 if form == "f32" else torch.bfloat16
    rows, q, new, weight = cuda(2, 2, 2, 96, 64, g=g), cuda(2, 8, 64, g=g, dtype=dtype), cuda(2, 2, 2, 64, g=g, dtype=dtype), torch.rand((2, 100), generator=g, device="cuda")
    table, lens = torch.randperm(12, generator=g, device="cuda").int().view(2, 6), ints([90, 33])

    def run():
        four, w, kw = [t.zero_() for t in (B.metok_kv4_cache(12, 2, 16, 64, "cuda") if form == "paged" else B.metok_kv4_cache(2, 2, 96, 64, "cuda"))], weight.clone(), {}
        if form == "paged":
            B.metok_kv4_pack_paged(rows[0], rows[1], *four, table)
        else:
            B.metok_kv4_pack(rows[0], rows[1], *four)
        if form in ("new", "paged"):
            kw.update(k_new=new[0], v_new=new[1])
        if form in ("weight", "paged"):
            kw.update(weight=w, scale=0.2, logit_cap=20)
        if form == "numpy_scale":
            import numpy as np
            kw.update(scale=np.float32(0.125))
        if form == "given":
            kw.update(out=dict(out=torch.empty_like(q), lse=torch.empty((2, 8), device="cuda")))
        if form == "workspace":
            kw.update(workspace=torch.empty(1 << 20, dtype=torch.int32, device="cuda"))
        if form == "wrong_type":
            four = [t.view(torch.int8) for t in four]
        res = B.metok_kv4_attention_paged(q, *four, table, lens, **kw) if form == "paged" else B.metok_kv4_attention(q, *four, lens, **kw)
        torch.cuda.synchronize()
        return dict(res, four=four, weight=w)

    if form == "wrong_type":
        with pytest.raises(ValueError, match="uint8"):
            run()
        return
    check_same(*both(monkeypatch, run, [True, form != "numpy_scale"]))


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("call", ["rotate", "pack", "unpack", "attention"])
def test_tables_without_pages_are_refused(monkeypatch, call, native):
    """A table of no columns is a table: the call is refused, also where the pool has as many pages as there are videos, and nothing is written."""
    if not native:
        monkeypatch.setattr(B, "_host", type("Declines", (), {"__getattr__": lambda self, name: lambda *a: None})())
    g = torch.Generator(device="cuda").manual_seed(4)
    lens, pos, freq = ints([3, 2]), ints([[[0, 1], [2, 3]]]), torch.rand(32, generator=g, device="cuda")
    for table in (torch.zeros((2, 0), dtype=torch.int32, device="cuda"), ints([[1, 0], [0, 1]])[:, :0]):
        if call == "rotate":
            qkv, pool, out = cuda(2, 2, 6, 64, g=g), cuda(2, 2, 2, 16, 64, g=g), {"q": cuda(2, 2, 2, 64, g=g)}
            args, kw = (B.metok_rotate_qk_paged, qkv[:, :, :2], qkv[:, :, 2:4], qkv[:, :, 4:], pos, freq, pool[0], pool[1], table), dict(out=out)
        else:
            pool, out = torch.randint(100, 140, (2, 2, 2, 1, 544), generator=g, device="cuda", dtype=torch.uint8), {x: cuda(2, 2, 2, 64, g=g) for x in "kv"}
            rows = cuda(2, 2, 2, 2, 64, g=g)
            args, kw = {"pack": ((B.metok_kv4_pack_paged, rows[0], rows[1], pool[0], pool[1], table), {}),
                        "unpack": ((B.metok_kv4_unpack_paged, pool[0], pool[1], table, lens, 2), dict(out=out)),
                        "attention": ((B.metok_kv4_attention_paged, rows[0, :, :, 0], pool[0], pool[1], table, lens), dict(k_new=rows[1, :, :, 0].contiguous(),
                                                                                                                     v_new=rows[1, :, :, 1].contiguous()))}[call]
            args = tuple(x.contiguous() if isinstance(x, torch.Tensor) and x is not table else x for x in args)
        before = [t.clone() for t in (pool, *out.values())]
        with pytest.raises(B.MetokError, match="page_table|capacity|pages_per_seq"):
            args[0](*args[1:], **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(before, (pool, *out.values())))
