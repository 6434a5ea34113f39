"""The operators around queries, keys and values of this repository as cases for measurement, with a plain form of each.

  rotate  metok_rotate_qk / metok_rotate_qk_paged: queries and keys of new tokens are normed for each head and rotated by positions of
          one to four axes (time, height, width), the queries laid out head by head, keys and values put into the dense or paged cache
  pack    metok_kv4_pack / metok_kv4_pack_paged, then metok_kv4_unpack / metok_kv4_unpack_paged: rows of K and V go into a cache held in 4 bits and
          come back as the values they now stand for
  attend  metok_kv4_attention / metok_kv4_attention_paged: attention of one new token per video over that cache, with the token's own
          row appended (its values come back by an unpack of that row) and the attention weight of every row accumulated

The cache in 4 bits: 32 neighbouring elements of a row share a scale s = 2^e, the smallest one with max |x| <= 7 s (-100 <= e <= 100); an
element is the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times s, with its sign, ties to the even code.  Rows lie in blocks of 16, 8.5 dh bytes each:
first the codes, two a byte, then the scales, e + 127 in a byte each.  With w = min(dh, 128), piece p = 0 .. dh / w - 1, row = 4 c + i:
  codes of K   [p][row][w / 2];   codes of V  [p][c][16][i][w / 32]: 16 runs of w / 16 elements, the four rows of a c beside each other
  scales       [p][c][w / 32][i]

A case is one call with its inputs resident on the GPU.  `own` says which side `run` takes: the library's calls, or elementary
torch operations in 32 bits (angles in 64).
"""
import math
import random

import torch

own = False
DEV = "cuda"


# ---------------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------------
def _rotate(**kw):
    c = dict(kind="rotate", dtype="bf16", batch=1, tokens=1, fewest=1, Hq=28, Hkv=4, dh=128, rot=128, axes=3, rounds=False, adjacent=False, norm=True,
             cap_rows=4096, held=0, page=0)
    c.update(kw)
    return c


def _pack(**kw):
    c = dict(kind="pack", dtype="bf16", batch=1, Hkv=4, dh=128, source_rows=4096, rows=4096, fewest=4096, listed=False, cap_rows=4096, held=0, page=0)
    c.update(kw)
    return c


def _attend(**kw):
    c = dict(kind="attend", dtype="bf16", batch=1, Hq=28, Hkv=4, dh=128, cap_rows=4096, shortest=4000, longest=4000, page=0,
             append=True, weights=False, logit_cap=0.0)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest call: one token of a small float32 decoder with ordinary positions, where launch and host are everything
        _rotate(name="rotate_token_f32", dtype="f32", Hq=8, Hkv=2, dh=32, rot=32, axes=1, norm=False, cap_rows=128, held=60),
        # a step of 64 requests: normed heads, positions of three axes, rows appended to pages of 16
        _rotate(name="rotate_64_tokens_paged", batch=64, cap_rows=512, held=300, page=16),
        # the prompt of a LongVA-shaped video pooled to 12 x 12 tokens a frame, with 128 text tokens, into an empty cache
        _rotate(name="rotate_prompt_18560", tokens=18560, fewest=18560, cap_rows=18560),
        # ragged prompts in float32, a quarter of each head rotated by adjacent pairs
        _rotate(name="rotate_4_ragged_f32", dtype="f32", batch=4, tokens=4571, fewest=1200, Hq=14, Hkv=2, dh=64, rot=16, axes=1, adjacent=True, norm=False,
                cap_rows=4608, held=33),
        # stage 3 with a cache in 4 bits as its end: the kept half of a long video's rows
        _pack(name="pack_half_of_18560", source_rows=18560, rows=9333, fewest=9333, listed=True, cap_rows=9344),
        # chunks of a batch's prompts in float32, appended behind rows that are there, in pages of 32
        _pack(name="pack_8_chunks_paged_f32", dtype="f32", batch=8, Hkv=2, dh=64, source_rows=1000, rows=1000, fewest=1, cap_rows=2048, held=777, page=32),
        # the smallest attention: a short cache of one request, float32 queries, small heads
        _attend(name="attend_tiny_f32", dtype="f32", Hq=8, Hkv=2, dh=32, cap_rows=128, shortest=60, longest=60, append=False),
        # one request of a LLaVA-OneVision service after adaptive pooling of 32 frames: latency of a decoding step, its row stored
        _attend(name="attend_1x2307", cap_rows=2560, shortest=2306, longest=2306),
        # continuous batching: 32 requests of very different lengths over pages of 16 rows
        _attend(name="attend_32_ragged_paged", batch=32, Hq=32, Hkv=8, cap_rows=8192, shortest=1, longest=8191, page=16),
        # one uncompressed long video whose rows are ranked while the answer is written
        _attend(name="attend_1x131072_weights", cap_rows=131072, shortest=131071, longest=131071, page=64, append=False, weights=True),
        # wide heads, capped scores, pages of 64 rows
        _attend(name="attend_8x3000_dh256_cap", batch=8, Hq=8, Hkv=2, dh=256, cap_rows=4096, shortest=700, longest=3000, page=64, append=False, logit_cap=30.0),
        # throughput: eight LongVA-shaped videos of 36864 visual tokens and 128 text tokens
        _attend(name="attend_8x36992", batch=8, cap_rows=36992, shortest=36992, longest=36992, append=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _whole(rows, unit):
    return -(-rows // unit) * unit


HEADS = ((28, 4, 128), (28, 4, 128), (40, 40, 128), (14, 2, 64), (32, 8, 128), (16, 16, 64), (8, 2, 256), (4, 4, 32), (71, 1, 64), (8, 1, 128))


def _draw_any(rng):
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    Hq, Hkv, dh = rng.choice(HEADS)
    if dh == 256:
        dtype = "bf16"
    kind = rng.random()
    if kind < 0.3:
        tokens, batch = rng.choice((1, _log(rng, 1, 20000), _log(rng, 1, 20000))), _log(rng, 1, 64)
        page, held = rng.choice((0, 0, 16, 64, 7, 1)), rng.choice((0, _log(rng, 1, 3000)))
        axes = rng.choice((1, 2, 3, 3, 4))
        return _rotate(dtype=dtype, batch=batch, tokens=tokens, fewest=rng.choice((tokens, rng.randint(0, tokens))), Hq=Hq, Hkv=Hkv, dh=dh,
                       rot=rng.choice((dh, dh, 16 * rng.randint(1, dh // 16))), axes=axes, rounds=rng.random() < 0.5, adjacent=rng.random() < 0.3,
                       norm=rng.random() < 0.6, cap_rows=_whole(held + tokens + rng.choice((0, 5)), page or 1), held=held, page=page)
    page = rng.choice((0, 0, 16, 16, 64, 128, 48))
    if kind < 0.5:
        source, held = _log(rng, 1, 40000), rng.choice((0, 0, _log(rng, 1, 3000)))
        picked = rng.random() < 0.5
        rows = rng.randint(1, source) if picked else source
        return _pack(dtype=dtype, batch=rng.choice((1, 1, 2, 4, 8)), Hkv=Hkv, dh=dh, source_rows=source, rows=rows,
                     fewest=rng.choice((rows, rng.randint(0, rows))), listed=picked, cap_rows=_whole(held + rows, page or 16), held=held, page=page)
    longest = _log(rng, 1, 40000)
    shortest = rng.choice((longest, max(1, longest // 2), rng.randint(0, longest), min(longest, 1)))
    rows = longest + 1 + rng.choice((0, 0, rng.randint(0, 200), longest))
    return _attend(dtype=dtype, batch=_log(rng, 1, 64), Hq=Hq, Hkv=Hkv, dh=dh, cap_rows=_whole(rows, page or 16), shortest=shortest, longest=longest, page=page,
                   append=rng.random() < 0.5, weights=rng.random() < 0.3, logit_cap=rng.choice((0.0, 0.0, 0.0, 30.0, 50.0)))


def draw(rng):
    most = max(_cost(c) for c in listed())
    memory = max(_memory(c) for c in listed())
    while True:
        c = _draw_any(rng)
        if _cost(c) <= most and _memory(c) <= memory:
            return c


def _cost(c):
    """A rough time of one pass, for the bound on drawn cases only."""
    w = work(c)
    return w["bytes"] / 5e12 + w["flops"] / 5e13 + _memory(c) / 5e13


def _memory(c):
    rows = c["batch"] * c["Hkv"] * c["dh"]
    if c["kind"] == "rotate":
        return rows * 2 * c["cap_rows"] * _esize(c) + 2 * c["batch"] * c["tokens"] * (c["Hq"] + 2 * c["Hkv"]) * c["dh"] * _esize(c)
    if c["kind"] == "pack":
        return rows * 2 * (c["source_rows"] + c["rows"]) * _esize(c) + rows * c["cap_rows"]
    return rows * c["cap_rows"] * 2        # of the plain form's indices and values there are many times as much


# ---------------------------------------------------------------------------------------------------------------------
# what one pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def _esize(c):
    return 2 if c["dtype"] == "bf16" else 4


def _between(c, lo, hi):
    """Sizes of the batch's members; they belong to the case, so that its work does not depend on the seed."""
    r = random.Random(hi * 131 + c["batch"])
    return [hi] + [int(round(math.exp(r.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1 for _ in range(c["batch"] - 1)]


def _held(c):
    """Rows that the caches hold before a rotate or pack."""
    return [max(0, c["held"] - 5 * b) for b in range(c["batch"])]


def work(case):
    c, e = case, _esize(case)
    Hkv, dh = c["Hkv"], c["dh"]
    if c["kind"] == "rotate":
        n = sum(_between(c, c["fewest"], c["tokens"]))
        heads = c["Hq"] + Hkv
        norm = 4 * heads * dh if c["norm"] else 0
        return {"bytes": n * (2 * (heads + Hkv) * dh * e + 4 * c["axes"]), "flops": n * (3 * heads * c["rot"] + norm)}
    row4 = Hkv * dh * 17 // 16                             # K and V of one row of a layer, 17 bits for two pairs of elements
    if c["kind"] == "pack":
        n = sum(_between(c, c["fewest"], c["rows"]))
        return {"bytes": n * (4 * Hkv * dh * e + 2 * row4 + (4 if c["listed"] else 0)), "flops": n * 6 * Hkv * dh}
    lens = _between(c, c["shortest"], c["longest"])
    rows = sum(lens) + (c["batch"] if c["append"] else 0)
    ends = c["batch"] * (c["Hq"] * (2 * dh * e + 4) + (row4 + 4 * Hkv * dh * e if c["append"] else 0))      # q, out, lse; the new row in, stored, and out
    return {"bytes": rows * row4 + ends + (8 * rows if c["weights"] else 0), "flops": 4 * rows * c["Hq"] * dh}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _torch_dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _pages(c, g):
    """(slabs of the cache, rows of a slab, page table or None)"""
    if c["page"] == 0:
        return c["batch"], c["cap_rows"], None
    per_seq, spare = c["cap_rows"] // c["page"], 3         # pages of the pool that belong to no sequence
    n = c["batch"] * per_seq
    return n + spare, c["page"], torch.randperm(n + spare, generator=g, device=DEV)[:n].int().view(c["batch"], per_seq).contiguous()


def _axis_of(c):
    """Axis of every pair: runs (a quarter of the pairs for the first axis, the others alike), or one pair of each in turn."""
    half, axes = c["rot"] // 2, c["axes"]
    if axes == 1 or c["rounds"]:
        return [i % axes for i in range(half)]
    first = max(1, half // 4)
    return [0 if i < first else 1 + (i - first) * (axes - 1) // (half - first) for i in range(half)]


def _prepare_rotate(c, seed):
    g, dt = torch.Generator(device=DEV).manual_seed(seed), _torch_dtype(c)
    Bn, n, Hq, Hkv, dh = c["batch"], c["tokens"], c["Hq"], c["Hkv"], c["dh"]
    # what one product leaves: queries, keys and values of a token beside each other
    qkv = torch.empty((Bn, n, Hq + 2 * Hkv, dh), dtype=dt, device=DEV).normal_(generator=g)
    slabs, rows, table = _pages(c, g)
    kv = torch.zeros((2, slabs, Hkv, rows, dh), dtype=dt, device=DEV)
    at = torch.arange(n, device=DEV)
    first = torch.randint(0, 100000, (Bn, 1), generator=g, device=DEV)        # videos of any age: far positions among them
    axes = [first + at // 144, first // 7 + at // 12 % 12, first // 11 + at % 12, first + at][:c["axes"]]
    held = _held(c)
    freq = torch.tensor([1e6 ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)], device=DEV)
    weights = 1.0 + 0.2 * torch.randn((2, dh), generator=g, device=DEV)
    return dict(case=c, q=qkv[:, :, :Hq], k=qkv[:, :, Hq:Hq + Hkv], v=qkv[:, :, Hq + Hkv:], pos=torch.stack(axes).int().contiguous(), freq=freq,
                axis=bytes(_axis_of(c)), axis_dev=torch.tensor(_axis_of(c), device=DEV), q_weight=weights[0].to(dt), k_weight=weights[1].to(dt),
                kv=kv, table=table, start=_i32(held), count=_i32(_between(c, c["fewest"], n)), q_out=torch.zeros((Bn, Hq, n, dh), dtype=dt, device=DEV))


def _blocks(c, slabs, rows):
    return torch.zeros((2, slabs, c["Hkv"], rows // 16, 17 * c["dh"] // 2), dtype=torch.uint8, device=DEV)


def _prepare_pack(c, seed):
    g, dt = torch.Generator(device=DEV).manual_seed(seed), _torch_dtype(c)
    Bn, Hkv, dh, n = c["batch"], c["Hkv"], c["dh"], c["rows"]
    kv = torch.empty((2, Bn, Hkv, c["source_rows"], dh), dtype=torch.float32, device=DEV).normal_(generator=g)
    kv *= torch.exp(0.7 * torch.randn((2, 1, Hkv, 1, dh), generator=g, device=DEV))       # some channels are larger than others, as keys have them
    kv = kv.to(dt)
    slabs, rows, table = _pages(c, g)
    idx = None
    if c["listed"]:
        idx = torch.stack([torch.randperm(c["source_rows"], generator=g, device=DEV)[:n].sort().values for _ in range(Bn)]).int()
    count, held = _between(c, c["fewest"], n), _held(c)
    return dict(case=c, kv=kv, k=kv[0], v=kv[1], idx=idx, cache=_blocks(c, slabs, rows), table=table, start=_i32(held), count=_i32(count),
                lens=_i32([x + y for x, y in zip(count, held)]), out=torch.zeros((2, Bn, Hkv, n, dh), dtype=dt, device=DEV))


def _prepare_attend(c, seed):
    g, dt = torch.Generator(device=DEV).manual_seed(seed), _torch_dtype(c)
    Bn, Hq, Hkv, dh = c["batch"], c["Hq"], c["Hkv"], c["dh"]
    slabs, rows, table = _pages(c, g)
    cache = _blocks(c, slabs, rows)
    for which in range(2):
        x = torch.empty((slabs, Hkv, rows, dh), dtype=torch.float32, device=DEV).normal_(generator=g)
        codes, scales = _quantise(x)
        at = torch.arange(rows, device=DEV)
        slab = torch.arange(slabs, device=DEV)
        _store(cache[which], which, slab[:, None].expand(slabs, rows), at[None].expand(slabs, rows), codes, scales)
    # logits of a standard deviation of two, as trained heads have them: a few rows draw most of the weight
    q = (2.0 * torch.randn((Bn, Hq, dh), generator=g, device=DEV)).to(dt)
    new = torch.randn((2, Bn, Hkv, dh), generator=g, device=DEV).to(dt)
    weight = torch.rand((Bn, c["cap_rows"]), generator=g, device=DEV) * (16.0 / c["cap_rows"])     # of some steps before
    lens = _i32(_between(c, c["shortest"], c["longest"]))
    return dict(case=c, q=q, cache=cache, k=cache[0], v=cache[1], table=table, new=new, k_new=new[0], v_new=new[1], weight=weight, lens=lens, lens_after=lens + 1,
                out=torch.zeros_like(q), lse=torch.zeros((Bn, Hq), device=DEV), row=torch.zeros((2, Bn, Hkv, 1, dh), dtype=dt, device=DEV))


def prepare(case, seed):
    return {"rotate": _prepare_rotate, "pack": _prepare_pack, "attend": _prepare_attend}[case["kind"]](case, seed)


# ---------------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    c = state["case"]
    if own:
        return {"rotate": _rotate_own, "pack": _pack_own, "attend": _attend_own}[c["kind"]](c, state)
    return {"rotate": _rotate_plain, "pack": _pack_plain, "attend": _attend_plain}[c["kind"]](c, state)


def _rotate_own(c, s):
    from paper_2506_02850_amd import binding as B

    kw = dict(start=s["start"], count=s["count"], pair_axis=s["axis"], pairs=B.PAIRS_ADJACENT if c["adjacent"] else B.PAIRS_HALVES, out={"q": s["q_out"]})
    if c["norm"]:
        kw.update(q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6)
    if c["page"]:
        B.metok_rotate_qk_paged(s["q"], s["k"], s["v"], s["pos"], s["freq"], s["kv"][0], s["kv"][1], s["table"], **kw)
    else:
        B.metok_rotate_qk(s["q"], s["k"], s["v"], s["pos"], s["freq"], s["kv"][0], s["kv"][1], **kw)
    return {"q": s["q_out"], "kv": s["kv"]}


def _pack_own(c, s):
    from paper_2506_02850_amd import binding as B

    k4, v4, out = s["cache"][0], s["cache"][1], {"k": s["out"][0], "v": s["out"][1]}
    if c["page"]:
        B.metok_kv4_pack_paged(s["k"], s["v"], k4, v4, s["table"], start=s["start"], count=s["count"], idx=s["idx"])
        B.metok_kv4_unpack_paged(k4, v4, s["table"], s["lens"], c["rows"], first=s["start"], out=out)
    else:
        B.metok_kv4_pack(s["k"], s["v"], k4, v4, start=s["start"], count=s["count"], idx=s["idx"])
        B.metok_kv4_unpack(k4, v4, s["lens"], c["rows"], first=s["start"], out=out)
    return {"kv": s["out"]}


def _attend_own(c, s):
    from paper_2506_02850_amd import binding as B

    if "workspace" not in s:
        code = B.BF16 if c["dtype"] == "bf16" else B.F32
        need = B.metok_kv4_attention_workspace_bytes(c["batch"], c["Hq"], c["Hkv"], c["cap_rows"], c["dh"], code, c["weights"])
        s["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
        s["into"] = dict(out=s["out"], lse=s["lse"])
    kw = dict(logit_cap=c["logit_cap"], workspace=s["workspace"], out=s["into"])
    if c["append"]:
        kw.update(k_new=s["k_new"], v_new=s["v_new"])
    if c["weights"]:
        kw.update(weight=s["weight"])
    if c["page"]:
        B.metok_kv4_attention_paged(s["q"], s["k"], s["v"], s["table"], s["lens"], **kw)
    else:
        B.metok_kv4_attention(s["q"], s["k"], s["v"], s["lens"], **kw)
    res = {"out": s["out"], "lse": s["lse"]}
    if c["weights"]:
        res["weight"] = s["weight"]
    if c["append"]:                                        # all that the call wrote into the cache, as the values it stands for
        out = {"k": s["row"][0], "v": s["row"][1]}
        if c["page"]:
            B.metok_kv4_unpack_paged(s["k"], s["v"], s["table"], s["lens_after"], 1, first=s["lens"], out=out)
        else:
            B.metok_kv4_unpack(s["k"], s["v"], s["lens_after"], 1, first=s["lens"], out=out)
        res["row"] = s["row"]
    return res


# ---- the same in elementary operations ----
def _place(c, s, row):
    """Where logical rows [B, n] are in the cache: (slab, row of the slab), [B, n] each."""
    if c["page"] == 0:
        return torch.arange(c["batch"], device=DEV)[:, None].expand_as(row), row
    return torch.gather(s["table"].long(), 1, row // c["page"]), row % c["page"]


def _rotate_plain(c, s):
    Bn, n, Hq, Hkv, dh, rot = c["batch"], c["tokens"], c["Hq"], c["Hkv"], c["dh"], c["rot"]
    angle = s["pos"].double()[s["axis_dev"]].permute(1, 2, 0) * s["freq"].double()           # [B, n, rot / 2]
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]

    def turned(x, weight):
        y = x.float()
        if c["norm"]:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * weight.float()
        z = y.clone()
        if c["adjacent"]:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            z[..., 0:rot:2], z[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
        else:
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            z[..., :rot // 2], z[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
        return z.to(x.dtype)

    there = torch.arange(n, device=DEV)[None] < s["count"].long()[:, None]
    q = turned(s["q"], s["q_weight"]).transpose(1, 2)
    s["q_out"].copy_(torch.where(there[:, None, :, None], q, s["q_out"]))
    slab, row = _place(c, s, s["start"].long()[:, None] + torch.arange(n, device=DEV)[None])
    for which, x in ((0, turned(s["k"], s["k_weight"])), (1, s["v"])):
        s["kv"][which][slab, :, row] = torch.where(there[:, :, None, None], x, s["kv"][which][slab, :, row])
    return {"q": s["q_out"], "kv": s["kv"]}


def _offsets(dh, which):
    """Byte offsets in a block: of the codes [16, dh / 2] of K (0) or V (1), and of the scales [16, dh / 32]."""
    w = min(dh, 128)
    P, G = dh // w, w // 32
    codes, scales = torch.arange(8 * dh, device=DEV), 8 * dh + torch.arange(dh // 2, device=DEV)
    if which == 0:
        codes = codes.view(P, 16, w // 2).permute(1, 0, 2)
    else:
        codes = codes.view(P, 4, 16, 4, G).permute(1, 3, 0, 2, 4)
    return codes.reshape(16, dh // 2), scales.view(P, 4, G, 4).permute(1, 3, 0, 2).reshape(16, dh // 32)


def _quantise(x):
    """[..., dh] float32 -> codes of 4 bits [..., dh], scale bytes [..., dh / 32]"""
    y = x.unflatten(-1, (-1, 32))
    mant, e = torch.frexp(y.abs().amax(-1, keepdim=True))                    # max = mant 2^e, 1/2 <= mant < 1
    e = torch.where(mant > 0.875, e - 2, e - 3).clamp(-100, 100)
    e = torch.where(mant == 0, -100, e)
    a = torch.ldexp(y.abs(), -e)
    codes = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    return (codes + 8 * torch.signbit(y)).flatten(-2), (e + 127).squeeze(-1)


def _base(c, cache, slab, row):
    """First byte of the blocks that rows are in, for every kv head: [B, Hkv, n]"""
    heads = torch.arange(c["Hkv"], device=DEV)[None, :, None]
    return ((slab[:, None] * c["Hkv"] + heads) * cache.shape[-2] + row[:, None] // 16) * cache.shape[-1]


def _store(cache, which, slab, row, codes, scales, there=None):
    """codes [B, Hkv, n, dh] and scales into the rows (slab, row) [B, n] of a cache, where `there`"""
    dh = codes.shape[-1]
    off, off_s = _offsets(dh, which)
    base = _base(dict(Hkv=codes.shape[1]), cache, slab, row)[..., None]
    at, at_s = base + off[row % 16][:, None], base + off_s[row % 16][:, None]
    packed = (codes[..., ::2] + 16 * codes[..., 1::2]).to(torch.uint8)
    scales = scales.to(torch.uint8)
    flat = cache.view(-1)
    if there is not None:                                  # the others are written back as they were
        pick = there[:, None, :, None]
        packed, scales = torch.where(pick, packed, flat[at]), torch.where(pick, scales, flat[at_s])
    flat[at] = packed
    flat[at_s] = scales


def _values(c, cache, which, slab, row):
    """The rows (slab, row) [B, n] of a cache as values, [B, Hkv, n, dh] float32"""
    off, off_s = _offsets(c["dh"], which)
    base = _base(c, cache, slab, row)[..., None]
    flat = cache.view(-1)
    code = torch.arange(16, device=DEV)
    low = (code % 8).float()
    grid = torch.where(low < 4, low / 2, torch.where(low < 6, low - 2, 2 * low - 8)) * (1 - 2 * (code // 8))
    byte = torch.arange(256, device=DEV)
    pair = torch.stack([grid[byte % 16], grid[byte // 16]], -1)
    x = pair[flat[base + off[row % 16][:, None]].int()].flatten(-2)
    scale = torch.exp2(flat[base + off_s[row % 16][:, None]].float() - 127.0)
    return (x.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2)


def _pack_plain(c, s):
    Bn, n = c["batch"], c["rows"]
    at = torch.arange(n, device=DEV)[None].expand(Bn, n)
    there = at < s["count"].long()[:, None]
    slab, row = _place(c, s, s["start"].long()[:, None] + at)
    for which in range(2):
        x = s["kv"][which]
        if c["listed"]:
            x = torch.gather(x, 2, s["idx"].long()[:, None, :, None].expand(Bn, c["Hkv"], n, c["dh"]))
        codes, scales = _quantise(x[:, :, :n].float())
        _store(s["cache"][which], which, slab, row, codes, scales, there)
        back = _values(c, s["cache"][which], which, slab, row).to(x.dtype)
        s["out"][which].copy_(torch.where(there[:, None, :, None], back, s["out"][which]))
    return {"kv": s["out"]}


def _attend_plain(c, s):
    Bn, Hq, Hkv, dh = c["batch"], c["Hq"], c["Hkv"], c["dh"]
    lens = s["lens"].long()
    res = {}
    if c["append"]:                                        # the new row goes behind the last one
        slab, row = _place(c, s, lens[:, None])
        for which in range(2):
            codes, scales = _quantise(s["new"][which].float()[:, :, None])
            _store(s["cache"][which], which, slab, row, codes, scales)
            s["row"][which].copy_(_values(c, s["cache"][which], which, slab, row).to(s["row"].dtype))
        res["row"] = s["row"]
        lens = lens + 1
    R = c["longest"] + (1 if c["append"] else 0)
    slab, row = _place(c, s, torch.arange(R, device=DEV)[None].expand(Bn, R))
    k, v = _values(c, s["k"], 0, slab, row), _values(c, s["v"], 1, slab, row)
    q = s["q"].float().view(Bn, Hkv, Hq // Hkv, dh)
    logits = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(dh)
    if c["logit_cap"]:
        logits = c["logit_cap"] * torch.tanh(logits / c["logit_cap"])
    seen = torch.arange(R, device=DEV)[None] < lens[:, None]
    logits = logits.masked_fill(~seen[:, None, None], -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-3e38)   # a video without rows has no maximum
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    p = p / total.clamp(min=1e-38)
    res["out"] = torch.matmul(p, v).view(Bn, Hq, dh).to(s["q"].dtype)
    res["lse"] = (top + torch.log(total)).view(Bn, Hq)
    if c["weights"]:
        old = s["weight"][:, :R]
        grown = p.sum((1, 2)) / Hq
        if c["append"]:
            old = old.masked_fill(torch.arange(R, device=DEV)[None] == lens[:, None] - 1, 0.0)
        s["weight"][:, :R] = torch.where(seen, old + grown, s["weight"][:, :R])
        res["weight"] = s["weight"]
    return res


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _nearest(x):
    """What rows [..., dh] stand for in 4 bits, from the definition: the scale by its logarithm's neighbours, the value by its distance to each
    of the eight."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    y = x.double().reshape(-1, 32)
    m = y.abs().amax(1)
    e = torch.floor(torch.log2(m.clamp(min=1e-40) / 7.0)).clamp(-100, 100) - 1
    for _ in range(3):
        e = torch.where((m > 7.0 * torch.exp2(e)) & (e < 100), e + 1, e)
    e = e.clamp(-100, 100)
    a = (y.abs() / torch.exp2(e)[:, None]).clamp(max=6.0)
    best, value = torch.full_like(a, math.inf), torch.zeros_like(a)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):                  # even codes first: they keep a tie
        d = (a - grid[code]).abs()
        value, best = torch.where(d < best, grid[code], value), torch.minimum(d, best)
    return torch.copysign(value * torch.exp2(e)[:, None], y).reshape(x.shape)


def _read(c, s, which, b, n):
    """Rows 0 .. n - 1 of video b as values [Hkv, n, dh] in float64, block by block as the layout is written down"""
    cache, dh, Hkv = s["cache"][which], c["dh"], c["Hkv"]
    if c["page"]:
        blocks = cache[s["table"][b].long()].transpose(0, 1).reshape(Hkv, -1, cache.shape[-1])
    else:
        blocks = cache[b]
    blocks = blocks[:, :-(-n // 16)]
    nb, w = blocks.shape[1], min(dh, 128)
    P, G = dh // w, w // 32
    code, scale = blocks[..., :8 * dh], blocks[..., 8 * dh:]
    code = torch.stack([code & 15, code >> 4], -1).reshape(Hkv, nb, 16 * dh)
    if which == 0:
        code = code.view(Hkv, nb, P, 16, w).transpose(2, 3)
    else:
        code = code.view(Hkv, nb, P, 4, 16, 4, w // 16).permute(0, 1, 3, 5, 2, 4, 6)
    code = code.reshape(Hkv, nb * 16, dh // 32, 32)
    scale = scale.view(Hkv, nb, P, 4, G, 4).permute(0, 1, 3, 5, 2, 4).reshape(Hkv, nb * 16, dh // 32, 1)
    low = (code & 7).double()
    value = torch.where(low < 4, low / 2, torch.where(low < 6, low - 2, 2 * low - 8))
    value = torch.where(code >= 8, -value, value) * torch.exp2(scale.double() - 127)
    return value.reshape(Hkv, nb * 16, dh)[:, :n]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    return {"rotate": _rotate_exact, "pack": _pack_exact, "attend": _attend_exact}[c["kind"]](c, s)


def _rotate_exact(c, s):
    q_out, kv, rot = s["q_out"].double(), s["kv"].double(), c["rot"]
    axis = torch.tensor(_axis_of(c), device=DEV)
    for b, (n, at) in enumerate(zip(_between(c, c["fewest"], c["tokens"]), _held(c))):
        angle = s["pos"][:, b, :n].double()[axis].T * s["freq"].double()     # [n, rot / 2]

        def turned(x, weight):
            y = x.double()
            if c["norm"]:
                y = y * torch.rsqrt(y.square().sum(-1, keepdim=True) / c["dh"] + 1e-6) * weight.double()
            first = torch.arange(0, rot, 2, device=DEV) if c["adjacent"] else torch.arange(rot // 2, device=DEV)
            second = first + (1 if c["adjacent"] else rot // 2)
            turn = torch.eye(c["dh"], dtype=torch.float64, device=DEV).repeat(n, 1, 1)         # [n, dh, dh]: the token's rotation as a matrix
            turn[:, first, first], turn[:, second, second] = torch.cos(angle), torch.cos(angle)
            turn[:, second, first], turn[:, first, second] = torch.sin(angle), -torch.sin(angle)
            return torch.matmul(y, turn.transpose(1, 2).contiguous())

        q_out[b, :, :n] = turned(s["q"][b, :n], s["q_weight"]).transpose(0, 1)
        rows = torch.arange(at, at + n, device=DEV)
        for which, x in ((0, turned(s["k"][b, :n], s["k_weight"])), (1, s["v"][b, :n].double())):
            if c["page"]:
                kv[which][s["table"][b].long()[rows // c["page"]], :, rows % c["page"]] = x
            else:
                kv[which, b, :, rows] = x.transpose(0, 1)
    return {"q": q_out, "kv": kv}


def _pack_exact(c, s):
    out = s["out"].double()
    for b, n in enumerate(_between(c, c["fewest"], c["rows"])):
        for which in range(2):
            x = s["kv"][which, b]
            out[which, b, :, :n] = _nearest(x[:, s["idx"][b, :n].long()] if c["listed"] else x[:, :n])
    return {"kv": out}


def _attend_exact(c, s):
    group, root = c["Hq"] // c["Hkv"], math.sqrt(c["dh"])
    outs, lses, weights = [], [], []
    new = _nearest(s["new"])
    for b, n in enumerate(_between(c, c["shortest"], c["longest"])):
        keys, vals = _read(c, s, 0, b, n), _read(c, s, 1, b, n)
        if c["append"]:
            keys, vals = torch.cat([keys, new[0, b][:, None]], 1), torch.cat([vals, new[1, b][:, None]], 1)
        total = torch.zeros(keys.shape[1], dtype=torch.float64, device=DEV)
        heads, norms = [], []
        for h in range(c["Hq"]):
            x = (keys[h // group] * s["q"][b, h].double()).sum(1) / root
            if c["logit_cap"]:
                x = c["logit_cap"] * torch.tanh(x / c["logit_cap"])
            p = torch.softmax(x, 0)
            total += p
            heads.append((p[:, None] * vals[h // group]).sum(0))
            norms.append(torch.logsumexp(x, 0))
        outs.append(torch.stack(heads))
        lses.append(torch.stack(norms))
        w = s["weight"][b].double()
        w[:total.numel()] += total / c["Hq"]
        if c["append"]:
            w[n] = total[n] / c["Hq"]
        weights.append(w)
    res = {"out": torch.stack(outs), "lse": torch.stack(lses)}
    if c["weights"]:
        res["weight"] = torch.stack(weights)
    if c["append"]:
        res["row"] = new[:, :, :, None]
    return res
