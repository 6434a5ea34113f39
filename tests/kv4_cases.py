"""Inputs, 64-bit results and tolerances of the operators around queries, keys and values, for their GPU tests."""
import numpy as np
import torch

from oracle import decode_oracle as D
from oracle import qkv_oracle as Q
from tests.decode_cases import HALF, TORCH, same, typed

U = 2.0 ** -24                                             # half a step of fp32


class Cache4:
    """A 4-bit cache on the host: K and V [slabs, Hkv, blocks, 17 dh / 2], what no row was stored into being random bytes (scaled: with scales that are ones)."""

    def __init__(self, B, Hkv, capacity, dh, page=0, seed=0, scaled=False):
        self.B, self.Hkv, self.capacity, self.dh, self.page = B, Hkv, capacity, dh, page
        rng = np.random.default_rng(1000 + seed)
        rows, slabs, self.table = capacity, B, None
        if page:
            per_seq, rows = capacity // page, page
            slabs = B * per_seq + 3                        # pages of nobody
            self.table = rng.permutation(slabs)[:B * per_seq].reshape(B, per_seq).astype(np.int32)
        self.data = rng.integers(0, 256, (2, slabs, Hkv, rows // 16, Q.block_bytes(dh)), dtype=np.uint8)
        if scaled:
            self.data[..., 8 * dh:] = rng.integers(27, 228, (2, slabs, Hkv, rows // 16, dh // 2), dtype=np.uint8)

    def there(self, b, rows):
        """Which of a video's rows have a page, and these rows' slabs and places in them."""
        rows = np.asarray(rows, dtype=np.int64)
        if not self.page:
            return np.ones(len(rows), dtype=bool), np.full(len(rows), b), rows
        slab = self.table[b, rows // self.page].astype(np.int64)
        ok = (slab >= 0) & (slab < self.data.shape[1])
        return ok, slab[ok], (rows % self.page)[ok]

    def put(self, which, b, rows, x):
        """x [n, Hkv, dh] into rows, where they have a page; what of it is stored then, as values"""
        ok, slab, at = self.there(b, rows)
        codes, e = Q.quantise(np.asarray(x)[ok])
        for h in range(self.Hkv):
            blocks = self.data[which, :, h].reshape(-1, self.data.shape[-1])         # a copy: heads are no outer dimension
            Q.store(blocks, which, slab * (self.data.shape[3] * 16) + at, codes[:, h].astype(np.uint8), e[:, h])
            self.data[which, :, h] = blocks.reshape(self.data[which, :, h].shape)
        return Q.values(codes, e)

    def get(self, which, b, row):
        """A row's values [Hkv, dh], None where it has no page"""
        ok, slab, at = self.there(b, [row])
        return np.stack([Q.load(self.data[which, slab[0], h], which, at, self.dh)[0] for h in range(self.Hkv)]) if ok[0] else None

    def device(self):
        t = torch.from_numpy(self.data.copy()).cuda()
        return t[0], t[1], None if self.table is None else torch.from_numpy(self.table.copy()).cuda()


def make(dtype, lens, Hq, Hkv, dh, capacity, page=0, append=True, weights=False, cap=0.0, spread=2.0, seed=0, broken=(), kind=Cache4):
    """The inputs of one attention over 4 bits, on the device, and what they are in float64.  broken: (video, page index, entry) of the table that are no
    pages of the pool."""
    rng = np.random.default_rng(seed)
    B = len(lens)
    q, q64 = typed(spread * rng.standard_normal((B, Hq, dh)), dtype)
    kn, kn64 = typed(rng.standard_normal((B, Hkv, dh)), dtype)
    vn, vn64 = typed(rng.standard_normal((B, Hkv, dh)), dtype)
    cache = kind(B, Hkv, capacity, dh, page, seed)
    for b, p, entry in broken:
        cache.table[b, p] = entry
    held, rows = [min(max(n, 0), capacity) for n in lens], [[], []]
    for which in range(2):
        for b, n in enumerate(held):
            x = rng.standard_normal((n, Hkv, dh)) * np.exp2(rng.integers(-2, 3, (1, Hkv, 1)))
            rows[which].append(cache.put(which, b, np.arange(n), x))
    weight = torch.rand((B, capacity + 3), generator=torch.Generator().manual_seed(seed)).cuda() if weights else None
    k, v, table = cache.device()
    return dict(dtype=dtype, lens=list(lens), held=held, Hq=Hq, Hkv=Hkv, dh=dh, capacity=capacity, page=page, append=append, cap=cap, q=q, q64=q64,
                k_new=kn if append else None, v_new=vn if append else None, new64=(kn64, vn64), rows64=rows, cache=cache, k=k, v=v, table=table,
                weight=weight, lens_dev=torch.tensor(lens, dtype=torch.int32, device="cuda"))


def call(B, c, **kw):
    args = dict(k_new=c["k_new"], v_new=c["v_new"], logit_cap=c["cap"], weight=c["weight"])
    args.update(kw)
    if c["page"]:
        return B.metok_kv4_attention_paged(c["q"], c["k"], c["v"], c["table"], c["lens_dev"], **args)
    return B.metok_kv4_attention(c["q"], c["k"], c["v"], c["lens_dev"], **args)


def attended(c):
    """Per video, the rows that the call attends to, in float64: K and V [n, Hkv, dh]; the new one as what 4 bits leave of it."""
    out = []
    for which in range(2):
        new = Q.values(*Q.quantise(c["new64"][which]))
        out.append([np.concatenate([x, new[b][None]]) if c["append"] else x for b, x in enumerate(c["rows64"][which])])
    return out


def tolerances(c, keys, values, scale):
    """What rounding can do to the results, worst case; the terms are those of decode_cases.tolerances with what is different here: the values of the cache
    are exact, and so is every product with a part of a query (one in bf16, three of 8 bits in fp32, which hold all 24 bits), so a logit is a sum of
    parts * dh products in fp32, off by at most parts dh u sum |q k|.  A probability is two bf16 numbers in bf16 (2^-16 of it) and three in fp32
    (u of it); 32 rows go into a product, so parts rows / 32 additions follow each other, and 64 more within the products and the join.
    Numbers below 2^-126 are 0 to exp2 and to the products: a probability that small beside the largest (which is 1) is dropped with its value, and so may be the
    second and third parts of a larger one, below 2^-126 each: at most 3 * 2^-126 < 2^-124 of every row's value, which shows where
    all larger rows have the value 0, as values of 4 bits have."""
    B, Hq, dh = c["q64"].shape
    qp, pp = (1, 2) if c["dtype"] == "bf16" else (3, 3)
    out_tol, lse_tol, p_tol = np.zeros((B, Hq, dh)), np.zeros((B, Hq)), []
    for b in range(B):
        n, rel = keys[b].shape[0], 0.0
        chain = (pp * n / 32 + 64) * U
        for h in range(Hq if n else 0):
            kv = h // (Hq // c["Hkv"])
            K, V = keys[b][:, kv], values[b][:, kv]
            s, dot = scale * (K @ c["q64"][b, h]), scale * (np.abs(K) @ np.abs(c["q64"][b, h]))
            if c["cap"] > 0:
                s = c["cap"] * np.tanh(s / c["cap"])
            d = qp * dh * U * dot.max() + 4 * U * np.abs(s).max() + (8 * U * c["cap"] if c["cap"] > 0 else 0) + 2 * U
            _, lse, p = D.attend(c["q64"][b, h], K, V, scale, c["cap"])
            out_tol[b, h] = p @ np.abs(V) * (2 * d + 3 * chain + (2.0 ** -16 if c["dtype"] == "bf16" else U)) + 2.0 ** -124 * np.abs(V).sum(0)
            lse_tol[b, h] = d + chain + 4 * U * (abs(lse) + 1)
            rel = max(rel, 2 * d + 2 * chain + 4 * U)
        p_tol.append(rel)
    return out_tol, lse_tol, p_tol


def check(c, res, weight_before=None, scale=None):
    scale = c["dh"] ** -0.5 if scale is None else scale
    keys, values = attended(c)
    out, lse, mean = D.decode_attention(c["q64"], keys, values, scale, c["cap"])
    out_tol, lse_tol, p_tol = tolerances(c, keys, values, scale)
    err = np.abs(res["out"].to(torch.float64).cpu().numpy() - out)
    limit = out_tol + HALF[c["dtype"]] * (np.abs(out) + out_tol) + 2.0 ** -133
    assert (err <= limit).all(), f"out: {int((~(err <= limit)).sum())} beyond the bound, worst {np.nanmax(err / np.maximum(limit, 1e-300)):.3g} of it"
    got, empty = res["lse"].to(torch.float64).cpu().numpy(), np.isneginf(lse)
    assert np.array_equal(np.isneginf(got), empty)
    err = np.abs(got[~empty] - lse[~empty])
    assert (err <= lse_tol[~empty] + U * np.abs(lse[~empty])).all(), f"lse: worst {np.max(err / lse_tol[~empty]):.3g} of the bound"
    if c["weight"] is not None:
        got, before = c["weight"].to(torch.float64).cpu().numpy(), weight_before.to(torch.float64).cpu().numpy()
        for b, n in enumerate(c["held"]):
            p = mean[b]
            placed = min(len(p), c["capacity"])
            want = p[:placed] + np.where(np.arange(placed) < n, before[b, :placed], 0.0)
            err = np.abs(got[b, :placed] - want)
            assert (err <= p[:placed] * p_tol[b] + U * want + 2.0 ** -126).all(), f"weights of video {b}"
            assert np.array_equal(got[b, placed:], before[b, placed:]), "weights behind the last row were written"


def check_cache(c):
    """The appended rows are there, bit for bit, everything else is as it was."""
    if c["append"]:
        for which in range(2):
            for b, n in enumerate(c["held"]):
                if n < c["capacity"]:
                    c["cache"].put(which, b, [n], c["new64"][which][b][None])
    for which, t in ((0, c["k"]), (1, c["v"])):
        assert np.array_equal(t.cpu().numpy(), c["cache"].data[which]), f"{'KV'[which]} is not what it was with the new rows"


def rotate_tolerance(x, weight, eps, want, dtype, dh, half, pairs):
    """Worst case of the roundings of a normed and rotated head.  The mean of the squares is off by at most (dh + 2) u of itself, its root by half of that and a
    unit, 1 / root and the two products by 3 u: (dh / 2 + 6) u of every element.  An angle, taken as a fraction of a revolution r (|r| <= 1/2, its rounding
    to fp32 2^-26, times 2 pi < 2^-23.3), gives a cosine and a sine off by that and by 4 u of their own, together < 2^-21.5; the two products and the sum
    3 u of |x| + |y|.  The result is rounded once more."""
    e = 2.0 ** -21.5 + 3 * U + ((dh / 2 + 6) * U if weight is not None else 0.0)
    x = np.abs(np.asarray(x, dtype=np.float64))
    if weight is not None:
        mean = np.mean(x * x, axis=-1, keepdims=True) + eps
        x = np.where(mean > 0, x / np.sqrt(np.where(mean > 0, mean, 1.0)), 0.0) * np.abs(weight)
    size = x.copy()
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs == Q.ADJACENT else (slice(0, half), slice(half, 2 * half))
    size[..., i] = size[..., j] = x[..., i] + x[..., j]
    return size * e * (1 + HALF[dtype]) + HALF[dtype] * np.abs(want) + 2.0 ** -133


__all__ = ["Cache4", "make", "call", "attended", "tolerances", "check", "check_cache", "rotate_tolerance", "typed", "same", "HALF", "TORCH", "U"]
