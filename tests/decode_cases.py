"""Inputs, 64-bit results and tolerances of the decoding-time operators, for their GPU tests."""
import numpy as np
import torch

from oracle import decode_oracle as D

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}       # half a step of a type, relative to the value
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def typed(x, dtype):
    """float32 array -> (device tensor of dtype, its values in float64)"""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(TORCH[dtype])
    return t.cuda(), t.to(torch.float64).numpy()


def make(dtype, lens, Hq, Hkv, dh, capacity, page=0, append=True, weights=False, cap=0.0, spread=2.0, seed=0, poison=float("nan")):
    """The inputs of one call on the device, and what they are in float64.  Rows behind a video's last one and pages of nobody hold
    `poison`."""
    rng = np.random.default_rng(seed)
    B = len(lens)
    q, q64 = typed(spread * rng.standard_normal((B, Hq, dh)), dtype)
    kn, kn64 = typed(rng.standard_normal((B, Hkv, dh)), dtype)
    vn, vn64 = typed(rng.standard_normal((B, Hkv, dh)), dtype)
    held = [min(max(n, 0), capacity) for n in lens]
    rows = [[typed(rng.standard_normal((n, Hkv, dh)), dtype) for n in held] for _ in range(2)]
    if page == 0:
        shape, table = (B, Hkv, capacity, dh), None
    else:
        assert capacity % page == 0
        per_seq = capacity // page
        table = rng.permutation(B * per_seq + 3)[:B * per_seq].reshape(B, per_seq).astype(np.int32)
        shape = (B * per_seq + 3, Hkv, page, dh)
    caches = []
    for which in range(2):
        c = torch.full(shape, poison, dtype=TORCH[dtype], device="cuda")
        for b, n in enumerate(held):
            if n == 0:
                continue
            x = rows[which][b][0]
            if page == 0:
                c[b, :, :n] = x.transpose(0, 1)
            else:
                j = torch.arange(n, device="cuda")
                c[torch.from_numpy(table[b]).cuda().long()[j // page], :, j % page] = x
        caches.append(c)
    weight = torch.rand((B, capacity + 3), generator=torch.Generator().manual_seed(seed)).cuda() if weights else None
    return dict(dtype=dtype, lens=list(lens), held=held, Hq=Hq, Hkv=Hkv, dh=dh, capacity=capacity, page=page, append=append, cap=cap,
                q=q, q64=q64, k_new=kn if append else None, v_new=vn if append else None, kn64=kn64, vn64=vn64, k=caches[0], v=caches[1],
                rows64=[[rows[w][b][1] for b in range(B)] for w in range(2)], table=table, weight=weight,
                lens_dev=torch.tensor(lens, dtype=torch.int32, device="cuda"), table_dev=None if table is None else torch.from_numpy(table).cuda())


def call(B, c, **kw):
    args = dict(k_new=c["k_new"], v_new=c["v_new"], logit_cap=c["cap"], weight=c["weight"])
    args.update(kw)
    if c["page"]:
        return B.metok_decode_attention_paged(c["q"], c["k"], c["v"], c["table_dev"], c["lens_dev"], **args)
    return B.metok_decode_attention(c["q"], c["k"], c["v"], c["lens_dev"], **args)


def attended(c):
    """Per video, the rows that the call attends to, in float64: K and V [n, Hkv, dh]."""
    out = []
    for w, new in ((0, c["kn64"]), (1, c["vn64"])):
        out.append([np.concatenate([x, new[b][None]]) if c["append"] else x for b, x in enumerate(c["rows64"][w])])
    return out


def tolerances(c, keys, values, scale):
    """What rounding can do to the results, worst case.  With u = 2^-24 (half a step of fp32):
    a logit is a dot product of dh products summed in fp32 in some order, error <= dh u sum |q k|, times scale and log2 e in one rounded
    factor (2 u |s|) and, capped, a tanh of 4 u and two more factors (<= 8 u |cap|, its argument's error passes at most whole); the
    difference to the maximum is rounded once (u (|s| + |max|)) and exp2 of it is 2 u off.  Both p and the sum carry that: p is off
    by at most 2 d + the summation error of the sum, relatively, d being the largest of these.  The weighted sum has at most
    rows / 16 + 64 additions in sequence, products of bf16 values with a probability in two bf16 parts (error 2^-16 of it, 0 in fp32)."""
    u = 2.0 ** -24
    B, Hq, dh = c["q64"].shape
    out_tol, lse_tol, p_tol = np.zeros((B, Hq, dh)), np.zeros((B, Hq)), []
    for b in range(B):
        n = keys[b].shape[0]
        rel = 0.0
        chain = (n / 16 + 64) * u
        for h in range(Hq):
            kv = h // (Hq // c["Hkv"])
            if n == 0:
                continue
            K, V = keys[b][:, kv], values[b][:, kv]
            s = scale * (K @ c["q64"][b, h])
            dot = scale * (np.abs(K) @ np.abs(c["q64"][b, h]))
            if c["cap"] > 0:
                s = c["cap"] * np.tanh(s / c["cap"])
            top = np.abs(s).max()
            # a row far below the maximum has no share in anything: its error counts with its probability
            d = dh * u * dot.max() + 2 * u * top + (8 * u * c["cap"] if c["cap"] > 0 else 0) + 2 * u * top + 2 * u
            _, lse, p = D.attend(c["q64"][b, h], K, V, scale, c["cap"])
            magnitude = p @ np.abs(V)
            out_tol[b, h] = magnitude * (2 * d + 3 * chain + (2.0 ** -16 if c["dtype"] == "bf16" else 0))
            lse_tol[b, h] = d + chain + 4 * u * (abs(lse) + 1)
            rel = max(rel, 2 * d + 2 * chain + 4 * u)
        p_tol.append(rel)
    return out_tol, lse_tol, p_tol


def check(c, res, weight_before=None, scale=None):
    scale = c["dh"] ** -0.5 if scale is None else scale
    keys, values = attended(c)
    out, lse, mean = D.decode_attention(c["q64"], keys, values, scale, c["cap"])
    out_tol, lse_tol, p_tol = tolerances(c, keys, values, scale)
    got = res["out"].to(torch.float64).cpu().numpy()
    err = np.abs(got - out)
    limit = out_tol + HALF[c["dtype"]] * (np.abs(out) + out_tol) + 2.0 ** -133
    assert (err <= limit).all(), f"out: {int((err > limit).sum())} beyond the bound, worst {np.nanmax(err / np.maximum(limit, 1e-300)):.3g} of it"
    got = res["lse"].to(torch.float64).cpu().numpy()
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(got), empty)
    err = np.abs(got[~empty] - lse[~empty])
    assert (err <= lse_tol[~empty] + 2.0 ** -24 * np.abs(lse[~empty])).all(), f"lse: worst {np.max(err / lse_tol[~empty]):.3g} of the bound"
    if c["weight"] is not None:
        got, before = c["weight"].to(torch.float64).cpu().numpy(), weight_before.to(torch.float64).cpu().numpy()
        for b, n in enumerate(c["held"]):
            p = mean[b]
            placed = min(len(p), c["capacity"])
            want = p[:placed] + np.where(np.arange(placed) < n, before[b, :placed], 0.0)
            limit = p[:placed] * p_tol[b] + 2.0 ** -24 * want + 2.0 ** -126
            err = np.abs(got[b, :placed] - want)
            assert (err <= limit).all(), f"weights of video {b}: worst {np.max(err / limit):.3g} of the bound"
            assert np.array_equal(got[b, placed:], before[b, placed:]), "weights behind the last row were written"


def same(a, b):
    """Bit for bit, NaNs included."""
    kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def check_caches(c, before):
    """The appended rows are there, everything else is as it was."""
    for name, new in (("k", c["k_new"]), ("v", c["v_new"])):
        want = before[name].clone()
        if c["append"]:
            for b, n in enumerate(c["held"]):
                if n < c["capacity"]:
                    if c["page"]:
                        want[int(c["table"][b, n // c["page"]]), :, n % c["page"]] = new[b]
                    else:
                        want[b, :, n] = new[b]
        assert same(c[name], want), f"the {name} cache is not what it was with the new rows"
