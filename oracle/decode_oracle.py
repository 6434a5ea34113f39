"""CPU oracle for the decoding-time operators: the definitions of metok_decode.h in numpy float64, one video and one head at a time.

TEST INFRASTRUCTURE, NOT PRODUCT CODE: shares no code with the HIP library.
"""
from __future__ import annotations

import math
from typing import List, Optional, Sequence, Tuple

import numpy as np

F64 = np.float64


def attend(q, keys, values, scale: float, cap: float = 0.0) -> Tuple[np.ndarray, float, np.ndarray]:
    """One query head [dh] over the rows keys / values [n, dh]: (output [dh], log of the sum, probabilities [n])."""
    q, keys, values = (np.asarray(x, dtype=F64) for x in (q, keys, values))
    n = keys.shape[0]
    if n == 0:
        return np.zeros(q.shape[0]), -math.inf, np.zeros(0)
    s = np.array([scale * float(np.dot(q, k)) for k in keys]) if n <= 64 else scale * (keys @ q)
    if cap > 0.0:
        s = cap * np.tanh(s / cap)
    top = float(s.max())
    e = np.exp(s - top)
    total = float(e.sum())
    p = e / total
    return p @ values, top + math.log(total), p


def decode_attention(q, keys: Sequence, values: Sequence, scale: float, cap: float = 0.0):
    """q [B, Hq, dh]; keys[b], values[b] [n_b, Hkv, dh], the appended row included.
    Returns out [B, Hq, dh], lse [B, Hq] and, per video, the mean over the heads of every row's probability."""
    q = np.asarray(q, dtype=F64)
    B, Hq, dh = q.shape
    out, lse, mean = np.zeros((B, Hq, dh)), np.zeros((B, Hq)), []
    for b in range(B):
        n, Hkv, _ = np.asarray(keys[b]).shape
        total = np.zeros(n)
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            out[b, h], lse[b, h], p = attend(q[b, h], keys[b][:, kv], values[b][:, kv], scale, cap)
            total += p
        mean.append(total / Hq)
    return out, lse, mean


def evict(weight, n: int, budget: int, n_first: int, n_last: int) -> List[int]:
    """The rows that one (layer, video) of n rows keeps, ascending: all of them within the budget, else the first n_first, the last
    n_last and the heaviest between, the lower index first among equals."""
    if n <= budget:
        return list(range(n))
    w = [float(x) for x in np.asarray(weight).reshape(-1)[:n]]
    middle = sorted(range(n_first, n - n_last), key=lambda j: (-w[j], j))[:budget - n_first - n_last]
    return list(range(n_first)) + sorted(middle) + list(range(n - n_last, n))


def index_list(kept: Sequence[int], budget: int) -> np.ndarray:
    """The list of one video as stage 3 takes it: a video that keeps fewer rows than the budget stays as it is."""
    return np.asarray(list(kept) + list(range(len(kept), budget)), dtype=np.int32)
