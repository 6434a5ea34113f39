"""Plain CPU oracle of the operators around queries, keys and values, in 64 bits: norm and rotation by positions, rows in 4 bits and where a cache
in 4 bits keeps them.  Test infrastructure only.  (The attention over such a cache is decode_oracle's over the values that it stands for.)"""
from __future__ import annotations

import functools
import math

import numpy as np

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
HALVES, ADJACENT = 0, 1


def rotate_head(x, weight, eps, pos, inv_freq, pair_axis, pairs):
    """One head [dh] of a token at pos [axes]: normed (weight None: not), then its first 2 len(inv_freq) elements rotated pair by pair."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        mean = float(np.mean(x * x)) + eps
        x = x / math.sqrt(mean) * weight if mean > 0 else np.zeros_like(x)
    y = x.copy()
    half = len(inv_freq)
    for p in range(half):
        angle = float(pos[pair_axis[p]]) * float(inv_freq[p])
        i, j = (2 * p, 2 * p + 1) if pairs == ADJACENT else (p, p + half)
        y[i] = x[i] * math.cos(angle) - x[j] * math.sin(angle)
        y[j] = x[j] * math.cos(angle) + x[i] * math.sin(angle)
    return y


def rotate(x, weight, eps, pos, inv_freq, pair_axis, pairs):
    """rotate_head of x [n, heads, dh] at pos [axes, n], all heads of a token at once."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        mean = np.mean(x * x, axis=-1, keepdims=True) + eps
        x = np.where(mean > 0, x / np.sqrt(np.where(mean > 0, mean, 1.0)) * weight, 0.0)
    half = len(inv_freq)
    angle = np.asarray(pos, dtype=np.float64)[np.asarray(pair_axis, dtype=np.int64)].T * np.asarray(inv_freq, dtype=np.float64)          # [n, half]
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs == ADJACENT else (slice(0, half), slice(half, 2 * half))
    y = x.copy()
    y[..., i] = x[..., i] * cos - x[..., j] * sin
    y[..., j] = x[..., j] * cos + x[..., i] * sin
    return y


def scale_exponent(m):
    """e of the smallest power of two with m <= 7 * 2^e, within -100 .. 100."""
    e = -100
    while e < 100 and m > 7.0 * 2.0 ** e:
        e += 1
    return e


def quantise(rows):
    """rows [..., dh] -> (codes [..., dh], exponents [..., dh / 32]): of each element the nearest of the eight, ties to the even code, its sign in bit 3."""
    x = np.asarray(rows, dtype=np.float64)
    groups = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(groups).max(axis=-1)
    mant, e = np.frexp(top)                                # top = mant 2^e, 1/2 <= mant < 1: 7 is 0.875 * 2^3
    e = np.where(top == 0, -100, np.clip(np.where(mant > 0.875, e - 2, e - 3), -100, 100)).astype(np.int64)
    a = np.abs(groups) / np.exp2(e.astype(np.float64))[..., None]
    distance = np.abs(a[..., None] - np.asarray(GRID))
    code = distance.argmin(axis=-1)                        # the lower one of two as near
    tie = (code < 7) & (np.take_along_axis(distance, np.minimum(code + 1, 7)[..., None], -1)[..., 0] == np.take_along_axis(distance, code[..., None], -1)[..., 0])
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    return (code + 8 * np.signbit(groups)).reshape(x.shape), e


def values(codes, exponents):
    """What codes [..., dh] with exponents [..., dh / 32] stand for."""
    c = np.asarray(codes)
    v = np.where(c >= 8, -1.0, 1.0) * np.asarray(GRID)[c & 7]
    return (v.reshape(*c.shape[:-1], c.shape[-1] // 32, 32) * np.exp2(np.asarray(exponents, dtype=np.float64))[..., None]).reshape(c.shape)


def block_bytes(dh):
    return 17 * dh // 2


def code_byte(which, row, element, dh):
    """Byte of a block, and whether its high half, where the code of an element of K (0) or V (1) in one of its 16 rows is."""
    w = min(dh, 128)
    p, x = divmod(element, w)
    if which == 0:
        return p * 8 * w + row * w // 2 + x // 2, x % 2
    u, z = divmod(x, w // 16)
    c, i = divmod(row, 4)
    return p * 8 * w + c * 2 * w + u * w // 8 + i * w // 32 + z // 2, x % 2


def scale_place(row, group, dh):
    """Byte of a block that holds e + 127 of a group of 32 elements of a row (K and V alike)."""
    w = min(dh, 128)
    p, g = divmod(group, w // 32)
    c, i = divmod(row, 4)
    return 8 * dh + p * w // 2 + c * w // 8 + g * 4 + i


@functools.lru_cache(maxsize=None)
def places(which, dh):
    """code_byte of all even elements [16, dh / 2] (the odd ones are in the same bytes) and scale_place of all groups [16, dh / 32]."""
    codes = np.array([[code_byte(which, r, x, dh)[0] for x in range(0, dh, 2)] for r in range(16)])
    scales = np.array([[scale_place(r, g, dh) for g in range(dh // 32)] for r in range(16)])
    return codes, scales


def store(blocks, which, rows, codes, exponents):
    """Codes [n, dh] and exponents [n, dh / 32] into rows (an int array, each once) of blocks [.., 17 dh / 2] (uint8, changed)."""
    at, at_s = places(which, codes.shape[-1])
    rows = np.asarray(rows, dtype=np.int64)
    blocks[(rows // 16)[:, None], at[rows % 16]] = codes[:, 0::2] | (codes[:, 1::2] << 4)
    blocks[(rows // 16)[:, None], at_s[rows % 16]] = exponents + 127


def load(blocks, which, rows, dh):
    """The values of rows (an int array) of blocks [.., 17 dh / 2]: [len(rows), dh]"""
    at, at_s = places(which, dh)
    rows = np.asarray(rows, dtype=np.int64)
    byte = blocks[(rows // 16)[:, None], at[rows % 16]].astype(np.int64)
    codes = np.stack([byte & 15, byte >> 4], -1).reshape(len(rows), dh)
    return values(codes, blocks[(rows // 16)[:, None], at_s[rows % 16]].astype(np.int64) - 127)
