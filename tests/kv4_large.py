"""Attention calls over 4 bits whose workers have several tiles: of one pair, of several pairs, of several videos."""
import random

import numpy as np

from oracle import qkv_oracle as Q
from tests import kv4_cases as K


class Cache(K.Cache4):
    """Cache4 that stores rows a few at a time and touches their bytes alone: for long caches and many videos."""

    def put(self, which, b, rows, x):
        ok, slab, at = self.there(b, rows)
        x, values = np.asarray(x)[ok], []
        codes_at, scales_at = Q.places(which, self.dh)
        for i in range(0, len(x), 1000):
            codes, e = Q.quantise(x[i:i + 1000])
            s, r = slab[i:i + 1000], at[i:i + 1000]
            for h in range(self.Hkv):
                self.data[which, s[:, None], h, (r // 16)[:, None], codes_at[r % 16]] = codes[:, h, 0::2] | (codes[:, h, 1::2] << 4)
                self.data[which, s[:, None], h, (r // 16)[:, None], scales_at[r % 16]] = e[:, h] + 127
            values.append(Q.values(codes, e))
        return np.concatenate(values) if values else np.zeros((0, self.Hkv, self.dh))


def _spread(n, least, most, seed):
    rng = random.Random(seed)
    return [rng.randint(least, most) for _ in range(n)]


# name: dtype, lens, Hq, Hkv, dh, capacity, and what differs from a dense cache, to which a row is appended, without weights and cap
CASES = {
    "long": ("bf16", [40011, 0, 30000], 12, 4, 128, 40032, {}),
    "long_paged_streamed_f32": ("f32", [30000, 29999, 5], 8, 4, 128, 82304, dict(page=16)),
    "long_paged_streamed_weights": ("bf16", [40011, 1], 16, 8, 128, 65536, dict(page=64, append=False, weights=True)),
    "long_weights_cap_f32": ("f32", [40000, 300], 8, 8, 64, 40016, dict(weights=True, cap=20.0)),
    "long_streamed_256": ("bf16", [26000, 12000, 40], 8, 8, 256, 26000, dict(append=False)),
    "long_paged_64": ("bf16", [30011, 1], 16, 8, 64, 30016, dict(page=32)),
    "long_f32": ("f32", [24000, 9000], 16, 8, 32, 24000, dict(append=False, cap=30.0)),
    "three_blocks_of_heads": ("bf16", [70000, 30000, 0], 40, 1, 64, 70016, {}),
    "short_pairs": ("bf16", _spread(2500, 0, 64, 1), 17, 1, 32, 64, dict(page=16)),
    "short_pairs_weights_f32": ("f32", _spread(1500, 0, 48, 2), 4, 2, 128, 48, dict(weights=True, append=False)),
    "ragged": ("bf16", _spread(200, 0, 1500, 3) + [2064, 2063, 0], 16, 2, 64, 2064, dict(page=48)),
    "ragged_streamed": ("bf16", _spread(100, 0, 300, 5) + _spread(30, 0, 2064, 6), 28, 4, 128, 2064, dict(append=False)),
}


def make(name):
    dtype, lens, Hq, Hkv, dh, capacity, kw = CASES[name]
    return K.make(dtype, lens, Hq, Hkv, dh, capacity, seed=len(lens) + dh, kind=Cache, **kw)
