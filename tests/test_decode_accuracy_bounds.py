"""CPU checks of decode_accuracy.py: plain fp32 arithmetic is within its bounds, arithmetic with fewer bits is not."""
import numpy as np
import pytest

from tests import decode_accuracy as A

F = np.float32


def inputs(dtype, dh, n, seed, B=4, Hq=8, Hkv=2):
    rng = np.random.default_rng(seed)
    kind = A.bf16 if dtype == "bf16" else lambda x: np.asarray(x, dtype=F).astype(np.float64)
    q = kind(2 * rng.standard_normal((B, Hq, dh)))
    return q, [kind(rng.standard_normal((n, Hkv, dh))) for _ in range(B)], [kind(rng.standard_normal((n, Hkv, dh))) for _ in range(B)]


def emulate(dtype, q, keys, values, scale, cut_qk=0, cut_v=0, p_bits=0, log_norm=False):
    """The arithmetic of the kernels in fp32, sums by numpy; with mistakes planted."""
    B, Hq, dh = q.shape
    out, lse, weights = np.zeros((B, Hq, dh)), np.zeros((B, Hq)), []
    c = F(scale * 1.4426950408889634)
    for b in range(B):
        total = np.zeros(len(keys[b]), dtype=F)
        for h in range(Hq):
            kv = h // (Hq // keys[b].shape[1])
            K, V, x = keys[b][:, kv], values[b][:, kv], q[b, h]
            if cut_qk:
                K, x = A.cut(K, cut_qk), A.cut(x, cut_qk)
            if cut_v:
                V = A.cut(V, cut_v)
            s = np.zeros(len(K), dtype=F)
            for i in range(dh):                          # one addition after the other
                s = s + K[:, i].astype(F) * F(x[i])
            top = s.max()
            p = np.exp2((s - top) * c)
            l = p.sum(dtype=F)
            if log_norm:
                p, l = np.exp2(s * c - F(top * c + np.log2(l))), F(1)
            in_product = p if dtype == "f32" else A.bf16(p) + A.bf16(p - A.bf16(p).astype(F))
            if p_bits:
                in_product = A.cut(p, p_bits)
            o = (in_product.astype(F)[:, None] * V.astype(F)).sum(0, dtype=F) / l
            out[b, h] = o if dtype == "f32" else A.bf16(o)
            lse[b, h] = F(top * c + np.log2(l)) * F(np.log(2.0)) if not log_norm else np.nan
            total += p / l
        weights.append((total / F(Hq)).astype(np.float64))
    return out, lse, weights


def said(dtype, dh, n, seed=0, **mistake):
    q, k, v = inputs(dtype, dh, n, seed)
    return A.faults(dtype, emulate(dtype, q, k, v, dh ** -0.5, **mistake), q, k, v, dh ** -0.5)


@pytest.mark.parametrize("n", [300, 2500])
@pytest.mark.parametrize("dtype,dh", [("f32", 32), ("f32", 128), ("bf16", 32), ("bf16", 128), ("bf16", 256)])
def test_fp32_arithmetic_is_within_the_bounds(dtype, dh, n):
    assert said(dtype, dh, n) == []


@pytest.mark.parametrize("n", [300, 2500])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_sixteen_bits_are_not_enough_for_fp32(dh, n):
    assert [x[:3] for x in said("f32", dh, n, cut_qk=16)] == ["out", "lse", "wei"]
    assert [x[:3] for x in said("f32", dh, n, p_bits=15)] == ["out"]
    assert [x[:3] for x in said("f32", dh, n, cut_v=15)] == ["out"]


@pytest.mark.parametrize("n", [300, 2500])
@pytest.mark.parametrize("dh", [32, 128, 256])
def test_one_bf16_number_is_not_enough_for_a_probability(dh, n):
    assert [x[:3] for x in said("bf16", dh, n, p_bits=8)] == ["out"]


def test_rounding_to_bf16():
    import torch
    x = np.random.default_rng(0).standard_normal(5000).astype(F) * np.exp2(np.random.default_rng(1).integers(-60, 60, 5000)).astype(F)
    np.testing.assert_array_equal(A.bf16(x), torch.from_numpy(x).to(torch.bfloat16).double().numpy())
    np.testing.assert_array_equal(A.cut(x.astype(np.float64), 8), A.bf16(x))


@pytest.mark.parametrize("n", [40, 2500])
def test_equal_values_show_a_sum_taken_through_its_logarithm(n):
    """Scores around 200: the result of values that are all 1 is within 32 u of 1 divided by the sum, and not through the rounded logarithm."""
    q, k, v = inputs("f32", 64, n, 3)
    q[..., 0] = 16.0
    for b in range(len(k)):
        k[b][..., 0], v[b][...] = 100.0, 1.0
    far = [np.abs(emulate("f32", q, k, v, 0.125, log_norm=x)[0] - 1).max() / A.U for x in (False, True)]
    assert far[0] <= 32 < 64 < far[1], far
