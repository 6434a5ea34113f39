"""How exact the one-token attention has to be on ordinary inputs: root mean square errors and misrounded results, beside decode_cases.py's
worst cases, which are a hundred times what happens.

Inputs: normal q (deviation 2), k and v, so that scores have a deviation of 2.  With u = 2^-24 and roundings taken as independent, uniform within
half a step (deviation u / sqrt 3 of the number rounded, 0.7 of that averaged over a binade):
  - a score, as its exponent: dh additions with partial sums of sqrt(t) 2, 0.8 sqrt(dh) u after the scale;
  - the distance to the maximum, some 8 there: two roundings, 2 to 4 u each; exp2, one step of its result;
  - the sums over the rows: chains of up to 60 additions, 3 u.
Together (sqrt(dh) + 8) u at most, relative to a probability, or to the deviation that the result would have if every row's part were wrong
independently, N = sqrt(sum (p_j (v_j - out))^2).  Three times that is the bound: independence is an assumption, the sums over thousands
of elements leave little to chance.
bf16: the products are exact, the scores as above; a probability in two bf16 parts is off by 2^-18 / sqrt 3 (26 u with the binade).  The result is rounded to bf16
once; an element is misrounded with probability |error| / step.  With an error of 27 u N and elements normal with deviation N or more that
is 0.8 c (1 + log(1 / c)), c = 0.8 * 1.39 * 2^7 * 27 u = 2.3e-4: 0.17 %.  The bound is 1 %; probabilities in one bf16 number give 29 %."""
import numpy as np

from oracle import decode_oracle as D

U = 2.0 ** -24


def bf16(x):
    """Rounded to bf16, as float64."""
    b = np.asarray(x, dtype=np.float32).view(np.uint32)
    return ((b + 0x7fff + ((b >> 16) & 1)) & np.uint32(0xffff0000)).view(np.float32).astype(np.float64)


def cut(x, bits):
    """Rounded to so many significant bits."""
    m, e = np.frexp(np.asarray(x, dtype=np.float64))
    return np.ldexp(np.rint(m * 2.0 ** bits) / 2.0 ** bits, e)


def bound(dh):
    return 3 * (dh ** 0.5 + 8) * U


MISROUNDED = 0.01


def spread_of(q, keys, values, scale):
    """N for every element [B, Hq, dh]."""
    B, Hq, dh = q.shape
    out = np.zeros((B, Hq, dh))
    for b in range(B):
        for h in range(Hq):
            kv = h // (Hq // keys[b].shape[1])
            o, _, p = D.attend(q[b, h], keys[b][:, kv], values[b][:, kv], scale)
            out[b, h] = np.sqrt((p[:, None] ** 2 * (values[b][:, kv] - o) ** 2).sum(0))
    return out


def faults(dtype, got, q, keys, values, scale):
    """got: out [B, Hq, dh], lse [B, Hq] and, or None, the weights of a first step per video, as float64.  Says what is too far off."""
    out, lse, mean = D.decode_attention(q, keys, values, scale)
    dh = q.shape[2]
    said = []
    if dtype == "f32":
        rms = np.sqrt(((got[0] - out) ** 2).mean() / (spread_of(q, keys, values, scale) ** 2).mean())
        if not rms <= bound(dh):
            said.append(f"out: {rms / U:.1f} u of {bound(dh) / U:.1f}")
    else:
        wrong = (got[0] != bf16(out)).mean()
        if not wrong <= MISROUNDED:
            said.append(f"out: {100 * wrong:.2f} % misrounded")
    rms, most = np.sqrt(((got[1] - lse) ** 2).mean()), bound(dh) / 3 + U * np.abs(lse).max()
    if not rms <= most:
        said.append(f"lse: {rms / U:.1f} u of {most / U:.1f}")
    if got[2] is not None:
        rms = np.sqrt(np.mean([((w[:len(p)] / p - 1) ** 2).mean() for w, p in zip(got[2], mean)]))
        if not rms <= bound(dh):
            said.append(f"weights: {rms / U:.1f} u of {bound(dh) / U:.1f}")
    return said
