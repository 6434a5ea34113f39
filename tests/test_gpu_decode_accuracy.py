"""GPU tests of how exact metok_decode_attention is, with bounds near its own roundings (those of decode_cases.py are worst cases)."""
import pytest
import torch

from tests import decode_accuracy as A
from tests import decode_cases as C

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                                   # half a step of fp32
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
# One launch (200 rows without weights) and split over the chip; some shares of a wave are a part, some a whole video.
FORMS = [(200, False), (200, True), (40, True), (3000, False), (3000, True), (20000, False)]


def mk():
    from paper_2506_02850_amd import binding as B
    return B


def around(offset, rows, dtype, seed, videos=4, heads=4, kv_heads=2, dh=64):
    """q and K whose scores lie around `offset`, with a standard deviation of about 1; all numbers fit both types."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = torch.randn((videos, kv_heads, rows, dh), generator=g, device="cuda")
    q = torch.randn((videos, heads, dh), generator=g, device="cuda")
    q[..., 0], k[..., 0] = 16.0, offset / 16.0 * dh ** 0.5
    return q.to(TORCH[dtype]), k.to(TORCH[dtype])


@pytest.mark.parametrize("rows,weights", FORMS)
@pytest.mark.parametrize("offset", [0.0, 60.0, 200.0, 700.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_values_come_out_as_they_are(rows, weights, offset, dtype):
    """All rows of V are 1: the result is the sum of the probabilities, 1 whatever the scores.  Output and sum add up the same fp32 numbers
    in other orders, some 240 additions in a chain at most, each off by u of the sum so far: 3 sqrt(240 / 3) u = 27 u at three
    standard deviations, 32 u with the division and the factors between the parts.  bf16: a probability in two parts is 2^-17 off at
    most, which rounds to 1."""
    q, k = around(offset, rows, dtype, seed=rows)
    v = torch.ones_like(k)
    lens = torch.tensor([rows, rows - 1, rows // 2, 1], dtype=torch.int32, device="cuda")
    res = mk().metok_decode_attention(q, k, v, lens, weight=torch.zeros((4, rows), device="cuda") if weights else None)
    far = (res["out"].double() - 1).abs().max().item()
    assert far <= (32 * U if dtype == "f32" else 0.0), f"{far / U:.1f} u"


@pytest.mark.parametrize("rows", [40, 200, 3000, 20000])
@pytest.mark.parametrize("offset", [0.0, 60.0, 200.0, 700.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_weights_of_a_step_add_up_to_one(rows, offset, dtype):
    """One query head, weights that start at 0, added up in 64 bits: the probabilities' sum.  The sum that they were divided by has the chains of
    the test above (27 u); the probabilities are computed once more for the weights, from the same scores: exponents up to 24 below
    the largest, each rounded once (17 u there, and of random sign), an exp2 of 2 u.  40 u."""
    videos = 6
    q, k = around(offset, rows, dtype, seed=rows + 1, videos=videos, heads=1, kv_heads=1)
    lens = torch.tensor([rows, rows - 1, rows // 2, 33, 16, 1], dtype=torch.int32, device="cuda")
    w = torch.zeros((videos, rows), device="cuda")
    mk().metok_decode_attention(q, k, torch.ones_like(k), lens, weight=w)
    far = (w.double().sum(1) - 1).abs().max().item()
    assert far <= 40 * U, f"{far / U:.1f} u"


@pytest.mark.parametrize("rows,weights", FORMS)
@pytest.mark.parametrize("exponent,cap", [(0, 0.0), (16, 0.0), (32, 0.0), (64, 0.0), (118, 0.0), (0, 2.0 ** 70), (16, 2.0 ** 70), (32, 2.0 ** 70),
                                          (118, 2.0 ** 70)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_of_any_size(rows, weights, exponent, cap, dtype):
    """Scores of 2^exponent times 1 to 15, exact in fp32.  From 2^16 on only the largest of a video count, with a probability of 1, and sums of
    the small whole numbers in V are exact: a quotient's roundings are left.  Scores of 1 to 15 are rounded in the log2 domain, to 21.6 u and,
    capped, twice, so that probabilities below 1 are off by 30 u at most: those have 0.37 of the sum, the values they draw to are 16
    apart at most, 0.37 * 30 u * 16 = 178 u, below 8 * 2^-19 = 256 u.  bf16: two parts of a probability are 2^-17 off, and the result is
    rounded.  A cap of 2^70 leaves scores up to 2^36 as they are and makes those of 2^118 equal: tanh is 1.  The logarithm is a product
    of three rounded factors, the weights are off as the probabilities are, and by the sum's 7 u."""
    videos, dh = 3, 64
    g = torch.Generator().manual_seed(rows + exponent)
    t = torch.randint(1, 16, (videos, 2, rows), generator=g)
    v = torch.randint(-8, 9, (videos, 2, rows, dh), generator=g).double()
    k = torch.zeros((videos, 2, rows, dh), dtype=torch.float64)
    k[..., 5] = t.double() * 2.0 ** (exponent - exponent // 2)
    q = torch.zeros((videos, 4, dh), dtype=torch.float64)
    q[..., 5] = 2.0 ** (exponent // 2)
    lens = [rows, rows - 1, rows // 2]
    x = 2.0 ** exponent * t.double()
    if cap:
        x = cap * torch.tanh(x / cap)
    want_w = torch.zeros((videos, rows), dtype=torch.float64)
    want, lse = torch.zeros((videos, 4, dh), dtype=torch.float64), torch.zeros((videos, 4), dtype=torch.float64)
    for b, n in enumerate(lens):
        p = torch.softmax(x[b, :, :n], -1)
        want_w[b, :n] = p.mean(0)
        want[b] = torch.matmul(p[:, None], v[b, :, :n])[:, 0].repeat_interleave(2, 0)
        lse[b] = torch.logsumexp(x[b, :, :n], -1).repeat_interleave(2, 0)
    to = lambda z: z.to(TORCH[dtype]).cuda()
    w = torch.zeros((videos, rows), device="cuda")
    res = mk().metok_decode_attention(to(q), to(k), to(v), torch.tensor(lens, dtype=torch.int32, device="cuda"), scale=1.0, logit_cap=cap,
                                      weight=w if weights else None)
    far = (res["out"].double().cpu() - want).abs()
    if dtype == "bf16":
        assert (far <= 2.0 ** -8 * want.abs() + 8 * 2.0 ** -15).all(), far.max()
    else:
        assert (far <= 8 * 2.0 ** -19).all(), far.max()
    assert ((res["lse"].double().cpu() - lse).abs() <= 8 * U * (lse.abs() + 1)).all()
    if weights:
        assert ((w.double().cpu() - want_w).abs() <= 2.0 ** -18 * want_w + 2.0 ** -126).all()


@pytest.mark.parametrize("dtype,dh", [("bf16", 32), ("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 32), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("page", [0, 16, 7])
@pytest.mark.parametrize("rows,weights,Hq,Hkv", [(300, False, 8, 2), (300, True, 8, 2), (4000, False, 8, 2), (4000, True, 14, 2), (700, True, 40, 1), (700, False, 64, 1)])
def test_errors_are_those_of_fp32(dtype, dh, page, rows, weights, Hq, Hkv):
    """Ordinary inputs: one launch, split and joined, many query heads; root mean squares as decode_accuracy.py derives them."""
    capacity = (rows + 10) if page == 0 else page * (-(-(rows + 10) // page))
    c = C.make(dtype, [rows, rows - 5, rows // 2, 200], Hq, Hkv, dh, capacity, page, append=weights, weights=weights, seed=rows + dh + page)
    if weights:
        c["weight"].zero_()
    res = C.call(mk(), c)
    keys, values = C.attended(c)
    got = [res["out"].double().cpu().numpy(), res["lse"].double().cpu().numpy(), None]
    if weights:
        w = c["weight"].double().cpu().numpy()
        got[2] = [w[b, :len(k)] for b, k in enumerate(keys)]
    assert A.faults(dtype, got, c["q64"], keys, values, dh ** -0.5) == []
