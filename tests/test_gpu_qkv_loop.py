"""The operators around queries, keys and values as a serving program runs them: a prompt's keys are rotated into a layer's cache, the rows that stage 3 keeps go into 4
bits, tokens are decoded over them (each is rotated, attends and joins the cache), rows are dropped, decoding goes on -- every stage against its oracle
on what the stages before have left, and a captured step against the eager one."""
import numpy as np
import pytest
import torch

from oracle import qkv_oracle as Q
from tests import kv4_cases as K
from tests.kv4_cases import same, typed

pytestmark = pytest.mark.gpu

VIDEOS, HQ, HKV, DH, AXES, ROT = 2, 8, 2, 64, 3, 48
PROMPT, COUNTS, KEPT, STEPS = 200, [200, 150], [120, 97], 20
FREQ = (np.float32(10000.0) ** (-np.arange(ROT // 2, dtype=np.float32) * 2 / ROT)).astype(np.float32)
AXIS = bytes(i % AXES for i in range(ROT // 2))


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class Layer:
    """A layer's weights of the norms, its 4-bit cache on the device and, row by row in float64, on the host."""

    def __init__(self, B, dtype, capacity, page, seed):
        self.B, self.dtype, self.capacity, self.page = B, dtype, capacity, page
        self.rng = np.random.default_rng(seed)
        self.norms = [typed(1 + 0.2 * self.rng.standard_normal(DH), dtype) for _ in range(2)]
        self.freq = torch.from_numpy(FREQ).cuda()
        self.cache = K.Cache4(VIDEOS, HKV, capacity, DH, page, seed)
        self.k4, self.v4, self.table = self.cache.device()
        self.rows = None                                   # [K, V][video] -> [n, Hkv, dh], what the codes stand for
        self.lens = i32([0] * VIDEOS)
        self.ws = torch.empty(max(256, B.metok_kv4_attention_workspace_bytes(VIDEOS, HQ, HKV, capacity, DH, B.BF16 if dtype == "bf16" else B.F32)), dtype=torch.uint8, device="cuda")

    def rotate(self, qkv, pos, k, v, count=None, out=None):
        return self.B.metok_rotate_qk(qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HKV], qkv[:, :, HQ + HKV:], pos, self.freq, k, v, count=count, pair_axis=AXIS,
                                      q_weight=self.norms[0][0], k_weight=self.norms[1][0], out=out)["q"]

    def rotated(self, x, pos, which):
        want = Q.rotate(x, self.norms[which][1], 1e-6, pos, FREQ, list(AXIS), Q.HALVES)
        return want, K.rotate_tolerance(x, self.norms[which][1], 1e-6, want, self.dtype, DH, ROT // 2, Q.HALVES)

    def attend(self, q, kn, vn, out=None):
        if self.page:
            return self.B.metok_kv4_attention_paged(q, self.k4, self.v4, self.table, self.lens, k_new=kn, v_new=vn, workspace=self.ws, out=out)
        return self.B.metok_kv4_attention(q, self.k4, self.v4, self.lens, k_new=kn, v_new=vn, workspace=self.ws, out=out)

    def step(self, qkv, pos, scratch, out=None):
        """One token of every video: its keys and values go through a cache of one row."""
        q = self.rotate(qkv, pos, *scratch, out=out)[:, :, 0]
        kn, vn = (x.view(VIDEOS, HKV, DH) for x in scratch)
        res = self.attend(q, kn, vn, out)
        self.lens += 1
        return q, kn, vn, res

    def pack(self, k, v, idx, count):
        if self.page:
            self.B.metok_kv4_pack_paged(k, v, self.k4, self.v4, self.table, count=i32(count), idx=idx)
        else:
            self.B.metok_kv4_pack(k, v, self.k4, self.v4, count=i32(count), idx=idx)
        self.lens.copy_(i32(count))

    def unpack(self, idx):
        if self.page:
            return self.B.metok_kv4_unpack_paged(self.k4, self.v4, self.table, self.lens, idx.shape[1], idx=idx, dtype=K.TORCH[self.dtype])
        return self.B.metok_kv4_unpack(self.k4, self.v4, self.lens, idx.shape[1], idx=idx, dtype=K.TORCH[self.dtype])

    def check_cache(self):
        for which, t in ((0, self.k4), (1, self.v4)):
            assert np.array_equal(t.cpu().numpy(), self.cache.data[which])

    def checked_step(self, scratch):
        x, x64 = typed(self.rng.standard_normal((VIDEOS, 1, HQ + 2 * HKV, DH)), self.dtype)
        pos = self.rng.integers(0, 5000, (AXES, VIDEOS, 1)).astype(np.int32)
        held = [len(r) for r in self.rows[0]]
        assert self.lens.tolist() == held
        q, kn, vn, res = self.step(x, i32(pos), scratch)
        got = [t.double().cpu().numpy() for t in (q, kn, vn)]
        for b in range(VIDEOS):
            for which, part in ((0, slice(0, HQ)), (1, slice(HQ, HQ + HKV))):
                want, limit = self.rotated(x64[b, :, part], pos[:, b], which)
                assert (np.abs(got[which][b] - want[0]) <= limit[0]).all()
            assert np.array_equal(got[2][b], x64[b, 0, HQ + HKV:])
        K.check(dict(dtype=self.dtype, held=held, Hq=HQ, Hkv=HKV, dh=DH, capacity=self.capacity, append=True, cap=0.0, q64=got[0], new64=got[1:], rows64=self.rows, weight=None), res)
        for which in range(2):
            for b in range(VIDEOS):
                self.rows[which][b] = np.concatenate([self.rows[which][b], self.cache.put(which, b, [held[b]], got[1 + which][b][None])])


@pytest.mark.parametrize("dtype,capacity,page", [("bf16", 256, 0), ("bf16", 2048, 32), ("f32", 256, 16)])
def test_prompt_pack_decode_drop_decode(dtype, capacity, page):
    from paper_2506_02850_amd import binding as B
    layer = Layer(B, dtype, capacity, page, seed=31)
    rng = layer.rng
    # the prompt
    x, x64 = typed(rng.standard_normal((VIDEOS, PROMPT, HQ + 2 * HKV, DH)), dtype)
    pos = rng.integers(0, 300, (AXES, VIDEOS, PROMPT)).astype(np.int32)
    k, v = (torch.full((VIDEOS, HKV, 224, DH), 9.0, dtype=K.TORCH[dtype], device="cuda") for _ in range(2))
    q = layer.rotate(x, i32(pos), k, v, count=i32(COUNTS)).double().cpu().numpy()
    k64, v64 = (t.double().cpu().numpy() for t in (k, v))
    for b, n in enumerate(COUNTS):
        for got, which, part in ((q, 0, slice(0, HQ)), (k64, 1, slice(HQ, HQ + HKV))):
            want, limit = layer.rotated(x64[b, :n, part], pos[:, b, :n], which)
            assert (np.abs(got[b, :, :n].transpose(1, 0, 2) - want) <= limit).all()
        assert np.array_equal(v64[b, :, :n].transpose(1, 0, 2), x64[b, :n, HQ + HKV:]) and (k64[b, :, n:] == 9.0).all() and (v64[b, :, n:] == 9.0).all()
    # the rows that stay
    idx = np.zeros((VIDEOS, max(KEPT)), dtype=np.int32)
    for b, n in enumerate(KEPT):
        idx[b, :n] = np.sort(rng.choice(COUNTS[b], n, replace=False))
    layer.pack(k, v, i32(idx), KEPT)
    layer.rows = [[layer.cache.put(w, b, np.arange(n), x64_[b][:, idx[b, :n]].transpose(1, 0, 2)) for b, n in enumerate(KEPT)] for w, x64_ in ((0, k64), (1, v64))]
    layer.check_cache()
    # decoding
    scratch = [torch.empty((VIDEOS, HKV, 1, DH), dtype=K.TORCH[dtype], device="cuda") for _ in range(2)]
    for _ in range(STEPS):
        layer.checked_step(scratch)
    layer.check_cache()
    # every other row goes, and what stays keeps its codes
    stay = [np.arange(b, KEPT[b] + STEPS, 2) for b in range(VIDEOS)]
    idx = np.full((VIDEOS, max(map(len, stay))), -1, dtype=np.int32)
    for b, s in enumerate(stay):
        idx[b, :len(s)] = s
    out = layer.unpack(i32(idx))
    for which, name in ((0, "k"), (1, "v")):
        got = out[name].double().cpu().numpy()
        for b, s in enumerate(stay):
            assert np.array_equal(got[b, :, :len(s)].transpose(1, 0, 2), layer.rows[which][b][s])
    layer.pack(out["k"], out["v"], None, [len(s) for s in stay])
    for which in range(2):
        for b, s in enumerate(stay):
            layer.rows[which][b] = layer.rows[which][b][s]
            assert np.array_equal(layer.cache.put(which, b, np.arange(len(s)), layer.rows[which][b]), layer.rows[which][b])
    layer.check_cache()
    for _ in range(STEPS):
        layer.checked_step(scratch)
    layer.check_cache()


@pytest.mark.parametrize("capacity,page", [(128, 0), (2048, 16)])
def test_a_captured_step_is_the_eager_one(capacity, page):
    """Rotation, attention and the lengths' step in one graph, replayed for thirty tokens; the eager steps run between the replays on a layer of their own."""
    from paper_2506_02850_amd import binding as B
    layers = [Layer(B, "bf16", capacity, page, seed=5) for _ in range(2)]
    k, v = (torch.randn((VIDEOS, HKV, 90, DH), generator=torch.Generator().manual_seed(s)).to(torch.bfloat16).cuda() for s in (1, 2))
    for layer in layers:
        layer.pack(k, v, None, [90, 61])
    x = torch.zeros((VIDEOS, 1, HQ + 2 * HKV, DH), dtype=torch.bfloat16, device="cuda")
    pos = i32(np.zeros((AXES, VIDEOS, 1)))
    scratch = [[torch.empty((VIDEOS, HKV, 1, DH), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    out = dict(q=torch.empty((VIDEOS, HQ, 1, DH), dtype=torch.bfloat16, device="cuda"), out=torch.empty((VIDEOS, HQ, DH), dtype=torch.bfloat16, device="cuda"),
               lse=torch.empty((VIDEOS, HQ), device="cuda"))
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        layers[0].step(x, pos, scratch[0], out)
        pos += 1
    pos_eager = torch.zeros_like(pos)
    assert int(pos.sum()) == 0 and layers[0].lens.tolist() == [90, 61]          # a capture runs nothing
    for token in range(30):
        x.normal_()
        graph.replay()
        q, _, _, res = layers[1].step(x, pos_eager, scratch[1])
        pos_eager += 1
        torch.cuda.synchronize()
        assert same(out["q"][:, :, 0], q) and same(out["out"], res["out"]) and same(out["lse"], res["lse"]), token
    assert same(layers[0].k4, layers[1].k4) and same(layers[0].v4, layers[1].v4) and layers[0].lens.tolist() == [120, 91]
