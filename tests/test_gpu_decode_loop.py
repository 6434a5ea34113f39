"""The decoding-time operators as a serving program runs them: stage 3 compacts the caches, tokens are decoded (each layer attends,
appends and accumulates), the caches are evicted down to a budget, decoding goes on -- over the dense cache, the paged one and the
one whose pages were relinked, against a 64-bit model of the same loop in plain lists of rows."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from tests import decode_cases as C

pytestmark = pytest.mark.gpu

LAYERS, VIDEOS, HQ, HKV, DH, PAGE, PER_SEQ = 3, 2, 8, 2, 64, 16, 20
S = PAGE * PER_SEQ
KEPT, STEPS, BUDGET, FIRST, LAST = 180, 70, 200, 4, 20


class Model:
    """Rows and weights per (layer, video) in float64."""

    def __init__(self, k, v):
        self.k, self.v = k, v                        # [layer][video] -> [n, Hkv, dh]
        self.w = [[np.zeros(len(x)) for x in layer] for layer in k]

    def compact(self, idx):
        for l in range(LAYERS):
            for b in range(VIDEOS):
                self.k[l][b], self.v[l][b], self.w[l][b] = self.k[l][b][idx[b]], self.v[l][b][idx[b]], self.w[l][b][idx[b]]

    def attend(self, l, q, k_new, v_new):
        for b in range(VIDEOS):
            self.k[l][b] = np.concatenate([self.k[l][b], k_new[b][None]])
            self.v[l][b] = np.concatenate([self.v[l][b], v_new[b][None]])
            self.w[l][b] = np.append(self.w[l][b], 0.0)
        out, _, mean = D.decode_attention(q, self.k[l], self.v[l], DH ** -0.5)
        for b in range(VIDEOS):
            self.w[l][b] += mean[b]
        return out


def typed(rng, shape):
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


@pytest.mark.parametrize("form", ["dense", "paged", "relinked"])
def test_compact_decode_evict_decode(form):
    from paper_2506_02850_amd import binding as B
    rng = np.random.default_rng(21)
    rows = [[[typed(rng, (S, HKV, DH)) for _ in range(VIDEOS)] for _ in range(LAYERS)] for _ in range(2)]
    model = Model(*[[[rows[w][l][b][1] for b in range(VIDEOS)] for l in range(LAYERS)] for w in range(2)])
    dense = [[torch.stack([rows[w][l][b][0].transpose(0, 1) for b in range(VIDEOS)]).contiguous() for l in range(LAYERS)] for w in range(2)]
    tables = None
    if form == "dense":
        k, v = dense
    else:
        table = rng.permutation(VIDEOS * PER_SEQ).reshape(VIDEOS, PER_SEQ).astype(np.int32)
        k, v = [], []
        for w, to in ((0, k), (1, v)):
            for l in range(LAYERS):
                pool = torch.empty((VIDEOS * PER_SEQ, HKV, PAGE, DH), dtype=torch.bfloat16, device="cuda")
                for b in range(VIDEOS):
                    pool[torch.from_numpy(table[b]).cuda().long()] = dense[w][l][b].view(HKV, PER_SEQ, PAGE, DH).transpose(0, 1)
                to.append(pool)
        tables = [torch.from_numpy(table).cuda()] * LAYERS
    weight = [torch.zeros((VIDEOS, S), device="cuda") for _ in range(LAYERS)]

    # stage 3
    idx = np.stack([np.sort(rng.choice(S, KEPT, replace=False)) for _ in range(VIDEOS)]).astype(np.int32)
    lists = [torch.from_numpy(idx).cuda()] * LAYERS
    if form == "dense":
        new_len = B.metok_kv_compact(k, v, lists)
    elif form == "paged":
        new_len = B.metok_kv_compact_paged(k, v, tables[0], lists)
    else:
        res = B.metok_kv_relink_paged(k, v, tables[0], lists)
        new_len = res["new_len"]
        # the pages that were released come back behind the new ones, as room to grow
        grown = res["page_table_out"].clone()
        used = -(-KEPT // PAGE)
        for l in range(LAYERS):
            for b in range(VIDEOS):
                n = int(res["n_free"][l, b])
                grown[l, b, used:used + n] = res["free_pages"][l, b, :n]
        tables = [grown[l].contiguous() for l in range(LAYERS)]
    lens = new_len[:, None].expand(LAYERS, VIDEOS).contiguous()
    model.compact(idx)

    def decode(steps):
        for _ in range(steps):
            for l in range(LAYERS):
                q, q64 = typed(rng, (VIDEOS, HQ, DH))
                kn, kn64 = typed(rng, (VIDEOS, HKV, DH))
                vn, vn64 = typed(rng, (VIDEOS, HKV, DH))
                if form == "dense":
                    res = B.metok_decode_attention(q, k[l], v[l], lens[l], k_new=kn, v_new=vn, weight=weight[l])
                else:
                    res = B.metok_decode_attention_paged(q, k[l], v[l], tables[l], lens[l], k_new=kn, v_new=vn, weight=weight[l])
                want = model.attend(l, q64, kn64, vn64)
                # half a step of bf16 on the result, and 2^-9 of its largest element for the fp32 steps before (2^-13 each at worst here)
                np.testing.assert_allclose(res["out"].double().cpu().numpy(), want, rtol=2.0 ** -8, atol=2.0 ** -9 * np.abs(want).max())
            lens.add_(1)

    def check_weights():
        for l in range(LAYERS):
            for b in range(VIDEOS):
                n = int(lens[l, b])
                assert n == len(model.w[l][b])
                np.testing.assert_allclose(weight[l][b, :n].double().cpu().numpy(), model.w[l][b], rtol=1e-4)

    decode(STEPS)
    assert int(lens[0, 0]) == KEPT + STEPS > BUDGET
    check_weights()
    # eviction by the weights that the GPU accumulated
    kept = [[D.evict(weight[l][b].cpu().numpy(), KEPT + STEPS, BUDGET, FIRST, LAST) for b in range(VIDEOS)] for l in range(LAYERS)]
    if form == "dense":
        res = B.metok_kv_evict(k, v, weight, lens, BUDGET, FIRST, LAST, new_len=lens)
    elif form == "paged":
        res = B.metok_kv_evict_paged(k, v, tables[0], weight, lens, BUDGET, FIRST, LAST, new_len=lens)
    else:
        res = B.metok_kv_evict_select(weight, lens, S, BUDGET, FIRST, LAST, new_len=lens)
        out = B.metok_kv_relink_paged(k, v, torch.stack(tables), res["idx"], len_in=[KEPT + STEPS] * LAYERS)
        grown = out["page_table_out"].clone()
        used = -(-BUDGET // PAGE)
        for l in range(LAYERS):
            for b in range(VIDEOS):
                n = int(out["n_free"][l, b])
                grown[l, b, used:used + n] = out["free_pages"][l, b, :n]
        tables = [grown[l].contiguous() for l in range(LAYERS)]
    for l in range(LAYERS):
        for b in range(VIDEOS):
            assert res["idx"][l][b].tolist() == kept[l][b] and int(lens[l, b]) == BUDGET
            model.k[l][b], model.v[l][b], model.w[l][b] = (x[l][b][kept[l][b]] for x in (model.k, model.v, model.w))
    check_weights()
    decode(15)
    check_weights()
