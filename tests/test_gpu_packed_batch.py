"""The packed operators run together by PackedBatch: prompts, drafts, single tokens, a pool that runs out, requests that end."""
import numpy as np
import pytest
import torch

import paper_2510_15312_amd as vf
from oracle import packed as op
from paper_2510_15312_amd.packed_batch import PackedBatch
from test_gpu_packed import DTYPES, Packed, _pool_rows
from util_gpu import DEV, i32

pytestmark = pytest.mark.gpu
LAYERS = 2


class Story:
    """A batch with the keys and values that it should hold, per layer and request."""

    def __init__(self, dtype, hq, hkv, hd, n, pages, tokens, part=None, pairs=vf.VF_ROTARY_HALF):
        self.batch = PackedBatch(n, LAYERS, hq, hkv, hd, pages, tokens, DTYPES[dtype], part, 1e4, pairs, DEV)
        self.hq, self.hkv, self.hd, self.dt, self.part, self.pairs = hq, hkv, hd, DTYPES[dtype], part or hd, pairs
        self.gen = torch.Generator(device=DEV).manual_seed(n)
        self.kept = [[np.zeros((2, 0, hkv, hd)) for _ in range(n)] for _ in range(LAYERS)]     # 0: unrotated keys, 1: values

    def step(self, new, granted):
        batch, lens = self.batch, list(self.batch.host_lens)
        row_off, pos = batch.begin(new)
        off = np.concatenate([[0], np.cumsum(new)])
        assert row_off.tolist() == off.tolist()
        outs = []
        for layer in range(LAYERS):
            qkv = torch.randn((int(off[-1]), self.hq + 2 * self.hkv, self.hd), generator=self.gen, device=DEV).to(self.dt)
            q, k, v = qkv.split((self.hq, self.hkv, self.hkv), 1)
            outs.append((q, batch.attend(layer, q, k, v)))
            for b in range(len(new)):
                if granted[b]:
                    rows = torch.stack((k, v))[:, off[b]:off[b + 1]].double().cpu().numpy()
                    self.kept[layer][b] = np.concatenate([self.kept[layer][b], rows], 1)
        assert batch.finish() == granted
        want = [h + w if g else h for h, w, g in zip(lens, new, granted)]
        assert batch.host_lens == want and batch.lens.tolist() == want
        assert batch.host_free == int(batch.n_free) == batch.free.numel() - sum(-(-n // 64) for n in want)
        for layer, (q, out) in enumerate(outs):
            self.check(layer, q, out, pos, off, [n if g else 0 for n, g in zip(want, granted)])
        pages = [p for b, n in enumerate(want) for p in batch.table[b, :-(-n // 64)].tolist()] + batch.free[:batch.host_free].tolist()
        assert sorted(pages) == list(range(batch.free.numel()))                     # every page has one owner

    def check(self, layer, q, out, pos, off, kv_len):
        batch, p = self.batch, Packed.__new__(Packed)
        p.hd, p.dt, p.row_off, p.kv_len, p.k, p.v = self.hd, self.dt, off, kv_len, [], []
        p.q = torch.empty_like(q.contiguous())
        nowhere = torch.full_like(pos, -1)
        vf.vf_rotary_append(q, q[:, :self.hkv], q[:, :self.hkv], batch.angles, pos, nowhere, p.q, batch.pools[layer], self.pairs)
        for b, n in enumerate(batch.host_lens):
            t = np.arange(n)
            slots = 64 * batch.table[b].cpu().numpy()[t // 64] + t % 64
            k, v = (x.double().cpu().numpy() for x in _pool_rows(batch.pools[layer], i32(slots), self.hd))
            angles = op.rotary_table(self.part, 1e4, n)
            want = op.rotate(self.kept[layer][b][0], angles, self.pairs == vf.VF_ROTARY_INTERLEAVED)
            # the angles' float32 rounding (2^-24 of a pair's two values) and three float32 operations, then the type's rounding
            size = 8 * 2.0 ** -24 * np.abs(want).max(initial=0)
            unit = 2.0 ** -8 if self.dt == torch.bfloat16 else 0.0
            assert (np.abs(k - want) <= 2 * size + unit * (np.abs(want) + size)).all()
            assert np.array_equal(v, self.kept[layer][b][1])
            p.k.append(k), p.v.append(v)
        p.check(out)

    def keep(self, request, tokens):
        self.batch.keep(request, tokens)
        for layer in self.kept:
            layer[request] = layer[request][:, :tokens]


@pytest.mark.parametrize("dtype,hq,hkv,hd,part,pairs", [("bf16", 12, 2, 128, None, vf.VF_ROTARY_HALF), ("bf16", 14, 2, 64, 32, vf.VF_ROTARY_INTERLEAVED),
                                                        ("f32", 4, 4, 64, None, vf.VF_ROTARY_HALF)])
def test_a_batch_is_served(dtype, hq, hkv, hd, part, pairs):
    s = Story(dtype, hq, hkv, hd, 4, pages=9, tokens=260, part=part, pairs=pairs)
    s.step([130, 1, 0, 64], [True, True, True, True])             # prompts: 3 + 1 + 0 + 1 pages of 9
    s.step([1, 1, 65, 1], [True, True, True, True])               # tokens, and a prompt: 2 + 1 more, one is left
    s.step([17, 130, 2, 33], [True, False, True, True])            # drafts; the second needs two pages
    s.keep(0, 133)                                                # two of the drafts were accepted
    s.keep(3, 66)
    s.step([1, 0, 1, 1], [True, True, True, True])
    s.batch.release(2)
    s.kept = [[x if b != 2 else x[:, :0] for b, x in enumerate(layer)] for layer in s.kept]
    s.step([1, 130, 0, 1], [True, True, True, True])               # now it has room
    s.step([0, 0, 330, 0], [True, True, False, True])             # longer than the table
    s.step([0, 0, 0, 0], [True] * 4)
    s.step([1, 1, 10, 1], [True] * 4)
    for b in range(4):
        s.batch.release(b)
    assert s.batch.host_free == 9 and not s.batch.lens.any() and (s.batch.table == -1).all()


def test_keep_refuses_what_a_request_does_not_hold():
    batch = PackedBatch(1, 1, 4, 4, 64, 2, 64, torch.float32)
    for tokens in (-1, 1):
        with pytest.raises(ValueError):
            batch.keep(0, tokens)
