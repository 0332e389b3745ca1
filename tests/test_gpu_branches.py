"""PackedBatch with requests that branch: norms of heads, forks, drafts cut back into shared pages, requests that end, another pool,
adjusted logits, against the float64 oracle; the same calls in a graph."""
import numpy as np
import pytest
import torch

import paper_2510_15312_amd as vf
from oracle import packed as op
from paper_2510_15312_amd.packed_batch import PackedBatch
from test_gpu_packed import DTYPES, Packed, _pool_rows, _rotary_inputs
from util_gpu import DEV, f32, i32

pytestmark = pytest.mark.gpu
LAYERS, EPS = 2, 1e-6


class Story:
    """A batch with the keys (normalised, not rotated) and values that it should hold, per layer and request."""

    def __init__(self, dtype, hq, hkv, hd, n, pages, tokens, norms):
        self.batch = PackedBatch(n, LAYERS, hq, hkv, hd, pages, tokens, DTYPES[dtype], None, 1e4, device=DEV)
        self.hq, self.hkv, self.hd, self.dt = hq, hkv, hd, DTYPES[dtype]
        self.gen = torch.Generator(device=DEV).manual_seed(n)
        self.norms = [None] * LAYERS
        if norms:
            self.norms = [(1 + 0.2 * torch.randn((hq, hd), generator=self.gen, device=DEV), 1 + 0.2 * torch.randn(hd, generator=self.gen, device=DEV), EPS)
                          for _ in range(LAYERS)]
        self.kept = [[np.zeros((2, 0, hkv, hd)) for _ in range(n)] for _ in range(LAYERS)]

    def step(self, new, granted=None):
        batch, lens = self.batch, list(self.batch.host_lens)
        granted = granted or [True] * len(new)
        _, pos = batch.begin(new)
        off, outs = np.concatenate([[0], np.cumsum(new)]), []
        for layer, norms in enumerate(self.norms):
            qkv = torch.randn((int(off[-1]), self.hq + 2 * self.hkv, self.hd), generator=self.gen, device=DEV).to(self.dt)
            q, k, v = qkv.split((self.hq, self.hkv, self.hkv), 1)
            outs.append((q, batch.attend(layer, q, k, v, norms)))
            keys = k.double().cpu().numpy() if norms is None else op.norm_heads(k.double().cpu().numpy(), norms[1].double().cpu().numpy(), EPS)
            for b in range(len(new)):
                if granted[b]:
                    rows = np.stack((keys, v.double().cpu().numpy()))[:, off[b]:off[b + 1]]
                    self.kept[layer][b] = np.concatenate([self.kept[layer][b], rows], 1)
        assert batch.finish() == granted
        want = [h + w if g else h for h, w, g in zip(lens, new, granted)]
        assert batch.host_lens == want
        for layer, (q, out) in enumerate(outs):
            self.check(layer, q, out, pos, off, [n if g else 0 for n, g in zip(want, granted)])
        self.owners()

    def check(self, layer, q, out, pos, off, kv_len):
        batch, p = self.batch, Packed.__new__(Packed)
        p.hd, p.dt, p.row_off, p.kv_len, p.k, p.v = self.hd, self.dt, off, kv_len, [], []
        p.q = torch.empty_like(q.contiguous())
        nowhere = torch.full_like(pos, -1)
        some = q[:, :self.hkv]
        if self.norms[layer] is None:
            vf.vf_rotary_append(q, some, some, batch.angles, pos, nowhere, p.q, batch.pools[layer])
        else:
            vf.vf_norm_rotary_append(q, some, some, *self.norms[layer], batch.angles, pos, nowhere, p.q, batch.pools[layer])
        for b, n in enumerate(batch.host_lens):
            t = np.arange(n)
            slots = 64 * batch.table[b].cpu().numpy()[t // 64] + t % 64
            k, v = (x.double().cpu().numpy() for x in _pool_rows(batch.pools[layer], i32(slots), self.hd))
            want = op.rotate(self.kept[layer][b][0], op.rotary_table(self.hd, 1e4, n), False)
            # norms: (hd + 3) / 2 + 7 roundings of 2^-24 (sum of squares, root, division, two products); angles 2^-24; rotation 3; each of a pair's size
            size = ((self.hd + 3) / 2 + 12) * 2.0 ** -24 * np.abs(want).max(initial=0)
            unit = 2.0 ** -8 if self.dt == torch.bfloat16 else 0.0
            assert (np.abs(k - want) <= 2 * size + unit * (np.abs(want) + size)).all()
            assert np.array_equal(v, self.kept[layer][b][1])
            p.k.append(k), p.v.append(v)
        p.check(out)

    def owners(self):
        """Every page is held as often as its count says, or is free once."""
        batch = self.batch
        held = np.zeros(batch.free.numel(), int)
        for b, n in enumerate(batch.host_lens):
            for p in batch.table[b, :-(-n // 64)].tolist():
                held[p] += 1
        free, shares = batch.free[:batch.host_free].tolist(), batch.shares.cpu().numpy()
        assert batch.lens.tolist() == batch.host_lens and int(batch.n_free) == batch.host_free
        assert sorted(free + np.flatnonzero(held).tolist()) == list(range(len(held))) and (shares == np.maximum(held - 1, 0)).all()

    def fork(self, src, dst, tokens=None, granted=None):
        assert self.batch.fork(src, dst, tokens) == (granted or [True] * len(src))
        for i, (s, d) in enumerate(zip(src, dst)):
            if granted is None or granted[i]:
                for layer in self.kept:
                    layer[d] = layer[s][:, :layer[s].shape[1] if tokens is None else tokens[i]]
        self.owners()

    def cut(self, held):
        for layer in self.kept:
            layer[:] = [x[:, :n] for x, n in zip(layer, held)]
        self.owners()


@pytest.mark.parametrize("dtype,hq,hkv,hd,norms", [("bf16", 12, 2, 128, True), ("bf16", 14, 2, 64, False), ("f32", 4, 4, 64, True)])
def test_a_batch_that_branches(dtype, hq, hkv, hd, norms):
    s = Story(dtype, hq, hkv, hd, 6, pages=13, tokens=400, norms=norms)
    s.step([150, 64, 0, 0, 0, 0])                                  # 3 + 1 pages of 13
    s.fork([0, 0, 1], [2, 3, 4])                                   # 1 + 1 + 0 more
    s.step([1, 1, 17, 5, 65, 0])                                   # they part: 0 + 1 + 0 + 0 + 2
    s.fork([2], [5], [130])
    with pytest.raises(ValueError):
        s.batch.fork([0], [5])
    assert s.batch.keep(2, 100) == 100                             # inside a page that 0, 3 and 5 hold
    s.cut([151, 65, 100, 155, 129, 130])
    s.step([1, 1, 3, 1, 1, 1])
    assert s.batch.keep_all([None, 64, 70, 0, 1, None]) == [152, 64, 70, 0, 1, 131]
    s.cut([152, 64, 70, 0, 1, 131])
    held = s.batch.free.numel() - s.batch.host_free
    for pages in (held, 9):
        s.batch.compact(pages)
        s.owners()
        s.step([1, 0, 2, 0, 0, 1])
    s.batch.release(0)
    s.cut([0, 64, 74, 0, 1, 133])
    s.step([1, 0, 1, 0, 0, 60])
    assert s.batch.keep_all([0] * 6) == [0] * 6 and s.batch.host_free == 9 and not s.batch.shared
    s.cut([0] * 6)
    s.step([30, 0, 64, 0, 65, 1])


def test_forks_and_cuts_that_find_no_page():
    s = Story("f32", 4, 4, 64, 5, pages=4, tokens=200, norms=False)
    s.step([100, 0, 0, 0, 0])
    s.fork([0, 0, 0], [1, 2, 3], granted=[True, True, False])
    assert s.batch.host_lens == [100, 100, 100, 0, 0] and s.batch.host_free == 0
    assert s.batch.keep(1, 30) == 30                               # its own page goes to the copy of the shared one
    s.cut([100, 30, 100, 0, 0])
    s.fork([0], [4], [64])
    s.fork([0], [3], [64])
    assert s.batch.keep(4, 63) == 0                                # no page is left, none is full
    s.cut([100, 30, 100, 64, 0])
    assert s.batch.keep_all([64, 0, 64, 20, None]) == [64, 0, 64, 20, 0]
    s.cut([64, 0, 64, 20, 0])
    s.step([1, 0, 60, 1, 0])


def test_compact_refuses_too_small_a_pool_and_open_steps():
    batch = PackedBatch(2, 1, 4, 4, 64, 6, 200, torch.float32, device=DEV)
    x = torch.randn((130, 12, 64), device=DEV)
    batch.begin([129, 1])
    for call in (lambda: batch.compact(6), lambda: batch.fork([0], [1]), lambda: batch.keep_all([0, 0])):
        with pytest.raises(RuntimeError):
            call()
    batch.attend(0, x[:, :4], x[:, 4:8], x[:, 8:])
    batch.finish()
    for call in (lambda: batch.compact(3), lambda: batch.fork([0], [1]), lambda: batch.fork([2], [1]), lambda: batch.fork([0], [1], [0, 1]),
                 lambda: batch.keep_all([1]), lambda: batch.keep_all([130, 0]), lambda: batch.keep_all([-2, 0])):
        with pytest.raises(ValueError):
            call()
    batch.release(1)
    for call in (lambda: batch.fork([0, 0], [1, 1]), lambda: batch.fork([0], [1], [130]), lambda: batch.fork([0], [-1])):
        with pytest.raises(ValueError):
            call()
    assert batch.fork([], []) == [] and batch.host_lens == [129, 0]


def test_logits_of_a_step():
    batch = PackedBatch(3, 1, 4, 4, 64, 6, 200, torch.float32, device=DEV)
    with pytest.raises(RuntimeError):
        batch.adjust(torch.zeros((1, 8), device=DEV))
    batch.begin([2, 0, 1])
    z, tokens = torch.randn((3, 500), device=DEV), i32([7, 9, 7])
    out = batch.adjust(z, tokens, penalties=f32([[2, 0.5, 0.25]] * 3), history=i32([[7], [8], [9]]), history_len=i32([1, 1, 1]))
    want = op.logits_adjust(z.double().cpu().numpy(), [0, 2, 2, 3], [[2, 0.5, 0.25]] * 3, [[7], [8], [9]], None, [7, 9, 7])
    assert np.allclose(out.cpu().numpy(), want, rtol=3 * 2.0 ** -24, atol=3 * 2.0 ** -24)
    assert batch.adjust(z, out=z).data_ptr() == z.data_ptr()


def test_on_another_stream_and_in_a_graph():
    """Forks, copies, norms with rotation, cuts and logits captured into one graph and replayed with other numbers, against eager calls."""
    rng = np.random.default_rng(12)
    n, pages, width, hq, hkv, hd, rows, vocab = 6, 24, 4, 6, 2, 64, 9, 5000
    q, k, v, pool0 = _rotary_inputs(rng, rows, hq, hkv, hd, "bf16", pages)
    pools0 = torch.stack([pool0, pool0 * 2])
    angles, gain = vf.vf_rotary_table(64, 1e4, 256), 1 + 0.1 * torch.randn(64, device=DEV)
    ints = lambda *m: torch.zeros(m, dtype=torch.int32, device=DEV)  # noqa: E731
    lens, keep, src, dst, tokens, pos, slot, ids = ints(n), ints(n), ints(3), ints(3), ints(3), ints(rows), ints(rows), ints(rows)
    table, shares, free, n_free, pools = ints(n, width), ints(pages), ints(pages), ints(1), pools0.clone()
    kv, kept, mid, left, copies, more, c, m = ints(n), ints(n), ints(1), ints(1), ints(3, 2), ints(n, 2), ints(1), ints(1)
    q_out, z, out = torch.empty_like(q.contiguous()), torch.randn((rows, vocab), device=DEV), torch.zeros((rows, vocab), device=DEV)
    new_table, new_shares, new_free, new_left, moved, moves, t = ints(n, width), ints(30), ints(30), ints(1), ints(pages), ints(pages, 2), ints(1)
    others = torch.zeros((2, 30, 2, hkv, 64 * hd), dtype=q.dtype, device=DEV)
    row_off, penalties = i32([0, 1, 5, 5, 6, 8, 9]), f32([[1.5, 0.1, 0.2]] * n)

    def step():
        vf.vf_pages_fork(src, dst, tokens, lens, free, n_free, table, shares, kv, mid, copies, c)
        vf.vf_pages_copy(pools, copies, c, pools)
        vf.vf_norm_rotary_append(q, k, v, gain, None, EPS, angles, pos, slot, q_out, pools[1])
        vf.vf_logits_adjust(z, row_off, out, penalties, ids.view(1, -1).expand(n, -1).contiguous(), kv, None, ids)
        vf.vf_pages_keep(kv, keep, free, mid, table, shares, kept, left, more, m)
        vf.vf_pages_copy(pools, more, m, pools)
        vf.vf_pages_compact(kept, table, shares, new_table, new_shares, new_free, new_left, moved, moves, t)
        vf.vf_pages_copy(pools, moves, t, others)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    results = (table, shares, free, kv, kept, mid, left, c, m, pools, q_out, out, new_table, new_shares, new_left, moved, t, others)
    for a, f, w in (([100, 0, 0, 64, 0, 7], ([0, 3, 0], [1, 2, 4], [-1, 9, 65]), [-1, 0, -1, 64, 3, 7]),
                    ([0, 200, 0, 0, 0, 0], ([1, 1, 1], [0, 2, 3], [-1, -1, 64]), [70, 70, 70, 1, 0, 0]),
                    ([256, 0, 0, 0, 0, 256], ([0, 5, 9], [3, 1, 2], [255, 256, 1]), [0, 0, -1, 100, -1, 0]),
                    ([100, 0, 0, 64, 0, 7], ([0, 3, 0], [1, 2, 4], [-1, 9, 65]), [-1, 0, -1, 64, 3, 7])):
        tables, at = np.full((n, width), -1), 0
        for b, h in enumerate(a):
            tables[b, :-(-h // 64)] = np.arange(at, at - (-h // 64))
            at -= -h // 64
        found = []
        for eager in (True, False):
            lens.copy_(i32(a)), keep.copy_(i32(w)), table.copy_(i32(tables)), shares.zero_(), pools.copy_(pools0), others.zero_(), out.zero_()
            for to, values in zip((src, dst, tokens), f):
                to.copy_(i32(values))
            free.copy_(i32(list(range(at, pages)) + [0] * at)), n_free.fill_(pages - at)
            pos.copy_(i32(rng.integers(0, 200, rows)) if eager else pos), slot.copy_(i32(64 * (pages - 1) + np.arange(rows)))
            ids.copy_(i32(rng.integers(0, 9, rows)) if eager else ids)
            step() if eager else graph.replay()
            torch.cuda.synchronize()
            found.append([x.clone() for x in results] + [copies[:int(c)].clone(), more[:int(m)].clone(), moves[:int(t)].clone(), new_free[:int(new_left)].clone()])
        for x, y in zip(*found):
            assert torch.equal(x, y)


def test_two_streams_at_once():
    """Two batches on two streams: nothing of a call is shared with another."""
    calls = []
    for seed in range(2):
        g = torch.Generator(device=DEV).manual_seed(seed)
        z = torch.randn((20, 40000), generator=g, device=DEV)
        history = torch.randint(0, 40000, (20, 5000), generator=g, device=DEV, dtype=torch.int32)
        calls.append((z, history, torch.cuda.Stream(), [torch.empty_like(z) for _ in range(2)]))
    args = dict(penalties=f32([[1.2, 0.5, 0.1]] * 20), history_len=i32([5000] * 20))
    offsets = i32(range(21))
    torch.cuda.synchronize()
    for z, history, _, (out, _) in calls:
        vf.vf_logits_adjust(z, offsets, out, history=history, **args)
    torch.cuda.synchronize()
    for _ in range(5):
        for z, history, stream, (_, out) in calls:
            with torch.cuda.stream(stream):
                vf.vf_logits_adjust(z, offsets, out, history=history, **args)
        torch.cuda.synchronize()
        assert all(torch.equal(*outs) for _, _, _, outs in calls)
