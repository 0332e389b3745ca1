"""The packed-batch operators against their float64 oracle: pages for a step, rotary embedding with the cache write,
attention of packed rows over the page pool."""
import numpy as np
import pytest
import torch

import paper_2510_15312_amd as vf
from oracle import packed as op
from util_gpu import DEV, i32

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- pages -------------------------------------------------------------------------------------

def _assign(lens, new, free, n_free, table, total):
    n = len(lens)
    t, junk = i32(table), -7
    full = lambda k: torch.full((k,), junk, dtype=torch.int32, device=DEV)  # noqa: E731
    row_off, pos, slot, kv, left = full(n + 1), full(total), full(total), full(n), full(1)
    vf.vf_pages_assign(i32(lens), i32(new), i32(free), i32([n_free]), t, row_off, pos, slot, kv, left)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (t, row_off, pos, slot, kv)] + [int(left)]


def _check_pages(lens, new, free, n_free, table, total):
    for got, want in zip(_assign(lens, new, free, n_free, table, total), op.pages_assign(lens, new, free, n_free, table, total)):
        assert np.array_equal(got, want)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("n,most", [(1, 1), (1, 200), (16, 1), (63, 70), (64, 130), (65, 3), (257, 40), (1000, 90), (4096, 9)])
def test_pages(n, most, seed):
    rng = np.random.default_rng(100 * n + seed)
    lens, new = rng.integers(0, 300, n), rng.integers(0, most + 1, n) if most > 1 else np.ones(n, int)
    width = int(max(-(-(lens + new) // 64)) if seed % 2 else 5) or 1      # a narrow table refuses some
    held = np.minimum(-(-lens // 64), width)
    table = np.full((n, width), -1)
    ids = rng.permutation(int(held.sum()) + 3000)
    at = 0
    for b in range(n):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    free = ids[at:]
    wanted = int((-(-(lens + new) // 64) - -(-lens // 64)).sum())
    n_free = min(len(free), [wanted, wanted // 2, 0, 3000, wanted - 1, wanted + 1][seed] if wanted else seed)
    _check_pages(lens, new, free, n_free, table, int(new.sum()))


def test_pages_lengths_that_are_refused():
    table = np.arange(12).reshape(6, 2)
    table[1, 0] = -1                                                     # a page that is missing
    for total in (0, 1, 40, 148, 200):                                   # fewer and more rows than the lengths say
        _check_pages([-3, 10, 128, 0, 127, 64], [5, 4, 1, -2, 1, 2**31 - 1], [50, 51, 52], 3, table, total)
    _check_pages([0, 0], [64, 65], [8], 99, np.full((2, 2), -1), 129)     # a count above the list's room
    _check_pages([0, 0], [64, 65], [8, 9], -1, np.full((2, 2), -1), 129)  # a negative one


def test_pages_table_rows_apart():
    wide = torch.full((3, 10), -1, dtype=torch.int32, device=DEV)
    table, out = wide[:, :2], [torch.zeros(k, dtype=torch.int32, device=DEV) for k in (4, 70, 70, 3, 1)]
    vf.vf_pages_assign(i32([0, 0, 0]), i32([1, 65, 4]), i32([7, 8, 9, 5]), i32([4]), table, *out)
    assert wide.cpu()[:, :2].tolist() == [[5, -1], [9, 8], [7, -1]] and (wide[:, 2:] == -1).all() and int(out[4]) == 0


# ---- rotary embedding ----------------------------------------------------------------------------

@pytest.mark.parametrize("scaling", ["unscaled", "positions", "base", "ramp"])
@pytest.mark.parametrize("dim,positions", [(16, 3), (64, 5000), (128, 70000)])
def test_rotary_table(dim, positions, scaling):
    kw = dict(factor=4.0, low=1.0, high=32.0, trained=4096.0, magnitude=1.25)
    got = vf.vf_rotary_table(dim, 1e6, positions, getattr(vf, "VF_ROTARY_" + scaling.upper()), **kw).cpu().numpy()
    want = op.rotary_table(dim, 1e6, positions, scaling, **kw)
    # float64 angles: position * f is off by a few 2^-53 of itself on either side (7e4 * 2^-50 = 6e-11), the rest is the
    # rounding to float32 of values up to 1.25
    assert np.abs(got - want).max() <= 1.25 * 2.0 ** -24 + 1e-10


def _pool_rows(pool, slots, hd):
    """K and V of the given slots, [n, kv heads, hd], from a pool [pages, 2, kv heads, 64 * hd]."""
    places = [torch.as_tensor(p, device=pool.device) for p in op.pool_place(hd)]
    page, key = slots.long() // 64, slots.long() % 64
    return [torch.gather(pool[page, i], 2, places[i][key][:, None].expand(-1, pool.shape[2], -1)) for i in range(2)]


def _rotary_inputs(rng, rows, hq, hkv, hd, dtype, pages, extra=0):
    gen = torch.Generator(device=DEV).manual_seed(int(rng.integers(1 << 30)))
    qkv = torch.randn((rows, hq + 2 * hkv + extra, hd), generator=gen, device=DEV).to(DTYPES[dtype])
    pool = torch.randn((pages, 2, hkv, 64 * hd), generator=gen, device=DEV).to(DTYPES[dtype])
    return qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:hq + 2 * hkv], pool


def _check_rotary(q, k, v, table, pos, slot, pool, interleaved, in_place=False):
    rows, hq, hd = q.shape
    before, q0 = pool.clone(), q.clone()
    out = q if in_place else torch.full((rows, hq, hd), 7.0, dtype=q.dtype, device=DEV)
    vf.vf_rotary_append(q, k, v, table, i32(pos), i32(slot), out, pool,
                        vf.VF_ROTARY_INTERLEAVED if interleaved else vf.VF_ROTARY_HALF)
    torch.cuda.synchronize()
    at = (pos >= 0) & (pos < table.shape[0])
    stored = at & (slot >= 0) & (slot < 64 * pool.shape[0])
    angles = table.double().cpu().numpy()[np.where(at, pos, 0)]
    # two products and a sum in float32, each rounded once (2^-24 of values up to twice the largest |x|), then the type's rounding
    unit = 2.0 ** -8 if q.dtype == torch.bfloat16 else 0.0
    for got, src in ((out, q0), (None, k)):
        x = src.double().cpu().numpy()
        want = op.rotate(x, angles, interleaved)
        off = 3 * 2.0 ** -24 * 2 * np.abs(x).max()
        bound = off + unit * (np.abs(want) + off)
        if got is not None:
            want[~at] = 0
            assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()
        elif stored.any():
            kept = _pool_rows(pool, i32(slot[stored]), hd)
            assert (np.abs(kept[0].double().cpu().numpy() - want[stored]) <= bound[stored]).all()
            assert torch.equal(kept[1], v[torch.as_tensor(stored, device=DEV)])
    # nothing else of the pool has changed
    page, key = i32(slot[stored]).long() // 64, i32(slot[stored]).long() % 64
    for i, place in enumerate(op.pool_place(hd)):
        at_place = torch.as_tensor(place, device=DEV)[key]
        for h in range(pool.shape[2]):
            before[page[:, None], i, h, at_place] = pool[page[:, None], i, h, at_place]
    assert torch.equal(before, pool)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,hq,hkv,hd,part", [("bf16", 14, 2, 64, 64), ("bf16", 12, 2, 128, 128), ("bf16", 24, 8, 128, 32),
                                                  ("f32", 4, 4, 64, 16), ("f32", 3, 1, 128, 112), ("bf16", 1, 1, 64, 48)])
@pytest.mark.parametrize("rows", [1, 7, 64, 333])
def test_rotary_append(rows, dtype, hq, hkv, hd, part, interleaved):
    rng = np.random.default_rng(rows + part)
    pages = rows // 64 + 9
    q, k, v, pool = _rotary_inputs(rng, rows, hq, hkv, hd, dtype, pages)
    table = vf.vf_rotary_table(part, 1e4, 900)
    # runs of neighbouring slots that start anywhere and end anywhere, and single rows
    pos, slot, start, perm = np.zeros(rows, int), np.zeros(rows, int), 0, rng.permutation(pages)
    p = int(rng.integers(0, 64))
    for r in range(rows):
        pos[r], slot[r] = (p + r) % 900, 64 * perm[(p + r) // 64] + (p + r) % 64
    if rows > 60:
        slot[10:50] = rng.permutation(slot[10:50])                       # no order at all
        slot[[3, 5]], pos[[6, 8, 55]] = [-1, 64 * pages], [-1, 900, 2**31 - 1]
    _check_rotary(q, k, v, table, pos, slot, pool, interleaved)


def test_rotary_in_place_and_wider_rows():
    rng = np.random.default_rng(5)
    for dtype in DTYPES:
        q, k, v, pool = _rotary_inputs(rng, 41, 6, 2, 64, dtype, 2, extra=3)
        _check_rotary(q, k, v, vf.vf_rotary_table(64, 1e4, 99), np.arange(41) + 20, np.arange(41) + 30, pool, False, in_place=True)


def test_rotary_non_finite_rows_stay_alone():
    rng = np.random.default_rng(6)
    q, k, v, pool = _rotary_inputs(rng, 16, 4, 2, 64, "bf16", 1)
    q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    q[3], k[3], v[3] = float("nan"), float("inf"), float("nan")
    out = torch.empty_like(q)
    vf.vf_rotary_append(q, k, v, vf.vf_rotary_table(64, 1e4, 16), i32(range(16)), i32(range(16)), out, pool)
    bad = torch.arange(16, device=DEV) == 3
    kept = _pool_rows(pool, i32(range(16)), 64)
    for x in (out, *kept):
        assert torch.isfinite(x[~bad]).all() and not torch.isfinite(x[bad]).any()


# ---- attention ---------------------------------------------------------------------------------

class Packed:
    """A pool, block tables of random pages and the same keys and values per sequence for the oracle."""

    def __init__(self, seqs, hq, hkv, hd, dtype, seed=0, std=1.5, spare=3, garbage=float("nan"), pool=None, ids=None):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.seqs, self.hd, self.dt = seqs, hd, DTYPES[dtype]
        need = [-(-max(n, 0) // 64) for n, _ in seqs]
        self.pool = torch.full((sum(need) + spare, 2, hkv, 64 * hd), garbage, dtype=self.dt, device=DEV) if pool is None else pool
        ids = rng.permutation(self.pool.shape[0])[:sum(need)] if ids is None else ids
        width = max(1, max(need))
        self.table = np.full((len(seqs), width), -1, np.int64)
        self.k, self.v, at = [], [], 0
        places = [torch.as_tensor(p, device=DEV) for p in op.pool_place(hd)]
        for b, (n, _) in enumerate(seqs):
            self.table[b, :need[b]] = ids[at:at + need[b]]
            at += need[b]
            kv = (torch.randn((2, n, hkv, hd), generator=gen, device=DEV) * std).to(self.dt)
            t = torch.arange(n, device=DEV)
            page = torch.as_tensor(self.table[b], device=DEV)[t // 64]
            for i in range(2):
                for h in range(hkv):
                    self.pool[page[:, None], i, h, places[i][t % 64]] = kv[i, :, h]
            self.k.append(kv[0].double().cpu().numpy())
            self.v.append(kv[1].double().cpu().numpy())
        self.row_off = np.concatenate([[0], np.cumsum([m for _, m in seqs])])
        self.kv_len = [n for n, _ in seqs]
        rows = int(self.row_off[-1])
        self.q = (torch.randn((rows, hq, hd), generator=gen, device=DEV) * std).to(self.dt)
        self.max_rows, self.max_keys = max(m for _, m in seqs), max(n for n, _ in seqs)

    def run(self, max_rows=None, max_keys=None, out=None, scale=0.0, q=None):
        q = self.q if q is None else q
        out = torch.full_like(self.q, 7.0) if out is None else out
        bounds = (self.max_rows if max_rows is None else max_rows, self.max_keys if max_keys is None else max_keys)
        table = i32(self.table)
        ws = vf.vf_attention_packed_workspace(q, self.pool, table, *bounds)
        ws.fill_(0xff)
        vf.vf_attention_packed(q, self.pool, table, i32(self.row_off), i32(self.kv_len), out, *bounds, ws, scale)
        torch.cuda.synchronize()
        return out

    def check(self, out, present=None, scale=None, rows=slice(None)):
        want, spread, size = op.attention_packed(self.q.double().cpu().numpy(), self.k, self.v, self.row_off, self.kv_len, scale, present)
        got = out.double().cpu().numpy()
        keys, hd = max(self.kv_len + [1]), self.hd
        # Scores: a sum of hd float32 products, off by hd 2^-24 of the sum of their sizes, scaled (two roundings) and taken from
        # the maximum (one): (hd + 4) 2^-24 size, twice (the maximum's own error cancels, the split's merges do not), and the
        # exponential's 2^-22.  A weight is off by that share of itself.  Sums over the keys: keys 2^-24 of the sum of sizes, for
        # the weights and for the products.  bfloat16: weights and result are rounded to 2^-8 of themselves (7 stored bits).
        share = 2 * (hd + 4) * 2.0 ** -24 * size + 2.0 ** -21 + 2 * (keys + 8) * 2.0 ** -24
        unit = 2.0 ** -8 if self.dt == torch.bfloat16 else 0.0
        bound = (share * 2 + unit) * spread + (unit + 2.0 ** -23) * np.abs(want) + 1e-30
        bad = ~(np.abs(got - want) <= 1.01 * bound)
        assert not bad[rows].any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])
        return want


SHAPES = [("bf16", 14, 2, 64), ("bf16", 12, 2, 128), ("bf16", 6, 2, 128), ("bf16", 16, 1, 64), ("bf16", 5, 5, 128),
          ("f32", 4, 4, 64), ("f32", 6, 3, 128), ("f32", 9, 1, 64)]
BATCHES = {
    "one_key": [(1, 1)],
    "page_edges": [(63, 1), (64, 1), (65, 1), (128, 1), (1, 1), (127, 1)],
    "prompts": [(1, 1), (64, 64), (65, 65), (17, 17), (130, 130)],
    "drafts": [(90, 33), (33, 33), (300, 2), (64, 17), (129, 8)],
    "mixed": [(257, 1), (40, 40), (0, 0), (200, 100), (5, 0), (66, 3)],
    "nothing_seen": [(0, 3), (2, 5), (0, 0), (70, 75), (0, 1)],
    "long": [(1500, 1), (700, 4)],
}


@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("dtype,hq,hkv,hd", SHAPES)
def test_attention(dtype, hq, hkv, hd, batch):
    p = Packed(BATCHES[batch], hq, hkv, hd, dtype, seed=len(batch))
    p.check(p.run())


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 12, 2, 128), ("bf16", 14, 2, 64), ("f32", 4, 2, 64)])
def test_attention_bounds_of_the_host_do_not_decide_the_result(dtype, hq, hkv, hd):
    """Loose bounds, tight ones and ones that are passed: other kernels and splits, the same sums."""
    p = Packed([(300, 1), (70, 70), (150, 20), (0, 2)], hq, hkv, hd, dtype, seed=4)
    for max_rows, max_keys in ((1, 1), (4, 100), (33, 300), (93, 5000), (2000, 100000), (0, 0)):
        p.check(p.run(max_rows, max_keys))


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_attention_many_sequences(dtype):
    rng = np.random.default_rng(8)
    seqs = [(int(n), int(min(n, m))) for n, m in zip(rng.integers(0, 90, 300), rng.choice([0, 1, 1, 2, 9], 300))]
    p = Packed(seqs, 4, 2, 64, dtype, seed=8)
    p.check(p.run())


@pytest.mark.parametrize("sequences", [9, 70])
@pytest.mark.parametrize("dtype,hkv", [("bf16", 2), ("f32", 7)])
def test_attention_more_tiles_than_compute_units(dtype, hkv, sequences):
    rng = np.random.default_rng(sequences)
    rows = rng.integers(0, 7000 // sequences, sequences)
    p = Packed([(int(m + rng.choice([0, 1, 90])), int(m)) for m in rows], 14, hkv, 64, dtype, seed=sequences)
    assert sum(-(-int(m) * (14 // hkv) // 128) for m in rows) * hkv > 256
    p.check(p.run())


@pytest.mark.parametrize("dtype,hq,hkv,hd,sequences,keys", [("bf16", 12, 2, 128, 150, 200), ("bf16", 24, 8, 128, 30, 1500), ("f32", 4, 4, 128, 70, 150),
                                                            ("f32", 4, 4, 64, 40, 1200), ("bf16", 14, 2, 64, 150, 300)])
def test_attention_more_single_tokens_than_compute_units(dtype, hq, hkv, hd, sequences, keys):
    rng = np.random.default_rng(sequences)
    p = Packed([(int(n), 1) for n in rng.integers(0, keys, sequences)], hq, hkv, hd, dtype, seed=sequences)
    p.check(p.run())
    p.check(p.run(max_keys=50 * keys))                        # in parts, wherever they end


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_attention_keys_a_row_does_not_see_add_nothing(dtype, rows):
    """The last key is infinite, then NaN: only the last row sees it."""
    for value in (float("inf"), float("nan"), -float("inf")):
        for what in (0, 1):
            p = Packed([(70, rows), (30, min(rows, 30))], 4, 2, 64, dtype, seed=3)
            page, key = int(p.table[0, 69 // 64]), 69 % 64
            place = torch.as_tensor(op.pool_place(64)[what][key], device=DEV)
            p.pool[page, what][:, place] = value
            out = p.run()
            p.k[0][69], p.v[0][69] = 0, 0            # the oracle's rows before the last do not see it either
            p.check(out, rows=np.arange(len(p.q)) != rows - 1)
            if what or value != -value:
                assert not torch.isfinite(out[rows - 1]).all()


def test_attention_pages_that_are_not_there():
    for bad in (-1, 10**6, 2**31 - 1):
        p = Packed([(200, 30), (100, 1), (64, 2)], 4, 2, 64, "bf16", seed=5)
        pages = p.table.copy()
        p.table[0, 1], p.table[1, 0], p.table[2, 0] = bad, bad, bad
        present = [np.ones(n, bool) for n in p.kv_len]
        present[0][64:128], present[1][:64], present[2][:] = False, False, False
        p.check(p.run(), present)
        assert pages.shape == p.table.shape


def test_attention_offsets_and_lengths_out_of_range():
    """Offsets beyond the rows, falling offsets, a length beyond the table: in bounds, and rows outside are not written."""
    p = Packed([(64, 5), (64, 5), (64, 5)], 4, 2, 64, "bf16", seed=9)
    p.row_off, p.kv_len = np.array([2, 7, 400, 12]), [64, 64, 70]
    out = p.run()
    assert (out[:2] == 7).all() and torch.isfinite(out).all()


def test_attention_strides_and_scale():
    p = Packed([(100, 50), (80, 1)], 6, 2, 64, "bf16", seed=6)
    wide_q, wide_o = (torch.full((51, 10, 64), 3.0, dtype=p.dt, device=DEV) for _ in range(2))
    wide_q[:, 2:8] = p.q
    p.run(q=wide_q[:, 2:8], out=wide_o[:, 1:7], scale=0.3)
    p.check(wide_o[:, 1:7], scale=np.float64(np.float32(0.3)))
    assert (wide_o[:, 0] == 3).all() and (wide_o[:, 7:] == 3).all()


def test_attention_large_scores():
    """Scores of hundreds: the running maximum moves by more than the exponent's range."""
    for dtype in DTYPES:
        p = Packed([(400, 130), (500, 1)], 4, 2, 64, dtype, seed=7, std=9.0)
        p.check(p.run())


def test_attention_pool_beyond_four_gigabytes():
    pages = 40000                                                         # 2.6 G elements of 2 bytes
    pool = torch.empty((pages, 2, 4, 64 * 128), dtype=torch.bfloat16, device=DEV)
    assert pool.numel() > 1 << 31
    p = Packed([(300, 20), (129, 129), (70, 1)], 8, 4, 128, "bf16", seed=11, pool=pool,
               ids=np.array([39999, 0, 39990, 32768, 16384, 39991, 32767, 1, 39992, 39993]))
    p.check(p.run())
    q, k, v, _ = _rotary_inputs(np.random.default_rng(1), 9, 8, 4, 128, "bf16", 1)
    slot = np.arange(9) + 64 * 39998 + 3
    vf.vf_rotary_append(q, k, v, vf.vf_rotary_table(128, 1e4, 9), i32(range(9)), i32(slot), torch.empty_like(q.contiguous()), pool)
    kept = _pool_rows(pool[39998:], i32(np.arange(9) + 3), 128)
    assert torch.equal(kept[1], v)


def test_packed_on_another_stream_and_in_a_graph():
    """The three operators captured into one graph and replayed with other lengths, against eager calls."""
    lens0, new0 = np.array([100, 0, 63, 10]), np.array([1, 70, 2, 1])
    hq, hkv, hd, total, width = 6, 2, 64, 74, 4
    rng = np.random.default_rng(12)
    q, k, v, pool0 = _rotary_inputs(rng, total, hq, hkv, hd, "bf16", 16)
    angles = vf.vf_rotary_table(64, 1e4, 256)
    table0 = np.full((4, width), -1)
    table0[0, :2], table0[2, 0], table0[3, 0] = [0, 1], 2, 3
    ints = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    lens, new, free, n_free = i32(lens0), i32(new0), i32(range(4, 16)), i32([12])
    table, row_off, pos, slot, kv_len, left = i32(table0), ints(5), ints(total), ints(total), ints(4), ints(1)
    pool, q_out, out = pool0.clone(), torch.empty_like(q.contiguous()), torch.zeros((total, hq, hd), dtype=q.dtype, device=DEV)
    ws = vf.vf_attention_packed_workspace(q_out, pool, table, total, 256)

    def step():
        vf.vf_pages_assign(lens, new, free, n_free, table, row_off, pos, slot, kv_len, left)
        vf.vf_rotary_append(q, k, v, angles, pos, slot, q_out, pool)
        vf.vf_attention_packed(q_out, pool, table, row_off, kv_len, out, total, 256, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for a, b in ((lens0, new0), ([5, 60, 0, 128], [3, 1, 69, 1]), ([1, 1, 1, 1], [64, 1, 8, 1]), (lens0, new0)):
        tables = np.full((4, width), -1)
        at = 0
        for s, n in enumerate(a):
            tables[s, :-(-n // 64)] = np.arange(at, at - (-n // 64))
            at += -(-n // 64)
        results = []
        for eager in (True, False):
            lens.copy_(i32(a)), new.copy_(i32(b)), table.copy_(i32(tables)), pool.copy_(pool0), out.zero_()
            free.copy_(i32(np.arange(4, 16)[::-1].copy()) if at <= 4 else i32(range(4, 16)))
            step() if eager else graph.replay()
            torch.cuda.synchronize()
            results.append([x.clone() for x in (table, row_off, pos, slot, kv_len, left, pool, q_out, out)])
        for x, y in zip(*results):
            assert torch.equal(x, y)


def test_the_binding_refuses_other_tensors():
    """Types, shapes and strides that the C entry points cannot see."""
    p = Packed([(70, 3), (5, 5)], 6, 2, 64, "bf16")
    table, row_off, kv_len, out = i32(p.table), i32(p.row_off), i32(p.kv_len), torch.zeros_like(p.q)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=DEV)
    good = dict(q=p.q, pool=p.pool, block_table=table, row_off=row_off, kv_len=kv_len, out=out, max_rows=5, max_keys=70, workspace=ws)
    vf.vf_attention_packed(**good)
    wrong = [("q", p.q.float()), ("q", p.q[:, :5]), ("q", p.q.cpu()), ("q", p.q.transpose(0, 1).contiguous().transpose(0, 1)),
             ("pool", p.pool.float()), ("pool", p.pool[:, :1]), ("pool", p.pool.transpose(1, 2)), ("pool", p.pool.cpu()),
             ("block_table", table.long()), ("block_table", table[0]), ("block_table", table.t()), ("block_table", table.cpu()),
             ("row_off", row_off[:2]), ("row_off", row_off.long()), ("kv_len", kv_len[:1]), ("kv_len", i32([[1, 2], [3, 4]]).t()[0]),
             ("out", out[:7]), ("out", out.float()), ("out", out[:, :, :32]), ("workspace", ws.float()),
             ("workspace", ws[:1].expand(1 << 20)), ("workspace", ws.cpu())]
    for name, value in wrong:
        with pytest.raises(vf.VfError):
            vf.vf_attention_packed(**{**good, name: value})
    k, angles, pos, slot = p.q[:, :2], vf.vf_rotary_table(64, 1e4, 100), i32(range(8)), i32(range(8))
    good = dict(q=p.q, k=k, v=k, table=angles, pos=pos, slot=slot, q_out=out, pool=p.pool)
    vf.vf_rotary_append(**good)
    for name, value in [("k", k.float()), ("v", k[:7]), ("v", p.q[:, :3]), ("table", angles.double()), ("table", angles[:, :, :1]),
                        ("table", angles.transpose(0, 1)), ("pos", pos[:7]), ("slot", slot.long()), ("q_out", out.transpose(0, 1)),
                        ("pool", p.pool[:, :, :, :64])]:
        with pytest.raises(vf.VfError):
            vf.vf_rotary_append(**{**good, name: value})
    lens = dict(lens=i32([0]), new=i32([5]), free_pages=i32([0, 1]), n_free=i32([2]), block_table=i32([[-1, -1]]), row_off=i32([0, 0]),
                pos=i32([0] * 5), slot=i32([0] * 5), kv_len=i32([0]), n_free_out=i32([0]))
    vf.vf_pages_assign(**lens)
    for name, value in [("lens", i32([])), ("new", lens["new"].long()), ("free_pages", lens["free_pages"].float()), ("n_free", i32([])),
                        ("row_off", i32([0])), ("slot", i32([0] * 4)), ("kv_len", lens["kv_len"].cpu()), ("block_table", i32([-1]))]:
        with pytest.raises(vf.VfError):
            vf.vf_pages_assign(**{**lens, name: value})


# ---- together with the rest of the framework ---------------------------------------------------

@pytest.mark.parametrize("dtype", list(DTYPES))
def test_the_pool_is_the_models_pool(dtype):
    """What vf_rotary_append stores is what vf_kv_read returns, in the layer it was given."""
    cfg = vf.make_config(3, 256, 4, 2, 64, 512, 4096, dtype, 1e4, 1e-6, 64, 512)
    gen = torch.Generator(device=DEV).manual_seed(1)
    mat = lambda *s: (torch.randn(s, generator=gen, device=DEV) * 0.02).to(DTYPES[dtype])  # noqa: E731
    ones = torch.ones(256, device=DEV)
    w = {"embed": mat(4096, 256), "final_norm": ones, "layers": [
        {"attn_norm": ones, "ffn_norm": ones, "wq": mat(256, 256), "wk": mat(128, 256), "wv": mat(128, 256), "wo": mat(256, 256),
         "w_gate": mat(512, 256), "w_up": mat(512, 256), "w_down": mat(256, 512)} for _ in range(3)]}
    model = vf.vf_model_create(cfg, w, DEV)
    memory = torch.zeros(vf.vf_kv_bytes(model, 64, 5), dtype=torch.uint8, device=DEV)
    table = i32([[4, 1, 2]])
    seq = vf.vf_seq_create(model, 192, memory, table[0], DEV)
    q, k, v, _ = _rotary_inputs(np.random.default_rng(2), 150, 4, 2, 64, dtype, 1)
    out, (row_off, pos, slot, kv_len, left) = torch.empty_like(q.contiguous()), [
        torch.zeros(n, dtype=torch.int32, device=DEV) for n in (2, 150, 150, 1, 1)]
    vf.vf_pages_assign(i32([0]), i32([150]), i32([2, 1, 4]), i32([3]), table, row_off, pos, slot, kv_len, left)
    assert table.cpu().tolist() == [[4, 1, 2]]
    vf.vf_rotary_append(q, k, v, vf.vf_rotary_table(64, 1e4, 512), pos, slot, out, vf.kv_layer(model, memory, 1))
    vf.vf_seq_set_len(seq, 150)
    kk, vv = vf.vf_kv_read(model, seq, 1, 0, 150)
    want = op.rotate(k.double().cpu().numpy(), op.rotary_table(64, 1e4, 150), False)
    assert torch.equal(vv, v.float())
    assert np.abs(kk.double().cpu().numpy() - want).max() <= np.abs(want).max() * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -21)
    for layer in (0, 2):
        kk, vv = vf.vf_kv_read(model, seq, layer, 0, 150)
        assert not kk.any() and not vv.any()
