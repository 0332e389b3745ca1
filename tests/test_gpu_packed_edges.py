"""Attention of packed rows where parts, tiles and page tables end inside one another, against the float64 oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2510_15312_amd as vf
from oracle import packed as op
from paper_2510_15312_amd.packed_batch import PackedBatch
from test_gpu_packed import Packed, _pool_rows
from util_gpu import DEV, i32

pytestmark = pytest.mark.gpu
TILES, TILES_TWO, FEW = 0, 1, 2     # kernels: 128 items a workgroup; the same with two groups of wavefronts; 16 items


def plan(p, max_rows=None, max_keys=None):
    """(kernel, parts, pages a part) that a call takes."""
    (rows, hq, hd), hkv, (n, width) = p.q.shape, p.pool.shape[2], p.table.shape
    max_rows, max_keys = p.max_rows if max_rows is None else max_rows, p.max_keys if max_keys is None else max_keys
    args = vf.vf_packed_args(vf.VF_F32 if p.dt == torch.float32 else vf.VF_BF16, hq, hkv, hd, n, rows, max_rows, max_keys,
                             p.pool.shape[0], width, width, 0.0, hq * hd, hq * hd)
    kernel, parts = C.c_int(), C.c_int()
    assert vf.lib.vf_debug_packed_plan(C.byref(args), C.byref(kernel), C.byref(parts)) == vf.VF_OK
    return kernel.value, parts.value, -(-max(1, min(width, -(-max_keys // 64))) // parts.value)


def check_rows(p, out, b, first, last, present=None, features=slice(None)):
    """Rows first .. last - 1 of sequence b against the oracle, as the last rows of a shorter sequence."""
    rows, n = int(p.row_off[b + 1] - p.row_off[b]), p.kv_len[b]
    end, at = n - (rows - last), slice(int(p.row_off[b]) + first, int(p.row_off[b]) + last)
    part = Packed.__new__(Packed)
    part.hd, part.dt, part.q, part.k, part.v = p.hd, p.dt, p.q[at], [p.k[b][:end]], [p.v[b][:end]]
    part.row_off, part.kv_len = np.array([0, last - first]), [end]
    part.check(out[at], None if present is None else [present[:end]], rows=np.s_[:, :, features])


# ---- records of a row whose heads lie in two tiles of 16 items -----------------------------------------------------

def split_lengths(rows, group, parts, part_pages, most):
    """Lengths (up to most) at which a row has heads in two tiles of 16 items whose last keys lie in different parts."""
    def used(tile, first_pos):
        last = first_pos + min(rows * group - 1, tile * 16 + 15) // group
        return min(parts, -(-(last // 64 + 1) // part_pages))
    return [n for n in range(rows, most + 1)
            if any(used(r * group // 16, n - rows) != used((r * group + group - 1) // 16, n - rows) for r in range(rows))]


@pytest.mark.parametrize("dtype,hq,hkv,hd", [("bf16", 12, 2, 128), ("bf16", 14, 2, 64), ("bf16", 6, 2, 128), ("f32", 6, 2, 64)])
@pytest.mark.parametrize("rows", [17, 33])
def test_rows_in_two_tiles_at_the_end_of_a_part(rows, dtype, hq, hkv, hd):
    probe = Packed([(2048, rows)], hq, hkv, hd, dtype)
    kernel, parts, part_pages = plan(probe)
    assert kernel == FEW and parts > 1
    lengths = split_lengths(rows, hq // hkv, parts, part_pages, 2048)
    assert lengths
    for n in (lengths[0], lengths[len(lengths) // 2], lengths[-1]):
        p = Packed([(n, rows)], hq, hkv, hd, dtype, seed=n)
        p.table = np.pad(p.table, ((0, 0), (0, 32 - p.table.shape[1])), constant_values=-1)   # as wide as the plan's keys
        p.check(p.run(rows, 2048))


def test_rows_in_two_tiles_where_the_bound_of_rows_is_passed():
    """One workgroup takes all tiles of a sequence, one after the other."""
    p = Packed([(1602, 17)], 12, 2, 128, "bf16", seed=17)
    kernel, parts, part_pages = plan(p, 1, 1602)
    assert kernel == FEW and parts > 1
    n = split_lengths(17, 6, parts, part_pages, 2048)[-1]
    p = Packed([(n, 17)], 12, 2, 128, "bf16", seed=18)
    p.table = np.pad(p.table, ((0, 0), (0, 40 - p.table.shape[1])), constant_values=-1)
    assert plan(p, 1, 1602) == (kernel, parts, part_pages)
    p.check(p.run(1, 1602))


def test_drafts_behind_1585_tokens():
    p = Packed([(1602, 17)], 12, 2, 128, "bf16", seed=19)
    assert plan(p) == (FEW, 6, 5)
    p.check(p.run())


# ---- more than 64 pages in a part ------------------------------------------------------------------------------------

def widen(p, pages):
    p.table = np.pad(p.table, ((0, 0), (0, pages - p.table.shape[1])), constant_values=-1)
    return p


def check_around(p, out, b, position, present=None):
    """Rows of sequence b in the tile of 128 items that holds a position: the tile's first, those around the position, the last."""
    rows, group = int(p.row_off[b + 1] - p.row_off[b]), p.q.shape[1] // p.pool.shape[2]
    first_pos = p.kv_len[b] - rows
    tile = (position - first_pos) * group // 128
    first, last = -(-tile * 128 // group), min(rows, (tile + 1) * 128 // group)
    for a, z in ((first, first + 3), (position - first_pos - 1, position - first_pos + 2), (last - 2, last)):
        check_rows(p, out, b, max(a, 0), min(z, rows), present)


@pytest.mark.parametrize("dtype,hq,hkv,hd,kernel,seqs,width,max_keys", [
    ("bf16", 12, 2, 128, TILES_TWO, [(5100, 5000)], 128, 5100), ("bf16", 14, 2, 64, TILES_TWO, [(5100, 5000)], 128, 5100),
    ("bf16", 24, 8, 128, TILES, [(5100, 5000)], 128, 5100), ("bf16", 12, 2, 128, TILES, [(8300, 8100)], 256, 8300),
    ("bf16", 14, 2, 64, TILES_TWO, [(8300, 8100)], 256, 8300),
    ("bf16", 12, 2, 128, TILES_TWO, [(4200 - n % 3, 256) for n in range(15)] + [(4352, 256)], 128, 4352),
    ("bf16", 14, 2, 64, TILES, [(4200, 900)] * 7 + [(4352, 900)], 70, 4352),
    ("f32", 4, 4, 64, TILES, [(5100, 5000)], 128, 64), ("f32", 6, 2, 128, TILES, [(5100, 5000)], 128, 64)])   # in one part: the bound of keys is passed
def test_chunks_that_cross_a_multiple_of_64_pages(dtype, hq, hkv, hd, kernel, seqs, width, max_keys):
    """Tables wider than the sequences, -1 behind their pages."""
    p = widen(Packed(seqs, hq, hkv, hd, dtype, seed=len(seqs)), width)
    assert plan(p, None, max_keys)[:2] == (kernel, 1)
    out = p.run(None, max_keys)
    for b in {0, len(seqs) // 2, len(seqs) - 1}:
        for position in range(4096, p.kv_len[b], 4096):
            check_around(p, out, b, position)
        check_rows(p, out, b, int(p.row_off[b + 1] - p.row_off[b]) - 2, int(p.row_off[b + 1] - p.row_off[b]))


@pytest.mark.parametrize("dtype,hq,hkv,hd,kernel", [("bf16", 12, 2, 128, TILES), ("bf16", 14, 2, 64, TILES_TWO), ("f32", 4, 4, 64, TILES)])
@pytest.mark.parametrize("missing", [[3], [62], [63], [64], [62, 63], [63, 128]])
def test_missing_pages_among_more_than_64(missing, dtype, hq, hkv, hd, kernel):
    """A page that is not there, in front of the 64th or there; entries 64 further on are pages."""
    p = widen(Packed([(8300, 8100)], hq, hkv, hd, dtype, seed=63), 200)
    max_keys = 64 if dtype == "f32" else 8300
    assert plan(p, None, max_keys)[:2] == (kernel, 1)
    p.table[0, missing] = -1
    present = np.ones(8300, bool)
    for page in missing:
        present[page * 64:page * 64 + 64] = False
    out = p.run(None, max_keys)
    for position in (4095, 4160, 8192, 8290):
        check_around(p, out, 0, position, present)


def test_a_chunk_behind_a_chunk_of_a_batch():
    """PackedBatch's tables are as wide as its requests may grow."""
    hq, hkv, hd = 12, 2, 128
    batch = PackedBatch(1, 1, hq, hkv, hd, pool_pages=100, max_tokens=8192, theta=1e4)
    gen = torch.Generator(device=DEV).manual_seed(100)
    for rows in (100, 5000):
        row_off, pos = batch.begin([rows])
        q, k, v = torch.randn((rows, hq + 2 * hkv, hd), generator=gen, device=DEV).to(torch.bfloat16).split((hq, hkv, hkv), 1)
        out = batch.attend(0, q, k, v)
        assert batch.finish() == [True]
    p, t = Packed.__new__(Packed), np.arange(5100)
    p.q = torch.empty_like(q.contiguous())
    vf.vf_rotary_append(q, k, v, batch.angles, pos, torch.full_like(pos, -1), p.q, batch.pools[0])
    slots = 64 * batch.table[0].cpu().numpy()[t // 64] + t % 64
    p.hd, p.dt, p.pool, p.row_off, p.kv_len = hd, torch.bfloat16, batch.pools[0], np.array([0, 5000]), [5100]
    p.k, p.v = ([x.double().cpu().numpy()] for x in _pool_rows(batch.pools[0], i32(slots), hd))
    check_around(p, out, 0, 4096)


# ---- values that are not finite -----------------------------------------------------------------------------------------

MASKED = [("bf16", 4, 64, 1500, 64, TILES), ("bf16", 4, 128, 1500, 64, TILES), ("bf16", 2, 128, 3000, 3000, TILES_TWO), ("f32", 4, 64, 1500, 64, TILES)]


@pytest.mark.parametrize("dtype,heads,hd,rows,max_keys,kernel", MASKED)
def test_a_row_that_is_not_a_number_stays_alone(dtype, heads, hd, rows, max_keys, kernel):
    """Rows 640 to 767 are a tile; those from 704 on see its first page, 640 to 703, whole."""
    p = Packed([(rows, rows)], heads, heads, hd, dtype, seed=rows)
    assert plan(p, None, max_keys)[0] == kernel
    p.q[710] = float("nan")
    out = p.run(None, max_keys)
    assert out[710].isnan().all()
    for first, last in ((640, 643), (670, 673), (700, 710), (711, 722), (733, 739), (765, 770)):
        check_rows(p, out, 0, first, last)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,heads,hd,rows,max_keys,kernel", MASKED)
def test_a_value_that_is_not_finite_stays_in_its_feature(dtype, heads, hd, rows, max_keys, kernel, value):
    p = Packed([(rows, rows)], heads, heads, hd, dtype, seed=rows + 1)
    assert plan(p, None, max_keys)[0] == kernel
    key, feature = 645, 3
    p.pool[int(p.table[0, key // 64]), 1, :, int(op.pool_place(hd)[1][key % 64, feature])] = value
    p.v[0][key, :, feature] = 0                          # the oracle's value where nobody sees it
    out = p.run(None, max_keys)
    sees = torch.arange(rows, device=DEV) >= key
    assert torch.isfinite(out[~sees]).all() and not torch.isfinite(out[sees][:, :, feature]).any()
    out[:, :, feature] = torch.where(sees[:, None], 0, out[:, :, feature])
    for first, last in ((640, 650), (700, 712), (760, 772), (830, 836)):
        check_rows(p, out, 0, first, last, features=[i for i in range(hd) if i != feature])
    check_rows(p, out, 0, 640, 645)


# ---- scores of any size -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("low,high,signs", [(101, 120, (-1,)), (60, 100, (-1, 1)), (26, 40, (-1, 1))])
@pytest.mark.parametrize("dtype,heads,hd,seq,max_keys,kernel,parts", [
    ("bf16", 4, 64, (1500, 1500), 64, TILES, 1), ("bf16", 4, 128, (1500, 1500), 64, TILES, 1), ("bf16", 2, 128, (3000, 3000), 3000, TILES_TWO, 6),
    ("f32", 4, 64, (1500, 1500), 64, TILES, 1), ("bf16", 4, 64, (300, 5), 300, FEW, 1), ("f32", 4, 128, (300, 5), 300, FEW, 1),
    ("bf16", 4, 128, (2048, 3), 2048, FEW, 8)])
def test_attention_of_scores_far_apart(dtype, heads, hd, seq, max_keys, kernel, parts, low, high, signs):
    """Scores of 2^26 to 2^121 whose differences are 2^19 or more, all of them negative or not: a row's result is the mean of
    the values of the keys with its highest score."""
    p = Packed([seq], heads, heads, hd, dtype, seed=low)
    assert plan(p, None, max_keys)[:2] == (kernel, parts)
    n, rows = seq
    rng = np.random.default_rng(high)
    score = (rng.choice(signs, 40) * (1 + rng.integers(0, 128, 40) / 128) * 2.0 ** rng.integers(low, high, 40))[rng.integers(0, 40, n)]
    p.q[:] = 0
    p.q[:, :, 0] = 1
    page, key = i32(p.table[0][np.arange(n) // 64]).long(), i32(np.arange(n) % 64).long()
    for h in range(heads):
        p.pool[page[:, None], 0, h, torch.as_tensor(op.pool_place(hd)[0], device=DEV)[key]] = 0
        p.pool[page, 0, h, torch.as_tensor(op.pool_place(hd)[0][:, 0], device=DEV)[key]] = torch.as_tensor(score, device=DEV).to(p.dt)
    out = p.run(None, max_keys, scale=1.0).double().cpu().numpy()
    sees = np.arange(n) <= n - rows + np.arange(rows)[:, None]
    highest = sees & (score == np.where(sees, score, -np.inf).max(1, keepdims=True))
    weight = highest / highest.sum(1, keepdims=True)
    want, spread = (np.einsum("rt,thd->rhd", weight, x) for x in (p.v[0], np.abs(p.v[0])))
    # the weights are equal and their sums are exact up to rounding: n 2^-24 of the sum of sizes; bfloat16's weights and results 2^-8
    unit = 2.0 ** -8 if dtype == "bf16" else 0.0
    assert (np.abs(out - want) <= (n + 8) * 2.0 ** -23 * spread + unit * (spread + np.abs(want))).all()


# ---- lengths that are none ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,hq,hkv,hd,rows,max_keys,kernel", [
    ("bf16", 4, 4, 64, 1500, 64, TILES), ("bf16", 12, 2, 128, 1500, 64, TILES), ("bf16", 12, 2, 128, 300, 2560, TILES_TWO), ("f32", 4, 4, 64, 1500, 64, TILES),
    ("bf16", 12, 2, 128, 2, 64, FEW), ("bf16", 12, 2, 128, 2, 5000, FEW), ("f32", 4, 2, 64, 9, 64, FEW)])
def test_attention_of_negative_lengths(dtype, hq, hkv, hd, rows, max_keys, kernel):
    """Down to the lowest: rows that see nothing, beside a sequence that stands."""
    p = widen(Packed([(64, rows), (64, rows), (100, min(rows, 100)), (64, rows)], hq, hkv, hd, dtype, seed=64), 40)
    assert plan(p, rows, max_keys)[0] == kernel
    p.kv_len = [-2 ** 31, -1, 100, -2 ** 31 + rows]
    out = p.run(rows, max_keys)
    a, z = int(p.row_off[2]), int(p.row_off[3])
    assert not out[:a].any() and not out[z:].any()
    check_rows(p, out, 2, 0, min(3, z - a))
    check_rows(p, out, 2, max(0, z - a - 3), z - a)
