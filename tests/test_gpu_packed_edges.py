"""Attention of packed rows where parts, tiles and page tables end inside one another, against the float64 oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2510_15312_amd as vf
from test_gpu_packed import Packed
from util_gpu import DEV

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


def check_rows(p, out, b, first, last, present=None):
    """Rows first .. last - 1 of sequence b against the oracle, as the last rows of a shorter sequence."""
    rows, n = int(p.row_off[b + 1] - p.row_off[b]), p.kv_len[b]
    end, at = n - (rows - last), slice(int(p.row_off[b]) + first, int(p.row_off[b]) + last)
    part = Packed.__new__(Packed)
    part.hd, part.dt, part.q, part.k, part.v = p.hd, p.dt, p.q[at], [p.k[b][:end]], [p.v[b][:end]]
    part.row_off, part.kv_len = np.array([0, last - first]), [end]
    part.check(out[at], None if present is None else [present[:end]])


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
