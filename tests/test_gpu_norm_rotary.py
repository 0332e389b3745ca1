"""vf_norm_rotary_append against the float64 oracle: norms of the heads, rotation, the write to the cache."""
import numpy as np
import pytest
import torch

import paper_2510_15312_amd as vf
from oracle import packed as op
from test_gpu_packed import _pool_rows, _rotary_inputs
from util_gpu import DEV, i32

pytestmark = pytest.mark.gpu
EPS = 1e-6


def _bounds(x, want, gain, hd, dtype):
    """What float32 may be off by.  The sum of hd squares: products and sums are rounded, so it is off by at most
    (hd + 1) 2^-24 of itself; the mean and eps add 2; a square root halves that; root, reciprocal and the two products with scale and gain
    add 2^-24 each (a division and a root are off by at most 2.5 units here).  The rotation's products and sum are off by 3 * 2^-24 of a
    pair's size, the angles are given.  Then the type's rounding."""
    u = 2.0 ** -24
    size = np.abs(op.norm_heads(x, gain, EPS))
    pair = np.broadcast_to(size.max(-1, keepdims=True), size.shape)      # a value's partner is at most this
    off = ((hd + 3) / 2 + 2 * 2.5 + 2) * u * 2 * pair + 3 * u * 2 * pair
    return off + (2.0 ** -8 if dtype == "bf16" else 0.0) * (np.abs(want) + off) + 1e-37


def _check(q, k, v, gains, table, pos, slot, pool, interleaved, dtype, in_place=False, eps=EPS):
    rows, hq, hd = q.shape
    before, q0 = pool.clone(), q.clone()
    out = q if in_place else torch.full((rows, hq, hd), 7.0, dtype=q.dtype, device=DEV)
    vf.vf_norm_rotary_append(q, k, v, *gains, eps, table, i32(pos), i32(slot), out, pool,
                             vf.VF_ROTARY_INTERLEAVED if interleaved else vf.VF_ROTARY_HALF)
    torch.cuda.synchronize()
    at = (pos >= 0) & (pos < table.shape[0])
    stored = at & (slot >= 0) & (slot < 64 * pool.shape[0])
    angles = table.double().cpu().numpy()[np.where(at, pos, 0)]
    gains = [None if g is None else g.double().cpu().numpy() for g in gains]
    for src, gain in zip((q0, k), gains):
        x = src.double().cpu().numpy()
        want = op.rotate(op.norm_heads(x, gain, eps), angles, interleaved)
        bound = _bounds(x, want, gain, hd, dtype)
        if src is q0:
            want[~at] = 0
            assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
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


def _gains(kind, hq, hkv, hd, seed=3):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if kind == "none":
        return None, None
    if kind == "q":
        return 1 + 0.3 * torch.randn(hd, generator=gen, device=DEV), None
    return [1 + 0.3 * torch.randn((h, hd) if kind == "heads" else (hd,), generator=gen, device=DEV) for h in (hq, hkv)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,hq,hkv,hd,part,kind", [
    ("bf16", 14, 2, 64, 64, "shared"), ("bf16", 12, 2, 128, 128, "heads"), ("bf16", 24, 8, 128, 32, "shared"), ("f32", 4, 4, 64, 16, "heads"),
    ("f32", 3, 1, 128, 112, "none"), ("bf16", 1, 1, 64, 48, "q"), ("bf16", 33, 9, 64, 32, "heads"), ("f32", 7, 7, 128, 64, "q")])
@pytest.mark.parametrize("rows", [1, 7, 64, 333])
def test_norm_rotary_append(rows, dtype, hq, hkv, hd, part, kind, interleaved):
    rng = np.random.default_rng(rows + part)
    pages = rows // 64 + 9
    q, k, v, pool = _rotary_inputs(rng, rows, hq, hkv, hd, dtype, pages)
    table = vf.vf_rotary_table(part, 1e4, 900)
    pos, slot, perm = np.zeros(rows, int), np.zeros(rows, int), rng.permutation(pages)
    p = int(rng.integers(0, 64))
    for r in range(rows):
        pos[r], slot[r] = (p + r) % 900, 64 * perm[(p + r) // 64] + (p + r) % 64
    _check(q, k, v, _gains(kind, hq, hkv, hd), table, pos, slot, pool, interleaved, dtype)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows,hkv", [(2100, 8), (9000, 2)])
def test_many_rows_in_place(rows, hkv, hd):
    """Enough rows for several heads a thread, v in tiles, rows that are not stored and positions outside the table among them."""
    rng = np.random.default_rng(rows)
    pages = rows // 64 + 2
    q, k, v, pool = _rotary_inputs(rng, rows, 9, hkv, hd, "bf16", pages)
    table = vf.vf_rotary_table(hd // 2, 1e4, rows + 80)
    pos, slot = np.arange(rows) + 33, np.arange(rows) + 33
    for i in range(0, rows, 97):
        pos[i] = [-1, rows + 80, 5][i % 3]
    for i in range(5, rows, 131):
        slot[i] = [-1, 64 * pages][i % 2]
    _check(q, k, v, _gains("shared", 9, hkv, hd), table, pos, slot, pool, False, "bf16", in_place=True)


def test_heads_of_zeros_and_small_ones():
    """eps is what a head of zeros is divided by; a head far below it too."""
    rows, hq, hkv, hd = 5, 3, 2, 64
    q, k, v, pool = _rotary_inputs(np.random.default_rng(1), rows, hq, hkv, hd, "f32", 3)
    q[0], q[1], k[2] = 0, q[1] * 1e-12, 0
    q[3] *= 1e15
    table = vf.vf_rotary_table(64, 1e4, 100)
    _check(q, k, v, _gains("shared", hq, hkv, hd), table, np.arange(rows), np.arange(rows), pool, False, "f32")
    assert torch.isfinite(pool).all()


def test_not_finite_values_stay_in_their_head():
    rows, hq, hkv, hd = 3, 4, 4, 128
    q, k, v, pool = _rotary_inputs(np.random.default_rng(1), rows, hq, hkv, hd, "bf16", 1)
    q[1, 2, 5], k[2, 1, 100] = float("nan"), float("inf")
    out = torch.empty_like(q.contiguous())
    vf.vf_norm_rotary_append(q, k, v, None, None, EPS, vf.vf_rotary_table(128, 1e4, 8), i32([0, 1, 2]), i32([3, 4, 5]), out, pool)
    bad = ~torch.isfinite(out).all(-1)
    assert bad.nonzero().tolist() == [[1, 2]]
    kept = _pool_rows(pool, i32([3, 4, 5]), hd)
    assert (~torch.isfinite(kept[0]).all(-1)).nonzero().tolist() == [[2, 1]] and torch.equal(kept[1], v)


def test_without_rotation_left_it_is_the_norm_alone():
    """Position 0 turns nothing: the oracle's norm, and vf_rotary_append on it is the identity."""
    q, k, v, pool = _rotary_inputs(np.random.default_rng(2), 9, 2, 2, 64, "f32", 1)
    out, gains = torch.empty_like(q.contiguous()), _gains("heads", 2, 2, 64)
    vf.vf_norm_rotary_append(q, k, v, *gains, EPS, vf.vf_rotary_table(64, 1e4, 1), i32([0] * 9), i32(np.arange(9)), out, pool)
    want = op.norm_heads(q.double().cpu().numpy(), gains[0].double().cpu().numpy(), EPS)
    assert np.allclose(out.double().cpu().numpy(), want, rtol=64 * 2.0 ** -24, atol=0)


def test_no_rows():
    q, k, v, pool = _rotary_inputs(np.random.default_rng(2), 0, 2, 2, 64, "f32", 1)
    vf.vf_norm_rotary_append(q, k, v, None, None, EPS, vf.vf_rotary_table(64, 1e4, 1), i32([]), i32([]), q.contiguous(), pool)
