"""Pins of the packed-batch oracle (CPU): hand-worked page assignments, rotations by other routes, attention against
dense softmax attention, page layout against the formula in include/vf.h."""
import numpy as np
import torch

from oracle import packed as op


def test_pages_worked_by_hand():
    # three requests; free pages 30, 31, 32 with the last taken first
    table = np.array([[5, -1, -1], [6, -1, -1], [-1, -1, -1]])
    t, off, pos, slot, kv, left = op.pages_assign([63, 64, 0], [2, 0, 65], [30, 31, 32], 3, table, 68)
    assert t.tolist() == [[5, 32, -1], [6, -1, -1], [31, 30, -1]]
    assert off.tolist() == [0, 2, 2, 67] and kv.tolist() == [65, 64, 65] and left == 0
    assert pos[:3].tolist() == [63, 64, 0] and slot[:3].tolist() == [5 * 64 + 63, 32 * 64, 31 * 64]
    assert slot[66] == 30 * 64 and (pos[67], slot[67]) == (-1, -1)


def test_pages_refusals_worked_by_hand():
    # one free page: the first request that needs two is refused, the next that needs one comes behind it and is refused
    # too, the last needs none; lengths that are negative or pass the table are refused and take nothing
    table = np.array([[1, -1], [2, -1], [3, -1], [4, -1], [7, -1]])
    t, off, pos, slot, kv, left = op.pages_assign([0, 64, 10, -1, 100], [100, 1, 5, 3, 29], [9], 1, table, 138)
    assert np.array_equal(t, table) and kv.tolist() == [0, 0, 15, 0, 0] and left == 1
    assert off.tolist() == [0, 100, 101, 106, 109, 138]
    assert (pos[:101] == -1).all() and pos[101:106].tolist() == list(range(10, 15)) and (slot[106:] == -1).all()


def test_offsets_stop_at_the_rows():
    _, off, pos, _, _, _ = op.pages_assign([0, 0], [5, 5], [0, 1], 2, np.full((2, 1), -1), 7)
    assert off.tolist() == [0, 5, 7] and pos.tolist() == [0, 1, 2, 3, 4, 0, 1]


def test_rotation_is_complex_multiplication_and_keeps_the_rest():
    rng = np.random.default_rng(1)
    x, table = rng.standard_normal((7, 3, 64)), op.rotary_table(32, 1e4, 50)
    pos = np.array([0, 1, 2, 3, 11, 48, 49])
    turn = np.exp(1j * pos[:, None] * 1e4 ** (-np.arange(16) / 16.0))[:, None]
    y = op.rotate(x, table[pos], True)
    z = (x[..., 0:32:2] + 1j * x[..., 1:32:2]) * turn
    assert np.allclose(y[..., 0:32:2], z.real) and np.allclose(y[..., 1:32:2], z.imag) and np.array_equal(y[..., 32:], x[..., 32:])
    y = op.rotate(x, table[pos], False)
    z = (x[..., :16] + 1j * x[..., 16:32]) * turn
    assert np.allclose(y[..., :16], z.real) and np.allclose(y[..., 16:32], z.imag)


def test_scalings():
    plain = op.rotary_table(64, 1e4, 64)
    assert np.allclose(op.rotary_table(64, 1e4, 256, "positions", 4.0)[::4], plain)     # position 4 t turns as t did
    base = op.rotary_table(64, 1e4, 9, "base", 8.0)
    assert np.allclose(base[:, 0], plain[:9, 0])                                        # the fastest pair is as it was
    assert np.allclose(base[8, -1], plain[1, -1])                                       # the slowest turns 8 times slower
    ramp = op.rotary_table(64, 1e4, 9, "ramp", 8.0, low=1.0, high=4.0, trained=512)
    turns = 512 * 1e4 ** (-np.arange(32) / 32.0) / (2 * np.pi)
    assert np.allclose(ramp[:, turns > 4], plain[:9, turns > 4]) and np.allclose(ramp[8, turns < 1], plain[1, turns < 1])
    assert np.allclose(op.rotary_table(64, 1e4, 9, magnitude=1.5), 1.5 * plain[:9])


def test_places_are_a_permutation():
    for hd in (64, 128):
        for place in op.pool_place(hd):
            assert sorted(place.ravel()) == list(range(64 * hd))


def test_attention_against_dense_softmax():
    rng = np.random.default_rng(2)
    lens, rows = [5, 0, 9], [5, 0, 3]
    q = rng.standard_normal((8, 4, 64))
    k, v = ([rng.standard_normal((n, 2, 64)) for n in lens] for _ in range(2))
    out, spread, _ = op.attention_packed(q, k, v, [0, 5, 5, 8], lens)
    at = 0
    for b, (n, m) in enumerate(zip(lens, rows)):
        if not m:
            continue
        mask = torch.arange(n)[None] <= torch.arange(n - m, n)[:, None]
        kk, vv = (torch.tensor(x[b]).repeat_interleave(2, 1).transpose(0, 1) for x in (k, v))
        want = torch.nn.functional.scaled_dot_product_attention(torch.tensor(q[at:at + m]).transpose(0, 1), kk, vv, attn_mask=mask)
        assert np.allclose(out[at:at + m], want.transpose(0, 1).numpy())
        at += m
    assert (spread >= np.abs(out) - 1e-12).all()


def test_rows_that_see_nothing_are_zero():
    rng = np.random.default_rng(3)
    q, k = rng.standard_normal((6, 2, 64)), [rng.standard_normal((4, 1, 64))]
    out, _, _ = op.attention_packed(q, k, k, [0, 6], [4])
    assert (out[:2] == 0).all() and np.allclose(out[2], k[0][0])          # the third row sees one key
    out, _, _ = op.attention_packed(q, k, k, [0, 6], [4], present=[[False] * 4])
    assert (out == 0).all()
