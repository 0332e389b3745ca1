"""vf_logits_adjust refuses results that share memory with the logits without being them (CPU: nothing is launched, every call here has
masks that are refused behind that)."""
import ctypes as C
import random

import pytest

import paper_2510_15312_amd as vf

L, BASE = vf.lib, 1 << 44
F32, BF16 = vf.VF_F32, vf.VF_BF16


def refused(shift, vocab, rows, in_stride, out_stride, dtype=F32):
    """Whether results `shift` bytes behind the logits are refused for shared memory."""
    p = C.c_void_p
    args = vf.vf_logits_args(dtype, 1, rows, vocab, 0, 0, -1, 0, in_stride, out_stride, 0, 0)
    assert L.vf_logits_adjust(C.byref(args), p(BASE), p(4096), p(BASE + shift), *[None] * 8, p(4096), None, None) == vf.VF_ERR_ARG
    assert b"shares memory" in L.vf_last_error() or b"masks" in L.vf_last_error()
    return b"shares memory" in L.vf_last_error()


def share(shift, vocab, rows, in_stride, out_stride, dtype=F32):
    """The same, row by row."""
    es = 4 if dtype == F32 else 2
    a = [(r * in_stride * es, r * in_stride * es + vocab * es) for r in range(rows)]
    b = [(shift + r * out_stride * 4, shift + r * out_stride * 4 + vocab * 4) for r in range(rows)]
    return any(x0 < y1 and y0 < x1 for x0, x1 in a for y0, y1 in b)


@pytest.mark.parametrize("shift,vocab,rows,in_stride,out_stride,dtype,want", [
    (0, 100, 3, 100, 100, F32, False),                  # the logits themselves
    (4, 100, 3, 100, 100, F32, True), (-4, 100, 3, 100, 100, F32, True), (400, 100, 3, 100, 100, F32, True),       # moved by an id, by a row
    (1200, 100, 3, 100, 100, F32, False), (-1200, 100, 3, 100, 100, F32, False), (1196, 100, 3, 100, 100, F32, True), (-1196, 100, 3, 100, 100, F32, True),
    (400, 100, 3, 200, 200, F32, False), (-400, 100, 3, 200, 200, F32, False), (396, 100, 3, 200, 200, F32, True),  # side by side in one matrix
    (404, 100, 3, 201, 201, F32, False), (408, 100, 3, 201, 201, F32, True), (404, 100, 1, 201, 201, F32, False),
    (400, 100, 3, 200, 300, F32, True), (400, 100, 2, 200, 300, F32, False),
    (200, 100, 3, 300, 150, BF16, False), (196, 100, 3, 300, 150, BF16, True), (200, 100, 3, 298, 150, BF16, True), (0, 100, 1, 100, 100, F32, False),
    (4 << 40, 1 << 24, 65536, 1 << 24, 1 << 24, F32, False), ((4 << 40) - 4, 1 << 24, 65536, 1 << 24, 1 << 24, F32, True),
    (4 << 24, 1 << 24, 65536, 1 << 25, 1 << 25, F32, False)])
def test_results_beside_the_logits(shift, vocab, rows, in_stride, out_stride, dtype, want):
    assert refused(shift, vocab, min(rows, vf.VF_PACKED_MAX_ROWS), in_stride, out_stride, dtype) == want


def test_any_layout():
    rng, seen = random.Random(1), set()
    for _ in range(20000):
        dtype, vocab, rows = rng.choice((F32, BF16)), rng.randint(1, 9), rng.randint(1, 6)
        layout = 4 * rng.randint(-120, 120), vocab, rows, vocab + rng.randint(0, 20), vocab + rng.randint(0, 20), dtype
        if layout[0]:
            assert refused(*layout) == share(*layout), layout
            seen.add(share(*layout))
    assert seen == {False, True}
