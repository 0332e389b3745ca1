"""Forks, tokens that stay, compaction and copies of pages against the oracle: whole numbers and copies, so equal."""
import numpy as np
import pytest
import torch

import paper_2510_15312_amd as vf
from oracle import packed as op
from util_gpu import DEV, i32

pytestmark = pytest.mark.gpu
JUNK = -7


def _full(*shape):
    return torch.full(shape, JUNK, dtype=torch.int32, device=DEV)


def _list(copies, n):
    return [tuple(p) for p in copies[:int(n)].tolist()]


def fork(src, dst, tokens, lens, free, n_free, table, shares):
    t, s, kv, left, copies, n = i32(table), i32(shares), _full(len(lens)), _full(1), _full(max(len(src), 1), 2), _full(1)
    vf.vf_pages_fork(i32(src), i32(dst), i32(tokens), i32(lens), i32(free), i32([n_free]), t, s, kv, left, copies, n)
    torch.cuda.synchronize()
    assert (copies[int(n):] == JUNK).all()
    return t.cpu().numpy(), s.cpu().numpy(), kv.cpu().numpy(), _list(copies, n), int(left)


def keep(lens, kept, free, n_free, table, shares):
    t, s, f, kv, left, copies, n = i32(table), i32(shares), i32(free), _full(len(lens)), _full(1), _full(len(lens), 2), _full(1)
    vf.vf_pages_keep(i32(lens), i32(kept), f, i32([n_free]), t, s, kv, left, copies, n)
    torch.cuda.synchronize()
    assert (copies[int(n):] == JUNK).all()
    return t.cpu().numpy(), s.cpu().numpy(), kv.cpu().numpy(), _list(copies, n), f[:int(left)].tolist()


def compact(lens, table, shares, room, in_place=False):
    t = i32(table)
    out = t if in_place else _full(*t.shape)
    s, f, left, moved, copies, n = _full(room), _full(room), _full(1), _full(len(shares)), _full(min(len(shares), room), 2), _full(1)
    vf.vf_pages_compact(i32(lens), t, i32(shares), out, s, f, left, moved, copies, n)
    torch.cuda.synchronize()
    assert (f[int(left):] == JUNK).all()
    return out.cpu().numpy(), s.cpu().numpy(), f[:int(left)].tolist(), moved.cpu().numpy(), _list(copies, n)


def same(got, want):
    for g, w in zip(got, want):
        assert np.array_equal(g, w), (g, w)


class Batch:
    """Lengths, tables, counts and free list of a batch whose requests share what forks left them."""

    def __init__(self, rng, n, most, spare, width=None):
        self.lens = rng.integers(0, most + 1, n)
        self.lens[rng.random(n) < 0.4] = 0                                       # places for forks
        self.width = width or int(-(-most // 64)) + 1
        held = -(-self.lens // 64)
        ids = rng.permutation(max(1, int(held.sum()) + spare))                    # (a pool has a page)
        self.table, at = np.full((n, self.width), -1), 0
        for b in range(n):
            self.table[b, :held[b]] = ids[at:at + held[b]]
            at += held[b]
        self.shares = np.zeros(len(ids), int)
        self.free = np.concatenate([ids[at:], np.full(at, -1)])                  # room for all pages
        self.n_free = len(ids) - at

    def owners(self):
        """Every page is held as often as its count says, or is free once."""
        held = np.zeros(len(self.shares), int)
        for b, n in enumerate(self.lens):
            for p in self.table[b, :-(-n // 64)]:
                held[p] += 1
        free = [int(p) for p in self.free[:self.n_free]]
        assert len(set(free)) == len(free) and not held[free].any()
        assert (held[held > 0] == self.shares[held > 0] + 1).all() and (held > 0).sum() + len(free) == len(self.shares)
        assert not self.shares[held == 0].any()

    def fork(self, src, dst, tokens):
        got = fork(src, dst, tokens, self.lens, self.free, self.n_free, self.table, self.shares)
        same(got, op.pages_fork(src, dst, tokens, self.lens, self.free, self.n_free, self.table, self.shares))
        self.table, self.shares, self.lens, _, self.n_free = got
        self.owners()

    def keep(self, kept):
        got = keep(self.lens, kept, self.free, self.n_free, self.table, self.shares)
        same(got, op.pages_keep(self.lens, kept, self.free, self.n_free, self.table, self.shares))
        self.table, self.shares, self.lens, _, free = got
        self.free[:len(free)], self.n_free = free, len(free)
        self.owners()

    def compact(self, spare):
        room = int((self.shares >= 0).sum()) - self.n_free + spare
        got = compact(self.lens, self.table, self.shares, max(room, 1))
        same(got, op.pages_compact(self.lens, self.table, self.shares, max(room, 1)))
        self.table, self.shares, free, _, _ = got
        self.free, self.n_free = np.array(free + [-1] * (len(self.shares) - len(free))), len(free)
        self.owners()


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("n,most", [(2, 1), (5, 64), (16, 700), (70, 200), (300, 130), (1500, 70), (4096, 65)])
def test_a_batch_branches_and_is_cut(n, most, seed):
    rng = np.random.default_rng(1000 * n + seed)
    b = Batch(rng, n, most, spare=[0, n // 3, n, 3 * n][seed])
    b.owners()
    for step in range(3):
        empty, full = np.flatnonzero(b.lens == 0), np.flatnonzero(b.lens > 0)
        if len(full) and len(empty):
            k = int(rng.integers(1, len(empty) + 1))
            dst = rng.permutation(empty)[:k]
            src = rng.choice(full, k) if step else np.full(k, full[0])           # all of one, then of any
            b.fork(src, dst, np.where(rng.random(k) < 0.5, -1, rng.integers(0, most + 9, k)))
        kept = np.where(rng.random(n) < 0.4, -1, (b.lens * rng.random(n)).astype(int))
        kept[rng.random(n) < 0.2] = 0
        if step == 1:
            kept = np.minimum(b.lens, 70)                                        # many cut inside the same pages
        b.keep(kept)
        if step == 1:
            b.compact(int(rng.integers(0, 9)))
    b.keep(np.zeros(n, int))
    assert b.n_free == len(b.shares) and not b.lens.any()


def test_forks_that_are_left_out():
    table = np.full((6, 3), -1)
    table[0, :3], table[1, 0] = [4, 5, 6], 7
    lens, shares, free = [150, 3, 0, 0, 0, -5], np.zeros(10, int), [8, 9]
    args = lens, free, 2, table, shares
    for src, dst, tokens in [([-1, 6, 0, 0], [2, 2, -1, 6], [-1] * 4),            # no such sequence
                             ([0, 1], [1, 0], [-1, -1]),                          # dst holds tokens
                             ([0, 1, 0], [2, 2, 3], [64, -1, 63]),                # the same dst twice
                             ([6, 0], [2, 2], [-1, -1]),                          # the first that names it counts, also where it is left out
                             ([2, 0, 3], [3, 2, 4], [-1, 70, -1]),                # a src that is filled by the same call was empty
                             ([2, 5], [2, 5], [-1, -1]),                          # itself
                             ([0, 0, 0], [2, 3, 4], [149, 128, 1]),               # no page for the last
                             ([0, 0, 1], [5, 2, 3], [0, 1 << 30, 2]), ([], [], [])]:
        same(fork(src, dst, tokens, *args), op.pages_fork(src, dst, tokens, *args))
    for n_free in (-3, 0, 1, 99):
        args = lens, free, n_free, table, shares
        same(fork([0, 0, 0], [4, 3, 2], [65, 100, 2], *args), op.pages_fork([0, 0, 0], [4, 3, 2], [65, 100, 2], *args))


def test_tables_with_pages_that_are_not_there():
    table = np.array([[0, -1, 9, 2], [-1, -1, -1, -1], [3, 99, 1, 7], [-1] * 4])
    lens, shares, free = [250, 0, 1 << 20, 0], [0] * 9, [4, 5, 6, 8, 0, 0, 0, 0, 0]    # a length past the table
    for tokens in ([-1, -1], [100, 70], [150, 255], [64, 256]):
        args = [0, 2], [1, 3], tokens, lens, free, 4, table, shares
        same(fork(*args), op.pages_fork(*args))
    for kept in ([0, 0, 0, 0], [70, -1, 100, 5], [130, 0, 64, -1], [-1, -1, 255, 0], [300, 1, 1 << 21, 1]):
        args = lens, kept, free, 4, table, shares
        same(keep(*args), op.pages_keep(*args))
    for room in (1, 3, 9, 40):
        same(compact(lens, table, shares, room), op.pages_compact(lens, table, shares, room))


def test_a_page_that_all_holders_give_back_at_once():
    """Three requests on the same pages: released together, one after the other's cut, all cut inside one page."""
    table = np.array([[3, 1, 2], [3, 1, 5], [3, 1, 6], [0, -1, -1]])
    lens, shares, free = [150, 140, 130, 10], [0, 2, 0, 2, 0, 0, 0], [4, 9, 9, 9, 9, 9, 9]
    for kept in ([0, 0, 0, 0], [0, 0, 0, -1], [70, 70, 70, -1], [100, 0, 70, 3], [0, 128, 65, -1], [1, 2, 3, 4], [64, 64, 1, -1], [-1, 100, -1, -1]):
        for n_free in (0, 1):
            args = lens, kept, free, n_free, table, shares
            same(keep(*args), op.pages_keep(*args))


def test_a_page_dropped_more_often_than_it_is_shared():
    """A table that names a page twice without a count: the page is free once."""
    args = [128, 64], [0, 0], [7, 0, 0, 0], 1, np.array([[2, 2], [2, -1]]), [0] * 4
    same(keep(*args), op.pages_keep(*args))


def test_a_free_list_without_room_loses_pages():
    args = [256], [0], [7, 0, 0], 1, np.array([[1, 2, 3, 4]]), [0] * 8
    same(keep(*args), op.pages_keep(*args))


def test_many_entries_at_once():
    """More entries than a pass of the one workgroup, half of them shared."""
    n, pages = 260, 100
    table = np.arange(n * pages).reshape(n, pages)
    table[1::2, :99] = table[0::2, :99]
    shares = np.zeros(n * pages, int)
    shares[table[0::2, :99].ravel()] = 1
    free = np.full(n * pages, -1)
    lens = np.full(n, 64 * pages)
    rng = np.random.default_rng(5)
    for kept in (np.zeros(n, int), rng.integers(0, 64 * pages, n), np.where(np.arange(n) % 2, 0, -1)):
        args = lens, kept, free, 0, table, shares
        same(keep(*args), op.pages_keep(*args))
    for in_place in (False, True):
        same(compact(lens, table, shares, n * pages, in_place), op.pages_compact(lens, table, shares, n * pages))
    args = [0] * 200, np.arange(n, n + 200), [-1] * 200, np.append(lens, [0] * 200), [5], 1, np.append(table, np.full((200, pages), -1), 0), shares
    same(fork(*args), op.pages_fork(*args))


def test_a_large_pool():
    """More pages than a word of bits for every thread."""
    rng, pool = np.random.default_rng(9), 200_003
    n, width = 300, 500
    lens = rng.integers(0, 64 * width, n)
    held = -(-lens // 64)
    ids = rng.permutation(pool)[:held.sum()]
    table, at = np.full((n, width), -1), 0
    for b in range(n):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    table[7, :held[7]][:20], shares = table[8, :held[8]][:20], np.zeros(pool, int)
    shares[table[8, :20]] = 1
    for room in (pool, int(held.sum()) - 30):
        same(compact(lens, table, shares, room), op.pages_compact(lens, table, shares, room))
    free = np.full(pool, -1)
    kept = rng.integers(0, 64 * width, n)
    args = lens, kept, free, 0, table, shares
    same(keep(*args), op.pages_keep(*args))
    with pytest.raises(vf.VfError):
        compact(lens, table, np.zeros(vf.VF_PAGES_MAX_POOL + 1, int), 5)


def test_table_rows_apart():
    wide = torch.full((4, 9), JUNK, dtype=torch.int32, device=DEV)
    table = wide[:, 2:5]
    table.copy_(i32([[3, 1, -1], [-1, -1, -1], [2, -1, -1], [-1, -1, -1]]))
    shares, free = i32([0] * 6), i32([0, 4, 5, 0, 0, 0])
    lens, kv, kv2, left, left2, copies, n = i32([100, 0, 5, 0]), _full(4), _full(4), _full(1), _full(1), _full(4, 2), _full(1)
    vf.vf_pages_fork(i32([0, 2]), i32([1, 3]), i32([-1, -1]), lens, free, i32([3]), table, shares, kv, left, copies, n)
    assert table.tolist() == [[3, 1, -1], [3, 5, -1], [2, -1, -1], [4, -1, -1]] and kv.tolist() == [100, 100, 5, 5] and left.tolist() == [1]
    out, moved = torch.full((4, 8), JUNK, dtype=torch.int32, device=DEV), _full(6)
    vf.vf_pages_compact(kv, table, shares, out[:, 3:6], _full(5), _full(5), left2, moved, _full(5, 2), n)
    assert out[:, 3:6].tolist() == [[2, 0, -1], [2, 4, -1], [1, -1, -1], [3, -1, -1]] and moved.tolist() == [-1, 0, 1, 2, 3, 4] and left2.tolist() == [0]
    vf.vf_pages_keep(kv, i32([0, 64, -1, 2]), free, left, table, shares, kv2, left2, copies, n)
    assert table.tolist() == [[-1, -1, -1], [3, -1, -1], [2, -1, -1], [4, -1, -1]] and kv2.tolist() == [0, 64, 5, 2]
    assert (wide[:, :2] == JUNK).all() and (wide[:, 5:] == JUNK).all() and (out[:, :3] == JUNK).all() and (out[:, 6:] == JUNK).all()
    assert free[:int(left2)].tolist() == [0, 1, 5]


# ---- copies --------------------------------------------------------------------------------------

@pytest.mark.parametrize("layers,hkv,hd,dtype", [(1, 1, 64, torch.bfloat16), (3, 2, 128, torch.bfloat16), (28, 2, 64, torch.bfloat16), (2, 5, 128, torch.float32)])
@pytest.mark.parametrize("n", [0, 1, 13])
def test_copies(n, layers, hkv, hd, dtype):
    gen, rng = torch.Generator(device=DEV).manual_seed(n), np.random.default_rng(n)
    pools = torch.randn((layers, 40, 2, hkv, 64 * hd), generator=gen, device=DEV).to(dtype)
    pairs = rng.permutation(40)[:2 * n].reshape(-1, 2)
    listed = i32(np.concatenate([pairs, [[0, 1]] * 4]))                          # entries behind n_copies are not read
    want = pools.clone()
    if n:
        want[:, pairs[:, 1]] = pools[:, pairs[:, 0]]
    vf.vf_pages_copy(pools, listed, i32([n]), pools)
    assert torch.equal(pools, want)
    other = torch.full((layers + 1, 50, 2, hkv, 64 * hd), 7.0, device=DEV, dtype=dtype)
    want = other.clone()
    if n:
        want[1:, pairs[:, 1]] = pools[:, pairs[:, 0]]
    vf.vf_pages_copy(pools, listed, i32([n]), other[1:])
    assert torch.equal(other, want)
    vf.vf_pages_copy(pools[0], listed, i32([n]), other[0])
    if n:
        want[0, pairs[:, 1]] = pools[0, pairs[:, 0]]
    assert torch.equal(other, want)


@pytest.mark.parametrize("shape", [(2, 1, 24), (2, 3, 4104), (2, 1, 2048), (2, 5, 4100)])
def test_pages_of_other_sizes(shape):
    """Pages that are no multiple of what a workgroup moves at a time; a view of some layers of a wider pool."""
    pools = torch.randn((4, 11, *shape), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    want = pools.clone()
    want[1:3, [0, 10]] = pools[1:3, [5, 3]]
    vf.vf_pages_copy(pools[1:3], i32([[5, 0], [3, 10]]), i32([2]), pools[1:3])
    assert torch.equal(pools, want)
    with pytest.raises(vf.VfError):
        vf.vf_pages_copy(pools.transpose(0, 1), i32([[3, 0]]), i32([1]), pools.transpose(0, 1))
    with pytest.raises(vf.VfError):
        vf.vf_pages_copy(pools[..., :-1], i32([[5, 0]]), i32([1]), pools[..., :-1])


def test_copies_that_are_left_out():
    pools = torch.arange(4.0, device=DEV)[None, :, None, None, None].expand(2, 4, 2, 1, 4096).contiguous()
    other = torch.full((2, 3, 2, 1, 4096), 9.0, device=DEV)
    vf.vf_pages_copy(pools, i32([[-1, 0], [4, 1], [3, 3], [3, -1], [2, 2], [1, 0]]), i32([99]), other)     # a number past the list's room
    assert [other[:, p].unique().tolist() for p in range(3)] == [[1.0], [9.0], [2.0]]
    vf.vf_pages_copy(pools, i32([[1, 1]]), i32([-4]), other)
    assert other[:, 1].unique().tolist() == [9.0]


def test_a_pool_past_32_bits():
    """Layers and pages more than 2^31 elements and bytes from the start."""
    pools = torch.empty((2, 5000, 2, 8, 64 * 128), dtype=torch.float32, device=DEV)      # 2.6e9 bytes a layer
    pools[0, 4999], pools[1, 4999], pools[:, 7] = 4.0, 5.0, 0.0
    vf.vf_pages_copy(pools, i32([[4999, 7]]), i32([1]), pools)
    assert [pools[layer, 7].unique().tolist() for layer in range(2)] == [[4.0], [5.0]]
    vf.vf_pages_copy(pools, i32([[7, 4998]]), i32([1]), pools)
    assert [pools[layer, 4998].unique().tolist() for layer in range(2)] == [[4.0], [5.0]]
