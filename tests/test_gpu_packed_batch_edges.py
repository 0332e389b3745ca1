"""PackedBatch: calls that it refuses, the bounds it gives, its memory on other streams."""
import pytest
import torch

from paper_2510_15312_amd.packed_batch import PackedBatch
from util_gpu import DEV

pytestmark = pytest.mark.gpu


def make(requests=3, pages=8, tokens=256):
    return PackedBatch(requests, 1, 4, 2, 64, pages, tokens, torch.float32, device=DEV)


def rows_of(n):
    x = torch.randn((n, 8, 64), device=DEV)
    return x[:, :4], x[:, 4:6], x[:, 6:]


def step(batch, new):
    batch.begin(new)
    batch.attend(0, *rows_of(sum(new)))
    return batch.finish()


def pages_of(batch):
    """All pages that a request or the free list holds."""
    held = [p for b, n in enumerate(batch.host_lens) for p in batch.table[b, :-(-n // 64)].tolist()]
    return sorted(held + batch.free[:batch.host_free].tolist())


@pytest.mark.parametrize("new", [[], [1], [1, 1], [1, 1, 1, 1]])
def test_begin_takes_a_number_for_every_request(new):
    batch = make()
    with pytest.raises(ValueError):
        batch.begin(new)
    assert step(batch, [70, 0, 1]) == [True] * 3 and pages_of(batch) == list(range(8))


def test_pages_are_not_given_back_within_a_step():
    batch = make()
    step(batch, [130, 64, 1])
    batch.begin([1, 1, 1])
    for call in (lambda: batch.keep(0, 5), lambda: batch.release(1)):
        with pytest.raises(RuntimeError):
            call()
    batch.attend(0, *rows_of(3))
    assert batch.finish() == [True] * 3
    assert batch.host_lens == [131, 65, 2] and pages_of(batch) == list(range(8)) and batch.host_free == 2
    batch.release(1)
    assert batch.host_lens == [131, 0, 2] and pages_of(batch) == list(range(8)) and batch.host_free == 4
    assert step(batch, [0, 256, 0]) == [True] * 3 and pages_of(batch) == list(range(8)) and batch.host_free == 0


def test_a_step_is_finished_once():
    batch = make()
    for call in (batch.finish, lambda: batch.attend(0, *rows_of(1))):     # no step yet
        with pytest.raises(RuntimeError):
            call()
    step(batch, [130, 64, 1])
    for call in (batch.finish, lambda: batch.attend(0, *rows_of(195))):   # the step is over
        with pytest.raises(RuntimeError):
            call()
    assert step(batch, [63, 65, 0]) == [True] * 3 and batch.host_lens == [193, 129, 1]
    assert pages_of(batch) == list(range(8)) and batch.host_free == 0


def test_a_step_may_begin_again():
    """The step before was given up: nothing of it stays."""
    batch = make()
    step(batch, [60, 0, 0])
    batch.begin([100, 100, 100])
    assert step(batch, [10, 64, 0]) == [True] * 3 and batch.host_lens == [70, 64, 0] and pages_of(batch) == list(range(8))
    batch.begin([100, 100, 100])
    with pytest.raises(ValueError):
        batch.begin([1])
    with pytest.raises(RuntimeError):                                     # no step is open
        batch.finish()
    batch.release(0)
    assert step(batch, [0, 1, 300]) == [True, True, False] and pages_of(batch) == list(range(8)) and batch.host_free == 6


def test_a_step_waits_for_the_device_once():
    """Nothing from begin to finish's copy waits, whatever is still running."""
    batch = make()
    step(batch, [130, 0, 1])
    step(batch, [1, 64, 1])                               # memory and kernels of such a step are there
    rows, before = rows_of(3), torch.cuda.get_sync_debug_mode()
    torch.cuda.set_sync_debug_mode("error")
    try:
        batch.begin([1, 1, 1])
        batch.attend(0, *rows)
    finally:
        torch.cuda.set_sync_debug_mode(before)
    assert batch.finish() == [True] * 3 and batch.host_lens == [132, 65, 3]


def test_numbers_of_tokens_are_those_of_their_begin():
    """Steps given up one after the other, faster than the device takes them: each has its own numbers on their way."""
    batch = make()
    torch.cuda._sleep(20_000_000)
    for i in range(200):
        batch.begin([i % 7, 1 + i % 64, 3])
    batch.begin([130, 5, 64])
    batch.attend(0, *rows_of(199))
    assert batch.row_off.tolist() == [0, 130, 135, 199]
    assert batch.finish() == [True] * 3 and batch.host_lens == [130, 5, 64] and pages_of(batch) == list(range(8))


def test_bounds_are_those_of_the_requests_in_the_step():
    """A long request without tokens in the step does not choose the others' kernel and parts."""
    batch = make(requests=3, pages=40, tokens=2048)
    step(batch, [2000, 10, 0])
    for new, rows, keys in (([0, 1, 0], 1, 11), ([0, 3, 70], 70, 70), ([1, 0, 0], 1, 2001), ([0, 0, 0], 0, 0), ([0, -4, 2], 2, 72)):
        batch.begin(new)
        assert (batch.max_rows, batch.max_keys) == (rows, keys)
        batch.attend(0, *rows_of(sum(max(0, w) for w in new)))
        assert batch.finish() == [w >= 0 for w in new]


def test_memory_of_a_step_waits_for_the_streams_that_use_it():
    """begin on one stream, a first attend on another, a second on a third: what they share is not handed out again before
    they are done with it."""
    batch = make(requests=2, pages=40, tokens=2048)
    step(batch, [2000, 10])
    rows, main = rows_of(2), torch.cuda.current_stream()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    batch.begin([1, 1])
    for before, stream in ((main, one), (one, two)):
        stream.wait_stream(before)
        with torch.cuda.stream(stream):
            torch.cuda._sleep(20_000_000)
            batch.attend(0, *rows)

    def given_again(name, stream):
        """Whether memory of a tensor that the batch lets go is given to others at once."""
        t = getattr(batch, name)
        shape, dtype, first, last = t.shape, t.dtype, t.data_ptr(), t.data_ptr() + t.nbytes
        del t
        setattr(batch, name, None)
        with torch.cuda.stream(stream):
            held = [torch.empty(shape, dtype=dtype, device=DEV) for _ in range(64)]     # (never written)
        return any(x.data_ptr() < last and first < x.data_ptr() + x.nbytes for x in held)
    assert batch.workspace.numel() > 0
    again = [given_again("workspace", one), given_again("pos", main), given_again("slot", main)]
    lens = batch.lens.data_ptr()
    main.wait_stream(two)
    assert batch.finish() == [True] * 2 and batch.lens.tolist() == [2001, 11]
    assert again == [False] * 3 and batch.lens.data_ptr() == lens
