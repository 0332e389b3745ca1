"""PackedBatch.keep and release by a request's number from the end, before and after requests share pages; numbers of no request."""
import pytest
import torch

from test_gpu_packed_batch_edges import make, pages_of, step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("forked", [False, True])
def test_requests_from_the_end(forked):
    batch = make(requests=4, pages=12)
    step(batch, [130, 64, 3, 0])
    if forked:
        assert batch.fork([0], [3]) == [True]
    held = list(batch.host_lens)
    assert batch.keep(-4, 70) == 70 and batch.host_lens == [70, *held[1:]]
    assert batch.keep(-2, 3) == 3 and batch.host_lens == [70, *held[1:]]
    batch.release(-3)
    assert batch.host_lens == [70, 0, *held[2:]]
    batch.release(-1)
    assert batch.host_lens == [70, 0, 3, 0] == batch.lens.tolist()
    assert batch.host_free == 12 - 2 - 1 == batch.n_free.item() and pages_of(batch) == list(range(12))


@pytest.mark.parametrize("forked", [False, True])
@pytest.mark.parametrize("request_", [4, -5, 100])
def test_numbers_of_no_request(forked, request_):
    batch = make(requests=4, pages=12)
    step(batch, [130, 64, 3, 0])
    if forked:
        batch.fork([0], [3])
    held = list(batch.host_lens)
    for call in (lambda: batch.keep(request_, 0), lambda: batch.release(request_)):
        with pytest.raises(IndexError):
            call()
    assert batch.host_lens == held == batch.lens.tolist()
    torch.cuda.synchronize()
