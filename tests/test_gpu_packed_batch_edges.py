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
