"""Which drafts a step of generate takes where only some ids may follow (CPU: nothing is launched)."""
import numpy as np
import pytest

from paper_2510_15312_amd.generate import _Adjust

VOCAB = 70


def _strict(admitted):
    """A grammar with the texts `admitted` {text: ids} that fails on others, and the texts that it was asked about."""
    asked = []

    def allowed(text):
        asked.append(tuple(text))
        return admitted[tuple(text)]
    return allowed, asked


def _make(allowed):
    return _Adjust(None, None, allowed, [5], 10, VOCAB, "cpu")


@pytest.mark.parametrize("admitted,drafts,taken", [
    ({(5,): [1, 2], (5, 1): [3], (5, 1, 3): [69]}, [1, 3], [1, 3]),
    ({(5,): [1, 2], (5, 1): [3]}, [1, 4, 9, 9], [1]),             # 4 is excluded, and with it what stands behind
    ({(5,): [1, 2]}, [0, 1, 2], []),
    ({(5,): []}, [0, 1], []),                                     # nothing is allowed: 0 follows, but no draft behind it is taken
    ({(5,): None, (5, 66): [7], (5, 66, 7): None, (5, 66, 7, 8): [2]}, [66, 7, 8], [66, 7, 8]),
    ({(5,): None, (5, 66): [7]}, [66, 8, 8], [66]),
    ({(5,): [1]}, [VOCAB, 1], []), ({(5,): [1]}, [-1, 1], []), ({(5,): [1]}, [], [])])
def test_drafts_that_are_excluded(admitted, drafts, taken):
    allowed, asked = _strict(admitted)
    a = _make(allowed)
    assert a.admitted([5], drafts) == taken
    assert asked == [(5, *taken[:i]) for i in range(len(taken) + 1)]
    words, rows = a.mask
    bits = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :VOCAB]
    assert len(words) == len(rows) == len(taken) + 1
    for i, row in enumerate(rows):
        ids = admitted[asked[i]]
        assert row == (-1 if ids is None else i)
        assert ids is None or np.flatnonzero(bits[i]).tolist() == sorted(ids)


@pytest.mark.parametrize("ids", [[VOCAB], [-1], [3, 1 << 40]])
def test_ids_outside_the_vocabulary(ids):
    with pytest.raises(ValueError):
        _make(lambda text: ids).admitted([5], [3])


def test_without_a_grammar_all_drafts_are_taken():
    a = _make(None)
    assert a.admitted([5], [1, 2, VOCAB]) == [1, 2, VOCAB] and a.mask is None
