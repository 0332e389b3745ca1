"""What the binding hands to vf_logits_adjust (CPU: stand-ins for tensors)."""
import pytest

import paper_2510_15312_amd as vf
from paper_2510_15312_amd import binding
from test_more_devices import BF16, F32, I32, LOGITS, Sized, _tensors, current, reached  # noqa: F401

NAMES = ["args", "logits", "row_off", "out", "penalties", "history", "history_len", "prompt_len", "tokens", "bias_off", "bias_id", "bias", "mask", "mask_row", "stream"]


@pytest.fixture
def handed(reached, current, monkeypatch):  # noqa: F811
    """The arguments of the calls, by name."""
    calls = []

    class Library:
        def vf_logits_adjust(self, *args):
            calls.append(dict(zip(NAMES, args), sizes=args[0]._obj))
            return 0
    monkeypatch.setattr(binding, "lib", Library())
    return calls


class Nowhere(Sized):
    """A tensor without elements, which has no address."""
    def data_ptr(self):
        return 0


@pytest.mark.parametrize("more", [{}, dict(prompt_len=None), dict(history_len=None, prompt_len=None)])
@pytest.mark.parametrize("kind", [Nowhere, Sized])
def test_a_history_of_no_columns_is_none(handed, kind, more):
    vf.vf_logits_adjust(**dict(_tensors(LOGITS, 1), history=kind(1, I32, 3, 0), **more))
    call, = handed
    assert not (call["history"] or call["history_len"] or call["prompt_len"]) and call["penalties"] and call["tokens"]
    assert call["sizes"].max_history == 0


@pytest.mark.parametrize("other", [dict(history_len=Sized(1, I32, 2)), dict(prompt_len=Sized(1, I32, 2)), dict(prompt_len=Sized(0, I32, 3))])
def test_lengths_of_no_columns_are_checked(handed, other):
    with pytest.raises(vf.VfError):
        vf.vf_logits_adjust(**dict(_tensors(LOGITS, 1), history=Nowhere(1, I32, 3, 0), **other))
    assert not handed


def test_a_history_with_columns_is_handed_on(handed):
    vf.vf_logits_adjust(**_tensors(LOGITS, 1))
    call, = handed
    assert call["history"] == call["history_len"] == call["prompt_len"] == 4096 and call["sizes"].max_history == 7


class Apart(Sized):
    """Rows four elements apart."""
    def stride(self):
        return 4, 1


def test_penalties_of_one_sequence_from_a_wider_row(handed):
    """One row is contiguous whatever lies between it and the next."""
    one = _tensors(dict(LOGITS, row_off=(I32, 2), history=(I32, 1, 7), history_len=(I32, 1), prompt_len=(I32, 1)), 1)
    vf.vf_logits_adjust(**dict(one, penalties=Apart(1, F32, 1, 3)))
    assert handed[0]["penalties"] == 4096
    with pytest.raises(vf.VfError):
        vf.vf_logits_adjust(**dict(_tensors(LOGITS, 1), penalties=Apart(1, F32, 3, 3)))
    assert len(handed) == 1
