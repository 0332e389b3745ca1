"""The binding's calls for norms with rotation, pages and logits refuse tensors of different devices, before anything is launched (CPU:
stand-ins for tensors)."""
import pytest
import torch

import paper_2510_15312_amd as vf
from paper_2510_15312_amd import binding
from test_packed_devices import BF16, F32, I32, ROTARY, On, reached  # noqa: F401


class Sized(On):
    def element_size(self):
        return {BF16: 2, F32: 4, I32: 4}[self.dtype]


@pytest.fixture
def current(monkeypatch):
    """The current device is 1; the devices that were made current for a call."""
    made = []
    monkeypatch.setattr(binding, "_current_device", lambda: 1)

    class Device:
        def __init__(self, number):
            self.number = number

        def __enter__(self):
            made.append(self.number)

        def __exit__(self, *args):
            pass
    monkeypatch.setattr(torch.cuda, "device", Device)
    return made


NORM = dict(ROTARY, q_gain=(F32, 64), k_gain=(F32, 2, 64))
FORK = dict(src=(I32, 2), dst=(I32, 2), tokens=(I32, 2), lens=(I32, 3), free_pages=(I32, 9), n_free=(I32, 1), block_table=(I32, 3, 4), shares=(I32, 9),
            kv_len=(I32, 3), n_free_out=(I32, 1), copies=(I32, 2, 2), n_copies=(I32, 1))
KEEP = dict(lens=(I32, 3), keep=(I32, 3), free_pages=(I32, 9), n_free=(I32, 1), block_table=(I32, 3, 4), shares=(I32, 9), kv_len=(I32, 3),
            n_free_out=(I32, 1), copies=(I32, 3, 2), n_copies=(I32, 1))
COMPACT = dict(lens=(I32, 3), block_table=(I32, 3, 4), shares=(I32, 9), table_out=(I32, 3, 4), shares_out=(I32, 5), free_out=(I32, 5), n_free_out=(I32, 1),
               moved=(I32, 9), copies=(I32, 9, 2), n_copies=(I32, 1))
COPY = dict(pools=(BF16, 2, 9, 2, 2, 4096), copies=(I32, 3, 2), n_copies=(I32, 1), to=(BF16, 2, 5, 2, 2, 4096))
LOGITS = dict(logits=(F32, 5, 100), row_off=(I32, 4), out=(F32, 5, 100), penalties=(F32, 3, 3), history=(I32, 3, 7), history_len=(I32, 3), prompt_len=(I32, 3),
              tokens=(I32, 5), mask=(I32, 6, 4), mask_row=(I32, 5))
CALLS = [(vf.vf_norm_rotary_append, NORM, dict(eps=1e-6)), (vf.vf_pages_fork, FORK, {}), (vf.vf_pages_keep, KEEP, {}), (vf.vf_pages_compact, COMPACT, {}),
         (vf.vf_pages_copy, COPY, {}), (vf.vf_logits_adjust, LOGITS, {})]
BIASES = ((I32, 4), (I32, 6), (F32, 6))


def _tensors(tensors, device, other=None, there=None):
    return {name: Sized(there if name == other else device, *spec) for name, spec in tensors.items()}


@pytest.mark.parametrize("call,tensors,more", CALLS)
def test_one_device(reached, current, call, tensors, more):  # noqa: F811
    call(**_tensors(tensors, 1), **more)
    assert reached == [call.__name__] and not current


@pytest.mark.parametrize("call,tensors,more", CALLS)
def test_a_device_that_is_not_the_current_one(reached, current, call, tensors, more):  # noqa: F811
    call(**_tensors(tensors, 2), **more)
    assert reached == [call.__name__] and current == [2]


@pytest.mark.parametrize("call,tensors,more,other", [(c, t, m, name) for c, t, m in CALLS for name in t])
@pytest.mark.parametrize("device", [0, -1])
def test_a_tensor_of_another_device(reached, call, tensors, more, other, device):  # noqa: F811
    with pytest.raises(vf.VfError):
        call(**_tensors(tensors, 1, other, device), **more)
    assert not reached


@pytest.mark.parametrize("other", [None, 0, 1, 2])
def test_biases(reached, current, other):  # noqa: F811
    biases = tuple(Sized(0 if i == other else 1, *spec) for i, spec in enumerate(BIASES))
    if other is None:
        vf.vf_logits_adjust(**_tensors(LOGITS, 1), biases=biases)
        assert reached == ["vf_logits_adjust"]
        return
    with pytest.raises(vf.VfError):
        vf.vf_logits_adjust(**_tensors(LOGITS, 1), biases=biases)
    assert not reached


WRONG = [  # (call, tensors, more, argument, another type or shape)
    (0, "q_gain", (BF16, 64)), (0, "q_gain", (F32, 2, 64)), (0, "k_gain", (F32, 4, 64)), (0, "k_gain", (F32, 128)), (0, "pos", (I32, 4)), (0, "k", (F32, 5, 2, 64)),
    (1, "dst", (I32, 1)), (1, "tokens", (F32, 2)), (1, "kv_len", (I32, 2)), (1, "copies", (I32, 1, 2)), (1, "block_table", (I32, 12)), (1, "shares", (F32, 9)),
    (1, "shares", (I32, 0)), (2, "keep", (I32, 2)), (2, "copies", (I32, 2, 2)), (2, "free_pages", (torch.int64, 9)),
    (3, "table_out", (I32, 3, 5)), (3, "table_out", (I32, 2, 4)), (3, "free_out", (I32, 4)), (3, "moved", (I32, 8)), (3, "copies", (I32, 4, 2)),
    (4, "to", (BF16, 1, 5, 2, 2, 4096)), (4, "to", (BF16, 2, 5, 2, 1, 4096)), (4, "to", (F32, 2, 5, 2, 2, 2048)), (4, "pools", (BF16, 9, 2)), (4, "copies", (F32, 3, 2)),
    (5, "logits", (F32, 500)), (5, "logits", (torch.float16, 5, 100)), (5, "out", (BF16, 5, 100)), (5, "out", (F32, 4, 100)), (5, "penalties", (F32, 3, 2)),
    (5, "penalties", (F32, 2, 3)), (5, "history", (I32, 2, 7)), (5, "history", (torch.int64, 3, 7)), (5, "tokens", (I32, 4)), (5, "mask", (I32, 6, 3)),
    (5, "mask_row", (I32, 4)), (5, "history_len", (I32, 2)), (5, "row_off", (F32, 4))]


@pytest.mark.parametrize("which,other,spec", WRONG)
def test_other_types_and_shapes(reached, which, other, spec):  # noqa: F811
    call, tensors, more = CALLS[which]
    with pytest.raises(vf.VfError):
        call(**_tensors(dict(tensors, **{other: spec}), 1), **more)
    assert not reached


def test_fewer_masks_than_rows(reached, current):  # noqa: F811
    args = _tensors(dict(LOGITS, mask=(I32, 4, 4)), 1)
    vf.vf_logits_adjust(**args)
    with pytest.raises(vf.VfError):
        vf.vf_logits_adjust(**dict(args, mask_row=None))
    assert reached == ["vf_logits_adjust"]


WIDE = 1 << 32      # sizes of which 32 bits would keep what looks right
TOO_LARGE = [
    (1, dict(free_pages=(I32, WIDE + 9))), (1, dict(shares=(I32, WIDE + 9))), (2, dict(free_pages=(I32, WIDE + 9))),
    (3, dict(shares_out=(I32, WIDE + 5), free_out=(I32, WIDE + 5), copies=(I32, 9, 2))),
    (4, dict(copies=(I32, WIDE, 2))), (4, dict(pools=(BF16, 2, WIDE + 9, 2, 2, 4096))), (4, dict(to=(BF16, 2, WIDE + 5, 2, 2, 4096))),
    (5, dict(logits=(F32, 5, WIDE + 100), out=(F32, 5, WIDE + 100), mask=(I32, 6, WIDE))), (5, dict(history=(I32, 3, WIDE + 7))),
    (5, dict(logits=(F32, WIDE + 5, 100), out=(F32, WIDE + 5, 100), tokens=(I32, WIDE + 5), mask_row=(I32, WIDE + 5)))]


@pytest.mark.parametrize("which,specs", TOO_LARGE)
def test_sizes_past_32_bits(reached, current, which, specs):  # noqa: F811
    call, tensors, more = CALLS[which]
    with pytest.raises(vf.VfError):
        call(**_tensors(dict(tensors, **specs), 1), **more)
    assert not reached
