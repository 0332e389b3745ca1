"""The binding's packed calls make their tensors' device the current one for the call, as those for norms, pages and logits do (CPU: stand-ins
for tensors)."""
import pytest
import torch

import paper_2510_15312_amd as vf
from paper_2510_15312_amd import binding
from test_more_devices import Sized, current  # noqa: F401
from test_packed_devices import CALLS, F32, reached  # noqa: F401


@pytest.mark.parametrize("call,tensors,more", CALLS)
@pytest.mark.parametrize("device,made", [(1, []), (2, [2]), (0, [0])])
def test_calls(reached, current, call, tensors, more, device, made):  # noqa: F811
    call(**{name: Sized(device, *spec) for name, spec in tensors.items()}, **more)
    assert reached == [call.__name__] and current == made


@pytest.mark.parametrize("device,made", [(1, []), (2, [2])])
def test_the_table_of_angles(reached, current, monkeypatch, device, made):  # noqa: F811
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: Sized(device, F32, *shape))
    assert vf.vf_rotary_table(64, 1e4, 10, device=device).shape == (10, 32, 2)
    assert reached == ["vf_rotary_table"] and current == made


def test_beside_one_device_none_is_asked_for(reached, monkeypatch):  # noqa: F811
    """... not even where a call knows the number of its tensors' device."""
    monkeypatch.setattr(binding, "_device_count", lambda: 1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: pytest.fail("asked for"))
    for call, tensors, more in CALLS:
        call(**{name: Sized(0, *spec) for name, spec in tensors.items()}, **more)
    assert reached == [call.__name__ for call, _, _ in CALLS]


def test_the_current_device(monkeypatch):
    monkeypatch.setattr(binding, "_device_count", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 2)
    assert binding._current_device() == 2
