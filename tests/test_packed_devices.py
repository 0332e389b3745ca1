"""The binding's packed calls refuse tensors of different devices, before anything is launched (CPU: stand-ins for tensors)."""
import pytest
import torch

import paper_2510_15312_amd as vf
from paper_2510_15312_amd import binding


class On:
    """What the binding asks of a tensor, on a device that is not here."""
    def __init__(self, device, dtype, *shape):
        self.device, self.dtype, self.shape, self.is_cuda = device, dtype, shape, device >= 0

    def get_device(self):
        return self.device

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def dim(self):
        return len(self.shape)

    def stride(self):
        out = [1]
        for x in reversed(self.shape[1:]):
            out.insert(0, out[0] * x)
        return tuple(out)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


I32, BF16, F32 = torch.int32, torch.bfloat16, torch.float32
ASSIGN = dict(lens=(I32, 2), new=(I32, 2), free_pages=(I32, 9), n_free=(I32, 1), block_table=(I32, 2, 4), row_off=(I32, 3), pos=(I32, 5),
              slot=(I32, 5), kv_len=(I32, 2), n_free_out=(I32, 1))
ROTARY = dict(q=(BF16, 5, 4, 64), k=(BF16, 5, 2, 64), v=(BF16, 5, 2, 64), table=(F32, 10, 32, 2), pos=(I32, 5), slot=(I32, 5),
              q_out=(BF16, 5, 4, 64), pool=(BF16, 3, 2, 2, 4096))
ATTENTION = dict(q=(BF16, 5, 4, 64), pool=(BF16, 3, 2, 2, 4096), block_table=(I32, 2, 4), row_off=(I32, 3), kv_len=(I32, 2),
                 out=(BF16, 5, 4, 64), workspace=(torch.uint8, 1 << 20))
CALLS = [(vf.vf_pages_assign, ASSIGN, {}), (vf.vf_rotary_append, ROTARY, {}), (vf.vf_attention_packed, ATTENTION, dict(max_rows=3, max_keys=200))]


@pytest.fixture
def reached(monkeypatch):
    """The entry points that were called, in place of calling them."""
    names = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: names.append(name) or 0
    monkeypatch.setattr(binding, "lib", Library())
    monkeypatch.setattr(binding, "_stream_of", lambda t: 0)
    monkeypatch.setattr(binding, "_several_devices", lambda: True, raising=False)
    return names


@pytest.mark.parametrize("call,tensors,more", CALLS)
def test_one_device(reached, call, tensors, more):
    call(**{name: On(1, *spec) for name, spec in tensors.items()}, **more)
    assert reached == [call.__name__]


@pytest.mark.parametrize("call,tensors,more,other", [(c, t, m, name) for c, t, m in CALLS for name in t])
@pytest.mark.parametrize("device", [0, -1])
def test_a_tensor_of_another_device(reached, call, tensors, more, other, device):
    args = {name: On(device if name == other else 1, *spec) for name, spec in tensors.items()}
    with pytest.raises(vf.VfError):
        call(**args, **more)
    assert not reached


def test_workspace_size_with_a_table_of_another_device(reached):
    args = [On(1, *ATTENTION["q"]), On(1, *ATTENTION["pool"]), On(0, *ATTENTION["block_table"])]
    with pytest.raises(vf.VfError):
        vf.vf_attention_packed_workspace(*args, 3, 200)
    assert not reached


@pytest.mark.parametrize("call,tensors,more,other", [(c, t, m, name) for c, t, m in CALLS for name in t])
def test_a_tensor_of_the_host_beside_one_device(reached, monkeypatch, call, tensors, more, other):
    monkeypatch.setattr(binding, "_several_devices", lambda: False, raising=False)
    args = {name: On(-1 if name == other else 0, *spec) for name, spec in tensors.items()}
    with pytest.raises(vf.VfError):
        call(**args, **more)
    assert not reached
