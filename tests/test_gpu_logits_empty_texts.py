"""vf_logits_adjust where no sequence has a text yet: a history of no columns."""
import numpy as np
import pytest
import torch

import paper_2510_15312_amd as vf
from oracle import packed as op
from util_gpu import DEV, f32, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [False, True])
@pytest.mark.parametrize("prompts", [False, True])
@pytest.mark.parametrize("view", [False, True])
def test_a_history_of_no_columns(view, prompts, tokens):
    n, vocab, off = 3, 1000, [0, 2, 2, 5]
    z = torch.randn((5, vocab), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    out = torch.empty_like(z)
    history = i32(np.arange(3 * 7).reshape(3, 7))[:, :0] if view else torch.empty((n, 0), dtype=torch.int32, device=DEV)
    ids, penalties = [4, 5, 6, 6, 999], [(1.5, 0.25, 0.125), (2.0, 1.0, 1.0), (0.5, -0.5, 0.25)]
    vf.vf_logits_adjust(z, i32(off), out, f32(penalties), history, i32([0, 3, -1]), i32([0, 2, 1]) if prompts else None, i32(ids) if tokens else None)
    want = op.logits_adjust(z.double().cpu().numpy(), off, penalties, [[]] * n, [0] * n if prompts else None, ids if tokens else None)
    # a quotient or product, alpha + beta n, a difference: each rounds once
    assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -24 * (4 * np.abs(z.double().cpu().numpy()) * 2 + 4)).all()


def test_a_prompt_without_a_history_is_refused():
    z = torch.zeros((1, 8), device=DEV)
    with pytest.raises(vf.VfError):
        vf.vf_logits_adjust(z, i32([0, 1]), z, f32([[1.5, 0, 0]]), prompt_len=i32([0]))
