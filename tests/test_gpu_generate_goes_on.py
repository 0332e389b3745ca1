"""generate without a prompt goes on from the sequence's pending token, with adjustments as without."""
import pytest
import torch

import workloads as wl
import paper_2510_15312_amd as vf
from paper_2510_15312_amd.generate import generate
from test_gpu_generate_adjusted import _prompt
from util_gpu import Pair, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("more", [{}, dict(biases={3: 0.0}), dict(penalties=(1.0, 0.0, 0.0)), dict(penalties=(1.5, 0.7, 0.3), biases={9: 1.0}),
                                  dict(allowed=lambda text: [v for v in range(4096) if v % 3 == len(text) % 3])])
def test_without_a_prompt(more):
    cfg = wl.CONFIGS["tiny_f32"]
    pair, prompt = Pair(cfg, max_rows=128, max_positions=600), _prompt(cfg)

    def run(**kw):
        seq = pair.new_seq(600)
        for c0 in range(0, len(prompt), 100):
            vf.vf_prefill_chunk(pair.model, seq, i32(prompt[c0:c0 + 100]), sample_first=c0 + 100 >= len(prompt))
        first = vf.vf_seq_get_state(seq)[1]
        junk = [torch.full((vf.VF_MAX_DRAFTS + 1, cfg.vocab), float(i), device="cuda") for i in range(4)]   # what fresh memory may hold
        for i, t in enumerate(junk):
            t[:, 77 + i] = 1e9
        del junk, t
        text, _ = generate(pair.model, seq, [], 25, **kw, **more)
        assert text[0] == first
        return text
    plain = run(k=0)
    assert run(k=8) == plain
    if more.get("biases") == {3: 0.0} or more.get("penalties") == (1.0, 0.0, 0.0):       # nothing is changed
        assert plain == generate(pair.model, pair.new_seq(600), prompt, 25, k=0, chunk=100)[0]
