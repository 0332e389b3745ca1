"""A step of generate waits for the device once, when it copies what the step has decided; with adjustments too."""
import warnings

import pytest
import torch

import workloads as wl
from paper_2510_15312_amd import binding
from paper_2510_15312_amd.generate import generate
from test_gpu_generate_adjusted import _grammar, _prompt
from util_gpu import Pair

pytestmark = pytest.mark.gpu
CFG = wl.CONFIGS["tiny_f32"]
KINDS = {"plain": {}, "penalties": dict(penalties=(1.3, 0.2, 0.1)), "biases": dict(biases={5: 3.0, 9: 2.5}), "allowed": dict(allowed=_grammar(CFG.vocab)),
         "all": dict(penalties=(1.1, 0.1, 0.05), biases={5: 1.0}, allowed=_grammar(CFG.vocab))}


@pytest.fixture
def between(monkeypatch):
    """Makes everything that would wait between vf_verify and vf_accept an error."""
    before, verify, accept = torch.cuda.get_sync_debug_mode(), binding.vf_verify, binding.vf_accept

    def verified(*args, **kw):
        verify(*args, **kw)
        torch.cuda.set_sync_debug_mode("error")

    def accepted(*args, **kw):
        accept(*args, **kw)
        torch.cuda.set_sync_debug_mode(before)
    monkeypatch.setattr(binding, "vf_verify", verified)
    monkeypatch.setattr(binding, "vf_accept", accepted)
    yield
    torch.cuda.set_sync_debug_mode(before)


@pytest.mark.parametrize("kind", KINDS)
def test_nothing_waits_between_verify_and_accept(between, kind):
    pair, prompt = Pair(CFG, max_rows=128, max_positions=600), _prompt(CFG)
    texts = [generate(pair.model, pair.new_seq(600), prompt, 20, k=k, chunk=64, **KINDS[kind])[0] for k in (0, 6)]
    assert texts[0] == texts[1]


@pytest.mark.parametrize("kind", KINDS)
def test_a_step_waits_once(kind):
    pair, prompt, waits, before = Pair(CFG, max_rows=128, max_positions=600), _prompt(CFG), [], torch.cuda.get_sync_debug_mode()
    for n_new in (10, 35):
        seq = pair.new_seq(600)
        with warnings.catch_warnings(record=True) as seen:
            warnings.simplefilter("always")
            torch.cuda.set_sync_debug_mode("warn")
            try:
                _, stats = generate(pair.model, seq, prompt, n_new, k=0, chunk=64, **KINDS[kind])
            finally:
                torch.cuda.set_sync_debug_mode(before)
        waits.append((stats["steps"], sum("synchroniz" in str(w.message) and "prototype" not in str(w.message) for w in seen)))
    (s0, w0), (s1, w1) = waits
    assert s1 > s0 and w1 - w0 == s1 - s0
