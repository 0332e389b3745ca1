"""Generation with penalties, biases and allowed ids: the text is what plain greedy decoding with the same adjustments gives."""
import numpy as np
import pytest

import oracle
from oracle import packed as op
import workloads as wl
from paper_2510_15312_amd.generate import generate
import torch

import paper_2510_15312_amd as vf
from util_gpu import DEV, Pair, f32, gpu_accept, i32, accept_margin_ok

pytestmark = pytest.mark.gpu


def _prompt(cfg):
    rng = np.random.default_rng(1)
    span = rng.integers(0, cfg.vocab, 23).tolist()
    return (span * 9)[:150] + rng.integers(0, cfg.vocab, 13).tolist() + span[:7]


def _grammar(vocab):
    """Ids of the last id's class and the next one; every fourth text may go on as it likes."""
    return lambda text: None if len(text) % 4 == 0 else [v for v in range(vocab) if (v - text[-1]) % 7 in (0, 1)]


KINDS = {"penalties": dict(penalties=(1.3, 0.2, 0.1)), "biases": dict(biases={5: 3.0, 9: 2.5, 100: -float("inf")}),
         "allowed": dict(allowed=True), "all": dict(penalties=(1.1, 0.1, 0.05), biases={5: 1.0}, allowed=True)}


@pytest.mark.parametrize("kind", KINDS)
def test_any_drafts_give_the_text_of_plain_decoding(kind):
    cfg = wl.CONFIGS["tiny_f32"]
    pair, prompt, kw = Pair(cfg, max_rows=128, max_positions=600), _prompt(cfg), dict(KINDS[kind])
    if "allowed" in kw:
        kw["allowed"] = _grammar(cfg.vocab)
    run = lambda **more: generate(pair.model, pair.new_seq(600), prompt, 40, chunk=64, **kw, **more)  # noqa: E731
    plain, _ = run(k=0)
    rng = np.random.default_rng(3)
    assert run(k=12)[0] == plain and run(k=5, drafter=lambda text, k: rng.integers(0, cfg.vocab, k).tolist())[0] == plain
    # drafts that are the text itself are all accepted
    told, stats = run(k=8, drafter=lambda text, k: plain[len(text) - len(prompt):][:k], reuse=False)
    assert told == plain and stats["accepted_drafts"] == stats["drafted"]
    # the same from the oracle's logits, wherever the best id is clear of the next by more than the logits' tolerance
    cache = oracle.KVCache(pair.spec, 600)
    z, text = oracle.prefill(pair.spec, pair.ow, cache, np.asarray(prompt), 128), list(prompt)
    clear = 0
    for t in plain:
        more = dict(penalties=[kw.get("penalties", (1, 0, 0))], history=[text], prompt_len=[len(prompt)], biases=[list(kw.get("biases", {}).items())])
        if "allowed" in kw and (ids := kw["allowed"](text)) is not None:
            more["mask"] = np.isin(np.arange(cfg.vocab), ids)[None]
        y = op.logits_adjust(z[None], [0, 1], **more)[0]
        best, second = np.sort(y)[-1:-3:-1]
        if best - second > 4e-5 * np.abs(z).max():
            assert int(y.argmax()) == t
            clear += 1
        text.append(t)
        z = oracle.forward(pair.spec, pair.ow, cache, [t])[0]
    assert clear > 30


def test_without_adjustments_nothing_changes():
    cfg = wl.CONFIGS["tiny_f32"]
    pair, prompt = Pair(cfg, max_rows=128, max_positions=600), _prompt(cfg)
    texts = [generate(pair.model, pair.new_seq(600), prompt, 30, k=6, chunk=64, **kw)[0] for kw in ({}, dict(penalties=(1.0, 0.0, 0.0)), dict(biases={3: 0.0}),
                                                                                       dict(allowed=lambda text: None))]
    assert all(t == texts[0] for t in texts)


def test_ids_outside_the_vocabulary_are_refused():
    cfg = wl.CONFIGS["tiny_f32"]
    pair = Pair(cfg, max_rows=128, max_positions=600)
    with pytest.raises(ValueError):
        generate(pair.model, pair.new_seq(600), _prompt(cfg), 3, chunk=64, allowed=lambda text: [cfg.vocab])


@pytest.mark.parametrize("mode", ["greedy", "stochastic"])
def test_verify_adjust_accept(mode):
    """The three calls of a step, with masks and penalties: accepted and emitted tokens are what the oracle's rule makes of the
    adjusted logits, and of the allowed ids."""
    cfg = wl.CONFIGS["tiny_f32"]
    pair, prompt, rng = Pair(cfg, max_rows=128, max_positions=600), _prompt(cfg), np.random.default_rng(8)
    seen = 0
    for step in range(6):
        seq = pair.new_seq(600)
        vf.vf_prefill_chunk(pair.model, seq, i32(prompt[:100]))
        vf.vf_prefill_chunk(pair.model, seq, i32(prompt[100:]), sample_first=True)
        _, pending = vf.vf_seq_get_state(seq)
        k = 5
        allowed = rng.random((k + 1, cfg.vocab)) < 0.03
        drafts = [int(rng.choice(np.flatnonzero(allowed[i]))) for i in range(k)]
        tokens, logits = i32([pending] + drafts), torch.empty((k + 1, cfg.vocab), device=DEV)
        vf.vf_verify(pair.model, [seq], tokens, [0, k + 1], logits)
        before = logits.double().cpu().numpy()
        words = torch.as_tensor(np.packbits(allowed, axis=1, bitorder="little").view(np.int32), device=DEV)
        vf.vf_logits_adjust(logits, i32([0, k + 1]), logits, f32([[1.2, 0.3, 0.1]]), i32([prompt]), i32([len(prompt)]), i32([len(prompt)]), tokens, mask=words)
        z = logits.cpu().numpy()
        want = op.logits_adjust(before, [0, k + 1], [(np.float32(1.2), np.float32(0.3), np.float32(0.1))], [prompt], [len(prompt)], [pending] + drafts, mask=allowed)
        assert np.array_equal(np.isneginf(z), ~allowed) and np.allclose(z[allowed], want[allowed], rtol=2.0 ** -21, atol=2.0 ** -21)
        if step % 2:                                                 # drafts that are accepted for a while
            tokens = i32([pending] + [int(v) for v in z[:k].argmax(1)])
            drafts = tokens.tolist()[1:]
        u = rng.random(2 * (k + 1)).astype(np.float32)
        temperature = 0.7
        params = [(vf.VF_GREEDY, 0.0, None, None)] if mode == "greedy" else [(vf.VF_STOCHASTIC, temperature, None, f32(u))]
        n_acc, out, y = gpu_accept(pair, [seq], tokens, [0, k + 1], params, logits)
        a = int(n_acc[0])
        assert allowed[a, out[a]] and all(allowed[i, out[i]] for i in range(a))
        if mode == "greedy":
            want_a, want_out, _ = oracle.greedy_accept(z, drafts)
        else:
            if not accept_margin_ok(z, drafts, mode, None, u, temperature, 1e-9):
                continue
            want_a, want_out, _ = oracle.stochastic_accept(z, drafts, None, u, temperature)
        assert a == want_a and np.array_equal(out[:a + 1], want_out) and np.array_equal(y, z.argmax(1))
        seen += 1
    assert seen >= 4
