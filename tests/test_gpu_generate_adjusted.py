"""Generation with penalties, biases and allowed ids: the text is what plain greedy decoding with the same adjustments gives."""
import numpy as np
import pytest

import oracle
from oracle import packed as op
import workloads as wl
from paper_2510_15312_amd.generate import generate
from util_gpu import Pair

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
