"""generate with a grammar that knows only its own texts: whatever the drafts, it is asked about no others, and the text is that of
plain decoding."""
import numpy as np
import pytest

import workloads as wl
from paper_2510_15312_amd.generate import generate
from test_gpu_generate_adjusted import _prompt
from util_gpu import Pair

pytestmark = pytest.mark.gpu


class Outside(Exception):
    pass


def _automaton(vocab, start):
    """States 0 .. 4 behind the first `start` ids; in state s an id v may follow with v % 5 in (s, s + 1), and leads to state v % 5.  In state 4
    only two ids may follow.  Fails on texts with an id that may not follow."""
    ids = [np.flatnonzero(np.isin(np.arange(vocab) % 5, (s, (s + 1) % 5))).tolist() for s in range(5)]
    ids[4] = [4, 10]

    def allowed(text):
        state = 0
        for t in text[start:]:
            if t not in ids[state]:
                raise Outside(text[start:])
            state = t % 5
        return ids[state]
    return allowed


@pytest.mark.parametrize("more", [{}, dict(penalties=(1.3, 0.2, 0.1), biases={10: 1.0})])
def test_a_grammar_that_fails_outside_its_texts(more):
    cfg = wl.CONFIGS["tiny_f32"]
    pair, prompt = Pair(cfg, max_rows=128, max_positions=600), _prompt(cfg)
    allowed = _automaton(cfg.vocab, len(prompt))
    run = lambda **kw: generate(pair.model, pair.new_seq(600), prompt, 40, chunk=64, allowed=allowed, **more, **kw)  # noqa: E731
    plain, _ = run(k=0)
    allowed(prompt + plain)
    rng = np.random.default_rng(3)
    assert run(k=12)[0] == plain
    random, stats = run(k=7, drafter=lambda text, k: rng.integers(0, cfg.vocab, k).tolist())
    assert random == plain and stats["drafted"] < 7 * stats["steps"]          # excluded drafts are not verified
    mixed = lambda text, k: plain[len(text) - len(prompt):][:3] + rng.integers(0, cfg.vocab, k - 3).tolist()  # noqa: E731
    told, stats = run(k=8, drafter=lambda text, k: mixed(text, k)[:k])
    assert told == plain and stats["accepted_drafts"] > 20


def test_where_nothing_may_follow():
    """0 follows, also where a draft says so, and the drafts behind it change nothing."""
    cfg = wl.CONFIGS["tiny_f32"]
    pair, prompt = Pair(cfg, max_rows=128, max_positions=600), _prompt(cfg)
    allowed = lambda text: [] if len(text) % 5 == 2 else [v for v in range(cfg.vocab) if v % 3 == len(text) % 3]  # noqa: E731
    run = lambda **kw: generate(pair.model, pair.new_seq(600), prompt, 30, chunk=64, allowed=allowed, **kw)[0]  # noqa: E731
    plain = run(k=0)
    assert [t for i, t in enumerate(plain) if (len(prompt) + i) % 5 == 2] == [0] * 6
    rng = np.random.default_rng(5)
    assert run(k=9, drafter=lambda text, k: plain[len(text) - len(prompt):][:k]) == plain
    assert run(k=9, drafter=lambda text, k: [0] + rng.integers(0, cfg.vocab, k - 1).tolist()) == plain
