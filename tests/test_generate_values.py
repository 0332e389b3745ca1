"""Penalties and biases of generate that would leave logits that are no numbers, and the first token where a logit is none (CPU)."""
import pytest
import torch

from paper_2510_15312_amd.generate import _Adjust, _best

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("penalties", [(INF, 0, 0), (1e39, 0, 0), (1e-50, 0, 0), (NAN, 0, 0), (-INF, 0, 0), (1.0, NAN, 0), (1.0, 0, NAN), (1.0, INF, -INF),
                                       (1.0, -1e39, 1e39)])
def test_penalties(penalties):
    with pytest.raises(ValueError, match="repetition"):
        _Adjust(penalties, None, None, [1, 2], 10, 20, "cpu")


@pytest.mark.parametrize("penalties", [(1.1, 0.5, -0.5), (1e-44, 0, 0), (3e38, 0, 0), (1.0, INF, 0), (1.0, INF, INF), (1.0, 0, -INF)])
def test_penalties_that_are_taken(penalties):
    assert _Adjust(penalties, None, None, [1, 2], 10, 20, "cpu").more["penalties"].tolist() == [torch.tensor(penalties, dtype=torch.float32).tolist()]


def test_biases():
    with pytest.raises(ValueError, match="biases"):
        _Adjust(None, {3: 1.0, 4: NAN}, None, [1, 2], 10, 20, "cpu")
    assert _Adjust(None, {3: INF, 4: -INF}, None, [1, 2], 10, 20, "cpu").more["biases"][2].tolist() == [INF, -INF]


@pytest.mark.parametrize("z,best", [([1.0, 3.0, 3.0, 2.0], 1), ([NAN, 3.0, 3.0, NAN], 1), ([-INF] * 4, 0), ([NAN] * 4, 0), ([NAN, -INF, -1e38, NAN], 2),
                                    ([0.0, INF, INF, NAN], 1)])
def test_the_best_id(z, best):
    assert _best(torch.tensor(z)) == best
