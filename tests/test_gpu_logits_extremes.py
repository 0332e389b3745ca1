"""vf_logits_adjust with repetitions and logits at the ends of the float32 range: the quotient and the product are those of the type."""
import numpy as np
import pytest
import torch

import paper_2510_15312_amd as vf
from util_gpu import DEV, f32, i32

pytestmark = pytest.mark.gpu
MOST, LEAST = float(np.finfo(np.float32).max), 2.0 ** -149
RHO = [float("inf"), MOST, 3e38, 2.0 ** 127, 2.0 ** 126, 1e30, 1.3, 1.0 - 2.0 ** -24, 1e-30, 2.0 ** -126, 1.5e-38, 2.0 ** -128, 2.9e-39, 1e-39, 3e-42, LEAST]
Z = [MOST, 3e38, 1e20, 7.0, 1.0, 0.3, 1e-10, 2e-38, 2.0 ** -126, 1e-39, 3e-45, LEAST, 0.0, -0.0, float("inf")]
Z += [-z for z in Z if z] + [float("nan")]


@pytest.mark.parametrize("dtype,in_place", [(torch.float32, False), (torch.float32, True), (torch.bfloat16, False)])
@pytest.mark.parametrize("vocab", [64, 1027])
def test_repetitions_at_the_ends_of_the_range(vocab, dtype, in_place):
    z = torch.zeros((len(RHO), vocab), dtype=dtype, device=DEV)
    z[:, 10:10 + len(Z)] = torch.tensor(Z, dtype=dtype, device=DEV)
    out = z if in_place else torch.empty(z.shape, dtype=torch.float32, device=DEV)
    n, before = len(RHO), z.float().cpu().numpy()
    vf.vf_logits_adjust(z, i32(range(n + 1)), out, penalties=f32([[r, 0.0, 0.0] for r in RHO]),
                        history=i32([list(range(10, 10 + len(Z)))] * n), history_len=i32([len(Z)] * n))
    got = out.cpu().numpy()
    seen = slice(10, 10 + len(Z))
    for rho, x, y in zip(np.float32(RHO), before[:, seen], got[:, seen]):
        with np.errstate(all="ignore"):
            exact = np.where(x > 0, x.astype(np.float64) / np.float64(rho), x.astype(np.float64) * np.float64(rho))
            want = exact.astype(np.float32)
        # the reciprocal and its product round, and where the correction is below the type's least value nothing takes that back: two roundings
        # of 2^-24 (each of 2^-150 below the normal values) and the last one
        finite = np.isfinite(want)
        assert np.array_equal(np.isnan(want), np.isnan(y)), rho
        assert np.array_equal(want[~finite & ~np.isnan(want)], y[~finite & ~np.isnan(want)]), rho
        assert (np.abs(y[finite].astype(np.float64) - exact[finite]) <= 3 * np.maximum(2.0 ** -24 * np.abs(exact[finite]), 2.0 ** -150)).all(), rho
    rest = np.ones(vocab, bool)
    rest[seen] = False
    assert not got[:, rest].any()


@pytest.mark.parametrize("rho", [float("inf"), 1e-39])
def test_with_the_other_penalties_a_bias_and_a_mask(rho):
    """rho = infinity takes a positive logit to 0, one of 1e-39 a small one to 10, before all else."""
    vocab, x = 4096, 2.0 if rho > 1 else 1e-38
    z = torch.full((3, vocab), x, device=DEV)
    out = torch.empty_like(z)
    vf.vf_logits_adjust(z, i32([0, 3]), out, penalties=f32([[rho, 0.5, 0.25]]), history=i32([[4, 5, 5]]), history_len=i32([3]), prompt_len=i32([1]),
                        tokens=i32([-1, 7, 5]), biases=(i32([0, 1]), i32([7]), f32([8.0])), mask=i32([[-1] * (vocab // 32)] * 2 + [[~(1 << 5)] + [-1] * (vocab // 32 - 1)]))
    want = np.full((3, vocab), np.float32(x))
    q = np.float32(np.float64(np.float32(x)) / np.float64(np.float32(rho)))
    want[:, 4], want[:, 5], want[:, 7] = q, q - np.float32(1.0), np.float32(x) + 8
    want[1:, 7], want[2, 5] = q - np.float32(0.75) + 8, -np.inf
    # quotient 2 roundings, sums 2
    assert np.allclose(out.cpu().numpy(), want, rtol=4 * 2.0 ** -24, atol=8 * 2.0 ** -24)
