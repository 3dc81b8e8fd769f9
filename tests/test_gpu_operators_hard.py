"""Rollout and policy operators on the GPU where a value, a size or a call's surroundings are hard: NaN rows, sums of a
million terms, calls that are prepared, captured or cut short.  Tolerances are those of test_gpu_operators.py."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _util import guarded_empty  # noqa: E402,F401
from test_gpu_operators import BF16, F32, api, plain_policy, policy_inputs, rule_sample, up  # noqa: E402,F401

INF, NAN = math.inf, float("nan")


def near_log_probs(got, want):
    want = torch.as_tensor(want, dtype=torch.float64, device=got.device)
    return ((got.double() - want).abs() <= 1e-5 + 2.0 ** -22 * want.abs()).all()


# ------------------------------------------------------------------------------------------ sampling
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,A", [(600, 5000), (3, 40000)])
@pytest.mark.parametrize("numbers", [1, 5, 40])
def test_sample_top_k_above_the_numbers_of_a_row(api, R, A, numbers, dtype):
    """Fewer numbers than top_k, the rest NaN, right behind a call that leaves the multiprocessors' shared memory full of words that
    would pass for keys of logits far above the row's own."""
    g = torch.Generator(device="cuda").manual_seed(numbers)
    full = torch.full((1200, 32768), -3.0, dtype=BF16, device="cuda")
    some = torch.zeros(1200, dtype=torch.int32, device="cuda")
    x = torch.full((R, A), NAN, device="cuda")
    at = torch.rand(R, A, device="cuda", generator=g).argsort(1)[:, :numbers]
    x.scatter_(1, at, torch.randn(R, numbers, device="cuda", generator=g) - 6)
    x = x.to(dtype)
    one, u = torch.ones(R, device="cuda"), torch.rand(R, device="cuda", generator=g)
    for k in (50, 192):
        for p in (1.0, 0.8):
            ks = torch.full((R,), k, dtype=torch.int32, device="cuda")
            want = rule_sample(x, u, one, ks, one * p, 0 * one)
            api.compute_log_probs(full, some)
            got = api.sample_actions(x, u, top_k=k, top_p=p)
            assert torch.equal(got[0], want[0])
            assert near_log_probs(got[1], want[1]) and near_log_probs(got[2], want[2])


