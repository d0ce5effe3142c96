"""Log-probabilities (asr_logit_rules) do not lose to the size of the logits.

Tolerance: z - M and the result are rounded once (half a step each), the logarithm is off by 2^-23 of
itself, and the sum's relative error (at most 48 additions of 2^-24, the exponential's 2^-22, and 2^-22 of
the mean distance from the maximum for the exponent's argument) is the logarithm's absolute one.  No term
grows with the maximum."""
import numpy as np
import pytest

from gpu_util import needs_gpu
from test_gpu_rules import F32, f, run

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("V", [2, 300, 51866])
@pytest.mark.parametrize("history", [40, 5000])
def test_size_of_the_logits_does_not_matter(V, history):
    rng = np.random.default_rng(30)
    tops = np.array([0.0, 20.0, 77.5, 300.0, 1000.25, 4095.0, 4100.0, -2500.0, 1e6], f)
    rows, k = len(tops), min(V, 4)
    logits = (tops[:, None] - np.exp(rng.uniform(0.5, 2.5, (rows, V))) - 3).astype(f)
    logits[np.arange(rows), rng.integers(0, V, rows)] = tops       # one near-certain token each
    # a history that changes nothing: the kernels for short and for long ones
    rules = {"history": np.zeros((rows, history), np.int32), "history_len": np.zeros(rows, np.int32)}
    _, token, logprob, _ = run(logits, rules, k)
    for r in range(rows):
        z = logits[r].astype(np.float64)
        M = z.max()
        e = np.exp(z - M)
        log_sum = np.log(e.sum())
        off = (e * (M - z)).sum() / e.sum() * 2.0 ** -22 + 48 * 2.0 ** -24 + 2.0 ** -22
        for t, v in zip(token[r], logprob[r]):
            want = (z[t] - M) - log_sum
            tol = off + 2.0 ** -24 * (abs(z[t] - M) + abs(want)) + 2.0 ** -23 * abs(log_sum)
            assert abs(v - want) <= tol, f"row {r} of {tops[r]}, token {t}: {v!r}, not {want!r} (within {tol:.1e})"
