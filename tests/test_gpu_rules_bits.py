"""Processed logits (asr_logit_rules) bit for bit as the definition has them, the sign of a zero included,
whatever else lies in the row."""
import numpy as np
import pytest
import torch

from gpu_util import needs_gpu
from test_gpu_rules import BF16, F32, all_rules, f, normal, processed, run

pytestmark = [pytest.mark.gpu, needs_gpu]


def same_bits(logits, rules, dtype):
    V = logits.shape[1]
    seen = torch.from_numpy(logits).to(dtype).float().numpy()
    z, _, _, _ = run(logits, rules, 0, dtype)
    for r in range(len(logits)):
        with np.errstate(all="ignore"):
            want = processed(seen[r], rules, r, V)
        number = ~np.isnan(want)
        assert np.array_equal(np.isnan(z[r]), ~number)
        off = np.flatnonzero((z[r].view(np.uint32) != want.view(np.uint32)) & number)
        assert not len(off), f"row {r}: {len(off)} differ, token {off[0]}: {z[r][off[0]]!r}, not {want[off[0]]!r}"


def with_zeros(rng, rows, V):
    """Ordinary logits with zeros of both signs among them; at the end of the row values that make a
    wave divide."""
    x = normal(rng, rows, V)
    x[:, ::5] = 0.0
    x[:, 2::7] = -0.0
    wild = (rng.standard_normal((rows, V)) * np.exp2(rng.uniform(-140, 126, (rows, V)))).astype(f)
    x[:, V - 900::3] = wild[:, V - 900::3]
    return x


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("names", [("temperature",), ("history", "history_len", "repetition"),
                                   ("bias_token", "bias_value", "bias_len"),
                                   ("bias_token", "bias_value", "bias_len", "temperature"),
                                   ("history", "history_len", "prompt_len", "frequency", "presence"), None],
                         ids=lambda n: "+".join(n) if n else "all")
@pytest.mark.parametrize("history", [3000, 5000])
def test_signs_of_zeros(names, history, dtype):
    rng = np.random.default_rng(20)
    rows, V = 6, 21000
    rules = all_rules(rng, rows, V, n=history, b=9)
    rules["bias_len"][:] = [9, 0, 1, 0, 3, -2]          # rows without any, and waves without any
    rules["bias_value"][:, 4] = -0.0
    rules["temperature"][:] = [0.7, 1.3, 1.0, 1e-25, 0.3, 1e25]
    rules["frequency"][0] = rules["presence"][0] = 0.0
    same_bits(with_zeros(rng, rows, V), rules if names is None else {n: rules[n] for n in names}, dtype)
