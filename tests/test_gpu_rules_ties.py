"""The k best of rows with many equal logits, over so many blocks that the join has more results at its
floor than it ranks at once: flat rows, a few values over whole vocabularies, masks that leave a part;
a single row (joined in its launch) and many (joined by a second kernel)."""
import numpy as np
import pytest

from gpu_util import needs_gpu
from test_gpu_rules import BF16, F32, check, f

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V,rows", [(51866, 1), (51866, 3), (51866, 40), (1 << 20, 1), (1 << 20, 3)])
def test_many_equal_logits(V, rows, dtype):
    rng = np.random.default_rng(V + rows)
    kinds = [np.zeros(V), np.full(V, -3.5), rng.integers(0, 3, V) * 1.0, -1.0 * (np.arange(V) % 4096 >= 4),
             np.where(np.arange(V) % 4096 >= 4090, 2.0, 1.0), np.where(rng.random(V) < 1e-3, 7.0, rng.standard_normal(V)),
             np.full(V, np.finfo(f).min)]
    logits = np.stack([kinds[(r + rows) % len(kinds)] for r in range(rows)]).astype(f)
    if dtype is BF16:
        logits[logits == np.finfo(f).min] = -3.3895313892515355e38
    check(logits, {}, 16, dtype, out=False)
    allowed = rng.random((3, V)) < np.array([0.5, 0.01, 0.9])[:, None]
    allowed[1, :V // 2] = False
    mask_of = rng.integers(-1, 3, rows).astype(np.int32)
    check(logits, {"allowed": allowed, "mask_of": mask_of}, 16, dtype, out=False)
    check(logits, {"allowed": allowed, "mask_of": mask_of}, 1, dtype, out=False)
    # long histories: blocks of 1024 threads
    rules = {"history": rng.integers(0, V, (rows, 4096)).astype(np.int32), "history_len": np.full(rows, 4096, np.int32),
             "presence": np.full(rows, 1.0, f)}
    check(logits, rules, 16, dtype, out=False)
