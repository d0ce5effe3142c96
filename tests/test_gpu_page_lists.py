"""Lists of starts on the paged cache's calls that say more than there is: rows and sequences that a batch of a fixed size does
not use are padded, and what is padded reads and writes nothing."""
import numpy as np
import pytest
import torch

from gpu_util import needs_gpu
from test_gpu_pages import BF16, F32, Attend

pytestmark = [pytest.mark.gpu, needs_gpu]

MOST = 2147483647


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("per", [2, 4])
@pytest.mark.parametrize("pad", [MOST, MOST - 1, 1 << 30, 6, 5])
def test_row_starts_padded_behind_the_rows(pad, per, dtype):
    """Sequences whose row starts lie behind the rows: the others' results bit for bit, and nothing else written.  (Five rows
    less 2^31 - 1, times 2 or 4 queries a row, are 12 or 24 in 32 bits.)  Up to 8 queries: a row's last block joins its parts."""
    case = Attend(81, [2, 1, 2], [1500, 300, 700], heads=2 * per, kv=2, page=128)
    case.max_rows = 8 // per
    want = case.run(dtype, part_keys=256)
    case.check(want)
    case.start = np.concatenate([case.start, np.full(4, pad)]).astype(np.int32)
    case.table = np.concatenate([case.table] * 3)[:7]
    around = torch.full((case.rows + 64, 2 * per * 64), 7.0, dtype=dtype, device="cuda")
    assert torch.equal(case.run(dtype, part_keys=256, out=around[:case.rows]), want)
    assert (around[case.rows:] == 7.0).all()
