"""Lists of starts on the paged cache's calls that say more than there is: rows and sequences that a batch of a fixed size does
not use are padded, and what is padded reads and writes nothing."""
import numpy as np
import pytest
import torch

import page_util as P
from gpu_util import needs_gpu
from test_gpu_pages import BF16, F32, Attend, Pool, dev, host, i32

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


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("max_new", [1, 40])
def test_token_starts_that_fall(max_new, dtype):
    """Sequences whose tokens end before they start, or start behind all, get none: by 1, or by more than 32 bits hold.  (3 tokens
    before -2^31 are 2^31 - 3 in 32 bits.)"""
    from paper_2603_11273_amd import asr
    start = np.array([0, 3, -MOST - 1, 50, 20, 30, 29, 60, MOST, 5, MOST, -MOST - 1], np.int32)
    n, tokens = len(start) - 1, 60
    held = np.array([5, 0, -1, 70, 9, 1, 2, 64, 3, 8, 4])      # (the third's tokens would start before all: it takes none)
    rng = np.random.default_rng(83)
    pool = Pool(84, 2 * n + 3, 2)
    table = rng.permutation(pool.pages)[:2 * n].reshape(n, 2).astype(np.int32)
    x = dev(rng.standard_normal((2, tokens, 128)).astype(np.float32)).to(dtype)
    codes, scales = pool.codes.copy(), pool.scales.copy()
    P.write(codes, scales, table, held, start, host(x[0].double()), host(x[1].double()), max_new)
    asr.PageWrite(pool.gpu_codes, pool.gpu_scales, i32(table), i32(held), tokens=tokens, dtype=dtype, max_new=max_new,
                  token_start=i32(start))(x[0], x[1])
    pool.check(codes, scales)
    assert (codes != pool.codes).any()
