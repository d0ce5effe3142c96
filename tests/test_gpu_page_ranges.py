"""The paged cache's calls and sampling at the ends of the ranges that include/asr.h states: many sequences, long prompts, pages of
4096 positions, 2^22 pages, 2^20 tokens.

Attention's tolerance is that of test_gpu_pages.attention, which counts 2^-17 for a weight as a pair of bf16; the first of the
pair is cut, not rounded (off by up to 2^-7), and the second rounds what is left (by up to 2^-9 of that): 2^-16, so another 2^-17 of
sum_j p_j |v_j| is added for a bf16 result.

Sampling's distance: weights are formed to 2^-44 of themselves and rounded to whole units, so with E the sum of what that moves and
S the sum of the kept weights (or of the first top_k), a share of S is off by up to 2 E / S, and by 2^-52 for the products in
doubles; a weight against min-p by 2^-43.  A row with a decision nearer than that says nothing, and the inputs hold none."""
import numpy as np
import pytest
import torch

import page_util as P
from gpu_util import needs_gpu
from test_gpu_pages import BF16, F32, Attend, Pool, attention, dev, host, i32, table_of, tables_case

pytestmark = [pytest.mark.gpu, needs_gpu]


def check(case, out, rows=None):
    """Attend.check, with the weights' 2^-16; rows: those that are written (default: of a sequence)."""
    got, bf = host(out.double()), out.dtype == BF16
    args = (case.table, case.start, case.first, case.length, case.q, case.heads, 0.125, bf)
    ref = attention(case.pool.codes, case.pool.scales, *args)
    plain = case.pool.codes.copy()
    plain[:, 1] &= 0x7f
    size = attention(plain, np.abs(case.pool.scales), *args) if bf else None      # sum_j p_j |v_j|
    for r, want in enumerate(ref):
        if want is None or (rows is not None and not rows[r]):
            assert (got[r] == 7.0).all(), f"row {r} was written"
            continue
        tol = want[1] + (2.0 ** -17 * size[r][0] if bf else 0)
        bad = ~(np.abs(got[r] - want[0]) <= tol)
        assert not bad.any(), f"row {r}: {np.nanmax(np.abs(got[r] - want[0])):.3e}, allowed {np.nanmax(tol):.3e}"


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("sequences", [64, 65, 129, 200])
@pytest.mark.parametrize("heads,kv", [(12, 1), (6, 6)])
def test_many_sequences_joined_by_a_second_kernel(heads, kv, sequences, dtype):
    """More than 8 queries a cache head, or more than 3 blocks a CU: rows find their sequence among 64 starts and more; some
    sequences are empty, the first rows and the last of none."""
    rng = np.random.default_rng(sequences)
    sizes = rng.choice([0, 1, 2], sequences) if kv == 1 else np.where(rng.random(sequences) < 0.2, 0, 1)
    sizes[[0, 5, 63]] = 0, 1, 1                      # (an empty one first, rows on both sides of a chunk's end)
    case = Attend(sequences, list(sizes), [300, 700, 64, 513, 1], heads=heads, kv=kv, mask="causal", uncovered=5)
    case.start += 2                                  # rows 0 and 1 before all, 3 behind: of none
    case.length[2:], case.first[2:] = case.length[:-2].copy(), case.first[:-2].copy()
    check(case, case.run(dtype, part_keys=256, max_rows=2))
    check(case, case.run(dtype, max_rows=2))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("window", [0, 100])
def test_prompts_of_hundreds_of_rows(window, dtype):
    case = Attend(91, [224, 1, 190], [224, 100, 700], heads=4, kv=2, mask="causal", page=128, window=window)
    check(case, case.run(dtype))
    check(case, case.run(dtype, part_keys=256))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads", [2, 10])
def test_rows_past_max_rows_stay(heads, dtype):
    """With the join in the launch (up to 8 queries) and by a second kernel."""
    case = Attend(93, [5, 2, 4], [700, 300, 900], heads=heads, kv=2)
    written = np.array([1, 1, 1, 0, 0, 1, 1, 1, 1, 1, 0], bool)
    check(case, case.run(dtype, part_keys=256, max_rows=3), written)
    check(case, case.run(dtype, max_rows=3), written)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("page", [4032, 4096])
def test_large_pages(page, dtype):
    from paper_2603_11273_amd import asr
    case = Attend(95, [1, 3, 1], [4095, 9000, 4097], heads=4, kv=2, page=page, mask="causal")
    check(case, case.run(dtype))
    check(case, case.run(dtype, part_keys=256))
    rng = np.random.default_rng(96)
    pool = Pool(97, 9, 2, page)
    held, new = np.array([page - 3, 0, 2 * page - 64, 100]), np.array([70, page + 1, 64, 1])
    table, start = table_of(rng, 9, [2, 2, 2, 1], 2), np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    x = dev(rng.standard_normal((2, int(start[-1]), 128)).astype(np.float32)).to(dtype)
    codes, scales = pool.codes.copy(), pool.scales.copy()
    P.write(codes, scales, table, held, start, host(x[0].double()), host(x[1].double()), page + 1)
    asr.PageWrite(pool.gpu_codes, pool.gpu_scales, i32(table), i32(held), tokens=int(start[-1]), dtype=dtype, max_new=page + 1,
                  token_start=i32(start))(x[0], x[1])
    pool.check(codes, scales)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("heads,sequences", [(4, 9), (12, 9), (4, 150)])
def test_the_same_bits_at_every_call(heads, sequences, dtype):
    """Parts joined in the launch by whichever block ends last, and by a second kernel."""
    case = Attend(99, [1, 2, 1] * (sequences // 3), [2500, 700, 64, 1500], heads=heads, kv=2, page=128)
    want = case.run(dtype)
    check(case, want)
    assert all(torch.equal(case.run(dtype), want) for _ in range(20))


# ---------------------------------------------------------------------------
# Tables
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("compact", [False, True], ids=["", "compact"])
@pytest.mark.parametrize("n,pages", [(40, (1 << 18) + 1), (1100, (1 << 18) + 33), (40, 1 << 22), (3, (1 << 22) - 31)])
def test_more_pages_than_their_bits_fit_in_lds(n, pages, compact):
    """2^18 pages is what the bits in LDS hold, 2^22 the most that is taken; no data is copied."""
    from paper_2603_11273_amd import asr
    columns, page, held = (700, 16, 11000) if n < 100 else (9, 64, 500)
    table, length, parent, want, had = tables_case(n, n, columns, page, 100, held)
    # the same pages, spread over all
    rng = np.random.default_rng(pages)
    place = rng.permutation(np.arange(1, pages - 1))[:had].astype(np.int32)
    place[:2] = pages - 1, 0
    table = np.where((table >= 0) & (table < had), place[table.clip(0, had - 1)], np.where(table >= had, pages, -1)).astype(np.int32)
    new, lens, room, info, _ = P.next_tables(table, length, parent, want, page, pages, compact)
    out = dict(new_table=i32(np.zeros((n, columns))), new_length=i32(np.zeros(n)), room=i32(np.zeros(n)), info=i32(np.zeros(4)))
    plan = asr.PageTables(None, None, i32(table), i32(length), parent=i32(parent), want=i32(want), page=page, pages=pages, **out)
    for _ in range(2):
        plan(compact=compact)
        for got, ref in ((out["new_table"], new), (out["new_length"], lens), (out["room"], room), (out["info"], info)):
            assert np.array_equal(host(got), ref)
    assert not compact or info[3] > 0


# ---------------------------------------------------------------------------
# Sampling
# ---------------------------------------------------------------------------
def weights(l, T, k):
    """Weights of a row in falling order, and by how much they may be off."""
    V = len(l)
    w = np.exp((l - l.max()) / T)
    unit = 2.0 ** (62 - max(int(np.ceil(np.log2(V))), 12))
    return np.sort(w)[::-1][:k], np.abs(np.rint(w * unit) / unit - w).sum() + 2.0 ** -44 * w.sum()


def sample(x, u, exact=False, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One set of parameters for all rows; exact: every weight and sum is exact, a distance is not needed."""
    from paper_2603_11273_amd import asr
    rows, V = x.shape
    one = lambda v, kind: dev(np.full(rows, v, kind))  # noqa: E731
    plan = asr.Sampler(rows, V, x.dtype, draws=u.shape[1], temperature=one(temperature, np.float32), top_k=one(top_k, np.int32),
                       top_p=one(top_p, np.float32), min_p=one(min_p, np.float32))
    token, kept = i32(np.full(u.shape, -7)), i32(np.full(rows, -7))
    logprob = torch.zeros(u.shape, device="cuda")
    plan(x.cuda(), dev(u), token, logprob, kept)
    for r in range(rows):
        l = x[r].double().numpy()
        T, p, m = np.float32(temperature), np.float32(top_p), np.float32(min_p)
        tokens, lp, n, slack = P.sample(l, u[r], T, top_k, p, m)
        best, moved = weights(l, float(T), n)
        assert exact or slack > max(2 * moved / best.sum() + 2.0 ** -52, 2.0 ** -43), f"row {r} is too near to decide: {slack:.1e}"
        assert host(kept)[r] == n and host(token)[r].tolist() == tokens, r
        # (rounded once, behind the logarithm of a sum: 2^-44 of the weights, 1024 tokens a lane added in doubles 2^-43)
        assert (np.abs(host(logprob)[r] - np.array(lp)) <= 2.0 ** -24 * np.abs(lp) + 2.0 ** -41).all(), r


CASES = {
    "no filter": dict(spread=3.0),
    "sharp": dict(spread=3.0, top_p=0.9, temperature=0.6),
    "top-p of a flat row": dict(spread=0.5, top_p=0.9),
    "top-k of a flat row": dict(spread=0.5, top_k=300001),
    "all filters, many kept": dict(spread=0.5, top_k=700000, top_p=0.97, min_p=0.01, temperature=1.2),
    "all filters, few kept": dict(spread=3.0, top_k=50, top_p=0.9, min_p=0.05, temperature=0.8),
    "top-k alone": dict(spread=3.0, top_k=6000),
}


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [1048575, 1048576])
@pytest.mark.parametrize("name", list(CASES))
def test_the_largest_vocabulary(name, V, dtype):
    kw = dict(CASES[name])
    rng = np.random.default_rng(V + len(name))
    x = torch.from_numpy((rng.standard_normal((2, V)) * kw.pop("spread") - 4).astype(np.float32)).to(dtype)
    sample(x, rng.random((2, 3)).astype(np.float32), **kw)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [1048575, 1048576])
def test_the_largest_sums(V, dtype):
    """Equal logits: each weight is the largest that there is, and 2^20 of them the largest sum, 2^62 units."""
    x = torch.full((2, V), -3.0, dtype=dtype)
    u = np.array([[0.0, 2 ** 23 + 1, 2 ** 24 - 1], [1, 12345679, 8388607]], np.float64).astype(np.float32) / np.float32(2 ** 24)
    for kw in ({}, dict(top_p=0.5), dict(top_k=V - 1), dict(top_k=V // 3, top_p=0.75), dict(min_p=1.0)):
        sample(x, u, exact=True, **kw)


@pytest.mark.parametrize("V", [1048575, 1048576])
def test_all_logits_within_the_first_bin(V):
    """Nearly equal logits, all less than 2^-12 below the largest: one bin takes every weight that the guess for top-p adds."""
    rng = np.random.default_rng(V)
    x = torch.from_numpy((rng.random((2, V)) * -2.0 ** -13).astype(np.float32))
    sample(x, rng.random((2, 3)).astype(np.float32), top_p=0.7)
    sample(x, rng.random((2, 3)).astype(np.float32), top_p=0.999)
