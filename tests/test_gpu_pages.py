"""Pages of 8 bits on the GPU: writing (asr_write_pages) and tables (asr_next_tables) equal their definitions byte for byte and
number for number; attention (asr_attend_pages) against softmax attention in 64 bits.

Tolerance of an attention's output: softmax weights move by at most e^{2 ds} - 1 when every score moves by at most ds, so an
output moves by 2 ds (1 + ds) sum_j p_j |v_j|.  Codes are exact in bf16; ds has the roundings of a dot product of 64 terms (66
steps of 2^-24 of sum |q_i k_i|; with a bf16 result 2^-17 for the query as a pair of bf16 values), of the scale and the
exponent's argument (2^-22 of the largest score) and the exponential (2^-22).  The weights' own rounding (2^-22 with their block's
scale, 2^-17 as a bf16 pair), the sums over n keys (2 n 2^-24) and the joins (32 of 2^-24) are relative to sum_j p_j |v_j| too.
The result is rounded once: half a step of its type."""
import numpy as np
import pytest
import torch

import page_util as P
from gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

F32, BF16 = torch.float32, torch.bfloat16


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(a):
    return dev(np.asarray(a, np.int32))


def host(t):
    return t.detach().cpu().numpy()


class Pool:
    """A pool on the GPU and the same on the CPU; layers > 1: the first of several layers' pages, the others NaN."""

    def __init__(self, seed, pages, heads, page=64, layers=1, layer=0, odd_scales=False):
        rng = np.random.default_rng(seed)
        shape = (pages, 2, heads, page // 64, 64, 64)
        self.codes = P.encode(rng.standard_normal(shape) * 60).astype(np.uint8)
        self.scales = (2.0 ** rng.integers(-8, -4, shape[:4])).astype(np.float32)
        if odd_scales:
            self.scales *= rng.uniform(1, 2, shape[:4]).astype(np.float32)
        whole = np.full((pages, layers, *shape[1:]), 0x7f, np.uint8)
        some = np.full((pages, layers, *shape[1:4]), np.nan, np.float32)
        whole[:, layer], some[:, layer] = self.codes, self.scales
        self.whole, self.some, self.layer = dev(whole), dev(some), layer
        self.page, self.pages, self.heads = page, pages, heads
        self.gpu_codes, self.gpu_scales = self.whole[:, layer], self.some[:, layer]

    def poke(self):
        """The CPU's codes and scales to the GPU."""
        self.gpu_codes.copy_(dev(self.codes))
        self.gpu_scales.copy_(dev(self.scales))

    def check(self, codes, scales):
        got, s = host(self.gpu_codes), host(self.gpu_scales)
        bad = (s != scales) & ~(np.isnan(s) & np.isnan(scales))
        assert not bad.any(), f"{bad.sum()} scales differ, the first at {np.argwhere(bad)[0]}"
        nan = (codes & 127) == 127
        bad = np.where((got & 127) == 127, 0x7f, got) != np.where(nan, 0x7f, codes)
        assert not bad.any(), f"{bad.sum()} codes differ, the first at {np.argwhere(bad)[0]}"
        others = [i for i in range(self.whole.shape[1]) if i != self.layer]
        assert (host(self.whole)[:, others] == 0x7f).all() and np.isnan(host(self.some)[:, others]).all()


def table_of(rng, pages, needs, columns):
    t = np.full((len(needs), columns), -1, np.int32)
    free = list(rng.permutation(pages))
    for s, n in enumerate(needs):
        for j in range(n):
            t[s, j] = free.pop()
    return t


# ---------------------------------------------------------------------------
# Writing
# ---------------------------------------------------------------------------
WRITES = {
    "first token": dict(held=[0], new=[1]),
    "tokens of a step": dict(held=[0, 1, 63, 64, 65, 127, 128, 300, 10], new=[1] * 9),
    "one token each, no starts": dict(held=[5, 0, 64, 200], new=[1] * 4, starts=False),
    "whole blocks": dict(held=[0, 64], new=[64, 128]),
    "odd lengths": dict(held=[3, 60, 0, 130, 17], new=[61, 9, 700, 1, 0]),
    "cut at max_new": dict(held=[3, 60], new=[61, 9], max_new=20),
    "pages of several blocks": dict(held=[100, 0, 511], new=[500, 1, 2], page=256),
    "a pool of three layers": dict(held=[100, 0, 31], new=[30, 1, 2], page=128, layers=3, layer=1),
    "one head": dict(held=[10, 7], new=[120, 3], heads=1),
    "seven heads": dict(held=[10, 7], new=[12, 70], heads=7),
    "past the table": dict(held=[120, 128, 190], new=[30, 5, 3], columns=2),
    "pages that are none": dict(held=[10, 60, 0, 0], new=[200, 100, 70, 5], holes=[(0, 1), (1, 0), (2, 99), (3, 0)]),
    "no sequence": dict(held=[-1, 5, -2147483648, 2147483647], new=[3, 3, 4, 2]),
    "large and small tokens": dict(held=[20, 30, 0, 63], new=[3, 80, 64, 1], amp=[1e-3, 1e4, 1e30, 1e-38]),
    "scales of the caller's own": dict(held=[20, 30, 40, 63], new=[3, 8, 4, 1], odd=True, amp=[1, 10, 0.1, 100]),
}


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("name", list(WRITES))
def test_write(name, dtype):
    from paper_2603_11273_amd import asr
    c = dict(heads=3, page=64, layers=1, layer=0, starts=True, odd=False, amp=[1.0], holes=[], max_new=None, columns=None) | WRITES[name]
    rng = np.random.default_rng(len(name) * 7 + 1)
    held, new, H, page = np.array(c["held"], np.int64), np.array(c["new"]), c["heads"], c["page"]
    needs = [max(0, -(-(min(h, 4096) + n) // page)) if h < 4096 else 0 for h, n in zip(held, new)]
    columns = c["columns"] or max(max(needs), 1)
    pool = Pool(3, sum(needs) + 4, H, page, c["layers"], c["layer"], c["odd"])
    table = table_of(rng, pool.pages, [min(n, columns) for n in needs], columns)
    for s, p in c["holes"]:
        table[s, p % columns] = (-1, pool.pages, -2147483648, 2147483647)[s]
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    tokens = int(new.sum())
    amp = np.repeat(np.array([c["amp"][s % len(c["amp"])] for s in range(len(new))]), new)[:, None]
    qkv = (rng.standard_normal((tokens, 3 * H * 64)) * np.concatenate([amp] * (3 * H * 64), 1)).astype(np.float32)
    x = dev(qkv).to(dtype)
    k, v = x[:, H * 64:2 * H * 64], x[:, 2 * H * 64:]
    most = c["max_new"] or max(int(new.max()), 1)
    plan = asr.PageWrite(pool.gpu_codes, pool.gpu_scales, i32(table), i32(held), tokens=tokens, dtype=dtype, max_new=most,
                         token_start=i32(start) if c["starts"] else None)
    codes, scales = pool.codes.copy(), pool.scales.copy()
    P.write(codes, scales, table, held, start, host(k.double()), host(v.double()), most)
    plan(k, v)
    pool.check(codes, scales)
    if not c["odd"]:
        plan(k, v)                       # the same tokens again: nothing changes
        pool.check(codes, scales)


def test_write_values_that_are_not_finite():
    from paper_2603_11273_amd import asr
    for rows, held in ((1, 5), (70, 0)):
        pool = Pool(5, 4, 2)
        x = np.random.default_rng(6).standard_normal((rows, 128)).astype(np.float32)
        y = x.copy()
        x[0, :4] = [np.nan, np.inf, -np.inf, 3e38]
        x[0, 64:] = np.nan                               # a head whose tokens hold nothing finite (with one token)
        y[:, 64:] = 0.0                                  # and one whose values are zeros
        table = np.array([[2, 0]], np.int32)
        codes, scales = pool.codes.copy(), pool.scales.copy()
        P.write(codes, scales, table, [held], [0, rows], x.astype(np.float64), y.astype(np.float64), rows)
        asr.PageWrite(pool.gpu_codes, pool.gpu_scales, i32(table), i32([held]), tokens=rows, dtype=F32, max_new=rows,
                      token_start=i32([0, rows]))(dev(x), dev(y))
        pool.check(codes, scales)


def test_write_scales_that_are_none():
    """Blocks whose scale is zero, negative, NaN, infinite, tiny or huge get a token."""
    from paper_2603_11273_amd import asr
    bad = np.array([0.0, -1.0, np.nan, np.inf, 1e-40, 1e-37, 2e38, 3.0], np.float32)
    pool = Pool(7, len(bad), 1)
    pool.scales[:] = bad[:, None, None, None]
    pool.poke()
    n = len(bad)
    x = np.random.default_rng(8).standard_normal((n, 64)).astype(np.float32)
    table = np.arange(n, dtype=np.int32)[:, None]
    codes, scales = pool.codes.copy(), pool.scales.copy()
    P.write(codes, scales, table, [9] * n, np.arange(n + 1), x.astype(np.float64), x.astype(np.float64), 1)
    asr.PageWrite(pool.gpu_codes, pool.gpu_scales, i32(table), i32([9] * n), tokens=n, dtype=F32)(dev(x), dev(x))
    pool.check(codes, scales)


def test_write_all_bf16_values():
    """Every finite bf16 value below 2^9 in magnitude, at the scale that 448 gives, and at one that makes the least codes."""
    from paper_2603_11273_amd import asr
    bits = np.arange(1 << 16, dtype=np.uint32)
    x = (bits << 16).astype(np.uint32).view(np.float32)
    x = x[np.isfinite(x) & (np.abs(x) <= 448)]
    for by in (1.0, 2.0 ** -7):
        y = np.concatenate([np.full(64, 448.0), x * by, np.zeros((-len(x)) % 64)]).astype(np.float32)
        y = np.where(np.abs(y) <= 448, y, 0).astype(np.float32)
        rows = len(y) // 64
        y = y.reshape(rows, 64)
        y[::64, 0] = 448.0                               # every block's largest
        pool = Pool(9, -(-rows // 64), 1)
        table = np.arange(pool.pages, dtype=np.int32)[None]
        codes, scales = pool.codes.copy(), pool.scales.copy()
        P.write(codes, scales, table, [0], [0, rows], y.astype(np.float64), y.astype(np.float64), rows)
        assert (scales[:rows // 64] == 1.0).all()
        asr.PageWrite(pool.gpu_codes, pool.gpu_scales, i32(table), i32([0]), tokens=rows, dtype=F32, max_new=rows,
                      token_start=i32([0, rows]))(dev(y), dev(y))
        pool.check(codes, scales)


def test_write_token_by_token_or_at_once():
    """Rising tokens one by one: the scale grows within a block, and what was there follows it."""
    from paper_2603_11273_amd import asr
    rng = np.random.default_rng(10)
    pool = Pool(11, 5, 2)
    table = np.array([[3, 1, 0]], np.int32)
    codes, scales = pool.codes.copy(), pool.scales.copy()
    length = i32([60])
    plan = asr.PageWrite(pool.gpu_codes, pool.gpu_scales, i32(table), length, tokens=1, dtype=F32)
    for t in range(12):
        x = (rng.standard_normal((2, 1, 128)) * 4.0 ** (t - 4)).astype(np.float32)
        plan(dev(x[0]), dev(x[1]))
        P.write(codes, scales, table, [60 + t], [0, 1], x[0].astype(np.float64), x[1].astype(np.float64), 1)
        length += 1
    pool.check(codes, scales)


def test_pages_far_apart():
    """Pages whose place in the pool passes 32 bits: written, attended to and copied."""
    from paper_2603_11273_amd import asr
    H, stride = 1, 3 << 30
    room = torch.zeros(2 * stride + 2 * 4096, dtype=torch.uint8, device="cuda")
    codes = room.as_strided((3, 2, H, 1, 64, 64), (stride, 4096, 4096, 4096, 64, 1))
    scales = torch.ones((3, 2, H, 1), device="cuda")
    rng = np.random.default_rng(12)
    x = rng.standard_normal((70, 64)).astype(np.float32)
    table, length = np.array([[1, 2]], np.int32), i32([0])
    asr.PageWrite(codes, scales, i32(table), length, tokens=70, dtype=F32, max_new=70, token_start=i32([0, 70]))(dev(x), dev(x))
    want, ws = np.zeros((3, 2, H, 1, 64, 64), np.uint8), np.ones((3, 2, H, 1), np.float32)
    P.write(want, ws, table, [0], [0, 70], x.astype(np.float64), x.astype(np.float64), 70)
    assert np.array_equal(np.stack([host(codes[p]) for p in range(3)]), want) and np.array_equal(host(scales), ws)
    q = dev(rng.standard_normal((1, 64)).astype(np.float32))
    out = asr.PagedAttention(codes, scales, i32(table), i32([70]), n_head=1, rows=1, dtype=F32)(q, torch.zeros_like(q))
    ref, tol = attention(want, ws, table, [0, 1], [0], [70], host(q), 1, 0.125, False)[0]
    assert (np.abs(host(out)[0] - ref) <= tol).all()
    t, n = i32([[1, 2], [0, -1]]), i32([70, 0])
    info = i32([0] * 4)
    asr.PageTables(codes, scales, t, n, parent=i32([1, 0]), want=i32([0, 70]), info=info)(compact=True)
    # the half page 2 is free to be kept by sequence 1, and moves to 0
    assert host(t).tolist() == [[-1, -1], [1, 0]] and host(info).tolist() == [2, 0, 0, 1]
    assert np.array_equal(host(codes[0]), want[2]) and np.array_equal(host(codes[1]), want[1])


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------
def attention(codes, scales, table, start, first, length, q, heads, scale, bf):
    """Per row (out, tolerance), None for rows of no sequence; first and length per row."""
    pages, _, kv, blocks = codes.shape[:4]
    page, per, res = blocks * 64, heads // kv, [None] * len(q)
    values = P.VALUE[codes] * scales.astype(np.float64)[..., None, None]
    for s in range(len(table)):
        for r in range(max(int(start[s]), 0), min(int(start[s + 1]), len(q))):
            pos = np.arange(max(int(first[r]), 0), min(int(length[r]), table.shape[1] * page))
            pg = table[s, pos // page]
            pos, pg = pos[(pg >= 0) & (pg < pages)], pg[(pg >= 0) & (pg < pages)]
            out, tol = np.zeros((heads, 64)), np.zeros((heads, 64))
            for h in range(heads):
                if len(pos):
                    K = values[pg, 0, h // per, pos % page // 64, pos % 64]
                    V = values[pg, 1, h // per, pos % page // 64, :, pos % 64]
                    x = q[r, h * 64:(h + 1) * 64].astype(np.float64) * scale
                    z = K @ x
                    p = np.exp(z - z.max())
                    p /= p.sum()
                    out[h] = p @ V
                    ds = (66 * 2.0 ** -24 + (2.0 ** -17 if bf else 0)) * (np.abs(K) @ np.abs(x)).max() \
                        + 2.0 ** -22 * np.abs(z).max() + 2.0 ** -22
                    tol[h] = (2 * ds * (1 + ds) + 2.0 ** -22 + (2.0 ** -17 if bf else 0) + (2 * len(pos) + 32) * 2.0 ** -24) \
                        * (p @ np.abs(V)) + np.abs(out[h]) * (2.0 ** -8 if bf else 2.0 ** -24)
            res[r] = (out.reshape(-1), tol.reshape(-1))
    return res


class Attend:
    def __init__(self, seed, sizes, keys, heads=4, kv=4, page=64, mask="same", window=0, uncovered=0, holes=0, kind="normal",
                 layers=1, odd=True, clean=True):
        rng = np.random.default_rng(seed)
        self.heads, self.kv, n = heads, kv, len(sizes)
        self.start = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        self.rows = int(self.start[-1]) + uncovered
        L = np.array([keys[i % len(keys)] for i in range(n)])
        needs = -(-L // page)
        columns = max(int(needs.max(initial=0)), 1)
        self.pool = Pool(seed + 1, int(needs.sum()) + 3, kv, page, layers, layers - 1, odd_scales=odd)
        self.table = table_of(rng, self.pool.pages, needs, columns)
        # what no row may see
        if clean:
            seen = np.zeros((self.pool.pages, page), bool)
            for s in range(n):
                for j in range(needs[s]):
                    seen[self.table[s, j], :min(page, L[s] - j * page)] = True
            blind = ~seen.reshape(-1, page // 64, 64)
            self.pool.codes[:, 0] = np.where(blind[:, None, :, :, None], 0xff, self.pool.codes[:, 0])
            self.pool.codes[:, 1] = np.where(blind[:, None, :, None, :], 0x7f, self.pool.codes[:, 1])
            self.pool.scales[np.broadcast_to(blind.all(-1)[:, None, None], self.pool.scales.shape)] = np.nan
            self.pool.poke()
        for s in range(holes):
            self.table[s % n, rng.integers(columns)] = (-1, self.pool.pages, 2147483647)[s % 3]
        self.length = np.zeros(self.rows, np.int32)
        for s in range(n):
            for i, r in enumerate(range(self.start[s], self.start[s + 1])):
                self.length[r] = L[s] if mask == "same" else max(L[s] - (self.start[s + 1] - 1 - r), 0) if mask == "causal" \
                    else rng.integers(0, L[s] + 1)
        self.first = np.maximum(self.length - window, -5).astype(np.int32) if window else np.zeros(self.rows, np.int32)
        if mask == "ragged":
            self.first = (self.length - rng.integers(-2, 200, self.rows)).astype(np.int32)
        amp = {"normal": 2.0, "sharp": 12.0, "flat": 0.0}[kind]
        self.q = (amp * rng.standard_normal((self.rows, heads * 64))).astype(np.float32)
        self.max_rows = max(sizes) if n else 1

    def run(self, dtype, part_keys=0, out=None, q=None, **kw):
        from paper_2603_11273_amd import asr
        out = torch.full((self.rows, self.heads * 64), 7.0, dtype=dtype, device="cuda") if out is None else out
        args = dict(n_head=self.heads, rows=self.rows, row_start=i32(self.start), max_rows=self.max_rows, first=i32(self.first),
                    scale=0.125, dtype=dtype, part_keys=part_keys)
        args.update(kw)
        plan = asr.PagedAttention(self.pool.gpu_codes, self.pool.gpu_scales, i32(self.table), i32(self.length), **args)
        return plan(dev(self.q) if q is None else q, out)

    def check(self, out):
        got, bf = host(out.double()), out.dtype == BF16
        ref = attention(self.pool.codes, self.pool.scales, self.table, self.start, self.first, self.length, self.q, self.heads,
                        0.125, bf)
        for r, want in enumerate(ref):
            if want is None:
                assert (got[r] == 7.0).all(), f"row {r} is of no sequence and was written"
                continue
            assert np.array_equal(np.isnan(got[r]), np.isnan(want[0])), f"row {r}: NaN at other places"
            bad = np.abs(got[r] - want[0]) > want[1]
            assert not bad.any(), f"row {r}: {np.nanmax(np.abs(got[r] - want[0])):.3e}, allowed {np.nanmax(want[1]):.3e}"


ATTENDS = {
    "one key": dict(sizes=[1], keys=[1]),
    "no keys": dict(sizes=[1, 2], keys=[0]),
    "around a block's end": dict(sizes=[1] * 8, keys=[15, 16, 17, 63, 64, 65, 127, 129]),
    "around a part's end": dict(sizes=[1] * 5, keys=[255, 256, 257, 511, 1025], page=128),
    "some without keys": dict(sizes=[1, 0, 3, 1], keys=[0, 40, 7, 300]),
    "hypotheses of a clip": dict(sizes=[5], keys=[1500], heads=6, kv=6, page=128),
    "a chunk under a causal mask": dict(sizes=[33, 1, 7], keys=[400, 90, 7], mask="causal"),
    "more new tokens than keys": dict(sizes=[9], keys=[5], mask="causal"),
    "lengths and windows at random": dict(sizes=[20, 3, 40], keys=[700, 64, 333], mask="ragged"),
    "a window": dict(sizes=[1, 4], keys=[900, 1000], mask="causal", window=100, page=256),
    "a window of one key": dict(sizes=[3], keys=[200], mask="causal", window=1),
    "shared key heads": dict(sizes=[1, 1, 1], keys=[200, 31, 1000], heads=8, kv=2),
    "one key head for 20": dict(sizes=[5, 2], keys=[400, 100], heads=20, kv=1),
    "more than 64 queries": dict(sizes=[70, 3], keys=[260, 1000], heads=2, kv=2, mask="causal"),
    "100 query heads a key head": dict(sizes=[2], keys=[300], heads=100, kv=1),
    "rows of no sequence": dict(sizes=[2, 1], keys=[130], uncovered=3),
    "pages that are none": dict(sizes=[1, 2, 1, 1], keys=[500, 300, 64, 900], holes=7),
    "a page alone that is none": dict(sizes=[2], keys=[60], holes=1),
    "sharp scores": dict(sizes=[1, 4], keys=[900, 100], kind="sharp"),
    "equal scores": dict(sizes=[3], keys=[1000], kind="flat"),
    "a pool of three layers": dict(sizes=[1, 2], keys=[150, 300], layers=3, page=192),
    "a long sequence": dict(sizes=[1], keys=[20011], heads=4, kv=2, page=256),
}


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("name", list(ATTENDS))
def test_attend(name, dtype):
    case = Attend(len(name) * 3 + 5, **ATTENDS[name])
    case.check(case.run(dtype))
    case.check(case.run(dtype, part_keys=256))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_attend_without_starts_and_bounds(dtype):
    case = Attend(31, [1, 1, 1], [100, 700, 64])
    case.first[:] = 0
    case.check(case.run(dtype, row_start=None, first=None))
    cut = case.length.copy()
    case.length = np.minimum(cut, 130)
    want = case.run(dtype, part_keys=256)
    case.length = cut
    assert torch.equal(case.run(dtype, part_keys=256, max_keys=130), want)
    case.length = np.array([2147483647, -2147483648, -1], np.int32)       # to the table's end; none
    out = host(case.run(dtype).double())
    assert (out[1:] == 0).all() and np.isnan(out[0]).any()                # (behind its keys there are NaN codes)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_nan_touches_the_rows_that_see_it(dtype):
    case = Attend(41, [6, 1, 2], [200, 130, 70], mask="causal", heads=4, kv=2)
    c, t = case.pool.codes, case.table
    c[t[0, 3], 1, 0, 0, 5, 197 % 64] = 0x7f            # a value of position 197: rows of the sequence that see it, dim 5
    c[t[0, 3], 0, 1, 0, 199 % 64, 8] = 0xff            # a key of position 199: its last row, whole heads
    c[t[1, 0], 1, 1, 0, 63, 0] = 0x7f
    c[t[2, 1], 0, 0, 0, 69 % 64, 63] = 0x7f
    case.pool.poke()
    case.check(case.run(dtype))
    case.check(case.run(dtype, part_keys=256))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_scales_that_are_not_finite_touch_the_rows_that_see_them(bad, dtype):
    """The scale of a block that only the last rows see, of keys or of values."""
    for m in (0, 1):
        case = Attend(45, [9, 3], [135, 70], mask="causal", heads=4, kv=2)
        case.pool.scales[case.table[0, 2], m, 1, 0] = bad          # positions 128 to 134: rows 2 to 8 of 0 to 8
        case.pool.poke()
        for part_keys in (0, 256):
            got = host(case.run(dtype, part_keys=part_keys).double())
            with np.errstate(all="ignore"):
                ref = attention(case.pool.codes, case.pool.scales, case.table, case.start, case.first, case.length, case.q, 4, 0.125,
                                dtype == BF16)
            for r, (want, tol) in enumerate(ref):
                sees = np.zeros(256, bool)
                sees[128:] = r < 9 and case.length[r] > 128        # query heads 2 and 3 are on cache head 1
                assert np.isfinite(want[~sees]).all() and (np.abs(got[r] - want)[~sees] <= tol[~sees]).all(), r
                if np.isnan(bad):                                  # (what an infinite one gives is not said)
                    assert np.isnan(got[r][sees]).all() and np.isnan(want[sees]).all(), r


def test_queries_that_are_not_finite():
    case = Attend(43, [3, 1], [100, 70])
    case.q[0, 3], case.q[1, 70], case.q[2, 130] = np.nan, np.inf, -np.inf
    for dtype in (F32, BF16):
        got = host(case.run(dtype).double())
        for r in range(4):
            for h in range(4):
                assert np.isnan(got[r, h * 64:h * 64 + 64]).all() == (r < 3 and h == r), (r, h)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_a_rows_bits_are_its_own(dtype):
    """A row alone, among others, at another place, in a chunk: with part_keys the same bits."""
    case = Attend(51, [1, 1, 1, 1], [700, 100, 1500, 64], heads=8, kv=4, page=128)
    whole = case.run(dtype, part_keys=512)
    for r in range(4):
        one = Attend(51, [1, 1, 1, 1], [700, 100, 1500, 64], heads=8, kv=4, page=128)
        one.start, one.rows, one.q = np.array([0, 1], np.int32), 1, case.q[r:r + 1]
        one.table, one.length, one.first = case.table[r:r + 1], case.length[r:r + 1], case.first[r:r + 1]
        assert torch.equal(one.run(dtype, part_keys=512, max_keys=1500)[0], whole[r])
    chunk = Attend(53, [40], [700], mask="causal")
    all_rows = chunk.run(dtype, part_keys=256)
    for r in (0, 17, 39):
        one = Attend(53, [40], [700], mask="causal")
        one.start, one.rows, one.q, one.max_rows = np.array([0, 1], np.int32), 1, chunk.q[r:r + 1], 1
        one.length, one.first = chunk.length[r:r + 1], chunk.first[r:r + 1]
        assert torch.equal(one.run(dtype, part_keys=256)[0], all_rows[r])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_rows_apart(dtype):
    """Rows of q and out further apart than their width; what lies between stays."""
    case = Attend(61, [2, 3], [90, 300])
    wide = dev(np.concatenate([case.q, np.full((case.rows, 12), np.nan, np.float32)], 1))
    out = torch.full((case.rows, case.heads * 64 + 20), 7.0, dtype=dtype, device="cuda")
    case.check(case.run(dtype, q=wide[:, :-12], out=out[:, :-20]))
    assert (out[:, -20:] == 7.0).all()


def test_attend_captured_and_replayed():
    from paper_2603_11273_amd import asr
    case = Attend(71, [1, 1, 5], [900, 100, 1500], heads=6, kv=6, page=128)
    q, length = dev(case.q), i32(case.length)
    outs = [torch.zeros((case.rows, 384), dtype=BF16, device="cuda") for _ in range(2)]
    plans = [asr.PagedAttention(case.pool.gpu_codes, case.pool.gpu_scales, i32(case.table), length, n_head=6, rows=case.rows,
                                row_start=i32(case.start), max_rows=5, part_keys=256) for _ in range(2)]
    plans[0](q, outs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        plans[1](q, outs[1])
    for step in range(4):
        q.copy_(dev(case.q * (1 + step)))
        length.copy_(i32(np.maximum(case.length - 37 * step, 0)))
        outs[1].fill_(9)
        graph.replay()
        plans[0](q, outs[0])
        torch.cuda.synchronize()
        assert torch.equal(*outs)


# ---------------------------------------------------------------------------
# Tables
# ---------------------------------------------------------------------------
def tables_case(seed, n, columns, page, spare, held, fork=0.5, ended=0.2, share=True, holes=0, want=None):
    """Tables of n sequences that share pages as forks leave them, and what they go on from."""
    rng = np.random.default_rng(seed)
    length = rng.integers(0, held + 1, n)
    needs = -(-length // page)
    table = table_of(rng, int(needs.sum()), needs, columns)
    table[np.arange(columns)[None] >= needs[:, None]] = rng.integers(-3, 1 << 20, int((np.arange(columns)[None] >= needs[:, None]).sum()))
    if share:
        for s in range(1, n):
            o = int(rng.integers(0, s))
            m = min(length[s], length[o]) // page
            if rng.random() < 0.6 and m:
                table[s, :m] = table[o, :m]
    pages = int(needs.sum()) + spare
    table = np.where(np.arange(columns)[None] < needs[:, None], rng.permutation(max(pages, 1))[table.clip(0, max(pages, 1) - 1)], table).astype(np.int32)
    for _ in range(holes):
        table[rng.integers(n), rng.integers(columns)] = (-1, pages, 2147483647, -2147483648)[rng.integers(4)]
    parent = np.where(rng.random(n) < fork, rng.integers(0, n, n), np.arange(n))
    parent = np.where(rng.random(n) < ended, rng.choice([-1, n, 2147483647, -2147483648], n), parent).astype(np.int32)
    if want is None:
        want = rng.integers(-5, held + 3 * page, n)
    return table, length.astype(np.int32), parent, np.asarray(want, np.int32), max(pages, 1)


TABLES = {
    "one sequence": dict(n=1, columns=3, page=64, spare=2, held=100),
    "one page": dict(n=2, columns=1, page=64, spare=1, held=64),
    "beams": dict(n=120, columns=8, page=64, spare=200, held=440, fork=1.0, ended=0.0),
    "requests end": dict(n=192, columns=8, page=64, spare=50, held=440, fork=0.0, ended=0.5),
    "too few pages": dict(n=60, columns=9, page=64, spare=4, held=500),
    "no free page": dict(n=30, columns=9, page=64, spare=0, held=500, ended=0.0, share=False),
    "pages that are none": dict(n=40, columns=9, page=64, spare=30, held=500, holes=40),
    "pages of one position": dict(n=20, columns=50, page=1, spare=100, held=50),
    "odd pages": dict(n=70, columns=130, page=7, spare=300, held=900),
    "many sequences": dict(n=2500, columns=4, page=64, spare=500, held=250),
    "many pages": dict(n=40, columns=700, page=16, spare=70000, held=11000),
    "far more than they can hold": dict(n=9, columns=4, page=64, spare=30, held=200, want=[2147483647, -2147483648] * 4 + [9999]),
}


@pytest.mark.parametrize("compact", [False, True], ids=["", "compact"])
@pytest.mark.parametrize("name", list(TABLES))
def test_tables(name, compact):
    from paper_2603_11273_amd import asr
    for seed in (1, 2):
        table, length, parent, want, pages = tables_case(seed * 100 + len(name), **TABLES[name])
        page = TABLES[name]["page"]
        new, lens, room, info, data = P.next_tables(table, length, parent, want, page, pages, compact)
        n, columns = table.shape
        pool = torch.randint(0, 1 << 30, (pages, 23), dtype=torch.int32, device="cuda").view(torch.uint8).view(pages, 4, 23)
        scales = torch.rand((pages, 5), device="cuda")
        c, s = host(pool).copy(), host(scales).copy()
        for a, b in data:
            c[b], s[b] = host(pool)[a], host(scales)[a]
        out = dict(new_table=i32(np.full((n, columns + 3), 77))[:, :columns], new_length=i32(np.zeros(n)), room=i32(np.zeros(n)),
                   info=i32(np.zeros(4)))
        t, l = i32(np.concatenate([table, table], 1))[:, :columns], i32(length)
        before = pool.clone(), scales.clone()
        plan = asr.PageTables(pool, scales, t, l, parent=i32(parent), want=i32(want), page=page, **out)
        for again in range(2):                       # the second call finds what the first did
            plan(compact=compact)
            for got, ref in ((out["new_table"], new), (out["new_length"], lens), (out["room"], room), (out["info"], info)):
                assert np.array_equal(host(got), ref)
            assert np.array_equal(host(pool), c) and np.array_equal(host(scales), s)
        # in place
        pool.copy_(before[0])
        scales.copy_(before[1])
        base = i32(np.concatenate([table, table], 1))
        t = base[:, :columns]
        asr.PageTables(pool, scales, t, l, parent=i32(parent), want=i32(want), page=page)(compact=compact)
        assert np.array_equal(host(t), new) and np.array_equal(host(l), lens)
        assert np.array_equal(host(base)[:, columns:], table)
        assert np.array_equal(host(pool), c) and np.array_equal(host(scales), s)


def test_tables_without_parents_wants_or_data():
    from paper_2603_11273_amd import asr
    table, length, _, _, pages = tables_case(5, 30, 6, 64, 20, 300)
    for parent, want in ((None, None), (None, 1), (1, None)):
        rng = np.random.default_rng(6)
        parent = None if parent is None else rng.integers(-1, 30, 30)
        want = None if want is None else rng.integers(0, 400, 30)
        new, lens, room, info, _ = P.next_tables(table, length, parent, want, 64, pages, True)
        t, l = i32(table), i32(length)
        asr.PageTables(None, None, t, l, parent=None if parent is None else i32(parent), want=None if want is None else i32(want),
                       page=64, pages=pages)(compact=True)
        assert np.array_equal(host(t), new) and np.array_equal(host(l), lens)
