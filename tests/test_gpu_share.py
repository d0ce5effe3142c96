"""Attention over shared keys (asr_attend_shared) against softmax attention in
64 bits, at the sizes where it can go wrong: lengths of zero, one and around a
tile's end, groups of one row and of many, query heads that share key heads,
other strides and orders, rows in no group, keys behind the lengths that hold
NaN, offsets past 32 bits, a captured and replayed call.

Tolerance of an output: softmax weights move by at most e^{2 ds} - 1 when every
score moves by at most ds, so an output moves by 2 ds (1 + ds) sum_j p_j |v_j|;
ds has the rounding of a dot product of 64 terms (64 steps of 2^-24 of
sum |q_i k_i|, and in bf16 the 2^-17 that the query's pair of bf16 values
leaves), of the exponent's argument (2^-23 of the score's distance from the
reference, at most twice the largest score) and the exponential itself (2^-22).
The weights' own rounding (2^-17 as a bf16 pair), the sums over n keys (n 2^-24)
and the joins (a few 2^-24) are relative to sum_j p_j |v_j| too.  The result is
rounded once: half a step of its type."""
import numpy as np
import pytest
import torch

from gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

F32, BF16 = torch.float32, torch.bfloat16


class Case:
    """Caches, groups and lengths on the GPU, and the same as numpy arrays."""

    def __init__(self, seed, dtype, sizes, prefix, own, heads=4, kv=4, first=0, order="heads", uncovered=0, scale=0.125,
                 kind="normal"):
        rng = np.random.default_rng(seed)
        self.dtype, self.heads, self.kv, self.scale = dtype, heads, kv, scale
        self.sizes, groups = list(sizes), len(sizes)
        covered = sum(sizes)
        self.rows = covered + uncovered
        self.prefix_len = np.array([prefix[g % len(prefix)] for g in range(groups)], np.int32)
        self.own_len = np.array([own[r % len(own)] for r in range(self.rows)], np.int32)
        self.first = np.array([(first * (r + 1)) % (first + 1) if first else 0 for r in range(self.rows)], np.int32)
        self.max_prefix, self.max_own = int(self.prefix_len.max()), int(self.own_len.max())
        self.row_of = rng.permutation(self.rows).astype(np.int32)
        self.start = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
        self.prefix_slot = rng.permutation(groups + 2)[:groups].astype(np.int32)
        self.own_slot = rng.permutation(self.rows + 2)[:self.rows].astype(np.int32)

        def cache(slots, positions):
            shape = (slots, 2, kv, positions, 64) if order == "heads" else (slots, positions, 2, kv, 64)
            t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dtype)
            return t.cuda(), (lambda x: (x[:, 0], x[:, 1])) if order == "heads" else (
                lambda x: (x[:, :, 0].transpose(1, 2), x[:, :, 1].transpose(1, 2)))
        pc, pv = cache(groups + 2, self.max_prefix + 3)
        oc, ov = cache(self.rows + 2, self.max_own + first + 3)
        self.pk, self.pv = pv(pc)
        self.ok, self.ov = ov(oc)
        # keys that no row may use
        for g in range(groups):
            for t in (self.pk, self.pv):
                t[self.prefix_slot[g], :, self.prefix_len[g]:] = float("nan")
        for r in range(self.rows):
            for t in (self.ok, self.ov):
                t[self.own_slot[r], :, :self.first[r]] = float("nan")
                t[self.own_slot[r], :, self.first[r] + self.own_len[r]:] = float("inf")
        amp = {"normal": 2.0, "sharp": 12.0, "flat": 0.0}[kind]
        self.q = torch.from_numpy((amp * rng.standard_normal((self.rows, heads * 64))).astype(np.float32)).cuda()
        self.out = torch.full((self.rows, heads * 64), 7.0, dtype=dtype, device="cuda")

    def dev(self, a):
        return torch.from_numpy(np.ascontiguousarray(a)).cuda()

    def plan(self, part_keys=0, **kw):
        from paper_2603_11273_amd import asr
        args = dict(n_head=self.heads, rows=self.rows, groups=len(self.sizes), max_group=max(max(self.sizes), 1),
                    group_start=self.dev(self.start), row_of=self.dev(self.row_of),
                    prefix_slot=self.dev(self.prefix_slot), prefix_len=self.dev(self.prefix_len),
                    max_prefix=self.max_prefix, own_slot=self.dev(self.own_slot), own_first=self.dev(self.first),
                    own_len=self.dev(self.own_len), max_own=self.max_own, scale=self.scale, part_keys=part_keys)
        args.update(kw)
        return asr.SharedAttention(self.pk, self.pv, self.ok, self.ov, **args)

    def reference(self, prefix_len=None, own_len=None):
        """(out, tolerance) in 64 bits, per covered row; rows in no group are None."""
        f = lambda t: t.detach().cpu().double().numpy()  # noqa: E731
        pk, pv, ok, ov, q = f(self.pk), f(self.pv), f(self.ok), f(self.ov), f(self.q)
        pl = self.prefix_len if prefix_len is None else prefix_len
        ol = self.own_len if own_len is None else own_len
        bf = self.dtype == BF16
        per, res = self.heads // self.kv, [None] * self.rows
        for g in range(len(self.sizes)):
            for i in range(self.start[g], self.start[g + 1]):
                r = self.row_of[i]
                out, tol = np.zeros((self.heads, 64)), np.zeros((self.heads, 64))
                for h in range(self.heads):
                    a, b = self.first[r], self.first[r] + ol[r]
                    K = np.concatenate([pk[self.prefix_slot[g], h // per, :pl[g]], ok[self.own_slot[r], h // per, a:b]])
                    V = np.concatenate([pv[self.prefix_slot[g], h // per, :pl[g]], ov[self.own_slot[r], h // per, a:b]])
                    n = len(K)
                    if n == 0:
                        continue
                    x = q[r, h * 64:(h + 1) * 64] * self.scale
                    s = K @ x
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[h] = p @ V
                    ds = (66 * 2.0 ** -24 + (2.0 ** -17 if bf else 0)) * (np.abs(K) @ np.abs(x)).max() \
                        + 2.0 ** -22 * np.abs(s).max() + 2.0 ** -22
                    w = p @ np.abs(V)
                    tol[h] = (2 * ds * (1 + ds) + (2.0 ** -17 if bf else 0) + (2 * n + 32) * 2.0 ** -24) * w \
                        + np.abs(out[h]) * (2.0 ** -8 if bf else 2.0 ** -24)
                res[r] = (out.reshape(-1), tol.reshape(-1))
        return res

    def check(self, out, **kw):
        got = out.detach().cpu().double().numpy()
        for r, want in enumerate(self.reference(**kw)):
            if want is None:
                assert (got[r] == 7.0).all(), f"row {r} is in no group and was written"
                continue
            bad = np.abs(got[r] - want[0]) > want[1]
            assert not bad.any() and not np.isnan(got[r]).any(), \
                f"row {r}: {np.abs(got[r] - want[0]).max():.3e}, allowed {want[1].max():.3e}"


CASES = {
    "one row, one key": dict(sizes=[1], prefix=[1], own=[0]),
    "one row, own key only": dict(sizes=[1], prefix=[0], own=[1]),
    "one row, one key of each": dict(sizes=[1], prefix=[1], own=[1]),
    "around a tile's end": dict(sizes=[1, 2, 3, 4, 5], prefix=[15, 16, 17, 31, 33], own=[0, 31, 32, 33, 16]),
    "around a part's end": dict(sizes=[3, 2, 5], prefix=[127, 128, 129], own=[255, 256, 257, 1]),
    "rows and groups without keys": dict(sizes=[2, 0, 3, 1], prefix=[0, 40, 0, 7], own=[0, 0, 5]),
    "no keys at all": dict(sizes=[2, 1], prefix=[0], own=[0]),
    "beams of one clip": dict(sizes=[5], prefix=[1500], own=[40, 41, 39], heads=6, kv=6, first=8),
    "16 and 17 queries": dict(sizes=[16, 17], prefix=[700], own=[3]),
    "40 queries": dict(sizes=[40, 1], prefix=[333, 500], own=[9, 0]),
    "more than 64 queries": dict(sizes=[70, 3], prefix=[260, 1000], own=[2, 130], heads=2, kv=2),
    "shared key heads": dict(sizes=[3, 1, 7], prefix=[200, 31, 1], own=[60, 0, 1], heads=8, kv=2, first=5),
    "one key head for 20": dict(sizes=[5, 2], prefix=[400], own=[33], heads=20, kv=1),
    "positions before heads": dict(sizes=[4, 2], prefix=[300, 77], own=[50, 3], order="positions", first=3),
    "rows in no group": dict(sizes=[2, 3], prefix=[130], own=[12], uncovered=4),
    "sharp scores": dict(sizes=[5, 4], prefix=[900, 100], own=[64, 7], kind="sharp"),
    "equal scores": dict(sizes=[3], prefix=[1000], own=[100], kind="flat"),
    "negative scale": dict(sizes=[3], prefix=[100], own=[30], scale=-0.3),
    "long": dict(sizes=[3, 2], prefix=[9001, 4000], own=[448, 1], heads=2, kv=2),
}


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("name", list(CASES))
def test_matches_64_bits(name, dtype):
    c = Case(sum(map(ord, name)), dtype, **CASES[name])
    plan = c.plan()
    c.check(plan(c.q, c.out))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("part", [128, 384, 8192])
def test_given_parts(dtype, part):
    c = Case(part, dtype, sizes=[3, 5, 1], prefix=[1500, 383, 0], own=[400, 0, 129], first=4)
    c.check(c.plan(part_keys=part)(c.q, c.out))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_a_row_does_not_depend_on_its_group(dtype):
    """The same row alone, among five and among 40 (other query tiles): the same bits."""
    c = Case(5, dtype, sizes=[40], prefix=[1500], own=[37, 0, 448, 129], heads=2, kv=2)
    whole = c.plan(part_keys=384)(c.q, c.out).clone()
    for rows in ([c.row_of[3]], list(c.row_of[7:12])):
        c.sizes, c.start = [len(rows)], np.array([0, len(rows)], np.int32)
        c.row_of = np.concatenate([rows, np.full(c.rows - len(rows), -1)]).astype(np.int32)
        out = torch.full_like(c.out, 7.0)
        c.plan(part_keys=384)(c.q, out)
        assert torch.equal(out[rows], whole[rows])
        others = [r for r in range(c.rows) if r not in rows]
        assert (out[others] == 7.0).all()


def test_wider_rows_and_bad_entries():
    """Rows further apart than their width; slots out of the cache have no keys, rows out of range
    are passed over, lengths past the bounds are cut."""
    c = Case(11, F32, sizes=[3, 2], prefix=[50, 60], own=[20], heads=2, kv=2, first=2)
    q = torch.zeros((c.rows, 200), device="cuda")
    q[:, :128] = c.q
    out = torch.full((c.rows, 132), 7.0, device="cuda")
    c.plan()(q[:, :128], out[:, :128])
    c.check(out[:, :128])
    assert (out[:, 128:] == 7.0).all()
    want = c.reference()
    slot = c.own_slot.copy()
    slot[c.row_of[0]], slot[c.row_of[1]] = -1, c.ok.shape[0]
    own = c.own_len.copy()
    own[c.row_of[0]] = own[c.row_of[1]] = 0
    out = torch.full_like(c.out, 7.0)
    c.plan(own_slot=c.dev(slot))(c.q, out)
    c.check(out, own_len=own)
    out = torch.full_like(c.out, 7.0)
    rows = c.row_of.copy()
    lost = rows[4]
    rows[4] = c.rows
    c.plan(row_of=c.dev(rows))(c.q, out)
    assert (out[lost] == 7.0).all() and want[lost] is not None
    out = torch.full_like(c.out, 7.0)
    c.plan(prefix_len=c.dev(np.array([1 << 30, -3], np.int32)), max_prefix=50)(c.q, out)
    c.check(out, prefix_len=np.array([50, 0]))


def test_infinite_value_and_nan_key_stay_with_their_row():
    c = Case(12, BF16, sizes=[2, 2], prefix=[40], own=[10], heads=2, kv=2)
    a, b, d = c.row_of[0], c.row_of[1], c.row_of[2]
    c.ov[c.own_slot[a], 0, 3, 5] = float("inf")
    c.ok[c.own_slot[b], 1, 2, 0] = float("nan")
    out = c.plan()(c.q, c.out)
    assert torch.isinf(out[a, 5]) and torch.isfinite(out[a, :5]).all() and torch.isfinite(out[a, 6:]).all()
    assert torch.isfinite(out[b, :64]).all() and torch.isnan(out[b, 64:]).all()
    assert torch.isfinite(out[d]).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_an_infinite_value_of_weight_one(dtype):
    c = Case(15, dtype, sizes=[1], prefix=[1], own=[0], heads=1, kv=1)
    c.pv[c.prefix_slot[0], 0, 0, :3] = torch.tensor([float("inf"), -float("inf"), 2.0]).to(dtype)
    assert c.plan()(c.q, c.out)[0, :3].tolist() == [float("inf"), -float("inf"), 2.0]


def test_offsets_past_32_bits():
    """Two slots more than 2^32 bytes apart, a group's shared keys in the far one."""
    n, gap = 300, (1 << 31) + 64
    c = Case(13, BF16, sizes=[3], prefix=[n], own=[4], heads=2, kv=2)
    block = torch.empty(gap + 2 * 2 * (n + 3) * 64, dtype=BF16, device="cuda")
    strides = (gap, (n + 3) * 64, 64, 1)
    k, v = (torch.as_strided(block, (2, 2, n + 3, 64), strides, i * 2 * (n + 3) * 64) for i in (0, 1))
    src = int(c.prefix_slot[0])
    k[1], v[1] = c.pk[src], c.pv[src]
    from paper_2603_11273_amd import asr
    out = torch.full_like(c.out, 7.0)
    asr.SharedAttention(k, v, c.ok, c.ov, n_head=2, rows=c.rows, groups=1, max_group=3, group_start=c.dev(c.start),
                        row_of=c.dev(c.row_of), prefix_slot=c.dev(np.array([1], np.int32)),
                        prefix_len=c.dev(c.prefix_len), max_prefix=n, own_slot=c.dev(c.own_slot),
                        own_len=c.dev(c.own_len), max_own=4)(c.q, out)
    c.check(out)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_capture_and_streams(dtype):
    """A captured call replayed with other lengths and queries, eager calls of a second plan in
    between, both on a stream of their own: bit-identical to eager calls."""
    c = Case(14, dtype, sizes=[4, 1, 6], prefix=[700, 30, 1500], own=[100, 3], heads=4, kv=2, first=3)
    lens = c.dev(c.prefix_len)
    plan, other = c.plan(prefix_len=lens), c.plan(prefix_len=lens)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        plan(c.q, c.out)
        eager = torch.empty_like(c.out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            plan(c.q, c.out)
        for step in range(4):
            lens.copy_(torch.tensor([700 - 97 * step, 30 // (step + 1), 1500 - step], dtype=torch.int32))
            c.q.mul_(1.01)
            c.out.zero_()
            graph.replay()
            other(c.q, eager)
            torch.cuda.synchronize()
            assert torch.equal(c.out, eager), step
    c.check(c.out, prefix_len=np.array([700 - 97 * 3, 30 // 4, 1500 - 3]))


def test_one_workspace_for_calls_of_many_sizes():
    """Attention of one part and of many, with and without own keys, and rules, one after the other over one
    block: what counts blocks in it is zeros again after every call."""
    from paper_2603_11273_amd import asr
    cases = [Case(20 + i, d, **kw) for i, (d, kw) in enumerate([
        (BF16, dict(sizes=[5], prefix=[1500], own=[40], heads=6, kv=6)), (F32, dict(sizes=[1, 3], prefix=[700, 0], own=[0, 90])),
        (BF16, dict(sizes=[20], prefix=[900], own=[5])), (F32, dict(sizes=[2], prefix=[0], own=[300, 0])),
        (BF16, dict(sizes=[1] * 9, prefix=[130, 0, 1], own=[1, 0, 500], heads=8, kv=2))])]
    size = max(c.plan().workspace_bytes for c in cases)
    block = torch.zeros(max(size, 1 << 20), dtype=torch.uint8, device="cuda")
    plans = [c.plan(workspace=block) for c in cases]
    logits = torch.randn((7, 50001), device="cuda")
    rules = [asr.LogitRules(n, 50001, F32, k=k, device="cuda:0", workspace=block) for n, k in ((7, 5), (2, 16))]
    token, logprob = (torch.zeros((7, 16), dtype=t, device="cuda") for t in (torch.int32, F32))
    want = torch.sort(logits, dim=1, descending=True, stable=True).indices
    for _ in range(3):
        for c, plan in zip(cases, plans):
            c.out.fill_(7.0)
            plan(c.q, c.out)
            for r, n, k in zip(rules, (7, 2), (5, 16)):
                r(logits[:n], token=token.view(-1)[:n * k].view(n, k), logprob=logprob.view(-1)[:n * k].view(n, k))
                assert torch.equal(token.view(-1)[:n * k].view(n, k).long(), want[:n, :k])
            assert not block[:16384].any()
    for c in cases:
        c.check(c.out)


def test_a_single_row_of_any_stride_and_refused_workspaces():
    """torch gives the stride of a dimension of one element as it likes."""
    c = Case(31, F32, sizes=[1], prefix=[70], own=[9])
    q = torch.empty((c.heads * 64, 1), device="cuda").copy_(c.q.t()).t()
    assert q.is_contiguous() and q.stride(0) == 1
    out = torch.full((c.heads * 64, 1), 7.0, device="cuda").t()
    c.plan()(q, out)
    c.check(out)
    for ws in (torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(1 << 20, device="cuda"),
               torch.zeros(1 << 21, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(TypeError):
            c.plan(workspace=ws)
