"""Rules on logits and the k best tokens (asr_logit_rules) against the definition.

The processed logits are float32 operations rounded one by one, so they and the
chosen tokens are compared bit for bit with the same operations in numpy.  The
log-probabilities are compared with 64 bits; their tolerance: 2^-24 of L = M +
log sum (one rounding; where |M| is 4096 or more, of z - M instead) and of the
result, 2^-23 of the logarithm, and a relative error of the sum that the
logarithm turns into an absolute one: at most 48 additions follow one another
(16 in a lane, then trees over lanes, waves and blocks of up to 13 lists), the
exponential is off by 2^-22 and its argument by 2^-23 of z - M, weighted with
the probabilities."""
import numpy as np
import pytest
import torch

from gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

F32, BF16 = torch.float32, torch.bfloat16
f = np.float32


def pack(allowed):
    """Bool [masks][vocab] as int32 words."""
    n, V = allowed.shape
    bits = np.zeros((n, (V + 31) // 32 * 32), np.uint8)
    bits[:, :V] = allowed
    return np.packbits(bits, axis=1, bitorder="little").view(np.int32)


def processed(logits, rules, r, V):
    """z of row r, float32, by the definition."""
    z = logits.astype(f).copy()
    s = int(rules["set"][r]) if "set" in rules else r
    n_sets = rules.get("sets", 10 ** 9)
    if s < 0 or s >= n_sets:
        return z
    if "history" in rules:
        n = min(max(int(rules["history_len"][s]), 0), rules["history"].shape[1])
        p = int(rules["prompt_len"][s]) if "prompt_len" in rules else 0
        h = rules["history"][s, :n]
        inside = (h >= 0) & (h < V)
        for v in np.unique(h[inside]):
            if "repetition" in rules:
                z[v] = z[v] / rules["repetition"][s] if z[v] > 0 else z[v] * rules["repetition"][s]
            c = int((h[max(p, 0):] == v).sum())
            if c:
                if "frequency" in rules:
                    z[v] = z[v] - rules["frequency"][s] * f(c)
                if "presence" in rules:
                    z[v] = z[v] - rules["presence"][s]
    if "bias_token" in rules:
        n = min(max(int(rules["bias_len"][s]), 0), rules["bias_token"].shape[1])
        total = np.zeros(V, f)
        for t, b in zip(rules["bias_token"][s, :n], rules["bias_value"][s, :n]):
            if 0 <= t < V:
                total[t] = total[t] + b
        z = z + total
    if "allowed" in rules:
        m = int(rules["mask_of"][s]) if "mask_of" in rules else s
        if 0 <= m < len(rules["allowed"]):
            z[~rules["allowed"][m]] = -np.inf
    if "temperature" in rules and rules["temperature"][s] > 0:
        z = z / rules["temperature"][s]
    return z


def best(z, k):
    """Tokens and 64-bit log-probabilities, (z - M) - log sum e^{z - M}, with their tolerances.  (Not
    z - (M + log sum): next to M = -3.4e38 even 64 bits, whose step there is 2^75, lose the logarithm.)"""
    key = np.where(np.isnan(z), np.inf, z).astype(np.float64)
    order = np.lexsort((np.arange(len(z)), -key, ~np.isnan(z)))[:k]
    token, logp, tol = np.full(k, -1), np.full(k, -np.inf), np.zeros(k)
    with np.errstate(invalid="ignore"):
        M = np.max(z[~np.isnan(z)], initial=-np.inf).astype(np.float64)
        if np.isnan(z).any() or M == np.inf:
            log_sum, off = np.nan, 0.0
        elif M == -np.inf:
            log_sum, off = -np.inf, 0.0
        else:
            e = np.exp(z.astype(np.float64) - M)
            d = np.where(e > 0, np.abs(z.astype(np.float64) - M), 0.0)
            off = float((e * np.where(np.isfinite(d), d, 0)).sum() / e.sum()) * 2.0 ** -22 + 48 * 2.0 ** -24 + 2.0 ** -22
            log_sum = np.log(e.sum())
    for i, v in enumerate(order):
        if not z[v] == -np.inf:
            token[i], logp[i] = v, (z[v].astype(np.float64) - M) - log_sum
            if np.isfinite(log_sum):
                rounded = abs(M + log_sum) if abs(M) < 4096 else abs(z[v] - M)
                tol[i] = off + 2.0 ** -24 * (rounded + abs(logp[i])) + 2.0 ** -23 * abs(log_sum)
    return token, logp, tol


def run(logits, rules, k, dtype=F32, out=True, in_place=False, ld=None):
    """(out, token, logprob) of the library, as numpy; logits float32 numpy [rows][V]."""
    from paper_2603_11273_amd import asr
    rows, V = logits.shape
    x = torch.empty((rows, ld or V), dtype=dtype, device="cuda").fill_(float("nan"))
    x[:, :V] = torch.from_numpy(logits).to(dtype)
    dev = {n: torch.from_numpy(np.ascontiguousarray(a)).cuda() for n, a in rules.items()
           if isinstance(a, np.ndarray) and n != "allowed"}
    if "allowed" in rules:
        dev["mask"] = torch.from_numpy(pack(rules["allowed"])).cuda()
    plan = asr.LogitRules(rows, V, dtype, k=k, sets=rules.get("sets"), device="cuda:0", **dev)
    view = x[:, :V]
    z = view if in_place else torch.full((rows, (ld or V) + 1), 7.0, device="cuda")[:, :V] if out else None
    token = torch.full((rows, k), -9, dtype=torch.int32, device="cuda")
    logprob = torch.full((rows, k), 9.0, device="cuda")
    plan(view, out=z, token=token if k else None, logprob=logprob if k else None)
    torch.cuda.synchronize()
    return (None if z is None else z.cpu().numpy(), token.cpu().numpy(), logprob.cpu().numpy(), dev)


def check(logits, rules, k, dtype=F32, **kw):
    rows, V = logits.shape
    seen = torch.from_numpy(logits).to(dtype).float().numpy()
    z, token, logprob, _ = run(logits, rules, k, dtype, **kw)
    for r in range(rows):
        want = processed(seen[r], rules, r, V)
        if z is not None:
            assert np.array_equal(z[r], want, equal_nan=True), f"row {r}: {np.flatnonzero(~(z[r] == want))[:5]}"
        if k:
            t, lp, tol = best(want, k)
            assert np.array_equal(token[r], t), f"row {r}"
            fine = np.isfinite(lp)
            assert np.array_equal(np.isnan(logprob[r]), np.isnan(lp)) and (logprob[r][~fine & ~np.isnan(lp)] == -np.inf).all()
            off = np.abs(logprob[r][fine] - lp[fine])
            assert (off <= tol[fine]).all(), f"row {r}: {off.max():.3e} of {tol.max():.3e}"


def all_rules(rng, rows, V, n=40, b=12, masks=3, **skip):
    r = {"history": rng.integers(0, V, (rows, n)).astype(np.int32),
         "history_len": rng.integers(0, n + 1, rows).astype(np.int32),
         "prompt_len": rng.integers(0, n + 1, rows).astype(np.int32),
         "repetition": rng.uniform(0.7, 1.6, rows).astype(f), "frequency": rng.uniform(-0.2, 0.6, rows).astype(f),
         "presence": rng.uniform(-0.5, 1.0, rows).astype(f),
         "bias_token": rng.integers(0, V, (rows, b)).astype(np.int32),
         "bias_value": rng.uniform(-5, 5, (rows, b)).astype(f), "bias_len": rng.integers(0, b + 1, rows).astype(np.int32),
         "allowed": rng.random((masks, V)) < 0.7, "mask_of": rng.integers(-1, masks + 1, rows).astype(np.int32),
         "temperature": rng.uniform(0.2, 2.0, rows).astype(f)}
    return {n: a for n, a in r.items() if n not in skip}


def normal(rng, rows, V):
    return (3 * rng.standard_normal((rows, V)) - 2).astype(f)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,k", [(1, 1, 1), (1, 1, 16), (3, 5, 3), (2, 31, 16), (5, 33, 5), (4, 4095, 2), (4, 4096, 10),
                                      (4, 4097, 16), (7, 8200, 1), (3, 51865, 1), (5, 51866, 10), (2, 131071, 16)])
def test_all_rules(rows, V, k, dtype):
    rng = np.random.default_rng(rows * V + k)
    check(normal(rng, rows, V), all_rules(rng, rows, V), k, dtype)


@pytest.mark.parametrize("names", [(), ("history", "history_len", "repetition"), ("history", "history_len", "frequency"),
                                   ("history", "history_len", "prompt_len", "presence"),
                                   ("bias_token", "bias_value", "bias_len"), ("allowed", "mask_of"), ("temperature",)],
                         ids=lambda n: n[0] if n else "none")
def test_each_rule_alone(names):
    rng = np.random.default_rng(len(names) + 1)
    rules = {n: a for n, a in all_rules(rng, 6, 9001).items() if n in names}
    check(normal(rng, 6, 9001), rules, 4)


def test_largest_vocabulary():
    """256 lists a row: every lane of the join goes down four."""
    rng = np.random.default_rng(3)
    logits = normal(rng, 2, 1 << 20)
    logits[0, -16:] = 40 + np.arange(16)
    logits[1, ::70000] = 50.0
    check(logits, all_rules(rng, 2, 1 << 20), 16)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_ties_take_the_lower_token(dtype):
    V = 9000
    logits = np.zeros((4, V), f)
    logits[1, ::2] = -0.0                                     # 0 and -0 are equal
    logits[2] = np.repeat(np.arange(V // 10), 10)[::-1]       # ten of each
    logits[3, [8999, 17, 4096, 4095]] = 3.0
    check(logits, {}, 16, dtype)


def test_rows_with_nothing_left_infinities_and_nan():
    V = 5000
    rng = np.random.default_rng(4)
    logits = normal(rng, 7, V)
    allowed = np.zeros((3, V), bool)
    allowed[1, [4, 4500]] = True
    allowed[2] = True
    logits[1, 7] = np.nan                                     # masked: gone
    logits[2, 7] = np.nan                                     # allowed: first, and every probability is a NaN
    logits[3, 9] = np.inf
    logits[4] = -np.inf                                       # nothing but -inf
    logits[5, :] = np.finfo(f).min                            # the type's lowest value is a value
    logits[6, 1] = np.inf                                     # masked
    rules = {"allowed": allowed, "mask_of": np.array([0, 1, 2, 2, 2, 2, 1], np.int32)}
    check(logits, rules, 5)
    z, token, logprob, _ = run(logits, rules, 5)
    assert (token[0] == -1).all() and (logprob[0] == -np.inf).all() and (z[0] == -np.inf).all()
    assert list(token[1][:2]) in ([4, 4500], [4500, 4]) and (token[1][2:] == -1).all()
    assert token[2, 0] == 7 and np.isnan(logprob[2]).all()
    assert (token[4] == -1).all()


def test_lists_with_repeats_and_tokens_outside():
    """A token given three biases has their sum in list order; tokens outside the vocabulary, negative
    lengths and lengths past the row are passed over or cut."""
    V = 4100
    rng = np.random.default_rng(5)
    rules = all_rules(rng, 5, V, n=64, b=70, masks=1)
    rules["bias_token"][:, :] = rng.integers(4090, 4100, (5, 70))
    rules["bias_token"][:, ::7] = [-1, V, 1 << 30, -(1 << 31), V + 3, 4099, 0, 4096, -7, V]
    rules["bias_value"][:] = rng.uniform(-1e3, 1e3, (5, 70))
    rules["bias_len"][:] = [70, 1 << 30, -5, 0, 69]
    rules["history"][:, ::5] = -1
    rules["history"][:, 1::9] = V
    rules["history"][1] = 77
    rules["history_len"][:] = [64, 64, -1, 1 << 30, 1]
    rules["prompt_len"][:] = [0, 3, 0, 64, -4]
    check(normal(rng, 5, V), rules, 8)


def test_rows_that_share_sets_and_rows_without():
    rng = np.random.default_rng(6)
    rules = all_rules(rng, 3, 5000)
    rules["set"] = np.array([2, 2, 0, -1, 3, 1, 0], np.int32)
    rules["sets"] = 3
    check(normal(rng, 7, 5000), rules, 3)


def test_long_history():
    rng = np.random.default_rng(7)
    rules = all_rules(rng, 3, 40000, n=70001)
    rules["history"][0] %= 50                                 # counts in the thousands
    rules["history_len"][:] = [70001, 69999, 4097]
    rules["prompt_len"][:] = [2049, 0, 4096]
    check(normal(rng, 3, 40000), rules, 5)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("ld", [5003, 5008])
def test_rows_apart(dtype, ld):
    rng = np.random.default_rng(8)
    check(normal(rng, 5, 5001), all_rules(rng, 5, 5001), 3, dtype, ld=ld)


def test_in_place_and_without_candidates():
    rng = np.random.default_rng(9)
    check(normal(rng, 5, 8195), all_rules(rng, 5, 8195), 3, in_place=True)
    check(normal(rng, 5, 8195), all_rules(rng, 5, 8195), 0)
    check(normal(rng, 5, 8195), all_rules(rng, 5, 8195), 2, out=False)


def test_no_temperature_below_or_at_zero():
    rng = np.random.default_rng(10)
    check(normal(rng, 4, 100), {"temperature": np.array([0.0, -1.0, np.nan, 1.0], f)}, 3)


def test_a_row_does_not_depend_on_its_batch():
    """The same logits and rules at other places of a batch (other alignments of an odd row; 40 rows, which
    another kernel joins): the same bits."""
    rng = np.random.default_rng(11)
    V, one = 51865, normal(np.random.default_rng(1), 1, 51865)
    for dtype in (F32, BF16):
        got = []
        for rows, at in ((1, 0), (4, 1), (4, 2), (6, 5), (40, 33)):
            logits = normal(rng, rows, V)
            logits[at] = one
            rules = all_rules(np.random.default_rng(2), 1, V)
            rules["set"], rules["sets"] = np.zeros(rows, np.int32), 1
            z, token, logprob, _ = run(logits, rules, 7, dtype)
            got.append((z[at], token[at], logprob[at]))
        for g in got[1:]:
            assert all(np.array_equal(a, b) for a, b in zip(g, got[0]))


def test_capture_and_replay():
    from paper_2603_11273_amd import asr
    rng = np.random.default_rng(12)
    V, rows, k = 20001, 5, 6
    rules = all_rules(rng, rows, V)
    dev = {n: torch.from_numpy(a).cuda() for n, a in rules.items() if n != "allowed"}
    dev["mask"] = torch.from_numpy(pack(rules["allowed"])).cuda()
    x = torch.from_numpy(normal(rng, rows, V)).cuda()

    def buffers():
        return dict(out=torch.zeros((rows, V), device="cuda"), token=torch.zeros((rows, k), dtype=torch.int32, device="cuda"),
                    logprob=torch.zeros((rows, k), device="cuda"))
    plan, other, a, b = asr.LogitRules(rows, V, F32, k=k, **dev), asr.LogitRules(rows, V, F32, k=k, **dev), buffers(), buffers()
    plan(x, **a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan(x, **a)
    for step in range(4):
        x.copy_(torch.from_numpy(normal(rng, rows, V)))
        dev["history_len"].copy_(torch.from_numpy(rng.integers(0, 41, rows).astype(np.int32)))
        for t in a.values():
            t.zero_()
        graph.replay()
        other(x, **b)
        torch.cuda.synchronize()
        assert all(torch.equal(a[n], b[n]) for n in a), step


def test_a_single_row_of_any_stride():
    from paper_2603_11273_amd import asr
    x = torch.from_numpy(normal(np.random.default_rng(13), 1, 5001)).cuda()
    column = torch.empty((5001, 1), device="cuda").copy_(x.t())
    plan = asr.LogitRules(1, 5001, F32, k=3, device="cuda:0")
    got = []
    for logits in (x, column.t()):
        token, logprob = torch.empty((1, 3), dtype=torch.int32, device="cuda"), torch.empty((1, 3), device="cuda")
        plan(logits, torch.empty((5001, 1), device="cuda").t(), token, logprob)
        got.append((token, logprob))
    assert column.t().stride(0) == 1 and torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [300, 4096])
def test_many_biases(n, dtype):
    """Hundreds of biases on few tokens and on many, sums in list order across the whole list."""
    V = 20011
    rng = np.random.default_rng(14)
    rules = all_rules(rng, 4, V, n=n, b=777)
    rules["bias_token"][0] = rng.integers(8100, 8300, 777)
    rules["bias_token"][1] = rng.integers(0, 3, 777) * 5000
    rules["bias_value"][:] = rng.uniform(-1e3, 1e3, (4, 777))
    rules["bias_len"][:] = [777, 770, 321, 65]
    check(normal(rng, 4, V), rules, 6, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_divisions_of_any_size(dtype):
    """Quotients are float32's own: ordinary values, all exponents, zeros, values at the range's ends."""
    rng = np.random.default_rng(15)
    by = np.array([0.7, np.float32(1) / 3, 1.9999999, 1.0000001, 2.0 ** -20, 2.0 ** 20, 1e-25, 1e25, 3.0, np.inf], f)
    rows, V = len(by), 9001
    x = normal(rng, rows, V)
    wild = (rng.standard_normal((rows, V)) * np.exp2(rng.uniform(-140, 126, (rows, V)))).astype(f)
    x[:, 4500:] = wild[:, 4500:]                            # whole waves of them, and some among ordinary ones
    x[:, :2000:50] = wild[:, :2000:50]
    x[:, 2000:4000:7] = 0.0
    rules = {"temperature": by, "history": rng.integers(0, V, (rows, 3000)).astype(np.int32),
             "history_len": np.full(rows, 3000, np.int32), "repetition": by[::-1].copy(),
             "allowed": rng.random((1, V)) < 0.9, "mask_of": np.zeros(rows, np.int32)}
    with np.errstate(all="ignore"):
        check(x, rules, 0, dtype)
        check(x, {"temperature": by}, 0, dtype)
