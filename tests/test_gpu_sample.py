"""Sampling (asr_sample) against its definition in 64 bits.  Tokens and counts have to be equal.  Weights are rounded to
multiples of 2^(n - 62), n at most 20, so a sum is off by at most 2^(n - 63) a token, 2^-22 of the largest weight at the very
worst and below 2^-40 of the sum at the sizes here: a row where a decision lies nearer to turning out otherwise than 2^-36 would
say nothing, and the inputs hold none.  A log-probability is rounded to float32 once (2^-24 of it), behind a logarithm and an
exponent in 64 bits."""
import numpy as np
import pytest
import torch

import page_util as P
from gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

F32, BF16 = torch.float32, torch.bfloat16


def dev(a, kind=np.float32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(kind))).cuda()


def check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, set=None, sets=None, ld=0, least=2.0 ** -36):
    """logits: a CPU tensor [rows][vocab]; parameters: lists."""
    from paper_2603_11273_amd import asr
    rows, V = logits.shape
    u = np.asarray(u, np.float32).reshape(rows, -1)
    params = {"temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p}
    plan = asr.Sampler(rows, V, logits.dtype, draws=u.shape[1], sets=sets, set=None if set is None else dev(set, np.int32), device="cuda:0",
                       **{n: dev(x, np.int32 if n == "top_k" else np.float32) for n, x in params.items() if x is not None})
    wide = torch.full((rows, V + ld), float("nan"), dtype=logits.dtype, device="cuda")
    wide[:, :V] = logits.cuda()
    token = torch.full(u.shape, -7, dtype=torch.int32, device="cuda")
    logprob, kept = torch.zeros(u.shape, device="cuda"), torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    plan(wide[:, :V], dev(u), token, logprob, kept)
    got, lp, n = token.cpu().numpy(), logprob.cpu().numpy().astype(np.float64), kept.cpu().numpy()
    l = logits.double().numpy()
    for r in range(rows):
        s = r if set is None else set[r]
        has = 0 <= s < (rows if sets is None else sets)
        one = lambda x: None if x is None or not has else np.float32(x[s])  # noqa: E731
        k = None if top_k is None or not has else int(top_k[s])
        want = P.sample(l[r], u[r], one(temperature), k, one(top_p), one(min_p))
        assert want[3] > least, f"row {r} is too near to decide: {want[3]:.1e}"
        assert n[r] == want[2], f"row {r}: kept {n[r]}, {want[2]}"
        assert got[r].tolist() == want[0], f"row {r}"
        ref = np.array(want[1], np.float64)
        assert np.array_equal(np.isnan(lp[r]), np.isnan(ref))
        fine = np.isfinite(ref)
        assert (lp[r][~fine & ~np.isnan(ref)] == ref[~fine & ~np.isnan(ref)]).all()
        assert (np.abs(lp[r] - ref)[fine] <= 2.0 ** -24 * np.abs(ref[fine]) + 2.0 ** -36).all(), f"row {r}: logprob"
    return got


def inputs(seed, rows, V, dtype, spread=3.0, draws=1):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy((rng.standard_normal((rows, V)) * spread - 4).astype(np.float32)).to(dtype)
    return x, rng.random((rows, draws)).astype(np.float32), rng


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 1000, 4095, 4096, 4097, 16383, 16385, 51865, 51866, 65536, 65537, 131071, 131073])
def test_sizes(V, dtype):
    rows = 4 if V < 20000 else 3
    x, u, rng = inputs(V, rows, V, dtype, draws=2)
    check(x, u)
    check(x, u, temperature=rng.uniform(0.2, 1.5, rows), top_k=rng.integers(1, V + 1, rows), top_p=rng.uniform(0.3, 0.99, rows),
          min_p=rng.uniform(0, 0.1, rows), ld=3)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("spread", [0.0, 0.01, 1.0, 30.0])
def test_each_filter(dtype, spread):
    """Flat rows, where nearly every token ties or is kept, to sharp ones, where one is."""
    x, u, rng = inputs(7, 6, 9001, dtype, spread)
    some = dict(temperature=rng.uniform(0.3, 2, 6), top_k=rng.choice([1, 2, 17, 4000, 9001, 99999], 6),
                top_p=rng.uniform(0.05, 0.999, 6), min_p=rng.uniform(0, 1, 6))
    for names in (["temperature"], ["top_k"], ["top_p"], ["min_p"], ["top_k", "top_p"], ["top_p", "min_p"], list(some)):
        check(x, u, **{n: some[n] for n in names})


def test_ties_at_the_cut():
    """Few values, many tokens of each: the lower tokens of equal logits are kept."""
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.integers(0, 4, (8, 5003)).astype(np.float32))
    u = rng.random((8, 3))
    for k in (1, 2, 700, 1250, 1251, 5002, 5003):
        check(x, u, top_k=[k] * 8)
    check(x, u, top_p=[0.1, 0.3, 0.5, 0.64, 0.65, 0.8, 0.95, 0.999])
    # (900 of some 1250 tokens with the largest logit: every weight is 1 and every sum exact, on a border too)
    check(x, u, least=-1, top_k=[900] * 8, top_p=[0.1, 0.3, 0.5, 0.64, 0.65, 0.8, 0.95, 0.999])


def test_parameters_that_are_off():
    x, u, _ = inputs(11, 8, 3001, F32)
    nan, inf = float("nan"), float("inf")
    check(x, u, temperature=[1, 0, -1, nan, inf, 1e-30, 1e30, 0.5])
    check(x, u, top_k=[0, -1, -2147483648, 2147483647, 1, 2, 3, 4], top_p=[nan, 1, 2, inf, 0.999, 0, -1, 1e-30],
          min_p=[nan, 0, -1, 1e-30, 1, 2, inf, 1e-6])


def test_random_numbers_at_their_ends():
    x, _, _ = inputs(13, 3, 700, F32, 1.0)
    u = np.array([[0.0, 1.0, 0.999999940395], [np.nan, -1.0, 2.0], [np.inf, 1e-38, 1 - 2.0 ** -24]], np.float32)
    check(x, u, least=-1)
    check(x, u, top_k=[5, 1, 300], least=-1)


def test_rows_that_have_no_token():
    x, u, _ = inputs(17, 9, 2050, F32, draws=3)
    x[0, 77], x[1, 2049], x[2, 0] = float("nan"), float("inf"), float("nan")
    x[3], x[4, 1:] = -float("inf"), -float("inf")
    x[5, ::2], x[6, :2000] = -float("inf"), -float("inf")
    x[7] = torch.finfo(F32).min
    x[8, 100:] = torch.finfo(F32).min
    check(x, u)
    check(x, u, top_k=[5] * 9, top_p=[0.9] * 9, min_p=[0.01] * 9, temperature=[0.7] * 9)
    check(x, u, temperature=[0.0] * 9)
    check(x, u, temperature=[float("inf")] * 9)
    check(x[:8].to(BF16), u[:8], top_k=[1500] * 8)


def test_zeros_of_either_sign_tie():
    x = torch.full((2, 300), -1.0)
    x[0, 5], x[0, 9], x[0, 200] = 0.0, -0.0, 0.0
    x[1, 5], x[1, 9], x[1, 200] = -0.0, 0.0, -0.0
    assert check(x, [[0.1], [0.9]], top_k=[1, 2]).reshape(-1).tolist() == [5, 9]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 40003])
def test_zeros_of_either_sign_are_the_largest(V, dtype):
    """Rows whose largest logits are zeros: of one sign, or of both in several parts of the row."""
    rng = np.random.default_rng(V)
    x = -np.abs(rng.standard_normal((5, V)).astype(np.float32)) - 0.5
    x[0, ::7], x[1, ::7] = -0.0, 0.0
    x[2, : V // 2 : 5], x[2, V // 2 :: 5] = -0.0, 0.0
    x[3, : V // 2 : 5], x[3, V // 2 :: 5] = 0.0, -0.0
    x[4, ::3] = np.where(rng.random(len(x[4, ::3])) < 0.5, 0.0, -0.0)
    x, u = torch.from_numpy(x).to(dtype), rng.random((5, 3)).astype(np.float32)
    for kw in ({}, dict(top_k=[7] * 5), dict(top_k=[V // 3] * 5), dict(top_p=[0.3] * 5), dict(top_k=[V // 2] * 5, top_p=[0.8] * 5),
               dict(min_p=[0.4] * 5), dict(temperature=[0.0] * 5), dict(top_k=[900] * 5)):
        check(x, u, least=-1, **kw)


@pytest.mark.parametrize("V", [9001, 60007])
def test_bf16_values(V):
    """Rows of bf16 logits that are counted by value, and those whose values lie too far apart for that."""
    rng = np.random.default_rng(V)
    rows = 9
    x = (rng.standard_normal((rows, V)) * 3 - 4).astype(np.float32)
    x[1, 100:] = -1e30                                   # masked by a large number
    x[2, 100:] = -np.inf
    x[3] = rng.integers(0, 3, V)                         # three values
    x[4] *= 2.0 ** rng.integers(-30, 6, V)               # thousands of values, tiny ones among them
    x[5] = x[5] * 100 + 3000                             # a large maximum: values down to it are out of reach
    x[6] = -np.abs(x[6]) * 1000
    x[7, ::2], x[7, 1::4] = 0.0, -0.0
    x[8] = 1e38 * np.sign(x[8])
    x = torch.from_numpy(x).to(BF16)
    u = rng.random((rows, 3)).astype(np.float32)
    k = [50, 99, 100, V // 2, 3000, 5000, 17, V // 3, V // 2 + 7]
    check(x, u, top_k=k)
    check(x, u, top_k=[101] * rows, top_p=[0.9] * rows)
    check(x, u, top_p=[0.9, 0.5, 0.99, 0.7, 0.6, 0.8, 0.3, 0.95, 0.9], temperature=[1, 2, 0.5, 1, 0.2, 30, 500, 1, 1])
    check(x, u, top_k=k, top_p=[0.97] * rows, min_p=[0.01, 0, 0.5, 0.1, 0.02, 1e-6, 0, 0.3, 0], temperature=[0.7] * rows)
    check(x, u, top_k=[V - 1] * rows, temperature=[float("inf"), 1e30, 1, 1e6, 1, 1e38, 1, 1e-3, 1])


def test_f32_rows_that_the_lists_cannot_hold():
    """Cuts among many tokens: wide distributions, many equal logits, logits in rising and falling order."""
    rng = np.random.default_rng(37)
    V, rows = 60007, 6
    x = (rng.standard_normal((rows, V)) * 0.5).astype(np.float32)
    x[1] = np.round(x[1] * 8) / 8
    x[2], x[3] = np.sort(x[2]), np.sort(x[3])[::-1]
    x[4] = 0.0
    x[5] = np.where(rng.random(V) < 0.7, 1.0, x[5])
    x = torch.from_numpy(x)
    u = rng.random((rows, 3)).astype(np.float32)
    check(x, u, top_k=[20000, 30000, 9000, 50000, 777, 44000])
    check(x, u, top_p=[0.91, 0.5, 0.99, 0.3, 0.7003, 0.95])
    # (all weights of row 4 are 1, which a min-p of 1 keeps: no distance, and nothing rounded)
    check(x, u, least=-1, top_k=[20000, 30000, 9000, 50000, 30001, 44000], top_p=[0.9, 0.6, 0.95, 0.4, 0.7003, 0.97], min_p=[0.3, 0.01, 0, 0.2, 1, 0])
    check(x, u, least=-1, min_p=[0.5, 0.6, 0.2, 0.1, 1.0, 0.9])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_one_token_holds_nearly_all(dtype):
    """What the other tokens weigh is far below a unit: the log-probability is 0 as it stands."""
    x, u, _ = inputs(41, 3, 70001, dtype, 1.0)
    x[:, 777] = 90.0
    for kw in ({}, dict(top_p=[0.5] * 3), dict(top_k=[5] * 3), dict(top_k=[5000] * 3, top_p=[0.9] * 3), dict(min_p=[0.1] * 3),
               dict(temperature=[0.0] * 3)):
        assert (check(x, u, **kw) == 777).all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_log_probabilities_near_zero(dtype):
    """A token that is all but certain: its log-probability is minus what tens of thousands of others weigh, each less than a unit."""
    x, u, _ = inputs(43, 6, 50113, dtype, 1.0)
    x[:, 31423] = torch.tensor([20.0, 24.0, 26.0, 28.0, 30.0, 34.0])
    for kw in ({}, dict(top_p=[0.99] * 6), dict(top_k=[5] * 6), dict(top_k=[40000] * 6, top_p=[0.9] * 6), dict(min_p=[0.1] * 6),
               dict(temperature=[0.0] * 6), dict(top_k=[5000] * 6)):
        assert (check(x, u, **kw) == 31423).all()


def test_parameter_sets():
    x, u, rng = inputs(19, 7, 1500, BF16, draws=2)
    check(x, u, temperature=[0.5, 1.5, 0.0], top_k=[3, 0, 50], set=[2, 0, 0, -1, 1, 3, 2147483647], sets=3)


def test_draws_of_a_row():
    """64 draws of one row are those of 64 rows of the same logits."""
    x, u, _ = inputs(23, 1, 51865, F32, draws=64)
    many = check(x, u, top_p=[0.95], temperature=[0.9])
    check(x.expand(64, -1).contiguous(), u.reshape(64, 1), top_p=[0.95] * 64, temperature=[0.9] * 64)
    assert len(set(many.reshape(-1).tolist())) > 20


def test_shares_of_many_draws():
    """4096 rows of a small distribution: counts within five deviations of their shares."""
    x = torch.log(torch.tensor([0.5, 0.25, 0.125, 0.0625, 0.0625]))[None].expand(4096, -1).contiguous()
    u = np.random.default_rng(29).random((4096, 1))
    got = np.bincount(check(x, u, least=-1).reshape(-1), minlength=5)
    share = np.array([0.5, 0.25, 0.125, 0.0625, 0.0625])
    assert (np.abs(got - 4096 * share) <= 5 * np.sqrt(4096 * share * (1 - share))).all()


def test_captured_and_replayed():
    from paper_2603_11273_amd import asr
    V = 51866
    x, u, _ = inputs(31, 4, V, F32)
    logits, rnd = x.cuda(), dev(u)
    params = dict(temperature=dev([0.5, 0.9, 1.1, 0.0]), top_p=dev([0.9] * 4), top_k=dev([0, 50, 1000, 0], np.int32))
    outs = [(torch.zeros((4, 1), dtype=torch.int32, device="cuda"), torch.zeros((4, 1), device="cuda"),
             torch.zeros(4, dtype=torch.int32, device="cuda")) for _ in range(2)]
    plans = [asr.Sampler(4, V, F32, **params) for _ in range(2)]
    plans[0](logits, rnd, *outs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        plans[1](logits, rnd, *outs[1])
    for step in range(4):
        logits.copy_(inputs(40 + step, 4, V, F32)[0].cuda())
        rnd.copy_(dev(inputs(50 + step, 4, 1, F32)[1]))
        for t in outs[1]:
            t.zero_()
        graph.replay()
        plans[0](logits, rnd, *outs[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs))
