"""Plans of the stateless operators used as the documentation allows: made on one stream and called at
once on another, dropped while their call is under way."""
import numpy as np
import pytest
import torch

from gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]


def busy(n=6):
    """Some ten milliseconds of work on the current stream."""
    x = torch.ones((8192, 8192), device="cuda")
    for _ in range(n):
        x = x @ x * 2.0 ** -13
    return x


def test_called_on_another_stream_as_soon_as_made():
    """The stream that a plan's scratch is cleared on has work before it; the call does not wait for that
    stream, and its blocks' counters have to be zeros all the same.  The memory held other values before."""
    from paper_2603_11273_amd import asr
    V, k = 51866, 5
    side = torch.cuda.Stream()
    logits = torch.randn((4, V), device="cuda")
    want = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    token = torch.zeros((4, k), dtype=torch.int32, device="cuda")
    logprob = torch.zeros((4, k), device="cuda")
    busy()
    torch.cuda.synchronize()
    for _ in range(3):
        for n in (1 << 14, 1 << 16, 1 << 18, 1 << 20):
            torch.full((n,), 0x55, dtype=torch.uint8, device="cuda")
        token.zero_()
        torch.cuda.synchronize()
        x = busy()
        plan = asr.LogitRules(4, V, torch.float32, k=k, device="cuda:0")
        plan(logits, token=token, logprob=logprob, stream=side)
        side.synchronize()
        assert torch.equal(token.long(), want)
        del x


def test_scratch_outlives_a_dropped_plan():
    """A plan is dropped while its call waits on a side stream: its scratch is not given to the next tensor
    of that size."""
    from paper_2603_11273_amd import asr
    V, k = 51866, 5
    side = torch.cuda.Stream()
    logits = torch.randn((4, V), device="cuda")
    want = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    token, logprob = torch.zeros((4, k), dtype=torch.int32, device="cuda"), torch.zeros((4, k), device="cuda")
    plan = asr.LogitRules(4, V, torch.float32, k=k, device="cuda:0")
    at, n = plan._ws_ptr, plan._ws_bytes
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = busy(20)
        plan(logits, token=token, logprob=logprob)
        done = torch.cuda.Event()
        done.record()
    del plan
    taken = [torch.full((n,), 0x55, dtype=torch.uint8, device="cuda") for _ in range(4)]
    pending = not done.query()
    assert not pending or all(t.data_ptr() != at for t in taken)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(token.long(), want) and pending and np.isfinite(logprob.cpu().numpy()).all()
    del x


@pytest.mark.parametrize("slots,heads,positions", [(1, 2, 40), (3, 1, 40), (3, 2, 1), (1, 1, 1)])
def test_caches_with_dimensions_of_one_element(slots, heads, positions):
    """torch gives the stride of a dimension of one element as it likes, and k and v different ones."""
    from paper_2603_11273_amd import asr
    g = torch.Generator(device="cuda").manual_seed(slots + heads + positions)
    k, v = (torch.randn((slots, heads, positions, 64), generator=g, device="cuda") for _ in range(2))
    q = torch.randn((slots, heads * 64), generator=g, device="cuda")
    odd = [k.as_strided(k.shape, [s if n > 1 else one for n, s, one in zip(k.shape, k.stride(), (7, 5, 3, 1))])] + \
          [v.as_strided(v.shape, [s if n > 1 else one for n, s, one in zip(v.shape, v.stride(), (1, 9, 64, 1))])]
    start = torch.arange(slots + 1, dtype=torch.int32, device="cuda")
    got = []
    for kk, vv in ((k, v), odd):
        plan = asr.SharedAttention(kk, vv, n_head=heads, rows=slots, groups=slots, max_group=1, group_start=start)
        got.append(plan(q, torch.empty_like(q)))
    assert torch.equal(*got)
    q64, k64, v64 = q.cpu().double().view(slots, heads, 64), k.cpu().double(), v.cpu().double()
    p = torch.softmax((q64[:, :, None] * k64).sum(-1) / 8, -1)
    want = (p[..., None] * v64).sum(2).reshape(slots, -1)
    # (scores of a few units: 66 steps of 2^-24 of sum |q k| below 100, twice that on the weights)
    assert (got[0].cpu().double() - want).abs().max() <= 4 * 66 * 2.0 ** -24 * 100 * v64.abs().max()
