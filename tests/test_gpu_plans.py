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
