"""A decode step over a paged cache and the sampler, captured into one graph and replayed, against the same step made eagerly; plans
that share a workspace; a plan on another stream than the current one."""
import numpy as np
import pytest
import torch

from gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

N, H, V, PAGE, COLUMNS, PAGES = 9, 3, 9001, 64, 12, 140


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).cuda()


class Step:
    """Tables, write, attend and sample of one step, on buffers of its own."""

    def __init__(self, seed, inputs, dtype, workspace=None):
        from paper_2603_11273_amd import asr
        g = torch.Generator(device="cuda").manual_seed(seed)
        shape = (PAGES, 2, H, PAGE // 64, 64, 64)
        self.codes = (torch.randn(shape, generator=g, device="cuda") * 60).to(torch.float8_e4m3fn).view(torch.uint8)
        self.scales = torch.full(shape[:4], 2.0 ** -6, device="cuda")
        held = np.array([0, 1, 63, 64, 65, 127, 300, 511, 640])
        table, free = np.full((N, COLUMNS), -1, np.int32), list(range(PAGES))
        for s in range(N):
            for j in range(-(-held[s] // PAGE)):
                table[s, j] = free.pop()
        self.table, self.length, self.seen = i32(table), i32(held), i32(np.zeros(N))
        self.room, self.info = i32(np.zeros(N)), i32(np.zeros(4))
        self.x, self.parent, self.want, self.u, self.logits = inputs
        self.out = torch.zeros((N, H * 64), dtype=dtype, device="cuda")
        self.token, self.kept = i32(np.zeros((N, 2))), i32(np.zeros(N))
        self.logprob = torch.zeros((N, 2), device="cuda")
        ws = {} if workspace is None else {"workspace": workspace}
        self.tables = asr.PageTables(self.codes, self.scales, self.table, self.length, parent=self.parent, want=self.want,
                                     room=self.room, info=self.info, **ws)
        self.write = asr.PageWrite(self.codes, self.scales, self.table, self.length, tokens=N, dtype=torch.float32)
        self.attend = asr.PagedAttention(self.codes, self.scales, self.table, self.seen, n_head=H, rows=N, dtype=dtype, part_keys=256,
                                         **ws)
        self.sample = asr.Sampler(N, V, torch.float32, draws=2, top_p=torch.full((N,), 0.9, device="cuda"),
                                  top_k=i32([0, 5, 900, 4000, 0, 1, 50, 0, 8000]), temperature=torch.linspace(0, 2, N, device="cuda"))

    def __call__(self):
        self.tables(compact=True)
        self.write(self.x[:, :H * 64], self.x[:, H * 64:2 * H * 64])
        torch.add(self.length, 1, out=self.seen)
        self.attend(self.x[:, 2 * H * 64:], self.out)
        self.sample(self.logits, self.u, self.token, self.logprob, self.kept)
        self.length.add_(1)

    def everything(self):
        return [self.codes, self.scales, self.table, self.length, self.room, self.info, self.out, self.token, self.kept, self.logprob]


def new_inputs(rng, inputs):
    x, parent, want, u, logits = inputs
    x.copy_(torch.from_numpy(rng.standard_normal(x.shape).astype(np.float32) * 2.0 ** rng.integers(-2, 5)))
    p = np.where(rng.random(N) < 0.3, rng.integers(0, N, N), np.arange(N))
    parent.copy_(i32(np.where(rng.random(N) < 0.1, -1, p)))
    want.copy_(i32(rng.integers(700, 720, N)))           # more than any holds: each has room for its token
    u.copy_(torch.from_numpy(rng.random(u.shape).astype(np.float32)))
    logits.copy_(torch.from_numpy((rng.standard_normal(logits.shape) * 3).astype(np.float32)))


def empty_inputs():
    return (torch.zeros((N, 3 * H * 64), device="cuda"), i32(np.arange(N)), i32(np.zeros(N)), torch.zeros((N, 2), device="cuda"),
            torch.zeros((N, V), device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_step_captured_and_replayed(dtype):
    rng = np.random.default_rng(3)
    inputs = empty_inputs()
    new_inputs(rng, inputs)
    eager, captured = Step(5, inputs, dtype), Step(5, inputs, dtype)
    eager()                                              # (the first calls outside of a graph)
    captured()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        captured()
    for _ in range(6):
        new_inputs(rng, inputs)
        graph.replay()
        eager()
        torch.cuda.synchronize()
        for a, b in zip(eager.everything(), captured.everything()):
            assert torch.equal(a, b)
        assert eager.info[1].item() == 0 and (eager.kept > 0).all()


def test_plans_that_share_a_workspace():
    """One after the other, and the counters are zeros behind every call."""
    rng = np.random.default_rng(7)
    inputs = empty_inputs()
    alone = Step(9, inputs, torch.float32)
    need = max(p.workspace_bytes for p in (alone.tables, alone.attend))
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    shared = Step(9, inputs, torch.float32, ws)
    for _ in range(3):
        new_inputs(rng, inputs)
        alone()
        shared()
        assert (ws[:4 * 4096] == 0).all()
        for a, b in zip(alone.everything(), shared.everything()):
            assert torch.equal(a, b)


def test_a_step_on_another_stream():
    rng = np.random.default_rng(11)
    inputs = empty_inputs()
    new_inputs(rng, inputs)
    here, there = Step(13, inputs, torch.bfloat16), Step(13, inputs, torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there()
    here()
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(here.everything(), there.everything()):
        assert torch.equal(a, b)
