"""Rows whose rules leave no token, in a running engine: they end, and nothing beside them does."""
import numpy as np
import pytest

from paper_2603_11273_amd import synth

from gpu_util import make_context, needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]

V = 2111


@pytest.mark.parametrize("overlap", [False, True])
def test_served_requests_end_where_their_rules_allow_nothing(overlap):
    """Three allowed tokens and a penalty that the second use of one makes infinite: six tokens are all that
    a request can have; one that asks for three has three."""
    shape, seed = synth.reduced_shape(synth.SHAPES["tiny"], 1, 2, vocab=V), 20261201
    ctx = make_context(shape, seed, max_slots=3, max_prefill=2, max_decode=3)
    ctx.bind_hypotheses(n_masks=1)
    allowed = np.zeros((1, V), bool)
    allowed[0, [5, 700, 2110]] = True
    ctx.set_masks(0, allowed)
    ctx.set_slot_rules(-1, mask=0, frequency=3.4e38)
    ctx.serve_config(max_admit=2, start_token=1, overlap=overlap)
    seconds = [6, 1, 5, 6, 1]
    for i, s in enumerate(seconds):
        ctx.submit(i, synth.pcm_clip(seed, i, 16000 * s))
    done = []
    for now in range(60):
        done += ctx.serve_step(now)["finished"]
        if len(done) == len(seconds):
            break
    assert sorted(done) == list(range(len(seconds)))
    for i, s in enumerate(seconds):
        tokens = ctx.serve_tokens(i)
        if s == 1:
            assert len(tokens) == len(set(tokens)) == 3
        else:
            assert sorted(tokens) == [5, 5, 700, 700, 2110, 2110]
    assert all(not ctx.slot_info(s)["occupied"] for s in range(3))
