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


@pytest.mark.parametrize("k", [0, 4])
def test_a_search_goes_on_beside_a_dead_end(k):
    """Of three hypotheses one comes to a mask that allows nothing: the error holds the others' results, and
    they are those of a step without the dead one."""
    from paper_2603_11273_amd import asr
    shape, seed = synth.reduced_shape(synth.SHAPES["base"], 0, 2, vocab=V, dtype="bf16"), 20261202
    got = []
    for dead in (False, True):
        ctx = make_context(shape, seed, max_slots=4, max_prefill=1, max_decode=4)
        ctx.bind_hypotheses(n_masks=2)
        ctx.set_masks(1, np.ones((1, V), bool))      # (row 0 stays as bound: nothing)
        ctx.debug_set_encoder_out([0], [-1], [40], synth.encoder_output(seed, 0, shape.d_model).numpy()[None])
        ctx.step(slots=[0], tokens=[3])
        for s in (1, 2):
            ctx.fork_slot(0, s)
            ctx.set_slot_rules(s, repetition=1.2, mask=1)
        ctx.set_slot_rules(0, presence=0.5)
        ctx.set_slot_mask(1, 0 if dead else 1)
        rows = []
        for t in (5, 6):
            if dead:
                with pytest.raises(asr.AsrError) as e:
                    ctx.step(slots=[0, 1, 2], tokens=[t, t + 1, t + 2], want_logits=True, topk=k)
                out = e.value.results
                assert e.value.status == asr.ASR_EDEVICE and out["argmax"][1] == -1
                if k:
                    assert (out["top_token"][1] == -1).all() and (out["top_logprob"][1] == -np.inf).all()
            else:
                out = ctx.step(slots=[0, 1, 2], tokens=[t, t + 1, t + 2], want_logits=True, topk=k)
            rows.append([out[n][i] for n in ("argmax", "logits") + (("top_token", "top_logprob") if k else ())
                         for i in (0, 2)] + [out["logits"][1]])
            assert ctx.slot_info(1)["position"] == t - 3
        got.append(rows)
    for a, b in zip(*got):
        assert all(np.array_equal(x, y) for x, y in zip(a, b))
