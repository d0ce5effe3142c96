"""Forked slots and per-slot rules through the C ABI, against slots that decode
the same tokens alone and against the oracle: families of hypotheses that share
audio and prompt, forks of forks, released roots, other rows beside them, the
best tokens under rules, and beam search over all of it."""
import numpy as np
import pytest

from oracle import whisper as OW
from paper_2603_11273_amd import synth

from gpu_util import TOL, cpu_params, make_context, needs_gpu, rel_err
from test_gpu_rules import best, processed

pytestmark = [pytest.mark.gpu, needs_gpu]

V = 2111


def shape_of(name, dtype):
    return synth.reduced_shape(synth.SHAPES[name], 0, 2, vocab=V, dtype=dtype)


def context(shape, seed, slots, clips=2, rows=None, **hyp):
    ctx = make_context(shape, seed, max_slots=slots, max_prefill=2, max_decode=rows or slots)
    if hyp.pop("bind", True):
        ctx.bind_hypotheses(**hyp)
    E = np.stack([synth.encoder_output(seed, b, shape.d_model).numpy() for b in range(clips)])
    ctx.debug_set_encoder_out(list(range(clips)), [-1] * clips, [40] * clips, E)
    return ctx, E


class Alone:
    """The oracle's sequence of one hypothesis."""

    def __init__(self, shape, P, ckv):
        self.args, self.ckv, self.st = (P, shape.n_dec, shape.n_head), ckv, OW.DecoderState(shape.n_dec, shape.d_model)
        self.tokens = []

    def prefill(self, kv, n):
        """Keys and values [n_dec][2][heads][448][64] of n positions whose tokens nobody knows."""
        self.tokens = [-1] * n
        for l in range(kv.shape[0]):
            for which, cache in ((0, self.st.k), (1, self.st.v)):
                cache[l] = kv[l, which, :, :n].astype(np.float64).transpose(1, 0, 2).reshape(n, -1)

    def step(self, token):
        P, n_dec, n_head = self.args
        self.tokens.append(int(token))
        return OW.decoder_step(int(token), self.st, self.ckv, P, n_dec, n_head)


def clone(seq):
    new = Alone.__new__(Alone)
    new.args, new.ckv, new.tokens = seq.args, seq.ckv, list(seq.tokens)
    import copy
    new.st = copy.deepcopy(seq.st)
    return new


@pytest.mark.parametrize("name,dtype", [("tiny", "f32"), ("base", "bf16")])
@pytest.mark.parametrize("graphs", [False, True])
@pytest.mark.parametrize("prompt", [0, 130])
def test_families_follow_the_oracle(name, dtype, graphs, prompt):
    """Two clips, with and without a prompt so long that a family shares it; clip 0 grows a family of five
    over forks of the root and of a hypothesis, and loses its root; clip 1 decodes beside it alone."""
    shape, seed = shape_of(name, dtype), 20261101
    ctx, E = context(shape, seed, 8)
    ctx.set_decode_graphs(graphs)
    P = cpu_params(shape, seed, bf16_rounded=dtype == "bf16")
    ckv = [OW.cross_kv(e.astype(np.float64), P, shape.n_dec) for e in E]
    seqs = {0: Alone(shape, P, ckv[0]), 1: Alone(shape, P, ckv[1])}
    rng = np.random.default_rng(seed)
    if prompt:
        for s in (0, 1):
            kv = synth.self_kv_prefix(seed, s, shape.n_dec, shape.n_head).numpy()
            ctx.debug_set_self_kv(s, kv, prompt)
            seqs[s].prefill(kv, prompt)

    def step(slots):
        tokens = rng.integers(0, V, len(slots))
        out = ctx.step(slots=slots, tokens=tokens, want_logits=True)
        for i, s in enumerate(slots):
            ref = seqs[s].step(tokens[i])
            assert rel_err(out["logits"][i], ref) <= TOL[dtype], f"slot {s} at {len(seqs[s].tokens)}"
            assert out["argmax"][i] == int(np.argmax(out["logits"][i]))
            assert ctx.slot_info(s)["position"] == len(seqs[s].tokens)

    def fork(src, dst):
        ctx.fork_slot(src, dst)
        seqs[dst] = clone(seqs[src])

    fork(0, 5)                                     # nothing decoded yet: only the audio is shared
    step([5, 0, 1])
    ctx.release_slot(5)
    del seqs[5]
    for _ in range(3):
        step([1, 0])
    fork(0, 2)
    fork(0, 3)
    for _ in range(3):
        step([3, 1, 0, 2])                         # the family's rows in no order, another row among them
    fork(3, 4)                                     # after 1 + 3 + 3 tokens, three of its own: copied
    fork(0, 5)
    for _ in range(2):
        step([0, 1, 2, 3, 4, 5])
    kv, own = ctx.debug_get_kv(4, 0), ctx.debug_get_kv(3, 0)
    assert np.array_equal(kv[:, :, :, :prompt + 7], own[:, :, :, :prompt + 7])
    assert not np.array_equal(kv[:, :, :, prompt + 7], own[:, :, :, prompt + 7])
    ctx.release_slot(0)                            # its caches stay: 2 to 5 read them
    del seqs[0]
    for _ in range(2):
        step([4, 2, 5, 3])
    step([1, 4])
    assert np.array_equal(ctx.debug_get_kv(2, 1), ctx.debug_get_kv(5, 1))
    for s in (2, 3, 5):
        ctx.release_slot(s)
        del seqs[s]
    step([4, 1])                                   # the last one reads its root's caches still


@pytest.mark.parametrize("prompt", [0, 200])
def test_rows_beside_a_family_and_hypotheses_of_any_batch_keep_their_bits(prompt):
    shape, seed = shape_of("base", "bf16"), 20261102
    got = []
    for plan in ("alone", "family"):
        ctx, _ = context(shape, seed, 8, bind=plan == "family")
        if prompt:
            ctx.debug_set_self_kv(0, synth.self_kv_prefix(seed, 0, shape.n_dec, shape.n_head).numpy(), prompt)
        rows = []
        for t in (5, 6, 7, 8):
            if plan == "family" and t == 6:
                for dst in (2, 3, 4, 5, 6):
                    ctx.fork_slot(0, dst)
            slots = [1] if plan == "alone" else [0, 1] if t < 6 else [2, 0, 3, 1, 4, 5, 6]
            out = ctx.step(slots=slots, tokens=[t] * len(slots), want_logits=True)
            rows.append(out["logits"][slots.index(1)])
            if t > 5 and plan == "family":           # the same token everywhere: the same bits everywhere
                for i, s in enumerate(slots):
                    if s != 1:
                        assert np.array_equal(out["logits"][i], out["logits"][0])
        got.append(rows)
        if plan == "family":                         # two of the seven: the bits that all seven have together
            kept = ctx.step(slots=[4, 5], tokens=[9, 9], want_logits=True)["logits"]
            rest = ctx.step(slots=[0, 2, 3, 6], tokens=[9] * 4, want_logits=True)["logits"]
            assert all(np.array_equal(x, kept[0]) for x in (kept[1], *rest))
    assert all(np.array_equal(a, b) for a, b in zip(*got))


def test_a_large_family():
    """40 hypotheses of one prompt (queries for every size of tile) give the bits that two of them give."""
    shape, seed = shape_of("base", "bf16"), 20261107
    got = []
    for n in (2, 20, 40):
        ctx, _ = context(shape, seed, 40, clips=1)
        ctx.debug_set_self_kv(0, synth.self_kv_prefix(seed, 0, shape.n_dec, shape.n_head).numpy(), 150)
        for dst in range(1, n):
            ctx.fork_slot(0, dst)
        for t in (5, 6, 7):
            out = ctx.step(slots=list(range(n)), tokens=[t] * n, want_logits=True, topk=3)
        assert all(np.array_equal(x, out["logits"][0]) for x in out["logits"])
        got.append((out["logits"][0], out["top_token"][n - 1], out["top_logprob"][n - 1]))
    assert all(np.array_equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))


def test_taken_and_held_slots():
    from paper_2603_11273_amd import asr
    shape, seed = shape_of("tiny", "f32"), 20261103
    ctx, E = context(shape, seed, 4, bind=False)

    def refused(status, f, *a, **kw):
        with pytest.raises(asr.AsrError) as e:
            f(*a, **kw)
        assert e.value.status == status, e.value

    refused(asr.ASR_ESTATE, ctx.fork_slot, 0, 2)
    refused(asr.ASR_ESTATE, ctx.set_slot_rules, 0)
    refused(asr.ASR_ESTATE, ctx.set_slot_mask, 0, 0)
    refused(asr.ASR_ESTATE, ctx.set_masks, 0, np.ones((1, V), bool))
    refused(asr.ASR_ESTATE, ctx.step, slots=[0], tokens=[1], topk=2)
    ctx.bind_hypotheses(max_bias=2, n_masks=1)
    for src, dst in ((2, 3), (0, 0), (0, 4), (0, -1), (-1, 2), (4, 2)):
        refused(asr.ASR_EINVAL, ctx.fork_slot, src, dst)
    refused(asr.ASR_EFULL, ctx.fork_slot, 0, 1)
    ctx.step(slots=[0], tokens=[3])
    ctx.fork_slot(0, 2)
    refused(asr.ASR_ESTATE, ctx.bind_hypotheses)
    kv = np.zeros((shape.n_dec, 2, shape.n_head, 448, 64), np.float32)
    refused(asr.ASR_EINVAL, ctx.debug_set_self_kv, 0, kv, 1)
    refused(asr.ASR_EINVAL, ctx.debug_set_self_kv, 2, kv, 1)
    refused(asr.ASR_EINVAL, ctx.debug_set_encoder_out, [0], [-1], [5], E[:1])
    ctx.release_slot(0)
    refused(asr.ASR_EINVAL, ctx.fork_slot, 0, 3)          # released
    refused(asr.ASR_EFULL, ctx.fork_slot, 2, 0)           # but its caches are read
    refused(asr.ASR_EINVAL, ctx.debug_set_encoder_out, [0], [-1], [5], E[:1])
    ctx.debug_set_encoder_out([2], [-1], [5], E[1:])       # a sequence of its own now: slot 0 is free
    ctx.debug_set_encoder_out([0], [-1], [5], E[:1])
    bad = [dict(repetition=0.0), dict(temperature=-1.0), dict(frequency=float("nan")), dict(presence=float("inf")),
           dict(n_prompt=-1), dict(mask=1), dict(mask=-2), dict(bias=[(1, 1.0)] * 3), dict(bias=[(V, 1.0)]),
           dict(bias=[(1, float("nan"))])]
    for kw in bad:
        refused(asr.ASR_EINVAL, ctx.set_slot_rules, 0, **kw)
    refused(asr.ASR_EINVAL, ctx.set_slot_rules, 3)
    refused(asr.ASR_EINVAL, ctx.set_slot_mask, 0, 1)
    refused(asr.ASR_EINVAL, ctx.set_masks, 1, np.ones((1, V), bool))
    refused(asr.ASR_EINVAL, ctx.step, slots=[0], tokens=[1], topk=17)
    # a mask that was never written allows nothing
    ctx.set_slot_rules(0, mask=0)
    refused(asr.ASR_EDEVICE, ctx.step, slots=[0], tokens=[1])


@pytest.mark.parametrize("name,dtype", [("tiny", "f32"), ("base", "bf16")])
def test_rules_of_slots(name, dtype):
    """Each row's best tokens are those of its own logits under its own rules; rows without rules keep
    their argmax; a fork takes its rules and history along; a slot filled anew starts with the defaults."""
    shape, seed = shape_of(name, dtype), 20261104
    ctx, E = context(shape, seed, 5, max_bias=6, n_masks=3)
    rng = np.random.default_rng(seed)
    allowed = rng.random((3, V)) < np.array([0.9, 0.3, 0.02])[:, None]
    ctx.set_masks(0, allowed)
    f = np.float32
    rules = {0: dict(repetition=1.3, frequency=0.25, presence=0.125, n_prompt=2, mask=1, temperature=0.7,
                     bias=[(7, 2.5), (11, -1.0), (7, 0.5)]), 1: None}
    ctx.set_slot_rules(0, **rules[0])
    said = {0: [], 1: []}

    def want(slot, logits):
        r = rules[slot]
        if r is None:
            return logits.astype(f)
        toks = np.array([b[0] for b in r.get("bias", ())] or [0], np.int32)
        vals = np.array([b[1] for b in r.get("bias", ())] or [0], f)
        return processed(logits, {
            "history": np.array([said[slot]], np.int32), "history_len": [len(said[slot])], "prompt_len": [r.get("n_prompt", 0)],
            "repetition": [f(r.get("repetition", 1))], "frequency": [f(r.get("frequency", 0))],
            "presence": [f(r.get("presence", 0))], "temperature": [f(r.get("temperature", 1))],
            "bias_token": toks[None], "bias_value": vals[None], "bias_len": [len(r.get("bias", ()))],
            "allowed": allowed, "mask_of": [r.get("mask", -1)]}, 0, V)

    def step(slots, k):
        tokens = [int(t) for t in rng.integers(0, 12, len(slots))]      # few words, so they repeat
        for s, t in zip(slots, tokens):
            said[s].append(t)
        out = ctx.step(slots=slots, tokens=tokens, want_logits=True, topk=k)
        for i, s in enumerate(slots):
            z = want(s, out["logits"][i])
            t, lp, tol = best(z, max(k, 1))
            assert out["argmax"][i] == t[0]
            if k:
                assert np.array_equal(out["top_token"][i], t)
                assert (np.abs(out["top_logprob"][i] - lp) <= tol).all()

    for k in (0, 3, 0, 3, 5, 0, 3):
        step([1, 0], k)
    ctx.fork_slot(0, 3)
    rules[3], said[3] = dict(rules[0]), list(said[0])
    for k in (4, 0, 4):
        step([3, 1, 0], k)
    ctx.set_slot_mask(3, 2)
    rules[3]["mask"] = 2
    ctx.set_slot_rules(0, frequency=0.5)
    rules[0] = dict(frequency=0.5)
    for k in (16, 0):
        step([0, 3, 1], k)
    ctx.clear_slot_rules(0)
    rules[0] = None
    step([0, 3], 0)
    step([0, 1], 0)
    # defaults of slots filled from now on, biases among them
    ctx.set_slot_rules(-1, mask=0, presence=1.0, bias=[(3, 9.0), (4, 8.0)])
    ctx.debug_set_encoder_out([4], [-1], [9], E[:1])
    rules[4], said[4] = dict(mask=0, presence=1.0, bias=[(3, 9.0), (4, 8.0)]), []
    for k in (2, 0, 2):
        step([4, 0], k)
    # a cache given from outside: which tokens it stands for is not known
    ctx.debug_set_self_kv(4, synth.self_kv_prefix(seed, 0, shape.n_dec, shape.n_head).numpy(), 20)
    said[4] = [-1] * 20
    step([4, 0], 2)


@pytest.mark.parametrize("name,dtype", [("tiny", "f32"), ("base", "bf16")])
def test_beam_search(name, dtype):
    """Three beams for each of two clips, a prompt of four tokens, a repetition penalty and a mask: at every
    step the six hypotheses' candidates are kept, forked and released as a beam search does; each one's
    log-probability follows the oracle's along its own tokens."""
    shape, seed = shape_of(name, dtype), 20261105
    n, steps = 3, 7
    ctx, E = context(shape, seed, 2 + 4 * n, rows=2 * n, n_masks=1)
    rng = np.random.default_rng(seed)
    allowed = rng.random((1, V)) < 0.5
    ctx.set_masks(0, allowed)
    P = cpu_params(shape, seed, bf16_rounded=dtype == "bf16")
    prompt = [3, 700, 12, 3]
    beams = []                                       # (score, slot, tokens, oracle), per clip
    for clip in (0, 1):
        seq = Alone(shape, P, OW.cross_kv(E[clip].astype(np.float64), P, shape.n_dec))
        for t in prompt[:-1]:
            ctx.step(slots=[clip], tokens=[t])
            seq.step(t)
        ctx.set_slot_rules(clip, repetition=1.2, mask=0, n_prompt=len(prompt))
        beams.append([(0.0, clip, list(prompt), seq)])
    free = list(range(2, 2 + 4 * n))
    for _ in range(steps):
        rows = [b for clip in beams for b in clip]
        out = ctx.step(slots=[b[1] for b in rows], tokens=[b[2][-1] for b in rows], topk=2 * n, want_logits=True)
        i = 0
        for c, clip in enumerate(beams):
            found = []
            for score, slot, tokens, seq in clip:
                ref = seq.step(tokens[-1])
                tol = TOL[dtype] * np.abs(ref).max()
                assert np.abs(out["logits"][i] - ref).max() <= tol
                z = processed(ref.astype(np.float32), {
                    "history": np.array([tokens], np.int32), "history_len": [len(tokens)], "prompt_len": [len(prompt)],
                    "repetition": [np.float32(1.2)], "allowed": allowed, "mask_of": [0]}, 0, V).astype(np.float64)
                lp = z - (z.max() + np.log(np.exp(z - z.max()).sum()))
                for t, v in zip(out["top_token"][i], out["top_logprob"][i]):
                    # logits off by tol move the penalised logit by 1.2 tol and the sum's logarithm by as much
                    assert abs(v - lp[t]) <= 2.4 * tol + 1e-5 and allowed[0, t]
                    found.append((score + float(v), slot, tokens + [int(t)], seq))
                i += 1
            found.sort(key=lambda b: -b[0])
            kept, used = [], set()
            for score, slot, tokens, seq in found[:n]:
                if slot in used:                     # its slot goes on with a better one: fork
                    dst = free.pop(0)
                    ctx.fork_slot(slot, dst)
                    slot, seq = dst, clone(seq)
                used.add(slot)
                kept.append((score, slot, tokens, seq))
            for _, slot, _, _ in clip:
                if slot not in used:
                    ctx.release_slot(slot)
                    if slot >= 2:
                        free.append(slot)
            beams[c] = kept
    assert all(len(b[2]) == len(prompt) + steps for clip in beams for b in clip)
    assert all(len({tuple(b[2]) for b in clip}) == n for clip in beams)


@pytest.mark.parametrize("overlap", [False, True])
def test_continuous_batching_under_default_rules(overlap):
    """Requests served with suppressed tokens and a repetition penalty: the tokens of each are those
    that its slot's rules choose, whatever is beside it."""
    shape = synth.reduced_shape(synth.SHAPES["tiny"], 1, 2, vocab=V)
    seed = 20261106
    allowed = np.random.default_rng(seed).random((1, V)) < 0.2
    ids = list(range(5))
    clips = [synth.pcm_clip(seed, i, 16000 * (2 + i)) for i in ids]

    def serve(admit):
        ctx = make_context(shape, seed, max_slots=3, max_prefill=2, max_decode=3)
        ctx.bind_hypotheses(max_bias=1, n_masks=1)
        ctx.set_masks(0, allowed)
        ctx.set_slot_rules(-1, repetition=1.5, presence=0.5, mask=0, bias=[(int(np.flatnonzero(allowed[0])[3]), 0.5)])
        ctx.serve_config(max_admit=admit, start_token=1, overlap=overlap and admit > 1)
        for i in ids:
            ctx.submit(i, clips[i])
        done = set()
        for now in range(200):
            done |= set(ctx.serve_step(now)["finished"])
            if len(done) == len(ids):
                break
        return [ctx.serve_tokens(i) for i in ids]

    together, single = serve(2), serve(1)
    assert together == single
    for t in together:
        assert len(t) > 3 and allowed[0, t].all()
