"""What the library does on the host for hypotheses and rules, without a GPU:
tests/hip_stub_hypotheses.cpp is linked with the library, stands in for the HIP
calls, makes up the results of the kernels and checks what becomes of them."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

asr = pytest.importorskip("paper_2603_11273_amd.asr")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def stub(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("stub") / "hypotheses")
    lib_dir = os.path.dirname(asr.LIB_PATH)
    cmd = ["g++", "-std=c++17", "-O1", "-Wall", "-rdynamic", "-I", os.path.join(ROOT, "include"),
           os.path.join(ROOT, "tests", "hip_stub_hypotheses.cpp"), "-L", lib_dir,
           "-l:" + os.path.basename(asr.LIB_PATH), "-Wl,-rpath," + lib_dir,
           "-Wl,--allow-shlib-undefined", "-o", exe]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout

    def run(name):
        r = subprocess.run([exe, name], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
        assert r.returncode == 0, r.stdout[-2000:]
        assert f"{name}: ok" in r.stdout
    return run


def test_a_row_without_a_next_token_ends_its_request_alone(stub):
    """Continuous batching: no allowed token, and a NaN, in one row of two."""
    stub("serve")


def test_a_row_without_rules_beside_one_with_rules(stub):
    """Infinite and NaN logits of a row without rules are answered as they are without the other row."""
    stub("beside")


def test_graphs_of_many_shapes_are_bounded(stub):
    """A search goes through more shapes of a step than graphs are kept of."""
    stub("shapes")


def test_biases_without_probabilities_are_refused(stub):
    stub("biases")


class FakeLibrary:
    """The entry points of a step: `status`, and what they write where they get so far."""

    def __init__(self, status, writes=True):
        self.status, self.writes = status, writes

    def asr_last_error(self):
        return b"a row of it"

    def asr_step(self, h, sin, sout):
        if self.writes:
            for i in range(sin._obj.n_decode):
                sout._obj.argmax[i] = i - 1
                sout._obj.done[i] = i % 2
        return self.status

    def asr_step_topk(self, h, sin, sout, k, token, logprob):
        if self.writes:
            for i in range(sin._obj.n_decode * k):
                token[i], logprob[i] = 10 + i, -i
        return self.asr_step(h, sin, sout)

    def asr_serve_step(self, h, now, out):
        if self.writes:
            o = out._obj
            o.policy, o.n_finished, o.finished[0] = 2, 1, 77
            o.n_decoded, o.decoded[0], o.token[0] = 1, 77, -1
        return self.status


@pytest.fixture
def context(monkeypatch):
    ctx = asr.Context.__new__(asr.Context)
    ctx.h, ctx.cfg, ctx._serve_cap = None, asr.ModelCfg(max_slots=4, vocab=9), 4

    def with_library(*a, **kw):
        monkeypatch.setattr(asr, "lib", FakeLibrary(*a, **kw))
        return ctx
    return with_library


def test_a_dead_row_does_not_take_the_others_results(context):
    """A step that reports a row without a next token hands its results over with the error; one that
    failed before it had any does not."""
    ctx = context(asr.ASR_EDEVICE)
    with pytest.raises(asr.AsrError) as e:
        ctx.step(slots=[0, 1, 2], tokens=[3, 4, 5], topk=2, want_logits=True)
    r = e.value.results
    assert list(r["argmax"]) == [-1, 0, 1] and list(r["done"]) == [False, True, False]
    assert r["top_token"].tolist() == [[10, 11], [12, 13], [14, 15]] and r["top_logprob"][2, 1] == -5
    assert r["logits"].shape == (3, 9)
    with pytest.raises(asr.AsrError) as e:
        ctx.step(slots=[0, 1], tokens=[3, 4])
    assert list(e.value.results["argmax"]) == [-1, 0]
    with pytest.raises(asr.AsrError) as e:
        ctx.serve_step(0)
    assert e.value.results["finished"] == [77] and e.value.results["token"] == [-1]
    for status in (asr.ASR_EDEVICE, asr.ASR_EINVAL):
        ctx = context(status, writes=False)
        for call in (lambda: ctx.step(slots=[0], tokens=[1]), lambda: ctx.step(slots=[0], tokens=[1], topk=3),
                     lambda: ctx.serve_step(0)):
            with pytest.raises(asr.AsrError) as e:
                call()
            assert e.value.results is None and e.value.status == status
    ctx = context(asr.ASR_OK)
    assert list(ctx.step(slots=[2], tokens=[1])["argmax"]) == [-1] and ctx.serve_step(1)["policy"] == 2


def test_biases_of_any_iterable(monkeypatch):
    """(token, value) pairs from a list, a dict's items, a zip or a generator."""
    got = []

    class Library:
        def asr_set_slot_rules(self, h, slot, r):
            r = r._obj
            got.append([(r.bias_token[i], r.bias_value[i]) for i in range(r.n_bias)])
            return asr.ASR_OK
    monkeypatch.setattr(asr, "lib", Library())
    ctx = asr.Context.__new__(asr.Context)
    ctx.h = None
    pairs = [(7, 2.5), (11, -1.0), (7, 0.5)]
    for bias in (pairs, zip([7, 11, 7], [2.5, -1.0, 0.5]), (p for p in pairs), tuple(pairs)):
        ctx.set_slot_rules(0, bias=bias)
    assert got == [pairs] * 4
    ctx.set_slot_rules(0, bias={3: 1.0}.items())
    ctx.set_slot_rules(0)
    assert got[4:] == [[(3, 1.0)], []]
