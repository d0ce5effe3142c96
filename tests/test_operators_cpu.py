"""Refusals of the stateless decode operators: every argument error is an
error status before anything is launched, so none of this needs a GPU."""
import ctypes as C

import pytest

asr = pytest.importorskip("paper_2603_11273_amd.asr")

BLOCK = C.create_string_buffer(4096)
A = (C.addressof(BLOCK) + 255) // 256 * 256        # an address that is never followed


def attention(**kw):
    a = asr.Attention(asr.BF16, 4, 2, 6, 2, 3, 100, 20, 0, 0.125, A, 256, A, 256, A, None,
                      asr.Keys(A, A, 2 * 100 * 64, 100 * 64, 64, 3, 100, None, None, None),
                      asr.Keys(A, A, 2 * 20 * 64, 20 * 64, 64, 8, 20, None, None, None))
    for name, value in kw.items():
        at, _, field = name.rpartition("__")
        setattr(getattr(a, at) if at else a, field, value)
    return a


def rules(**kw):
    r = asr.Rules(asr.F32, 3, 1000, 3, 1, 2, A, 1000, None, A, 10, A, None, None, None, None, A, A, 5, A, A, 32, None,
                  None, A, 1000, A, A)
    for name, value in kw.items():
        setattr(r, name, value)
    return r


def size(fn, args):
    n = C.c_size_t()
    return fn(C.byref(args) if args is not None else None, C.byref(n)), n.value


def test_sizes():
    st, n = size(asr.lib.asr_attend_shared_size, attention(part_keys=128))
    assert st == asr.ASR_OK and n == 16384 + 6 * 4 * 2 * 66 * 4  # two parts: shared and own
    st, n = size(asr.lib.asr_attend_shared_size, attention(max_own=0))
    assert st == asr.ASR_OK and n == 0                           # one part: no records
    st, n = size(asr.lib.asr_logit_rules_size, rules(vocab=4097, mask_ld=129))
    assert st == asr.ASR_OK and n == 16384 + 3 * 2 * (1 + 2) * 8
    assert size(asr.lib.asr_logit_rules_size, rules(k=0)) == (asr.ASR_OK, 0)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(n_head=0), dict(rows=1 << 25, n_head=8), dict(n_kv_head=3), dict(n_kv_head=0), dict(n_head=1 << 20, n_kv_head=1), dict(rows=-1),
    dict(groups=-1), dict(max_group=0), dict(max_group=7), dict(max_prefix=-1), dict(max_own=-1), dict(max_prefix=101),
    dict(max_own=21), dict(part_keys=64), dict(part_keys=200), dict(part_keys=8320), dict(part_keys=-128),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(prefix__k=None), dict(own__v=None), dict(prefix__k=A + 8),
    dict(own__v=A + 2), dict(prefix__slots=0), dict(own__positions=0), dict(prefix__pos_stride=32),
    dict(prefix__pos_stride=68), dict(own__head_stride=-64), dict(own__slot_stride=100), dict(prefix__pos_stride=1 << 18),
], ids=str)
def test_attention_sizes_refused(kw):
    assert size(asr.lib.asr_attend_shared_size, attention(**kw))[0] == asr.ASR_EINVAL
    assert asr.lib.asr_attend_shared(C.byref(attention(**kw)), A, 1 << 30, None) == asr.ASR_EINVAL
    assert asr.lib.asr_last_error()


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(group_start=None), dict(q=A + 4), dict(out=A + 8),
                                dict(q_ld=252), dict(q_ld=258), dict(out_ld=255), dict(out_ld=64)], ids=str)
def test_attention_call_refused(kw):
    assert asr.lib.asr_attend_shared(C.byref(attention(**kw)), A, 1 << 30, None) == asr.ASR_EINVAL


def test_attention_scratch_refused():
    need = size(asr.lib.asr_attend_shared_size, attention())[1]
    call = lambda ws, n: asr.lib.asr_attend_shared(C.byref(attention()), ws, n, None)  # noqa: E731
    assert call(A, need - 1) == asr.ASR_ENOMEM
    assert call(None, need) == asr.ASR_EINVAL
    assert call(A + 128, need) == asr.ASR_EINVAL
    assert asr.lib.asr_attend_shared(None, A, need, None) == asr.ASR_EINVAL
    assert asr.lib.asr_attend_shared_size(C.byref(attention()), None) == asr.ASR_EINVAL
    # nothing to do is no error, and reads nothing
    assert asr.lib.asr_attend_shared(C.byref(attention(rows=0, q=None, out=None)), None, 0, None) == asr.ASR_OK
    assert asr.lib.asr_attend_shared(C.byref(attention(groups=0, out=None)), A, need, None) == asr.ASR_OK


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(rows=-1), dict(rows=65536), dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(k=-1), dict(k=17),
    dict(sets=-1), dict(masks=-1), dict(history_len=None), dict(history_ld=-1), dict(history_ld=1 << 31),
    dict(bias_value=None), dict(bias_len=None), dict(bias_ld=-1), dict(mask_ld=31)], ids=str)
def test_rules_sizes_refused(kw):
    assert size(asr.lib.asr_logit_rules_size, rules(**kw))[0] == asr.ASR_EINVAL
    assert asr.lib.asr_logit_rules(C.byref(rules(**kw)), A, 1 << 30, None) == asr.ASR_EINVAL


@pytest.mark.parametrize("kw", [dict(logits=None), dict(ld=999), dict(logits=A + 2), dict(out_ld=999), dict(out=A + 2),
                                dict(out=A, dtype=asr.BF16), dict(out=A, out_ld=1001), dict(token=None),
                                dict(logprob=None), dict(out=None, k=0)], ids=str)
def test_rules_call_refused(kw):
    assert asr.lib.asr_logit_rules(C.byref(rules(**kw)), A, 1 << 30, None) == asr.ASR_EINVAL


def test_rules_scratch_refused():
    need = size(asr.lib.asr_logit_rules_size, rules())[1]
    call = lambda ws, n: asr.lib.asr_logit_rules(C.byref(rules()), ws, n, None)  # noqa: E731
    assert call(A, need - 1) == asr.ASR_ENOMEM
    assert call(None, need) == asr.ASR_EINVAL
    assert call(A + 8, need) == asr.ASR_EINVAL
    assert asr.lib.asr_logit_rules(None, A, need, None) == asr.ASR_EINVAL
    assert asr.lib.asr_logit_rules_size(C.byref(rules()), None) == asr.ASR_EINVAL
    assert asr.lib.asr_logit_rules(C.byref(rules(rows=0, logits=None)), None, 0, None) == asr.ASR_OK


def test_plans_refuse_host_memory():
    torch = pytest.importorskip("torch")
    zeros = lambda *shape, **kw: torch.zeros(*shape, **kw)  # noqa: E731
    with pytest.raises(TypeError):
        asr.LogitRules(2, 100, torch.float32, k=1, device="cpu")
    with pytest.raises(TypeError):
        asr.LogitRules(2, 100, torch.float32, k=1, temperature=zeros(2))
    with pytest.raises(TypeError):
        asr.LogitRules(2, 100, torch.float32, k=1, device="cuda:0", temperature=zeros(2))
    with pytest.raises(TypeError):
        asr.LogitRules(2, 100, torch.float32, k=1, device="cuda:0", workspace=zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(TypeError):
        keys = zeros(1, 2, 8, 64)
        asr.SharedAttention(keys, keys, n_head=2, rows=1, groups=1, max_group=1,
                            group_start=zeros(2, dtype=torch.int32))


@pytest.mark.parametrize("name", ["history_ld", "bias_ld"])
def test_lists_that_32_bits_would_not_step_through(name):
    """The kernels read a list 8192 entries at a time with 32-bit places; past 2^31 - 8192 entries the
    last of them would wrap round to places before the list."""
    assert size(asr.lib.asr_logit_rules_size, rules(**{name: 1 << 30}))[0] == asr.ASR_OK
    for n in ((1 << 30) + 1, (1 << 31) - 1):
        assert size(asr.lib.asr_logit_rules_size, rules(**{name: n}))[0] == asr.ASR_EINVAL
        assert asr.lib.asr_logit_rules(C.byref(rules(**{name: n})), A, 1 << 30, None) == asr.ASR_EINVAL
