"""The CPU side of the paged cache and of sampling: codes pinned to the format, the plain implementations pinned to worked
examples, and every refusal of the calls, none of which needs a GPU."""
import ctypes as C

import numpy as np
import pytest

import page_util as P

asr = pytest.importorskip("paper_2603_11273_amd.asr")

BLOCK = C.create_string_buffer(4096)
A = (C.addressof(BLOCK) + 255) // 256 * 256        # an address that is never followed
PAGE = 2 * 2 * 1 * 4096                            # bytes of a page of 64 positions and two heads


def pages(**kw):
    p = dict(kv_heads=2, page=64, pages=9, codes=A, page_stride=PAGE, scales=A, scale_stride=4, table=A, table_ld=5,
             sequences=3, columns=5)
    p.update(kw)
    return asr.Pages(*[p[n] for n, _ in asr.Pages._fields_])


def make(kind, fields, **kw):
    cache = {n[7:]: kw.pop(n) for n in list(kw) if n.startswith("cache__")}
    values = dict(fields, **kw)
    if "cache" in [n for n, _ in kind._fields_]:
        values["cache"] = pages(**cache)
    return kind(**values)


def write(**kw):
    return make(asr.PageTokens, dict(dtype=asr.F32, tokens=7, max_new=7, k=A, v=A, ld=128, token_start=A, length=A), **kw)


def attend(**kw):
    return make(asr.PageQueries, dict(dtype=asr.BF16, n_head=4, rows=6, max_rows=4, max_keys=300, part_keys=0, scale=0.125, q=A,
                                      q_ld=256, out=A, out_ld=256, row_start=A, first=None, length=A), **kw)


def tables(**kw):
    return make(asr.NextTables, dict(sequences=3, columns=5, page=64, pages=9, compact=0, table=A, table_ld=5, length=A + 1024,
                                     parent=A, want=A, new_table=A + 512, new_ld=5, new_length=A + 1280, room=A, info=A,
                                     codes=A, code_stride=PAGE, code_bytes=PAGE, scales=A, scale_stride=16, scale_bytes=16), **kw)


def sampling(**kw):
    return make(asr.Sampling, dict(dtype=asr.F32, rows=3, vocab=100, sets=3, draws=2, logits=A, ld=100, u=A, set=None,
                                   temperature=A, top_k=A, top_p=A, min_p=A, token=A, logprob=A, kept=A), **kw)


CALLS = {"write": lambda a, ws=A, n=1 << 40: asr.lib.asr_write_pages(C.byref(a), None),
         "attend": lambda a, ws=A, n=1 << 40: asr.lib.asr_attend_pages(C.byref(a), ws, n, None),
         "tables": lambda a, ws=A, n=1 << 40: asr.lib.asr_next_tables(C.byref(a), ws, n, None),
         "sample": lambda a, ws=A, n=1 << 40: asr.lib.asr_sample(C.byref(a), ws, n, None)}
SIZES = {"attend": asr.lib.asr_attend_pages_size, "tables": asr.lib.asr_next_tables_size, "sample": asr.lib.asr_sample_size}
MAKE = {"write": write, "attend": attend, "tables": tables, "sample": sampling}

POOL = [dict(cache__kv_heads=0), dict(cache__kv_heads=65537), dict(cache__page=0), dict(cache__page=32), dict(cache__page=96),
        dict(cache__page=8192), dict(cache__pages=0), dict(cache__sequences=-1), dict(cache__columns=0), dict(cache__codes=None),
        dict(cache__codes=A + 8), dict(cache__scales=None), dict(cache__scales=A + 2), dict(cache__page_stride=PAGE - 16),
        dict(cache__page_stride=PAGE + 8), dict(cache__scale_stride=3), dict(cache__table=None), dict(cache__table_ld=4),
        dict(cache__columns=1 << 25, cache__table_ld=1 << 25)]
REFUSED = {
    "write": POOL + [dict(dtype=2), dict(tokens=-1), dict(max_new=-1), dict(token_start=None, tokens=2), dict(k=None), dict(v=None),
                     dict(length=None), dict(k=A + 4), dict(v=A + 8), dict(ld=124), dict(ld=130), dict(ld=132, dtype=asr.BF16),
                     dict(cache__sequences=1 << 20, cache__kv_heads=8, cache__page_stride=4 * PAGE, cache__scale_stride=16, ld=512,
                          tokens=1 << 30, max_new=1 << 20)],
    "attend": POOL + [dict(dtype=-1), dict(n_head=0), dict(n_head=3), dict(n_head=1 << 17), dict(rows=-1), dict(max_keys=-1),
                      dict(max_rows=0), dict(max_rows=7), dict(row_start=None), dict(part_keys=128), dict(part_keys=300),
                      dict(part_keys=1 << 15), dict(part_keys=-256), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=None),
                      dict(out=None), dict(length=None), dict(q=A + 4), dict(out=A + 8), dict(q_ld=252), dict(q_ld=258),
                      dict(out_ld=64), dict(rows=1 << 25, n_head=8)],
    "tables": [dict(sequences=-1), dict(columns=0), dict(page=0), dict(pages=0), dict(pages=(1 << 22) + 1), dict(page=1 << 28),
               dict(sequences=1 << 25), dict(table_ld=4), dict(new_ld=4), dict(table=None), dict(new_table=None), dict(length=None),
               dict(new_length=None), dict(new_table=A + 8), dict(new_length=A + 1028), dict(new_table=A), dict(new_length=A + 1024),
               dict(new_table=A, new_length=A + 1024, new_ld=6), dict(codes=A + 2), dict(code_bytes=-4), dict(code_bytes=6),
               dict(code_stride=PAGE - 4), dict(scales=A + 2), dict(scale_bytes=10), dict(scale_stride=12)],
    "sample": [dict(dtype=2), dict(rows=-1), dict(rows=65536), dict(vocab=0), dict(vocab=(1 << 20) + 1, ld=1 << 21), dict(draws=0),
               dict(draws=65), dict(sets=-1), dict(logits=None), dict(ld=99), dict(logits=A + 2), dict(u=None), dict(token=None)]}


@pytest.mark.parametrize("op,kw", [(op, kw) for op in REFUSED for kw in REFUSED[op]], ids=str)
def test_refused(op, kw):
    assert CALLS[op](MAKE[op](**kw)) == asr.ASR_EINVAL
    assert asr.lib.asr_last_error()


@pytest.mark.parametrize("op", list(CALLS))
def test_null_arguments_refused(op):
    fn = {"write": asr.lib.asr_write_pages, "attend": asr.lib.asr_attend_pages, "tables": asr.lib.asr_next_tables,
          "sample": asr.lib.asr_sample}[op]
    assert fn(None, None) == asr.ASR_EINVAL if op == "write" else fn(None, A, 1 << 30, None) == asr.ASR_EINVAL
    if op in SIZES:
        assert SIZES[op](C.byref(MAKE[op]()), None) == asr.ASR_EINVAL
        assert SIZES[op](None, C.byref(C.c_size_t())) == asr.ASR_EINVAL


@pytest.mark.parametrize("op", list(SIZES))
def test_scratch_refused(op):
    n = C.c_size_t()
    args = MAKE[op](**(dict(part_keys=256) if op == "attend" else {}))
    assert SIZES[op](C.byref(args), C.byref(n)) == asr.ASR_OK
    if n.value:
        assert CALLS[op](args, A, n.value - 1) == asr.ASR_ENOMEM
        assert CALLS[op](args, None, n.value) == asr.ASR_EINVAL
        assert CALLS[op](args, A + 128, n.value) == asr.ASR_EINVAL


def test_nothing_to_do_is_no_error_and_reads_nothing():
    for kw in (dict(tokens=0, k=None, v=None, length=None), dict(max_new=0, k=None), dict(cache__sequences=0, k=None, length=None)):
        assert CALLS["write"](write(**kw)) == asr.ASR_OK
    for kw in (dict(rows=0, q=None, out=None), dict(cache__sequences=0, q=None)):
        assert CALLS["attend"](attend(**kw), None, 0) in (asr.ASR_OK,)
    assert CALLS["sample"](sampling(rows=0, logits=None, u=None, token=None), None, 0) == asr.ASR_OK


def test_plans_refuse_host_memory():
    torch = pytest.importorskip("torch")
    codes, scales = torch.zeros((3, 2, 2, 1, 64, 64), dtype=torch.uint8), torch.zeros((3, 2, 2, 1))
    table, length = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        asr.PageWrite(codes, scales, table, length, tokens=2, dtype=torch.float32)
    with pytest.raises(TypeError):
        asr.PagedAttention(codes, scales, table, length, n_head=2, rows=2)
    with pytest.raises(TypeError):
        asr.PageTables(codes, scales, table, length)
    with pytest.raises(TypeError):
        asr.Sampler(2, 100, torch.float32, device="cpu")
    with pytest.raises(TypeError):
        asr.Sampler(2, 100, torch.float16, device="cuda:0")
    with pytest.raises(TypeError):
        asr.Sampler(2, 100, torch.float32, temperature=torch.zeros(2))


def test_codes_are_those_of_the_format():
    assert P.VALUE[0x7e] == 448 and P.VALUE[0x01] == 2.0 ** -9 and P.VALUE[0x08] == 2.0 ** -6 and P.VALUE[0x38] == 1.0
    assert np.isnan(P.VALUE[[0x7f, 0xff]]).all() and (np.diff(P.STEPS) > 0).all()
    fine = np.arange(256)[~np.isnan(P.VALUE)]
    assert (P.encode(P.VALUE[fine]) == fine).all()
    mid = (P.STEPS[1:] + P.STEPS[:-1]) / 2
    assert (P.encode(mid) % 2 == 0).all() and (P.encode(-mid) % 2 == 0).all()
    assert P.encode([1e9, -1e9, np.inf, np.nan]).tolist() == [0x7e, 0xfe, 0x7f, 0x7f]
    torch = pytest.importorskip("torch")
    x = np.concatenate([np.random.default_rng(1).standard_normal(20000) * 2.0 ** np.arange(-10, 10).repeat(1000), mid])
    x = x[np.abs(x) <= 448].astype(np.float32)
    assert (torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy() == P.encode(x)).all()


def test_scales():
    for x in (448.0, 447.9, 448.1, 1.0, 0.0, 1e-30, 3e38, 449 * 2.0 ** -7, 448 * 2.0 ** -7):
        s = P.power_at_least(x / 448)
        assert np.log2(s) % 1 == 0 and (x <= 448 * s or s == 2.0 ** 120) and (s == 2.0 ** -120 or x > 224 * s)


def test_tables_of_a_worked_example():
    """Pages of four positions, eight of them.  Sequence 0 holds 6 positions on pages 5, 2; sequence 1 4 on page 7."""
    table, length = np.array([[5, 2, -1], [7, -1, -1]]), np.array([6, 4])
    # both go on from 0: the first keeps its half page, the second gets a copy; 7 is free
    new, lens, room, info, data = P.next_tables(table, length, np.array([0, 0]), np.array([7, 9]), 4, 8, False)
    assert new.tolist() == [[5, 2, -1], [5, 0, 1]] and lens.tolist() == [6, 6] and room.tolist() == [8, 12]
    assert info.tolist() == [4, 0, 1, 0] and data == [(2, 0)]
    # sequence 0 ends and starts anew with room for one position; compact: 7 moves to 0, the new page is 1
    new, lens, room, info, data = P.next_tables(table, length, np.array([-1, 1]), np.array([1, 4]), 4, 8, True)
    assert new.tolist() == [[1, -1, -1], [0, -1, -1]] and lens.tolist() == [0, 4] and data == [(7, 0)]
    assert info.tolist() == [2, 0, 0, 1]
    # no page left for the copy
    new, lens, room, info, data = P.next_tables(np.array([[0, 1, 2]] * 2), np.array([12, 9]), np.array([0, 1]), None, 4, 3, False)
    assert new.tolist() == [[0, 1, 2], [0, 1, -1]] and room.tolist() == [12, 8] and info.tolist() == [3, 1, 0, 0]


def test_sampling_of_a_worked_example():
    """Weights 4 : 2 : 1 : 1 at tokens 2, 0, 1, 3."""
    l = np.log([2.0, 1.0, 4.0, 1.0])
    assert P.sample(l, [0.0, 0.249, 0.251, 0.374, 0.376, 0.874, 0.876, 0.999])[0] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert P.sample(l, [0.1], k=3)[2] == 3 and P.sample(l, [0.99], k=3)[0] == [2]       # the lower of equal tokens is in
    assert P.sample(l, [0.1], p=0.5)[2] == 1 and P.sample(l, [0.1], p=0.51)[2] == 2
    assert P.sample(l, [0.1], k=2, p=0.66)[2] == 1 and P.sample(l, [0.1], k=2, p=0.67)[2] == 2
    assert P.sample(l, [0.1], m=0.3)[2] == 2 and P.sample(l, [0.1], T=0.0)[0] == [2]
    assert abs(P.sample(l, [0.1], T=0.5)[1][0] - np.log(4 / 22)) < 1e-12
    assert P.sample([-np.inf, -np.inf], [0.5])[:3] == ([-1], [-np.inf], 0)
    assert P.sample([0.0, np.nan], [0.5])[0] == [-1]
