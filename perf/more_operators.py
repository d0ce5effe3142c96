"""What a decode step needs to keep its keys and values in pages of 8 bits and to choose tokens by chance, as a user's program
calls it.

Four operators, each over the sizes it is used at:

* write    new keys and values into pages of e4m3 codes, one power-of-two scale per head and block of 64 tokens: asr.PageWrite;
* attend   new tokens attend over the pages of their sequence: asr.PagedAttention;
* tables   the page tables of the next step: sequences forked, ended, extended, the pool compacted: asr.PageTables;
* sample   tokens drawn from logits under temperature, top-k, top-p and min-p with given random numbers: asr.Sampler.

A program keeps its pool, tables and parameters in device memory and a plan per batch shape.  Lengths are spread evenly between
their bounds and dealt to the sequences by the seed, so a case's work does not depend on it.
"""
import math

import numpy as np
import torch

own = False

HEAD = 64
BLOCK = 64
LEAST = 2.0 ** -120
F8 = torch.float8_e4m3fn
# what a drawn case has at most, as the largest listed ones: values written, bytes of keys and values, scores, table entries,
# bytes of a pool that pages are copied in, logits
MOST_WRITTEN = 24 * 1500 * 20 * HEAD
MOST_BYTES = 16 * 65536 * 8 * 2 * HEAD
MOST_SCORES = 16 * 65536 * 32
MOST_POOL = 4.0e8
MOST_LOGITS = 256 * 131071


def listed():
    return [
        # one decode step of 128 running sequences: a token each, behind texts of all lengths
        {"name": "write_step_128", "op": "write", "dtype": "f32", "heads": 20, "page": 64, "sequences": 128, "new_lo": 1,
         "new_hi": 1, "held_lo": 10, "held_hi": 400},
        # the audio of 24 clips after their prefill, bf16 as the projection leaves it
        {"name": "write_audio_24", "op": "write", "dtype": "bf16", "heads": 20, "page": 128, "sequences": 24, "new_lo": 1500,
         "new_hi": 1500, "held_lo": 0, "held_hi": 0},
        # the small model on a development machine: one row, one clip
        {"name": "attend_tiny_1", "op": "attend", "dtype": "f32", "heads": 6, "kv_heads": 6, "page": 64, "sequences": 1,
         "rows_lo": 1, "rows_hi": 1, "keys_lo": 1500, "keys_hi": 1500, "causal": False, "window": 0},
        # a full decode batch: 24 clips, five hypotheses on each one's audio
        {"name": "attend_audio_24x5", "op": "attend", "dtype": "bf16", "heads": 20, "kv_heads": 20, "page": 128, "sequences": 24,
         "rows_lo": 5, "rows_hi": 5, "keys_lo": 1500, "keys_hi": 1500, "causal": False, "window": 0},
        # chunks of text prompts: up to 33 new tokens a sequence, each seeing those before it, a window of 1000 positions
        {"name": "attend_chunk_7", "op": "attend", "dtype": "f32", "heads": 8, "kv_heads": 8, "page": 64, "sequences": 7,
         "rows_lo": 1, "rows_hi": 33, "keys_lo": 33, "keys_hi": 4001, "causal": True, "window": 1000},
        # 64 sequences of uneven length on a decoder whose query heads share key heads
        {"name": "attend_shared_heads_64", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "page": 128,
         "sequences": 64, "rows_lo": 1, "rows_hi": 1, "keys_lo": 515, "keys_hi": 8191, "causal": False, "window": 0},
        # the largest: sixteen recordings of many hours as the context
        {"name": "attend_long_16", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "page": 256, "sequences": 16,
         "rows_lo": 1, "rows_hi": 1, "keys_lo": 65536, "keys_hi": 65536, "causal": False, "window": 0},
        # one step of beam search: 24 clips x 5 hypotheses of one layer's pages, parents drawn anew in each clip
        {"name": "tables_beams_120", "op": "tables", "heads": 20, "layers": 1, "page": 64, "family": 5, "sequences": 120,
         "held_lo": 1, "held_hi": 448, "spare": 1.5, "ended": 0.0, "compact": False},
        # after many requests ended: the pages of the others packed to the front of the pool, all of a model's layers in a page
        {"name": "tables_compact_192", "op": "tables", "heads": 6, "layers": 4, "page": 64, "family": 1, "sequences": 192,
         "held_lo": 1, "held_hi": 448, "spare": 2.0, "ended": 0.4, "compact": True},
        # a lone clip, temperature fallback
        {"name": "sample_1", "op": "sample", "dtype": "f32", "rows": 1, "vocab": 51865, "draws": 1, "top_k": 0, "top_p": True,
         "min_p": False, "spread": 3.0},
        # every decode slot busy, all filters on
        {"name": "sample_128", "op": "sample", "dtype": "f32", "rows": 128, "vocab": 51866, "draws": 1, "top_k": 400,
         "top_p": True, "min_p": True, "spread": 3.0},
        # the largest: a big vocabulary, five tokens of each row, filters that keep many
        {"name": "sample_256x5", "op": "sample", "dtype": "bf16", "rows": 256, "vocab": 131071, "draws": 5, "top_k": 50000,
         "top_p": True, "min_p": False, "spread": 1.5},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["write", "attend", "attend", "tables", "sample"])
    if op == "write":
        heads = rng.choice([1, 2, 4, 6, 8, 12, 16, 20])
        n = _log_int(rng, 1, 128)
        hi = _log_int(rng, 1, min(4096, max(1, MOST_WRITTEN // (n * heads * HEAD))))
        held = rng.randint(0, 448)
        return {"op": op, "dtype": rng.choice(["f32", "bf16"]), "heads": heads, "page": rng.choice([64, 128, 192, 256]),
                "sequences": n, "new_lo": rng.choice([0, 1, hi]), "new_hi": hi, "held_lo": rng.randint(0, held), "held_hi": held}
    if op == "attend":
        kv = rng.choice([1, 2, 4, 6, 8, 12, 16, 20])
        per = rng.choice([1, 1, 1, 2, 4, 5, 8])
        if kv * per > 40:
            per = 1
        n = _log_int(rng, 1, 64)
        rows = _log_int(rng, 1, min(40, 256 // n))
        room = min(MOST_BYTES / (n * kv * 2 * HEAD), MOST_SCORES / (n * rows * kv * per))
        keys = _log_int(rng, 1, int(min(65536, room)))
        return {"op": op, "dtype": rng.choice(["bf16", "bf16", "f32"]), "heads": kv * per, "kv_heads": kv,
                "page": rng.choice([64, 128, 192, 256]), "sequences": n, "rows_lo": rng.randint(1, rows), "rows_hi": rows,
                "keys_lo": rng.choice([0, 1, keys // 2, keys]), "keys_hi": keys, "causal": rng.random() < 0.5,
                "window": rng.choice([0, 0, 0, 1, 77, 1000])}
    if op == "tables":
        heads, layers, page = rng.choice([1, 4, 6, 8, 20]), rng.choice([1, 1, 2, 4]), rng.choice([64, 128, 256])
        spare = rng.choice([1.0, 1.2, 2.0])
        most = MOST_POOL / (spare * layers * 2 * heads * page * HEAD)
        n = _log_int(rng, 1, int(min(400, max(1, most / 2))))
        held = _log_int(rng, 1, int(min(8192, max(1, most / n - 1) * page)))
        return {"op": op, "heads": heads, "layers": layers, "page": page, "family": rng.choice([1, 1, 4, 5, 8]), "sequences": n,
                "held_lo": rng.randint(0, held), "held_hi": held, "spare": spare, "ended": rng.choice([0.0, 0.1, 0.5]),
                "compact": rng.random() < 0.5}
    rows = _log_int(rng, 1, 256)
    vocab = _log_int(rng, 33, min(131071, MOST_LOGITS // rows))
    return {"op": op, "dtype": rng.choice(["bf16", "f32"]), "rows": rows, "vocab": vocab, "draws": rng.choice([1, 1, 2, 5]),
            "top_k": rng.choice([0, 1, 50, vocab // 2]), "top_p": rng.random() < 0.6, "min_p": rng.random() < 0.4,
            "spread": rng.choice([0.5, 1.5, 3.0])}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _spread(lo, hi, n):
    """n whole numbers spread evenly over [lo, hi]."""
    return np.rint(np.linspace(hi, lo, n)).astype(np.int32) if n > 1 else np.array([hi], np.int32)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _pool(g, pages, layers, heads, page):
    """Codes and scales of values with a deviation of 1, as a pool that has been in use holds them; one page more than a plan is
    told of, so that the plain form has somewhere to send what is not to be written."""
    blocks = page // BLOCK
    codes = torch.empty((pages + 1, layers, 2, heads, blocks, 64, 64), dtype=torch.uint8, device="cuda")
    for some in codes.split(max(1, (1 << 28) // codes[0].numel())):
        some.copy_((torch.randn(some.shape, generator=g, device="cuda") * 64).clamp(-448, 448).to(F8).view(torch.uint8))
    scales = torch.full((pages + 1, layers, 2, heads, blocks), 2.0 ** -6, device="cuda")
    return codes, scales


def _tables(rng, needs, pages, columns):
    """Tables of sequences that hold needs[i] pages each, taken from anywhere in the pool; -1 behind them."""
    table = np.full((len(needs), columns), -1, np.int32)
    table[np.arange(columns) < needs[:, None]] = rng.permutation(pages)[:int(needs.sum())]
    return table


def _write_inputs(case, seed):
    rng = np.random.default_rng([seed, 11])
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, page, wide = case["sequences"], case["page"], case["heads"] * HEAD
    new = rng.permutation(_spread(case["new_lo"], case["new_hi"], n))
    held = rng.permutation(_spread(case["held_lo"], case["held_hi"], n))
    needs = (new + held + page - 1) // page
    # (as many pages whatever the seed deals to whom)
    pages, tokens = int(((new + page - 1) // page + (held + page - 1) // page).sum()) + 3, max(1, int(new.sum()))
    columns = max(1, (case["new_hi"] + case["held_hi"] + page - 1) // page)
    codes, scales = _pool(g, pages, 1, case["heads"], page)
    # keys, values and the queries beside them, as the projection leaves them; some tokens larger than what the blocks hold
    qkv = torch.randn((tokens, 3 * wide), generator=g, device="cuda")
    qkv *= 2.0 ** _dev(rng.integers(-1, 3, (tokens, 1)).astype(np.float32))
    if case["dtype"] == "bf16":
        qkv = qkv.to(torch.bfloat16)
    return {"case": case, "k": qkv[:, wide:2 * wide], "v": qkv[:, 2 * wide:], "codes": codes[:, 0], "scales": scales[:, 0],
            "pages": pages, "tokens": tokens, "table": _dev(_tables(rng, needs, pages, columns)),
            "length": _dev(held), "token_start": _dev(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))}


def _attend_inputs(case, seed):
    rng = np.random.default_rng([seed, 13])
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, page = case["sequences"], case["page"]
    sizes = rng.permutation(_spread(case["rows_lo"], case["rows_hi"], n))
    keys = rng.permutation(_spread(case["keys_lo"], case["keys_hi"], n))
    needs = (keys + page - 1) // page
    pages, rows = int(needs.sum()) + 3, int(sizes.sum())
    codes, scales = _pool(g, pages, 1, case["kv_heads"], page)
    start = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    length = np.repeat(keys, sizes)
    if case["causal"]:
        # the sequence's last tokens: each sees itself and what is before it
        length = length - (np.repeat(start[1:], sizes) - 1 - np.arange(rows, dtype=np.int32))
    length = np.maximum(length, 0).astype(np.int32)
    # queries that make some keys matter: scores of a few units
    q = 2.0 * torch.randn((rows, case["heads"] * HEAD), generator=g, device="cuda")
    kind = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    state = {"case": case, "rows": rows, "q": q, "out": torch.zeros((rows, case["heads"] * HEAD), dtype=kind, device="cuda"),
             "codes": codes[:, 0], "scales": scales[:, 0], "pages": pages, "most": int(sizes.max()),
             "table": _dev(_tables(rng, needs, pages, max(1, (case["keys_hi"] + page - 1) // page))), "row_start": _dev(start),
             "length": _dev(length)}
    if case["window"]:
        state["first"] = _dev(np.maximum(length - case["window"], 0).astype(np.int32))
    return state


def _tables_inputs(case, seed):
    rng = np.random.default_rng([seed, 17])
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, page, family = case["sequences"], case["page"], case["family"]
    # the hypotheses of a family are as long as each other and share the full pages of the first half of their text
    clips = (n + family - 1) // family
    texts = _spread(case["held_lo"], case["held_hi"], clips)
    held = np.repeat(rng.permutation(texts), family)[:n].astype(np.int32)
    first = np.arange(n) // family * family
    needs, shared = (held + page - 1) // page, held // 2 // page
    columns = int((held.max() + 1 + page - 1) // page)
    pages = int(int(((texts + page - 1) // page).sum()) * family * case["spare"]) + n
    table = _tables(rng, needs, pages, columns)
    at = np.arange(columns)
    table = np.where(at < shared[:, None], table[first], table).astype(np.int32)
    codes, scales = _pool(g, pages, case["layers"], case["heads"], page)
    parent = (first + rng.integers(0, family, n)).clip(max=n - 1).astype(np.int32)
    ended = np.zeros(n, bool)
    ended[rng.permutation(n)[:int(n * case["ended"])]] = True
    parent[ended] = -1
    # each sequence that goes on gets room for one token more; an ended one is filled with a new prompt or stays empty
    want = np.where(ended, rng.integers(0, 2, n) * min(page, columns * page), held[np.maximum(parent, 0)] + 1).astype(np.int32)
    return {"case": case, "codes": codes, "scales": scales, "pages": pages, "table": _dev(table), "length": _dev(held),
            "parent": _dev(parent), "want": _dev(want), "new_table": _dev(np.zeros_like(table)),
            "new_length": _dev(np.zeros(n, np.int32)), "room": _dev(np.zeros(n, np.int32)), "info": _dev(np.zeros(4, np.int32))}


def _sample_inputs(case, seed):
    rng = np.random.default_rng([seed, 19])
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, V = case["rows"], case["vocab"]
    x = torch.randn((rows, V), generator=g, device="cuda") * case["spread"] - 4.0
    state = {"case": case, "logits": x.to(torch.bfloat16) if case["dtype"] == "bf16" else x,
             "u": torch.rand((rows, case["draws"]), generator=g, device="cuda"),
             "temperature": _dev(np.where(rng.random(rows) < 0.05, 0.0, rng.uniform(0.2, 1.2, rows)).astype(np.float32)),
             "token": torch.empty((rows, case["draws"]), dtype=torch.int32, device="cuda"),
             "logprob": torch.empty((rows, case["draws"]), device="cuda"),
             "kept": torch.empty((rows,), dtype=torch.int32, device="cuda")}
    if case["top_k"]:
        state["top_k"] = _dev(rng.integers(1, case["top_k"] + 1, rows).astype(np.int32))
    if case["top_p"]:
        state["top_p"] = _dev(rng.uniform(0.5, 1.0, rows).astype(np.float32))
    if case["min_p"]:
        state["min_p"] = _dev(rng.uniform(0.0, 0.1, rows).astype(np.float32))
    return state


def prepare(case, seed):
    return {"write": _write_inputs, "attend": _attend_inputs, "tables": _tables_inputs, "sample": _sample_inputs}[case["op"]](case, seed)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _plan(s):
    """The plan that a program makes once for a batch shape and the buffers it keeps."""
    from paper_2603_11273_amd import asr
    c = s["case"]
    if c["op"] == "sample":
        names = ("temperature", "top_k", "top_p", "min_p")
        return asr.Sampler(c["rows"], c["vocab"], s["logits"].dtype, draws=c["draws"], **{n: s[n] for n in names if n in s})
    codes, scales = s["codes"][:s["pages"]], s["scales"][:s["pages"]]
    if c["op"] == "write":
        return asr.PageWrite(codes, scales, s["table"], s["length"], tokens=s["tokens"], dtype=s["k"].dtype, max_new=c["new_hi"],
                             token_start=s["token_start"])
    if c["op"] == "attend":
        return asr.PagedAttention(codes, scales, s["table"], s["length"], n_head=c["heads"], rows=s["rows"],
                                  row_start=s["row_start"], max_rows=s["most"], first=s.get("first"), max_keys=c["keys_hi"],
                                  scale=HEAD ** -0.5, dtype=s["out"].dtype)
    return asr.PageTables(codes, scales, s["table"], s["length"], parent=s["parent"], want=s["want"], new_table=s["new_table"],
                          new_length=s["new_length"], room=s["room"], info=s["info"])


def _pool_out(s):
    """The pool as the values that its codes stand for, and their scales."""
    return {"codes": s["codes"][:s["pages"]].view(F8), "scales": s["scales"][:s["pages"]]}


def _run_own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    op = s["case"]["op"]
    if op == "write":
        s["plan"](s["k"], s["v"])
        return _pool_out(s)
    if op == "attend":
        return {"out": s["plan"](s["q"], s["out"])}
    if op == "tables":
        s["plan"](compact=s["case"]["compact"])
        return {n: s[n] for n in ("new_table", "new_length", "room", "info")} | _pool_out(s)
    s["plan"](s["logits"], s["u"], s["token"], s["logprob"], s["kept"])
    return {n: s[n] for n in ("token", "logprob", "kept")}


def _write(s):
    c, n, page, H = s["case"], s["case"]["sequences"], s["case"]["page"], s["case"]["heads"]
    most = (c["new_hi"] + BLOCK - 1) // BLOCK + 1            # blocks that a sequence's new tokens can touch
    start, length = s["token_start"].long(), s["length"].long()
    end = length + start[1:] - start[:-1]
    block = length[:, None] // BLOCK + torch.arange(most, device="cuda")                      # [n][most]
    there = block * BLOCK < end[:, None]
    pos = block[..., None] * BLOCK + torch.arange(BLOCK, device="cuda")                       # [n][most][64]
    old = pos < length[:, None, None]
    new = (pos >= length[:, None, None]) & (pos < end[:, None, None])
    slot = (block * BLOCK // page).clamp(max=s["table"].shape[1] - 1)
    at = torch.where(there, s["table"].long().gather(1, slot), torch.full_like(block, s["pages"]))
    inner = torch.where(there, block % (page // BLOCK), torch.zeros_like(block))
    token = (start[:-1, None, None] + pos - length[:, None, None]).clamp(0, s["tokens"] - 1)
    x = torch.stack([s[m][token.view(-1)].float().view(n, most, BLOCK, H, HEAD) for m in ("k", "v")], 2)
    x = x.permute(0, 1, 2, 4, 3, 5)                                                           # [n][most][2][H][64 tokens][64]
    code = s["codes"].permute(0, 3, 1, 2, 4, 5)[at, inner]                                    # [n][most][2][H][64][64]
    code[:, :, 1] = code[:, :, 1].transpose(-1, -2).clone()
    scale = s["scales"].permute(0, 3, 1, 2)[at, inner]                                        # [n][most][2][H]
    new6, old6 = new[:, :, None, None, :, None], old[:, :, None, None, :, None]
    top = torch.where(new6, x.abs(), torch.zeros_like(x)).amax((-1, -2))
    part, power = torch.frexp(top)
    need = torch.ldexp(torch.ones_like(top), (power - 9 + (part > 0.875).int()).clamp(min=-120))
    need = torch.where(top > 0, need, torch.full_like(need, LEAST))
    held = old.any(-1)[:, :, None, None]
    to = torch.where(held, torch.maximum(scale, need), need)
    moved = (code.view(F8).float() * (scale / to)[..., None, None]).to(F8).view(torch.uint8)
    fresh = (torch.where(new6, x, torch.zeros_like(x)) / to[..., None, None]).to(F8).view(torch.uint8)
    code = torch.where(new6, fresh, torch.where(old6, moved, code))
    code[:, :, 1] = code[:, :, 1].transpose(-1, -2).clone()
    s["codes"].permute(0, 3, 1, 2, 4, 5)[at, inner] = code
    s["scales"].permute(0, 3, 1, 2)[at, inner] = to
    return _pool_out(s)


def _attend(s):
    c, rows, kv, page = s["case"], s["rows"], s["case"]["kv_heads"], s["case"]["page"]
    per, n, most, L = c["heads"] // kv, c["sequences"], s["most"], c["keys_hi"]
    start, table = s["row_start"].long(), s["table"].long().clamp(min=0)
    x = s["codes"][table].view(F8).float() * s["scales"][table][..., None, None]              # [n][pages][2][kv][blocks][64][64]
    K = x[:, :, 0].permute(0, 2, 1, 3, 4, 5).reshape(n, kv, -1, HEAD)[:, :, :L]
    V = x[:, :, 1].permute(0, 2, 1, 3, 5, 4).reshape(n, kv, -1, HEAD)[:, :, :L]
    member = (start[:-1, None] + torch.arange(most, device="cuda")).clamp(max=rows - 1)       # repeated past a sequence's end
    q = (s["q"] * HEAD ** -0.5).view(rows, kv, per, HEAD)[member].transpose(1, 2).reshape(n, kv, most * per, HEAD)
    at = torch.arange(L, device="cuda")
    there = at < s["length"][:, None]
    if "first" in s:
        there &= at >= s["first"][:, None]
    there = there[member][:, None, :, None, :]                                                # [n][1][most][1][L]
    z = torch.matmul(q, K.transpose(2, 3)).view(n, kv, most, per, L).masked_fill(~there, -math.inf)
    top = z.amax(-1, keepdim=True) if L else z.new_zeros((n, kv, most, per, 1))
    e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    value = torch.matmul(e.view(n, kv, most * per, L), V).view(n, kv, most, per, HEAD)
    value = torch.where(total > 0, value / total, torch.zeros_like(value)).transpose(1, 2)    # [n][most][kv][per][64]
    place = torch.arange(rows, device="cuda")
    group = torch.searchsorted(start, place, right=True) - 1
    s["out"].copy_(value[group, place - start[group]].reshape(rows, c["heads"] * HEAD))
    return {"out": s["out"]}


def _next_tables(s):
    c, n, page, pages = s["case"], s["case"]["sequences"], s["case"]["page"], s["pages"]
    columns, far = s["table"].shape[1], 1 << 30
    parent, at = s["parent"].long(), torch.arange(columns, device="cuda")
    goes_on = (parent >= 0) & (parent < n)
    length = torch.where(goes_on, s["length"].long()[parent.clamp(0, n - 1)], torch.zeros_like(parent))
    kept = (length + page - 1) // page
    old = s["table"].long()[parent.clamp(0, n - 1)]
    mine = (at < kept[:, None]) & (old >= 0) & (old < pages)
    last = (at == length[:, None] // page) & mine                                             # pages that will be written
    # who keeps a page: a sequence that only reads it, or else the first of those that will write it
    claim = torch.where(last, 1 + torch.arange(n, device="cuda")[:, None], torch.zeros_like(old))
    owner = torch.full((pages + 1,), far, dtype=torch.long, device="cuda")
    owner.scatter_reduce_(0, torch.where(mine, old, torch.full_like(old, pages)).view(-1), claim.view(-1), "amin")
    copied = last & (owner[old.clamp(0, pages)] != claim)
    extra = (at >= kept[:, None]) & (at < ((s["want"].long() + page - 1) // page)[:, None])
    asked = copied | extra
    used = owner[:pages] < far
    free = torch.cumsum(~used, 0)
    in_use, granted = used.sum(), torch.minimum(asked.sum(), (~used).sum())
    # the free pages in order: first those that pages are moved into, then what the sequences ask for
    spots = torch.full((pages + 1,), -1, dtype=torch.long, device="cuda")
    number = torch.arange(pages, device="cuda")
    spots[torch.where(used, torch.full_like(free, pages), free - 1)] = torch.where(used, torch.full_like(number, -1), number)
    moves = used & (number >= in_use + granted) if c["compact"] else torch.zeros_like(used)
    n_moves = moves.sum()
    to = torch.where(moves, spots[(torch.cumsum(moves, 0) - 1).clamp(min=0)], number)
    rank = torch.cumsum(asked.view(-1), 0).view(n, columns) - 1
    spots[pages] = -1
    new = torch.where(rank < granted, spots[(n_moves + rank).clamp(0, pages - 1)], torch.full_like(rank, -1))
    s["new_table"].copy_(torch.where(asked, new, torch.where(mine, to[old.clamp(0, pages - 1)], torch.full_like(old, -1))))
    s["new_length"].copy_(length)
    s["room"].copy_((s["new_table"] >= 0).long().cumprod(1).sum(1) * page)
    took = copied & (new >= 0)
    s["info"].copy_(torch.stack([in_use + granted, asked.sum() - granted, took.sum(), n_moves]))
    for name in ("codes", "scales"):
        pool = s[name]
        src, dst = torch.cat([old[took], number[moves]]), torch.cat([new[took], to[moves]])
        pool[dst] = pool[src]
    return {n: s[n] for n in ("new_table", "new_length", "room", "info")} | _pool_out(s)


def _sample(s):
    c, rows, V = s["case"], s["case"]["rows"], s["case"]["vocab"]
    greedy = ~(s["temperature"] > 0)[:, None]
    T = torch.where(greedy, torch.ones_like(greedy, dtype=torch.float32), s["temperature"][:, None]).double()
    x = s["logits"].double()
    top = x.amax(1, keepdim=True)
    x = (x - top) / T
    w = torch.exp(x)
    order = torch.sort(s["logits"], dim=1, descending=True, stable=True).indices
    ws, rank = w.gather(1, order), torch.arange(V, device="cuda")
    k = torch.where(greedy, 1, s["top_k"][:, None] if "top_k" in s else V)
    ws = ws * (rank < k)
    keep = rank < k
    if "min_p" in s:
        keep &= ws >= s["min_p"][:, None].double()
    if "top_p" in s:
        p = torch.where(s["top_p"] < 1, s["top_p"].double(), torch.full_like(s["top_p"], math.inf, dtype=torch.float64))
        run = torch.cumsum(ws, 1)
        keep &= run - ws < p[:, None] * run[:, -1:]
    keep[:, 0] = True
    s["kept"].copy_(keep.sum(1))
    run = torch.cumsum(w * torch.zeros_like(keep).scatter_(1, order, keep), 1)
    s["token"].copy_(torch.searchsorted(run, s["u"].double() * run[:, -1:], right=True).clamp(max=V - 1))
    s["logprob"].copy_(x.gather(1, s["token"].long()) - torch.log(w.sum(1, keepdim=True)))
    return {n: s[n] for n in ("token", "logprob", "kept")}


def run(state):
    if own:
        return _run_own(state)
    return {"write": _write, "attend": _attend, "tables": _next_tables, "sample": _sample}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["op"] == "write":
        values = 2.0 * HEAD * case["heads"] * float(_spread(case["new_lo"], case["new_hi"], case["sequences"]).sum())
        return {"bytes": values * (1 + (2 if case["dtype"] == "bf16" else 4)) + 8.0 * case["sequences"], "flops": 2.0 * values}
    if case["op"] == "attend":
        rows = float(_spread(case["rows_lo"], case["rows_hi"], case["sequences"]).sum())
        keys = _spread(case["keys_lo"], case["keys_hi"], case["sequences"]).astype(np.float64)
        if case["window"]:
            keys = np.minimum(keys, case["window"])
        return {"bytes": float(keys.sum()) * case["kv_heads"] * (2 * HEAD + 8 / BLOCK)
                + rows * case["heads"] * HEAD * (4 + (2 if case["dtype"] == "bf16" else 4)) + 4 * rows,
                "flops": 4.0 * HEAD * case["heads"] * float(keys.sum()) * rows / case["sequences"]}
    if case["op"] == "tables":
        n, page = case["sequences"], case["page"]
        held = _spread(case["held_lo"], case["held_hi"], n).astype(np.float64)
        entries = float(((held + page) // page).sum())
        # pages copied: of a family of F the F (1 - (1 - 1/F)^F) that go on keep their last page, the others take a copy
        F = case["family"]
        copied = n * (1 - case["ended"]) * (1 - 1 / F) ** F if F > 1 else 0.0
        # pages moved: those in use behind the place of the last of them, of a pool that is evenly filled
        if case["compact"]:
            alive = entries * (1 - case["ended"])
            copied += alive * (1 - min(1.0, alive / (entries * case["spare"] + n)))
        return {"bytes": 8.0 * entries + 24.0 * n + 2 * copied * case["layers"] * 2 * case["heads"] * page * HEAD, "flops": 4.0 * entries}
    rows, V = case["rows"], case["vocab"]
    return {"bytes": float(rows) * V * (2 if case["dtype"] == "bf16" else 4) + rows * (24 + 12 * case["draws"]), "flops": 20.0 * rows * V}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------
def _e4m3_64(x):
    """Doubles of at most 448 in magnitude, rounded to the nearest of e4m3 (ties to even): steps of 2^-9 up to 2^-6, then of an
    eighth of the power of two below."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))).clamp(min=-6.0) - 3)
    return torch.round(x / step) * step


def _write64(s):
    c, page, blocks = s["case"], s["case"]["page"], s["case"]["page"] // BLOCK
    values, scales = s["codes"].view(F8).double(), s["scales"].double()
    start, table, held = s["token_start"].tolist(), s["table"].tolist(), s["length"].tolist()
    for i in range(c["sequences"]):
        done, count = held[i], start[i + 1] - start[i]
        while done < held[i] + count:
            b, first = done // BLOCK, done % BLOCK
            n = min(BLOCK - first, held[i] + count - done)
            p, j = table[i][b // (page // BLOCK)], b % blocks
            row = start[i] + done - held[i]
            for m, name in enumerate(("k", "v")):
                x = s[name][row:row + n].double().view(n, c["heads"], HEAD).transpose(0, 1)         # [H][n][64]
                top = x.abs().amax((1, 2))
                need = torch.exp2(torch.ceil(torch.log2((top / 448).clamp(min=LEAST))))
                need = torch.where(need * 224 >= top, need / 2, need).clamp(min=LEAST)              # (log2 is not exact)
                need = torch.where(need * 448 < top, need * 2, need)
                was = values[p, m, :, j] if m == 0 else values[p, m, :, j].transpose(1, 2)          # [H][tokens][64]
                to = torch.maximum(scales[p, m, :, j], need) if first else need
                if first:
                    was[:, :first] = _e4m3_64(was[:, :first] * (scales[p, m, :, j] / to)[:, None, None])
                was[:, first:first + n] = _e4m3_64(x / to[:, None, None])
                scales[p, m, :, j] = to
            done += n
    return {"codes": values[:s["pages"]], "scales": scales[:s["pages"]]}


def _attend64(s):
    c, kv, page = s["case"], s["case"]["kv_heads"], s["case"]["page"]
    per = c["heads"] // kv
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    start, length = s["row_start"].tolist(), s["length"].tolist()
    first = s["first"].tolist() if "first" in s else [0] * s["rows"]
    for i in range(c["sequences"]):
        rows = range(start[i], start[i + 1])
        top = max(length[r] for r in rows)
        if top == 0:
            continue
        t = s["table"][i, :(top + page - 1) // page].long()
        x = s["codes"][t].view(F8).double() * s["scales"][t].double()[..., None, None]              # [pages][2][kv][blocks][64][64]
        for h in range(kv):
            k, v = x[:, 0, h].reshape(-1, HEAD), x[:, 1, h].transpose(-1, -2).reshape(-1, HEAD)
            cols = slice(h * per * HEAD, (h + 1) * per * HEAD)
            for r in rows:
                a, b = first[r], length[r]
                if a < b:
                    q = s["q"][r, cols].double().view(per, HEAD) / math.sqrt(HEAD)
                    out[r, cols] = (torch.softmax(q @ k[a:b].T, 1) @ v[a:b]).reshape(-1)
    return {"out": out}


def _tables64(s):
    c, page, pages, n = s["case"], s["case"]["page"], s["pages"], s["case"]["sequences"]
    table, held, parent, want = (s[m].tolist() for m in ("table", "length", "parent", "want"))
    columns = len(table[0])
    length = [held[p] if 0 <= p < n else 0 for p in parent]
    read, write = set(), {}
    for i in range(n):
        for j in range((length[i] + page - 1) // page):
            p = table[parent[i]][j]
            if j < length[i] // page:
                read.add(p)
            else:
                write.setdefault(p, i)
    used = read | set(write)
    spots = [p for p in range(pages) if p not in used]
    asks, new, copies = [], [[-1] * columns for _ in range(n)], []
    for i in range(n):
        for j in range(max((length[i] + page - 1) // page, (want[i] + page - 1) // page)):
            if j * page >= length[i]:
                asks.append((i, j, None))
            elif j >= length[i] // page and (table[parent[i]][j] in read or write[table[parent[i]][j]] != i):
                asks.append((i, j, table[parent[i]][j]))
            else:
                new[i][j] = table[parent[i]][j]
    granted = min(len(asks), len(spots))
    end = len(used) + granted
    moves = {p: spots[m] for m, p in enumerate(sorted(p for p in used if p >= end))} if c["compact"] else {}
    new = [[moves.get(p, p) for p in row] for row in new]
    for a, (i, j, p) in enumerate(asks[:granted]):
        new[i][j] = spots[len(moves) + a]
        if p is not None:
            copies.append((p, new[i][j]))
    info = [end, len(asks) - granted, len(copies), len(moves)]
    copies += list(moves.items())
    codes, scales = s["codes"][:pages].view(F8).double(), s["scales"][:pages].double()
    for src, dst in copies:
        codes[dst], scales[dst] = codes[src], scales[src]
    room = [(row + [-1]).index(-1) * page for row in new]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"new_table": i32(new), "new_length": i32(length), "room": i32(room), "info": i32(info), "codes": codes, "scales": scales}


def _sample64(s):
    c, V = s["case"], s["case"]["vocab"]
    get = {m: s[m].cpu().numpy() for m in ("u", "temperature", "top_k", "top_p", "min_p") if m in s}
    token, logprob, kept = [], [], []
    for r in range(c["rows"]):
        x = s["logits"][r].double().cpu().numpy()
        T = float(get["temperature"][r])
        order = np.argsort(-x, kind="stable")
        z = (x - x[order[0]]) / (T if T > 0 else 1.0)
        w = np.exp(z)
        n = min(int(get["top_k"][r]), V) if "top_k" in get else V
        best = w[order[:n]]
        if "top_p" in get and get["top_p"][r] < 1:
            before = np.concatenate([[0.0], np.cumsum(best)[:-1]])
            n = min(n, int(np.sum(before < float(get["top_p"][r]) * best.sum())))
        if "min_p" in get:
            n = min(n, int(np.sum(best >= float(get["min_p"][r]))))
        n = max(n, 1) if T > 0 else 1
        some = np.zeros(V)
        some[order[:n]] = w[order[:n]]
        run = np.cumsum(some)
        t = np.searchsorted(run, get["u"][r].astype(np.float64) * run[-1], side="right")
        token.append(t)
        logprob.append(z[t] - np.log(w.sum()))
        kept.append(n)
    return {"token": _dev(np.stack(token).astype(np.int32)), "logprob": _dev(np.stack(logprob)), "kept": _dev(np.array(kept, np.int32))}


def exact(case, seed):
    s = prepare(case, seed)
    # loops over rows and heads, or over sequences and blocks: some tens of thousands of small steps are what fits the time
    if case["op"] == "attend" and s["rows"] * case["kv_heads"] > 12000:
        return None
    return {"write": _write64, "attend": _attend64, "tables": _tables64, "sample": _sample64}[case["op"]](s)
