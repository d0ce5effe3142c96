"""What a decode step needs to carry several hypotheses of one clip, as a user's program calls it.

Two operators, each over the sizes it is used at:

* attend   one new token per hypothesis attends over the keys that its group shares (a clip's audio, a prompt) and over the
           hypothesis's own keys behind them: asr.SharedAttention;
* rules    penalties for repeated tokens, biases and grammar masks on the logits of a step, then the k best tokens with their
           log-probabilities: asr.LogitRules.

A program keeps its caches, histories and masks in device memory and a plan per batch shape, and sends it new queries or new
logits.  Lengths are spread evenly between their bounds and dealt to the rows by the seed, so a case's work does not depend on it.
"""
import math

import numpy as np
import torch

own = False

HEAD = 64
# what a drawn case has at most, as the largest listed ones: bytes of keys and values, scores, logits
MOST_BYTES = 2.8e9
MOST_SCORES = 128 * 20 * 65536
MOST_LOGITS = 256 * 131071


def listed():
    return [
        # the float32 model on a development machine: one row, one clip, a few tokens in
        {"name": "attend_tiny_1", "op": "attend", "dtype": "f32", "heads": 6, "kv_heads": 6, "groups": 1, "group_lo": 1,
         "group_hi": 1, "prefix_lo": 1500, "prefix_hi": 1500, "own_lo": 17, "own_hi": 17},
        # five beams of one clip on the large model: what a lone request waits for at every token
        {"name": "attend_large_5", "op": "attend", "dtype": "bf16", "heads": 20, "kv_heads": 20, "groups": 1, "group_lo": 5,
         "group_hi": 5, "prefix_lo": 1500, "prefix_hi": 1500, "own_lo": 40, "own_hi": 40},
        # a full decode batch of beams, five to a clip, their texts of all lengths (one of them empty)
        {"name": "attend_large_24x5", "op": "attend", "dtype": "bf16", "heads": 20, "kv_heads": 20, "groups": 24, "group_lo": 5,
         "group_hi": 5, "prefix_lo": 1500, "prefix_hi": 1500, "own_lo": 0, "own_hi": 224},
        # float32, ragged everywhere: prompts from one token on, groups of one hypothesis to eight
        {"name": "attend_f32_ragged_11", "op": "attend", "dtype": "f32", "heads": 8, "kv_heads": 8, "groups": 11, "group_lo": 1,
         "group_hi": 8, "prefix_lo": 1, "prefix_hi": 1499, "own_lo": 0, "own_hi": 447},
        # one recording of many segments as the shared context of 64 rows
        {"name": "attend_long_1x64", "op": "attend", "dtype": "bf16", "heads": 20, "kv_heads": 20, "groups": 1, "group_lo": 64,
         "group_hi": 64, "prefix_lo": 30011, "prefix_hi": 30011, "own_lo": 1, "own_hi": 448},
        # a decoder whose query heads share key heads, ragged prompts
        {"name": "attend_shared_heads_16", "op": "attend", "dtype": "bf16", "heads": 32, "kv_heads": 8, "groups": 16,
         "group_lo": 1, "group_hi": 8, "prefix_lo": 515, "prefix_hi": 8191, "own_lo": 1, "own_hi": 512},
        # the largest: eight long recordings, sixteen rows on each
        {"name": "attend_long_8x16", "op": "attend", "dtype": "bf16", "heads": 20, "kv_heads": 20, "groups": 8, "group_lo": 16,
         "group_hi": 16, "prefix_lo": 65536, "prefix_hi": 65536, "own_lo": 1, "own_hi": 448},
        # greedy decoding of one clip with suppressed tokens and a repetition penalty
        {"name": "rules_greedy_1", "op": "rules", "dtype": "f32", "rows": 1, "vocab": 51865, "k": 1, "out": False, "history": 24,
         "prompt": 4, "penalties": True, "biases": 0, "masks": 1, "temperature": False},
        # five beams: twice as many candidates, hot words, a grammar state each
        {"name": "rules_beam_5", "op": "rules", "dtype": "f32", "rows": 5, "vocab": 51866, "k": 10, "out": False, "history": 224,
         "prompt": 56, "penalties": True, "biases": 50, "masks": 3, "temperature": False},
        # every decode slot busy, greedy
        {"name": "rules_greedy_128", "op": "rules", "dtype": "f32", "rows": 128, "vocab": 51866, "k": 1, "out": False,
         "history": 447, "prompt": 4, "penalties": True, "biases": 0, "masks": 2, "temperature": False},
        # bf16 logits of another tokenizer, processed logits returned for a sampler of the program's own
        {"name": "rules_sample_37", "op": "rules", "dtype": "bf16", "rows": 37, "vocab": 32771, "k": 0, "out": True,
         "history": 300, "prompt": 100, "penalties": True, "biases": 7, "masks": 0, "temperature": True},
        # the largest: a big vocabulary, long contexts, logits and candidates
        {"name": "rules_long_256", "op": "rules", "dtype": "bf16", "rows": 256, "vocab": 131071, "k": 5, "out": True,
         "history": 32768, "prompt": 30000, "penalties": True, "biases": 300, "masks": 9, "temperature": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.5:
        kv = rng.choice([1, 2, 4, 6, 8, 12, 16, 20])
        per = rng.choice([1, 1, 1, 2, 4, 5, 8])
        if kv * per > 40:
            per = 1
        dtype = rng.choice(["bf16", "bf16", "f32"])
        groups = _log_int(rng, 1, 32)
        hi = _log_int(rng, 1, min(64, 128 // groups))
        room = min(MOST_BYTES / (groups * kv * HEAD * 2 * (2 if dtype == "bf16" else 4)), MOST_SCORES / (groups * hi * kv * per))
        prefix_hi = _log_int(rng, 1, int(min(65536, room)))
        own_hi = rng.randint(0, 512)
        return {"op": "attend", "dtype": dtype, "heads": kv * per, "kv_heads": kv, "groups": groups,
                "group_lo": rng.randint(1, hi), "group_hi": hi, "prefix_lo": rng.choice([0, 1, prefix_hi // 2, prefix_hi]),
                "prefix_hi": prefix_hi, "own_lo": rng.randint(0, own_hi), "own_hi": own_hi}
    rows = _log_int(rng, 1, 256)
    k = rng.choice([0, 1, 1, 2, 5, 10, 16])
    history = _log_int(rng, 1, 32768)
    return {"op": "rules", "dtype": rng.choice(["bf16", "f32"]), "rows": rows,
            "vocab": _log_int(rng, 33, min(131071, MOST_LOGITS // rows)), "k": k, "out": k == 0 or rng.random() < 0.4,
            "history": history, "prompt": rng.randint(0, history), "penalties": rng.random() < 0.8,
            "biases": rng.choice([0, 1, 20, 300]), "masks": rng.choice([0, 1, 5, 40]), "temperature": rng.random() < 0.5}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _spread(lo, hi, n):
    """n whole numbers spread evenly over [lo, hi]."""
    return np.rint(np.linspace(hi, lo, n)).astype(np.int32) if n > 1 else np.array([hi], np.int32)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _sizes(case):
    """Rows of each group, in the order of the groups, for one seed's dealing or none."""
    return _spread(case["group_lo"], case["group_hi"], case["groups"])


def _attend_inputs(case, seed):
    rng = np.random.default_rng([seed, 3])
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    sizes = rng.permutation(_sizes(case))
    rows, groups, kv = int(sizes.sum()), case["groups"], case["kv_heads"]
    # a pool of cache slots, a few more than are in use, taken in any order; a row's own keys start somewhere in its slot,
    # as the text of a hypothesis starts behind the prompt
    first = rng.integers(0, 9, rows).astype(np.int32)
    prefix = torch.randn((groups + 1, 2, kv, case["prefix_hi"], HEAD), generator=g, dtype=kind, device="cuda")
    text = torch.randn((rows + 1, 2, kv, case["own_hi"] + 9, HEAD), generator=g, dtype=kind, device="cuda")
    # queries that make some keys matter: scores of a few units
    q = 2.0 * torch.randn((rows, case["heads"] * HEAD), generator=g, dtype=torch.float32, device="cuda")
    return {
        "case": case, "rows": rows, "q": q, "out": torch.zeros((rows, case["heads"] * HEAD), dtype=kind, device="cuda"),
        "prefix_k": prefix[:, 0], "prefix_v": prefix[:, 1], "own_k": text[:, 0], "own_v": text[:, 1],
        "group_start": _dev(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)),
        "row_of": _dev(rng.permutation(rows).astype(np.int32)),
        "prefix_slot": _dev(rng.permutation(groups + 1)[:groups].astype(np.int32)),
        "prefix_len": _dev(rng.permutation(_spread(case["prefix_lo"], case["prefix_hi"], groups))),
        "own_slot": _dev(rng.permutation(rows + 1)[:rows].astype(np.int32)), "own_first": _dev(first),
        "own_len": _dev(rng.permutation(_spread(case["own_lo"], case["own_hi"], rows))),
    }


def _rules_inputs(case, seed):
    rng = np.random.default_rng([seed, 5])
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, V, n = case["rows"], case["vocab"], case["history"]
    x = torch.randn((rows, V), generator=g, dtype=torch.float32, device="cuda") * 3.0 - 4.0
    state = {"case": case, "logits": x.to(torch.bfloat16) if case["dtype"] == "bf16" else x}
    if case["out"]:
        state["out"] = torch.empty((rows, V), dtype=torch.float32, device="cuda")
    if case["k"]:
        state["token"] = torch.empty((rows, case["k"]), dtype=torch.int32, device="cuda")
        state["logprob"] = torch.empty((rows, case["k"]), dtype=torch.float32, device="cuda")
    if case["penalties"]:
        # tokens as texts repeat them: few often, many once; histories from one token to the longest
        words = torch.rand((rows, n), generator=g, dtype=torch.float64, device="cuda")
        state["history"] = (torch.exp(words * math.log(V)) - 1.0).clamp(0, V - 1).to(torch.int32)
        lens = rng.permutation(_spread(max(1, n // 8), n, rows)).astype(np.int32)
        state["history_len"] = _dev(lens)
        state["prompt_len"] = _dev(np.minimum(lens, case["prompt"]).astype(np.int32))
        state["repetition"] = _dev(rng.uniform(1.0, 1.5, rows).astype(np.float32))
        state["frequency"] = _dev(rng.uniform(0.0, 0.5, rows).astype(np.float32))
        state["presence"] = _dev(rng.uniform(0.0, 1.0, rows).astype(np.float32))
    if case["biases"]:
        b = min(case["biases"], V)
        state["bias_token"] = _dev(np.stack([rng.choice(V, b, replace=False) for _ in range(rows)]).astype(np.int32))
        state["bias_value"] = _dev(rng.uniform(-4.0, 6.0, (rows, b)).astype(np.float32))
        state["bias_len"] = _dev(rng.integers(0, b + 1, rows).astype(np.int32))
    if case["masks"]:
        # grammar states: some forbid a few tokens, some allow a few, and the last of many allows none
        words = (V + 31) // 32
        share = np.linspace(0.98, 0.02, case["masks"])
        allowed = torch.rand((case["masks"], words * 32), generator=g, device="cuda") < _dev(share.astype(np.float32))[:, None]
        if case["masks"] > 4:
            allowed[-1] = False
        weights = 2 ** torch.arange(32, dtype=torch.int64, device="cuda")
        packed = (allowed.view(case["masks"], words, 32).long() * weights).sum(-1)
        state["mask"] = torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).to(torch.int32)
        state["mask_of"] = _dev(rng.integers(-1 if case["masks"] > 1 else 0, case["masks"], rows).astype(np.int32))
    if case["temperature"]:
        state["temperature"] = _dev(rng.uniform(0.2, 1.2, rows).astype(np.float32))
    return state


def prepare(case, seed):
    return _attend_inputs(case, seed) if case["op"] == "attend" else _rules_inputs(case, seed)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _plan(s):
    """The plan that a program makes once for a batch shape and the buffers it keeps."""
    from paper_2603_11273_amd import asr
    c = s["case"]
    if c["op"] == "attend":
        return asr.SharedAttention(
            s["prefix_k"], s["prefix_v"], s["own_k"], s["own_v"], n_head=c["heads"], rows=s["rows"], groups=c["groups"],
            max_group=c["group_hi"], group_start=s["group_start"], row_of=s["row_of"], prefix_slot=s["prefix_slot"],
            prefix_len=s["prefix_len"], max_prefix=c["prefix_hi"], own_slot=s["own_slot"], own_first=s["own_first"],
            own_len=s["own_len"], max_own=c["own_hi"], scale=HEAD ** -0.5)
    names = ("history", "history_len", "prompt_len", "repetition", "frequency", "presence", "bias_token", "bias_value",
             "bias_len", "mask", "mask_of", "temperature")
    return asr.LogitRules(c["rows"], c["vocab"], s["logits"].dtype, k=c["k"], **{n: s[n] for n in names if n in s})


def _run_own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    if s["case"]["op"] == "attend":
        s["plan"](s["q"], s["out"])
    else:
        s["plan"](s["logits"], out=s.get("out"), token=s.get("token"), logprob=s.get("logprob"))
    return {n: s[n] for n in (("out",) if s["case"]["op"] == "attend" else ("out", "token", "logprob")) if n in s}


def _attend(s):
    c, rows, kv = s["case"], s["rows"], s["case"]["kv_heads"]
    per, L, O, most = c["heads"] // kv, c["prefix_hi"], c["own_hi"], c["group_hi"]
    start, row_of = s["group_start"].long(), s["row_of"].long()
    at = start[:-1, None] + torch.arange(most, device="cuda")
    member = row_of[at.clamp(max=rows - 1)]                                     # [groups][most], repeated past a group's end
    q = s["q"].view(rows, kv, per, HEAD) * HEAD ** -0.5
    # the shared keys, once for the queries of a group and key head
    slot = s["prefix_slot"].long()
    K, V = s["prefix_k"][slot].float(), s["prefix_v"][slot].float()
    qg = q[member].transpose(1, 2).reshape(c["groups"], kv, most * per, HEAD)
    there = torch.arange(L, device="cuda") < s["prefix_len"][:, None]
    shared = torch.matmul(qg, K.transpose(2, 3)).masked_fill(~there[:, None, None], -math.inf)
    # each row's own keys
    pos = s["own_first"].long()[:, None] + torch.arange(O, device="cuda")
    owns = s["own_slot"].long()[:, None]
    Ko, Vo = s["own_k"].transpose(1, 2)[owns, pos].float(), s["own_v"].transpose(1, 2)[owns, pos].float()   # [rows][O][kv][64]
    mine = torch.matmul(q, Ko.permute(0, 2, 3, 1))
    mine = mine.masked_fill(~(torch.arange(O, device="cuda") < s["own_len"][:, None])[:, None, None], -math.inf)
    # back to rows: place `j` of group `g` holds row row_of[start[g] + j]
    place = torch.empty_like(row_of)
    place[row_of] = torch.arange(rows, device="cuda")
    group = torch.searchsorted(start, place, right=True) - 1
    j = place - start[group]
    shared_rows = shared.view(c["groups"], kv, most, per, L)
    top = shared_rows.amax(-1).transpose(1, 2)[group, j]                        # [rows][kv][per]
    if O:
        top = torch.maximum(top, mine.amax(-1))
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    top_g = top[member].transpose(1, 2).reshape(c["groups"], kv, most * per, 1)
    e, eo = torch.exp(shared - top_g), torch.exp(mine - top[..., None])
    total = e.sum(-1).view(c["groups"], kv, most, per).transpose(1, 2)[group, j] + eo.sum(-1)
    value = torch.matmul(e, V).view(c["groups"], kv, most, per, HEAD).transpose(1, 2)[group, j]
    value = value + torch.matmul(eo, Vo.transpose(1, 2))
    value = torch.where(total[..., None] > 0, value / total[..., None], torch.zeros_like(value))
    s["out"].copy_(value.reshape(rows, c["heads"] * HEAD))
    return {"out": s["out"]}


def _rules(s):
    c, V = s["case"], s["case"]["vocab"]
    z = s["logits"].float()
    if c["penalties"]:
        at = torch.arange(c["history"], device="cuda")
        there = at < s["history_len"][:, None]
        said = there & (at >= s["prompt_len"][:, None])
        tokens = s["history"].long()
        count = torch.zeros(z.shape, dtype=torch.int32, device="cuda").scatter_add_(1, tokens, said.int())
        seen = torch.zeros(z.shape, dtype=torch.int32, device="cuda").scatter_add_(1, tokens, there.int()) > 0
        r = s["repetition"][:, None]
        z = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
        z = torch.where(count > 0, (z - s["frequency"][:, None] * count.float()) - s["presence"][:, None], z)
    if c["biases"]:
        there = torch.arange(s["bias_token"].shape[1], device="cuda") < s["bias_len"][:, None]
        value = torch.where(there, s["bias_value"], torch.zeros_like(s["bias_value"]))
        z = z + torch.zeros_like(z).scatter_add_(1, s["bias_token"].long(), value)
    if c["masks"]:
        v = torch.arange(V, device="cuda")
        allowed = (s["mask"][:, v // 32] >> (v % 32).int()) & 1
        of = s["mask_of"].long()
        z = z.masked_fill((of >= 0)[:, None] & (allowed[of.clamp(min=0)] == 0), -math.inf)
    if c["temperature"]:
        z = z / s["temperature"][:, None]
    result = {}
    if c["out"]:
        result["out"] = s["out"].copy_(z)
    if c["k"]:
        k = min(c["k"], V)
        value, token = torch.sort(z, dim=1, descending=True, stable=True)
        value, token = value[:, :k], token[:, :k]
        top = torch.where(value[:, :1] == -math.inf, torch.zeros_like(value[:, :1]), value[:, :1])
        total = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
        none = value == -math.inf
        s["token"].fill_(-1)
        s["logprob"].fill_(-math.inf)
        s["token"][:, :k] = torch.where(none, torch.full_like(token, -1), token).int()
        s["logprob"][:, :k] = torch.where(none, value, value - total)
        result |= {"token": s["token"], "logprob": s["logprob"]}
    return result


def run(state):
    if own:
        return _run_own(state)
    return _attend(state) if state["case"]["op"] == "attend" else _rules(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "attend":
        sizes = _sizes(case)
        rows = int(sizes.sum())
        prefix = float(_spread(case["prefix_lo"], case["prefix_hi"], case["groups"]).sum())
        text = float(_spread(case["own_lo"], case["own_hi"], rows).sum())
        row_bytes = 2.0 * case["kv_heads"] * HEAD * es
        keys = prefix * rows / case["groups"] + text
        return {"bytes": (prefix + text) * row_bytes + rows * case["heads"] * HEAD * (4 + es),
                "flops": 4.0 * HEAD * case["heads"] * keys}
    rows, V = case["rows"], case["vocab"]
    n = rows * V * (es + (4 if case["out"] else 0)) + rows * case["k"] * 8
    if case["penalties"]:
        n += 4 * int(_spread(max(1, case["history"] // 8), case["history"], rows).sum())
    if case["biases"]:
        n += rows * min(case["biases"], V) * 4
    if case["masks"]:
        n += min(case["masks"], rows) * ((V + 31) // 32) * 4
    return {"bytes": float(n), "flops": 8.0 * rows * V}


# ---------------------------------------------------------------------------
# The same in 64 bits
# ---------------------------------------------------------------------------
def _attend64(s):
    c, kv = s["case"], s["case"]["kv_heads"]
    per = c["heads"] // kv
    start, row_of = s["group_start"].tolist(), s["row_of"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    slots, lens = s["prefix_slot"].tolist(), s["prefix_len"].tolist()
    own_slot, first, own_len = s["own_slot"].tolist(), s["own_first"].tolist(), s["own_len"].tolist()
    for g in range(c["groups"]):
        for h in range(kv):
            k, v = (s[n][slots[g], h, :lens[g]].double() for n in ("prefix_k", "prefix_v"))
            rows = [row_of[i] for i in range(start[g], start[g + 1])]
            cols = slice(h * per * HEAD, (h + 1) * per * HEAD)
            q = s["q"][rows, cols].double().view(len(rows), per, HEAD) / math.sqrt(HEAD)
            shared = q @ k.T
            for i, r in enumerate(rows):
                a, b = first[r], first[r] + own_len[r]
                ko, vo = (s[n][own_slot[r], h, a:b].double() for n in ("own_k", "own_v"))
                if lens[g] + own_len[r] == 0:
                    continue
                p = torch.softmax(torch.cat([shared[i], q[i] @ ko.T], 1), 1)
                out[r, cols] = (p[:, :lens[g]] @ v + p[:, lens[g]:] @ vo).reshape(-1)
    return {"out": out}


def _rules64(s):
    c, V = s["case"], s["case"]["vocab"]
    get = {n: s[n].cpu().numpy() for n in s if isinstance(s[n], torch.Tensor) and n not in ("logits", "out", "token", "logprob")}
    rows, k = c["rows"], c["k"]
    out = torch.empty((rows, V), dtype=torch.float64, device="cuda")
    for r in range(rows):
        z = s["logits"][r].double()
        if c["penalties"]:
            n, p = int(get["history_len"][r]), int(get["prompt_len"][r])
            seen = torch.from_numpy(np.unique(get["history"][r, :n]).astype(np.int64)).cuda()
            z[seen] = torch.where(z[seen] > 0, z[seen] / float(get["repetition"][r]), z[seen] * float(get["repetition"][r]))
            token, count = np.unique(get["history"][r, p:n], return_counts=True)
            token, count = torch.from_numpy(token.astype(np.int64)).cuda(), torch.from_numpy(count).cuda()
            z[token] -= count * float(get["frequency"][r]) + float(get["presence"][r])
        if c["biases"]:
            n = int(get["bias_len"][r])
            z[_dev(get["bias_token"][r, :n].astype(np.int64))] += _dev(get["bias_value"][r, :n].astype(np.float64))
        if c["masks"] and get["mask_of"][r] >= 0:
            bits = np.unpackbits(get["mask"][get["mask_of"][r]].view(np.uint8), bitorder="little")[:V]
            z[_dev(bits == 0)] = -math.inf
        if c["temperature"]:
            z = z / float(get["temperature"][r])
        out[r] = z
    result = {"out": out} if c["out"] else {}
    if k:
        m = min(k, V)
        order = torch.sort(out, dim=1, descending=True, stable=True)
        token = torch.full((rows, k), -1, dtype=torch.int32, device="cuda")
        logprob = torch.full((rows, k), -math.inf, dtype=torch.float64, device="cuda")
        none = order.values[:, :m] == -math.inf
        token[:, :m] = order.indices[:, :m].int().masked_fill(none, -1)
        logprob[:, :m] = torch.log_softmax(out, 1).gather(1, order.indices[:, :m]).masked_fill(none, -math.inf)
        result |= {"token": token, "logprob": logprob}
    return result


def exact(case, seed):
    s = prepare(case, seed)
    # a loop over rows and key heads: some tens of thousands of small steps are what fits the time
    if case["op"] == "attend" and s["rows"] * case["kv_heads"] > 12000:
        return None
    return _attend64(s) if case["op"] == "attend" else _rules64(s)
