"""Pages of e4m3 codes on the CPU: what codes stand for, rounding to them, writing, the next step's tables, attention and sampling,
each from its definition in include/asr.h, in 64 bits or whole numbers."""
import numpy as np


def _values():
    v = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = np.nan if c & 127 == 127 else (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        v[c] = -x if c & 128 else x
    return v


VALUE = _values()
STEPS = VALUE[:127]                                   # 0 .. 448, rising


def encode(x):
    """Codes of doubles: the nearest value, ties to the even code, past 448 448; what is not finite NaN (0x7f)."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.nan_to_num(np.abs(x), nan=0.0, posinf=448.0), 448.0)
    hi = np.searchsorted(STEPS, a).clip(max=126)      # STEPS[hi - 1] < a <= STEPS[hi]
    lo = np.maximum(hi - 1, 0)
    mid = (STEPS[lo] + STEPS[hi]) / 2
    code = np.where(a > mid, hi, np.where(a < mid, lo, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(a == STEPS[hi], hi, code)
    return np.where(np.isfinite(x), code | np.where(np.signbit(x), 128, 0), 0x7f).astype(np.uint8)


def power_at_least(x):
    """The smallest power of two in [2^-120, 2^120] that is not below x > 0."""
    if not x <= 2.0 ** 120:
        return 2.0 ** 120
    m, e = np.frexp(max(float(x), 2.0 ** -120))
    return 2.0 ** (e - 1 if m == 0.5 else e)


def write(codes, scales, table, length, start, k, v, max_new):
    """In place: codes uint8 [pages][2][H][blocks][64][64], scales float32; k, v [tokens][H * 64] doubles."""
    pages, _, H, blocks = codes.shape[:4]
    page, columns = blocks * 64, table.shape[1]
    for s in range(len(table)):
        a, b = max(int(start[s]), 0), min(int(start[s + 1]), len(k))
        n = min(b - a, max_new)
        if length[s] < 0 or n <= 0:
            continue
        p0, end = int(length[s]), min(int(length[s]) + n, columns * page)
        while p0 < end:
            p1 = min(p0 // 64 * 64 + 64, end)
            pg, j, i = table[s, p0 // page], p0 % page // 64, p0 % 64
            if 0 <= pg < pages:
                for m, src in enumerate((k, v)):
                    for h in range(H):
                        block = codes[pg, m, h, j] if m == 0 else codes[pg, m, h, j].T      # [position][dim], a view
                        x = src[a + p0 - length[s]:a + p1 - length[s], h * 64:h * 64 + 64]
                        fine = np.abs(x[np.isfinite(x)])
                        scale = power_at_least(fine.max(initial=0.0) / 448)
                        if i:
                            was = float(scales[pg, m, h, j])
                            held = power_at_least(was) if was > 0 else 2.0 ** -120
                            scale = max(scale, held)
                            if was != scale:
                                by = (was if was > 0 else 2.0 ** -120) / scale
                                with np.errstate(invalid="ignore"):
                                    block[:i] = encode(VALUE[block[:i]] * by)
                        block[i:i + p1 - p0] = encode(x / scale)
                        scales[pg, m, h, j] = scale
            p0 = p1


def next_tables(table, length, parent, want, page, pages, compact):
    """(new table, new length, room, info, [(from, to), ..] of pages whose data moves)."""
    n, columns = table.shape
    parent = np.arange(n) if parent is None else parent
    want = np.zeros(n, int) if want is None else want
    clip = lambda x: int(min(max(int(x), 0), columns * page))  # noqa: E731
    lens = [clip(length[p]) if 0 <= p < n else 0 for p in parent]
    ok = lambda p: 0 <= p < pages  # noqa: E731
    readers, writer = set(), {}
    for s in range(n):
        for j in range(-(-lens[s] // page)):
            p = int(table[parent[s], j])
            if ok(p):
                if j < lens[s] // page:
                    readers.add(p)
                else:
                    writer.setdefault(p, s)
    used = readers | set(writer)
    free = [p for p in range(pages) if p not in used]
    new = np.full((n, columns), -1, np.int64)
    asks = []
    for s in range(n):
        kept = -(-lens[s] // page)
        for j in range(max(kept, -(-clip(want[s]) // page))):
            if j >= kept:
                asks.append((s, j, None))
                continue
            p = int(table[parent[s], j])
            if not ok(p):
                continue
            if j == lens[s] // page and (p in readers or writer[p] != s):
                asks.append((s, j, p))
            else:
                new[s, j] = p
    granted = min(len(asks), len(free))
    end = len(used) + granted
    moved = [p for p in sorted(used) if p >= end] if compact else []
    to = dict(zip(moved, free))
    new = np.vectorize(lambda p: to.get(int(p), int(p)), otypes=[np.int64])(new) if new.size else new
    copies = []
    for (s, j, p), spot in zip(asks, free[len(moved):]):
        new[s, j] = spot
        if p is not None:
            copies.append((p, spot))
    room = [page * (list(row) + [-1]).index(-1) if -1 in row else page * columns for row in new.tolist()]
    info = [end, len(asks) - granted, len(copies), len(moved)]
    return new, np.array(lens), np.array(room), np.array(info), copies + sorted(to.items())


def sample(logits, u, T=None, k=None, p=None, m=None):
    """One row: (tokens, logprobs, kept, slack): slack is how near a decision lies to turning out otherwise."""
    l = np.asarray(logits, np.float64)
    V = len(l)
    if np.isnan(l).any() or (l == np.inf).any():
        return [-1] * len(u), [np.nan] * len(u), 0, 1.0
    if not (l > -np.inf).any():
        return [-1] * len(u), [-np.inf] * len(u), 0, 1.0
    greedy = T is not None and not T > 0
    T = 1.0 if T is None or greedy else float(T)
    order = np.argsort(-l, kind="stable")
    z = np.where(l > -np.inf, l - l[order[0]], -np.inf)
    z = np.where(l > -np.inf, z / T, -np.inf)
    w = np.exp(z)
    some = int((l > -np.inf).sum())
    n = 1 if greedy else min(some, int(k)) if k is not None and k > 0 else some
    slack = 1.0
    if not greedy:
        best = w[order[:n]]
        first = n
        if p is not None and p < 1:
            run = np.cumsum(best)
            before = np.concatenate([[0.0], run[:-1]])
            first = max(1, int((before < float(p) * run[-1]).sum()))
            slack = min(slack, np.abs(before[1:] / run[-1] - float(p)).min(initial=1.0))
        if m is not None and m > 0:
            first = min(first, max(1, int((best >= float(m)).sum())))
            slack = min(slack, np.abs(best[1:] - float(m)).min(initial=1.0))
        n = first
    some = np.zeros(V)
    some[order[:n]] = w[order[:n]]
    run = np.cumsum(some)
    tokens = []
    for x in u:
        x = min(max(float(x), 0.0), 1 - 2.0 ** -24) if x == x else 0.0
        tokens.append(int(np.searchsorted(run, x * run[-1], side="right")))
        slack = min(slack, np.abs(run / run[-1] - x).min() if x > 0 else 1.0)
    return tokens, [z[t] - np.log(w.sum()) for t in tokens], n, slack
