"""The paged cache and the sampler together, as a program decodes with them: prompts are written, tokens drawn, sequences forked,
ended and refilled by tables, new keys written and attended to, step after step, one of the steps with the pool compacted.  A
plain list of keys and values for each sequence follows the same decisions."""
import numpy as np
import pytest
import torch

import page_util as P
from gpu_util import needs_gpu

pytestmark = [pytest.mark.gpu, needs_gpu]


def dev(a, kind=np.int32):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a).astype(kind))).cuda()


@pytest.mark.parametrize("layers", [1, 2])
def test_decoding_by_chance(layers):
    from paper_2603_11273_amd import asr
    rng = np.random.default_rng(layers)
    n, H, V, page, columns, pages = 7, 2, 211, 64, 5, 26
    shape = (pages, layers, 2, H, page // 64, 64, 64)
    codes, scales = torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda"), torch.full(shape[:5], float("nan"), device="cuda")
    table, length = dev(np.full((n, columns), -1)), dev(np.zeros(n))
    parent, want, room, info = dev(np.full(n, -1)), dev(np.zeros(n)), dev(np.zeros(n)), dev(np.zeros(4))
    rows = dev(np.zeros(n))                                 # keys that each row sees
    tables = asr.PageTables(codes, scales, table, length, parent=parent, want=want, room=room, info=info, page=page)
    write = [asr.PageWrite(codes[:, i], scales[:, i], table, length, tokens=n, dtype=torch.float32) for i in range(layers)]
    attend = [asr.PagedAttention(codes[:, i], scales[:, i], table, rows, n_head=2 * H, rows=n, dtype=torch.float32) for i in range(layers)]
    temperature, top_k = dev(np.full(n, 0.8), np.float32), dev(np.full(n, 40))
    sampler = asr.Sampler(n, V, torch.float32, temperature=temperature, top_k=top_k)
    emb = rng.standard_normal((V, 2 * H * 64)).astype(np.float32)       # a token's query; keys and values are cut from it
    out_w = rng.standard_normal((2 * H * 64, V)).astype(np.float32) * 0.3
    E, W = dev(emb, np.float32), dev(out_w, np.float32)
    # the plain side: per sequence and layer one page pool of its own that P.write fills
    plain = [None] * n

    def fresh():
        return [(np.zeros((columns, 2, H, 1, 64, 64), np.uint8), np.zeros((columns, 2, H, 1), np.float32)) for _ in range(layers)]

    tokens = dev(rng.integers(0, V, (n, 1)))
    held = [0] * n
    # prompts of several lengths, written at once
    prompt = np.array([1, 63, 64, 65, 5, 130, 0])
    want.copy_(dev(prompt + 1))
    tables()
    assert room.cpu().numpy().min() >= page and info.cpu().numpy()[1] == 0
    start = np.concatenate([[0], np.cumsum(prompt)])
    text = rng.integers(0, V, prompt.sum())
    for i in range(layers):
        k, v = emb[text] * (1 + i), emb[text][:, ::-1] * (1 + i)
        k, v = np.ascontiguousarray(k[:, :H * 64]), np.ascontiguousarray(v[:, :H * 64])
        asr.PageWrite(codes[:, i], scales[:, i], table, length, tokens=len(text), dtype=torch.float32, max_new=int(prompt.max()),
                      token_start=dev(start))(dev(k, np.float32), dev(v, np.float32))
        for s in range(n):
            plain[s] = plain[s] or fresh()
            P.write(*plain[s][i], np.arange(columns)[None], [0], [0, prompt[s]], k[start[s]:start[s + 1]].astype(np.float64),
                    v[start[s]:start[s + 1]].astype(np.float64), 1 << 20)
    held = list(prompt)
    length.copy_(dev(prompt))
    ident = np.arange(n)
    choices = [ident, [0, 0, 2, 2, 2, 5, 5], ident, [1, 0, 2, 3, -1, 5, 5], ident, [5, 5, 5, 5, 5, 5, 5], [0, 1, -1, -1, 4, -1, 6], ident,
               [0, 0, 0, 0, 0, 0, 0], ident]
    for step, choice in enumerate(choices):
        parent.copy_(dev(choice))
        grown = [held[c] + 1 if c >= 0 else 1 for c in choice]
        want.copy_(dev(grown))
        tables(compact=step in (3, 6))
        assert info.cpu().numpy()[1] == 0 and (room.cpu().numpy() >= grown).all()
        assert step not in (3, 6) or table.max().item() + 1 == info[0].item()
        plain = [[(a.copy(), b.copy()) for a, b in plain[c]] if c >= 0 else fresh() for c in choice]
        held = [g - 1 for g in grown]
        assert length.cpu().tolist() == held
        x = E[tokens.view(-1).long()]
        for i in range(layers):
            k, v = (x * (1 + i))[:, :H * 64].contiguous(), (x.flip(1) * (1 + i))[:, :H * 64].contiguous()
            write[i](k, v)
            for s in range(n):
                P.write(*plain[s][i], np.arange(columns)[None], [held[s]], [0, 1], k[s:s + 1].double().cpu().numpy(),
                        v[s:s + 1].double().cpu().numpy(), 1)
        rows.copy_(length + 1)
        mix = torch.zeros((n, 2 * H * 64), device="cuda")
        for i in range(layers):
            o = attend[i](x.contiguous(), torch.empty_like(mix))
            got, q = o.double().cpu().numpy(), x.double().cpu().numpy()
            for s in range(n):
                a, b = plain[s][i]
                value = P.VALUE[a] * b[..., None, None].astype(np.float64)
                for h in range(2 * H):
                    K = value[:, 0, h // 2].reshape(-1, 64)[:held[s] + 1]
                    U = value[:, 1, h // 2].transpose(0, 1, 3, 2).reshape(-1, 64)[:held[s] + 1]
                    z = K @ q[s, h * 64:h * 64 + 64] / 8
                    p = np.exp(z - z.max())
                    ref = p / p.sum() @ U
                    # (scores below 40 in sums |q k| below 160: 66 steps of 2^-24 of that and 2^-22 of the score, twice on the weights)
                    assert np.abs(got[s, h * 64:h * 64 + 64] - ref).max() <= 2 * (66 * 160 + 4 * 40 + 2 * 400) * 2.0 ** -24 * np.abs(U).max()
            mix += o
        logits = mix @ W
        u = torch.rand((n, 1), device="cuda")
        sampler(logits, u, tokens)
        l = logits.double().cpu().numpy()
        for s in range(n):
            t, _, _, slack = P.sample(l[s], u[s].cpu().numpy(), np.float32(0.8), 40)
            assert tokens[s, 0].item() == t[0] or slack < 2.0 ** -36
        length.add_(1)
        held = grown
