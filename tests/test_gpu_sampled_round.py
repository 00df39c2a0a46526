"""Rounds of a serving program that samples, every operator fed by the one before on the device: pages for the
lengths, rotary positions of a common projection's rows, attention of each layer, logits under penalties, sampled
tokens, acceptance, append, new lengths.  A first round brings prompts in beside a request that decodes, later ones verify trees.
The oracle runs the same rounds."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32, to_dev
from oracle import tr_oracle as O
from oracle import tr_prompt as P
from oracle import tr_serve as S
from paper_2406_17404_amd import binding as b
from paper_2406_17404_amd import inputs as I
from serve_util import ints, offsets_of

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


def rotated(x, at, freqs, got):
    """The oracle's rows in 16 bits; the device's have to be these but for a rounding, and go on as they are."""
    want = P.rotary(x, at, freqs, 1.0, False)
    assert (np.abs(got - want) <= HALF * np.abs(want) + 2.0 ** -20 * np.abs(x).max()).all()


@pytest.mark.parametrize("dh,scaling", [(64, b.ROTARY_PLAIN), (128, b.ROTARY_TURNS)])
def test_prompts_then_sampled_trees(dh, scaling):
    rng = np.random.default_rng(dh)
    B, layers, kv_heads, heads, V, width, n_blocks = 3, 2, 2, 4, 900, 12, 30
    rounds = [[150, 1, 70], [9, 1, 33], [9, 20, 33]]
    host = {w: np.full((layers, kv_heads, n_blocks, 32 * dh), 127, np.uint8) for w in "kv"}
    hscale = {w: np.full((layers, kv_heads, n_blocks), np.nan, np.float32) for w in "kv"}
    pool, scale = ({w: to_dev(x[w]) for w in "kv"} for x in (host, hscale))
    freqs, magnitude = b.trj_rotary_freqs(dh, 1e4, scaling, 8.0, 1.0, 4.0, 64)
    table, held, free, count, prefix = np.full((B, width), -1), np.zeros(B, int), np.arange(n_blocks), n_blocks, np.zeros(B, int)
    d = dict(table=i32(table), held=[i32(held), ints(B)], free=i32(free), count=[i32([count]), ints(1)], prefix=i32(prefix), new_len=ints(B))
    rules = np.array([[0.8, 40, 0.95, 0], [1, 0, 0.9, 0.02], [0, 0, 1, 0]], np.float32)
    pen = np.tile(np.array([[1.2, 0.3, 0.1]], np.float32), (B, 1))
    ctx = [list(rng.integers(0, 30, 5)) for _ in range(B)]
    for step, size in enumerate(rounds):
        chain = step == 0
        off, T = offsets_of(size), int(sum(size))
        parents = [np.arange(n) - 1 if chain else I.tree_random(n, rng) for n in size]
        at = [prefix[s] + (np.arange(n) if chain else P.depths(parents[s])) for s, n in enumerate(size)]
        qkv = torch.from_numpy(rng.normal(size=(layers, T, (heads + 2 * kv_heads) * dh)).astype(np.float32)).bfloat16()
        x = (rng.normal(size=(T, V)) * 3).astype(np.float32)
        u, tok = rng.random(T).astype(np.float32), rng.integers(0, V, T)
        if not chain:
            for s in range(B):  # drafts that are right more often than not
                for i in range(1, size[s]):
                    r, j = slice(off[s], off[s + 1]), off[s] + parents[s][i]
                    if rng.random() < 0.7:
                        y, _ = S.tree_logits(x[r], tok[r], parents[s], ctx[s], 5, pen[s], None, None, np.float32)
                        tok[off[s] + i] = P.sample(y[parents[s][i]], rules[s], u[j])[0]
        # ---- the device's round
        g = dict(off=i32(off), parent=i32(np.concatenate(parents)), tok=i32(tok), qkv=qkv.to(DEV))
        a, z, status, slot = step % 2, 1 - step % 2, [ints(B) for _ in range(7)], ints(T)
        b.kv_block_tables(d["table"], d["held"][a], d["prefix"], g["off"], T, d["free"], d["count"][a], d["held"][z], d["count"][z],
                          slot, status[0])
        outs, parts = [], []
        for l in range(layers):
            q, k, v = (t.unflatten(1, (-1, dh)) for t in g["qkv"][l].split([heads * dh, kv_heads * dh, kv_heads * dh], 1))
            b.rotary_rows(q, k, None if chain else g["parent"], g["off"], d["prefix"], freqs.to(DEV), magnitude, b.ROTARY_HALVES, q, k,
                          status[1])
            outs.append(torch.zeros(T, heads, dh, dtype=torch.bfloat16, device=DEV))
            cache = (pool["k"][l], pool["v"][l], scale["k"][l], scale["v"][l], k, v)
            if chain:
                ws = torch.empty(b.chunk_attention_q8_workspace_bytes(B, T, heads, kv_heads, dh, width * 32), dtype=torch.uint8, device=DEV)
                b.chunk_attention_q8(q, *cache, g["off"], d["table"], d["prefix"], width * 32, dh ** -0.5, ws, outs[-1], status[2])
            else:
                ws = torch.empty(b.tree_attention_q8_workspace_bytes(B, T, heads, kv_heads, dh, width * 32), dtype=torch.uint8, device=DEV)
                b.tree_attention_q8(q, *cache, g["parent"], g["off"], d["table"], d["prefix"], width * 32, dh ** -0.5, ws, outs[-1], status[2])
            parts.append((q, k, v))
        kr, vr = (torch.stack([p[i] for p in parts]) for i in (1, 2))
        if chain:
            b.kv_append_q8(pool["k"], pool["v"], scale["k"], scale["v"], kr, vr, None, None, g["off"], d["table"], d["prefix"],
                           d["new_len"], status[3])
        else:
            logits, token, prob = to_dev(x), ints(T), torch.zeros(T, device=DEV)
            ws = torch.empty(b.tree_logits_workspace_bytes(B, T, V), dtype=torch.uint8, device=DEV)
            b.tree_logits(logits, g["tok"], g["parent"], g["off"], i32(np.concatenate(ctx)), i32(offsets_of([len(c) for c in ctx])),
                          i32([5] * B), to_dev(pen), None, None, None, None, logits, None, ws, status[4])
            ws = torch.empty(b.tree_sample_workspace_bytes(B, T, V), dtype=torch.uint8, device=DEV)
            b.tree_sample(logits, g["off"], to_dev(rules), to_dev(u), token, prob, ws, status[5])
            acc, best, path, bonus = ints(B), ints(B), ints((B, 128)), ints(B)
            b.accept_path(None, g["tok"], g["parent"], g["off"], B, T, V, token, acc, best, path, bonus, status[6])
            b.kv_append_q8(pool["k"], pool["v"], scale["k"], scale["v"], kr, vr, path, acc, g["off"], d["table"], d["prefix"],
                           d["new_len"], status[3])
        d["prefix"].copy_(d["new_len"])
        torch.cuda.synchronize()
        # ---- the same by the oracle
        table, held, free, count, want_slot, refused = S.block_tables(table, held, prefix, off, T, free, count, n_blocks)
        assert np.array_equal(d["table"].cpu().numpy(), table) and not refused.any() and np.array_equal(slot.cpu().numpy(), want_slot)
        rows = [[t.float().cpu().numpy() for t in p] for p in parts]
        want_path, want_acc = np.full((B, 128), -1), np.full(B, -1)
        for s in range(B):
            r, pages = slice(off[s], off[s + 1]), table[s, :-(-prefix[s] // 32)]
            for l in range(layers):
                raw = qkv[l, r].float().numpy().reshape(size[s], -1, dh)
                rotated(raw[:, :heads], at[s], freqs.numpy(), rows[l][0][r])
                rotated(raw[:, heads:heads + kv_heads], at[s], freqs.numpy(), rows[l][1][r])
                assert np.array_equal(rows[l][2][r], raw[:, heads + kv_heads:])
                kv = [S.page_values(host[w][l], hscale[w][l], w)[:, pages].reshape(kv_heads, -1, dh)[:, :prefix[s]] for w in "kv"]
                want, mean = S.attention(rows[l][0][r], *kv, rows[l][1][r], rows[l][2][r], parents[s], dh ** -0.5)
                tol = HALF * (np.abs(want) + mean) * (1 + HALF) + 2.0 ** -12 * mean
                assert (np.abs(outs[l][r].float().cpu().numpy() - want) <= tol).all()
            if not chain:
                y, _ = S.tree_logits(x[r], tok[r], parents[s], ctx[s], 5, pen[s], None, None, np.float32)
                picks = [P.sample(y[i], rules[s], u[off[s] + i])[0] for i in range(size[s])]
                assert np.array_equal(token[r].cpu().numpy(), picks)
                n_acc, _, p, bonus_tok = O.accept_path(np.array(picks), tok[r], parents[s])
                want_acc[s], want_path[s, :len(p)] = n_acc, p
                ctx[s] += [int(tok[off[s] + i]) for i in p[1:]] + [int(bonus_tok)]
        if not chain:
            assert np.array_equal(acc.cpu().numpy(), want_acc) and np.array_equal(path.cpu().numpy(), want_path)
        k_all, v_all = (np.stack([rw[i] for rw in rows]) for i in (1, 2))
        prefix, bad = S.append(host["k"], host["v"], hscale["k"], hscale["v"], k_all, v_all, None if chain else want_path, want_acc, off, table, prefix)
        assert np.array_equal(d["new_len"].cpu().numpy(), prefix) and not bad.any()
        for w in "kv":
            assert np.array_equal(pool[w].cpu().numpy(), host[w]) and np.array_equal(scale[w].cpu().numpy(), hscale[w], equal_nan=True)
        assert not any(t.gt(0).any() for t in status)
    assert prefix[0] > 153


def test_a_round_captured_into_a_graph():
    """Two graphs of the same round with workspaces of their own, replayed in turn from a state that they change, with eager
    rounds between them: every replay is the eager round from the same state."""
    rng = np.random.default_rng(22)
    B, kv_heads, heads, dh, V, width, n_blocks = 3, 2, 8, 64, 40000, 16, 60
    size = [7, 1, 90]
    off, T = offsets_of(size), sum(size)
    qkv = torch.from_numpy(rng.normal(size=(T, heads + 2 * kv_heads, dh)).astype(np.float32)).bfloat16().to(DEV)
    x, node_off, u = to_dev((rng.normal(size=(T, V)) * 3).astype(np.float32)), i32(off), to_dev(rng.random(T).astype(np.float32))
    rules = to_dev(np.array([[0.8, 40, 0.95, 0], [1, 0, 0.9, 0.02], [1, 0, 1, 0]], np.float32))
    freqs, _ = b.trj_rotary_freqs(dh, 1e4)
    freqs = freqs.to(DEV)
    pool, scale = ([torch.full((kv_heads, n_blocks) + s, v, dtype=t, device=DEV) for _ in "kv"]
                   for s, t, v in (((32 * dh,), torch.uint8, 0x38), ((), torch.float32, 1.0)))
    table, held, count, prefix, free = i32(np.full((B, width), -1)), ints(B), i32([n_blocks]), i32([0] * B), i32(np.arange(n_blocks))
    held.zero_()
    held2, count2, new_len, slot, token = ints(B), ints(1), ints(B), ints(T), ints(T)
    q, k, out = (torch.zeros(T, h, dh, dtype=torch.bfloat16, device=DEV) for h in (heads, kv_heads, heads))
    v, prob, status = qkv[:, heads + kv_heads:].contiguous(), torch.zeros(T, device=DEV), [ints(B) for _ in range(4)]
    state = [*pool, *scale, table, held, count, prefix, free]
    results = [slot, q, k, out, token, prob, new_len, *status, *state]

    def a_round(ws, sws):
        b.kv_block_tables(table, held, prefix, node_off, T, free, count, held2, count2, slot, status[0])
        b.rotary_rows(qkv[:, :heads], qkv[:, heads:heads + kv_heads], None, node_off, prefix, freqs, 1.0, b.ROTARY_PAIRS, q, k, status[1])
        b.chunk_attention_q8(q, *pool, *scale, k, v, node_off, table, prefix, width * 32, dh ** -0.5, ws, out, status[2])
        b.tree_sample(x, node_off, rules, u, token, prob, sws, status[3])
        b.kv_append_q8(*pool, *scale, k, v, None, None, node_off, table, prefix, new_len, status[0])
        held.copy_(held2)
        count.copy_(count2)
        prefix.copy_(new_len)

    def workspaces():
        return [torch.empty(n, dtype=torch.uint8, device=DEV) for n in (
            b.chunk_attention_q8_workspace_bytes(B, T, heads, kv_heads, dh, width * 32), b.tree_sample_workspace_bytes(B, T, V))]

    spaces = [workspaces() for _ in range(3)]
    a_round(*spaces[0])
    torch.cuda.synchronize()
    graphs = []
    for ws in spaces[1:]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            a_round(*ws)
    for i in range(4):
        start = [t.clone() for t in state]
        a_round(*spaces[0])
        want = [t.clone() for t in results]
        torch.cuda.synchronize()
        for t, s in zip(state, start):
            t.copy_(s)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(results, want))
        assert not any(t.any() for t in status)
    assert int(prefix[2]) == 450
