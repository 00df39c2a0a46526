"""Rounds of a serving program on the paged 8-bit cache, every operator fed by the one before on the
device: pages for the lengths, attention of each layer over the cache and the tree's rows,
logits under penalties and a grammar, acceptance, append of the accepted rows, new lengths.
The oracle runs the same rounds; requests begin, end and run out of pages on the way."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32, to_dev
from oracle import tr_oracle as O
from oracle import tr_serve as S
from paper_2406_17404_amd import binding as b
from paper_2406_17404_amd import inputs as I
from serve_util import bf16, ints, offsets_of
from test_gpu_tree_logits import words_of

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


@pytest.mark.parametrize("dh,n_blocks", [(64, 64), (128, 11)])
def test_rounds(dh, n_blocks):
    rng = np.random.default_rng(dh)
    B, layers, kv_heads, heads, V, width = 4, 2, 2, 4, 700, 6
    sizes = [[9, 1, 33, 0], [9, 1, 33, 20], [0, 1, 33, 20], [0, 40, 33, 20]]  # a request ends, one begins
    host = {w: np.full((layers, kv_heads, n_blocks, 32 * dh), 127, np.uint8) for w in "kv"}
    hscale = {w: np.full((layers, kv_heads, n_blocks), np.nan, np.float32) for w in "kv"}
    pool, scale = ({w: to_dev(x[w]) for w in "kv"} for x in (host, hscale))
    table, held, free, count = np.full((B, width), -1), np.zeros(B, int), np.arange(n_blocks), n_blocks
    d = dict(table=i32(table), free=i32(free), held=[i32(held), ints(B)], count=[i32([count]), ints(1)],
             prefix=i32([0] * B), new_len=ints(B), argmax=None)
    prefix, ctx = np.zeros(B, int), [list(rng.integers(0, 30, 5)) for _ in range(B)]
    for step, size in enumerate(sizes):
        if step == 2:  # the first request has ended
            prefix[0] = 0
            d["prefix"][0] = 0
        off, T = offsets_of(size), int(sum(size))
        parents = [I.tree_random(n, rng) if n else np.zeros(0, int) for n in size]
        parent = np.concatenate(parents)
        q, kr, vr = (bf16(rng.normal(size=(layers, T, h, dh))) for h in (heads, kv_heads, kv_heads))
        x = (rng.normal(size=(T, V)) * 3).astype(np.float32)
        allowed = rng.random((T, V)) < 0.5
        pen = np.tile(np.array([[1.2, 0.3, 0.1]], np.float32), (B, 1))
        tok = rng.integers(0, V, T)
        for s in range(B):  # drafts that are right half of the time
            for i in range(1, size[s]):
                r = slice(off[s], off[s + 1])
                if rng.random() < 0.7:
                    tok[off[s] + i] = S.tree_logits(x[r], tok[r], parents[s], ctx[s], 5, pen[s], None, allowed[r], np.float32)[1][parents[s][i]]
        # ---- the device's round
        dev = dict(off=i32(off), parent=i32(parent), tok=i32(tok), q=q.to(DEV), kr=kr.to(DEV), vr=vr.to(DEV))
        slot, status = ints(T), [ints(B) for _ in range(5)]
        a, z = step % 2, 1 - step % 2
        b.kv_block_tables(d["table"], d["held"][a], d["prefix"], dev["off"], T, d["free"], d["count"][a], d["held"][z],
                          d["count"][z], slot, status[0])
        ws = torch.empty(b.tree_attention_q8_workspace_bytes(B, T, heads, kv_heads, dh, width * 32), dtype=torch.uint8, device=DEV)
        outs = []
        for l in range(layers):
            outs.append(torch.zeros(T, heads, dh, dtype=torch.bfloat16, device=DEV))
            b.tree_attention_q8(dev["q"][l], pool["k"][l], pool["v"][l], scale["k"][l], scale["v"][l], dev["kr"][l], dev["vr"][l],
                                dev["parent"], dev["off"], d["table"], d["prefix"], width * 32, dh ** -0.5, ws, outs[-1], status[1])
        argmax, logits = ints(T), to_dev(x)
        lws = torch.empty(b.tree_logits_workspace_bytes(B, T, V), dtype=torch.uint8, device=DEV)
        b.tree_logits(logits, dev["tok"], dev["parent"], dev["off"], i32(np.concatenate(ctx)),
                      i32(offsets_of([len(c) for c in ctx])), i32([5] * B), to_dev(pen), None, None, None, words_of(allowed),
                      logits, argmax, lws, status[2])
        acc, best, path, bonus = ints(B), ints(B), ints((B, 128)), ints(B)
        b.accept_path(None, dev["tok"], dev["parent"], dev["off"], B, T, V, argmax, acc, best, path, bonus, status[3])
        b.kv_append_q8(pool["k"], pool["v"], scale["k"], scale["v"], dev["kr"], dev["vr"], path, acc, dev["off"], d["table"],
                       d["prefix"], d["new_len"], status[4])
        before = d["prefix"].clone()
        d["prefix"].copy_(d["new_len"])
        torch.cuda.synchronize()
        # ---- the same by the oracle
        assert np.array_equal(before.cpu().numpy(), prefix)
        table, held, free, count, want_slot, refused = S.block_tables(table, held, prefix, off, T, free, count, n_blocks)
        assert np.array_equal(d["table"].cpu().numpy(), table) and np.array_equal(slot.cpu().numpy(), want_slot)
        assert np.array_equal(status[0].cpu().numpy(), refused) and int(d["count"][z]) == count
        want_path, want_acc = np.full((B, 128), -1), np.full(B, -1)
        for s in range(B):
            r = slice(off[s], off[s + 1])
            if size[s] == 0:
                continue
            pages = table[s, :-(-prefix[s] // 32)]
            for l in range(layers):
                kv = [S.page_values(host[w][l], hscale[w][l], w)[:, pages].reshape(kv_heads, -1, dh)[:, :prefix[s]] for w in "kv"]
                want, mean = S.attention(q[l, r].float().numpy(), *kv, kr[l, r].float().numpy(), vr[l, r].float().numpy(),
                                         parents[s], dh ** -0.5)
                tol = HALF * (np.abs(want) + mean) * (1 + HALF) + 2.0 ** -12 * mean
                assert (np.abs(outs[l][r].float().cpu().numpy() - want) <= tol).all()
            y, picks = S.tree_logits(x[r], tok[r], parents[s], ctx[s], 5, pen[s], None, allowed[r], np.float32)
            assert np.array_equal(logits[r].cpu().numpy(), y) and np.array_equal(argmax[r].cpu().numpy(), picks)
            n_acc, _, p, bonus_tok = O.accept_path(picks, tok[r], parents[s])
            want_acc[s], want_path[s, :len(p)] = n_acc, p
            ctx[s] += [int(tok[off[s] + i]) for i in p[1:]] + [int(bonus_tok)]
        assert np.array_equal(acc.cpu().numpy(), want_acc) and np.array_equal(path.cpu().numpy(), want_path)
        new_len, bad = S.append(host["k"], host["v"], hscale["k"], hscale["v"], kr.float().numpy(), vr.float().numpy(),
                                want_path, want_acc, off, table, prefix)
        for w in "kv":
            assert np.array_equal(pool[w].cpu().numpy(), host[w])
            assert np.array_equal(scale[w].cpu().numpy(), hscale[w], equal_nan=True)
        assert np.array_equal(d["new_len"].cpu().numpy(), new_len) and np.array_equal(status[4].cpu().numpy(), bad)
        prefix = new_len
    assert max(prefix) > 4


def test_a_round_captured_into_a_graph():
    """Replayed from a state that it has changed, with other lengths, and between eager rounds: every replay is the
    eager round from the same state."""
    rng = np.random.default_rng(21)
    B, layers, kv_heads, heads, dh, V, width, n_blocks = 3, 2, 2, 8, 64, 1500, 8, 40
    size = [7, 1, 40]
    off, T = offsets_of(size), sum(size)
    parent = i32(np.concatenate([I.tree_random(n, rng) for n in size]))
    q, kr, vr = (bf16(rng.normal(size=(layers, T, h, dh))).to(DEV) for h in (heads, kv_heads, kv_heads))
    x, tok, node_off = to_dev((rng.normal(size=(T, V)) * 3).astype(np.float32)), i32(rng.integers(0, V, T)), i32(off)
    ctx, ctx_off, gen = i32(rng.integers(0, V, 60)), i32([0, 10, 40, 60]), i32([4, 4, 4])
    pen = to_dev(np.tile(np.array([[1.3, 0.2, 0.1]], np.float32), (B, 1)))
    pool, scale = ([torch.full((layers, kv_heads, n_blocks) + s, v, dtype=t, device=DEV) for _ in "kv"]
                   for s, t, v in (((32 * dh,), torch.uint8, 0x38), ((), torch.float32, 1.0)))
    table, held, count, prefix = i32(np.full((B, width), -1)), ints(B), i32([n_blocks]), i32([0] * B)
    free = i32(np.arange(n_blocks))
    held.zero_()
    held2, count2, new_len, slot, argmax = ints(B), ints(1), ints(B), ints(T), ints(T)
    out, y = torch.zeros_like(q), torch.zeros_like(x)
    acc, best, path, bonus, status = ints(B), ints(B), ints((B, 128)), ints(B), [ints(B) for _ in range(4)]
    ws = torch.empty(b.tree_attention_q8_workspace_bytes(B, T, heads, kv_heads, dh, width * 32), dtype=torch.uint8, device=DEV)
    lws = torch.empty(b.tree_logits_workspace_bytes(B, T, V), dtype=torch.uint8, device=DEV)
    state = [*pool, *scale, table, held, count, prefix, free]
    results = [slot, out, y, argmax, acc, path, new_len, *status, *state]

    def a_round():
        b.kv_block_tables(table, held, prefix, node_off, T, free, count, held2, count2, slot, status[0])
        for l in range(layers):
            b.tree_attention_q8(q[l], pool[0][l], pool[1][l], scale[0][l], scale[1][l], kr[l], vr[l], parent, node_off, table, prefix,
                                width * 32, dh ** -0.5, ws, out[l], status[1])
        b.tree_logits(x, tok, parent, node_off, ctx, ctx_off, gen, pen, None, None, None, None, y, argmax, lws, status[2])
        b.accept_path(None, tok, parent, node_off, B, T, V, argmax, acc, best, path, bonus, status[3])
        b.kv_append_q8(*pool, *scale, kr, vr, path, acc, node_off, table, prefix, new_len, status[3])
        held.copy_(held2)
        count.copy_(count2)
        prefix.copy_(new_len)

    a_round()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a_round()
    for _ in range(4):
        start = [t.clone() for t in state]
        a_round()
        want = [t.clone() for t in results]
        torch.cuda.synchronize()
        for t, s in zip(state, start):
            t.copy_(s)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(results, want))
        assert not status[0].any() and not status[3].any()
    assert (prefix >= 5).all()
