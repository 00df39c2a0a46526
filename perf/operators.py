"""The operators of serving from a paged 8-bit KV cache, and what their speed is measured on:
block tables and row slots from request lengths, the append that quantises rows into the cache,
tree attention over it, and penalties, biases and grammar masks on the logits of a tree.

``run`` computes an operator in plain torch (32 bits, rounded once at the end) or, with ``own``,
through ``paper_2406_17404_amd.binding``, on the same buffers.  Layouts are those of
``include/trjacobi.h``: pages of 32 slots, e4m3 codes in tiles, one power-of-two scale for the K
and one for the V of a page and head.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
PAGE = 32
K_MIN = -100  # the smallest scale's exponent


# ------------------------------------------------------------------------------ the cases
def listed():
    return [
        # one token of one short chat, grouped-query heads: plain decoding, latency alone
        _attention("attn_500x1", prefix=500, nodes=1, kv_heads=8),
        # the paper's template of 69 rows on grouped-query heads (8B class), a ragged length
        _attention("attn_gqa_3001x69", prefix=3001, nodes=69, kv_heads=8),
        # 64 drafts on a long document, as many K/V heads as query heads
        _attention("attn_32768x64", prefix=32768, nodes=64),
        # sixteen requests of different lengths verified together
        _attention("attn_packed16", prefix=4096, nodes=64, seqs=16),
        # the token of one request that decodes plainly, one layer
        _append("append_1", prefix=500, rows=1, kv_heads=8),
        # a prompt chunk of 4096 tokens behind a short system prompt, one layer of the 7B shape
        _append("append_prompt_4096", prefix=77, rows=4096),
        # the accepted paths of sixteen requests, all layers of the grouped-query shape at once
        _append("append_commit16", prefix=1024, rows=64, seqs=16, kv_heads=8, layers=32, accepted=5),
        # the next round of sixteen requests
        _tables("tables_16", prefix=4096, seqs=16, rows=64),
        # a full server: requests that go on, that ended, and that begin
        _tables("tables_1024", prefix=4096, seqs=1024, rows=5),
        # one request's plain decoding step with penalties
        _logits("logits_1x32000", ctx=500, nodes=1, vocab=32000),
        # a 64-node tree under a grammar, penalties and biases, large vocabulary
        _logits("logits_69x128256", ctx=3001, nodes=69, vocab=128256, masked=True, biases=100),
        # sixteen packed trees; only the predictions are wanted
        _logits("logits_packed16", ctx=4096, nodes=64, seqs=16, vocab=32000, masked=True, biases=20, keep=False),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["attention"] * 5 + ["append"] * 3 + ["tables"] * 2 + ["logits"] * 3)
    most = {c["kind"]: max(_cost(x) for x in listed() if x["kind"] == c["kind"]) for c in listed()}[kind]
    while True:
        if kind == "attention":
            seqs = rng.choice([1, 1, log(2, 32)])
            heads, kv_heads, dh = rng.choice([(32, 32, 128), (32, 8, 128), (32, 8, 128), (16, 16, 64), (16, 2, 64), (12, 4, 128)])
            c = _attention(None, prefix=log(1, 32768) if seqs == 1 else log(16, 4096),
                           nodes=rng.choice([1, log(1, 128), rng.randint(1, 128)]), seqs=seqs, heads=heads,
                           kv_heads=kv_heads, head_dim=dh)
        elif kind == "append":
            kv_heads, dh = rng.choice([(32, 128), (8, 128), (8, 128), (16, 64), (2, 64)])
            if rng.random() < 0.5:
                c = _append(None, prefix=rng.choice([0, log(1, 4096)]), rows=log(1, 4096), seqs=log(1, 8),
                            kv_heads=kv_heads, head_dim=dh)
            else:
                rows = rng.randint(2, 128)
                c = _append(None, prefix=log(1, 4096), rows=rows, seqs=log(1, 64), kv_heads=kv_heads, head_dim=dh,
                            layers=rng.choice([1, 4, 32]), accepted=rng.randint(0, min(15, rows - 1)))
        elif kind == "tables":
            c = _tables(None, prefix=log(32, 32768), seqs=log(1, 2048), rows=log(1, 128))
        else:
            c = _logits(None, ctx=log(1, 8192), nodes=rng.choice([1, log(1, 128), rng.randint(1, 128)]),
                        seqs=rng.choice([1, 1, log(2, 32)]), vocab=rng.choice([2048, 32000, 32256, 128256, log(1000, 130000)]),
                        masked=rng.random() < 0.5, biases=rng.choice([0, 0, log(1, 300)]), keep=rng.random() < 0.7)
        c["mix"] = rng.randint(0, 10 ** 6)
        if _cost(c) <= most:
            break
    del c["name"]
    return c


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 1.3e15)


def _attention(name, prefix, nodes, seqs=1, heads=32, kv_heads=None, head_dim=128):
    return {"name": name, "kind": "attention", "prefix": prefix, "nodes": nodes, "seqs": seqs, "heads": heads,
            "kv_heads": kv_heads or heads, "head_dim": head_dim, "mix": 1}


def _append(name, prefix, rows, seqs=1, kv_heads=32, head_dim=128, layers=1, accepted=-1):
    """accepted >= 0: of the trees of `rows` nodes a path with so many drafts (plus or minus one) is kept."""
    return {"name": name, "kind": "append", "prefix": prefix, "rows": rows, "seqs": seqs, "kv_heads": kv_heads,
            "head_dim": head_dim, "layers": layers, "accepted": accepted, "mix": 1}


def _tables(name, prefix, seqs, rows):
    return {"name": name, "kind": "tables", "prefix": prefix, "seqs": seqs, "rows": rows, "mix": 1}


def _logits(name, ctx, nodes, vocab, seqs=1, masked=False, biases=0, keep=True):
    return {"name": name, "kind": "logits", "ctx": ctx, "nodes": nodes, "seqs": seqs, "vocab": vocab,
            "masked": masked, "biases": biases, "keep": keep, "mix": 1}


# ------------------------------------------------------------------------------ inputs
def _lengths(case, key="prefix"):
    """One sequence: as stated; several: ragged between an eighth of it and all."""
    if case["seqs"] == 1:
        return [case[key]]
    rng = random.Random(case["mix"])
    return [rng.randint(case[key] // 8, case[key]) for _ in range(case["seqs"])]


def _counts(case):
    """Rows per sequence of an append, and how many of them are kept."""
    rng = random.Random(case["mix"] + 1)
    if case["accepted"] < 0:
        rows = [case["rows"] if case["seqs"] == 1 else rng.randint(1, case["rows"]) for _ in range(case["seqs"])]
        return rows, rows
    kept = [min(case["rows"], max(1, case["accepted"] + 1 + rng.randint(-1, 1))) for _ in range(case["seqs"])]
    return [case["rows"]] * case["seqs"], kept


def _requests(case):
    """Per request: tokens it had room for, committed tokens now, rows now.  A tenth ended, a tenth begins."""
    rng = random.Random(case["mix"] + 2)
    had, prefix, rows = [], [], []
    for l in _lengths(case):
        what = rng.random() if case["seqs"] > 1 else 0.5
        if what < 0.1:
            h, p, n = l + case["rows"], 0, 0
        elif what < 0.2:
            h, p, n = 0, 0, rng.randint(1, 4 * case["rows"])
        else:
            kept = rng.randint(1, case["rows"])
            h, p, n = l + case["rows"], l + kept, case["rows"]
        had.append(h), prefix.append(p), rows.append(n)
    return had, prefix, rows


def _gen(seed, key):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 64 + key) % (1 << 62))
    return g


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _offsets(sizes):
    return _ints(np.concatenate([[0], np.cumsum(sizes)]))


def _trees(nodes, seqs, rng):
    """Every node's parent any earlier node."""
    p = (rng.random((seqs, nodes)) * np.arange(nodes)).astype(np.int64)
    p[:, 0] = -1
    return p


def _pages(lens, rng, spare=3):
    """A table of shuffled pages with room for `lens` tokens each, and the number of pages."""
    need = [-(-l // PAGE) for l in lens]
    width, total = max(max(need), 1) + 1, sum(need) + spare
    ids, table, at = rng.permutation(total), np.full((len(lens), width), -1), 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at:at + n]
        at += n
    return _ints(table), total


def _cache(gen, layers, heads, pages, dh):
    """Codes of normal values and the scales that pages of them have; in a tenth half of that, which new rows raise."""
    n = layers * heads * pages
    x = torch.empty(n, PAGE * dh, dtype=torch.uint8, device=DEV)
    for at in range(0, n, 4096):
        v = torch.randn(min(4096, n - at), PAGE * dh, generator=gen, device=DEV) * 64
        x[at:at + 4096] = v.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    k = -6 - (torch.rand(layers, heads, pages, generator=gen, device=DEV) < 0.1).int()
    return x.view(layers, heads, pages, PAGE * dh), torch.ldexp(torch.ones(k.shape, device=DEV), k)


def prepare(case, seed):
    rng = np.random.default_rng([int(seed), 11])
    s = {"case": case}
    if case["kind"] == "attention":
        B, n, dh, lens = case["seqs"], case["nodes"], case["head_dim"], _lengths(case)
        s["table"], pages = _pages(lens, rng)
        s["k"], s["ks"] = (t[0] for t in _cache(_gen(seed, 1), 1, case["kv_heads"], pages, dh))
        s["v"], s["vs"] = (t[0] for t in _cache(_gen(seed, 2), 1, case["kv_heads"], pages, dh))
        s["q"] = torch.randn(B * n, case["heads"], dh, generator=_gen(seed, 3), device=DEV).bfloat16()
        rows = torch.randn(2, B * n, case["kv_heads"], dh, generator=_gen(seed, 4), device=DEV).bfloat16()
        s.update(k_rows=rows[0], v_rows=rows[1], parent=_ints(_trees(n, B, rng).ravel()), off=_offsets([n] * B),
                 prefix=_ints(lens), longest=max(lens), out=torch.zeros_like(s["q"]),
                 status=torch.zeros(B, dtype=torch.int32, device=DEV))
    elif case["kind"] == "append":
        B, dh, H, lens = case["seqs"], case["head_dim"], case["kv_heads"], _lengths(case)
        rows, kept = _counts(case)
        s["table"], pages = _pages([l + m for l, m in zip(lens, kept)], rng)
        s["k"], s["ks"] = _cache(_gen(seed, 1), case["layers"], H, pages, dh)
        s["v"], s["vs"] = _cache(_gen(seed, 2), case["layers"], H, pages, dh)
        x = torch.randn(2, case["layers"], sum(rows), H, dh, generator=_gen(seed, 3), device=DEV).bfloat16()
        s.update(k_rows=x[0], v_rows=x[1], off=_offsets(rows), prefix=_ints(lens), most=max(kept), path=None, acc=None,
                 new_len=torch.zeros(B, dtype=torch.int32, device=DEV),
                 status=torch.zeros(B, dtype=torch.int32, device=DEV))
        if case["accepted"] >= 0:
            path = np.full((B, 128), -1)
            for b, m in enumerate(kept):
                path[b, 0] = 0
                path[b, 1:m] = 1 + np.sort(rng.permutation(case["rows"] - 1)[:m - 1])
            s.update(path=_ints(path), acc=_ints([m - 1 for m in kept]))
    elif case["kind"] == "tables":
        had, prefix, rows = _requests(case)
        need = [-(-(p + n) // PAGE) for p, n in zip(prefix, rows)]
        held = [-(-h // PAGE) for h in had]
        spare = sum(max(0, a - b) for a, b in zip(need, held)) + 8
        ids = rng.permutation(sum(held) + spare)
        width = max(max(held), max(need)) + 1
        table, at = np.full((case["seqs"], width), -1), 0
        for b, n in enumerate(held):
            table[b, :n] = ids[at:at + n]
            at += n
        free = np.full(len(ids), -1)
        free[:spare] = ids[at:]
        s.update(table=_ints(table), held=_ints(held), prefix=_ints(prefix), off=_offsets(rows), T=sum(rows),
                 free=_ints(free), count=_ints([spare]), held_out=_ints(held), count_out=_ints([0]),
                 slot=_ints([0] * max(1, sum(rows))), status=_ints([0] * case["seqs"]))
    else:
        B, n, V, lens = case["seqs"], case["nodes"], case["vocab"], _lengths(case, "ctx")
        g = _gen(seed, 1)
        s["x"] = torch.randn(B * n, V, generator=g, device=DEV) * 3
        # frequent tokens come again and again
        zipf = lambda k: (torch.rand(k, generator=g, device=DEV) ** 3 * V).int().clamp(max=V - 1)  # noqa: E731
        s.update(tok=zipf(B * n), parent=_ints(_trees(n, B, rng).ravel()), off=_offsets([n] * B), ctx=zipf(sum(lens)),
                 ctx_off=_offsets(lens), gen=_ints([l // 2 for l in lens]), status=_ints([0] * B))
        s["pen"] = torch.rand(B, 3, generator=g, device=DEV) * 0.5 + torch.tensor([1.0, 0.0, 0.0], device=DEV)
        s["allowed"] = s["bias_tok"] = s["bias_val"] = s["bias_off"] = None
        if case["masked"]:
            words = -(-V // 32)
            s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (B * n, words), generator=g, device=DEV).int()
        if case["biases"]:
            k = min(case["biases"], V)
            s["bias_tok"] = _ints(np.concatenate([rng.choice(V, k, replace=False) for _ in range(B)]))
            s["bias_val"] = torch.randn(B * k, generator=g, device=DEV) * 2
            s["bias_off"] = _offsets([k] * B)
        s["out"] = torch.zeros_like(s["x"]) if case["keep"] else None
        s["argmax"] = torch.zeros(B * n, dtype=torch.int32, device=DEV)
    return s


# ------------------------------------------------------------------------------ the calls
def run(s):
    return _own(s) if own else _PLAIN[s["case"]["kind"]](s)


def _own(s):
    from paper_2406_17404_amd import binding as B
    c = s["case"]
    if c["kind"] == "attention":
        T = c["seqs"] * c["nodes"]
        if "ws" not in s:
            s["ws"] = torch.empty(B.tree_attention_q8_workspace_bytes(c["seqs"], T, c["heads"], c["kv_heads"],
                                                                      c["head_dim"], s["longest"]),
                                  dtype=torch.uint8, device=DEV)
        B.tree_attention_q8(s["q"], s["k"], s["v"], s["ks"], s["vs"], s["k_rows"], s["v_rows"], s["parent"], s["off"],
                            s["table"], s["prefix"], s["longest"], 1.0 / math.sqrt(c["head_dim"]), s["ws"], s["out"],
                            s["status"])
        return s["out"]
    if c["kind"] == "append":
        B.kv_append_q8(s["k"], s["v"], s["ks"], s["vs"], s["k_rows"], s["v_rows"], s["path"], s["acc"], s["off"],
                       s["table"], s["prefix"], s["new_len"], s["status"])
        return _cache_out(s)
    if c["kind"] == "tables":
        B.kv_block_tables(s["table"], s["held"], s["prefix"], s["off"], s["T"], s["free"], s["count"], s["held_out"],
                          s["count_out"], s["slot"], s["status"])
        return {"table": s["table"], "held": s["held_out"], "free": s["free"], "count": s["count_out"],
                "slot": s["slot"], "status": s["status"]}
    if "ws" not in s:
        s["ws"] = torch.empty(B.tree_logits_workspace_bytes(c["seqs"], c["seqs"] * c["nodes"], c["vocab"]),
                              dtype=torch.uint8, device=DEV)
    B.tree_logits(s["x"], s["tok"], s["parent"], s["off"], s["ctx"], s["ctx_off"], s["gen"], s["pen"], s["bias_tok"],
                  s["bias_val"], s["bias_off"], s["allowed"], s["out"], s["argmax"], s["ws"], s["status"])
    return {"logits": s["out"], "argmax": s["argmax"]} if c["keep"] else {"argmax": s["argmax"]}


def _cache_out(s):
    f8 = torch.float8_e4m3fn
    return {"k": s["k"].view(f8), "v": s["v"].view(f8), "k_scale": s["ks"], "v_scale": s["vs"], "len": s["new_len"]}


# ------------------------------------------------------------------------------ plain forms
def _untile_k(x, dh):
    """[.., 32 * dh] as laid out in a page -> [.., 32, dh]."""
    lead = x.shape[:-1]
    return x.view(*lead, dh // 32, 2, 32, 16).movedim(-2, -4).reshape(*lead, 32, dh)


def _tile_k(x, dh):
    lead = x.shape[:-2]
    return x.reshape(*lead, 32, dh // 32, 2, 16).movedim(-4, -2).reshape(*lead, 32 * dh)


def _untile_v(x, dh):
    lead, n = x.shape[:-1], x.dim() - 1  # a page: [dh/32][slot/4%2][32 columns][slot/16][slot/8%2][slot%4]
    x = x.view(*lead, dh // 32, 2, 32, 2, 2, 4)
    return x.permute(*range(n), n + 3, n + 4, n + 1, n + 5, n, n + 2).reshape(*lead, 32, dh)


def _tile_v(x, dh):
    lead, n = x.shape[:-2], x.dim() - 2
    x = x.reshape(*lead, 2, 2, 2, 4, dh // 32, 32)
    return x.permute(*range(n), n + 4, n + 2, n + 5, n, n + 1, n + 3).reshape(*lead, 32 * dh)


def _values(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _paths(parent, B, n):
    """[B, n, n]: whether node j is on the path from the root to node i, itself included."""
    p = parent.view(B, n).long()
    step = (p[:, :, None] == torch.arange(n, device=DEV)).double() + torch.eye(n, device=DEV, dtype=torch.float64)
    return torch.linalg.matrix_power(step, max(1, n - 1)) > 0


def _plain_attention(s):
    c = s["case"]
    B, n, H, Hk, dh = c["seqs"], c["nodes"], c["heads"], c["kv_heads"], c["head_dim"]
    page = s["table"].long()[:, :-1].clamp(min=0)  # [B, pages of the longest]
    k = _untile_k(_values(s["k"])[:, page] * s["ks"][:, page][..., None], dh).reshape(Hk, B, -1, dh)
    v = _untile_v(_values(s["v"])[:, page] * s["vs"][:, page][..., None], dh).reshape(Hk, B, -1, dh)
    there = torch.arange(k.shape[2], device=DEV) < s["prefix"][:, None]  # [B, slots]
    k = torch.cat([k, s["k_rows"].float().view(B, n, Hk, dh).permute(2, 0, 1, 3)], 2)
    v = torch.cat([v * there[:, :, None], s["v_rows"].float().view(B, n, Hk, dh).permute(2, 0, 1, 3)], 2)
    sees = torch.cat([there[:, None].expand(B, n, there.shape[1]), _paths(s["parent"], B, n)], 2)  # [B, n, keys]
    q = s["q"].float().view(B, n, Hk, H // Hk, dh).permute(2, 0, 3, 1, 4).reshape(Hk, B, -1, dh)
    score = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(dh))
    score = score.view(Hk, B, H // Hk, n, -1).masked_fill(~sees[None, :, None], -math.inf)
    p = (score - score.amax(-1, keepdim=True)).exp()
    p = (p / p.sum(-1, keepdim=True)).view(Hk, B, (H // Hk) * n, -1)
    o = torch.matmul(p, v).view(Hk, B, H // Hk, n, dh).permute(1, 3, 0, 2, 4)
    return o.reshape(B * n, H, dh).bfloat16()


def _plain_append(s):
    c = s["case"]
    dh, prefix = c["head_dim"], s["prefix"].long()
    off = s["off"].long()
    count = off[1:] - off[:-1] if s["path"] is None else s["acc"].long() + 1
    touched = (prefix // PAGE)[:, None] + torch.arange(s["most"] // PAGE + 2, device=DEV)
    seq, nth = ((touched * PAGE < (prefix + count)[:, None]) & (count > 0)[:, None]).nonzero(as_tuple=True)
    at = touched[seq, nth]
    pos = at[:, None] * PAGE + torch.arange(PAGE, device=DEV)  # [pages, 32]
    j = pos - prefix[seq][:, None]
    new, old = (j >= 0) & (j < count[seq][:, None]), j < 0
    j = j.clamp(min=0).minimum(count[seq][:, None] - 1)
    row = off[seq][:, None] + (j if s["path"] is None else s["path"].long()[seq[:, None], j])
    page = s["table"].long()[seq, at]
    for_all = lambda m: m[:, :, None]  # noqa: E731

    def write(pool, scales, rows, untile, tile):
        codes = untile(pool[:, :, page], dh)  # [layers, heads, pages, 32, dh]
        had = torch.where(old.any(1), scales[:, :, page], torch.zeros((), device=DEV))
        x = rows.float()[:, row].permute(0, 3, 1, 2, 4) * for_all(new)
        m, e = torch.frexp(x.abs().amax((3, 4)))
        k = torch.where(m > 0.875, e - 8, e - 9)  # the least with max|x| <= 448 * 2^k
        k = torch.where(m == 0, torch.full_like(k, K_MIN), k).clamp(min=K_MIN)
        scale = torch.maximum(torch.ldexp(torch.ones_like(had), k), had)
        kept = (_values(codes) * (had / scale)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        put = (x / scale[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        codes = torch.where(for_all(new), put, torch.where(for_all(old), kept, codes))
        pool[:, :, page] = tile(codes, dh)
        scales[:, :, page] = scale

    write(s["k"], s["ks"], s["k_rows"], _untile_k, _tile_k)
    write(s["v"], s["vs"], s["v_rows"], _untile_v, _tile_v)
    s["new_len"].copy_(prefix + count)
    return _cache_out(s)


def _plain_tables(s):
    held, prefix, off = s["held"].long(), s["prefix"].long(), s["off"].long()
    n_seq, width = s["table"].shape
    want = (prefix + off[1:] - off[:-1] + PAGE - 1) // PAGE
    need, over = (want - held).clamp(min=0), (held - want).clamp(min=0)
    j = torch.arange(width, device=DEV)
    # released pages go on top of the stack, sequence by sequence
    gives = (j >= want[:, None]) & (j < held[:, None])
    place = s["count"].long() + (over.cumsum(0) - over)[:, None] + j - want[:, None]
    sink = s["free"].numel()
    free = torch.cat([s["free"], s["free"].new_zeros(1)]).scatter(0, torch.where(gives, place, sink).view(-1), s["table"].view(-1))
    have = s["count"].long() + over.sum()
    fits = need.cumsum(0) <= have
    take = torch.where(fits, need, torch.zeros_like(need))
    # and the pages that are needed come from its top
    from_top = (need.cumsum(0) - need)[:, None] + j - held[:, None]
    gets = (j >= held[:, None]) & (j < (held + take)[:, None])
    table = torch.where(gets, free[torch.where(gets, have - 1 - from_top, sink)], s["table"])
    held_out = torch.where(fits, want, held)
    t = torch.arange(s["T"], device=DEV)
    seq = torch.searchsorted(off, t, right=True) - 1
    pos = prefix[seq] + t - off[seq]
    slot = table[seq, (pos // PAGE).clamp(max=width - 1)].long() * PAGE + pos % PAGE
    return {"table": table, "held": held_out.int(), "free": free[:-1], "count": (have - take.sum()).int().view(1),
            "slot": torch.where(fits[seq], slot, torch.full_like(slot, -1)).int(), "status": (~fits).int()}


def _plain_logits(s):
    c = s["case"]
    B, n, V = c["seqs"], c["nodes"], c["vocab"]
    x, ctx_off = s["x"].view(B, n, V), s["ctx_off"].long()
    at = torch.arange(s["ctx"].numel(), device=DEV)
    seq = torch.searchsorted(ctx_off, at, right=True) - 1
    one = torch.ones((), device=DEV)
    flat = seq * V + s["ctx"]
    made = (at - ctx_off[seq] >= s["gen"][seq]).float()
    seen = torch.zeros(B * V, device=DEV).index_put((flat,), one.expand(flat.shape), accumulate=True)
    count = torch.zeros(B * V, device=DEV).index_put((flat,), made, accumulate=True)
    drafts = _paths(s["parent"], B, n).float()
    drafts[:, :, 0] = 0  # the root is the context's last token
    here = s["tok"].long().view(B, 1, n).expand(B, n, n)
    above = torch.zeros(B, n, V, device=DEV).scatter_add(2, here, drafts)
    seen = (seen.view(B, 1, V) + above) > 0
    count = count.view(B, 1, V) + above
    r, f, p = (s["pen"][:, k, None, None] for k in range(3))
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - f * count
    x = x - p * (count > 0)
    if s["bias_tok"] is not None:
        k = s["bias_tok"].numel() // B
        bias = torch.zeros(B, V, device=DEV).scatter(1, s["bias_tok"].long().view(B, k), s["bias_val"].view(B, k))
        x = x + bias[:, None]
    x = x.reshape(B * n, V)
    v = torch.arange(V, device=DEV)
    if s["allowed"] is not None:
        x = torch.where((s["allowed"][:, v // 32] >> (v % 32)) & 1 == 1, x, torch.full((), -math.inf, device=DEV))
    best = torch.where(x == x.amax(1, keepdim=True), v, V).amin(1)
    return {"logits": x, "argmax": best.int()} if c["keep"] else {"argmax": best.int()}


_PLAIN = {"attention": _plain_attention, "append": _plain_append, "tables": _plain_tables, "logits": _plain_logits}


# ------------------------------------------------------------------------------ the work
def work(case):
    kind = case["kind"]
    if kind == "attention":
        n, H, Hk, dh, lens = case["nodes"], case["heads"], case["kv_heads"], case["head_dim"], _lengths(case)
        rows = n * len(lens)
        pages = sum(-(-l // PAGE) for l in lens)
        return {"bytes": sum(lens) * 2 * Hk * dh + pages * (8 * Hk + 4) + rows * (4 * Hk * dh + 4 * H * dh + 4),
                "flops": sum(4 * n * (l + n) * H * dh for l in lens)}
    if kind == "append":
        lens, (_, kept) = _lengths(case), _counts(case)
        width = case["layers"] * case["kv_heads"] * case["head_dim"]
        values = sum(kept) * width * 2
        pages = sum((l + m - 1) // PAGE - l // PAGE + 1 for l, m in zip(lens, kept))
        return {"bytes": 3 * values + 8 * pages * case["layers"] * case["kv_heads"], "flops": 2 * values}
    if kind == "tables":
        had, prefix, rows = _requests(case)
        moved = sum(abs(-(-h // PAGE) + (-(p + n) // PAGE)) for h, p, n in zip(had, prefix, rows))
        return {"bytes": 20 * case["seqs"] + 8 * moved + 4 * sum(rows) + 4 * sum(rows) // PAGE, "flops": 0}
    rows, V = case["nodes"] * case["seqs"], case["vocab"]
    each = 4 * V * (2 if case["keep"] else 1) + (-(-V // 32) * 4 if case["masked"] else 0) + 12
    return {"bytes": rows * each + 4 * sum(_lengths(case, "ctx")) + 8 * case["biases"] * case["seqs"],
            "flops": 6 * rows * V}


# ------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(case, s)
    if case["kind"] == "append":
        return _exact_append(case, s)
    return None if case["kind"] == "tables" else _exact_logits(case, s)


def _code_values():
    """The 256 values of e4m3: sign, four bits of exponent, three of mantissa; 0x7f and 0xff are no numbers."""
    b = torch.arange(256, device=DEV)
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * torch.exp2(e.double() - 7))
    v[(b & 127) == 127] = math.nan
    return torch.where(b >= 128, -v, v)


def _places(dh):
    """Where a page keeps (slot r, column c), for K and for V."""
    r, c = torch.arange(32, device=DEV)[:, None], torch.arange(dh, device=DEV)
    k = ((c // 32 * 2 + c % 32 // 16) * 32 + r) * 16 + c % 16
    v = ((c // 32 * 2 + r // 4 % 2) * 32 + c % 32) * 16 + r // 16 * 8 + r // 8 % 2 * 4 + r % 4
    return k, v


def _exact_attention(case, s):
    dh, Hk, n = case["head_dim"], case["kv_heads"], case["nodes"]
    group, values, places = case["heads"] // Hk, _code_values(), _places(dh)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    parent = s["parent"].cpu().numpy().reshape(-1, n)
    for b, L in enumerate(_lengths(case)):
        on_path = np.eye(n, dtype=bool)
        for i in range(1, n):
            on_path[i] |= on_path[parent[b, i]]
        seen = torch.from_numpy(on_path).to(DEV)
        rows, pages = slice(b * n, (b + 1) * n), s["table"][b, :-(-L // PAGE)].long()
        for h in range(Hk):
            kv = []
            for pool, scale, own_rows, place in ((s["k"], s["ks"], s["k_rows"], places[0]), (s["v"], s["vs"], s["v_rows"], places[1])):
                x = values[pool[h, pages].long()[:, place.reshape(-1)]].view(-1, 32, dh) * scale[h, pages].double()[:, None, None]
                kv.append(torch.cat([x.reshape(-1, dh)[:L], own_rows[rows, h].double()]))
            for g in range(h * group, (h + 1) * group):
                score = s["q"][rows, g].double() @ kv[0].t().contiguous() / math.sqrt(dh)
                score[:, L:][~seen] = -math.inf
                out[rows, g] = torch.softmax(score, 1) @ kv[1]
    return out


def _round_e4m3(x):
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -20))).clamp(min=-6) - 3)
    return torch.round(x / step) * step


def _exact_append(case, s):
    dh, values, off = case["head_dim"], _code_values(), s["off"].tolist()
    out = {}
    for name, place in zip("kv", _places(dh)):
        x, scale = values[s[name].long()], s[name + "s"].double()
        flat = place.reshape(-1)
        rows = s[name + "_rows"].double()
        for b, (L, m) in enumerate(zip(_lengths(case), _counts(case)[1])):
            picked = list(range(m)) if s["path"] is None else s["path"][b, :m].tolist()
            for page in range(L // PAGE, (L + m - 1) // PAGE + 1):
                a, z = max(L, page * PAGE), min(L + m, (page + 1) * PAGE)
                at = int(s["table"][b, page])
                new = rows[:, [off[b] + i for i in picked[a - L:z - L]]].transpose(1, 2)  # [layers, heads, .., dh]
                top = new.abs().amax((2, 3)) / 448
                k = torch.ceil(torch.log2(top.clamp(min=2.0 ** K_MIN)))
                k = torch.where(torch.exp2(k - 1) >= top, k - 1, k).clamp(min=K_MIN)
                to = torch.exp2(k)
                full = x[:, :, at][..., flat].view(*scale.shape[:2], 32, dh)
                if a > page * PAGE:
                    to = torch.maximum(to, scale[:, :, at])
                    full[:, :, :a - page * PAGE] = _round_e4m3(full[:, :, :a - page * PAGE] * (scale[:, :, at] / to)[..., None, None])
                full[:, :, a - page * PAGE:z - page * PAGE] = _round_e4m3(new / to[..., None, None])
                scale[:, :, at] = to
                back = torch.empty_like(x[:, :, at])
                back[..., flat] = full.reshape(*scale.shape[:2], -1)
                x[:, :, at] = back
        out[name], out[name + "_scale"] = x, scale
    return {**out, "len": None}


def _exact_logits(case, s):
    if not case["keep"]:
        return None
    n, V, off = case["nodes"], case["vocab"], s["ctx_off"].tolist()
    parent, x = s["parent"].view(-1, n).tolist(), s["x"].double()
    pen, tok = s["pen"].double(), s["tok"].view(-1, n).tolist()
    for b in range(case["seqs"]):
        ctx = s["ctx"][off[b]:off[b + 1]].long()
        seen, count = torch.bincount(ctx, minlength=V), torch.bincount(ctx[int(s["gen"][b]):], minlength=V)
        bias = torch.zeros(V, dtype=torch.float64, device=DEV)
        if s["bias_tok"] is not None:
            part = slice(int(s["bias_off"][b]), int(s["bias_off"][b + 1]))
            bias[s["bias_tok"][part].long()] = s["bias_val"][part].double()
        for i in range(n):
            drafts, j = [], i
            while j > 0:
                drafts.append(tok[b][j])
                j = parent[b][j]
            own_count = torch.bincount(torch.tensor(drafts, device=DEV, dtype=torch.long), minlength=V)
            y, made = x[b * n + i], count + own_count
            y = torch.where(seen + own_count > 0, torch.where(y > 0, y / pen[b, 0], y * pen[b, 0]), y)
            x[b * n + i] = y - pen[b, 1] * made - pen[b, 2] * (made > 0) + bias
    if s["allowed"] is not None:
        bits = torch.stack([(s["allowed"] >> k) & 1 for k in range(32)], 2).flatten(1)[:, :V]
        x[bits == 0] = -math.inf
    return {"logits": x, "argmax": None}
