"""Prompts and sampled tokens on the paged 8-bit cache, and what their speed is measured on: rotary
positions of query and key rows, causal attention of a chunk of new rows over the cache, and
sampling with temperature, top-k, top-p and min-p at every row of logits.

``run`` computes an operator in plain torch (32 bits, 64 for angles and long sums, rounded once at
the end) or, with ``own``, through ``paper_2406_17404_amd.binding``, on the same buffers.  Layouts
are those of ``include/trjacobi.h``.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
PAGE = 32
UNIT = 2.0 ** 38  # what a sampling weight of 1 is held as


# ------------------------------------------------------------------------------ the cases
def listed():
    return [
        # the row of one request that decodes plainly, grouped-query heads: latency alone
        _rotary("rotary_1", prefix=500, rows=1, kv_heads=8),
        # 69 nodes of a tree far into a long text, 32 bits
        _rotary("rotary_fp32_69", prefix=100000, rows=69, heads=16, head_dim=64, dtype="f32", tree=True),
        # sixteen packed trees of a small model that rotates neighbours, in half of a head, for a longer context
        _rotary("rotary_trees16_pairs", prefix=4096, rows=64, seqs=16, heads=16, kv_heads=2, head_dim=64, rot_dim=32,
                pairs=True, scaled=True, tree=True),
        # a prompt chunk of the 7B shape
        _rotary("rotary_prompt_4096", prefix=77, rows=4096),
        # the last few tokens of a prompt, behind a cached system prompt
        _chunk("chunk_40_after_500", prefix=500, rows=40, kv_heads=8),
        # a further turn of a chat, ragged
        _chunk("chunk_517_after_3001", prefix=3001, rows=517, kv_heads=8),
        # a whole prompt, nothing cached
        _chunk("chunk_prompt_4096", prefix=0, rows=4096, kv_heads=8),
        # the next chunk of a long document, as many K/V heads as query heads
        _chunk("chunk_2048_after_16384", prefix=16384, rows=2048),
        # requests that decode beside requests whose prompts come in
        _chunk("chunk_mixed16", prefix=4096, rows=512, seqs=16, kv_heads=8),
        # one request's plain decoding step, all rules
        _sample("sample_1x32000", nodes=1, vocab=32000, rules="kpm"),
        # a 69-node tree, large vocabulary, top-k and top-p
        _sample("sample_69x128256", nodes=69, vocab=128256, rules="kp"),
        # sixteen packed trees under a grammar, every request with rules of its own, logits of 16 bits (ties)
        _sample("sample_packed16", nodes=64, seqs=16, vocab=32000, rules="mixed", masked=True, coarse=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotary"] * 3 + ["chunk"] * 5 + ["sample"] * 4)
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    while True:
        heads, kv_heads, dh = rng.choice([(32, 32, 128), (32, 8, 128), (32, 8, 128), (16, 16, 64), (16, 2, 64), (12, 4, 128)])
        if kind == "rotary":
            tree = rng.random() < 0.5
            c = _rotary(None, prefix=rng.choice([0, log(1, 10 ** 6)]), rows=log(1, 128) if tree else log(1, 4096),
                        seqs=rng.choice([1, log(1, 32)]), heads=heads, kv_heads=kv_heads, head_dim=dh,
                        rot_dim=rng.choice([dh, dh, dh // 2, dh // 4, 2 * rng.randint(1, dh // 2)]),
                        pairs=rng.random() < 0.5, scaled=rng.random() < 0.5, tree=tree,
                        dtype=rng.choice(["bf16", "bf16", "f32"]))
        elif kind == "chunk":
            seqs = rng.choice([1, 1, log(2, 32)])
            c = _chunk(None, prefix=rng.choice([0, log(1, 32768), log(1, 32768)]) if seqs == 1 else log(16, 4096),
                       rows=log(1, 4096) if seqs == 1 else log(1, 1024), seqs=seqs, heads=heads, kv_heads=kv_heads, head_dim=dh)
        else:
            c = _sample(None, nodes=rng.choice([1, log(1, 128), rng.randint(1, 128)]), seqs=rng.choice([1, 1, log(2, 32)]),
                        vocab=rng.choice([2048, 32000, 32256, 128256, log(1000, 130000)]),
                        rules=rng.choice(["", "k", "p", "m", "kp", "kpm", "mixed"]), masked=rng.random() < 0.3,
                        coarse=rng.random() < 0.4)
        c["mix"] = rng.randint(0, 10 ** 6)
        if _cost(c) <= most:
            break
    del c["name"]
    return c


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / 1.3e15)


def _rotary(name, prefix, rows, seqs=1, heads=32, kv_heads=None, head_dim=128, rot_dim=None, pairs=False, scaled=False,
            tree=False, dtype="bf16"):
    return {"name": name, "kind": "rotary", "prefix": prefix, "rows": rows, "seqs": seqs, "heads": heads,
            "kv_heads": kv_heads or heads, "head_dim": head_dim, "rot_dim": rot_dim or head_dim, "pairs": pairs,
            "scaled": scaled, "tree": tree, "dtype": dtype, "mix": 1}


def _chunk(name, prefix, rows, seqs=1, heads=32, kv_heads=None, head_dim=128):
    return {"name": name, "kind": "chunk", "prefix": prefix, "rows": rows, "seqs": seqs, "heads": heads,
            "kv_heads": kv_heads or heads, "head_dim": head_dim, "mix": 1}


def _sample(name, nodes, vocab, rules, seqs=1, masked=False, coarse=False):
    """rules: which of top-k (k), top-p (p) and min-p (m) are on; "mixed": another choice for every request."""
    return {"name": name, "kind": "sample", "nodes": nodes, "seqs": seqs, "vocab": vocab, "rules": rules,
            "masked": masked, "coarse": coarse, "mix": 1}


# ------------------------------------------------------------------------------ inputs
def _lengths(case):
    """One sequence: as stated; several: ragged between an eighth of it and all."""
    if case["seqs"] == 1:
        return [case["prefix"]]
    rng = random.Random(case["mix"])
    return [rng.randint(case["prefix"] // 8, case["prefix"]) for _ in range(case["seqs"])]


def _rows(case):
    """Rows of every sequence; of several that attend together half decode a token each."""
    if case["seqs"] == 1 or case["kind"] == "rotary":
        return [case["rows"]] * case["seqs"]
    rng = random.Random(case["mix"] + 1)
    return [1 if s % 2 else max(1, int(round(case["rows"] ** rng.uniform(0.5, 1)))) for s in range(case["seqs"])]


def _gen(seed, key):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 64 + key) % (1 << 62))
    return g


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _offsets(sizes):
    return _ints(np.concatenate([[0], np.cumsum(sizes)]))


def _pages(lens, rng, spare=3):
    """A table of shuffled pages with room for `lens` tokens each, and the number of pages."""
    need = [-(-l // PAGE) for l in lens]
    width, total = max(max(need), 1) + 1, sum(need) + spare
    ids, table, at = rng.permutation(total), np.full((len(lens), width), -1), 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at:at + n]
        at += n
    return _ints(table), total


def _cache(gen, heads, pages, dh):
    """Codes of normal values and the scales that pages of them have."""
    n = heads * pages
    x = torch.empty(n, PAGE * dh, dtype=torch.uint8, device=DEV)
    for at in range(0, n, 4096):
        v = torch.randn(min(4096, n - at), PAGE * dh, generator=gen, device=DEV) * 64
        x[at:at + 4096] = v.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    k = -6 - (torch.rand(heads, pages, generator=gen, device=DEV) < 0.1).int()
    return x.view(heads, pages, PAGE * dh), torch.ldexp(torch.ones(k.shape, device=DEV), k)


def _frequencies(case):
    """theta^(-2j / rot_dim); for a longer context the low ones are divided by 8, those between blended."""
    n = case["rot_dim"] // 2
    f = 10000.0 ** (-np.arange(n) / n)
    if case["scaled"]:
        share = np.clip((2048 * f / (2 * math.pi) - 1) / 3, 0, 1)  # turns within the first 2048 tokens: 1 .. 4
        f = f / 8 * (1 - share) + f * share
    return f


def prepare(case, seed):
    rng = np.random.default_rng([int(seed), 17])
    s = {"case": case}
    if case["kind"] == "rotary":
        rows, H, Hk, dh = _rows(case), case["heads"], case["kv_heads"], case["head_dim"]
        T, kind = sum(rows), torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s["qkv"] = torch.randn(T, (H + 2 * Hk) * dh, generator=_gen(seed, 1), device=DEV).to(kind)
        s["q"] = s["qkv"][:, :H * dh].view(T, H, dh)  # as the common projection leaves them
        s["k"] = s["qkv"][:, H * dh:(H + Hk) * dh].view(T, Hk, dh)
        s["parent"] = None
        if case["tree"]:  # every node's parent any earlier node
            p = [np.concatenate([[-1], (rng.random(n - 1) * np.arange(1, n)).astype(np.int64)]) for n in rows]
            s["parent"] = _ints(np.concatenate(p))
        s.update(off=_offsets(rows), prefix=_ints(_lengths(case)), freqs=torch.from_numpy(_frequencies(case)).to(DEV),
                 magnitude=1.0 + 0.1 * math.log(8) if case["scaled"] else 1.0,
                 q_out=torch.zeros(T, H, dh, dtype=kind, device=DEV), k_out=torch.zeros(T, Hk, dh, dtype=kind, device=DEV),
                 status=_ints([0] * case["seqs"]))
    elif case["kind"] == "chunk":
        rows, H, Hk, dh, lens = _rows(case), case["heads"], case["kv_heads"], case["head_dim"], _lengths(case)
        T = sum(rows)
        s["table"], pages = _pages(lens, rng)
        s["k"], s["ks"] = _cache(_gen(seed, 1), Hk, pages, dh)
        s["v"], s["vs"] = _cache(_gen(seed, 2), Hk, pages, dh)
        s["q"] = torch.randn(T, H, dh, generator=_gen(seed, 3), device=DEV).bfloat16()
        new = torch.randn(2, T, Hk, dh, generator=_gen(seed, 4), device=DEV).bfloat16()
        s.update(k_rows=new[0], v_rows=new[1], off=_offsets(rows), prefix=_ints(lens), longest=max(lens),
                 out=torch.zeros_like(s["q"]), status=_ints([0] * case["seqs"]))
    else:
        B, n, V, g = case["seqs"], case["nodes"], case["vocab"], _gen(seed, 1)
        x = torch.randn(B * n, V, generator=g, device=DEV) * 3
        if case["coarse"]:
            x = x.bfloat16().float()
        if case["masked"]:
            x = x.masked_fill(torch.rand(B * n, V, generator=g, device=DEV) < 0.5, -math.inf)
        rules = np.zeros((B, 4), dtype=np.float32)  # temperature, top-k, top-p, min-p
        for b in range(B):
            on = case["rules"] if case["rules"] != "mixed" else ["", "k", "p", "m", "kp", "kpm"][rng.integers(6)]
            rules[b] = [rng.uniform(0.6, 1.3), rng.integers(1, 200) if "k" in on else 0,
                        rng.uniform(0.5, 0.98) if "p" in on else 1, rng.uniform(0.01, 0.2) if "m" in on else 0]
            if case["rules"] == "mixed" and rng.random() < 0.1:
                rules[b, 0] = 0
        s.update(x=x, rules=torch.from_numpy(rules).to(DEV), u=torch.rand(B * n, generator=g, device=DEV),
                 off=_offsets([n] * B), token=_ints([0] * (B * n)), prob=torch.zeros(B * n, device=DEV), status=_ints([0] * B))
    return s


# ------------------------------------------------------------------------------ the calls
def run(s):
    return _own(s) if own else _PLAIN[s["case"]["kind"]](s)


def _own(s):
    from paper_2406_17404_amd import binding as B
    c = s["case"]
    if c["kind"] == "rotary":
        B.rotary_rows(s["q"], s["k"], s["parent"], s["off"], s["prefix"], s["freqs"], s["magnitude"],
                      B.ROTARY_PAIRS if c["pairs"] else B.ROTARY_HALVES, s["q_out"], s["k_out"], s["status"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["kind"] == "chunk":
        if "ws" not in s:
            s["ws"] = torch.empty(B.chunk_attention_q8_workspace_bytes(c["seqs"], s["q"].shape[0], c["heads"], c["kv_heads"],
                                                                       c["head_dim"], s["longest"]),
                                  dtype=torch.uint8, device=DEV)
        B.chunk_attention_q8(s["q"], s["k"], s["v"], s["ks"], s["vs"], s["k_rows"], s["v_rows"], s["off"], s["table"],
                             s["prefix"], s["longest"], 1.0 / math.sqrt(c["head_dim"]), s["ws"], s["out"], s["status"])
        return s["out"]
    if "ws" not in s:
        s["ws"] = torch.empty(B.tree_sample_workspace_bytes(c["seqs"], s["x"].shape[0], c["vocab"]), dtype=torch.uint8,
                              device=DEV)
    B.tree_sample(s["x"], s["off"], s["rules"], s["u"], s["token"], s["prob"], s["ws"], s["status"])
    return {"token": s["token"], "prob": s["prob"]}


# ------------------------------------------------------------------------------ plain forms
def _depths(parent, sizes):
    """Of every node of trees of equal size, parent by parent."""
    B, n = len(sizes), sizes[0]
    p = parent.view(B, n).long()
    at, depth = p, torch.zeros_like(p)
    while bool((at >= 0).any()):
        depth = depth + (at >= 0)
        at = torch.where(at >= 0, p.gather(1, at.clamp(min=0)), at)
    return depth.view(-1)


def _plain_rotary(s):
    c, off = s["case"], s["off"].long()
    t = torch.arange(s["q"].shape[0], device=DEV)
    seq = torch.searchsorted(off, t, right=True) - 1
    j = t - off[seq] if s["parent"] is None else _depths(s["parent"], _rows(c))
    angle = (s["prefix"].long()[seq] + j).double()[:, None] * s["freqs"]
    cos, sin = ((f(angle) * s["magnitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    n = c["rot_dim"] // 2

    def turn(x):
        y = x.float()
        if c["pairs"]:
            a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        else:
            a, b = y[..., :n], y[..., n:2 * n]
        a, b = a * cos - b * sin, a * sin + b * cos
        front = torch.stack([a, b], -1).flatten(-2) if c["pairs"] else torch.cat([a, b], -1)
        return torch.cat([front, y[..., 2 * n:]], -1).to(x.dtype)

    return {"q": turn(s["q"]), "k": turn(s["k"])}


def _untile_k(x, dh):
    """[.., 32 * dh] as laid out in a page -> [.., 32, dh]."""
    lead = x.shape[:-1]
    return x.view(*lead, dh // 32, 2, 32, 16).movedim(-2, -4).reshape(*lead, 32, dh)


def _untile_v(x, dh):
    lead, n = x.shape[:-1], x.dim() - 1  # a page: [dh/32][slot/4%2][32 columns][slot/16][slot/8%2][slot%4]
    x = x.view(*lead, dh // 32, 2, 32, 2, 2, 4)
    return x.permute(*range(n), n + 3, n + 4, n + 1, n + 5, n, n + 2).reshape(*lead, 32, dh)


def _plain_chunk(s):
    c = s["case"]
    H, Hk, dh = c["heads"], c["kv_heads"], c["head_dim"]
    out, r = torch.empty_like(s["q"]), 0
    for b, (L, n) in enumerate(zip(_lengths(c), _rows(c))):
        pages = s["table"][b, :-(-L // PAGE)].long()
        keys = L + n
        seen = torch.arange(keys, device=DEV) <= L + torch.arange(n, device=DEV)[:, None]  # [n, keys]
        heads = Hk if H * n * keys < 1 << 29 else 1  # K/V heads at a time
        for h in range(0, Hk, heads):
            kv = []
            for pool, scale, rows, untile in ((s["k"], s["ks"], s["k_rows"], _untile_k), (s["v"], s["vs"], s["v_rows"], _untile_v)):
                x = pool[h:h + heads, pages].view(torch.float8_e4m3fn).float() * scale[h:h + heads, pages][..., None]
                x = untile(x, dh).reshape(heads, -1, dh)[:, :L]
                kv.append(torch.cat([x, rows[r:r + n, h:h + heads].float().transpose(0, 1)], 1))
            q = s["q"][r:r + n].float().view(n, Hk, H // Hk, dh)[:, h:h + heads].permute(1, 2, 0, 3).reshape(heads, -1, dh)
            score = torch.matmul(q, kv[0].transpose(1, 2)) * (1.0 / math.sqrt(dh))
            score = score.view(heads, H // Hk, n, keys).masked_fill(~seen, -math.inf)
            p = (score - score.amax(-1, keepdim=True)).exp()
            p = (p / p.sum(-1, keepdim=True)).view(heads, -1, keys)
            o = torch.matmul(p, kv[1]).view(heads, H // Hk, n, dh).permute(2, 0, 1, 3)
            out[r:r + n].view(n, Hk, H // Hk, dh)[:, h:h + heads] = o.bfloat16()
        r += n
    return out


def _plain_sample(s):
    c = s["case"]
    V = c["vocab"]
    x, order = torch.sort(s["x"], dim=1, descending=True, stable=True)
    t, k, p, least = (s["rules"].repeat_interleave(c["nodes"], 0)[:, i:i + 1].double() for i in range(4))
    greedy = t == 0
    w = torch.round(torch.exp((x.double() - x[:, :1].double()) / torch.where(greedy, torch.ones_like(t), t)) * UNIT).long()
    place = torch.arange(V, device=DEV)
    w = w * (place < torch.where(k >= 1, k, torch.full_like(k, V)))
    upto = w.cumsum(1)
    enough = torch.where(p < 1, torch.ceil(p * upto[:, -1:].double()), upto[:, -1:].double()).long()
    keep = (place == 0) | ((upto - w < enough) & (w >= torch.ceil(least * UNIT).long()))
    keep = torch.where(greedy, place == 0, keep)
    w = w * keep
    upto = w.cumsum(1)
    target = torch.floor(s["u"].double()[:, None] * upto[:, -1:].double()).long().minimum(upto[:, -1:] - 1)
    at = (upto <= target).sum(1, keepdim=True)
    prob = w.gather(1, at).double() / upto[:, -1:].double()
    return {"token": order.gather(1, at)[:, 0].int(), "prob": prob[:, 0].float()}


_PLAIN = {"rotary": _plain_rotary, "chunk": _plain_chunk, "sample": _plain_sample}


# ------------------------------------------------------------------------------ the work
def work(case):
    if case["kind"] == "rotary":
        rows, width = sum(_rows(case)), (case["heads"] + case["kv_heads"]) * case["head_dim"]
        turned = (case["heads"] + case["kv_heads"]) * case["rot_dim"]
        return {"bytes": rows * (2 * width * (2 if case["dtype"] == "bf16" else 4) + 4) + 4 * case["rot_dim"],
                "flops": 3 * rows * turned}
    if case["kind"] == "chunk":
        H, Hk, dh, lens, rows = case["heads"], case["kv_heads"], case["head_dim"], _lengths(case), _rows(case)
        pages = sum(-(-l // PAGE) for l in lens)
        return {"bytes": sum(lens) * 2 * Hk * dh + pages * (8 * Hk + 4) + sum(rows) * (4 * Hk * dh + 4 * H * dh),
                "flops": sum(4 * H * dh * (n * l + n * (n + 1) // 2) for l, n in zip(lens, rows))}
    rows = case["nodes"] * case["seqs"]
    return {"bytes": rows * (4 * case["vocab"] + 12) + 16 * case["seqs"], "flops": 20 * rows * case["vocab"]}


# ------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "chunk": _exact_chunk, "sample": _exact_sample}[case["kind"]](case, s)


def _exact_rotary(case, s):
    n, at = case["rot_dim"] // 2, []
    parent = None if s["parent"] is None else s["parent"].tolist()
    r = 0
    for L, rows in zip(_lengths(case), _rows(case)):
        depth = list(range(rows))
        if parent is not None:
            for i in range(rows):
                depth[i] = 0 if i == 0 else depth[parent[r + i]] + 1
        at += [L + d for d in depth]
        r += rows
    angle = torch.tensor(at, device=DEV, dtype=torch.float64)[:, None] * s["freqs"]
    by = torch.polar(torch.full_like(angle, s["magnitude"]), angle)[:, None]
    out = {}
    for name in "qk":
        x = s[name].double().clone()
        a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if case["pairs"] else (x[..., :n], x[..., n:2 * n])
        z = torch.complex(a.contiguous(), b.contiguous()) * by
        a.copy_(z.real), b.copy_(z.imag)
        out[name] = x
    return out


def _exact_chunk(case, s):
    dh, Hk, group = case["head_dim"], case["kv_heads"], case["heads"] // case["kv_heads"]
    code = torch.arange(256, device=DEV)  # e4m3: sign, four bits of exponent, three of mantissa
    e, m = (code >> 3) & 15, (code & 7).double()
    values = torch.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * torch.exp2(e.double() - 7))
    values = torch.where(code >= 128, -values, values)
    r, col = torch.arange(32, device=DEV)[:, None], torch.arange(dh, device=DEV)  # where a page keeps (slot r, column)
    place_k = ((col // 32 * 2 + col % 32 // 16) * 32 + r) * 16 + col % 16
    place_v = ((col // 32 * 2 + r // 4 % 2) * 32 + col % 32) * 16 + r // 16 * 8 + r // 8 % 2 * 4 + r % 4
    out, first = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV), 0
    for b, (L, n) in enumerate(zip(_lengths(case), _rows(case))):
        rows, pages = slice(first, first + n), s["table"][b, :-(-L // PAGE)].long()
        later = torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1)
        for h in range(Hk):
            kv = []
            for pool, scale, new, place in ((s["k"], s["ks"], s["k_rows"], place_k), (s["v"], s["vs"], s["v_rows"], place_v)):
                x = values[pool[h, pages].long()[:, place.reshape(-1)]].view(-1, 32, dh) * scale[h, pages].double()[:, None, None]
                kv.append(torch.cat([x.reshape(-1, dh)[:L], new[rows, h].double()]))
            for g in range(h * group, (h + 1) * group):
                score = s["q"][rows, g].double() @ kv[0].t().contiguous() / math.sqrt(dh)
                score[:, L:].masked_fill_(later, -math.inf)
                out[rows, g] = torch.softmax(score, 1) @ kv[1]
        first += n
    return out


def _exact_sample(case, s):
    x, u, rules = s["x"].cpu().numpy().astype(np.float64), s["u"].double().tolist(), s["rules"].double().tolist()
    token, prob = [], []
    for i, row in enumerate(x):
        t, k, p, least = rules[i // case["nodes"]]
        top = row.max()
        if t == 0:
            token.append(int(np.flatnonzero(row == top)[0])), prob.append(1.0)
            continue
        some = np.flatnonzero(row >= top - 28 * t)  # what lies lower weighs nothing
        some = some[np.lexsort((some, -row[some]))]
        if k >= 1:
            some = some[:int(k)]
        w = np.rint(np.exp((row[some] - top) / t) * UNIT).astype(np.int64)
        n = len(w)
        if p < 1:
            n = max(1, int(np.searchsorted(np.cumsum(w), math.ceil(p * float(w.sum())))) + 1)
        w = w[:n]
        w = w[:max(1, int((w >= math.ceil(least * UNIT)).sum()))]
        total = int(w.sum())
        at = int(np.searchsorted(np.cumsum(w), min(math.floor(u[i] * float(total)), total - 1), side="right"))
        token.append(int(some[at])), prob.append(float(w[at]) / total)
    return {"token": torch.tensor(token, dtype=torch.int32, device=DEV), "prob": torch.tensor(prob, dtype=torch.float64, device=DEV)}
