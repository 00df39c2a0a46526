"""CPU oracle of serving from the paged 8-bit cache (numpy, 64 bits, one sequence at a time): pages
that follow lengths, the quantising append, tree attention over the cache, logits under
penalties, biases and masks.  Written from the rules in include/trjacobi.h; test infrastructure
only.  Layouts are spelled out slot by slot."""
import numpy as np

PAGE = 32
MAX_PAGES = (2 ** 31 - 1) // PAGE  # positions are int32, to the end of their page
MIN_EXP = -100


# ---------------------------------------------------------------- e4m3
def _e4m3_values():
    v = np.zeros(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[b] = np.nan if (b & 127) == 127 else (-x if b & 128 else x)
    return v


E4M3 = _e4m3_values()
_POS = E4M3[:127]  # ascending


def encode(x):
    """Nearest code of every number of x (|x| <= 448), ties to the even code; NaN and infinities to NaN."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    a = np.where(fine, np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POS, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(a == 0, 0, code)
    code = np.where(np.signbit(x), code | 128, code)
    return np.where(fine, code, 127).astype(np.uint8)


def scale_exp(top):
    """Exponent of the smallest power of two, from 2^-100 on, with which `top` fits into 448."""
    e = MIN_EXP
    while 448.0 * 2.0 ** e < top:
        e += 1
    return e


# ---------------------------------------------------------------- page layout
def k_off(r, c):
    return ((c // 32 * 2 + c % 32 // 16) * 32 + r) * 16 + c % 16


def v_off(r, c):
    return ((c // 32 * 2 + r // 4 % 2) * 32 + c % 32) * 16 + r // 16 * 8 + r // 8 % 2 * 4 + r % 4


def offsets(dh, which):
    """[32, dh] byte places of a page."""
    r, c = np.arange(32)[:, None], np.arange(dh)[None]
    return (k_off if which == "k" else v_off)(r, c)


def page_values(pool, scale, which):
    """[.., n_blocks, 32 * dh] codes and [.., n_blocks] scales -> [.., n_blocks, 32, dh] numbers."""
    dh = pool.shape[-1] // 32
    return E4M3[pool[..., offsets(dh, which)]] * scale[..., None, None].astype(np.float64)


# ---------------------------------------------------------------- tables
def block_tables(table, held, prefix, off, T, free, count, n_blocks):
    """Returns table, held, free list, count, row slots, status as they are afterwards."""
    table, free = table.copy(), free.copy()
    B, width = table.shape
    status, held_out, want, wish = np.zeros(B, int), held.copy(), np.zeros(B, int), np.zeros(B, int)
    for s in range(B):
        n = int(off[s + 1]) - int(off[s])
        want[s] = -(-(int(prefix[s]) + n) // PAGE)
        if n >= 0 and prefix[s] >= 0 and 0 <= held[s] <= width:
            wish[s] = min(want[s], width)
        if n < 0 or off[s] < 0 or off[s + 1] > T or prefix[s] < 0 or not 0 <= held[s] <= width or want[s] > min(width, MAX_PAGES):
            status[s], want[s] = 1, held[s]
    stack = [int(free[i]) for i in range(count)] if 0 <= count <= n_blocks else []
    for s in range(B):
        for j in range(want[s], held[s]):
            if len(stack) < n_blocks:
                stack.append(int(table[s, j]))
                free[len(stack) - 1] = stack[-1]
        held_out[s] = min(want[s], held[s])
    full = False
    for s in range(B):
        need = want[s] - held[s]
        if need <= 0:
            continue
        full = full or need > len(stack)
        if full:
            status[s] = 1
            continue
        for j in range(held[s], want[s]):
            table[s, j] = stack.pop()
        held_out[s] = want[s]
    for s in range(B):
        if status[s]:  # what it wanted beyond what it holds is nowhere
            table[s, max(held[s], 0):wish[s]] = -1
    slot = np.full(T, -1)
    for s in range(B):
        if status[s] == 0:
            for t in range(off[s], off[s + 1]):
                p = int(prefix[s]) + t - int(off[s])
                slot[t] = int(table[s, p // PAGE]) * PAGE + p % PAGE
    return table, held_out, free, len(stack), slot, status


# ---------------------------------------------------------------- append
def append(k_pool, v_pool, k_scale, v_scale, k_rows, v_rows, path, accept, off, table, prefix):
    """pools [layers, heads, n_blocks, 32 * dh] and scales change in place; rows [layers, T, heads, dh].
    Returns new lengths and status."""
    layers, heads, n_blocks, size = k_pool.shape
    dh, T, B = size // 32, k_rows.shape[1], len(prefix)
    new_len, status = np.asarray(prefix).copy(), np.zeros(B, int)
    for s in range(B):
        L, n = int(prefix[s]), int(off[s + 1]) - int(off[s])
        ok = n >= 0 and off[s] >= 0 and off[s + 1] <= T and L >= 0
        picked = list(range(max(n, 0)))
        if ok and path is not None:
            ok = n <= 128 and 0 <= accept[s] < n
            if ok:
                picked = [int(i) for i in path[s][:accept[s] + 1]]
                ok = all(0 <= i < n for i in picked)
        m = len(picked)
        ok = ok and L + m <= min(table.shape[1], MAX_PAGES) * PAGE
        pages = range(L // PAGE, (L + m - 1) // PAGE + 1) if ok and m else range(0)
        ok = ok and all(0 <= table[s, p] < n_blocks for p in pages)
        if not ok:
            status[s] = 1
            continue
        new_len[s] = L + m
        for p in pages:
            a, z = max(L, p * PAGE), min(L + m, (p + 1) * PAGE)
            src = [int(off[s]) + i for i in picked[a - L:z - L]]
            at, r0, r1 = int(table[s, p]), a - p * PAGE, z - p * PAGE
            for pool, scale, rows, which in ((k_pool, k_scale, k_rows, "k"), (v_pool, v_scale, v_rows, "v")):
                place = offsets(dh, which)
                for l in range(layers):
                    for h in range(heads):
                        x = rows[l, src, h].astype(np.float64)
                        e = scale_exp(np.abs(np.where(np.isfinite(x), x, 0)).max())
                        if r0 > 0:
                            old = float(scale[l, h, at])
                            e = max(e, int(np.log2(old)))
                            if 2.0 ** e != old:
                                was = E4M3[pool[l, h, at, place[:r0]]]
                                pool[l, h, at, place[:r0]] = encode(was * (old / 2.0 ** e))
                        pool[l, h, at, place[r0:r1]] = encode(x / 2.0 ** e)
                        scale[l, h, at] = 2.0 ** e
    return new_len, status


# ---------------------------------------------------------------- attention
def on_path(parent):
    n = len(parent)
    see = np.eye(n, dtype=bool)
    for i in range(1, n):
        see[i] |= see[parent[i]]
    return see


def attention(q, keys, values, k_rows, v_rows, parent, scale):
    """One sequence: q [n, H, dh], keys and values [Hkv, L, dh] of the cache, rows [n, Hkv, dh].  Returns
    the result and the same weights' mean of |v|, which errors of the weights are bounded by."""
    n, H, dh = q.shape
    group = H // keys.shape[0]
    see = np.concatenate([np.ones((n, keys.shape[1]), bool), on_path(parent)], 1)
    out, mean = np.zeros((n, H, dh)), np.zeros((n, H, dh))
    for h in range(H):
        k = np.concatenate([keys[h // group], k_rows[:, h // group]]).astype(np.float64)
        v = np.concatenate([values[h // group], v_rows[:, h // group]]).astype(np.float64)
        for i in range(n):
            score = scale * (k[see[i]] @ q[i, h].astype(np.float64))
            w = np.exp(score - score.max())
            w /= w.sum()
            out[i, h], mean[i, h] = w @ v[see[i]], w @ np.abs(v[see[i]])
    return out, mean


# ---------------------------------------------------------------- logits
def tree_logits(x, tok, parent, ctx, gen_start, pen, bias, allowed, dtype=np.float64):
    """One sequence: x [n, V]; pen (repetition, frequency, presence) or None; bias list of (token, value) or
    None; allowed bool [n, V] or None.  Every step in `dtype`.  Returns logits and predictions."""
    n, V = x.shape
    y, best = x.astype(dtype), np.zeros(n, int)
    see = on_path(parent)
    ctx = np.asarray(ctx, int)
    valid = lambda t: t[(t >= 0) & (t < V)]  # noqa: E731
    for i in range(n):
        drafts = valid(np.asarray([tok[j] for j in range(1, n) if see[i, j]], int))
        if pen is not None:
            r, f, p = (dtype(v) for v in pen)
            seen = np.bincount(valid(ctx), minlength=V) + np.bincount(drafts, minlength=V)
            made = np.bincount(valid(ctx[max(0, gen_start):]), minlength=V) + np.bincount(drafts, minlength=V)
            with np.errstate(all="ignore"):
                y[i] = np.where(seen > 0, np.where(y[i] > 0, y[i] / r, y[i] * r), y[i])
                y[i] = y[i] - f * made.astype(dtype)
                y[i] = y[i] - np.where(made > 0, p, dtype(0))
        if bias is not None:
            add = np.zeros(V, dtype)
            for t, v in bias:
                if 0 <= t < V:
                    add[t] = dtype(v)
            y[i] = y[i] + add
        ok = np.ones(V, bool) if allowed is None else allowed[i]
        y[i][~ok] = -np.inf
        key = np.where(np.isnan(y[i]), -np.inf, y[i])
        nums = ok & ~np.isnan(y[i])
        if not ok.any():
            best[i] = -1
        elif not nums.any():
            best[i] = int(np.flatnonzero(ok)[0])
        else:
            best[i] = int(np.flatnonzero(nums & (key == key[nums].max()))[0])
    return y, best
