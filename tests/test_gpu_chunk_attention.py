"""chunk_attention_q8 against the 64-bit oracle, element by element.

Tolerance: the result is rounded to bf16 (half a step, 2^-8 of it) and so is every weight
(2^-8 each, so at most 2^-8 of the weighted mean of |v|, which the oracle returns); codes times
scales are exact.  The rest is 32-bit: scores below 64 in magnitude and their sums are off by less
than 2^-13, and so is a weight's exponent."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32
from oracle import tr_prompt as P
from paper_2406_17404_amd import binding as b
from serve_util import NAN_CODE, Paged, bf16, ints, offsets_of
from oracle import tr_serve as S

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


class Call:
    def __init__(self, rng, lens, sizes, heads, kv_heads, dh, wide=0, behind=0, exps=(-8, -4), scale=None):
        self.cache = Paged(rng, lens, kv_heads, dh, exps=exps)
        self.off, self.heads, self.dh = offsets_of(sizes), heads, dh
        T = self.T = int(self.off[-1]) + behind
        self.q, self.kr, self.vr = (bf16(rng.normal(size=(T, h, dh))) for h in (heads, kv_heads, kv_heads))
        self.scale, self.wide = scale or 1 / np.sqrt(dh), wide

    def device(self):
        rows = []
        for x in (self.q, self.kr, self.vr):
            buf = torch.full((self.T, x.shape[1] * self.dh + self.wide), float("nan"), dtype=torch.bfloat16, device=DEV)
            buf[:, :x.shape[1] * self.dh] = x.reshape(self.T, -1).to(DEV)
            rows.append(buf[:, :x.shape[1] * self.dh].unflatten(1, x.shape[1:]))
        d = self.cache.device()
        most = max([0] + [l for l in self.cache.lens if 0 <= l < 1 << 20])
        B, Hk = len(self.cache.lens), self.cache.heads
        ws = torch.full((b.chunk_attention_q8_workspace_bytes(B, self.T, self.heads, Hk, self.dh, most),), 255,
                        dtype=torch.uint8, device=DEV)
        out = torch.full((self.T, self.heads, self.dh), 5.0, dtype=torch.bfloat16, device=DEV)
        return [rows[0], *(d[n][0] for n in ("k", "v", "ks", "vs")), rows[1], rows[2], i32(self.off), d["table"],
                d["prefix"], most, float(self.scale), ws, out, ints(B)]

    def run(self):
        args = self.device()
        b.chunk_attention_q8(*args)
        torch.cuda.synchronize()
        self.status = args[-1].cpu().numpy()
        return args[-2].float().cpu().numpy()

    def check(self, got=None, skip=()):
        got = self.run() if got is None else got
        covered = np.zeros(self.T, bool)
        for s in range(len(self.cache.lens)):
            r = slice(max(self.off[s], 0), self.off[s + 1])
            covered[r] = True
            if s in skip or self.off[s] == self.off[s + 1]:
                continue
            want, mean = P.chunk_attention(self.q[r].float().numpy(), self.cache.values("k", s), self.cache.values("v", s),
                                           self.kr[r].float().numpy(), self.vr[r].float().numpy(), self.scale)
            tol = HALF * (np.abs(want) + mean) * (1 + HALF) + 2.0 ** -12 * mean
            bad = ~(np.abs(got[r] - want) <= tol)
            assert not bad.any(), (s, np.argwhere(bad)[:4], np.abs(got[r] - want).max(), np.abs(want).max())
        assert (got[~covered] == 5.0).all()
        return got


@pytest.mark.parametrize("heads,kv_heads,dh", [(4, 4, 64), (4, 1, 128), (6, 2, 128), (2, 2, 128), (5, 1, 64)])
@pytest.mark.parametrize("L,n", [(0, 1), (0, 2), (0, 33), (0, 64), (0, 65), (1, 1), (31, 1), (32, 1), (33, 7), (63, 5), (64, 32),
                                 (65, 3), (100, 33), (257, 64), (500, 128), (1000, 69), (2100, 5), (96, 300), (130, 700)])
def test_single_sequences(heads, kv_heads, dh, L, n):
    c = Call(np.random.default_rng(31 * L + n + dh), [L], [n], heads, kv_heads, dh, wide=8 * (n % 2))
    c.check()
    assert list(c.status) == [0]


@pytest.mark.parametrize("seed", range(8))
def test_packed_sequences_of_any_lengths(seed):
    rng = np.random.default_rng(800 + seed)
    B = int(rng.integers(2, 9))
    kv_heads, group, dh = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 8])), int(rng.choice([64, 128]))
    lens = [int(rng.choice([0, 1, 31, 32, 33, 64, 500, 1500])) if rng.random() < 0.5 else int(rng.integers(0, 900)) for _ in range(B)]
    sizes = [int(rng.choice([0, 1, 1, 2, 31, 32, 33, 64, 65, 128, 129, 257, 400])) for _ in range(B)]
    sizes[0] = max(sizes[0], 1)
    c = Call(rng, lens, sizes, kv_heads * group, kv_heads, dh, behind=int(rng.integers(0, 3)))
    c.check()
    assert not c.status.any()


def test_many_sequences():
    rng = np.random.default_rng(1)
    lens = rng.integers(0, 200, 150)
    lens[70] = 3000  # far longer than the others
    sizes = [1] * 150
    sizes[20], sizes[149], sizes[33] = 200, 70, 0
    Call(rng, lens, sizes, 2, 1, 64).check()


def test_long_sequences_are_split_and_merged():
    rng = np.random.default_rng(2)
    Call(rng, [20000, 40], [3, 270], 2, 1, 128).check()
    Call(rng, [9000], [1], 16, 2, 64).check()


def test_a_range_that_goes_down_leaves_the_others():
    rng = np.random.default_rng(4)
    c = Call(rng, [50, 90], [20, 30], 4, 2, 64)
    c.check()
    args = c.device()
    args[7] = i32([20, 50, 20])
    b.chunk_attention_q8(*args)
    torch.cuda.synchronize()
    assert list(args[-1].cpu().numpy()) == [0, 1] and (args[-2][:20] == 5.0).all()


def test_scores_far_from_zero():
    rng = np.random.default_rng(5)
    c = Call(rng, [40], [100], 2, 1, 64, exps=(40, 41))
    c.cache.scale["v"][:] = 1.0
    c.q = (c.q.float() * 2.0 ** 70).bfloat16()
    got = c.run()
    keys = np.concatenate([c.cache.values("k", 0)[0], c.kr[:, 0].float().numpy()])
    vals = np.concatenate([c.cache.values("v", 0)[0], c.vr[:, 0].float().numpy()])
    for i in range(100):
        for h in range(2):
            score = keys[:40 + i + 1] @ c.q[i, h].float().numpy().astype(np.float64)
            v = vals[score.argmax()]
            assert np.abs(got[i, h] - v).max() <= HALF * np.abs(v).max()
    c = Call(rng, [40], [70], 1, 1, 64, scale=1e30)
    c.q = -c.q.abs()
    c.cache.pool["k"][:] &= 127  # every score below -1e30
    c.kr = c.kr.abs()
    assert np.isfinite(c.run()).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("L,n", [(45, 7), (45, 40), (0, 200), (9000, 70)])
def test_what_is_not_finite_stays_with_those_who_see_it(value, L, n):
    rng = np.random.default_rng(6)
    c = Call(rng, [L], [n], 4, 2, 64)
    clean = c.check()
    j = n - 3  # seen by itself and two more
    c.kr[j, 0, 3] = value
    c.vr[j, 1, 5] = value
    got = c.run()
    assert np.array_equal(got[:j], clean[:j])
    if value == value:  # K/V head 1 belongs to query heads 2, 3
        assert (got[j:, 2:, 5] == value).all()
    else:
        assert np.isnan(got[j:, 2:, 5]).all() and np.isnan(got[j:, :2]).all()
    keep = [d for d in range(64) if d != 5]
    assert np.array_equal(got[j:, 2:][:, :, keep], clean[j:, 2:][:, :, keep])
    c.vr[0, 0, 9] = value  # the first row: all see it
    assert not np.isfinite(c.run()[:, 0, 9]).any()


def test_unused_slots_and_pages_may_hold_anything():
    rng = np.random.default_rng(7)
    c = Call(rng, [33], [4], 2, 1, 128)
    a = c.check()
    for code in (NAN_CODE, 255, 126, 0):
        for w in "kv":
            page = c.cache.pool[w][:, :, c.cache.table[0, 1]]
            page[..., S.offsets(128, w)[1:]] = code
            c.cache.pool[w][:, :, c.cache.table[0, 1]] = page
        assert np.array_equal(c.run(), a)
    others = [p for p in range(c.cache.n_blocks) if p not in c.cache.table[0, :2]]
    for w in "kv":
        c.cache.scale[w][..., others] = np.nan
    assert np.array_equal(c.run(), a)


def test_sequences_may_share_pages():
    rng = np.random.default_rng(8)
    c = Call(rng, [64, 90], [70, 5], 2, 1, 64)
    c.cache.table[1, :2] = c.cache.table[0, :2]
    c.check()


@pytest.mark.parametrize("what", ["long prefix", "negative prefix", "rows", "pages", "wide"])
def test_malformed_sequences(what):
    rng = np.random.default_rng(9)
    c = Call(rng, [70, 100, 40], [5, 300, 9], 4, 2, 64)
    zero = True
    if what == "long prefix":
        c.cache.lens[1] = 1 << 21
    elif what == "negative prefix":
        c.cache.lens[1] = -1
    elif what == "rows":
        c.off, zero = np.array([0, 5, 305, 315]), False
    elif what == "pages":
        c.cache.table[1, 2], zero = c.cache.n_blocks, None
    elif what == "wide":
        c.cache.lens[1] = c.cache.width * 32 + 1
    got = c.run()
    bad = 2 if what == "rows" else 1
    assert list(c.status) == [int(s == bad) for s in range(3)]
    rows = got[c.off[bad]:c.off[bad + 1]]
    assert (rows == 0).all() if zero else np.isnan(rows).all() if zero is None else (rows == 5.0).all()
    c.check(got, skip=(bad,))


def test_bad_pages_of_long_sequences():
    rng = np.random.default_rng(10)
    c = Call(rng, [9000, 9000], [4, 4], 2, 1, 64)
    c.cache.table[1, 200] = -5
    got = c.run()
    assert list(c.status) == [0, 1] and np.isnan(got[4:]).all()
    c.check(got, skip=(1,))


def test_same_bits_every_time():
    rng = np.random.default_rng(13)
    c = Call(rng, [5000, 77], [3, 200], 4, 2, 128)
    a = c.run()
    assert all(np.array_equal(a, c.run()) for _ in range(3))


def test_captured_and_replayed_with_other_lengths():
    rng = np.random.default_rng(11)
    c = Call(rng, [3000, 700], [130, 40], 4, 2, 128)
    args = c.device()
    b.chunk_attention_q8(*args)
    torch.cuda.synchronize()
    want = args[-2].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.chunk_attention_q8(*args)
    shorter = i32([1000, 0])
    for _ in range(3):
        keep = args[9].clone()
        args[9].copy_(shorter)
        g.replay()
        torch.cuda.synchronize()
        other = args[-2].clone()
        b.chunk_attention_q8(*args)
        torch.cuda.synchronize()
        assert torch.equal(other, args[-2]) and not torch.equal(other, want)
        args[9].copy_(keep)
        args[-2].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(args[-2], want)


def test_two_streams_with_workspaces_of_their_own():
    rng = np.random.default_rng(12)
    calls = [Call(rng, [4000], [150], 4, 2, 128), Call(rng, [2500, 100], [7, 264], 4, 1, 64)]
    args = [c.device() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for st, a in zip(streams, args):
            with torch.cuda.stream(st):
                b.chunk_attention_q8(*a)
    torch.cuda.synchronize()
    for c, a in zip(calls, args):
        c.check(a[-2].float().cpu().numpy())


@pytest.mark.parametrize("B,n,heads", [(65, 320, 4), (65, 1280, 1), (80, 300, 4), (70, 260, 5)])
def test_many_prompts_at_once(B, n, heads):
    # beyond 64 sequences, all of a length at which they are just split: every split has room for its partials
    c = Call(np.random.default_rng(B + n), [0] * B, [n] * B, heads, 1, 64)
    c.check()
    assert not c.status.any()


@pytest.mark.parametrize("seed", range(4))
def test_many_sequences_of_any_lengths(seed):
    rng = np.random.default_rng(900 + seed)
    B, kv_heads, group = int(rng.integers(65, 200)), int(rng.integers(1, 3)), int(rng.integers(1, 6))
    lens = rng.integers(0, 25, B) ** 2 * int(rng.integers(0, 2))
    sizes = [int(x) for x in rng.integers(0, int(rng.choice([3, 60, 200])), B)]
    sizes[B // 2] = 70
    c = Call(rng, [int(x) for x in lens], sizes, kv_heads * group, kv_heads, 64, behind=2)
    c.check()
    assert not c.status.any()


def test_an_unaligned_workspace():
    c = Call(np.random.default_rng(15), [5000, 64], [3, 100], 4, 2, 64)
    want, args = c.run(), c.device()
    args[12] = torch.full((args[12].numel() + 13,), 255, dtype=torch.uint8, device=DEV)[13:]
    b.chunk_attention_q8(*args)
    torch.cuda.synchronize()
    assert np.array_equal(args[13].float().cpu().numpy(), want)


def pieces(c):
    d = c.device()
    return d[0], d[1:5], d[5:7], d[7:]


def test_fractions_of_scales_do_not_count():
    rng = np.random.default_rng(16)
    c = Call(rng, [300, 45], [20, 7], 4, 2, 128)
    want = c.run()
    for w in "kv":
        c.cache.scale[w] = (c.cache.scale[w] * rng.uniform(1, 1.999, c.cache.scale[w].shape)).astype(np.float32)
    assert np.array_equal(c.run(), want)


@pytest.mark.parametrize("dh,n_blocks", [(128, 800_000), (64, 1_500_000)])
def test_pools_beyond_4_gib(dh, n_blocks):
    c = Call(np.random.default_rng(dh), [700, 45], [20, 70], 4, 2, dh)
    want = c.run()
    q, pools, rows, rest = pieces(c)
    shift = n_blocks - c.cache.n_blocks  # the same pages at the end of pools of 6.5 and 6.1 GB
    big = [torch.empty((2, n_blocks) + t.shape[2:], dtype=t.dtype, device=DEV) for t in pools]
    for x, y in zip(big, pools):
        x[:, shift:] = y
    assert big[0].numel() > 2 ** 32
    rest[1] = torch.where(rest[1] >= 0, rest[1] + shift, rest[1])
    b.chunk_attention_q8(q, *big, *rows, *rest)
    torch.cuda.synchronize()
    assert np.array_equal(rest[-2].float().cpu().numpy(), want) and not rest[-1].any()


def test_rows_beyond_2_to_the_32_elements():
    c = Call(np.random.default_rng(17), [50, 33, 100], [128, 100, 72], 4, 2, 64)
    c.vr[299, 1, 3] = float("inf")
    want = c.run()
    q, pools, rows, rest = pieces(c)
    wide = torch.empty(300, 1 << 24, dtype=torch.bfloat16, device=DEV)  # the longest stride, 10 GB
    far, at = [], (1 << 24) - 1024
    for x in (q, *rows):
        n = x.shape[1] * 64
        wide[:, at:at + n] = x.reshape(300, n)
        far.append(wide[:, at:at + n].unflatten(1, (x.shape[1], 64)))
        at += n
    b.chunk_attention_q8(far[0], *pools, *far[1:], *rest)
    torch.cuda.synchronize()
    assert np.array_equal(rest[-2].float().cpu().numpy(), want) and np.isinf(want[299, 2:, 3]).all()


@pytest.mark.parametrize("n", [1, 70])
def test_the_longest_prefix(n):
    # as long as positions go: few pages, named over and over
    rng = np.random.default_rng(18)
    L, n_blocks, dh = 2 ** 31 - 65 - n, 3, 64
    pages = (L + 31) // 32
    pool = {w: S.encode((rng.normal(size=(1, n_blocks, 32 * dh)) * 60).clip(-448, 448)) for w in "kv"}
    scale = {w: np.full((1, n_blocks), 2.0 ** -6, np.float32) for w in "kv"}
    q, kr, vr = (bf16(rng.normal(size=(n, 1, dh))) for _ in range(3))
    table = (torch.arange(pages, device=DEV) % n_blocks).int()[None]
    ws = torch.empty(b.chunk_attention_q8_workspace_bytes(1, n, 1, 1, dh, L), dtype=torch.uint8, device=DEV)
    out, status = torch.full((n, 1, dh), 5.0, dtype=torch.bfloat16, device=DEV), ints(1)
    b.chunk_attention_q8(q.to(DEV), *(torch.from_numpy(pool[w]).to(DEV) for w in "kv"),
                         *(torch.from_numpy(scale[w]).to(DEV) for w in "kv"), kr.to(DEV), vr.to(DEV), i32([0, n]), table, i32([L]),
                         L, dh ** -0.5, ws, out, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0]
    times = np.zeros((n_blocks, 32))
    for p in range(n_blocks):
        times[p] = len(range(p, pages, n_blocks))
    if L % 32:
        times[(pages - 1) % n_blocks, L % 32:] -= 1
    keys, values = (S.page_values(pool[w][0], scale[w][0], w).reshape(-1, dh) for w in "kv")
    # as for short ones, and 32-bit sums over a split's blocks, 2^25 / 32 of them at most: half a step of 2^-23 for each
    # that the sum of weights adds, and for each product of 16 keys (four of a block) that the values' sums add
    long_sum = 2.0 ** 20 * (2 * 2.0 ** -24 + 4 * 2.0 ** -23)
    got = out.float().cpu().numpy()
    for i in range(n):
        f = q[i, 0].float().numpy().astype(np.float64)
        k = np.concatenate([keys, kr[:i + 1, 0].float().numpy()])
        v = np.concatenate([values, vr[:i + 1, 0].float().numpy()])
        w = np.concatenate([times.ravel(), np.ones(i + 1)]) * np.exp(dh ** -0.5 * (k @ f))
        w /= w.sum()
        want, mean = w @ v, w @ np.abs(v)
        tol = HALF * (np.abs(want) + mean) * (1 + HALF) + (long_sum + 2.0 ** -12) * mean
        assert (np.abs(got[i, 0] - want) <= tol).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("L,n,heads", [(9000, 7, 4), (9000, 16, 4), (0, 3, 4), (64, 5, 6), (9000, 100, 4)])
def test_what_is_not_finite_in_split_sequences_and_short_ones(value, L, n, heads):
    rng = np.random.default_rng(19)
    c = Call(rng, [L], [n], heads, 2, 64)
    clean = c.check()
    j, g = n - 2, heads // 2
    c.kr[j, 0, 3] = value
    c.vr[j, 1, 5] = value
    got = c.run()
    assert np.array_equal(got[:j], clean[:j])
    if value == value:
        assert (got[j:, g:, 5] == value).all()
    else:
        assert np.isnan(got[j:, g:, 5]).all() and np.isnan(got[j:, :g]).all()
    keep = [d for d in range(64) if d != 5]
    assert np.array_equal(got[j:, g:][:, :, keep], clean[j:, g:][:, :, keep])


@pytest.mark.parametrize("L,n", [(33, 40), (33, 1), (65, 200), (9001, 3), (9001, 90)])
def test_unused_slots_of_the_last_page_may_hold_anything(L, n):
    c = Call(np.random.default_rng(20), [L], [n], 2, 1, 128)
    want = c.check()
    last, used = c.cache.table[0, (L - 1) // 32], (L - 1) % 32 + 1
    for code in (NAN_CODE, 255, 126):
        for w in "kv":
            page = c.cache.pool[w][:, :, last]
            page[..., S.offsets(128, w)[used:]] = code
            c.cache.pool[w][:, :, last] = page
        assert np.array_equal(c.run(), want)


@pytest.mark.parametrize("n", [3, 60])
def test_pages_that_are_not_there(n):
    c = Call(np.random.default_rng(21), [9000, 9000, 70], [n] * 3, 2, 1, 64)
    c.cache.table[0, 200], c.cache.table[2, 0] = -1, c.cache.n_blocks
    got = c.run()
    assert list(c.status) == [1, 0, 1] and np.isnan(got[:n]).all() and np.isnan(got[2 * n:]).all()
    c.check(got, skip=(0, 2))


@pytest.mark.parametrize("n", [1, 10])
def test_scores_far_from_zero_of_few_queries(n):
    rng = np.random.default_rng(22)
    c = Call(rng, [40], [n], 2, 1, 64, exps=(40, 41))
    c.cache.scale["v"][:] = 1.0
    c.q = (c.q.float() * 2.0 ** 70).bfloat16()
    got = c.run()
    keys = np.concatenate([c.cache.values("k", 0)[0], c.kr[:, 0].float().numpy()])
    vals = np.concatenate([c.cache.values("v", 0)[0], c.vr[:, 0].float().numpy()])
    for i in range(n):
        for h in range(2):
            v = vals[(keys[:40 + i + 1] @ c.q[i, h].float().numpy().astype(np.float64)).argmax()]
            assert np.abs(got[i, h] - v).max() <= HALF * np.abs(v).max()
    c = Call(rng, [40], [n], 1, 1, 64, scale=1e30)
    c.q = -c.q.abs()
    c.cache.pool["k"][:] &= 127  # every score below -1e30
    c.kr = c.kr.abs()
    assert np.isfinite(c.run()).all()


@pytest.mark.parametrize("dh,n", [(64, 1), (128, 3), (64, 40)])
def test_many_pages_of_one_workgroup(dh, n):
    # so many heads that nothing is split: a wavefront looks pages up several times
    rng = np.random.default_rng(23)
    L, heads, n_blocks = 40000 - 5, 256, 40
    pages = (L + 31) // 32
    codes = {w: (rng.normal(size=(heads, n_blocks, 32 * dh)) * 60).clip(-448, 448) for w in "kv"}
    pool = {w: S.encode(codes[w]) for w in "kv"}
    scale = {w: (2.0 ** rng.integers(-8, -4, (heads, n_blocks))).astype(np.float32) for w in "kv"}
    table = rng.integers(0, n_blocks, pages)
    q, kr, vr = (bf16(rng.normal(size=(n, heads, dh))) for _ in range(3))
    ws = torch.empty(b.chunk_attention_q8_workspace_bytes(1, n, heads, heads, dh, L), dtype=torch.uint8, device=DEV)
    out, status = torch.full((n, heads, dh), 5.0, dtype=torch.bfloat16, device=DEV), ints(1)
    b.chunk_attention_q8(q.to(DEV), *(torch.from_numpy(pool[w]).to(DEV) for w in "kv"),
                         *(torch.from_numpy(scale[w]).to(DEV) for w in "kv"), kr.to(DEV), vr.to(DEV), i32([0, n]),
                         i32(table[None]), i32([L]), L, dh ** -0.5, ws, out, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0]
    got = out.float().cpu().numpy()
    for h in (0, 100, 255):
        k, v = (S.page_values(pool[w][h], scale[w][h], w)[table].reshape(-1, dh)[:L] for w in "kv")
        rows = [x[:, h:h + 1].float().numpy() for x in (q, kr, vr)]
        want, mean = P.chunk_attention(rows[0], k[None], v[None], rows[1], rows[2], dh ** -0.5)
        # 32-bit sums of up to 625 blocks in a row: half a step of 2^-23 for the weights', one for each product of the values'
        tol = HALF * (np.abs(want) + mean) * (1 + HALF) + (625 * 2 * (2.0 ** -24 + 2 * 2.0 ** -23) + 2.0 ** -12) * mean
        assert (np.abs(got[:, h:h + 1] - want) <= tol).all()


@pytest.mark.parametrize("L,n", [(0, 33), (0, 64), (0, 65), (1, 33), (31, 40), (32, 64), (33, 63), (63, 33), (64, 64), (65, 50), (100, 96),
                                 (257, 130)])
def test_short_sequences_of_many_heads(L, n):
    # more tiles of 32 queries than are taken one by one
    c = Call(np.random.default_rng(7 * L + n), [L], [n], 140, 140, 64)
    c.check()


@pytest.mark.parametrize("heads,kv_heads,dh", [(2, 1, 64), (4, 2, 128), (3, 1, 128)])
@pytest.mark.parametrize("L,n", [(0, 1100), (1, 1089), (33, 1025), (95, 1030), (1000, 17), (1023, 90), (1025, 33)])
def test_sequences_just_beyond_short_ones(heads, kv_heads, dh, L, n):
    Call(np.random.default_rng(L + n), [L], [n], heads, kv_heads, dh).check()


@pytest.mark.parametrize("seed", range(4))
def test_short_sequences_beside_long_ones(seed):
    rng = np.random.default_rng(950 + seed)
    kv_heads, group, dh = int(rng.integers(1, 4)), int(rng.choice([1, 4, 8])), int(rng.choice([64, 128]))
    lens = [int(x) for x in rng.choice([0, 20, 300, 800, 1500, 3000], 6)]
    sizes = [int(x) for x in rng.choice([1, 5, 33, 50, 90], 6)]
    c = Call(rng, lens, sizes, kv_heads * group, kv_heads, dh, behind=1)
    c.check()
    assert not c.status.any()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("j", [0, 40, 63, 64, 100, 149])
def test_what_is_not_finite_in_a_short_prompt(value, j):
    c = Call(np.random.default_rng(24), [30], [150], 4, 2, 64)
    clean = c.check()
    c.kr[j, 0, 3] = value
    c.vr[j, 1, 5] = value
    got = c.run()
    assert np.array_equal(got[:j], clean[:j])
    assert (np.isnan if value != value else np.isinf)(got[j:, 2:, 5]).all()
    if value != value:
        assert np.isnan(got[j:, :2]).all()
    keep = [d for d in range(64) if d != 5]
    assert np.array_equal(got[j:, 2:][:, :, keep], clean[j:, 2:][:, :, keep])


@pytest.mark.parametrize("L,n", [(0, 129), (0, 192), (0, 193), (1, 130), (31, 160), (33, 129), (63, 255), (64, 256), (65, 257), (100, 150),
                                 (257, 130), (1000, 133)])
def test_longer_sequences_of_many_heads(L, n):
    # and more than 128 queries of a head
    c = Call(np.random.default_rng(9 * L + n), [L], [n], 140, 140, 64, wide=8 * (n % 2))
    c.check()


@pytest.mark.parametrize("dh,heads", [(64, 140), (128, 70)])
def test_packed_sequences_of_many_heads(dh, heads):
    c = Call(np.random.default_rng(dh), [70, 0, 1000, 33], [150, 140, 1, 260], heads, heads // 2, dh, behind=2)
    c.check()
    assert not c.status.any()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("j", [0, 63, 64, 100, 149])
def test_what_is_not_finite_with_many_heads(value, j):
    c = Call(np.random.default_rng(25), [30], [150], 140, 70, 64)
    clean = c.check()
    c.kr[j, 0, 3] = value
    c.vr[j, 1, 5] = value
    got = c.run()
    assert np.array_equal(got[:j], clean[:j])
    assert (np.isnan if value != value else np.isinf)(got[j:, 2:4, 5]).all()
    if value != value:
        assert np.isnan(got[j:, :2]).all()
    keep = [d for d in range(64) if d != 5]
    assert np.array_equal(got[j:, 2:][:, :, keep], clean[j:, 2:][:, :, keep])


@pytest.mark.parametrize("n", [129, 200])
def test_far_scores_and_unused_slots_with_many_heads(n):
    c = Call(np.random.default_rng(26), [41], [n], 140, 140, 64)
    want = c.check()
    for w in "kv":
        page = c.cache.pool[w][:, :, c.cache.table[0, 1]]
        page[..., S.offsets(64, w)[9:]] = NAN_CODE
        c.cache.pool[w][:, :, c.cache.table[0, 1]] = page
    assert np.array_equal(c.run(), want)
    c = Call(np.random.default_rng(27), [40], [n], 140, 140, 64, scale=1e30)
    c.q = -c.q.abs()
    c.cache.pool["k"][:] &= 127  # every score below -1e30
    c.kr = c.kr.abs()
    assert np.isfinite(c.run()).all()


@pytest.mark.parametrize("heads,kv_heads,dh,n", [(16, 8, 64, 100), (16, 8, 128, 77), (40, 8, 64, 130), (24, 24, 64, 140)])
@pytest.mark.parametrize("L", [9000, 6500 - 31, 12001])
def test_long_sequences_of_several_heads(heads, kv_heads, dh, n, L):
    # split, in tiles of 256 queries
    c = Call(np.random.default_rng(L + n), [L], [n], heads, kv_heads, dh)
    clean = c.check()
    assert list(c.status) == [0]
    last, used = c.cache.table[0, (L - 1) // 32], (L - 1) % 32 + 1
    for w in "kv":
        page = c.cache.pool[w][:, :, last]
        page[..., S.offsets(dh, w)[used:]] = NAN_CODE
        c.cache.pool[w][:, :, last] = page
    assert np.array_equal(c.run(), clean)
    j, g = n - 20, heads // kv_heads
    c.kr[j, 0, 3] = c.vr[j, 1, 5] = float("nan")
    got = c.run()
    assert np.array_equal(got[:j], clean[:j]) and np.isnan(got[j:, :g]).all() and np.isnan(got[j:, g:2 * g, 5]).all()
    keep = [d for d in range(dh) if d != 5]
    assert np.array_equal(got[j:, g:][:, :, keep], clean[j:, g:][:, :, keep])
    c.cache.table[0, 100] = -1
    assert np.isnan(c.run()).all() and list(c.status) == [1]


@pytest.mark.parametrize("n,heads,dh", [(1, 1, 64), (200, 8, 64), (1, 1, 128)])
def test_the_last_position_of_the_longest_prefix(n, heads, dh):
    # every page is the first but the last one, in which the last position outweighs all others: e^60 to 2^31
    L = 2 ** 31 - 64 - n
    pages, last = (L + 31) // 32, (L - 1) % 32
    k, v = (np.zeros((1, 2, 32 * dh), np.uint8) for _ in "kv")
    places = {w: S.offsets(dh, w) for w in "kv"}
    k[0, 1, places["k"][last, 0]] = S.encode(np.array(60.0))
    v[0, 0], v[0, 1] = S.encode(np.array(1.0)), NAN_CODE
    v[0, 1, places["v"][:last]], v[0, 1, places["v"][last]] = S.encode(np.array(1.0)), S.encode(np.array(3.0))
    table = torch.zeros((1, pages), dtype=torch.int32, device=DEV)
    table[0, -1] = 1
    scale = torch.ones(1, 2, device=DEV)
    q = torch.zeros(n, heads, dh, dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 1.0
    own = torch.zeros(n, 1, dh, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(b.chunk_attention_q8_workspace_bytes(1, n, heads, 1, dh, L), dtype=torch.uint8, device=DEV)
    out, status = torch.full((n, heads, dh), 5.0, dtype=torch.bfloat16, device=DEV), ints(1)
    b.chunk_attention_q8(q, torch.from_numpy(k).to(DEV), torch.from_numpy(v).to(DEV), scale, scale, own, own, i32([0, n]), table,
                         i32([L]), L, 1.0, ws, out, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0] and (out.float() - 3).abs().max() <= 2 * HALF * 3


@pytest.mark.parametrize("B", [9, 16, 33, 64])
@pytest.mark.parametrize("kind", ["any", "long and short", "alike", "many heads"])
def test_up_to_64_sequences_come_longest_first(B, kind):
    rng = np.random.default_rng(1000 + B + len(kind))
    lens, sizes = [int(x) for x in rng.integers(0, 400, B)], [int(x) for x in rng.choice([1, 1, 2, 9, 40], B)]
    heads, kv_heads = 4, 2
    if kind == "long and short":  # what is split lies at either end and in the middle
        for s in (0, B // 2, B - 1):
            lens[s], sizes[s] = int(rng.integers(5000, 9000)), int(rng.choice([1, 70]))
    elif kind == "alike":
        lens, sizes = [700] * B, [3] * B
    elif kind == "many heads":  # tiles of 256 queries
        heads, kv_heads, lens = 32, 8, [x // 3 for x in lens]
        sizes = [int(x) for x in rng.choice([1, 20, 70, 130], B)]
    sizes[3] = 0
    c = Call(rng, lens, sizes, heads, kv_heads, 64, behind=1)
    bad = B // 3 + 1
    c.cache.lens[bad] = -1
    got = c.run()
    assert list(c.status) == [int(s == bad and sizes[s] > 0) for s in range(B)]
    assert (got[c.off[bad]:c.off[bad + 1]] == 0).all()
    c.check(got, skip=(bad,))
