"""tree_attention_q8 against the 64-bit oracle, element by element.

Tolerance: the result is rounded to bf16 (half a step, 2^-8 of it) and so is every weight
(2^-8 each, so at most 2^-8 of the weighted mean of |v|, which the oracle returns); codes times
scales are exact.  The rest is 32-bit: scores below 64 in magnitude and their sums are off by less
than 2^-13, and so is a weight's exponent."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32
from oracle import tr_serve as S
from paper_2406_17404_amd import binding as b
from paper_2406_17404_amd import inputs as I
from serve_util import NAN_CODE, Paged, bf16, ints, offsets_of

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


class Call:
    def __init__(self, rng, lens, sizes, heads, kv_heads, dh, wide=0, behind=0, parents=None, exps=(-8, -4), scale=None):
        self.cache = Paged(rng, lens, kv_heads, dh, exps=exps)
        self.off, self.heads, self.dh = offsets_of(sizes), heads, dh
        T = self.T = int(self.off[-1]) + behind
        self.q, self.kr, self.vr = (bf16(rng.normal(size=(T, h, dh))) for h in (heads, kv_heads, kv_heads))
        self.parents = parents or [I.tree_random(n, rng) if n else np.zeros(0, int) for n in sizes]
        self.scale = scale or 1 / np.sqrt(dh)
        self.wide = wide

    def device(self):
        rows = []
        for x in (self.q, self.kr, self.vr):
            buf = torch.full((self.T, x.shape[1] * self.dh + self.wide), float("nan"), dtype=torch.bfloat16, device=DEV)
            buf[:, :x.shape[1] * self.dh] = x.reshape(self.T, -1).to(DEV)
            rows.append(buf[:, :x.shape[1] * self.dh].unflatten(1, x.shape[1:]))
        parent = np.full(self.T, 99)
        for s, p in enumerate(self.parents):
            parent[self.off[s]:self.off[s] + len(p)] = p
        d = self.cache.device()
        most = max([0] + [l for l in self.cache.lens if 0 <= l < 1 << 20])
        B, Hk = len(self.cache.lens), self.cache.heads
        ws = torch.full((b.tree_attention_q8_workspace_bytes(B, self.T, self.heads, Hk, self.dh, most),), 255,
                        dtype=torch.uint8, device=DEV)
        out = torch.full((self.T, self.heads, self.dh), 5.0, dtype=torch.bfloat16, device=DEV)
        return (rows[0], *(d[n][0] for n in ("k", "v", "ks", "vs")), rows[1], rows[2], i32(parent), i32(self.off), d["table"],
                d["prefix"], most, float(self.scale), ws, out, ints(B))

    def run(self):
        args = self.device()
        b.tree_attention_q8(*args)
        torch.cuda.synchronize()
        self.status = args[-1].cpu().numpy()
        return args[-2].float().cpu().numpy()

    def want(self, s):
        r = slice(self.off[s], self.off[s + 1])
        return S.attention(*(x[r].float().numpy() if i == 0 else x for i, x in enumerate(
            (self.q, self.cache.values("k", s), self.cache.values("v", s), self.kr[r].float().numpy(), self.vr[r].float().numpy()))),
            self.parents[s], self.scale)

    def check(self, got=None, skip=()):
        got = self.run() if got is None else got
        for s in range(len(self.cache.lens)):
            if s in skip or self.off[s] == self.off[s + 1]:
                continue
            want, mean = self.want(s)
            g = got[self.off[s]:self.off[s + 1]]
            tol = HALF * (np.abs(want) + mean) * (1 + HALF) + 2.0 ** -12 * mean
            bad = ~(np.abs(g - want) <= tol)
            assert not bad.any(), (s, np.argwhere(bad)[:4], np.abs(g - want).max(), np.abs(want).max())
        covered = np.zeros(self.T, bool)
        for s in range(len(self.cache.lens)):
            covered[max(self.off[s], 0):self.off[s + 1]] = True
        assert (got[~covered] == 5.0).all()
        return got


@pytest.mark.parametrize("heads,kv_heads,dh", [(4, 4, 64), (4, 1, 128), (6, 2, 128), (2, 2, 128)])
@pytest.mark.parametrize("L,n", [(0, 1), (0, 2), (0, 33), (1, 1), (31, 1), (32, 1), (33, 7), (64, 32), (100, 33), (257, 64),
                                 (500, 128), (1000, 69), (2100, 5)])
def test_single_sequences(heads, kv_heads, dh, L, n):
    c = Call(np.random.default_rng(31 * L + n + dh), [L], [n], heads, kv_heads, dh, wide=8 * (n % 2))
    c.check()
    assert list(c.status) == [0]


@pytest.mark.parametrize("seed", range(8))
def test_packed_sequences_of_any_lengths(seed):
    rng = np.random.default_rng(700 + seed)
    B = int(rng.integers(2, 9))
    kv_heads, group, dh = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 8])), int(rng.choice([64, 128]))
    lens = [int(rng.choice([0, 1, 31, 32, 33, 500, 1500])) if rng.random() < 0.5 else int(rng.integers(0, 900)) for _ in range(B)]
    sizes = [int(rng.choice([0, 1, 2, 31, 32, 33, 64, 65, 128])) for _ in range(B)]
    sizes[0] = max(sizes[0], 1)
    Call(rng, lens, sizes, kv_heads * group, kv_heads, dh, behind=int(rng.integers(0, 3))).check()


def test_many_sequences_of_one_token():
    rng = np.random.default_rng(1)
    lens = rng.integers(0, 200, 150)
    lens[70] = 3000  # far longer than the others
    Call(rng, lens, [1] * 150, 2, 1, 64).check()


def test_long_sequence_is_split_and_merged():
    rng = np.random.default_rng(2)
    Call(rng, [20000, 40], [3, 70], 2, 1, 128).check()


@pytest.mark.parametrize("tree", ["chain", "star"])
def test_chains_and_stars(tree):
    n = 128
    parent = np.arange(n) - 1 if tree == "chain" else np.array([-1] + [0] * (n - 1))
    Call(np.random.default_rng(3), [77], [n], 2, 1, 128, parents=[parent]).check()


def test_a_range_that_goes_down_leaves_the_others():
    rng = np.random.default_rng(4)
    c = Call(rng, [50, 90], [20, 30], 4, 2, 64)
    want = c.check()
    args = list(c.device())
    args[8] = i32([20, 50, 20])  # the second range goes down: only the first sequence is one
    b.tree_attention_q8(*args)
    torch.cuda.synchronize()
    assert list(args[-1].cpu().numpy()) == [0, 1] and np.isfinite(want).all()


def test_scores_far_from_zero():
    # scores beyond any finite stand-in for "not visible", and rows whose weights all underflow but one
    rng = np.random.default_rng(5)
    c = Call(rng, [40], [10], 2, 1, 64, exps=(40, 41))
    c.cache.scale["v"][:] = 1.0
    c.q = (c.q.float() * 2.0 ** 70).bfloat16()
    got = c.run()
    keys = np.concatenate([c.cache.values("k", 0)[0], c.kr[:, 0].float().numpy()])
    vals = np.concatenate([c.cache.values("v", 0)[0], c.vr[:, 0].float().numpy()])
    see = np.concatenate([np.ones((10, 40), bool), S.on_path(c.parents[0])], 1)
    for i in range(10):
        for h in range(2):
            score = np.where(see[i], keys @ c.q[i, h].float().numpy().astype(np.float64), -np.inf)
            v = vals[score.argmax()]
            assert np.abs(got[i, h] - v).max() <= HALF * np.abs(v).max()
    c = Call(rng, [40], [6], 1, 1, 64, scale=1e30)
    c.q = -c.q.abs()
    c.cache.pool["k"][:] &= 127  # every score below -1e30
    c.kr = c.kr.abs()
    assert np.isfinite(c.run()).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n", [7, 40, 100])
def test_what_is_not_finite_stays_with_those_who_see_it(value, n):
    rng = np.random.default_rng(6)
    c = Call(rng, [45], [n], 4, 2, 64, parents=[np.array([-1] + [0] * (n - 1))])
    clean = c.check()
    j = n - 2  # seen by itself alone
    c.kr[j, 0, 3] = value
    c.vr[j, 1, 5] = value
    got = c.run()
    others = [i for i in range(n) if i != j]
    assert np.array_equal(got[others], clean[others])
    if value == value:  # K/V head 1 belongs to query heads 2, 3
        assert (got[j, 2:, 5] == value).all()
    else:
        assert np.isnan(got[j, 2:, 5]).all() and np.isnan(got[j, :2]).all()
    keep = [d for d in range(64) if d != 5]
    assert np.array_equal(got[j, 2:][:, keep], clean[j, 2:][:, keep])
    c.vr[0, 0, 9] = value  # the root: all see it
    assert not np.isfinite(c.run()[:, 0, 9]).any()


def test_unused_slots_may_hold_anything():
    rng = np.random.default_rng(7)
    c = Call(rng, [33], [4], 2, 1, 128)
    a = c.check()
    for code in (NAN_CODE, 255, 126, 0):
        for w in "kv":
            page = c.cache.pool[w][:, :, c.cache.table[0, 1]]
            page[..., S.offsets(128, w)[1:]] = code
            c.cache.pool[w][:, :, c.cache.table[0, 1]] = page
        assert np.array_equal(c.run(), a)


def test_sequences_may_share_pages():
    rng = np.random.default_rng(8)
    c = Call(rng, [64, 90], [3, 5], 2, 1, 64)
    c.cache.table[1, :2] = c.cache.table[0, :2]
    c.check()


@pytest.mark.parametrize("what", ["tree", "self parent", "root", "long tree", "long prefix", "negative prefix", "rows", "pages"])
def test_malformed_sequences(what):
    rng = np.random.default_rng(9)
    sizes = [5, 140, 9] if what == "long tree" else [5, 20, 9]
    c = Call(rng, [70, 100, 40], sizes, 4, 2, 64, parents=[np.arange(n) - 1 for n in sizes])
    zero = True
    if what == "tree":
        c.parents[1][3] = 4
    elif what == "self parent":
        c.parents[1][3] = 3
    elif what == "root":
        c.parents[1][0] = 0
    elif what == "long prefix":
        c.cache.lens[1] = 1 << 21
    elif what == "negative prefix":
        c.cache.lens[1] = -1
    elif what == "rows":
        c.off, zero = np.array([0, 5, 25, 35]), False
    elif what == "pages":
        c.cache.table[1, 2], zero = c.cache.n_blocks, None
    got = c.run()
    bad = 2 if what == "rows" else 1
    assert list(c.status) == [int(s == bad) for s in range(3)]
    rows = got[c.off[bad]:c.off[bad + 1]]
    assert (rows == 0).all() if zero else np.isnan(rows).all() if zero is None else (rows == 5.0).all()
    c.check(got, skip=(bad,))


def test_malformed_long_sequences_among_split_ones():
    rng = np.random.default_rng(10)
    c = Call(rng, [9000, 9000, 9000], [4, 4, 4], 2, 1, 64)
    c.parents[1][2] = 7
    c.cache.table[2, 200] = -5
    got = c.run()
    assert list(c.status) == [0, 1, 1]
    assert (got[4:8] == 0).all() and np.isnan(got[8:]).all()
    c.check(got, skip=(1, 2))


def test_captured_and_replayed_with_other_lengths():
    rng = np.random.default_rng(11)
    c = Call(rng, [3000, 700], [30, 40], 4, 2, 128)
    args = c.device()
    b.tree_attention_q8(*args)
    torch.cuda.synchronize()
    want = args[-2].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.tree_attention_q8(*args)
    shorter = i32([1000, 0])
    for _ in range(3):
        keep = args[10].clone()
        args[10].copy_(shorter)
        g.replay()
        torch.cuda.synchronize()
        other = args[-2].clone()
        b.tree_attention_q8(*args)
        torch.cuda.synchronize()
        assert torch.equal(other, args[-2]) and not torch.equal(other, want)
        args[10].copy_(keep)
        args[-2].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(args[-2], want)


def test_two_streams_with_workspaces_of_their_own():
    rng = np.random.default_rng(12)
    calls = [Call(rng, [4000], [20], 4, 2, 128), Call(rng, [2500, 100], [7, 64], 4, 1, 64)]
    args = [c.device() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(3):
        for st, a in zip(streams, args):
            with torch.cuda.stream(st):
                b.tree_attention_q8(*a)
    torch.cuda.synchronize()
    for c, a in zip(calls, args):
        c.check(a[-2].float().cpu().numpy())
