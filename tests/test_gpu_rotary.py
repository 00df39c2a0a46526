"""rotary_rows against the 64-bit oracle, element by element.

Tolerance: cosine and sine are rounded to 32 bits (half a step each, 2^-24), so is every product, and their sum:
2^-24 (2 (|x1| + |x2|) + |y|) times the magnitude, which is rounded in the same way; and the result's own
rounding, 2^-8 |y| for bf16, 2^-24 |y| for fp32 (its sum is the result).  Angles are off by less than 2^-52 of
themselves and 7e-12 (the polynomials); positions here stay below 2^31 and their angles below 2^31, so by 2^-21 where
they are largest, which is added for them."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32, to_dev
from oracle import tr_prompt as P
from paper_2406_17404_amd import binding as b
from paper_2406_17404_amd import inputs as I
from serve_util import ints, offsets_of

pytestmark = pytest.mark.gpu
KEEP = 5.0


class Call:
    def __init__(self, rng, prefix, sizes, heads, kv_heads, dh, rot, pairs, dtype=torch.bfloat16, tree=False, theta=1e4,
                 magnitude=1.0, behind=0, wide=0, scale=1.0):
        self.prefix, self.sizes, self.off = list(prefix), list(sizes), offsets_of(sizes)
        self.T, self.pairs, self.dtype, self.magnitude, self.wide = int(self.off[-1]) + behind, pairs, dtype, magnitude, wide
        self.q, self.k = (torch.from_numpy((rng.normal(size=(self.T, h, dh)) * scale).astype(np.float32)).to(dtype) for h in (heads, kv_heads))
        self.parents = [I.tree_random(n, rng) if n else np.zeros(0, int) for n in sizes] if tree else None
        self.freqs = P.rotary_freqs(rot, theta)[0]

    def rows(self, x, value):
        buf = torch.full((self.T, x.shape[1] * x.shape[2] + self.wide), value, dtype=self.dtype, device=DEV)
        part = buf[:, :x.shape[1] * x.shape[2]].unflatten(1, x.shape[1:])
        return buf, part

    def device(self, in_place=False):
        rows = [self.rows(x, float("nan")) for x in (self.q, self.k)]
        for (_, part), x in zip(rows, (self.q, self.k)):
            part.copy_(x.to(DEV))
        outs = rows if in_place else [self.rows(x, KEEP) for x in (self.q, self.k)]
        self.bufs = [o[0] for o in outs]
        parent = None
        if self.parents is not None:
            parent = np.full(self.T, 99)
            for s, p in enumerate(self.parents):
                parent[self.off[s]:self.off[s] + len(p)] = p
            parent = i32(parent)
        return [rows[0][1], rows[1][1], parent, i32(self.off), i32(self.prefix), to_dev(self.freqs), self.magnitude,
                b.ROTARY_PAIRS if self.pairs else b.ROTARY_HALVES, outs[0][1], outs[1][1], ints(len(self.sizes))]

    def run(self, in_place=False):
        args = self.device(in_place)
        b.rotary_rows(*args)
        torch.cuda.synchronize()
        self.status = list(args[-1].cpu().numpy())
        return [x.float().cpu().numpy() for x in (args[8], args[9])]

    def check(self, got=None, bad=(), in_place=False):
        got = self.run(in_place) if got is None else got
        half = 2.0 ** -8 if self.dtype == torch.bfloat16 else 2.0 ** -24
        for x, g in zip((self.q, self.k), got):
            x = x.double().numpy()
            covered = np.zeros(self.T, bool)
            for s, n in enumerate(self.sizes):
                r = slice(self.off[s], self.off[s] + n)
                if s in bad or n == 0:
                    continue
                covered[r] = True
                at = np.arange(n) if self.parents is None else P.depths(self.parents[s])
                want = P.rotary(x[r], self.prefix[s] + at, self.freqs, self.magnitude, self.pairs)
                mix = P.rotary(np.abs(x[r]), [0] * n, self.freqs, 1.0, self.pairs)
                m = len(self.freqs)
                a, z = (mix[..., 0:2 * m:2], mix[..., 1:2 * m:2]) if self.pairs else (mix[..., :m], mix[..., m:2 * m])
                both = np.zeros_like(mix)
                both[..., 0:2 * m:2] = both[..., 1:2 * m:2] = a + z
                if not self.pairs:
                    both[..., :m] = both[..., m:2 * m] = a + z
                far = 2.0 ** -21 if max(self.prefix) > 1 << 24 else 2.0 ** -37
                tol = (2.0 ** -23 + far) * abs(self.magnitude) * both * (1 + half) + (half + 2.0 ** -24) * np.abs(want)
                exact = np.arange(x.shape[-1]) >= 2 * m
                assert np.array_equal(g[r][..., exact], x[r][..., exact])
                worst = np.abs(g[r] - want) - tol
                assert (worst <= 0).all(), (s, np.argwhere(worst > 0)[:4], worst.max())
            rest = x[~covered] if in_place else KEEP
            assert (g[~covered] == rest).all()
        for buf, x in zip(self.bufs, (self.q, self.k)):  # beside the rows
            side = buf[:, x.shape[1] * x.shape[2]:].float().cpu().numpy()
            assert (np.isnan(side) if in_place else side == KEEP).all()
        return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("dh,rot", [(128, 128), (128, 64), (64, 64), (64, 32), (128, 2), (128, 126), (64, 12), (64, 20), (8, 8),
                                    (24, 16), (80, 80), (1024, 1024), (1024, 1000)])
def test_layouts_and_parts_of_heads(dtype, pairs, dh, rot):
    rng = np.random.default_rng(dh + rot)
    c = Call(rng, [1234], [5], 3, 2, dh, rot, pairs, dtype, wide=8)
    c.check()
    c.check(in_place=True)
    assert c.status == [0]


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("seed", range(4))
def test_packed_sequences(tree, seed):
    rng = np.random.default_rng(50 + seed)
    B = int(rng.integers(2, 9))
    sizes = [int(rng.choice([0, 1, 2, 31, 64, 65, 128])) for _ in range(B)]
    sizes[0] = max(sizes[0], 1)
    prefix = [int(rng.choice([0, 1, 77, 5000, 123456])) for _ in range(B)]
    c = Call(rng, prefix, sizes, 4, 2, 64, 64, bool(seed % 2), tree=tree, behind=3, magnitude=1.25)
    c.check()
    assert c.status == [0] * B


def test_many_sequences_and_many_rows():
    rng = np.random.default_rng(3)
    Call(rng, rng.integers(0, 1000, 150), [1] * 150, 2, 1, 64, 32, False).check()
    Call(rng, [9, 100], [4100, 37], 1, 1, 16, 16, True).check()  # several rows per workgroup, an odd end
    Call(rng, [0] * 70, [59 + s % 2 for s in range(70)], 1, 1, 8, 8, False, tree=True).check()


@pytest.mark.parametrize("prefix", [1 << 20, (1 << 31) - 4])
def test_far_positions(prefix):
    Call(np.random.default_rng(4), [prefix], [4], 2, 1, 64, 64, False, torch.float32).check()


def test_chains_and_trees_that_are_chains_agree():
    rng = np.random.default_rng(5)
    c = Call(rng, [70, 3], [100, 28], 2, 2, 128, 128, False)
    got = c.run()
    c.parents = [np.arange(100) - 1, np.arange(28) - 1]
    again = c.check()
    assert all(np.array_equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("what", ["tree", "root", "long tree", "negative prefix", "too far", "rows", "descending"])
def test_malformed_sequences(what):
    rng = np.random.default_rng(6)
    sizes = [5, 140 if what == "long tree" else 20, 9]
    tree = what in ("tree", "root", "long tree")
    c = Call(rng, [70, 100, 40], sizes, 2, 1, 64, 64, False, tree=False)
    if tree:
        c.parents = [np.arange(n) - 1 for n in sizes]
    if what == "tree":
        c.parents[1][3] = 4
    elif what == "root":
        c.parents[1][0] = 0
    elif what == "negative prefix":
        c.prefix[1] = -1
    elif what == "too far":
        c.prefix[1] = (1 << 31) - 20 + 1
    args = c.device()
    if what == "rows":
        args[3] = i32([0, 5, 25, 35])
    elif what == "descending":
        args[3] = i32([0, 5, 3, 3])
    b.rotary_rows(*args)
    torch.cuda.synchronize()
    got = [x.float().cpu().numpy() for x in (args[8], args[9])]
    bad = 2 if what == "rows" else 1
    assert list(args[-1].cpu().numpy()) == [int(s == bad) for s in range(3)]
    c.check(got, bad=(1, 2) if what == "descending" else (bad,))


def test_values_that_are_not_finite_stay_in_their_pair():
    rng = np.random.default_rng(7)
    c = Call(rng, [10], [3], 2, 1, 64, 64, False)
    clean = c.run()
    c.q[1, 0, 3] = float("nan")
    got = c.run()
    hit = np.zeros(got[0].shape, bool)
    hit[1, 0, [3, 35]] = True
    assert np.isnan(got[0][hit]).all() and np.array_equal(got[0][~hit], clean[0][~hit]) and np.array_equal(got[1], clean[1])


def test_captured_replayed_and_on_another_stream():
    rng = np.random.default_rng(8)
    c = Call(rng, [3000, 700], [30, 40], 4, 2, 128, 128, False, tree=True)
    args = c.device()
    b.rotary_rows(*args)
    torch.cuda.synchronize()
    want = args[8].clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.rotary_rows(*args)
    for _ in range(3):
        args[4].copy_(i32([5, 9]))
        g.replay()
        torch.cuda.synchronize()
        other = args[8].clone()
        assert not torch.equal(other, want)
        args[4].copy_(i32(c.prefix))
        args[8].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(args[8], want)
    st = torch.cuda.Stream()
    args[8].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        b.rotary_rows(*args)
    st.synchronize()
    assert torch.equal(args[8], want)
