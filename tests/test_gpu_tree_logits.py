"""tree_logits against the oracle: with its steps in 32 bits bit for bit, with its steps in 64 bits to
the roundings of the four steps."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32, to_dev
from oracle import tr_serve as S
from paper_2406_17404_amd import binding as b
from paper_2406_17404_amd import inputs as I
from serve_util import ints, offsets_of

pytestmark = pytest.mark.gpu


def words_of(allowed):
    n, V = allowed.shape
    w = -(-V // 32)
    bits = np.zeros((n, w * 32), np.uint64)
    bits[:, :V] = allowed
    out = (bits.reshape(n, w, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32)
    return torch.from_numpy(out.view(np.int32)).to(DEV)


class Call:
    def __init__(self, rng, sizes, V, ctx_lens, pen=True, bias=0, masked=False, behind=0, ctx=True):
        B = len(sizes)
        self.V, self.off, self.T = V, offsets_of(sizes), int(sum(sizes)) + behind
        self.x = (rng.normal(size=(self.T, V)) * 3).astype(np.float32)
        few = max(1, min(V, 50))  # tokens repeat
        self.tok = rng.integers(0, few, self.T)
        self.parents = [I.tree_random(n, rng) if n else np.zeros(0, int) for n in sizes]
        self.ctx = [rng.integers(0, V if rng.random() < 0.3 else few, l) for l in ctx_lens] if ctx else [np.zeros(0, int)] * B
        self.has_ctx = ctx
        self.gen = [int(rng.integers(0, len(c) + 2)) for c in self.ctx]
        self.pen = np.stack([rng.uniform(0.8, 2, B), rng.uniform(-0.5, 1, B), rng.uniform(0, 1, B)], 1).astype(np.float32) if pen else None
        self.bias = [[(int(t), np.float32(v)) for t, v in zip(rng.integers(-2, V + 2, bias), rng.normal(size=bias) * 4)]
                     for _ in range(B)] if bias else None
        self.allowed = rng.random((self.T, V)) < rng.choice([0.02, 0.5, 0.99], (self.T, 1)) if masked else None

    def device(self, keep=True, argmax=True, in_place=False):
        flat = lambda rows: np.concatenate([np.asarray(r) for r in rows]) if rows else np.zeros(0)  # noqa: E731
        parent = np.full(self.T, 50)
        parent[:self.off[-1]] = flat(self.parents) if self.off[-1] else 0
        x = to_dev(self.x)
        bias = [None] * 3
        if self.bias is not None:
            pairs = [p for s in self.bias for p in s]
            bias = [i32([p[0] for p in pairs]), to_dev(np.array([p[1] for p in pairs], np.float32)),
                    i32(offsets_of([len(s) for s in self.bias]))]
        ctx = [None] * 3
        if self.has_ctx:
            ctx = [i32(np.concatenate([flat(self.ctx), [0]])), i32(offsets_of([len(c) for c in self.ctx])), i32(self.gen)]
        ws = torch.full((b.tree_logits_workspace_bytes(len(self.parents), self.T, self.V),), 255, dtype=torch.uint8, device=DEV)
        out = x if in_place else torch.full_like(x, 5.0) if keep else None
        return [x, i32(self.tok), i32(parent), i32(self.off), *ctx, None if self.pen is None else to_dev(self.pen), *bias,
                None if self.allowed is None else words_of(self.allowed), out, ints(self.T) if argmax else None, ws,
                ints(len(self.parents))]

    def want(self, s, dtype):
        r = slice(self.off[s], self.off[s + 1])
        return S.tree_logits(self.x[r], self.tok[r], self.parents[s], self.ctx[s], self.gen[s],
                             None if self.pen is None else self.pen[s], None if self.bias is None else self.bias[s],
                             None if self.allowed is None else self.allowed[r], dtype)

    def check(self, skip=(), **how):
        args = self.device(**how)
        b.tree_logits(*args)
        torch.cuda.synchronize()
        out, best = (None if t is None else t.cpu().numpy() for t in args[12:14])
        for s in range(len(self.parents)):
            r = slice(self.off[s], self.off[s + 1])
            if s in skip or r.start == r.stop:
                continue
            y, picks = self.want(s, np.float32)
            if out is not None:
                assert np.array_equal(out[r], y, equal_nan=True), np.argwhere(out[r] != y)[:4]
                z, _ = self.want(s, np.float64)
                # what 64 bits hold and 32 do not (the lowest logit times a repetition of 1.5) rounds to infinity:
                # compared above
                fine = np.abs(z) <= np.finfo(np.float32).max
                # a rounding of half a step for each of: penalty, product, two differences, sum
                size = 40 + np.abs(self.x[r]).astype(np.float64) * 2 + 2 * len(self.ctx[s])
                assert (np.abs(out[r][fine].astype(np.float64) - z[fine]) <= (5 * 2.0 ** -24 * size)[fine]).all()
            if best is not None:
                assert np.array_equal(best[r], picks), (s, np.argwhere(best[r] != picks)[:4])
        rest = np.ones(self.T, bool)
        rest[:self.off[-1]] = False
        if out is not None and out.base is None and not how.get("in_place"):
            assert (out[rest] == 5.0).all()
        if best is not None:
            assert (best[rest] == -7).all()
        self.status = args[-1].cpu().numpy()
        return out, best


@pytest.mark.parametrize("V", [1, 3, 32, 33, 1023, 1024, 1025, 2048, 5001, 32000])
@pytest.mark.parametrize("n,L", [(1, 1), (7, 300), (128, 33)])
def test_sizes(V, n, L):
    rng = np.random.default_rng(V + n)
    c = Call(rng, [n], V, [L], bias=9, masked=True)
    c.check()
    assert list(c.status) == [0]


@pytest.mark.parametrize("pen", [False, True])
@pytest.mark.parametrize("bias", [0, 30])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("how", [dict(), dict(keep=False), dict(argmax=False), dict(in_place=True)])
def test_parts_that_are_left_out(pen, bias, masked, how):
    rng = np.random.default_rng(3)
    Call(rng, [5, 1, 0, 40], 1500, [10, 0, 4, 700], pen, bias, masked, behind=2).check(**how)


def test_no_context():
    Call(np.random.default_rng(4), [30, 2], 4100, [0, 0], ctx=False).check()


@pytest.mark.parametrize("seed", range(4))
def test_packed_batches(seed):
    rng = np.random.default_rng(40 + seed)
    B = [3, 16, 70, 200][seed]
    sizes = rng.choice([0, 1, 5, 33, 64] if B < 70 else [0, 1, 2], B)
    sizes[0] = 1
    Call(rng, sizes, [32000, 3000, 1025, 130][seed], rng.integers(0, 500, B), bias=4, masked=True).check()


def test_long_context():
    rng = np.random.default_rng(5)
    Call(rng, [3, 2], 2500, [70000, 5]).check()


def test_ties_take_the_lowest_token_and_nan_never_wins():
    rng = np.random.default_rng(6)
    c = Call(rng, [6], 3000, [4], pen=False)
    c.x[:] = -1.0
    c.x[0, [7, 2999]] = 2.0
    c.x[1, 5], c.x[1, 1400] = np.nan, 0.5
    c.x[2] = np.nan
    c.x[3] = -np.inf
    c.x[4, 2000], c.x[4, 2500] = -0.0, 0.0
    c.x[5, 100] = np.inf
    _, best = c.check()
    assert list(best) == [7, 1400, 0, 0, 2000, 100]


def test_masks_that_leave_little_or_nothing():
    rng = np.random.default_rng(7)
    c = Call(rng, [5], 2100, [20], masked=True)
    c.allowed[:] = False
    c.allowed[1, 2099] = True
    c.allowed[2, [40, 1500]] = True
    c.x[2, 40], c.x[2, 1500] = np.nan, -np.inf  # a number, if only minus infinity, before NaN
    c.allowed[3, [11, 12]] = True
    c.x[3, [11, 12]] = np.nan
    c.allowed[4], c.x[4] = True, np.finfo(np.float32).min
    out, best = c.check()
    assert best[0] == -1 and best[1] == 2099 and best[2] == 1500 and best[3] == 11 and np.isneginf(out[0]).all()


def test_repeated_and_foreign_tokens():
    rng = np.random.default_rng(8)
    c = Call(rng, [12], 1100, [60])
    c.tok[1:4] = c.tok[0]  # drafts that repeat
    c.parents = [np.arange(12) - 1]
    c.tok[5:8] = [-1, 1100, 2 ** 31 - 1]
    c.ctx[0][:6] = [-1, 1100, -2 ** 31, 2 ** 31 - 1, 1030, 1030]
    c.gen = [0]
    c.bias = [[(1030, 1.0), (1030, 2.0), (3, 5.0), (1030, -3.0), (1099, 1.0)]]
    c.check()


@pytest.mark.parametrize("rep", [1.5, 1.0, 2.0 ** -30, 2.0 ** 30, 1e-12, 1e12, 0.0, float("inf")])
@pytest.mark.parametrize("masked", [False, True])
def test_quotients_of_numbers_of_any_size(rep, masked):
    """Seen tokens from the smallest subnormal to infinity: bit for bit what a division gives."""
    rng = np.random.default_rng(11)
    c = Call(rng, [9, 3], 1100, [200, 5], masked=masked)
    seen = np.unique(c.ctx[0][c.ctx[0] < 1100])
    size = np.ldexp(rng.uniform(1, 2, (9, len(seen))), rng.integers(-149, 127, (9, len(seen))))
    c.x[:9, seen] = (size * rng.choice([-1, 1], size.shape)).astype(np.float32)
    c.x[3, seen[:4]] = [0.0, -0.0, np.inf, -np.inf]
    c.x[4, seen[0]] = np.nan
    c.x[5, :] = 3.0  # nothing unusual in this row
    c.pen[:, 0] = rep
    args = c.device()
    b.tree_logits(*args)
    torch.cuda.synchronize()
    out, best = args[12].cpu().numpy(), args[13].cpu().numpy()
    with np.errstate(all="ignore"):
        for s in range(2):
            r = slice(c.off[s], c.off[s + 1])
            y, picks = c.want(s, np.float32)
            assert np.array_equal(out[r], y, equal_nan=True), np.argwhere(~((out[r] == y) | np.isnan(y)))[:4]
            assert np.array_equal(best[r], picks)


@pytest.mark.parametrize("gen", [-5, 0, 59, 60, 1000])
def test_where_generation_starts(gen):
    c = Call(np.random.default_rng(9), [4], 200, [60])
    c.gen = [gen]
    c.check()


@pytest.mark.parametrize("what", ["tree", "rows", "ctx", "ctx end", "bias", "bias end", "long"])
def test_malformed_sequences_are_left_as_they_were(what):
    rng = np.random.default_rng(10)
    c = Call(rng, [4, 140 if what == "long" else 6, 5], 1300, [9, 9, 9], bias=3)
    if what == "long":
        c.parents[1] = np.arange(140) - 1
    if what == "tree":
        c.parents[1][2] = 2
    args = c.device()
    bad = [1]
    if what == "rows":
        args[3] = i32([0, 4, 10, 16])
        bad = [2]
    for name, k, at in (("ctx", 5, [0, 9, 4, 27]), ("ctx end", 5, [0, 9, 18, 29]), ("bias", 10, [0, -1, 6, 9]),
                        ("bias end", 10, [0, 3, 10, 9])):
        if what == name:
            args[k] = i32(at)
            bad = {"ctx": [1], "ctx end": [2], "bias": [0, 1], "bias end": [1, 2]}[name]
    b.tree_logits(*args)
    torch.cuda.synchronize()
    assert [s for s in range(3) if args[-1][s]] == bad
    for s in range(3):
        r = slice(c.off[s], c.off[s + 1])
        got = args[12][r].cpu().numpy(), args[13][r].cpu().numpy()
        if s in bad:
            assert (got[0] == 5.0).all() and (got[1] == -7).all()
        elif what in ("rows", "tree", "long"):
            assert np.array_equal(got[0], c.want(s, np.float32)[0])


def test_captured_and_replayed():
    c = Call(np.random.default_rng(11), [20, 64], 32000, [100, 3000], bias=10, masked=True)
    args = c.device()
    b.tree_logits(*args)
    torch.cuda.synchronize()
    want = [t.clone() for t in args[12:14]]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.tree_logits(*args)
    for _ in range(3):
        args[12].zero_(), args[13].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(args[12], want[0]) and torch.equal(args[13], want[1])
