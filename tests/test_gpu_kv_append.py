"""kv_append_q8 against the oracle: codes and scales are decided by exact arithmetic, so they
are equal bit for bit, and bytes that nothing is stored to are what they were."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32
from oracle import tr_serve as S
from paper_2406_17404_amd import binding as b
from serve_util import Paged, bf16, ints, offsets_of

pytestmark = pytest.mark.gpu


def check(cache, k_rows, v_rows, off, path=None, accept=None, wide=0):
    """rows [layers, T, heads, dh] bf16 tensors.  wide: elements behind every row."""
    dev = cache.device()
    want = [x.copy() for x in (cache.pool["k"], cache.pool["v"], cache.scale["k"], cache.scale["v"])]
    new_len, status = S.append(*want, k_rows.float().numpy(), v_rows.float().numpy(), path, accept, off, cache.table, cache.lens)
    layers, T, heads, dh = k_rows.shape
    rows = []
    for x in (k_rows, v_rows):
        buf = torch.full((layers, T, heads * dh + wide), 7.0, dtype=torch.bfloat16, device=DEV)
        buf[:, :, :heads * dh] = x.reshape(layers, T, -1).to(DEV)
        rows.append(buf[:, :, :heads * dh].unflatten(2, (heads, dh)))
    got_len, got_status = ints(len(cache.lens)), ints(len(cache.lens))
    args = (dev["k"], dev["v"], dev["ks"], dev["vs"], *rows, None if path is None else i32(path),
            None if accept is None else i32(accept), i32(off), dev["table"], dev["prefix"], got_len, got_status)
    for again in range(2):  # repeating it changes nothing
        b.kv_append_q8(*args)
        torch.cuda.synchronize()
        for name, g, w in zip(("k", "v", "ks", "vs"), (dev["k"], dev["v"], dev["ks"], dev["vs"]), want):
            g = g.cpu().numpy()
            assert np.array_equal(g, w), (name, again, np.argwhere(g != w)[:5])
        assert np.array_equal(got_len.cpu().numpy(), new_len) and np.array_equal(got_status.cpu().numpy(), status)
    return status


def rows_of(rng, layers, T, heads, dh, std=1.0):
    return [bf16(rng.normal(size=(layers, T, heads, dh)) * std) for _ in range(2)]


@pytest.mark.parametrize("dh,heads,layers", [(64, 1, 1), (64, 3, 2), (128, 2, 1), (128, 8, 2)])
@pytest.mark.parametrize("lens,sizes", [
    ([0], [1]), ([0], [32]), ([31], [1]), ([31], [2]), ([32], [1]), ([5], [100]), ([0, 40, 17], [33, 1, 64]),
    ([7, 64, 0, 63], [0, 3, 0, 1]), ([20], [300])])
def test_all_rows(dh, heads, layers, lens, sizes):
    rng = np.random.default_rng(dh + 10 * len(lens) + sizes[0])
    cache = Paged(rng, lens, heads, dh, layers, room=max(sizes))
    off = offsets_of(sizes)
    check(cache, *rows_of(rng, layers, int(off[-1]) + 2, heads, dh), off, wide=8 * (lens[0] % 3))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("L", [3, 8, 15, 16, 17, 20, 31])
@pytest.mark.parametrize("n,std", [(1, 100.0), (1, 0.01), (7, 30.0), (14, 1e-3)])
def test_pages_that_fill_up_while_their_scales_grow_or_stay(dh, L, n, std):
    rng = np.random.default_rng(L * 100 + n)
    cache = Paged(rng, [L, L + 32], 2, dh, room=40)
    check(cache, *rows_of(rng, 1, 2 * n, 2, dh, std), offsets_of([n, n]))


@pytest.mark.parametrize("n", [65 * 32, 520 * 32 + 7])
@pytest.mark.parametrize("bad", [None, 0, -1])
def test_long_prompts(n, bad):
    rng = np.random.default_rng(n)
    cache = Paged(rng, [20, 5], 1, 64, room=n)
    if bad is not None:  # one page that does not exist, of all that rows go to: nothing is stored
        cache.table[0, bad if bad == 0 else (20 + n - 1) // 32] = cache.n_blocks
    status = check(cache, *rows_of(rng, 1, n + 3, 1, 64), offsets_of([n, 3]))
    assert list(status) == [bad is not None, 0]


@pytest.mark.parametrize("B", [64, 65, 128, 129, 300])
def test_many_sequences(B):
    rng = np.random.default_rng(B)
    sizes = rng.choice([0, 1, 3], B)
    cache = Paged(rng, rng.choice([0, 1, 31, 40], B), 1, 64, room=4)
    check(cache, *rows_of(rng, 1, int(sum(sizes)) + 1, 1, 64), offsets_of(sizes))


@pytest.mark.parametrize("seed", range(6))
def test_accepted_paths(seed):
    rng = np.random.default_rng(50 + seed)
    B, dh, heads, layers = int(rng.integers(1, 9)), (64, 128)[seed % 2], int(rng.integers(1, 5)), int(rng.integers(1, 4))
    lens, sizes = rng.choice([0, 1, 30, 31, 32, 63, 90], B), rng.choice([1, 5, 64, 128], B)
    cache = Paged(rng, lens, heads, dh, layers, room=130)
    path, accept = np.full((B, 128), -1), np.zeros(B, int)
    for s, n in enumerate(sizes):
        accept[s] = rng.integers(0, n) if seed != 3 else n - 1
        path[s, :accept[s] + 1] = np.sort(rng.permutation(n)[:accept[s] + 1])
    off = offsets_of(sizes)
    check(cache, *rows_of(rng, layers, int(off[-1]), heads, dh), off, path, accept)


def test_more_sequences_than_a_wavefront_has_lanes():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 70, 150)
    cache = Paged(rng, lens, 2, 64, room=3)
    off = offsets_of(rng.integers(0, 4, 150))
    check(cache, *rows_of(rng, 1, int(off[-1]), 2, 64), off)


@pytest.mark.parametrize("std", [1e-38, 1e-30, 1e-3, 1.0, 300.0, 1e30])
def test_any_magnitude_grows_or_keeps_the_scale(std):
    rng = np.random.default_rng(6)
    cache = Paged(rng, [20, 33], 2, 128, room=40, exps=(-12, 12))
    check(cache, *rows_of(rng, 1, 50, 2, 128, std), offsets_of([40, 10]))


def test_ties_subnormals_zeros_and_what_is_not_finite():
    rng = np.random.default_rng(7)
    cache = Paged(rng, [3], 1, 64, room=64, exps=(-9, -8))
    k, v = rows_of(rng, 1, 64, 1, 64)
    steps = torch.arange(64, dtype=torch.float32)
    k[0, 0, 0] = (steps * 2.0 ** -11).bfloat16()  # around the smallest codes
    k[0, 1, 0] = ((16 + steps) / 16 * 0.25).bfloat16()  # ties
    k[0, 2, 0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0]).bfloat16()
    v[0, 2, 0, 5] = float("nan")
    k[0, 40:] = 0.0
    v[0, 29:61] = 0.0  # a page of zeros
    check(cache, k, v, offsets_of([64]))


@pytest.mark.parametrize("what", ["page", "negative page", "path", "accept -1", "accept n", "length", "negative length", "rows",
                                  "descending", "tree"])
def test_a_malformed_sequence_stores_nothing(what):
    rng = np.random.default_rng(8)
    cache = Paged(rng, [10, 30, 50], 2, 64, room=140)
    sizes = [5, 6, 7]
    path, accept = np.tile(np.arange(128), (3, 1)), np.array([2, 5, 0])
    off = offsets_of(sizes)
    T = 18
    if what == "page":
        cache.table[1, 0] = cache.n_blocks
    elif what == "negative page":
        cache.table[1, 0] = -1
    elif what == "path":
        path[1, 3] = 6
    elif what == "accept -1":
        accept[1] = -1
    elif what == "accept n":
        accept[1] = 6
    elif what == "length":
        cache.lens[1] = cache.width * 32 - 5
    elif what == "negative length":
        cache.lens[1] = -4
    elif what == "rows":
        off = np.array([0, 5, 11, 19])
    elif what == "descending":
        off = np.array([0, 5, 3, 18])
        accept[2] = 0
    elif what == "tree":
        off, T = np.array([0, 5, 140, 147]), 147
    status = check(cache, *rows_of(rng, 1, T, 2, 64), off, path, accept)
    assert list(status) == [0, 1, 0] or what == "rows" and list(status) == [0, 0, 1]


def test_captured_and_replayed():
    rng = np.random.default_rng(9)
    cache = Paged(rng, [31, 5], 2, 128, room=40)
    k, v = rows_of(rng, 1, 20, 2, 128)
    dev, off, new_len, status = cache.device(), i32(offsets_of([12, 8])), ints(2), ints(2)
    args = (dev["k"], dev["v"], dev["ks"], dev["vs"], k.to(DEV), v.to(DEV), None, None, off, dev["table"], dev["prefix"], new_len,
            status)
    start = {n: t.clone() for n, t in dev.items()}
    b.kv_append_q8(*args)
    torch.cuda.synchronize()
    want = {n: t.clone() for n, t in dev.items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.kv_append_q8(*args)
    for _ in range(3):
        for n, t in dev.items():
            t.copy_(start[n])
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(dev[n], want[n]) for n in dev)
