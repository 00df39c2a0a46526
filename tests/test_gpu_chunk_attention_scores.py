"""chunk_attention_q8 where scores are far from zero, against the 64-bit oracle.

Scores here are exact in 32 bits before they are multiplied by the scale (few columns, whole numbers), so the tolerance of
test_gpu_chunk_attention.py holds without its part for scores below 64: weights that differ do so by the exact scores, and the
reference's rounding is common to all weights of a query."""
import numpy as np
import pytest

from oracle import tr_serve as S
from serve_util import bf16
from test_gpu_chunk_attention import Call

pytestmark = pytest.mark.gpu
# many heads, and a long sequence that is split, both in tiles of 256 queries; short ones in tiles of 32
SHAPES = {"many heads": ([137], [140], 140, 140, 64), "split": ([9001], [100], 16, 8, 64), "128 columns": ([137], [150], 70, 70, 128),
          "few": ([137], [20], 4, 2, 64)}


def put(c, w, columns):
    """Whole cache: pool `w` holds columns[c][page][row] in its first columns, 0 in the others, scales 1."""
    place = S.offsets(c.dh, w)
    c.cache.scale[w][:] = 1.0
    c.cache.pool[w][:] = 0
    for p, page in enumerate(c.cache.table[0, :-(-c.cache.lens[0] // 32)]):
        for col, x in enumerate(columns):
            c.cache.pool[w][:, :, page, place[:, col]] = S.encode(np.broadcast_to(x[p], (1, c.cache.heads, 32)).astype(np.float64))


def rows(x, *columns):
    y = np.zeros(tuple(x.shape), np.float32)
    for col, v in enumerate(columns):
        y[..., col] = v
    return bf16(y)


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("exp", [2, 13, 14, 15, 16, 17, 18, 19, 22, 40])
def test_equal_keys_weigh_alike(shape, sign, exp):
    # references of about 2^exp; the first page's values are 1, all others 0, so that its share is seen
    rng = np.random.default_rng(100 * exp + sign)
    c = Call(rng, *SHAPES[shape], scale=0.125)
    pages = -(-c.cache.lens[0] // 32)
    put(c, "k", [np.ones((pages, 32))])
    put(c, "v", [(np.arange(pages) == 0)[:, None] * np.ones(32)])
    c.q = rows(c.q, sign * 2.0 ** (exp + 3) / np.log2(np.e) * rng.uniform(0.5, 1, c.q.shape[:2]))
    c.kr, c.vr = rows(c.kr, 1.0), rows(c.vr, 0.0)
    got = c.check()
    assert (got[..., 0] > 0).all()


@pytest.mark.parametrize("shape", ["many heads", "split", "128 columns"])
@pytest.mark.parametrize("exp", [10, 14, 16, 18, 19])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
def test_near_keys_far_from_zero(shape, exp, order):
    # the second column's products lie 0 to 100 apart, the first's are all the same and large: in 32 bits their sum is exact
    rng = np.random.default_rng(exp)
    c = Call(rng, *SHAPES[shape], scale=0.125)
    L, pages = c.cache.lens[0], -(-c.cache.lens[0] // 32)
    steps = np.sort(S.E4M3[S.encode(rng.uniform(20, 400, pages))])
    steps = steps[::-1] if order == "falling" else rng.permutation(steps) if order == "mixed" else steps
    near = S.E4M3[S.encode(np.repeat(steps, 32).reshape(pages, 32) * rng.uniform(0.9, 1, (pages, 32)))]
    put(c, "k", [np.ones((pages, 32)), near])
    put(c, "v", [rng.normal(size=(pages, 32)) for _ in range(4)])
    n, H = c.q.shape[:2]
    c.q = rows(c.q, 2.0 ** (exp + 3) * np.floor(rng.uniform(64, 128, (n, H))) / 128, rng.integers(1, 3, (n, H)))
    c.kr = rows(c.kr, 1.0, np.floor(rng.uniform(0, 256, c.kr.shape[:2])))
    c.vr = rows(c.vr, *(rng.normal(size=c.vr.shape[:2]) for _ in range(4)))
    c.check()


@pytest.mark.parametrize("shape", ["many heads", "split", "128 columns", "few"])
@pytest.mark.parametrize("size", [1.0, 2.0 ** 12])
def test_a_query_does_not_depend_on_those_beside_it(shape, size):
    # every second row's scores become far ones, and ones that rise from page to page
    rng = np.random.default_rng(3)
    c = Call(rng, *SHAPES[shape])
    c.q = (c.q.float() * size).bfloat16()
    clean = c.run()
    for factor in (2.0 ** -30, 2.0 ** 5, 2.0 ** 11, 2.0 ** 20, 2.0 ** 60):
        q = c.q.clone()
        c.q[1::2] = (c.q[1::2].float() * factor).bfloat16()
        got = c.run()
        assert np.array_equal(got[::2], clean[::2]) and not np.array_equal(got[1::2], clean[1::2])
        c.q = q


@pytest.mark.parametrize("lens,sizes,heads,kv_heads,dh", [([40], [100], 2, 1, 64), ([40], [70], 1, 1, 64), ([40], [1], 1, 1, 64),
                                                          ([40], [10], 1, 1, 64), ([40], [129], 140, 140, 64),
                                                          ([77], [200], 140, 140, 64), ([9001], [100], 16, 8, 64),
                                                          ([130], [150], 70, 70, 128)])
@pytest.mark.parametrize("sign", [1, -1])
def test_the_largest_of_scores_beyond_1e30(lens, sizes, heads, kv_heads, dh, sign):
    # whole numbers times 1e30: the largest take all, in equal shares
    rng = np.random.default_rng(dh + sizes[0])
    c = Call(rng, lens, sizes, heads, kv_heads, dh, scale=1e30)
    c.cache.scale["k"][:] = 1.0
    c.cache.pool["k"][:] = S.encode(rng.integers(0, 5, c.cache.pool["k"].shape).astype(np.float64))
    c.q = bf16(sign * rng.integers(1, 4, c.q.shape))
    c.kr = bf16(rng.integers(0, 5, c.kr.shape))
    c.check()
