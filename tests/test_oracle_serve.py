"""Pins of the serving oracle that do not repeat its formulas: torch's own 8-bit type, the 16-bit
oracle's attention, token-by-token counting, and page accounting."""
import numpy as np
import pytest
import torch

from oracle import tr_oracle as O
from oracle import tr_serve as S
from paper_2406_17404_amd import inputs as I


def test_codes_are_those_of_the_library_type():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(S.E4M3, want, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * 2.0 ** rng.integers(-12, 8, 4000), (want[:126] + want[1:127]) / 2,
                        [0.0, -0.0, 448.0, -448.0, np.nan, np.inf]]).clip(-448, 448)
    x[-1] = np.inf
    got = S.encode(x)
    lib = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    keep = np.isfinite(x) & (x.astype(np.float32) == x)
    assert keep.sum() > 100 and np.array_equal(got[keep], lib[keep])
    assert (got[~np.isfinite(x)] == 127).all()


@pytest.mark.parametrize("top,e", [(448.0, 0), (449.0, 1), (1.75, -8), (1.7578125, -7), (1.0, -8), (0.0, -100), (1e-38, -100)])
def test_scale_is_the_smallest_that_fits(top, e):
    assert S.scale_exp(top) == e


def test_page_places_are_a_permutation():
    for dh in (64, 128):
        for which in "kv":
            assert sorted(S.offsets(dh, which).ravel()) == list(range(32 * dh))


def test_attention_equals_the_16_bit_oracle():
    q, k, v, parent = I.gen_attention_case(3, 4, 64, 50, 9, "bf16", 2)
    got, mean = S.attention(q, k[:, :50], v[:, :50], k[:, 50:].transpose(1, 0, 2), v[:, 50:].transpose(1, 0, 2), parent,
                            1 / np.sqrt(64))
    assert np.abs(got - O.tree_attention(q, k, v, parent, 50)).max() < 1e-12
    assert (mean >= np.abs(got) - 1e-12).all()


def test_append_holds_rows_to_half_a_step_and_keeps_the_rest():
    rng = np.random.default_rng(1)
    pool = rng.integers(0, 255, (1, 2, 6, 32 * 64)).astype(np.uint8)
    scale = np.full((1, 2, 6), 2.0 ** -7, np.float32)
    pools, scales = [pool.copy(), pool.copy()], [scale.copy(), scale.copy()]
    rows = rng.normal(size=(2, 1, 50, 2, 64)).astype(np.float32)
    table = np.array([[4, 1, 0], [2, 5, 3]])
    new_len, status = S.append(*pools, *scales, *rows, None, None, [0, 40, 50], table, [20, 0])
    assert list(new_len) == [60, 10] and not status.any()
    for which, p, s, x in zip("kv", pools, scales, rows):
        val = S.page_values(p, s, which)
        flat = np.concatenate([val[:, :, 4], val[:, :, 1]], 2)[0, :, 20:60]
        assert np.abs(flat - x[0, :40].transpose(1, 0, 2)).max() <= np.abs(x).max() * 2.0 ** -4
        for page, rest in ((1, slice(28, 32)), (2, slice(10, 32)), (3, slice(0, 32))):
            assert np.array_equal(p[:, :, page][..., S.offsets(64, which)[rest]], pool[:, :, page][..., S.offsets(64, which)[rest]])


def test_pages_are_handed_out_once():
    rng = np.random.default_rng(2)
    n_blocks, B, width = 64, 12, 10
    table, held = np.full((B, width), -1), np.zeros(B, int)
    free, count = rng.permutation(n_blocks), n_blocks
    for step in range(40):
        prefix, rows = rng.integers(0, 260, B), rng.integers(0, 40, B)
        off = np.concatenate([[0], np.cumsum(rows)])
        table, held, free, count, slot, status = S.block_tables(table, held, prefix, off, int(off[-1]), free, count, n_blocks)
        owned = [p for s in range(B) for p in table[s, :held[s]]]
        assert sorted(owned + list(free[:count])) == list(range(n_blocks))
        for s in range(B):
            if status[s] == 0:
                assert held[s] == -(-(prefix[s] + rows[s]) // 32)


def test_logits_equal_decoding_token_by_token():
    rng = np.random.default_rng(3)
    V, parent, tok = 40, np.array([-1, 0, 1, 1, 0]), np.array([7, 3, 3, 9, 3])
    x, ctx = rng.normal(size=(5, V)), [3, 8, 8, 7]
    y, best = S.tree_logits(x, tok, parent, ctx, 2, (1.3, 0.2, 0.4), [(5, 9.0), (5, 1.0), (99, 1.0)], None)
    for i, text in ((0, []), (1, [3]), (2, [3, 3]), (3, [3, 9]), (4, [3])):
        whole = ctx + text
        for v in range(V):
            z = x[i, v]
            if v in whole:
                z = z / 1.3 if z > 0 else z * 1.3
            c = whole[2:].count(v)
            z = z - 0.2 * c - (0.4 if c else 0) + (1.0 if v == 5 else 0)
            assert abs(y[i, v] - z) < 1e-12
        assert best[i] == y[i].argmax()
