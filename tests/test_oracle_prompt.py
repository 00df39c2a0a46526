"""Pins of the oracle of rotary positions, chunk attention and sampling that do not repeat its formulas."""
import itertools

import numpy as np
import pytest
import torch

from oracle import tr_oracle as O
from oracle import tr_prompt as P
from oracle import tr_serve as S
from paper_2406_17404_amd import binding as b


@pytest.mark.parametrize("pairs", [False, True])
def test_rotary_is_a_complex_product_and_keeps_relative_positions(pairs):
    rng = np.random.default_rng(0)
    f, _ = P.rotary_freqs(8, 100.0)
    x, y = rng.normal(size=(2, 1, 3, 12))
    at = lambda v, p: P.rotary(v, [p], f, 1.0, pairs)  # noqa: E731
    z = x[..., 0:8:2] + 1j * x[..., 1:8:2] if pairs else x[..., :4] + 1j * x[..., 4:8]
    z = z * np.exp(1j * 5 * f)
    got = at(x, 5)
    assert np.allclose(got[..., 0:8:2] if pairs else got[..., :4], z.real, atol=1e-14)
    assert np.allclose(got[..., 1:8:2] if pairs else got[..., 4:8], z.imag, atol=1e-14)
    assert np.array_equal(got[..., 8:], x[..., 8:]) and np.array_equal(at(x, 0), x)
    dot = lambda p, q: (at(x, p) * at(y, q)).sum(-1)  # noqa: E731
    assert np.allclose(dot(3, 11), dot(1003, 1011), atol=1e-12)


def test_halves_at_full_width_are_the_step_oracles_rotation():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(5, 2, 16))
    pos = np.array([0, 3, 4, 100, 77])
    f, _ = P.rotary_freqs(16, 10000.0)
    assert np.allclose(P.rotary(x, pos, f, 1.0, False), O.rope(x, pos, 10000.0), atol=1e-12)


def test_depths_are_lengths_of_walks():
    parent = [-1, 0, 0, 1, 3, 2, 4]
    assert list(P.depths(parent)) == [0, 1, 1, 2, 3, 2, 4]


def test_frequencies():
    # hand-worked: theta = 16, four columns: 1 and 1/4
    assert np.allclose(P.rotary_freqs(4, 16.0)[0], [1, 0.25])
    assert np.allclose(P.rotary_freqs(4, 16.0, "linear", 4)[0], [0.25, 0.0625])
    # 2 pi * 8 trained tokens: 8 and 2 turns; low 1, high 3: the second pair keeps half
    trained = 50  # 7.96 and 1.99 turns
    f = P.rotary_freqs(4, 16.0, "turns", 4, 1, 3, trained)[0]
    g = (trained * 0.25 / (2 * np.pi) - 1) / 2
    assert f[0] == 1 and np.isclose(f[1], 0.0625 + g * (0.25 - 0.0625))
    ramp, mag = P.rotary_freqs(64, 10000.0, "ramp", 8, 1, 32, 4096)
    plain = P.rotary_freqs(64, 10000.0)[0]
    turns = 4096 * plain / (2 * np.pi)
    assert (ramp[turns > 40] == plain[turns > 40]).all() and np.allclose(ramp[turns < 0.7], plain[turns < 0.7] / 8)
    assert (np.diff(ramp / plain) <= 1e-12).all() and np.isclose(mag, 1 + 0.1 * np.log(8))


@pytest.mark.parametrize("scaling", ["plain", "linear", "turns", "ramp"])
@pytest.mark.parametrize("rot,theta,factor,low,high,trained", [(128, 10000.0, 8.0, 1.0, 4.0, 8192), (64, 5e5, 32.0, 1.0, 32.0, 4096),
                                                              (2, 10.0, 1.0, 0.5, 0.75, 1), (10, 1e4, 3.5, 1.0, 2.0, 100)])
def test_frequencies_of_the_library(scaling, rot, theta, factor, low, high, trained):
    code = dict(plain=b.ROTARY_PLAIN, linear=b.ROTARY_LINEAR, turns=b.ROTARY_TURNS, ramp=b.ROTARY_RAMP)[scaling]
    got, mag = b.trj_rotary_freqs(rot, theta, code, factor, low, high, trained)
    want, want_mag = P.rotary_freqs(rot, float(np.float32(theta)), scaling, float(np.float32(factor)), float(np.float32(low)), float(np.float32(high)), trained)
    assert np.allclose(got.numpy(), want, rtol=1e-13) and abs(mag - want_mag) <= 2.0 ** -24 * want_mag


def test_chunk_is_the_attention_of_a_chain():
    rng = np.random.default_rng(2)
    q, kr, vr = (rng.normal(size=(9, h, 8)) for h in (4, 2, 2))
    keys, values = rng.normal(size=(2, 2, 13, 8))
    got = P.chunk_attention(q, keys, values, kr, vr, 0.3)
    want = S.attention(q, keys, values, kr, vr, np.arange(9) - 1, 0.3)
    assert np.allclose(got, want, atol=1e-13)


def test_chunk_is_the_library_types_causal_attention():
    rng = np.random.default_rng(3)
    q, kr, vr = (torch.from_numpy(rng.normal(size=(7, 3, 8))) for _ in range(3))
    want = torch.nn.functional.scaled_dot_product_attention(*(x.transpose(0, 1) for x in (q, kr, vr)), is_causal=True, scale=0.5)
    none = np.zeros((3, 0, 8))
    got, _ = P.chunk_attention(q.numpy(), none, none, kr.numpy(), vr.numpy(), 0.5)
    assert np.allclose(got, want.transpose(0, 1).numpy(), atol=1e-12)


def test_sampling_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert P.order(x) == [1, 3, 2, 0]
    draw = lambda u, *rules: P.sample(x, rules, u)[0]  # noqa: E731
    assert [draw(u, 1, 0, 1, 0) for u in (0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91, 0.999)] == [1, 1, 3, 3, 2, 2, 0, 0]
    assert [draw(u, 1, 2, 1, 0) for u in (0, 0.56, 0.58, 0.999)] == [1, 1, 3, 3]      # 4/7, 3/7
    assert [draw(u, 1, 0, 0.65, 0) for u in (0.56, 0.58, 0.999)] == [1, 3, 3]
    assert [draw(u, 1, 0, 0.75, 0) for u in (0.999, 0.44, 0.45)] == [2, 1, 3]         # 4/9, 3/9, 2/9
    assert [draw(u, 1, 0, 1, 0.6) for u in (0.999,)] == [3] and draw(0.999, 1, 0, 1, 0.8) == 1
    assert draw(0.999, 0, 0, 1, 0) == 1 and draw(0.999, 1, 0, 0, 0) == 1 and draw(0.999, 1, 1, 1, 0) == 1
    assert P.sample(x, (1, 3, 0.9, 0.1), 0.999)[1] == pytest.approx(2 / 9)             # 0.9 of 0.9: all three
    # temperature 2: square roots
    assert P.sample(x, (2, 2, 1, 0), 0.0)[1] == pytest.approx(2 / (2 + 3 ** 0.5))


def test_sampling_of_rows_without_numbers_and_with_ties():
    inf, nan = np.inf, np.nan
    assert P.sample(np.array([-inf, nan, -inf]), (1, 0, 1, 0), 0.5) == (-1, 0.0)
    assert P.sample(np.array([-inf, nan, -3.0]), (1, 0, 1, 0), 0.5) == (2, 1.0)
    assert P.sample(np.array([0.0, inf, 1.0, inf]), (1, 0, 1, 0), 0.6) == (3, 0.5)
    flat = np.zeros(10)
    assert [P.sample(flat, (1, 0, 1, 0), u)[0] for u in (0, 0.1, 0.25, 0.999)] == [0, 1, 2, 9]
    assert [P.sample(flat, (1, 4, 1, 0), u)[0] for u in (0, 0.25, 0.999)] == [0, 1, 3]
    assert P.sample(np.array([-0.0, 0.0]), (1, 1, 1, 0), 0.9)[0] == 0


def test_shares_of_an_even_grid_of_numbers_are_the_kept_probabilities():
    rng = np.random.default_rng(4)
    x = rng.normal(size=12) * 2
    for t, k, p, m in itertools.product((0.5, 1.0), (0, 5), (1.0, 0.8), (0.0, 0.1)):
        w = np.exp(x / t) / np.exp(x / t).sum()
        by = sorted(range(12), key=lambda i: -w[i])
        keep = by[:k] if k else by
        run = np.cumsum(w[keep]) / w[keep].sum()
        keep = [v for v, before in zip(keep, np.concatenate([[0], run[:-1]])) if before < p]
        keep = [v for v in keep if w[v] >= m * w.max()]
        want = {v: w[v] / w[keep].sum() for v in keep}
        n = 4000
        got = np.bincount([P.sample(x, (t, k, p, m), (i + 0.5) / n)[0] for i in range(n)], minlength=12) / n
        assert all(abs(got[v] - want.get(v, 0)) <= 1 / n for v in range(12)), (t, k, p, m)
