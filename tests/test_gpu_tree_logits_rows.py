"""tree_logits: rows that no sequence owns stay as they were in both outputs, and NaN of either kind."""
import numpy as np
import pytest
import torch

from paper_2406_17404_amd import binding as b
from test_gpu_tree_logits import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [33, 1024, 1500, 5001])
@pytest.mark.parametrize("rules", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("argmax", [False, True])
def test_rows_behind_the_last_sequence(V, rules, in_place, argmax):
    c = Call(np.random.default_rng(V), [5, 0, 40], V, [10, 3, 700], pen=rules, bias=9 * rules, masked=rules, behind=3)
    args = c.device(in_place=in_place, argmax=argmax)
    b.tree_logits(*args)
    torch.cuda.synchronize()
    out = args[12].cpu().numpy()
    assert out.shape == (48, V)
    assert np.array_equal(out[45:], c.x[45:]) if in_place else (out[45:] == 5.0).all()
    assert not argmax or (args[13][45:] == -7).all()
    for s in (0, 2):
        rows = slice(c.off[s], c.off[s + 1])
        y, picks = c.want(s, np.float32)
        assert np.array_equal(out[rows], y) and (not argmax or np.array_equal(args[13][rows].cpu().numpy(), picks))


@pytest.mark.parametrize("bits", [0x7f800001, 0xff800001, 0x7fc00000, 0xffc00000, 0xffffffff])
@pytest.mark.parametrize("masked", [False, True])
def test_nan_of_any_kind_never_wins(bits, masked):
    c = Call(np.random.default_rng(1), [6], 2100, [4], pen=False, masked=masked)
    nan = np.array([bits], np.uint32).view(np.float32)[0]
    raw = c.x.view(np.uint32)
    raw[0, :2099] = bits  # one number among NaN
    raw[1, 1:] = bits
    raw[2, 3:700] = bits
    raw[3, ::2] = bits
    raw[4] = bits
    c.x[5] = -np.inf
    raw[5, :100] = bits
    assert np.isnan(nan)
    args = c.device()
    b.tree_logits(*args)
    torch.cuda.synchronize()
    assert np.array_equal(args[13].cpu().numpy(), c.want(0, np.float32)[1])
