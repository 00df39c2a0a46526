"""tree_attention_q8 over tens of millions of positions (few pages, named over and over): the split of the
keys has to be one that the partial results' space holds, whatever it would cost."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32
from oracle import tr_serve as S
from paper_2406_17404_amd import binding as b
from serve_util import bf16, ints

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8


def repeated_pages(q, keys, values, times, kr, vr, scale):
    """One row over `times` of every key and its own: the result and the weights' mean of |v|."""
    k, v = np.concatenate([keys, kr[None]]), np.concatenate([values, vr[None]])
    w = np.concatenate([times, [1]]) * np.exp(scale * (k @ q))
    w /= w.sum()
    return w @ v, w @ np.abs(v)


@pytest.mark.parametrize("pages,heads", [(1_100_003, 255), (1_100_003, 40)])
def test_single_rows(pages, heads):
    rng = np.random.default_rng(heads)
    dh, n_blocks, L = 64, 3, 32 * pages - 7
    pool = {w: S.encode((rng.normal(size=(heads, n_blocks, 32 * dh)) * 60).clip(-448, 448)) for w in "kv"}
    scale = {w: np.full((heads, n_blocks), 2.0 ** -6, np.float32) for w in "kv"}
    q, kr, vr = (bf16(rng.normal(size=(1, heads, dh))) for _ in range(3))
    table = (torch.arange(pages, device=DEV) % n_blocks).int()[None]
    ws = torch.empty(b.tree_attention_q8_workspace_bytes(1, 1, heads, heads, dh, L), dtype=torch.uint8, device=DEV)
    out, status = torch.full((1, heads, dh), 5.0, dtype=torch.bfloat16, device=DEV), ints(1)
    b.tree_attention_q8(q.to(DEV), *(torch.from_numpy(pool[w]).to(DEV) for w in "kv"),
                        *(torch.from_numpy(scale[w]).to(DEV) for w in "kv"), kr.to(DEV), vr.to(DEV), i32([-1]), i32([0, 1]), table,
                        i32([L]), L, dh ** -0.5, ws, out, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0]
    # how often a page's slots occur: the last page has 25 of them
    times = np.zeros((n_blocks, 32))
    for p in range(n_blocks):
        times[p] = len(range(p, pages, n_blocks))
    times[(pages - 1) % n_blocks, 25:] -= 1
    got = out.float().cpu().numpy()[0]
    # Roundings to bf16 of weights and result, half a step each; and sums of up to pages / 8 blocks in a row in 32 bits:
    # half a step (2^-24) for each that the sum of weights adds, a whole one for each of the two products of
    # a block that the values' sums add
    long_sum = pages / 8 * (2.0 ** -24 + 2 * 2.0 ** -23)
    for h in range(heads):
        keys, values = (S.page_values(pool[w][h], scale[w][h], w).reshape(-1, dh) for w in "kv")
        f = [x[0, h].float().numpy().astype(np.float64) for x in (q, kr, vr)]
        want, mean = repeated_pages(f[0], keys, values, times.ravel(), f[1], f[2], dh ** -0.5)
        tol = HALF * (np.abs(want) + mean) * (1 + HALF) + (long_sum + 2.0 ** -12) * mean
        bad = ~(np.abs(got[h] - want) <= tol)
        assert not bad.any(), (h, np.abs(got[h] - want).max(), np.abs(want).max())
