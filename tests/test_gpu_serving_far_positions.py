"""Tables so wide that positions would pass 2^31: the last page that int32 positions reach is a page like
any other, and a sequence that would go beyond it is refused."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32
from oracle import tr_serve as S
from paper_2406_17404_amd import binding as b
from serve_util import bf16, ints

pytestmark = pytest.mark.gpu
PAGES = (2 ** 31 - 1) // 32
END = PAGES * 32  # 2^31 - 32


@pytest.fixture(scope="module")
def table():
    t = torch.zeros(1, PAGES + 8, dtype=torch.int32, device=DEV)
    t[0, PAGES - 1], t[0, PAGES:] = 2, 1
    return t


@pytest.mark.parametrize("prefix,n", [(END - 5, 5), (END - 5, 6), (END, 1), (2 ** 31 - 1, 40), (2 ** 31 - 33, 2 ** 15)])
def test_tables(table, prefix, n):
    free, held_out, count, slot, status = i32(np.arange(5)), ints(1), ints(1), ints(n), ints(1)
    before = table.clone()
    b.kv_block_tables(table, i32([PAGES if prefix + n == END else PAGES + 8]), i32([prefix]), i32([0, n]), n, free, i32([1]),
                      held_out, count, slot, status)
    torch.cuda.synchronize()
    fits = prefix + n <= END
    assert int(status) == (not fits) and torch.equal(table, before) and int(count) == 1
    assert int(held_out) == (PAGES if fits else PAGES + 8)
    assert slot.tolist() == ([2 * 32 + (prefix + j) % 32 for j in range(n)] if fits else [-1] * n)


@pytest.mark.parametrize("paths", [False, True])
@pytest.mark.parametrize("prefix,n", [(END - 5, 5), (END - 5, 6), (END, 1), (2 ** 31 - 1, 40), (2 ** 31 - 10, 20)])
def test_append(table, prefix, n, paths):
    rng = np.random.default_rng(n)
    pools = [torch.zeros(1, 3, 32 * 64, dtype=torch.uint8, device=DEV) for _ in "kv"]
    scales = [torch.ones(1, 3, device=DEV) for _ in "kv"]
    rows = [bf16(rng.normal(size=(n, 1, 64))) for _ in "kv"]
    new_len, status = ints(1), ints(1)
    path, accept = (i32(np.arange(128)[None]), i32([n - 1])) if paths else (None, None)
    b.kv_append_q8(*pools, *scales, *(r.to(DEV) for r in rows), path, accept, i32([0, n]), table, i32([prefix]), new_len, status)
    torch.cuda.synchronize()
    fits = prefix + n <= END
    assert int(status) == (not fits) and int(new_len) == (END if fits else prefix)
    for pool, scale, row, which in zip(pools, scales, rows, "kv"):
        p = pool.cpu().numpy()
        assert not p[0, :2].any()
        if not fits:
            assert not p.any() and (scale == 1).all()
            continue
        x = row.float().numpy()[:, 0]
        e = max(S.scale_exp(np.abs(x).max()), 0)  # the page's scale was 1
        assert float(scale[0, 2]) == 2.0 ** e
        assert np.array_equal(p[0, 2][S.offsets(64, which)[32 - n:]], S.encode(x / 2.0 ** e))


@pytest.mark.parametrize("prefix", [END + 1, 2 ** 31 - 1])
@pytest.mark.parametrize("dh,n", [(64, 3), (128, 40)])
def test_attention_refuses_what_is_longer(table, prefix, dh, n):
    """Beside a sequence of an ordinary length, which it leaves alone."""
    rng = np.random.default_rng(dh)
    two = torch.cat([table, table])
    two[1, :2] = i32([2, 0])
    pools = [torch.from_numpy(S.encode(rng.normal(size=(1, 3, 32 * dh)))).to(DEV) for _ in "kv"]
    scales = [torch.ones(1, 3, device=DEV) for _ in "kv"]
    q, kr, vr = (bf16(rng.normal(size=(2 * n, 1, dh))) for _ in range(3))
    parent = np.arange(n) - 1
    ws = torch.empty(b.tree_attention_q8_workspace_bytes(2, 2 * n, 1, 1, dh, 2 ** 31 - 1), dtype=torch.uint8, device=DEV)
    out, status = torch.full((2 * n, 1, dh), 5.0, dtype=torch.bfloat16, device=DEV), ints(2)
    b.tree_attention_q8(q.to(DEV), *pools, *scales, kr.to(DEV), vr.to(DEV), i32(np.tile(parent, 2)), i32([0, n, 2 * n]), two,
                        i32([prefix, 40]), 2 ** 31 - 1, dh ** -0.5, ws, out, status)
    torch.cuda.synchronize()
    assert status.tolist() == [1, 0]
    got = out.float().cpu().numpy()
    assert (got[:n] == 0).all()
    k, v = (S.page_values(p.cpu().numpy(), np.ones((1, 3), np.float32), w)[:, [2, 0]].reshape(1, 64, dh)[:, :40]
            for p, w in zip(pools, "kv"))
    f = [x[n:].float().numpy() for x in (q, kr, vr)]
    want, mean = S.attention(f[0], k, v, f[1], f[2], parent, dh ** -0.5)
    # result and weights are rounded to bf16 (half a step: 2^-8), the rest is 32-bit
    tol = 2.0 ** -8 * (np.abs(want) + mean) * (1 + 2.0 ** -8) + 2.0 ** -12 * mean
    assert (np.abs(got[n:] - want) <= tol).all()
