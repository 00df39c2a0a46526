"""Offsets beyond 32 bits in every operator on the paged cache, and scales that are not powers of two: results
equal those of the same call on small or plain buffers, bit for bit."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, i32
from paper_2406_17404_amd import binding as b
from paper_2406_17404_amd import inputs as I
from serve_util import Paged, bf16, ints, offsets_of

pytestmark = pytest.mark.gpu


def attend(q, k, v, ks, vs, kr, vr, parent, off, table, prefix, most):
    B, T, heads, dh = table.shape[0], *q.shape
    ws = torch.empty(b.tree_attention_q8_workspace_bytes(B, T, heads, ks.shape[0], dh, most), dtype=torch.uint8, device=DEV)
    out, status = torch.zeros(T, heads, dh, dtype=torch.bfloat16, device=DEV), ints(B)
    b.tree_attention_q8(q, k, v, ks, vs, kr, vr, parent, off, table, prefix, most, dh ** -0.5, ws, out, status)
    torch.cuda.synchronize()
    assert not status.any()
    return out


def append(k, v, ks, vs, kr, vr, off, table, prefix):
    new_len, status = ints(table.shape[0]), ints(table.shape[0])
    b.kv_append_q8(k, v, ks, vs, kr, vr, None, None, off, table, prefix, new_len, status)
    torch.cuda.synchronize()
    assert not status.any()


@pytest.mark.parametrize("dh,n_blocks", [(128, 800_000), (64, 1_500_000)])
def test_pools_beyond_4_gib(dh, n_blocks):
    rng = np.random.default_rng(dh)
    heads, lens, sizes = 2, [300, 45], [20, 7]
    cache = Paged(rng, lens, heads, dh, room=40)
    d = cache.device()
    q, kr, vr = (bf16(rng.normal(size=(27, h, dh))).to(DEV) for h in (4, heads, heads))
    parent, off = i32(np.concatenate([I.tree_random(n, rng) for n in sizes])), i32(offsets_of(sizes))
    small = [d[n][0] for n in ("k", "v", "ks", "vs")]
    # the same pages at the end of pools of 6.5 and 6.1 GB
    shift = n_blocks - cache.n_blocks
    big = [torch.empty((heads, n_blocks) + t.shape[2:], dtype=t.dtype, device=DEV) for t in small]
    for x, y in zip(big, small):
        x[:, shift:] = y
    assert big[0].numel() > 2 ** 32
    far = torch.where(d["table"] >= 0, d["table"] + shift, d["table"])
    assert torch.equal(attend(q, *small, kr, vr, parent, off, d["table"], d["prefix"], 300),
                       attend(q, *big, kr, vr, parent, off, far, d["prefix"], 300))
    append(*small, kr, vr, off, d["table"], d["prefix"])
    append(*big, kr, vr, off, far, d["prefix"])
    assert all(torch.equal(x[:, shift:], y) for x, y in zip(big, small))


def test_rows_beyond_2_to_the_32_elements():
    rng = np.random.default_rng(1)
    heads, dh, lens, sizes = 2, 64, [50, 33, 100], [128, 100, 72]
    cache = Paged(rng, lens, heads, dh, room=130)
    d = cache.device()
    q, kr, vr = (bf16(rng.normal(size=(300, h, dh))).to(DEV) for h in (4, heads, heads))
    vr[299, 1, 3] = float("inf")
    wide = torch.empty(300, 1 << 24, dtype=torch.bfloat16, device=DEV)  # the longest stride, 10 GB
    far, at = [], (1 << 24) - 1024
    for x in (q, kr, vr):
        n = x.shape[1] * dh
        wide[:, at:at + n] = x.view(300, n)
        far.append(wide[:, at:at + n].unflatten(1, (x.shape[1], dh)))
        at += n
    parent, off = i32(np.concatenate([I.tree_random(n, rng) for n in sizes])), i32(offsets_of(sizes))
    pools = [d[n][0] for n in ("k", "v", "ks", "vs")]
    near = attend(q, *pools, kr, vr, parent, off, d["table"], d["prefix"], 100)
    got = attend(far[0], *pools, far[1], far[2], parent, off, d["table"], d["prefix"], 100)
    assert torch.equal(near.view(torch.int16), got.view(torch.int16)) and torch.isinf(near[299, 2:, 3]).all()
    other = [t.clone() for t in pools]
    append(*pools, kr, vr, off, d["table"], d["prefix"])
    append(*other, far[1], far[2], off, d["table"], d["prefix"])
    assert all(torch.equal(x, y) for x, y in zip(pools, other))


@pytest.mark.parametrize("masked", [False, True])
def test_logits_beyond_2_to_the_31_elements(masked):
    V, sizes = 1 << 24, [100, 30]
    T = sum(sizes)
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.randn(T, V, generator=g, device=DEV)
    rng = np.random.default_rng(3)
    parent = np.concatenate([I.tree_random(n, rng) for n in sizes])
    words = torch.randint(-2 ** 31, 2 ** 31, (T, V // 32), generator=g, device=DEV).int() if masked else None
    bias_tok = torch.tensor([V - 1, 5, V - 2], dtype=torch.int32, device=DEV)
    bias_val = torch.tensor([3.0, -2.0, 1.0], device=DEV)
    ws = torch.empty(b.tree_logits_workspace_bytes(2, T, V), dtype=torch.uint8, device=DEV)
    out, best, status = torch.empty_like(x), ints(T), ints(2)
    b.tree_logits(x, ints(T, 7), i32(parent), i32(offsets_of(sizes)), None, None, None, None, bias_tok, bias_val,
                  i32([0, 1, 3]), words, out, best, ws, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0, 0]
    bit = torch.arange(32, device=DEV)
    for t in range(T):
        y = x[t].clone()
        for tok, v in ([(V - 1, 3.0)] if t < 100 else [(5, -2.0), (V - 2, 1.0)]):
            y[tok] += v
        if masked:
            y[((words[t][:, None] >> bit) & 1).view(-1) == 0] = -float("inf")
        assert torch.equal(out[t], y), t
        assert int(best[t]) == int((y == y.max()).nonzero()[0]), t


def test_fractions_of_scales_do_not_count():
    rng = np.random.default_rng(4)
    heads, dh, lens, sizes = 2, 128, [300, 45], [20, 7]
    cache = Paged(rng, lens, heads, dh, room=40)
    q, kr, vr = (bf16(rng.normal(size=(27, h, dh))).to(DEV) for h in (4, heads, heads))
    parent, off = i32(np.concatenate([I.tree_random(n, rng) for n in sizes])), i32(offsets_of(sizes))
    plain = cache.device()
    for w in "kv":
        cache.scale[w] = (cache.scale[w] * rng.uniform(1, 1.999, cache.scale[w].shape)).astype(np.float32)
    odd = cache.device()
    outs = []
    for d in (plain, odd):
        pools = [d[n][0] for n in ("k", "v", "ks", "vs")]
        outs.append(attend(q, *pools, kr, vr, parent, off, d["table"], d["prefix"], 300))
        append(*pools, kr, vr, off, d["table"], d["prefix"])
    assert torch.equal(*outs) and all(torch.equal(plain[n], odd[n]) for n in "kv")
    for n in ("ks", "vs"):  # pages that rows went to have powers of two now
        assert torch.equal(plain[n], torch.exp2(torch.floor(torch.log2(odd[n]))))
        for s, l in enumerate(lens):
            page = int(cache.table[s, l // 32])
            assert torch.equal(plain[n][:, :, page], odd[n][:, :, page])
