"""Calls of the paged 8-bit cache and the logits that the host refuses: the status comes before
anything is enqueued, so no GPU is needed and the pointers are never followed."""
import ctypes

import pytest
import torch

from paper_2406_17404_amd import binding as b

NULL, SHAPE, DTYPE, TREE, WS = -1, -2, -3, -4, -5
P = 1 << 20  # an aligned address


def call(name, order, base, **change):
    return getattr(b.lib(), name)(*[{**base, **change}[k] for k in order], None)


TABLES = dict(block_table=P, max_blocks=8, held=P, prefix=P, off=P, B=4, T=9, free=P, n_blocks=64, count=P,
              held_out=2 * P, count_out=2 * P, slot=P, status=P)


@pytest.mark.parametrize("change,status", [
    (dict(held=None), NULL), (dict(slot=None), NULL), (dict(free=None), NULL), (dict(status=None), NULL),
    (dict(B=0), SHAPE), (dict(B=4097), SHAPE), (dict(T=-1), SHAPE), (dict(max_blocks=0), SHAPE), (dict(n_blocks=0), SHAPE),
    (dict(n_blocks=1 << 27), SHAPE), (dict(B=4096, max_blocks=1 << 20), SHAPE), (dict(held_out=P), SHAPE),
    (dict(held_out=P + 12), SHAPE), (dict(held_out=P - 12), SHAPE), (dict(count_out=P), SHAPE)])
def test_tables(change, status):
    assert call("kv_block_tables", list(TABLES), TABLES, **change) == status


APPEND = dict(k=P, v=P, ks=P, vs=P, kr=P, vr=P, stride=1024, layer=1 << 20, path=None, acc=None, off=P, table=P, max_blocks=8,
              prefix=P, B=4, T=9, layers=2, heads=8, dh=128, n_blocks=64, dtype=b.BF16, new_len=2 * P, status=P)


@pytest.mark.parametrize("change,status", [
    (dict(k=None), NULL), (dict(vr=None), NULL), (dict(new_len=None), NULL), (dict(path=P), NULL),
    (dict(dtype=b.F32), DTYPE), (dict(dtype=9), DTYPE), (dict(dh=96), SHAPE), (dict(dh=32), SHAPE), (dict(T=0), SHAPE),
    (dict(layers=0), SHAPE), (dict(layers=40000), SHAPE), (dict(heads=0), SHAPE), (dict(heads=70000), SHAPE),
    (dict(stride=1016), SHAPE), (dict(stride=1028), SHAPE), (dict(layer=4), SHAPE), (dict(kr=P + 8), SHAPE),
    (dict(v=P + 2), SHAPE), (dict(n_blocks=0), SHAPE), (dict(B=5000), SHAPE), (dict(max_blocks=0), SHAPE),
    (dict(new_len=P), SHAPE), (dict(new_len=P + 12), SHAPE), (dict(new_len=P - 12), SHAPE)])
def test_append(change, status):
    assert call("kv_append_q8", list(APPEND), APPEND, **change) == status


ATTN = dict(q=P, q_stride=4096, k=P, v=P, ks=P, vs=P, kr=P, vr=P, stride=1024, parent=P, off=P, table=P, max_blocks=8, prefix=P,
            B=4, T=9, H=32, Hk=8, dh=128, n_blocks=64, most=200, dtype=b.BF16, scale=0.1, ws=P, ws_bytes=1 << 30, out=P,
            status=P)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), NULL), (dict(ws=None), NULL), (dict(status=None), NULL), (dict(parent=None), NULL),
    (dict(dtype=b.F32), DTYPE), (dict(H=30), SHAPE), (dict(Hk=0), SHAPE), (dict(dh=256), SHAPE), (dict(T=0), SHAPE),
    (dict(T=513), TREE), (dict(B=0), SHAPE), (dict(B=4097), SHAPE), (dict(most=-1), SHAPE), (dict(scale=0.0), SHAPE),
    (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
    (dict(q_stride=4088), SHAPE), (dict(q_stride=4100), SHAPE), (dict(stride=1000), SHAPE), (dict(q=P + 4), SHAPE),
    (dict(out=P + 8), SHAPE), (dict(n_blocks=-3), SHAPE), (dict(ws_bytes=0, ws=P + 4, most=1 << 20), WS),
    (dict(ws_bytes=1 << 10, most=1 << 20), WS)])
def test_attention(change, status):
    assert call("tree_attention_q8", list(ATTN), ATTN, **change) == status


LOGITS = dict(x=P, tok=P, parent=P, off=P, B=4, T=9, V=32000, ctx=P, n_ctx=7, ctx_off=P, gen=P, pen=P, bt=P, bv=P, n_bias=3,
              bo=P, allowed=P, out=P, argmax=P, ws=P, ws_bytes=1 << 20, status=P)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), NULL), (dict(tok=None), NULL), (dict(ctx_off=None), NULL), (dict(gen=None), NULL), (dict(bv=None), NULL),
    (dict(out=None, argmax=None), NULL), (dict(ws=None), NULL), (dict(status=None), NULL), (dict(V=0), SHAPE),
    (dict(V=1 << 25), SHAPE), (dict(T=0), SHAPE), (dict(T=513), TREE), (dict(n_ctx=-1), SHAPE), (dict(n_bias=-1), SHAPE),
    (dict(n_ctx=(1 << 30) + 1), SHAPE), (dict(n_bias=(1 << 30) + 1), SHAPE),
    (dict(B=4097, T=4097), SHAPE), (dict(ws_bytes=8), WS)])
def test_logits(change, status):
    assert call("tree_logits", list(LOGITS), LOGITS, **change) == status


def test_workspace_queries():
    n = ctypes.c_size_t(0)
    assert b.lib().tree_attention_q8_workspace_bytes(1, 64, 32, 32, 128, 4096, None) == NULL
    assert b.lib().tree_attention_q8_workspace_bytes(1, 64, 32, 5, 128, 4096, ctypes.byref(n)) == SHAPE
    assert b.lib().tree_attention_q8_workspace_bytes(1, 129, 32, 8, 128, 4096, ctypes.byref(n)) == TREE
    assert b.lib().tree_logits_workspace_bytes(1, 1, 0, ctypes.byref(n)) == SHAPE
    # bounded whatever the length
    assert b.tree_attention_q8_workspace_bytes(1, 64, 32, 32, 128, 1 << 24) <= 64 << 20
    assert b.tree_attention_q8_workspace_bytes(64, 64, 32, 8, 128, 1 << 20) <= 64 << 20
    assert b.tree_logits_workspace_bytes(16, 1024, 128256) <= 4 << 20


def test_binding_refuses_what_is_not_laid_out_as_stated():
    cpu = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        b._rows(cpu)
    with pytest.raises(ValueError, match="device tensor"):
        b.kv_block_tables(torch.zeros(2, 3, dtype=torch.int32), *[cpu] * 3, 1, cpu, *[cpu] * 5)
