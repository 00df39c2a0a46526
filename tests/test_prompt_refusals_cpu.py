"""Calls of rotary positions, chunk attention and sampling that the host refuses: the status comes before
anything is enqueued, so no GPU is needed and the pointers are never followed."""
import ctypes

import pytest
import torch

from paper_2406_17404_amd import binding as b

NULL, SHAPE, DTYPE, WS = -1, -2, -3, -5
P = 1 << 20  # an aligned address
INF, NAN = float("inf"), float("nan")


def call(name, order, base, **change):
    return getattr(b.lib(), name)(*[{**base, **change}[k] for k in order], None)


ROTARY = dict(q=P, q_stride=4096, k=P, k_stride=1024, parent=None, off=P, prefix=P, B=4, T=9, H=32, Hk=8, dh=128, rot=64,
              layout=0, freqs=P, mag=1.0, dtype=b.BF16, qo=2 * P, qo_stride=4096, ko=2 * P, ko_stride=1024, status=P)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(off=None), NULL), (dict(prefix=None), NULL), (dict(freqs=None), NULL),
    (dict(qo=None), NULL), (dict(ko=None), NULL), (dict(status=None), NULL), (dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE),
    (dict(B=0), SHAPE), (dict(B=4097), SHAPE), (dict(T=0), SHAPE), (dict(T=(1 << 20) + 1), SHAPE), (dict(H=0), SHAPE),
    (dict(Hk=0), SHAPE), (dict(Hk=65536), SHAPE), (dict(dh=132), SHAPE), (dict(dh=1032, rot=64), SHAPE), (dict(dh=0), SHAPE),
    (dict(rot=0), SHAPE), (dict(rot=63), SHAPE), (dict(rot=130), SHAPE), (dict(layout=2), SHAPE), (dict(layout=-1), SHAPE),
    (dict(mag=INF), SHAPE), (dict(mag=NAN), SHAPE), (dict(q_stride=4088), SHAPE), (dict(k_stride=1020), SHAPE),
    (dict(qo_stride=4092), SHAPE), (dict(ko_stride=1016), SHAPE), (dict(ko_stride=(1 << 24) + 8), SHAPE), (dict(q=P + 8), SHAPE),
    (dict(ko=P + 2), SHAPE), (dict(freqs=P + 4), SHAPE), (dict(qo=P, qo_stride=4104), SHAPE), (dict(ko=P, k_stride=1032), SHAPE)])
def test_rotary(change, status):
    assert call("rotary_rows", list(ROTARY), ROTARY, **change) == status


@pytest.mark.parametrize("change", [
    dict(rot=0), dict(rot=7), dict(rot=-2), dict(theta=1.0), dict(theta=INF), dict(theta=NAN), dict(scaling=-1), dict(scaling=4),
    dict(scaling=1, factor=0.5), dict(scaling=1, factor=NAN), dict(scaling=2, factor=INF), dict(scaling=2, low=0.0),
    dict(scaling=2, low=4.0), dict(scaling=3, high=NAN), dict(scaling=3, trained=0), dict(scaling=2, high=INF)])
def test_frequencies(change):
    a = {**dict(rot=64, theta=1e4, scaling=0, factor=2.0, low=1.0, high=4.0, trained=4096), **change}
    f, m = (ctypes.c_double * 32)(), ctypes.c_float(0)
    assert b.lib().trj_rotary_freqs(*a.values(), f, ctypes.byref(m)) == SHAPE
    assert b.lib().trj_rotary_freqs(64, 1e4, 0, NAN, NAN, NAN, 0, f, ctypes.byref(m)) == 0  # not read
    assert b.lib().trj_rotary_freqs(64, 1e4, 0, 1, 1, 1, 1, None, ctypes.byref(m)) == NULL
    assert b.lib().trj_rotary_freqs(64, 1e4, 0, 1, 1, 1, 1, f, None) == NULL


ATTN = dict(q=P, q_stride=4096, k=P, v=P, ks=P, vs=P, kr=P, vr=P, stride=1024, off=P, table=P, max_blocks=8, prefix=P,
            B=4, T=1000, H=32, Hk=8, dh=128, n_blocks=64, most=200, dtype=b.BF16, scale=0.1, ws=P, ws_bytes=1 << 30, out=P,
            status=P)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(vr=None), NULL), (dict(off=None), NULL), (dict(table=None), NULL),
    (dict(ws=None), NULL), (dict(out=None), NULL), (dict(status=None), NULL), (dict(dtype=b.F32), DTYPE), (dict(H=30), SHAPE),
    (dict(Hk=0), SHAPE), (dict(dh=96), SHAPE), (dict(T=0), SHAPE), (dict(T=(1 << 20) + 1), SHAPE), (dict(B=0), SHAPE),
    (dict(T=1 << 20, H=2048, q_stride=1 << 18), SHAPE), (dict(B=4097), SHAPE), (dict(most=-1), SHAPE),
    (dict(most=(1 << 31) - 1000), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=NAN), SHAPE), (dict(scale=3e38), SHAPE),
    (dict(q_stride=4088), SHAPE), (dict(stride=1000), SHAPE), (dict(stride=(1 << 24) + 8), SHAPE), (dict(q=P + 4), SHAPE),
    (dict(kr=P + 8), SHAPE), (dict(out=P + 8), SHAPE), (dict(n_blocks=0), SHAPE), (dict(n_blocks=1 << 27), SHAPE),
    (dict(max_blocks=0), SHAPE), (dict(ws_bytes=0, ws=P + 4), WS), (dict(ws_bytes=1 << 10), WS)])
def test_chunk_attention(change, status):
    assert call("chunk_attention_q8", list(ATTN), ATTN, **change) == status


SAMPLE = dict(x=P, off=P, B=4, T=9, V=32000, rules=P, u=P, token=P, prob=None, ws=P, ws_bytes=1 << 26, status=P)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), NULL), (dict(off=None), NULL), (dict(rules=None), NULL), (dict(u=None), NULL), (dict(token=None), NULL),
    (dict(ws=None), NULL), (dict(status=None), NULL), (dict(V=0), SHAPE), (dict(V=(1 << 24) + 1), SHAPE), (dict(T=0), SHAPE),
    (dict(T=(1 << 20) + 1), SHAPE), (dict(B=0), SHAPE), (dict(B=4097), SHAPE), (dict(ws_bytes=8), WS),
    (dict(ws_bytes=0, ws=P + 4), WS)])
def test_sample(change, status):
    assert call("tree_sample", list(SAMPLE), SAMPLE, **change) == status


def test_workspace_queries():
    n = ctypes.c_size_t(0)
    assert b.lib().chunk_attention_q8_workspace_bytes(1, 64, 32, 32, 128, 4096, None) == NULL
    assert b.lib().chunk_attention_q8_workspace_bytes(1, 64, 32, 5, 128, 4096, ctypes.byref(n)) == SHAPE
    assert b.lib().tree_sample_workspace_bytes(1, 1, 0, ctypes.byref(n)) == SHAPE
    assert b.lib().tree_sample_workspace_bytes(1, 1, 1, None) == NULL
    # bounded whatever the length
    assert b.chunk_attention_q8_workspace_bytes(1, 4096, 32, 32, 128, 1 << 24) <= 128 << 20
    assert b.chunk_attention_q8_workspace_bytes(4096, 1 << 20, 32, 8, 128, 1 << 20) <= 128 << 20


def test_binding_refuses_host_tensors_and_other_types():
    x, i = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    f = torch.zeros(8, dtype=torch.float64)
    with pytest.raises(ValueError, match="device tensor"):
        b.rotary_rows(x, x, None, i, i, f, 1.0, b.ROTARY_HALVES, x, x, i)
    with pytest.raises(ValueError, match="64 bits"):
        b.rotary_rows(x, x, None, i, i, f.float(), 1.0, b.ROTARY_HALVES, x, x, i)
    with pytest.raises(ValueError, match="same type"):
        b.rotary_rows(x, x, None, i, i, f, 1.0, b.ROTARY_HALVES, x.float(), x, i)
    with pytest.raises(ValueError, match="fp32"):
        b.tree_sample(torch.zeros(3, 8, dtype=torch.bfloat16), i, i, i, i, None, i, i)


@pytest.mark.parametrize("T", [1, 1000, 1 << 20])
def test_chunk_attention_takes_what_the_header_says_it_takes(T):
    n, most = ctypes.c_size_t(0), (1 << 31) - 64 - T
    small = dict(T=T, ws_bytes=8)  # (so that no call is made)
    assert call("chunk_attention_q8", list(ATTN), ATTN, most=most, **small) == WS
    assert call("chunk_attention_q8", list(ATTN), ATTN, most=most + 1, **small) == SHAPE
    sizes = b.lib().chunk_attention_q8_workspace_bytes
    assert sizes(4, T, 32, 8, 128, most, ctypes.byref(n)) == 0 and n.value > 0
    assert sizes(4, T, 32, 8, 128, most + 1, ctypes.byref(n)) == SHAPE
