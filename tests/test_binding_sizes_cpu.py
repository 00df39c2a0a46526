"""Buffers of 32-bit numbers that hold fewer bytes than the sequences and rows of a call are refused before anything
is launched: the kernels would go past their ends.  On host tensors, so that buffers that are large enough are refused too, as
such, and no call is ever made."""
import pytest
import torch

from paper_2406_17404_amd import binding as b

B, T, H, DH, PAGES, V = 3, 5, 2, 64, 4, 40


def i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def rows(*lead):
    return torch.zeros(*lead, T, H, DH, dtype=torch.bfloat16)


def cache(*lead):
    codes = [torch.zeros(*lead, H, PAGES, 32 * DH, dtype=torch.uint8) for _ in "kv"]
    return dict(zip(("k_pool", "v_pool", "k_scale", "v_scale"), codes + [torch.ones(*lead, H, PAGES) for _ in "kv"]))


CALLS = {  # arguments, and how many words each named one has to hold
    "tree_sample": (dict(logits=torch.zeros(T, V), node_off=i(B + 1), rules=torch.zeros(B, 4), uniform=torch.zeros(T), token_out=i(T),
                         prob_out=None, workspace=i(64), status_dev=i(B)),
                    dict(token_out=T, node_off=B + 1, status_dev=B)),
    "rotary_rows": (dict(q_rows=rows(), k_rows=rows(), parent=i(T), node_off=i(B + 1), prefix_len=i(B),
                         freqs=torch.zeros(DH // 2, dtype=torch.float64), magnitude=1.0, layout=b.ROTARY_HALVES, q_out=rows(), k_out=rows(),
                         status_dev=i(B)),
                    dict(parent=T, node_off=B + 1, prefix_len=B, status_dev=B)),
    "chunk_attention_q8": (dict(q_rows=rows(), **cache(), k_rows=rows(), v_rows=rows(), node_off=i(B + 1), block_table=i(B, PAGES),
                                prefix_len=i(B), max_prefix=100, scale=0.1, workspace=i(64), out=rows(), status_dev=i(B)),
                           dict(node_off=B + 1, block_table=B * PAGES, prefix_len=B, status_dev=B)),
}


def refused(name, **change):
    with pytest.raises(ValueError) as e:
        getattr(b, name)(*{**CALLS[name][0], **change}.values())
    return str(e.value)


@pytest.mark.parametrize("name", CALLS)
def test_buffers_that_are_large_enough(name):
    assert "device tensor" in refused(name)


@pytest.mark.parametrize("name,what", [(n, w) for n, (_, needs) in CALLS.items() for w in needs])
def test_buffers_that_are_too_small(name, what):
    args, needs = CALLS[name]
    words, t = needs[what], args[what]
    shape = t.shape
    assert t.numel() == words
    assert "smaller" in refused(name, **{what: t.to(torch.int16)})
    assert "smaller" in refused(name, **{what: t.to(torch.int8)})
    if len(shape) == 1 and (what != "node_off" or "block_table" in args):  # (else they are as many as these say)
        assert "smaller" in refused(name, **{what: t[:-1].contiguous()})
