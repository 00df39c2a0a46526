"""Buffers of 32-bit numbers that hold fewer bytes than the sequences and rows of a call are refused before anything
is launched: the kernels would go past their ends.  On host tensors, so that buffers that are large enough are refused too, as
such, and no call is ever made."""
import pytest
import torch

from paper_2406_17404_amd import binding as b

B, T, V = 3, 5, 40


def i(*shape):
    return torch.zeros(shape, dtype=torch.int32)


CALLS = {  # arguments, and how many words each named one has to hold
    "tree_sample": (dict(logits=torch.zeros(T, V), node_off=i(B + 1), rules=torch.zeros(B, 4), uniform=torch.zeros(T), token_out=i(T),
                         prob_out=None, workspace=i(64), status_dev=i(B)),
                    dict(token_out=T)),
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
    if len(shape) == 1 and what != "node_off":  # (the number of sequences comes from its own length)
        assert "smaller" in refused(name, **{what: t[:-1].contiguous()})
