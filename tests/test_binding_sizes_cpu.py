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
    "kv_block_tables": (dict(block_table=i(B, PAGES), held=i(B), prefix_len=i(B), node_off=i(B + 1), T=T, free_list=i(9), free_count=i(1),
                             held_out=i(B), free_count_out=i(1), row_slot=i(T), status_dev=i(B)),
                        dict(block_table=B * PAGES, held=B, prefix_len=B, node_off=B + 1, free_list=9, free_count=1, held_out=B,
                             free_count_out=1, row_slot=T, status_dev=B)),
    "kv_append_q8": (dict(**cache(2), k_rows=rows(2), v_rows=rows(2), path=i(B * 128), accept_len=i(B), node_off=i(B + 1),
                          block_table=i(B, PAGES), prefix_len=i(B), new_len=i(B), status_dev=i(B)),
                     dict(path=B * 128, accept_len=B, node_off=B + 1, block_table=B * PAGES, prefix_len=B, new_len=B, status_dev=B)),
    "tree_attention_q8": (dict(q_rows=rows(), **cache(), k_rows=rows(), v_rows=rows(), parent=i(T), node_off=i(B + 1),
                               block_table=i(B, PAGES), prefix_len=i(B), max_prefix=100, scale=0.1, workspace=i(64), out=rows(),
                               status_dev=i(B)),
                          dict(parent=T, node_off=B + 1, block_table=B * PAGES, prefix_len=B, status_dev=B)),
    "tree_logits": (dict(logits=torch.zeros(T, V), tok=i(T), parent=i(T), node_off=i(B + 1), ctx=i(20), ctx_off=i(B + 1), gen_start=i(B),
                         penalties=torch.ones(3 * B), bias_tok=i(7), bias_val=torch.zeros(7), bias_off=i(B + 1), allowed=None,
                         logits_out=None, argmax_out=i(T), workspace=i(64), status_dev=i(B)),
                    dict(tok=T, parent=T, node_off=B + 1, ctx_off=B + 1, gen_start=B, penalties=3 * B, bias_off=B + 1, argmax_out=T,
                         status_dev=B)),
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
    if len(shape) == 1 and what != "free_list" and (what != "node_off" or "block_table" in args):  # (else they are as many as these say)
        assert "smaller" in refused(name, **{what: t[:-1].contiguous()})


def test_parts_that_are_left_out_or_not_looked_at_are_not_measured():
    assert "device tensor" in refused("kv_append_q8", path=None, accept_len=None)
    assert "device tensor" in refused("kv_block_tables", T=0, row_slot=None)
    assert "device tensor" in refused("rotary_rows", parent=None)
    none = dict.fromkeys(("ctx", "ctx_off", "gen_start", "penalties", "bias_tok", "bias_val", "bias_off"))
    assert "device tensor" in refused("tree_logits", **none)
    assert "device tensor" in refused("tree_logits", **{**none, "tok": i(1)})
    assert "device tensor" in refused("tree_logits", penalties=None, ctx_off=i(1), gen_start=i(1))


def test_texts_and_biases_count_as_many_words_as_they_have_bytes_for(monkeypatch):
    given = []

    class Library:
        def tree_logits(self, *args):
            given.append((args[8], args[14]))
            return 0

    monkeypatch.setattr(b, "lib", Library)
    monkeypatch.setattr(b, "_ptr", lambda t: None)
    monkeypatch.setattr(b, "_stream", lambda: None)
    args = CALLS["tree_logits"][0]
    for change, want in ((dict(), (20, 7)), (dict(ctx=i(20).to(torch.int16)), (10, 7)), (dict(ctx=i(20).to(torch.int64)), (20, 7)),
                         (dict(bias_tok=i(7).to(torch.int16)), (20, 3)), (dict(bias_val=torch.zeros(7).bfloat16()), (20, 3)),
                         (dict(bias_val=torch.zeros(5)), (20, 5)), (dict(ctx=None, bias_tok=None, bias_val=None, bias_off=None), (0, 0))):
        b.tree_logits(*{**args, **change}.values())
        assert given.pop() == want
