"""Buffers that are too small or of another type for what the shapes say are refused before anything is
launched: the kernels would go past their ends."""
import pytest
import torch

from gpu_util import DEV, i32
from paper_2406_17404_amd import binding as b
from serve_util import ints

pytestmark = pytest.mark.gpu
LAYERS, HEADS, PAGES, DH, T = 2, 2, 3, 64, 4


def buffers(layers=(LAYERS,)):
    pools = [torch.zeros(*layers, HEADS, PAGES, 32 * DH, dtype=torch.uint8, device=DEV) for _ in "kv"]
    scales = [torch.ones(*layers, HEADS, PAGES, device=DEV) for _ in "kv"]
    rows = [torch.zeros(*layers, T, HEADS, DH, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    return pools + scales + rows


BAD = {  # which buffer, and what is there instead
    "scales of one layer": (2, lambda t: t[0]), "V scales of one layer": (3, lambda t: t[0]), "16-bit scales": (2, lambda t: t.bfloat16()),
    "V scales of fewer pages": (3, lambda t: t[..., :2].contiguous()), "a pool of one layer": (0, lambda t: t[0].clone()),
    "a V pool of one layer": (1, lambda t: t[0].clone()), "a 16-bit pool": (0, lambda t: t.bfloat16()),
    "rows of other heads": (4, lambda t: t[:, :, :1].contiguous())}


@pytest.mark.parametrize("what", [None, *BAD])
def test_append(what):
    x = buffers()
    if what:
        at, change = BAD[what]
        x[at] = change(x[at])
        if at == 4:
            x[5] = change(x[5])
    call = lambda: b.kv_append_q8(*x, None, None, i32([0, T]), i32([[0]]), i32([5]), ints(1), ints(1))  # noqa: E731
    if what:
        with pytest.raises(ValueError):
            call()
    else:
        call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("what", [None, "16-bit scales", "V scales of fewer pages", "a 16-bit pool", "out"])
def test_attention(what):
    x = buffers(())
    if what in BAD:
        at, change = BAD[what]
        x[at] = change(x[at])
    q = torch.zeros(T, 4, DH, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(T - (what == "out"), 4, DH, dtype=torch.bfloat16, device=DEV)
    ws = torch.zeros(b.tree_attention_q8_workspace_bytes(1, T, 4, HEADS, DH, 5), dtype=torch.uint8, device=DEV)
    call = lambda: b.tree_attention_q8(q, *x, i32([-1, 0, 0, 1]), i32([0, T]), i32([[0]]), i32([5]), 5, 0.1, ws, out, ints(1))  # noqa: E731
    if what:
        with pytest.raises(ValueError):
            call()
    else:
        call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("what", [None, "16-bit logits", "fewer rows out", "16-bit out", "fewer words", "bytes"])
def test_logits(what):
    V = 70
    x = torch.zeros(T, V, device=DEV)
    out, allowed = torch.zeros_like(x), torch.full((T, 3), -1, dtype=torch.int32, device=DEV)
    if what == "16-bit logits":
        x = x.bfloat16()
    elif what == "fewer rows out":
        out = out[:3]
    elif what == "16-bit out":
        out = out.bfloat16()
    elif what == "fewer words":
        allowed = allowed[:, :2].contiguous()
    elif what == "bytes":
        allowed = allowed.bool()
    ws = torch.zeros(b.tree_logits_workspace_bytes(1, T, V), dtype=torch.uint8, device=DEV)
    call = lambda: b.tree_logits(x, ints(T), i32([-1, 0, 0, 1]), i32([0, T]), *[None] * 7, allowed, out, ints(T), ws, ints(1))  # noqa: E731
    if what:
        with pytest.raises(ValueError):
            call()
    else:
        call()
    torch.cuda.synchronize()
