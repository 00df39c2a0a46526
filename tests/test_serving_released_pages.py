"""A sequence that gave pages back and is refused new ones must not store through the table entries it
left: those pages may be another's.  Once by the oracle's rules alone, once on the device."""
import numpy as np
import pytest
import torch

from oracle import tr_serve as S
from serve_util import bf16, ints, offsets_of

WIDTH, N_BLOCKS = 3, 4
# the second round: prefix and rows of the first sequence.  No page is left for the first; the second asks for more
# than a table row holds
SECOND = {"no pages left": (32, 4), "beyond the table": (32, 80)}


def first_round():
    """Sequence 0 shrinks from three pages to one, sequence 1 takes the two that come back."""
    table = np.array([[2, 0, 3], [1, -1, -1]])
    return table, np.array([3, 1]), np.array([28, 30]), offsets_of([4, 60]), 64, np.full(N_BLOCKS, -1), 0


def second_round(what):
    prefix, rows = SECOND[what]
    return np.array([prefix, 90]), offsets_of([rows, 0]), rows


@pytest.mark.parametrize("what", SECOND)
@pytest.mark.parametrize("paths", [False, True])
def test_rules(what, paths):
    table, held, prefix, off, T, free, count = first_round()
    table, held, free, count, _, status = S.block_tables(table, held, prefix, off, T, free, count, N_BLOCKS)
    assert list(held) == [1, 3] and not status.any()
    prefix, off, T = second_round(what)
    table, held, free, count, slot, status = S.block_tables(table, held, prefix, off, T, free, count, N_BLOCKS)
    assert list(held) == [1, 3] and list(status) == [1, 0] and (slot == -1).all()
    rng = np.random.default_rng(0)
    pools = [rng.integers(0, 120, (1, 1, N_BLOCKS, 32 * 64)).astype(np.uint8) for _ in "kv"]
    scales = [np.full((1, 1, N_BLOCKS), 2.0 ** -6, np.float32) for _ in "kv"]
    before = [x.copy() for x in pools + scales]
    rows = [rng.normal(size=(1, T, 1, 64)) for _ in "kv"]
    path, accept = (np.tile(np.arange(128), (2, 1)), np.array([3, -1])) if paths else (None, None)
    new_len, status = S.append(*pools, *scales, *rows, path, accept, off, table, prefix)
    assert status[0] == 1 and list(new_len) == [32, 90]
    assert all(np.array_equal(a, b) for a, b in zip(before, pools + scales))


@pytest.mark.gpu
@pytest.mark.parametrize("what", SECOND)
@pytest.mark.parametrize("paths", [False, True])
@pytest.mark.parametrize("dh", [64, 128])
def test_device(what, paths, dh):
    from gpu_util import DEV, i32, to_dev
    from paper_2406_17404_amd import binding as b

    table, held, prefix, off, T, free, count = first_round()
    d = dict(table=i32(table), free=i32(free), held=[i32(held), ints(2)], count=[i32([count]), ints(1)])
    slot, status = ints(80), ints(2)
    b.kv_block_tables(d["table"], d["held"][0], i32(prefix), i32(off), T, d["free"], d["count"][0], d["held"][1],
                      d["count"][1], slot, status)
    assert list(d["held"][1].cpu().numpy()) == [1, 3] and not status.any()
    prefix, off, T = second_round(what)
    for again in range(2):  # repeating it changes nothing
        b.kv_block_tables(d["table"], d["held"][1], i32(prefix), i32(off), T, d["free"], d["count"][1], d["held"][0],
                          d["count"][0], slot, status)
        assert list(d["held"][0].cpu().numpy()) == [1, 3] and list(status.cpu().numpy()) == [1, 0]
        assert (slot[:T] == -1).all()
    owned = d["table"][1].cpu().numpy()
    assert sorted(owned) == [0, 1, 3] and int(d["table"][0, 0]) == 2
    rng = np.random.default_rng(dh)
    layers, heads = 2, 2
    pools = [to_dev(rng.integers(0, 120, (layers, heads, N_BLOCKS, 32 * dh)).astype(np.uint8)) for _ in "kv"]
    scales = [torch.full((layers, heads, N_BLOCKS), 2.0 ** -6, device=DEV) for _ in "kv"]
    before = [x.clone() for x in pools + scales]
    rows = [bf16(rng.normal(size=(layers, T, heads, dh))).to(DEV) for _ in "kv"]
    path, accept = (i32(np.tile(np.arange(128), (2, 1))), i32([3, -1])) if paths else (None, None)
    new_len, status = ints(2), ints(2)
    b.kv_append_q8(*pools, *scales, *rows, path, accept, i32(off), d["table"], i32(prefix), new_len, status)
    torch.cuda.synchronize()
    assert int(status[0]) == 1 and list(new_len.cpu().numpy()) == [32, 90]
    assert all(torch.equal(x, y) for x, y in zip(before, pools + scales))


def rounds(seed, B):
    """Requests that grow, shrink, end, and now and then ask for what is malformed."""
    rng = np.random.default_rng(seed)
    width, n_blocks = 6, 3 * B
    for _ in range(8):
        rows = rng.choice([0, 1, 30, 60], B)
        prefix = rng.integers(0, width * 32 - 60, B)
        prefix = np.where(rng.random(B) < 0.1, rng.choice([-5, width * 32, 2 ** 31 - 1], B), prefix)
        off = offsets_of(rows)
        yield width, n_blocks, prefix, off, int(off[-1])


@pytest.mark.parametrize("seed,B", [(1, 1), (2, 5), (3, 70)])
def test_no_entry_of_a_refused_sequence_names_a_page_of_another(seed, B):
    """By the rules alone: whatever a refused sequence could append to is its own or nothing."""
    table, held, free, count, refused = np.full((B, 6), -1), np.zeros(B, int), np.arange(3 * B), 3 * B, 0
    for width, n_blocks, prefix, off, T in rounds(seed, B):
        table, held, free, count, _, status = S.block_tables(table, held, prefix, off, T, free, count, n_blocks)
        assert sorted([p for s in range(B) for p in table[s, :held[s]]] + list(free[:count])) == list(range(n_blocks))
        for s in np.flatnonzero(status):
            end = min(width, -(-(max(prefix[s], 0) + off[s + 1] - off[s]) // 32)) if prefix[s] >= 0 else 0
            assert (table[s, held[s]:end] == -1).all()
            refused += 1
    assert refused > 0


@pytest.mark.gpu
@pytest.mark.parametrize("seed,B", [(1, 1), (2, 5), (3, 70), (4, 300)])
def test_rounds_equal_the_rules(seed, B):
    from gpu_util import i32
    from paper_2406_17404_amd import binding as b

    table, held, free, count = np.full((B, 6), -1), np.zeros(B, int), np.arange(3 * B), 3 * B
    d = dict(table=i32(table), free=i32(free), held=[i32(held), ints(B)], count=[i32([count]), ints(1)])
    for step, (width, n_blocks, prefix, off, T) in enumerate(rounds(seed, B)):
        table, held, free, count, slot, status = S.block_tables(table, held, prefix, off, T, free, count, n_blocks)
        a, z = step % 2, 1 - step % 2
        got_slot, got_status = ints(max(T, 1)), ints(B)
        for again in range(2):
            b.kv_block_tables(d["table"], d["held"][a], i32(prefix), i32(off), T, d["free"], d["count"][a], d["held"][z],
                              d["count"][z], got_slot, got_status)
            for g, w in ((d["table"], table), (d["held"][z], held), (d["free"], free), (d["count"][z], [count]),
                         (got_slot[:T], slot), (got_status, status)):
                assert np.array_equal(g.cpu().numpy(), w), (step, again)
