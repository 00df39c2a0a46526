"""kv_block_tables against the oracle: whole numbers, equal in every output."""
import numpy as np
import pytest
import torch

from gpu_util import i32
from oracle import tr_serve as S
from paper_2406_17404_amd import binding as b
from serve_util import ints, offsets_of

pytestmark = pytest.mark.gpu


def run(table, held, prefix, off, T, free, count):
    """One call on device copies; returns what the oracle returns."""
    dev = dict(table=i32(table), held=i32(held), prefix=i32(prefix), off=i32(off), free=i32(free), count=i32([count]),
               held_out=ints(len(held)), count_out=ints(1), slot=ints(max(T, 1)), status=ints(len(held)))
    args = (dev["table"], dev["held"], dev["prefix"], dev["off"], T, dev["free"], dev["count"], dev["held_out"],
            dev["count_out"], dev["slot"] if T else None, dev["status"])
    b.kv_block_tables(*args)
    first = {k: v.clone() for k, v in dev.items()}
    b.kv_block_tables(*args)  # nothing it reads was overwritten
    torch.cuda.synchronize()
    assert all(torch.equal(first[k], dev[k]) for k in dev)
    return (dev["table"].cpu().numpy(), dev["held_out"].cpu().numpy(), dev["free"].cpu().numpy(), int(dev["count_out"]),
            dev["slot"].cpu().numpy()[:T], dev["status"].cpu().numpy())


def check(table, held, prefix, off, T, free, count):
    table, held, prefix, off, free = (np.asarray(x, np.int64) for x in (table, held, prefix, off, free))
    want = S.block_tables(table, held, prefix, off, T, free, count, len(free))
    got = run(table, held, prefix, off, T, free, count)
    for name, g, w in zip(("table", "held", "free", "count", "slot", "status"), got, want):
        assert np.array_equal(g, w), (name, g, w)
    return got


def state(rng, B, width, n_blocks, most):
    held = rng.integers(0, most + 1, B)
    ids, table, at = rng.permutation(n_blocks), np.full((B, width), -1), 0
    for s in range(B):
        table[s, :held[s]] = ids[at:at + held[s]]
        at += held[s]
    free = np.full(n_blocks, -1)
    free[:n_blocks - at] = ids[at:]
    return table, held, free, n_blocks - at


@pytest.mark.parametrize("B,width,most", [(1, 1, 0), (1, 5, 3), (2, 4, 4), (63, 6, 4), (64, 6, 4), (65, 9, 7), (257, 5, 4),
                                          (1024, 8, 6), (4096, 4, 3)])
@pytest.mark.parametrize("seed", range(3))
def test_random_batches(B, width, most, seed):
    rng = np.random.default_rng(100 * B + seed)
    room = [0, B, 4 * B][seed]  # from too few pages to enough
    table, held, free, count = state(rng, B, width, B * most + room + 1, most)
    rows = rng.choice([0, 1, 5, 31, 32, 33, 64], B)
    prefix = np.minimum(rng.choice([0, 1, 31, 32, 33, 63, 64, 100], B) + rng.integers(0, 3, B), width * 32 - rows).clip(0)
    off = offsets_of(rows)
    check(table, held, prefix, off, int(off[-1]) + seed, free, count)  # and rows behind the last sequence


def test_pages_released_in_a_call_are_taken_in_it():
    table = np.array([[5, 6, 7, 8], [1, -1, -1, -1], [9, 2, -1, -1]])
    got = check(table, [4, 1, 2], [30, 90, 64], [0, 1, 7, 7], 7, [3, 4, -1, -1, -1, -1, -1, -1, -1, -1], 2)
    assert got[3] == 2 + 3 - 2 and not got[5].any()


def test_no_room_stops_the_sequence_and_those_behind_that_want_more():
    table = np.full((4, 6), -1)
    got = check(table, [0, 0, 0, 0], [30, 100, 0, 30], [0, 2, 8, 8, 10], 10, [0, 1, 2, -1], 3)
    assert list(got[5]) == [0, 1, 0, 1] and list(got[1]) == [1, 0, 0, 0] and got[3] == 2


@pytest.mark.parametrize("change", [
    dict(prefix=[-1, 10, 10]), dict(off=[0, 9, 4, 8]), dict(off=[-1, 2, 4, 8]), dict(off=[0, 2, 4, 40]), dict(held=[9, 1, 1]),
    dict(held=[-2, 1, 1]), dict(prefix=[10, 1000, 10]), dict(count=-3), dict(count=99), dict(prefix=[10, 2 ** 31 - 1, 10])])
def test_what_is_wrong_with_one_sequence_leaves_the_others(change):
    base = dict(table=np.array([[0, -1, -1], [1, -1, -1], [2, -1, -1]]), held=[1, 1, 1], prefix=[40, 10, 10], off=[0, 2, 4, 8],
                T=8, free=[3, 4, 5, 6, -1, -1, -1], count=4)
    base.update(change)
    got = check(**base)
    assert got[5].any() or "count" in change


def test_pages_held_twice_do_not_run_over_the_stack():
    # more pages come back than there are
    table = np.array([[0, 1, 2, 3], [0, 1, 2, 3]])
    got = check(table, [4, 4], [0, 0], [0, 0, 0], 0, [0, 1, -1, -1], 2)
    assert got[3] == 4
