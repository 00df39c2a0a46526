"""Inputs of the paged-cache tests: a cache with its codes, scales and table, on host and device."""
import numpy as np
import torch

from gpu_util import DEV, i32, to_dev
from oracle import tr_serve as S

NAN_CODE = 127


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).bfloat16()


class Paged:
    """A cache of `lens` tokens per sequence plus `room` more; unused slots and pages hold NaN codes."""

    def __init__(self, rng, lens, heads, dh, layers=1, room=0, spare=2, exps=(-8, -4)):
        self.lens, self.heads, self.dh, self.layers = list(lens), heads, dh, layers
        need = [-(-(l + room) // 32) for l in lens]
        self.n_blocks, self.width = sum(need) + spare, max(max(need), 1) + 1
        ids, self.table, at = rng.permutation(self.n_blocks), np.full((len(lens), self.width), -1), 0
        for s, n in enumerate(need):
            self.table[s, :n] = ids[at:at + n]
            at += n
        shape = (layers, heads, self.n_blocks)
        self.pool, self.scale = {}, {}
        for w in "kv":
            self.pool[w] = np.full(shape + (32 * dh,), NAN_CODE, np.uint8)
            self.scale[w] = 2.0 ** rng.integers(*exps, shape).astype(np.float32)
            place = S.offsets(dh, w)
            for s, l in enumerate(lens):
                for p in range(-(-l // 32)):
                    rows = min(32, l - 32 * p)
                    codes = S.encode((rng.normal(size=(layers, heads, rows, dh)) * 60).clip(-448, 448))
                    page = self.pool[w][:, :, self.table[s, p]]
                    page[..., place[:rows]] = codes
                    self.pool[w][:, :, self.table[s, p]] = page

    def values(self, which, s, layer=0):
        """[heads, len, dh] numbers of sequence s."""
        n = -(-self.lens[s] // 32)
        v = S.page_values(self.pool[which][layer], self.scale[which][layer], which)[:, self.table[s, :n]]
        return v.reshape(self.heads, -1, self.dh)[:, :self.lens[s]]

    def device(self):
        return dict(k=to_dev(self.pool["k"]), v=to_dev(self.pool["v"]), ks=to_dev(self.scale["k"]), vs=to_dev(self.scale["v"]),
                    table=i32(self.table), prefix=i32(self.lens))


def offsets_of(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)


def ints(n, value=-7):
    return torch.full((n,) if isinstance(n, int) else n, value, dtype=torch.int32, device=DEV)
