"""What the bounds that the attention tests hold the rows to can see: a tile of 64 tokens lost from any place of the sequence."""
import numpy as np
import pytest

from cache_util import RowBound, World, seen_by_rows, tree_words
from oracle import cache as oc
from test_gpu_cache import ATTENTION


@pytest.mark.parametrize("case", [c for c in ATTENTION if max(c[5]) >= 64], ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_a_lost_tile_is_seen(case):
    dtype, H, KV, dh, T, past, fresh, page, bits, tree = case
    w = World(1000 + T + dh, dtype, H, KV, dh, T, past, page, bits, fresh)
    for b in range(w.B):
        n = int(w.fresh[b])
        oc.append(w.pool, w.table, page, b, int(w.past[b]), w.normal(n, KV, dh), w.normal(n, KV, dh), bits)
    q = w.normal(w.B * T, H, dh, std=1.5).reshape(w.B, T, H, dh)
    words = tree_words(w.rng, w.B, T) if tree else None
    b = int(w.past.argmax())
    new = min(int(w.fresh[b]), 8)                                        # the first rows do
    k, v, see = seen_by_rows(w, words, b)
    whole = RowBound(dtype, q[b, :new], k, v, see[:new])
    tiles = range(0, int(w.past[b]) - 63, 64)
    for j in list(tiles)[:: max(1, len(tiles) // 12)]:
        for twice in (False, True):                                      # left out, or counted twice
            if twice:
                part = np.arange(j, j + 64)
                other = RowBound(dtype, q[b, :new], *(np.concatenate([a, a[part]]) for a in (k, v)),
                                 np.concatenate([see[:new], see[:new, part]], 1))
            else:
                less = see[:new].copy()
                less[:, j:j + 64] = False
                other = RowBound(dtype, q[b, :new], k, v, less)
            assert (np.abs(other.out - whole.out) / whole.bound).max() > 2, (j, twice)
