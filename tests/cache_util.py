"""Inputs, pools and the oracle's side for the tests of the key / value cache."""
import numpy as np
import torch

from oracle import cache as oc

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def tree_words(rng, B, T):
    """Ancestor masks of random trees: every token sees itself and what the earlier token that it hangs on sees."""
    words = np.zeros((B, T), dtype=np.uint64)
    for b in range(B):
        for t in range(T):
            up = words[b, rng.integers(0, t)] if t else np.uint64(0)
            words[b, t] = up | (np.uint64(1) << np.uint64(t))
    return words


class World:
    """A pool with the past of some sequences in it, on the host (the oracle's) and on the GPU."""

    def __init__(self, seed, dtype, H, KV, dh, T, past, page, scale_bits, fresh=None, spare=1, holes=True):
        self.rng = rng = np.random.default_rng(seed)
        self.dtype, self.H, self.KV, self.dh, self.T, self.page, self.scale_bits = dtype, H, KV, dh, T, page, scale_bits
        self.past = np.array(past, dtype=np.int32)
        self.B = B = len(past)
        self.fresh = np.full(B, T, dtype=np.int32) if fresh is None else np.array(fresh, dtype=np.int32)
        self.table_pages = max(1, -(-int(max(0, self.past.max()) + T) // page)) + spare
        pages = B * self.table_pages + 3
        order = rng.permutation(pages)[:B * self.table_pages]
        self.table = order.reshape(B, self.table_pages).astype(np.int32)
        # what no token has been written to: codes that encoding never gives and scales that are no numbers
        nb = dh // 64
        self.pool = {"k_codes": np.full((pages, KV, page, dh), -128, np.int8), "v_codes": np.full((pages, KV, dh, page), -128, np.int8),
                     "k_scales": np.full((pages, KV, nb, page), np.nan, np.float32),
                     "v_scales": np.full((pages, KV, nb, page), np.nan, np.float32)}
        for b in range(B):
            n = int(max(0, self.past[b]))
            self.k_past = rng.standard_normal((n, KV, dh)).astype(np.float32)
            oc.append(self.pool, self.table, page, b, 0, self.k_past, rng.standard_normal((n, KV, dh)).astype(np.float32), scale_bits)

    def normal(self, *shape, std=1.0):
        """float64 values that the dtype holds exactly."""
        x = torch.from_numpy((self.rng.standard_normal(shape) * std).astype(np.float32))
        return x.to(TORCH[self.dtype]).double().numpy()

    def config(self):
        import paper_2301_11913_amd as sw
        return sw.CacheConfig(self.H, self.KV, self.dh, self.page, self.pool["k_codes"].shape[0], self.B, self.table_pages,
                              self.dtype, self.scale_bits)

    def upload(self):
        import paper_2301_11913_amd as sw
        cfg = self.config()
        dev = {n: torch.from_numpy(a.copy()).cuda() for n, a in self.pool.items()}
        if self.scale_bits == 16:
            for n in ("k_scales", "v_scales"):
                dev[n] = dev[n].to(torch.bfloat16)
        return cfg, sw.Cache(cfg, **dev)

    def ints(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    def dev(self, x):
        return torch.from_numpy(np.ascontiguousarray(x)).to(TORCH[self.dtype]).cuda()


def pool_of(cache):
    """The GPU's pool as numpy (scales as fp32 values)."""
    out = {}
    for n, t in cache.tensors.items():
        out[n] = (t if n.endswith("codes") else t.float()).cpu().numpy()
    return out


def same_pool(a, b):
    return all(np.array_equal(a[n], b[n], equal_nan=n.endswith("scales")) for n in a)


def attention_bound(dtype, out, mean_abs, size, n, v_max):
    """How far a row of attention may be from its value, elementwise.  Every weight p_j has a relative error eps:
      its score is a sum of d_head / 64 products of whole numbers and two scales, about 16 roundings of 2^-24 of at most
      `size` each, which the exponential turns into a relative error; the exponent and the maximum it is taken from have the
      same size (8 more), exp itself and the running sums add one rounding per 64 tokens and 64 for the rest;
      bf16: the weight itself may be rounded to fp16 (2^-11).
    Numerator and denominator each carry it: 2 eps of the weighted mean of |v|.  Weights may also be held as whole numbers of
    2^-22 of the largest one (bf16; below fp16's normal range 2^-24) or 2^-30 (fp32): n of them against a sum of at least 1.  At the end half a
    step of the type."""
    eps = 2.0 ** -24 * (24 * size[..., None] + n / 64 + 64) + (2.0 ** -11 if dtype == "bf16" else 0.0)
    whole = n * v_max * (2.0 ** -22 if dtype == "bf16" else 2.0 ** -30)
    return 2 * eps * mean_abs + whole + HALF_STEP[dtype] * np.abs(out) + 1e-30
