"""Attention over the cache where values differ by many powers of two: every row within a bound of what that row sees."""
import numpy as np
import pytest
import torch

from cache_util import RowBound, World, check_rows, seen_by_rows, tree_words
from oracle import cache as oc
from test_gpu_cache import ATTENTION, run_attention

pytestmark = pytest.mark.gpu

ROWS = [("f32", 64, 3), ("f32", 64, 13), ("f32", 128, 9), ("f32", 128, 40), ("bf16", 64, 3), ("bf16", 64, 7), ("bf16", 128, 3),
        ("bf16", 64, 20), ("bf16", 64, 100), ("bf16", 128, 20), ("bf16", 128, 64), ("bf16", 128, 100)]


def world(seed, dtype, dh, T, past, bits=32):
    """Two heads; the new tokens' keys and values are there to be changed before they are appended."""
    w = World(seed, dtype, 2, 2, dh, T, [past], 32, bits)
    return w, w.normal(T, 2, dh), w.normal(T, 2, dh), w.normal(T, 2, dh)


def both_cuts(w, q, words):
    for max_len in (64, 1024):                                           # one workgroup for a sequence, and several
        check_rows(w, q, words, run_attention(w, q, words, max_len))


@pytest.mark.parametrize("power", [14, 22, 30, 100])
@pytest.mark.parametrize("past", [0, 200])
@pytest.mark.parametrize("dtype,dh,T", ROWS)
def test_what_a_row_does_not_see_costs_it_nothing(dtype, dh, T, past, power):
    """A later token of a prompt, or another branch of a tree, with values of another size."""
    w, q, k, v = world(8000 + T + power, dtype, dh, T, past)
    v[T // 2] *= 2.0 ** power
    oc.append(w.pool, w.table, 32, 0, past, k, v, 32)
    both_cuts(w, q, None)
    if T <= 64:
        words = tree_words(w.rng, 1, T)
        words[0] &= ~np.uint64(1 << (T // 2))                            # of the branch, its own token alone sees it
        words[0, T // 2] |= np.uint64(1 << (T // 2))
        both_cuts(w, q, words)


@pytest.mark.parametrize("power", [24, 60])
@pytest.mark.parametrize("at", [3, 90, 240])
@pytest.mark.parametrize("dtype,dh,T", ROWS)
def test_what_a_row_sees_with_next_to_no_weight_costs_it_nothing(dtype, dh, T, at, power):
    """One token's values are 2^24 (2^60) times the others', its weight e^-60 (e^-85) of theirs."""
    n = 256
    w = World(8200 + T + at, dtype, 2, 2, dh, T, [n], 32, 32)
    k, v = w.normal(n + T, 2, dh), w.normal(n + T, 2, dh)
    q = w.normal(T, 2, dh)
    q[..., 0] = 8.0
    k[..., 0] = 0.0
    k[at, :, 0] = -(60.0 if power == 24 else 85.0) * np.sqrt(dh) / 8
    v[at] *= 2.0 ** power
    oc.append(w.pool, w.table, 32, 0, 0, k, v, 32)
    both_cuts(w, q, None)


@pytest.mark.parametrize("dtype,dh,T", ROWS)
@pytest.mark.parametrize("how", ["rising", "falling", "mixed", "far apart", "one element", "tiny", "zero first"])
def test_values_of_any_size(dtype, dh, T, how):
    """Scales that change from token to token and tile to tile.  `one element`: a value is large in one place and its other codes are 0,
    so that the rest of the row's elements are the other tokens' alone."""
    n = 400
    w = World(8400 + T, dtype, 2, 2, dh, T, [n], 32, 32)
    size = {"rising": np.linspace(-40, 10, n + T), "falling": np.linspace(10, -40, n + T), "mixed": w.rng.uniform(-12, 12, n + T),
            "far apart": w.rng.choice([-100.0, -50.0, 0.0, 50.0, 90.0], n + T), "tiny": np.full(n + T, -100.0)}.get(how, np.zeros(n + T))
    k, v = w.normal(n + T, 2, dh), w.normal(n + T, 2, dh) * 2.0 ** size[:, None, None]
    if how == "one element":
        v[::50, :, 5] = 2.0 ** 20
    if how == "zero first":
        v[:200] = 0.0
    oc.append(w.pool, w.table, 32, 0, 0, k, v, 32)
    both_cuts(w, w.normal(T, 2, dh), None)


@pytest.mark.parametrize("bits", [32, 16])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("dtype,dh,T", [r for r in ROWS if r[1] == 128])
def test_a_scale_that_is_no_number_is_its_blocks_alone(dtype, dh, T, bad, bits):
    """One block of a value of the past (head 0) and one of a new token (head 1): NaN in that block of the rows that see it, and nowhere else."""
    w, q, k, v = world(8600 + T, dtype, dh, T, 150, bits)
    oc.append(w.pool, w.table, 32, 0, 150, k, v, bits)
    at = [(0, 40, 1), (1, 150 + T // 2, 0)]                              # head, token, block
    finite = {n: a.copy() for n, a in w.pool.items()}
    for h, j, blk in at:
        w.pool["v_scales"][w.table[0, j // 32], h, blk, j % 32] = bad
        finite["v_scales"][w.table[0, j // 32], h, blk, j % 32] = 1.0
    for max_len in (64, 1024):
        got = run_attention(w, q, None, max_len)
        for h, j, blk in at:
            mine = got[0, max(0, j - 150):, h, 64 * blk:64 * blk + 64]
            assert np.all(np.isnan(mine))
        assert np.isnan(got).sum() == sum(64 * (T - max(0, j - 150)) for _, j, _ in at)
        broken, w.pool = w.pool, finite
        want = RowBound(dtype, q, *seen_by_rows(w, None, 0)).out
        got[0] = np.where(np.isnan(got[0]), want, got[0])
        check_rows(w, q, None, got)
        w.pool = broken


@pytest.mark.parametrize("pattern", [0x7FC00000, 0x7FFFFFFF, 0xFFFFFFFF, 0x7F800001])
@pytest.mark.parametrize("T", [1, 6, 40])
def test_no_number_of_any_pattern_stays_one(T, pattern):
    """fp32 scales that are NaN, whatever their bits, are NaN in bf16 too: read back, as keys and as values."""
    import paper_2301_11913_amd as sw
    w, q, k, v = world(8800 + T, "bf16", 64, T, 40)
    oc.append(w.pool, w.table, 32, 0, 40, k, v, 32)
    bad = np.array([pattern], dtype=np.uint32).view(np.float32)[0]
    w.pool["k_scales"][w.table[0, 0], 0, 0, 7] = bad
    w.pool["v_scales"][w.table[0, 0], 1, 0, 9] = bad
    for max_len in (64, 1024):
        assert np.all(np.isnan(run_attention(w, q, None, max_len)))      # head 0 by the key, head 1 by the value
    cfg, cache = w.upload()
    out = [torch.zeros((40, 2 * 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    sw.swarm_cache_read(cfg, cache, w.ints(w.table), w.ints([0]), None, 40, *out)
    for got, token, head in ((out[0], 7, 0), (out[1], 9, 1)):
        none = torch.isnan(got).cpu().reshape(40, 2, 64)
        assert bool(none[token, head].all()) and int(none.sum()) == 64


def test_read_rounds_as_torch_does():
    """code * scale of every code, with scales of all sizes down to the smallest: the bf16 value next to the fp32 product."""
    import paper_2301_11913_amd as sw
    n = 512
    cfg = sw.CacheConfig(1, 1, 64, 16, n // 16, 1, n // 16, "bf16", 32)
    gen = torch.Generator(device="cuda").manual_seed(3)
    pool = {name: torch.zeros(shape, dtype=dt, device="cuda") for name, (shape, dt) in cfg.shapes().items()}
    codes = torch.randint(-127, 128, (n, 64), generator=gen, device="cuda", dtype=torch.int32).to(torch.int8)
    scales = torch.ldexp(1 + torch.rand(n, generator=gen, device="cuda"), torch.arange(n, device="cuda") % 250 - 140)
    pool["k_codes"].copy_(codes.reshape(n // 16, 1, 16, 64))
    pool["v_codes"].copy_(codes.reshape(n // 16, 1, 16, 64).transpose(2, 3))
    for name in ("k_scales", "v_scales"):
        pool[name].copy_(scales.reshape(n // 16, 1, 1, 16))
    out = [torch.zeros((n, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    sw.swarm_cache_read(cfg, sw.Cache(cfg, **pool), torch.arange(n // 16, dtype=torch.int32, device="cuda"), zero, None, n, *out)
    want = (codes.float() * scales[:, None]).to(torch.bfloat16)
    assert torch.equal(out[0], want) and torch.equal(out[1], want)


def case_world(case):
    dtype, H, KV, dh, T, past, fresh, page, bits, tree = case
    w = World(9000 + T + dh, dtype, H, KV, dh, T, past, page, bits, fresh)
    for b in range(w.B):
        n = int(w.fresh[b])
        oc.append(w.pool, w.table, page, b, int(w.past[b]), w.normal(n, KV, dh), w.normal(n, KV, dh), bits)
    return w, w.normal(w.B * T, H, dh, std=1.5), tree_words(w.rng, w.B, T) if tree else None


@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_every_row_within_its_own_bound(case):
    """A bound that a tile of 64 tokens lost or counted twice exceeds, at all of these lengths."""
    w, q, words = case_world(case)
    for max_len in (0, 64, int((w.past + w.fresh).max())):
        check_rows(w, q, words, run_attention(w, q, words, max_len))


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dtype,rows", [("f32", 2), ("f32", 8), ("f32", 17), ("bf16", 4), ("bf16", 5), ("bf16", 8), ("bf16", 9), ("bf16", 33),
                                        ("bf16", 65), ("bf16", 129)])
def test_every_number_of_rows_within_its_own_bound(dtype, rows, dh, page):
    w, q, words = case_world((dtype, 2, 2, dh, rows, [650, 64], [rows, rows - 1], page, 32, rows <= 64))
    for max_len in (64, 1024):
        check_rows(w, q, words, run_attention(w, q, words, max_len))


@pytest.mark.parametrize("dtype,T", [("f32", 3), ("bf16", 1), ("bf16", 20), ("bf16", 140)])
def test_shared_heads_within_their_own_bounds(dtype, T):
    w, q, words = case_world((dtype, 12, 3, 64, T, [1500, 90], None, 64, 16, T <= 64))
    check_rows(w, q, words, run_attention(w, q, words, 2048))


@pytest.mark.parametrize("dtype,dh,T", ROWS + [("bf16", 64, 40), ("bf16", 64, 64)])
def test_scores_far_below_zero_and_splits_without_tokens(dtype, dh, T):
    """Every score is about -300, and the short sequence leaves most of the workgroups that share its rows without a token."""
    w = World(9300 + T, dtype, 2, 2, dh, T, [1900, 30], 32, 32)
    q = w.normal(w.B * T, 2, dh)
    q[..., 0] = 30.0
    for b in range(2):
        n = int(w.past[b]) + T
        k = w.normal(n, 2, dh)
        k[..., 0] = -10.0 * np.sqrt(dh)
        oc.append(w.pool, w.table, 32, b, 0, k, w.normal(n, 2, dh), 32)
    for max_len in (64, 2048):
        check_rows(w, q, None, run_attention(w, q, None, max_len))


@pytest.mark.parametrize("bits", [32, 16])
@pytest.mark.parametrize("dtype,dh,T", ROWS)
def test_scales_of_either_sign(dtype, dh, T, bits):
    """A pool that another quantiser filled: scales below zero, and zeros of both signs."""
    w, q, k, v = world(9500 + T, dtype, dh, T, 150, bits)
    oc.append(w.pool, w.table, 32, 0, 150, k, v, bits)
    for name in ("k_scales", "v_scales"):
        a = w.pool[name]
        a *= np.where(w.rng.random(a.shape) < 0.5, -1.0, 1.0).astype(np.float32)
        a[w.rng.random(a.shape) < 0.1] = -0.0
    both_cuts(w, q, None)


@pytest.mark.parametrize("seed", list(range(24)) + [231])
def test_anything_at_once(seed):
    """Random shapes, trees, pages, cuts, scores some hundreds apart and values of sizes that change by token, by tile or not at all."""
    rng = np.random.default_rng(9700 + seed)
    dtype, dh = ("bf16", "bf16", "f32")[seed % 3], (64, 128)[seed // 3 % 2]
    T, KV, group = int(rng.choice([1, 2, 5, 9, 17, 33, 40, 64, 100, 150])), int(rng.integers(1, 4)), int(rng.choice([1, 1, 2, 4]))
    past = [int(x) for x in rng.integers(0, 700, 3)]
    fresh = [T, int(rng.integers(0, T + 1)), int(rng.integers(1, T + 1))]
    page = int(rng.choice([16, 32, 64, 128]))
    w = World(9800 + seed, dtype, KV * group, KV, dh, T, past, page, int(rng.choice([16, 32])), fresh)
    q = w.normal(3 * T, KV * group, dh) * 2.0 ** rng.integers(-3, 4)
    for b in range(3):
        n = past[b] + fresh[b]
        if n == 0:
            continue
        size = [np.zeros(n), rng.uniform(-3, 3, n), rng.uniform(-20, 20, n), np.repeat(rng.uniform(-30, 30, n // 64 + 1), 64)[:n],
                rng.choice([0.0, 0.0, 0.0, -12.0, 25.0], n)][int(rng.integers(0, 5))]
        v = w.normal(n, KV, dh) * 2.0 ** size[:, None, None]
        if dh == 128 and rng.random() < 0.5:                             # the second block's sizes go another way
            v[..., 64:] = w.normal(n, KV, 64) * 2.0 ** -size[:, None, None]
        v[rng.random(n) < 0.05] = 0.0
        k = w.normal(n, KV, dh) * rng.choice([0.1, 1.0, 4.0])
        oc.append(w.pool, w.table, page, b, 0, k, v, w.scale_bits)
    words = tree_words(w.rng, 3, T) if T <= 64 and rng.random() < 0.6 else None
    if words is not None and rng.random() < 0.5:
        words &= w.rng.integers(0, 1 << 63, words.shape, dtype=np.uint64) * np.uint64(2) + np.uint64(1)     # holes, some rows blind of themselves
    for max_len in (0, 64, 700 + T):
        check_rows(w, q, words, run_attention(w, q, words, max_len))
