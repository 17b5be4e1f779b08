"""The paged int8 key / value cache: append, read, keep, and attention over it, against the oracle."""
import numpy as np
import pytest
import torch

from cache_util import HALF_STEP, TORCH, World, attention_bound, pool_of, same_pool, tree_words
from oracle import cache as oc

pytestmark = pytest.mark.gpu

FAR = 1_000_003


# ------------------------------------------------------------------------------------------------ append and read
@pytest.mark.parametrize("dtype,H,KV,dh,T,past,fresh,page,bits,pad", [
    ("f32", 4, 4, 64, 1, [0], None, 16, 32, 0),
    ("f32", 4, 4, 64, 1, [15, 16, 63, 64], None, 16, 32, 8),
    ("f32", 3, 3, 128, 17, [0, 5, 127], [17, 0, 3], 32, 16, 0),
    ("bf16", 16, 16, 64, 1, [170], None, 64, 32, 0),
    ("bf16", 8, 2, 128, 65, [63, 1], [65, 64], 64, 16, 16),
    ("bf16", 12, 12, 64, 130, [31, 0, 200], [130, 129, 1], 256, 32, 0),
    ("bf16", 5, 1, 128, 3, [2046, 0], None, 1024, 16, 0)])
def test_append_then_read_without_rotation(dtype, H, KV, dh, T, past, fresh, page, bits, pad):
    """Bit for bit the codec's codes and scales, and nothing else in the pool or the outputs is touched."""
    import paper_2301_11913_amd as sw
    w = World(1 + T, dtype, H, KV, dh, T, past, page, bits, fresh)
    cfg, cache = w.upload()
    rows = w.B * T
    x = w.normal(rows, (H + 2 * KV) * dh + pad, std=2.0)
    x[0, H * dh:H * dh + 64] = 0.0                                     # a block of zeros
    dev = w.dev(x)
    k, v = dev[:, H * dh:(H + KV) * dh], dev[:, (H + KV) * dh:(H + 2 * KV) * dh]
    table, past_d, fresh_d = w.ints(w.table), w.ints(w.past), w.ints(w.fresh)
    sw.swarm_cache_append(cfg, cache, table, past_d, fresh_d, T, k, v)
    k_out, v_out = (torch.full((rows, KV * dh), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2))
    sw.swarm_cache_read(cfg, cache, table, past_d, fresh_d, T, k_out, v_out)
    torch.cuda.synchronize()
    x = x.reshape(w.B, T, -1)
    want_k, want_v = np.full((w.B, T, KV * dh), 7.0), np.full((w.B, T, KV * dh), 7.0)
    for b in range(w.B):
        n = int(w.fresh[b])
        oc.append(w.pool, w.table, page, b, int(w.past[b]), x[b, :n, H * dh:(H + KV) * dh].reshape(n, KV, dh),
                  x[b, :n, (H + KV) * dh:(H + 2 * KV) * dh].reshape(n, KV, dh), bits)
        rk, rv, _ = oc.read(w.pool, w.table, page, b, list(range(w.past[b], w.past[b] + n)))
        want_k[b, :n], want_v[b, :n] = rk.reshape(n, KV * dh), rv.reshape(n, KV * dh)
    assert same_pool(pool_of(cache), w.pool)
    # code * scale is exact in 64 bits: one fp32 product, for bf16 a second rounding
    tol = 2.0 ** -24 + (HALF_STEP["bf16"] if dtype == "bf16" else 0.0)
    for got, want in ((k_out, want_k), (v_out, want_v)):
        got = got.double().cpu().numpy().reshape(want.shape)
        assert np.all(np.abs(got - want) <= tol * np.abs(want))


@pytest.mark.parametrize("dtype,H,KV,dh,T,past,page,bits,where", [
    ("f32", 4, 4, 64, 5, [0, 130], 16, 32, "past"),
    ("f32", 2, 2, 128, 33, [7], 64, 32, "far"),
    ("bf16", 8, 2, 64, 64, [100, 3], 32, 16, "given"),
    ("bf16", 16, 16, 128, 20, [40], 128, 32, "past")])
def test_append_rotates(dtype, H, KV, dh, T, past, page, bits, where):
    """Rotation in 64 bits: q_out within half a step of its type, keys the codes of the rotated rows.  A rotated key may come
    out one fp32 step apart (2^-53 of an angle of up to 10^6 radians against 2^-24: about 1 value in 100), which moves a code only
    next to a border between two: none by more than one, fewer than 1 in 10^4."""
    import paper_2301_11913_amd as sw
    w = World(17 + T, dtype, H, KV, dh, T, past, page, bits)
    cfg, cache = w.upload()
    rows = w.B * T
    x = w.normal(rows, (H + 2 * KV) * dh)
    pos = np.concatenate([p + np.arange(T) for p in w.past])
    if where == "far":
        pos = FAR + np.arange(rows)
    if where == "given":
        pos = w.rng.integers(0, 4096, rows)                              # a tree: several tokens at one depth
        pos[0] = -5
    positions = None if where == "past" else w.ints(pos)
    dev = w.dev(x)
    q, k, v = dev.split([H * dh, KV * dh, KV * dh], 1)
    q_out = torch.full((rows, H * dh + 8), 7.0, dtype=TORCH[dtype], device="cuda")
    table, past_d = w.ints(w.table), w.ints(w.past)
    sw.swarm_cache_append(cfg, cache, table, past_d, None, T, k, v, q=q, q_out=q_out[:, :H * dh], positions=positions, rotary=True)
    torch.cuda.synchronize()
    got = q_out.double().cpu().numpy()
    assert np.all(got[:, H * dh:] == 7.0)
    want = oc.rotate(x[:, :H * dh].reshape(rows, H, dh), pos).reshape(rows, -1)
    size = np.abs(x[:, :H * dh]).max()
    step = HALF_STEP["f32"] + (HALF_STEP["bf16"] if dtype == "bf16" else 0.0)
    assert np.all(np.abs(got[:, :H * dh] - want) <= step * np.abs(want) + 2.0 ** -45 * size)
    kr = oc.rotate(x[:, H * dh:(H + KV) * dh].reshape(rows, KV, dh), pos).astype(np.float32).reshape(w.B, T, KV, dh)
    for b in range(w.B):
        oc.append(w.pool, w.table, page, b, int(w.past[b]), kr[b], x[:, (H + KV) * dh:].reshape(w.B, T, KV, dh)[b], bits)
    pool = pool_of(cache)
    for n in ("v_codes", "v_scales"):
        assert np.array_equal(pool[n], w.pool[n], equal_nan=n.endswith("scales"))
    off = np.abs(pool["k_codes"].astype(int) - w.pool["k_codes"].astype(int))
    assert off.max() <= 1 and off.mean() < 1e-4
    fine = np.isfinite(w.pool["k_scales"])
    assert np.array_equal(fine, np.isfinite(pool["k_scales"]))
    scale_step = 2.0 ** -22 if bits == 32 else 2.0 ** -7
    assert np.all(np.abs(pool["k_scales"][fine] - w.pool["k_scales"][fine]) <= scale_step * w.pool["k_scales"][fine])
    # in place: the same values
    sw.swarm_cache_append(cfg, cache, table, past_d, None, T, k, v, q=q, q_out=q, positions=positions, rotary=True)
    torch.cuda.synchronize()
    assert np.array_equal(q.double().cpu().numpy(), got[:, :H * dh])


@pytest.mark.parametrize("bits", [32, 16])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_is_the_codec(dtype, bits):
    """Rows of all sizes, infinities and no numbers among them: the bits that swarm_codec_encode gives."""
    import paper_2301_11913_amd as sw
    KV, dh, T, page = 3, 128, 40, 16
    w = World(99, dtype, KV, KV, dh, T, [9], page, bits)
    cfg, cache = w.upload()
    x = w.normal(T, KV * dh)
    x *= 2.0 ** w.rng.integers(-60, 60, (T, 1))
    x[3, 5], x[4, 70], x[5, :64], x[6, 130] = np.inf, np.nan, -np.inf, -np.inf
    x[7] *= 2.0 ** -130 / np.abs(x[7]).max()
    dev = w.dev(x)
    sw.swarm_cache_append(cfg, cache, w.ints(w.table), w.ints(w.past), None, T, dev, dev)
    codes = torch.empty(dev.numel(), dtype=torch.int8, device="cuda")
    scales = torch.empty(dev.numel() // 64, dtype=torch.float32 if bits == 32 else torch.bfloat16, device="cuda")
    (sw.swarm_codec_encode if bits == 32 else sw.swarm_codec_encode_s16)(dev, codes, scales)
    torch.cuda.synchronize()
    codes, raw = codes.cpu().numpy().reshape(T, KV, dh), torch.int32 if bits == 32 else torch.int16
    scales = scales.view(raw).cpu().numpy().reshape(T, KV, 2)
    got = {n: (t if n.endswith("codes") else t.view(raw)).cpu().numpy() for n, t in cache.tensors.items()}
    for t in range(T):
        p, o = w.table[0, (9 + t) // page], (9 + t) % page
        assert np.array_equal(got["k_codes"][p, :, o], codes[t]) and np.array_equal(got["v_codes"][p, :, :, o], codes[t])
        assert np.array_equal(got["k_scales"][p, :, :, o], scales[t]) and np.array_equal(got["v_scales"][p, :, :, o], scales[t])


def test_append_leaves_out_what_is_out_of_range():
    """Sequences whose lengths do not fit and pages that are none: nothing of them is written, everything else is."""
    import paper_2301_11913_amd as sw
    page, T, KV, dh = 16, 4, 2, 64
    w = World(5, "f32", KV, KV, dh, T, [10, 0, 14, 12], page, 32, fresh=[4, 4, 4, 5])
    cfg, cache = w.upload()
    past = w.past.copy()
    past[0], past[1] = -1, w.table_pages * page - 3          # negative; one token too many.  The last one has fresh > tokens
    w.table[2, 1] = w.pool["k_codes"].shape[0]               # tokens 16, 17 of the third lie on a page that is none
    x = w.normal(w.B * T, KV * dh)
    dev = w.dev(x)
    args = (w.ints(w.table), w.ints(past), w.ints(w.fresh), T)
    sw.swarm_cache_append(cfg, cache, *args, dev, dev)
    out = [torch.full((w.B * T, KV * dh), 7.0, device="cuda") for _ in range(2)]
    sw.swarm_cache_read(cfg, cache, *args, *out)
    torch.cuda.synchronize()
    rows = x.reshape(w.B, T, KV, dh)[2]
    oc.append(w.pool, w.table, page, 2, 14, rows, rows, 32)
    assert same_pool(pool_of(cache), w.pool)
    got = out[0].cpu().numpy().reshape(w.B, T, -1)
    assert np.all(got[[0, 1, 3]] == 7.0) and np.all(got[2, 2:] == 0.0) and np.all(np.any(got[2, :2] != 0.0, axis=1))


# ------------------------------------------------------------------------------------------------ keep
@pytest.mark.parametrize("KV,dh,T,past,kept,page,bits", [
    (2, 64, 8, [0, 171], [[0, 2, 5], [7]], 16, 32),
    (4, 128, 64, [63, 1, 500], [list(range(64)), [], [63, 62, 1, 1, 0]], 64, 16),
    (1, 128, 64, [15], [[(7 * i) % 64 for i in range(64)]], 32, 32),
    (3, 64, 1, [16, 31], [[0], [0]], 16, 16),
    (2, 64, 5, [30], [[4, -1, 9, 0]], 16, 32)])                         # indices that are none of the draft's
def test_keep(KV, dh, T, past, kept, page, bits):
    import paper_2301_11913_amd as sw
    w = World(T + 40, "bf16", KV, KV, dh, T, past, page, bits)
    for b in range(w.B):
        oc.append(w.pool, w.table, page, b, past[b], w.normal(T, KV, dh), w.normal(T, KV, dh), bits)
    cfg, cache = w.upload()
    idx = np.full((w.B, T), 12345, dtype=np.int32)
    for b, ks in enumerate(kept):
        idx[b, :len(ks)] = ks
        oc.keep(w.pool, w.table, page, b, past[b], ks, T)
    sw.swarm_cache_keep(cfg, cache, w.ints(w.table), w.ints(w.past), w.ints(idx), w.ints([len(k) for k in kept]), T)
    torch.cuda.synchronize()
    assert same_pool(pool_of(cache), w.pool)


def test_keep_at_the_end_of_the_table_and_on_pages_that_are_none():
    import paper_2301_11913_amd as sw
    page, T, KV, dh = 16, 8, 2, 64
    w = World(77, "bf16", KV, KV, dh, T, [28, 28, 28, 28], page, 32, spare=0)
    cap = w.table_pages * page
    for b in range(4):
        oc.append(w.pool, w.table, page, b, 28, w.normal(T, KV, dh), w.normal(T, KV, dh), 32)
    cfg, cache = w.upload()
    past = np.array([cap - 3, 28, -1, 28], dtype=np.int32)
    n = np.array([3, 8, 2, 9], dtype=np.int32)                          # the last two are out of range
    idx = np.tile(np.array([[2, 5, 0, 7, 6, 1, 3, 4]], dtype=np.int32), (4, 1))
    w.table[1, 2] = -7                                                   # tokens 32.. of the second are on no page
    for b in (0, 1):
        oc.keep(w.pool, w.table, page, b, int(past[b]), idx[b, :n[b]], T)
    sw.swarm_cache_keep(cfg, cache, w.ints(w.table), w.ints(past), w.ints(idx), w.ints(n), T)
    torch.cuda.synchronize()
    assert same_pool(pool_of(cache), w.pool)


# ------------------------------------------------------------------------------------------------ attention
def run_attention(w, q, words, max_len=0, pads=(0, 0)):
    """out [B, T, H, dh] float64 (7 where nothing was written) of the GPU."""
    import paper_2301_11913_amd as sw
    cfg, cache = w.upload()
    rows, width = w.B * w.T, w.H * w.dh
    qd = w.dev(np.concatenate([q.reshape(rows, width), np.full((rows, pads[0]), 99.0)], 1))[:, :width]
    buf = torch.full((rows, width + pads[1]), 7.0, dtype=TORCH[w.dtype], device="cuda")
    tree = None if words is None else torch.from_numpy(words.view(np.int64)).cuda()
    n = sw.swarm_cache_attention_workspace_bytes(cfg, w.T, max_len)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    past, fresh = w.ints(w.past), w.ints(w.fresh)
    sw.swarm_cache_attention(cfg, cache, w.ints(w.table), past, fresh, w.T, qd, buf[:, :width], ws, tree=tree, max_len=max_len)
    torch.cuda.synchronize()
    got = buf.double().cpu().numpy()
    assert np.all(got[:, width:] == 7.0)
    return got[:, :width].reshape(w.B, w.T, w.H, w.dh)


def check_attention(w, q, words, got, skip=()):
    for b in range(w.B):
        n, new = int(w.past[b]), int(w.fresh[b])
        assert np.all(got[b, 0 if b in skip else new:] == 7.0)
        if b in skip or new == 0:
            continue
        k, v, there = oc.read(w.pool, w.table, w.page, b, list(range(n + new)))
        see = np.ones((new, n + new), dtype=bool)
        for t in range(new):
            for u in range(new):
                see[t, n + u] = u <= t if words is None else bool(int(words[b, t]) >> u & 1)
        see &= there[None]
        unseen = ~see.any(axis=0)
        k[unseen], v[unseen] = 0.0, 0.0                                 # whatever lies there
        out, mean_abs, size = oc.attention(q.reshape(w.B, w.T, w.H, w.dh)[b, :new], k, v, see)
        bound = attention_bound(w.dtype, out, mean_abs, size, n + new, np.abs(v).max(initial=0.0))
        assert np.all(np.isfinite(got[b, :new]))
        off = np.abs(got[b, :new] - out)
        assert np.all(off <= bound), (b, float((off / bound).max()))
        blind = ~see.any(axis=1)
        assert np.all(got[b, :new][blind] == 0.0)


ATTENTION = [
    # dtype, H, KV, dh, T, past, fresh, page, scale bits, tree
    ("f32", 1, 1, 64, 1, [0], None, 16, 32, False),                      # one token, nothing before it
    ("f32", 4, 4, 64, 1, [0, 1, 15, 16, 17, 62, 63, 64, 65, 127, 128], None, 16, 32, False),
    ("f32", 4, 4, 64, 9, [500, 250, 3], None, 32, 32, True),
    ("f32", 6, 2, 128, 5, [40, 0], [5, 2], 64, 16, True),
    ("f32", 4, 2, 64, 150, [0, 70], [150, 149], 64, 32, False),          # a prompt, causal
    ("f32", 2, 2, 128, 1, [5000], None, 256, 32, False),
    ("bf16", 1, 1, 128, 1, [0, 3], None, 16, 32, False),
    ("bf16", 16, 16, 64, 1, [170], None, 16, 32, False),
    ("bf16", 32, 8, 128, 1, [1000, 0, 77, 4095], None, 64, 16, False),   # shared heads
    ("bf16", 10, 2, 64, 1, [300], None, 32, 32, False),                  # five to a head
    ("bf16", 16, 1, 128, 1, [129], None, 16, 32, False),                 # one for all
    ("bf16", 8, 8, 128, 33, [200, 101, 0], [33, 17, 30], 64, 32, True),
    ("bf16", 4, 4, 64, 64, [64, 1], None, 128, 16, True),                # the widest tree
    ("bf16", 4, 1, 64, 64, [31], [63], 16, 32, True),
    ("bf16", 4, 4, 128, 16, [48, 0], [16, 0], 16, 32, False),
    ("bf16", 4, 4, 128, 200, [0, 57], [200, 130], 64, 32, False),        # prompts
    ("bf16", 4, 2, 64, 129, [700], None, 32, 16, False),
    ("bf16", 2, 2, 128, 1, [30000], None, 1024, 32, False),              # spread over many workgroups
]


@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: "-".join(str(x) for x in c).replace(" ", ""))
def test_attention(case):
    dtype, H, KV, dh, T, past, fresh, page, bits, tree = case
    w = World(1000 + T + dh, dtype, H, KV, dh, T, past, page, bits, fresh)
    for b in range(w.B):
        n = int(w.fresh[b])
        oc.append(w.pool, w.table, page, b, int(w.past[b]), w.normal(n, KV, dh), w.normal(n, KV, dh), bits)
    q = w.normal(w.B * T, H, dh, std=1.5)
    words = tree_words(w.rng, w.B, T) if tree else None
    check_attention(w, q, words, run_attention(w, q, words, max_len=int((w.past + w.fresh).max()), pads=(8, 16)))


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("bits", [32, 16])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("dtype,rows", [("f32", 3), ("f32", 7), ("f32", 13), ("bf16", 3), ("bf16", 7), ("bf16", 40), ("bf16", 100)])
def test_attention_at_every_number_of_rows(dtype, rows, dh, bits, page):
    """Each kernel's row counts, head sizes, scales, page sizes: over several tiles and splits, with and without a tree."""
    w = World(7000 + rows + dh + bits + page, dtype, 2, 2, dh, rows, [700, 129], page, bits, fresh=[rows, rows - 1])
    for b in range(w.B):
        n = int(w.fresh[b])
        oc.append(w.pool, w.table, page, b, int(w.past[b]), w.normal(n, 2, dh), w.normal(n, 2, dh), bits)
    q = w.normal(w.B * rows, 2, dh, std=1.5)
    words = tree_words(w.rng, w.B, rows) if rows <= 64 else None
    for tree in ([None, words] if rows <= 64 else [None]):
        for max_len in (64, 1024):                                       # one workgroup for a sequence, and several
            check_attention(w, q, tree, run_attention(w, q, tree, max_len))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [3, 40])
def test_attention_masks_that_leave_rows_empty(dtype, T):
    """Trees that say nothing (zeros where nothing lies before), that leave a token itself out, that name tokens that are not there;
    what a mask hides may be infinite or no number."""
    w = World(2000 + T, dtype, 4, 4, 64, T, [0, 20], 16, 32, fresh=[T, T - 1])
    for b in range(w.B):
        n = int(w.fresh[b])
        oc.append(w.pool, w.table, 16, b, int(w.past[b]), w.normal(n, 4, 64), w.normal(n, 4, 64), 32)
    words = np.zeros((2, T), dtype=np.uint64)
    words[:, 0] = 0                                                      # blind: zeros, or the past alone
    words[:, 1] = 1 << 0                                                 # its parent, not itself
    words[:, 2] = (1 << 2) | (1 << 63)                                   # itself, and a token that is none
    words[:, 3:] = 1 << 1
    hidden = T - 2                                                       # seen by nobody
    for b in range(2):
        p, o = w.table[b, (w.past[b] + hidden) // 16], (w.past[b] + hidden) % 16
        if hidden > 2:
            w.pool["k_scales"][p, :, :, o] = np.inf
            w.pool["v_scales"][p, :, :, o] = np.nan
            w.pool["k_codes"][p, :, o] = -128
    q = w.normal(2 * T, 4, 64)
    check_attention(w, q, words, run_attention(w, q, words, max_len=64))


@pytest.mark.parametrize("dtype,T,tree", [("f32", 2, True), ("bf16", 2, True), ("bf16", 70, False)])
def test_attention_of_sequences_and_pages_out_of_range(dtype, T, tree):
    w = World(3000 + T, dtype, 2, 2, 128, T, [90, 40, 5, 33], 16, 32, fresh=[T, T, T, T])
    for b in range(w.B):
        oc.append(w.pool, w.table, 16, b, int(w.past[b]), w.normal(T, 2, 128), w.normal(T, 2, 128), 32)
    w.table[0, 1] = w.pool["k_codes"].shape[0] + 5                      # tokens 16..31: not attended to
    w.table[0, 3] = -1
    w.table[2, :] = -1                                                   # none at all: zeros
    w.past[1] = -3
    w.past[3] = w.table_pages * 16
    q = w.normal(4 * T, 2, 128)
    words = tree_words(w.rng, 4, T) if tree else None
    check_attention(w, q, words, run_attention(w, q, words), skip=(1, 3))


@pytest.mark.parametrize("dtype,T", [("f32", 1), ("bf16", 1), ("bf16", 80)])
def test_attention_of_queries_of_any_size(dtype, T):
    """Zero, tiny and large queries; a large one makes the softmax a choice of one key."""
    w = World(4000 + T, dtype, 4, 4, 128, T, [300], 64, 32)
    oc.append(w.pool, w.table, 64, 0, 300, w.normal(T, 4, 128), w.normal(T, 4, 128), 32)
    q = w.normal(T, 4, 128)
    q[:, 0] = 0.0
    q[:, 1] *= 2.0 ** -100
    q[:, 2, :64] *= 2.0 ** -40
    q[:, 3] *= 64.0
    check_attention(w, q, None, run_attention(w, q, None))


@pytest.mark.parametrize("dtype,T", [("f32", 1), ("f32", 9), ("bf16", 1), ("bf16", 7), ("bf16", 40), ("bf16", 100)])
@pytest.mark.parametrize("how", ["rising", "falling", "mixed", "tiny", "large", "zero first"])
def test_attention_of_values_of_any_size(dtype, T, how):
    """Values whose scales differ by many powers of two from token to token and tile to tile."""
    w = World(4700 + T, dtype, 2, 2, 128, T, [0], 32, 32)
    n = 400
    w.past[0] = n
    w.table_pages = -(-(n + T) // 32)
    w.table = w.rng.permutation(w.table_pages + 2)[:w.table_pages].reshape(1, -1).astype(np.int32)
    for name, a in list(w.pool.items()):
        w.pool[name] = np.zeros((w.table_pages + 2,) + a.shape[1:], a.dtype)
    size = {"rising": np.linspace(-40, 10, n + T), "falling": np.linspace(10, -40, n + T), "mixed": w.rng.uniform(-12, 12, n + T),
            "tiny": np.full(n + T, -100.0), "large": np.full(n + T, 90.0), "zero first": np.zeros(n + T)}[how]
    v = w.normal(n + T, 2, 128) * 2.0 ** size[:, None, None]
    if how == "zero first":
        v[:200] = 0.0
    oc.append(w.pool, w.table, 32, 0, 0, w.normal(n + T, 2, 128), v, 32)
    q = w.normal(T, 2, 128)
    for max_len in (64, 1024):
        check_attention(w, q, None, run_attention(w, q, None, max_len))


@pytest.mark.parametrize("dtype,T", [("f32", 1), ("bf16", 1), ("bf16", 80)])
def test_what_is_no_number_reaches_the_rows_that_see_it(dtype, T):
    w = World(4500 + T, dtype, 2, 2, 64, T, [100, 30], 16, 32)
    for b in range(2):
        oc.append(w.pool, w.table, 16, b, int(w.past[b]), w.normal(T, 2, 64), w.normal(T, 2, 64), 32)
    q = w.normal(2 * T, 2, 64)
    q[0, 0, 5] = np.nan
    w.pool["v_scales"][w.table[1, 1], 1, 0, 3] = np.nan                  # a value of the second sequence's head 1
    w.pool["k_scales"][w.table[1, 1], 0, 0, 3] = np.nan                  # a key of its head 0
    got = run_attention(w, q, None)
    assert np.all(np.isnan(got[0, 0, 0])) and np.all(np.isnan(got[1]))
    assert np.all(np.isfinite(got[0, 0, 1])) and np.all(np.isfinite(got[0, 1:]))


@pytest.mark.parametrize("dtype,T,past", [("f32", 3, 900), ("bf16", 1, 9000), ("bf16", 20, 700), ("bf16", 140, 300)])
def test_attention_does_not_depend_on_the_given_bound_beyond_rounding_and_repeats(dtype, T, past):
    w = World(5000 + T, dtype, 4, 4, 64, T, [past, past // 3], 32, 16)
    for b in range(w.B):
        oc.append(w.pool, w.table, 32, b, int(w.past[b]), w.normal(T, 4, 64), w.normal(T, 4, 64), 16)
    q = w.normal(w.B * T, 4, 64)
    for max_len in (0, 1, past + T, 1 << 29):                            # also far too small and far too large
        a = run_attention(w, q, None, max_len)
        check_attention(w, q, None, a)
        assert np.array_equal(a, run_attention(w, q, None, max_len))


def test_pools_beyond_32_bits():
    """A pool of more than 4 GiB of codes: the sequence's pages lie at its two ends."""
    import paper_2301_11913_amd as sw
    KV, dh, page, T = 8, 128, 1024, 3
    pages = (5 << 30) // (KV * dh * page)
    w = World(6000, "bf16", 8, KV, dh, T, [2000], page, 32)
    oc.append(w.pool, w.table, page, 0, 2000, w.normal(T, KV, dh), w.normal(T, KV, dh), 32)
    small = w.table.copy()
    where = np.array([[pages - 1, 0, pages - 2][:w.table_pages]], dtype=np.int32)
    cfg = sw.CacheConfig(8, KV, dh, page, pages, 1, w.table_pages, "bf16", 32)
    dev = {n: torch.empty(shape, dtype=dt, device="cuda") for n, (shape, dt) in cfg.shapes().items()}
    for i in range(w.table_pages):
        for n in dev:
            dev[n][where[0, i]] = torch.from_numpy(w.pool[n][small[0, i]]).cuda()
    cache = sw.Cache(cfg, **dev)
    q = w.normal(T, 8, dh)
    out = torch.full((T, 8 * dh), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(sw.swarm_cache_attention_workspace_bytes(cfg, T, 2003), dtype=torch.uint8, device="cuda")
    table, past = w.ints(where), w.ints(w.past)
    sw.swarm_cache_attention(cfg, cache, table, past, None, T, w.dev(q.reshape(T, -1)), out, ws, max_len=2003)
    torch.cuda.synchronize()
    check_attention(w, q, None, out.double().cpu().numpy().reshape(1, T, 8, dh))
    x = w.dev(w.normal(T, KV * dh))
    sw.swarm_cache_append(cfg, cache, table, past, None, T, x, x)
    back = [torch.empty((T, KV * dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    sw.swarm_cache_read(cfg, cache, table, past, None, T, *back)
    torch.cuda.synchronize()
    # half a code step of a block of 64: its largest magnitude / 254, and a bf16 rounding
    top = x.float().reshape(T, -1, 64).abs().amax(2, keepdim=True)
    for got in back:
        off = (got.float() - x.float()).reshape(T, -1, 64).abs()
        assert bool((off <= top * (1 / 254 + 2.0 ** -8) * 1.0001).all())


def test_calls_on_another_stream():
    """Work goes to the stream that is given, or to torch's current one."""
    import paper_2301_11913_amd as sw
    T = 4
    w = World(6500, "bf16", 4, 4, 64, T, [100, 50], 16, 32)
    cfg, cache = w.upload()
    x = w.normal(w.B * T, 3 * 4 * 64)
    q, k, v = w.dev(x).split(256, 1)
    table, past = w.ints(w.table), w.ints(w.past)
    ws = torch.empty(sw.swarm_cache_attention_workspace_bytes(cfg, T, 0), dtype=torch.uint8, device="cuda")
    outs = []
    for how in ("given", "current", "default"):
        out = torch.zeros((w.B * T, 256), dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        call = lambda st: (sw.swarm_cache_append(cfg, cache, table, past, None, T, k, v, stream=st),  # noqa: E731
                           sw.swarm_cache_attention(cfg, cache, table, past, None, T, q, out, ws, stream=st))
        if how == "given":
            call(s)
        elif how == "current":
            with torch.cuda.stream(s):
                call(None)
        else:
            call(None)
        torch.cuda.synchronize()
        outs.append(out.clone())
    assert bool((outs[0] != 0).any()) and torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_a_decoding_step_replays_from_a_graph():
    """append, attention and keep recorded once, replayed with new inputs and lengths in the same buffers; every replay against
    the eager calls."""
    import paper_2301_11913_amd as sw
    T, H, dh = 5, 4, 128
    w = World(6600, "bf16", H, H, dh, T, [700, 61], 32, 32)
    cfg, cache = w.upload()
    _, eager = w.upload()
    x = w.dev(w.normal(w.B * T, 3 * H * dh))
    q, k, v = x.split(H * dh, 1)
    table, past, n_kept = w.ints(w.table), w.ints(w.past), w.ints([2, 2])
    tree = torch.from_numpy(tree_words(w.rng, w.B, T).view(np.int64)).cuda()
    kept = w.ints(np.tile(np.arange(T), (w.B, 1)))
    q_out, out = (torch.zeros((w.B * T, H * dh), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    max_len = 1024
    ws = torch.empty(sw.swarm_cache_attention_workspace_bytes(cfg, T, max_len), dtype=torch.uint8, device="cuda")

    def step(pool):
        sw.swarm_cache_append(cfg, pool, table, past, None, T, k, v, q=q, q_out=q_out, rotary=True)
        sw.swarm_cache_attention(cfg, pool, table, past, None, T, q_out, out, ws, tree=tree, max_len=max_len)
        sw.swarm_cache_keep(cfg, pool, table, past, kept, n_kept, T)

    step(eager)                                                           # once outside a capture
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step(cache)
    torch.cuda.synchronize()
    for i in range(4):
        x.copy_(w.dev(w.normal(w.B * T, 3 * H * dh)))
        kept.copy_(w.ints(np.stack([np.sort(w.rng.permutation(T)) for _ in range(w.B)])))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, out) and same_pool(pool_of(cache), pool_of(eager))
        past.add_(2)
