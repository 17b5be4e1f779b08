"""Generation at its edges: one sequence of one token, rows of logits that start anywhere, a page table that ends with the tokens."""
import numpy as np
import pytest
import torch

import swarm_synth as synth
from cache_util import World, check_rows, pool_of, same_pool
from oracle import cache as oc
from stage_util import max_norm_err, to_dev
from test_gpu_cache import run_attention
from test_gpu_extend import Generator

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block", ["gelu", "rotary_geglu"])
@pytest.mark.parametrize("dtype,d,H,f", [("f32", 64, 1, 64), ("bf16", 64, 1, 64), ("bf16", 128, 1, 192), ("bf16", 1024, 16, 2048)])
def test_one_sequence_token_by_token(dtype, d, H, f, block):
    """From nothing to the end of its only page, without `fresh`, `max_len` and positions."""
    import paper_2301_11913_amd as sw
    bar, dh, page = 1e-4 if dtype == "f32" else 2e-2, d // H, 16
    wl = synth.Workload(name="edges", dtype=dtype, d_model=d, n_heads=H, d_ffn=f, seq=1, batch=1, n_layers=1, n_repeat=1, grad_sigma=1.0,
                        seed=d + f, block=block)
    params = synth.make_params(wl)
    dev = [{k: to_dev(p[k], wl) for k in sw.PARAM_FIELDS} for p in params]
    cfg = sw.StageConfig(d, H, f, 1, 1, 1, 1, dtype, wl.ln_eps, block)
    cc = sw.CacheConfig(H, H, dh, page, 1, 1, 1, dtype, 32)
    cache = sw.Cache(cc, **{n: torch.zeros(s, dtype=t, device="cuda") for n, (s, t) in cc.shapes().items()})
    table = np.zeros((1, 1), dtype=np.int32)
    oracle = Generator(wl, params, [pool_of(cache)], table, page, 32)
    ws = torch.full((sw.swarm_stage_extend_workspace_bytes(cfg, cc),), 255, dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(d)
    past = torch.zeros(1, dtype=torch.int32, device="cuda")
    for t in range(page):
        xd = to_dev(rng.standard_normal((1, d)).astype(np.float32), wl)
        y = torch.zeros_like(xd)
        sw.swarm_stage_extend(cfg, dev, cc, [cache], torch.zeros(1, 1, dtype=torch.int32, device="cuda"), past, None, xd, y, ws)
        torch.cuda.synchronize()
        want = oracle.extend(0, t, xd.double().cpu().numpy(), np.array([t]), np.ones((1, 1), dtype=bool))
        assert max_norm_err(y.double().cpu().numpy(), want) < bar
        past += 1
    y.fill_(7.0)                                                         # the page is full: the sequence is left out
    before = pool_of(cache)
    sw.swarm_stage_extend(cfg, dev, cc, [cache], torch.zeros(1, 1, dtype=torch.int32, device="cuda"), past, None, xd, y, ws)
    torch.cuda.synchronize()
    assert same_pool(before, pool_of(cache))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pitch,out_pitch", [(1, 8191, 8191), (3, 8193, 8195), (0, 8190, 8189)])
def test_logits_rows_that_start_anywhere(dtype, offset, pitch, out_pitch):
    """Odd pitches and first elements, columns of whole workgroups among them."""
    import paper_2301_11913_amd as sw
    rows, vocab = 4, 8189
    gen = torch.Generator(device="cuda").manual_seed(pitch)
    flat = torch.randn(offset + rows * pitch, generator=gen, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    x = flat[offset:].as_strided((rows, vocab), (pitch, 1))
    buf = torch.full((offset + rows * out_pitch,), 7.0, device="cuda")
    out = buf[offset:].as_strided((rows, vocab), (out_pitch, 1))
    seen = torch.randint(0, vocab, (rows, 50), generator=gen, device="cuda", dtype=torch.int32)
    rules = sw.LogitsRules(rows, vocab, history=seen, history_len=torch.full((rows,), 50, dtype=torch.int32, device="cuda"),
                           presence=torch.full((rows,), 2.0, device="cuda"))
    sw.swarm_logits_adjust(rules, x, out)
    want = x.float().clone()
    for r in range(rows):
        want[r, seen[r].long().unique()] -= 2.0
    assert torch.equal(out, want)
    left = torch.ones_like(buf, dtype=torch.bool)
    left[offset:].as_strided((rows, vocab), (out_pitch, 1)).fill_(False)
    assert bool((buf[left] == 7.0).all())


@pytest.mark.parametrize("dtype,T", [("f32", 5), ("bf16", 1), ("bf16", 7), ("bf16", 50)])
@pytest.mark.parametrize("page", [16, 64])
def test_a_table_that_ends_with_the_tokens(dtype, T, page):
    """past + tokens is all that the table can hold, and the last page of the pool is the last of the table."""
    past = 4 * page - T % page if T % page else 4 * page
    w = World(77 + T, dtype, 2, 2, 64, T, [past], page, 32, spare=0)
    assert w.table_pages * page == past + T
    pages = w.pool["k_codes"].shape[0]
    old = int(w.table[0, -1])
    w.table[0, -1] = pages - 1
    for name in w.pool:                                                  # what lay in the page moves with it
        w.pool[name][[old, pages - 1]] = w.pool[name][[pages - 1, old]]
    w.table[0, :-1][w.table[0, :-1] == pages - 1] = old
    oc.append(w.pool, w.table, page, 0, past, w.normal(T, 2, 64), w.normal(T, 2, 64), 32)
    q = w.normal(T, 2, 64)
    for max_len in (0, 64, past + T):
        check_rows(w, q, None, run_attention(w, q, None, max_len))


@pytest.mark.parametrize("rotary", [False, True])
@pytest.mark.parametrize("dtype,dh", [("f32", 64), ("bf16", 64), ("bf16", 128)])
def test_a_first_sequence_without_new_tokens(dtype, dh, rotary):
    """fresh 0 behind a past that ends anywhere: nothing of it is read or written, and what the others append is theirs.  The values lie at the
    start of an allocation of their own, in front of which there is nothing."""
    import paper_2301_11913_amd as sw
    T, KV, page = 3, 2, 16
    w = World(31, dtype, KV, KV, dh, T, [17, 40, 63, 130], page, 32, fresh=[0, 3, 0, 2])
    cfg, cache = w.upload()
    x = w.normal(w.B * T, KV * dh)
    big = torch.empty((32 << 20,), dtype=w.dev(x).dtype, device="cuda")
    v = big[:w.B * T * KV * dh].reshape(w.B * T, KV * dh)
    v.copy_(w.dev(x))
    args = (cfg, cache, w.ints(w.table), w.ints(w.past), w.ints(w.fresh), T)
    if rotary:
        q = torch.zeros_like(v)
        sw.swarm_cache_append(*args, v.clone(), v, q=q, q_out=q, positions=torch.zeros(w.B * T, dtype=torch.int32, device="cuda"), rotary=True)
    else:
        sw.swarm_cache_append(*args, v, v)
    torch.cuda.synchronize()
    for b in range(w.B):
        n = int(w.fresh[b])
        rows = x.reshape(w.B, T, KV, dh)[b, :n]
        if n:
            oc.append(w.pool, w.table, page, b, int(w.past[b]), rows, rows, 32)
    assert same_pool(pool_of(cache), w.pool)
    out = [torch.full((w.B * T, KV * dh), 7.0, dtype=v.dtype, device="cuda") for _ in range(2)]
    sw.swarm_cache_read(*args, *out)
    got = out[1].double().cpu().numpy().reshape(w.B, T, -1)
    assert np.all(got[[0, 2]] == 7.0) and np.all(got[3, 2] == 7.0) and np.all(got[1] != 7.0)
