"""Generation with a stage: swarm_stage_extend over prompts of different lengths, single tokens and a drafted tree whose accepted
tokens are kept, then the head's logits and the rules on them, against the oracle at every step."""
import numpy as np
import pytest
import torch

import swarm_synth as synth
from cache_util import pool_of, same_pool
from oracle import cache as oc
from oracle import stage as osg
from stage_util import max_norm_err, to_dev

pytestmark = pytest.mark.gpu


class Generator:
    """The oracle's side: float64 blocks over the pools' values, which each append puts through the codec."""

    def __init__(self, wl, params, pools, table, page, scale_bits):
        self.wl, self.params, self.pools, self.table, self.page, self.bits = wl, params, pools, table, page, scale_bits

    def extend(self, b, past, x, pos, see):
        """x [n, d] of sequence b; see [n, n] among the new tokens."""
        wl, H = self.wl, self.wl.n_heads
        d, n, dh = wl.d_model, x.shape[0], wl.d_model // wl.n_heads
        app = 0
        for p in self.params:
            p = {k: np.asarray(a, dtype=np.float64) for k, a in p.items()}
            for _ in range(wl.n_repeat):
                a, _, _ = osg.layernorm_fwd(x, p["ln1_g"], p["ln1_b"], wl.ln_eps)
                q, k, v = ((a @ p["w_qkv"].T + p["b_qkv"])[:, i * d:(i + 1) * d].reshape(n, H, dh) for i in range(3))
                if wl.block == "rotary_geglu":
                    q, k = oc.rotate(q, pos), oc.rotate(k, pos)
                oc.append(self.pools[app], self.table, self.page, b, past, k, v, self.bits)
                kc, vc, _ = oc.read(self.pools[app], self.table, self.page, b, list(range(past + n)))
                o, _, _ = oc.attention(q, kc, vc, np.concatenate([np.ones((n, past), dtype=bool), see], 1))
                h = x + o.reshape(n, d) @ p["w_o"].T + p["b_o"]
                c, _, _ = osg.layernorm_fwd(h, p["ln2_g"], p["ln2_b"], wl.ln_eps)
                u = c @ p["w_1"].T + p["b_1"]
                g = osg.gelu(u[:, :wl.d_ffn]) * u[:, wl.d_ffn:] if wl.block == "rotary_geglu" else osg.gelu(u)
                x = h + g @ p["w_2"].T + p["b_2"]
                app += 1
        return x


@pytest.mark.parametrize("dtype,d,H,f,L,R,block,page,bits", [
    ("f32", 256, 4, 512, 2, 1, "gelu", 16, 32),
    ("f32", 128, 1, 256, 1, 2, "rotary_geglu", 32, 32),
    ("bf16", 256, 2, 512, 1, 3, "rotary_geglu", 16, 16),
    ("bf16", 512, 8, 1024, 2, 2, "gelu", 64, 32)])
def test_generation(dtype, d, H, f, L, R, block, page, bits):
    import paper_2301_11913_amd as sw
    bar = 1e-4 if dtype == "f32" else 2e-2
    B, dh, apps = 3, d // H, L * R
    wl = synth.Workload(name="extend", dtype=dtype, d_model=d, n_heads=H, d_ffn=f, seq=1, batch=B, n_layers=L, n_repeat=R,
                        grad_sigma=1.0, seed=d + f, block=block)
    params = synth.make_params(wl)
    dev_params = [{k: to_dev(p[k], wl) for k in sw.PARAM_FIELDS} for p in params]
    rng = np.random.default_rng(d + page)
    draw = lambda n: torch.from_numpy(rng.standard_normal((n, d)).astype(np.float32)).to(  # noqa: E731
        torch.float32 if dtype == "f32" else torch.bfloat16).double().numpy()
    table_pages = -(-80 // page)
    pages = B * table_pages
    table = rng.permutation(pages).reshape(B, table_pages).astype(np.int32)
    cc = sw.CacheConfig(H, H, dh, page, pages, B, table_pages, dtype, bits)
    caches = [sw.Cache(cc, **{n: torch.zeros(s, dtype=t, device="cuda") for n, (s, t) in cc.shapes().items()}) for _ in range(apps)]
    oracle = Generator(wl, params, [pool_of(c) for c in caches], table, page, bits)
    ints = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    table_d = ints(table)
    past = np.zeros(B, dtype=np.int32)

    def step(T, fresh, depth=None, words=None):
        """One call and the oracle's; the rows that are there agree."""
        cfg = sw.StageConfig(d, H, f, L, R, B, T, dtype, wl.ln_eps, block)
        x = draw(B * T)
        for b in range(B):
            x.reshape(B, T, d)[b, fresh[b]:] = np.nan if dtype == "f32" else 1e30        # what is not there reaches nothing
        xd = to_dev(x.astype(np.float32), wl)
        y = torch.zeros_like(xd)
        ws = torch.full((sw.swarm_stage_extend_workspace_bytes(cfg, cc, 80),), 255, dtype=torch.uint8, device="cuda")
        pos = past[:, None] + (np.arange(T)[None] if depth is None else depth)
        given = ints(pos) if depth is not None and block == "rotary_geglu" else None
        tree = None if words is None else torch.from_numpy(words.view(np.int64)).cuda()
        sw.swarm_stage_extend(cfg, dev_params, cc, caches, table_d, ints(past), ints(fresh), xd, y, ws, positions=given, tree=tree,
                              max_len=80)
        torch.cuda.synchronize()
        y = y.double().cpu().numpy().reshape(B, T, d)
        for b in range(B):
            n = fresh[b]
            if not n:
                continue
            see = np.tril(np.ones((n, n), dtype=bool))
            if words is not None:
                see = np.array([[bool(int(words[b, t]) >> u & 1) for u in range(n)] for t in range(n)])
            want = oracle.extend(b, int(past[b]), x.reshape(B, T, d)[b, :n], pos[b, :n], see)
            assert max_norm_err(y[b, :n], want) < bar
        return y

    step(37, [37, 20, 0])                                                # prompts, one not there yet
    past += [37, 20, 0]
    step(1, [1, 1, 1])
    past += 1
    # a tree of six: 0 - 1 - 2, 0 - 3 - 4, 5 beside 0
    parent, depth = [-1, 0, 1, 0, 3, -1], np.array([0, 1, 2, 1, 2, 0])
    words = np.zeros((B, 6), dtype=np.uint64)
    for t in range(6):
        words[:, t] = (words[:, parent[t]] if parent[t] >= 0 else np.uint64(0)) | (np.uint64(1) << np.uint64(t))
    step(6, [6, 6, 6], depth=depth, words=words)
    kept = np.tile(np.array([0, 3, 4, 0, 0, 0], dtype=np.int32), (B, 1))
    n_kept = np.array([3, 2, 1], dtype=np.int32)
    for i, c in enumerate(caches):
        sw.swarm_cache_keep(cc, c, table_d, ints(past), ints(kept), ints(n_kept), 6)
        for b in range(B):
            oc.keep(oracle.pools[i], table, page, b, int(past[b]), kept[b, :n_kept[b]], 6)
    past += n_kept
    y = step(1, [1, 1, 1])                                               # goes on behind the kept tokens
    if dtype == "f32":                                                   # codes: equal but for keys and values next to a border
        for c, want in zip(caches, oracle.pools):
            got = pool_of(c)
            off = np.abs(got["k_codes"].astype(int) - want["k_codes"].astype(int))
            assert off.max() <= 1 and off.mean() < 1e-3

    # the last stage: logits of the three tokens, a rule on them, the choice
    vocab, rows = 300, 320
    head = {"ln_g": np.ones(d), "ln_b": np.zeros(d), "w_vocab": rng.standard_normal((rows, d)) / np.sqrt(d)}
    head_d = {k: to_dev(a.astype(np.float32), wl) for k, a in head.items()}
    hc = sw.HeadConfig(d, vocab, rows, B, dtype)
    ws = torch.empty(sw.swarm_head_workspace_bytes(hc, False), dtype=torch.uint8, device="cuda")
    xd = to_dev(y.reshape(B, d).astype(np.float32), wl)
    logits = torch.zeros((B, rows), dtype=xd.dtype, device="cuda")
    sw.swarm_head_logits(hc, head_d, xd, logits, ws)
    top = logits[:, :vocab].float().argmax(1).int()
    allowed = torch.full((B, -(-vocab // 32)), -1, dtype=torch.int32, device="cuda")
    rules = sw.LogitsRules(B, vocab, history=top[:, None].contiguous(), history_len=ints(np.ones(B)),
                           repetition=torch.full((B,), 1e6, device="cuda"), allowed=allowed)
    out = torch.empty((B, vocab), device="cuda")
    sw.swarm_logits_adjust(rules, logits, out)
    second = logits[:, :vocab].float().scatter(1, top.long()[:, None], -np.inf).argmax(1)
    assert torch.equal(out.argmax(1), second)
    assert torch.equal(out.gather(1, second[:, None]), logits.float().gather(1, second[:, None]))


def test_extend_replays_from_a_graph():
    """One token at a time: recorded once, replayed while `past` grows on the device."""
    import paper_2301_11913_amd as sw
    d, H, f, B, page = 256, 2, 512, 2, 16
    wl = synth.Workload(name="extend_graph", dtype="bf16", d_model=d, n_heads=H, d_ffn=f, seq=1, batch=B, n_layers=1, n_repeat=2,
                        grad_sigma=1.0, seed=3, block="rotary_geglu")
    params = [{k: to_dev(p[k], wl) for k in sw.PARAM_FIELDS} for p in synth.make_params(wl)]
    cfg = sw.StageConfig(d, H, f, 1, 2, B, 1, "bf16", wl.ln_eps, "rotary_geglu")
    cc = sw.CacheConfig(H, H, 128, page, 2 * 8, B, 8, "bf16", 32)
    make = lambda: [sw.Cache(cc, **{n: torch.zeros(s, dtype=t, device="cuda") for n, (s, t) in cc.shapes().items()}) for _ in range(2)]  # noqa: E731
    table = torch.arange(16, dtype=torch.int32, device="cuda").reshape(2, 8)
    ws = torch.empty(sw.swarm_stage_extend_workspace_bytes(cfg, cc, 128), dtype=torch.uint8, device="cuda")
    x = torch.zeros((B, d), dtype=torch.bfloat16, device="cuda")
    y = torch.zeros_like(x)
    past = torch.zeros(B, dtype=torch.int32, device="cuda")
    replayed, eager = make(), make()
    run = lambda pools: sw.swarm_stage_extend(cfg, params, cc, pools, table, past, None, x, y, ws, max_len=128)  # noqa: E731
    run(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            run(replayed)
    torch.cuda.synchronize()
    gen = torch.Generator(device="cuda").manual_seed(5)
    for _ in range(20):
        x.copy_(torch.randn((B, d), generator=gen, device="cuda"))
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.zero_()
        run(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, y) and bool(torch.isfinite(y).all())
        past.add_(1)
    assert all(same_pool(pool_of(a), pool_of(b)) for a, b in zip(replayed, eager))
