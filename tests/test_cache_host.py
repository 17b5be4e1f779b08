"""Host-only checks of the cache, extend and logits calls: what they refuse, before anything is launched."""
import ctypes as C
import os

import pytest
import torch

import paper_2301_11913_amd as sw
from paper_2301_11913_amd import binding

NULL, SHAPE, DTYPE, WORKSPACE = -1, -2, -3, -4
A = 1 << 20                        # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sw.lib_path()):
        pytest.skip("libswarm_stage.so not built")
    return sw.load_library()


def config(**other):
    values = dict(n_heads=8, n_kv_heads=4, d_head=64, page_tokens=16, n_pages=10, batch=2, table_pages=5, dtype="bf16", scale_bits=32)
    values.update(other)
    return sw.CacheConfig(**values)


def pool(**other):
    values = dict(k_codes=A, v_codes=A, k_scales=A, v_scales=A)
    values.update(other)
    return binding._Cache(**values)


BAD = [("n_heads", 6), ("n_heads", 0), ("n_kv_heads", 0), ("n_heads", 2048), ("d_head", 96), ("d_head", 32), ("page_tokens", 8),
       ("page_tokens", 48), ("page_tokens", 1 << 17), ("n_pages", 0), ("batch", 0), ("table_pages", 0), ("table_pages", 1 << 27),
       ("scale_bits", 8)]


def calls(lib, cfg, cache, tokens=3, **other):
    """The status of every call of the cache with otherwise good arguments; `other` replaces some by name."""
    v = dict(table=A, past=A, fresh=A, q=A, k=A, v=A, pitch=1024, positions=None, rotary=1, q_out=A, q_out_pitch=512, k_out=A,
             v_out=2 * A, kept=A, n_kept=A, max_len=80, q_pitch=512, tree=None, out=2 * A, out_pitch=512, ws=A, ws_bytes=1 << 30)
    v.update(other)
    ref, pref = C.byref(cfg.c), C.byref(cache) if cache is not None else None
    return {
        "append": lambda: lib.swarm_cache_append(ref, pref, v["table"], v["past"], v["fresh"], tokens, v["q"], v["k"], v["v"], v["pitch"],
                                                 v["positions"], v["rotary"], v["q_out"], v["q_out_pitch"], None),
        "read": lambda: lib.swarm_cache_read(ref, pref, v["table"], v["past"], v["fresh"], tokens, v["k_out"], v["v_out"], None),
        "keep": lambda: lib.swarm_cache_keep(ref, pref, v["table"], v["past"], v["kept"], v["n_kept"], tokens, None),
        "attention": lambda: lib.swarm_cache_attention(ref, pref, v["table"], v["past"], v["fresh"], tokens, v["max_len"], v["q"],
                                                       v["q_pitch"], v["tree"], v["out"], v["out_pitch"], v["ws"], v["ws_bytes"], None)}


@pytest.mark.parametrize("name,value", BAD)
def test_configurations_that_are_none(lib, name, value):
    cfg = config(**{name: value})
    assert sw.swarm_cache_attention_workspace_bytes(cfg, 3, 80) == 0
    for call in calls(lib, cfg, pool()).values():
        assert call() == SHAPE


def test_dtype_tokens_and_null(lib):
    cfg = config()
    cfg.c.dtype = 7
    assert all(call() == DTYPE for call in calls(lib, cfg, pool()).values())
    cfg = config()
    shared = config(n_heads=1024, n_kv_heads=1, batch=1)
    assert calls(lib, shared, pool(), (1 << 14) + 1, q_pitch=1 << 16, out_pitch=1 << 16)["attention"]() == SHAPE
    assert sw.swarm_cache_attention_workspace_bytes(shared, (1 << 14) + 1, 80) == 0
    for tokens in (0, -1, (1 << 23) + 1):
        assert all(call() == SHAPE for call in calls(lib, cfg, pool(), tokens).values())
    assert all(call() == NULL for call in calls(lib, cfg, None).values())
    for field in ("k_codes", "v_codes", "k_scales", "v_scales"):
        assert all(call() == NULL for call in calls(lib, cfg, pool(**{field: None})).values())
        assert all(call() == SHAPE for call in calls(lib, cfg, pool(**{field: A + 8})).values())
    for field in ("table", "past"):
        assert all(call() == NULL for call in calls(lib, cfg, pool(), **{field: None}).values())


@pytest.mark.parametrize("name,status,other", [
    ("append", NULL, dict(k=None)), ("append", NULL, dict(v=None)), ("append", NULL, dict(q=None)), ("append", NULL, dict(q_out=None)),
    ("append", SHAPE, dict(rotary=0)),                                   # q and q_out without a rotation
    ("append", SHAPE, dict(rotary=0, q=None, q_out=None, positions=A)),
    ("append", SHAPE, dict(pitch=511)), ("append", SHAPE, dict(pitch=1028)), ("append", SHAPE, dict(k=A + 2)),
    ("append", SHAPE, dict(q_out_pitch=256)), ("append", SHAPE, dict(q=2 * A, q_out=2 * A)),
    ("read", NULL, dict(k_out=None)), ("read", NULL, dict(v_out=None)), ("read", SHAPE, dict(k_out=A + 4)), ("read", SHAPE, dict(v_out=A)),
    ("keep", NULL, dict(kept=None)), ("keep", NULL, dict(n_kept=None)), ("keep", SHAPE, dict(tokens=65)),
    ("attention", NULL, dict(q=None)), ("attention", NULL, dict(out=None)), ("attention", SHAPE, dict(max_len=-1)),
    ("attention", SHAPE, dict(tokens=65, tree=A)), ("attention", SHAPE, dict(tree=A + 4)), ("attention", SHAPE, dict(out=A)),
    ("attention", SHAPE, dict(q_pitch=511)), ("attention", SHAPE, dict(q_pitch=516)), ("attention", SHAPE, dict(out_pitch=500)),
    ("attention", SHAPE, dict(ws=A + 128)), ("attention", SHAPE, dict(q=A + 8))])
def test_arguments_that_do_not_fit(lib, name, status, other):
    other = dict(other)
    assert calls(lib, config(), pool(), other.pop("tokens", 3), **other)[name]() == status


def test_attention_workspace(lib):
    """Long sequences of few rows are spread over workgroups, which leave partial results: no more than the size that is asked for."""
    cfg = config(table_pages=4096, page_tokens=16, n_pages=8192)
    need = sw.swarm_cache_attention_workspace_bytes(cfg, 1, 0)
    assert need % 256 == 0 and need <= 64 << 20
    if need:
        assert calls(lib, cfg, pool(), 1, max_len=0, ws_bytes=need - 1)["attention"]() == WORKSPACE
        assert calls(lib, cfg, pool(), 1, max_len=0, ws=None, ws_bytes=0)["attention"]() == NULL


def test_extend_refuses(lib):
    cfg = sw.StageConfig(256, 4, 512, 1, 2, 2, 3, "bf16", block_kind="rotary_geglu")
    cc = config(n_heads=4, n_kv_heads=4)
    assert sw.swarm_stage_extend_workspace_bytes(cfg, cc, 80) >= sw.swarm_stage_workspace_bytes(cfg, False) > 0
    params = (binding._BlockPtrs * 1)(binding._BlockPtrs(*[A] * 12))
    pools = (binding._Cache * 2)(pool(), pool())

    def call(cfg=cfg, cc=cc, params=params, pools=pools, positions=None, tree=None, x_in=A, x_out=2 * A, ws=A, n=1 << 40):
        return lib.swarm_stage_extend(C.byref(cfg.c), params, C.byref(cc.c), pools, A, A, None, positions, tree, 80, x_in, x_out, ws, n, None)

    assert call(n=100) == WORKSPACE
    assert call(x_in=None) == NULL and call(ws=None) == NULL
    assert call(params=(binding._BlockPtrs * 1)()) == NULL
    assert call(pools=(binding._Cache * 2)(pool(), pool(v_scales=None))) == NULL
    assert call(pools=(binding._Cache * 2)(pool(), pool(v_scales=A + 4))) == SHAPE
    assert call(x_out=A) == SHAPE and call(x_in=A + 8) == SHAPE and call(ws=A + 16) == SHAPE and call(tree=A + 4) == SHAPE
    for other in (dict(batch=3), dict(n_heads=8, n_kv_heads=4), dict(n_heads=2, n_kv_heads=2), dict(d_head=128), dict(dtype="f32"),
                  dict(page_tokens=24)):
        assert call(cc=config(**dict(dict(n_heads=4, n_kv_heads=4), **other))) == SHAPE
        assert sw.swarm_stage_extend_workspace_bytes(cfg, config(**dict(dict(n_heads=4, n_kv_heads=4), **other)), 80) == 0
    gelu = sw.StageConfig(256, 4, 512, 1, 2, 2, 3, "bf16")
    assert call(cfg=gelu, positions=A) == SHAPE
    assert call(cfg=sw.StageConfig(256, 4, 512, 1, 2, 2, 65, "bf16"), tree=A) == SHAPE


def test_logits_refuse(lib):
    fields = [n for n, _ in binding._LogitsRules._fields_]

    def call(dtype=1, logits=A, pitch=100, out=2 * A, out_pitch=100, **other):
        v = dict(rows=2, vocab=100, history_max=4, bias_max=4, history=A, history_len=A, repetition=A, frequency=A, presence=A, bias_ids=A,
                 bias=A, bias_len=A, allowed=A)
        v.update(other)
        return lib.swarm_logits_adjust(C.byref(binding._LogitsRules(*(v[n] for n in fields))), logits, dtype, pitch, out, out_pitch, None)

    for other in (dict(logits=None), dict(out=None), dict(history_len=None), dict(bias=None), dict(bias_len=None)):
        assert call(**other) == NULL
    assert call(dtype=5) == DTYPE
    for other in (dict(rows=0), dict(rows=65536), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(history_max=-1), dict(history_max=1 << 20), dict(bias_max=-1),
                  dict(bias_max=1025), dict(pitch=99), dict(out_pitch=99), dict(logits=A + 1), dict(out=A + 2), dict(out=A)):
        assert call(**other) == SHAPE
    assert call(dtype=0, out=A, out_pitch=101) == SHAPE                   # in place with another pitch


def test_head_logits_refuse(lib):
    cfg = sw.HeadConfig(64, 50, 56, 3, "f32")
    good = binding._Ptrs3(A, A, A)
    call = lambda p=good, x=A, out=2 * A, ws=A, n=1 << 30: lib.swarm_head_logits(C.byref(cfg.c), C.byref(p), x, out, ws, n, None)  # noqa: E731
    assert call(p=binding._Ptrs3(A, A, None)) == NULL and call(x=None) == NULL and call(out=None) == NULL
    assert call(out=A) == SHAPE and call(x=A + 8) == SHAPE and call(out=A + 8) == SHAPE and call(ws=A + 4) == SHAPE
    assert call(n=10) == WORKSPACE


def test_binding_checks_tensors(monkeypatch):
    """Shapes and types that the C side cannot see are refused by the binding."""
    cfg = config()
    make = lambda c: sw.Cache(c, **{n: torch.zeros(s, dtype=d) for n, (s, d) in c.shapes().items()})  # noqa: E731
    cache = make(cfg)
    with pytest.raises(ValueError):
        sw.Cache(config(n_pages=11), **cache.tensors)
    with pytest.raises(TypeError):
        sw.Cache(config(scale_bits=16), **cache.tensors)
    table, past = torch.zeros((2, 5), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    k = torch.zeros((6, 256), dtype=torch.bfloat16)
    q = torch.zeros((6, 512), dtype=torch.bfloat16)
    ok = (cfg, cache, table, past, None, 3)
    append, attention = sw.swarm_cache_append, sw.swarm_cache_attention
    wide = torch.zeros((6, 300), dtype=torch.bfloat16)[:, :256]
    for why, call in [
            ("page_table must be", lambda: append(cfg, cache, table.long(), past, None, 3, k, k)),
            ("page_table has 8 elements", lambda: append(cfg, cache, table[:, :4].contiguous(), past, None, 3, k, k)),
            ("past has 1 elements", lambda: append(cfg, cache, table, past[:1], None, 3, k, k)),
            ("fresh must be", lambda: append(cfg, cache, table, past, past.float(), 3, k, k)),
            ("k has shape", lambda: append(cfg, cache, table, past, None, 4, k, k)),
            ("k must be", lambda: append(*ok, k.float(), k)),
            ("k has shape", lambda: append(*ok, k[:, :128], k)),
            ("same row pitch", lambda: append(*ok, k, wide)),
            ("another configuration", lambda: append(cfg, make(config(n_pages=9)), table, past, None, 3, k, k)),
            ("not on the current GPU", lambda: append(*ok, k, k)),
            ("k_out has", lambda: sw.swarm_cache_read(cfg, cache, table, past, None, 4, k, k)),
            ("k_out must be", lambda: sw.swarm_cache_read(cfg, cache, table, past, None, 3, k.float(), k)),
            ("kept has 4 elements", lambda: sw.swarm_cache_keep(cfg, cache, table, past, torch.zeros((2, 2), dtype=torch.int32), past, 3)),
            ("tree must be", lambda: attention(*ok, q, q.clone(), None, tree=torch.zeros((2, 3), dtype=torch.int32))),
            ("tree has 4 elements", lambda: attention(*ok, q, q.clone(), None, tree=torch.zeros((2, 2), dtype=torch.int64))),
            ("out must be contiguous|elements of a row of out", lambda: attention(*ok, q, q.clone().t().contiguous().t(), None)),
            ("another configuration", lambda: attention(cfg, make(config(page_tokens=32)), table, past, None, 3, q, q.clone(), None)),
            ("history must be", lambda: sw.LogitsRules(2, 100, history=torch.zeros((2, 3)), history_len=past)),
            ("allowed has shape", lambda: sw.LogitsRules(2, 100, allowed=torch.zeros((2, 3), dtype=torch.int32))),
            ("vocab or more", lambda: sw.swarm_logits_adjust(sw.LogitsRules(2, 100), torch.zeros((2, 99)), torch.zeros((2, 100)))),
            ("out must be", lambda: sw.swarm_logits_adjust(sw.LogitsRules(2, 100), torch.zeros((2, 100)),
                                                           torch.zeros((2, 100), dtype=torch.bfloat16)))]:
        with monkeypatch.context() as m:
            if why != "not on the current GPU":
                m.setattr(binding, "_device", lambda: -1)               # as if the tensors' device, the CPU, were the current one
            with pytest.raises((ValueError, TypeError), match=why):
                call()
