"""Pins of the generation oracle: rotation against the stage oracle's, attention over a cache against the stage oracle's causal
attention and closed forms, the pool's layout against the codec, the rules on logits against hand-made rows."""
import numpy as np

from oracle import cache as oc
from oracle import codec
from oracle import stage as osg


def empty_pool(pages, kv, page, dh):
    return {"k_codes": np.zeros((pages, kv, page, dh), np.int8), "v_codes": np.zeros((pages, kv, dh, page), np.int8),
            "k_scales": np.zeros((pages, kv, dh // 64, page), np.float32), "v_scales": np.zeros((pages, kv, dh // 64, page), np.float32)}


def test_rotation_is_the_stage_oracles():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((9, 3, 64))
    cos, sin = osg.rotary_angles(9, 64, np.float64)
    want = osg.rotary(x.transpose(1, 0, 2)[None], cos, sin)[0].transpose(1, 0, 2)
    assert np.allclose(oc.rotate(x, np.arange(9)), want, rtol=0, atol=1e-14)
    # a rotation: lengths of pairs stay, and q.k depends on the distance alone
    assert np.allclose((oc.rotate(x, np.full(9, 77)) ** 2).sum(2), (x ** 2).sum(2))
    a, b = x[:1], x[1:2]
    dot = lambda i, j: (oc.rotate(a, [i]) * oc.rotate(b, [j])).sum()  # noqa: E731
    assert abs(dot(5, 2) - dot(1005, 1002)) < 1e-10


def test_attention_is_causal_attention_and_shares_heads():
    rng = np.random.default_rng(2)
    q, k, v = (rng.standard_normal((7, 4, 64)) for _ in range(3))
    out, mean_abs, _ = oc.attention(q, k, v, np.tril(np.ones((7, 7), bool)))
    to = lambda x: x.transpose(1, 0, 2)[None]  # noqa: E731
    want, _ = osg.attention_fwd(to(q), to(k), to(v))
    assert np.allclose(out, want[0].transpose(1, 0, 2), rtol=0, atol=1e-13) and np.all(mean_abs >= np.abs(out) - 1e-13)
    shared, _, _ = oc.attention(q, k[:, :2], v[:, :2], np.ones((7, 7), bool))
    twice, _, _ = oc.attention(q, np.repeat(k[:, :2], 2, 1), np.repeat(v[:, :2], 2, 1), np.ones((7, 7), bool))
    assert np.array_equal(shared, twice)
    see = np.zeros((7, 7), bool)
    see[2, 5] = True                                                     # one token: its value; none: zeros
    out, _, _ = oc.attention(q, k, v, see)
    assert np.allclose(out[2], v[5]) and np.all(out[[0, 1, 3, 4, 5, 6]] == 0)


def test_append_read_and_keep():
    rng = np.random.default_rng(3)
    page, kv, dh = 16, 2, 128
    table = np.array([[3, 0], [2, 9]])                                   # page 9 is none of the pool's
    pool = empty_pool(4, kv, page, dh)
    k, v = (rng.standard_normal((12, kv, dh)).astype(np.float32) for _ in range(2))
    for b in range(2):
        oc.append(pool, table, page, b, 10, k, v, 32)
    got_k, got_v, there = oc.read(pool, table, page, 0, list(range(10, 22)))
    assert there.all()
    for got, x in ((got_k, k), (got_v, v)):
        assert np.allclose(got.reshape(-1), codec.decode(*codec.encode(x.reshape(-1))), rtol=2.0 ** -23, atol=0)
    assert np.array_equal(pool["v_codes"][0, :, :, 2], codec.encode(v.reshape(-1))[0].reshape(12, kv, dh)[8])
    assert list(oc.read(pool, table, page, 1, list(range(10, 22)))[2]) == [True] * 6 + [False] * 6
    before = oc.read(pool, table, page, 0, list(range(10, 22)))[0]
    oc.keep(pool, table, page, 0, 10, [3, 3, 11, 0, 99], 12)
    after = oc.read(pool, table, page, 0, list(range(10, 22)))[0]
    assert np.array_equal(after[:4], before[[3, 3, 11, 0]]) and np.array_equal(after[4:], before[4:])


def test_rules_on_logits():
    x = np.array([2.0, -2.0, 1.0, 0.0, 5.0])
    allowed = np.array([True, True, True, True, False])
    out = oc.adjust(x, [0, 1, 1, -1, 7], 2.0, 0.5, 0.25, [2, 2, 0, 9], [1.0, 2.0, -1.0, 5.0], allowed)
    assert np.array_equal(out, [2.0 / 2 - 0.5 - 0.25 - 1.0, -4.0 - 1.0 - 0.25, 4.0, 0.0, -np.inf])
