"""Rules on logits, and the head's logits, against the oracle."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from oracle.stage import layernorm_fwd

pytestmark = pytest.mark.gpu


def bits_of(allowed):
    rows, vocab = allowed.shape
    words = -(-vocab // 32)
    padded = np.zeros((rows, words * 32), dtype=np.uint64)
    padded[:, :vocab] = allowed
    return (padded.reshape(rows, words, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)


def check(got, want, x, what):
    """fp32: a division or product, a product and two differences, a sum over the biases, each half a step of a value no larger than
    the terms' magnitudes."""
    fine = np.isfinite(want)
    assert np.array_equal(np.isneginf(got), np.isneginf(want)) and np.all(np.isfinite(got) == fine)
    tol = 2.0 ** -24 * what
    assert np.all(np.abs(got[fine] - want[fine]) <= tol[fine])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,history,biases,pads", [
    (1, 1, 1, 1, (0, 0)), (1, 50257, 171, 16, (175, 0)), (3, 2048, 0, 5, (0, 3)), (5, 2049, 700, 0, (7, 0)), (2, 4127, 3000, 300, (1, 1)),
    (4, 31, 64, 8, (0, 0))])
def test_rules(dtype, rows, vocab, history, biases, pads):
    import paper_2301_11913_amd as sw
    rng = np.random.default_rng(rows * vocab + history)
    t = torch.from_numpy(rng.standard_normal((rows, vocab + pads[0])).astype(np.float32) * 4)
    t[:, 0] = 0.0
    if vocab > 40:
        t[0, 7], t[0, 8] = -np.inf, 0.0
    t = t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    x = t.double().numpy()[:, :vocab]
    hist = rng.integers(-3, vocab + 3, (rows, max(history, 1))).astype(np.int32)      # some are no tokens
    if vocab > 40:
        hist[:, : history // 2] %= 40                                                  # many are often there
    hist_len = rng.integers(0, history + 1, rows).astype(np.int32)
    hist_len[0] = history + 5                                                          # counts as all of them
    ids = rng.integers(-2, vocab + 2, (rows, max(biases, 1))).astype(np.int32)
    if biases > 3:
        ids[:, 2] = ids[:, 0]                                                          # the same one twice
    val = rng.standard_normal(ids.shape).astype(np.float32) * 5
    n_bias = np.full(rows, biases, dtype=np.int32)
    n_bias[-1] = -1 if rows > 1 else biases                                            # none
    rep = (1 + rng.random(rows)).astype(np.float32)
    freq, pres = rng.random(rows).astype(np.float32), rng.random(rows).astype(np.float32)
    allowed = rng.random((rows, vocab)) < 0.7
    if rows > 2:
        allowed[1] = False                                                             # nothing at all
        allowed[2] = True
    g = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    rules = sw.LogitsRules(rows, vocab, history=g(hist) if history else None, history_len=g(hist_len) if history else None,
                           repetition=g(rep), frequency=g(freq), presence=g(pres), bias_ids=g(ids) if biases else None,
                           bias=g(val) if biases else None, bias_len=g(n_bias) if biases else None, allowed=g(bits_of(allowed)))
    src = t.cuda()
    out = torch.full((rows, vocab + pads[1]), 7.0, device="cuda")
    sw.swarm_logits_adjust(rules, src, out)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    assert np.all(got[:, vocab:] == 7.0)
    for r in range(rows):
        n = min(max(int(hist_len[r]), 0), history)
        m = min(max(int(n_bias[r]), 0), biases)
        want = oc.adjust(x[r], hist[r, :n], float(rep[r]), float(freq[r]), float(pres[r]), ids[r, :m], val[r, :m].astype(np.float64), allowed[r])
        big = np.where(np.isfinite(x[r]), np.abs(x[r]), 0.0) * 2.0
        big = 6 * (big + freq[r] * n + pres[r] + np.abs(val[r, :m]).sum())
        check(got[r, :vocab], want, x[r], big)
    if dtype == "f32" and not pads[0]:                                                 # in place: the same
        sw.swarm_logits_adjust(rules, src, src)
        torch.cuda.synchronize()
        assert torch.equal(src, out[:, :vocab]) or bool((torch.isnan(src) == torch.isnan(out[:, :vocab])).all())


def test_no_rule_at_all_copies():
    import paper_2301_11913_amd as sw
    x = torch.randn((7, 333), device="cuda").to(torch.bfloat16)
    out = torch.zeros((7, 333), device="cuda")
    sw.swarm_logits_adjust(sw.LogitsRules(7, 333), x, out)
    assert torch.equal(out, x.float())


@pytest.mark.parametrize("dtype,d,vocab,vocab_rows,T", [("f32", 64, 50, 56, 3), ("bf16", 128, 500, 512, 1), ("bf16", 1024, 4000, 4096, 130)])
def test_head_logits(dtype, d, vocab, vocab_rows, T):
    """Products of LayerNormed rows; against the head's parity bars (max-normalised 1e-4 and 2e-2)."""
    import paper_2301_11913_amd as sw
    rng = np.random.default_rng(d)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    made = {"x": rng.standard_normal((T, d)), "ln_g": 1 + 0.1 * rng.standard_normal(d), "ln_b": 0.1 * rng.standard_normal(d),
            "w_vocab": rng.standard_normal((vocab_rows, d)) / np.sqrt(d)}
    dev = {n: torch.from_numpy(a.astype(np.float32)).to(dt).cuda() for n, a in made.items()}
    host = {n: t.double().cpu().numpy() for n, t in dev.items()}
    cfg = sw.HeadConfig(d, vocab, vocab_rows, T, dtype)
    ws = torch.empty(sw.swarm_head_workspace_bytes(cfg, False), dtype=torch.uint8, device="cuda")
    logits = torch.zeros((T, vocab_rows), dtype=dt, device="cuda")
    sw.swarm_head_logits(cfg, dev, dev["x"], logits, ws)
    torch.cuda.synchronize()
    n, _, _ = layernorm_fwd(host["x"], host["ln_g"], host["ln_b"], 1e-5)
    want = n @ host["w_vocab"].T
    off = np.abs(logits.double().cpu().numpy() - want).max() / np.abs(want).max()
    assert off < (1e-4 if dtype == "f32" else 2e-2)
