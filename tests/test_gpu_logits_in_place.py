"""swarm_logits_adjust where the output is the input: the same values as in another place, to the bit."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from test_gpu_logits import bits_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,vocab,history,biases,pad", [
    (1, 1, 1, 1, 0), (4, 31, 64, 8, 0), (2, 4127, 3000, 300, 0), (3, 4096, 900, 20, 0), (5, 2049, 700, 0, 3), (3, 8192, 0, 40, 1), (7, 50257, 200, 9, 175)])
def test_in_place(rows, vocab, history, biases, pad):
    import paper_2301_11913_amd as sw
    rng = np.random.default_rng(vocab + history)
    x = (rng.standard_normal((rows, vocab + pad)) * 4).astype(np.float32)
    hist = rng.integers(0, vocab, (rows, max(history, 1))).astype(np.int32)
    ids = rng.integers(0, vocab, (rows, max(biases, 1))).astype(np.int32)
    val = rng.standard_normal(ids.shape).astype(np.float32) * 5
    rep, freq, pres = (1 + rng.random(rows)).astype(np.float32), rng.random(rows).astype(np.float32), rng.random(rows).astype(np.float32)
    allowed = rng.random((rows, vocab)) < 0.7
    g = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    full = lambda n: torch.full((rows,), n, dtype=torch.int32, device="cuda")  # noqa: E731
    rules = sw.LogitsRules(rows, vocab, history=g(hist) if history else None, history_len=full(history) if history else None,
                           repetition=g(rep), frequency=g(freq), presence=g(pres), bias_ids=g(ids) if biases else None,
                           bias=g(val) if biases else None, bias_len=full(biases) if biases else None, allowed=g(bits_of(allowed)))
    src = g(x)
    out = torch.full_like(src, 7.0)
    sw.swarm_logits_adjust(rules, src, out)
    assert torch.equal(src.cpu(), torch.from_numpy(x))                   # the input is left as it was
    sw.swarm_logits_adjust(rules, src, src)
    torch.cuda.synchronize()
    assert torch.equal(src[:, :vocab], out[:, :vocab])
    assert torch.equal(src[:, vocab:].cpu(), torch.from_numpy(x[:, vocab:]))
    if vocab > 1:                                                        # and not what they were: something was asked for in every row
        assert bool((src[:, :vocab].cpu() != torch.from_numpy(x[:, :vocab])).any(1).all())
    for r in range(rows):
        want = oc.adjust(x[r, :vocab].astype(np.float64), hist[r, :history], float(rep[r]), float(freq[r]), float(pres[r]), ids[r, :biases],
                         val[r, :biases].astype(np.float64), allowed[r])
        got = src[r, :vocab].double().cpu().numpy()
        fine = np.isfinite(want)
        assert np.array_equal(np.isfinite(got), fine)
        # six roundings of 2^-24 of no more than the terms' magnitudes
        big = 6 * 2.0 ** -24 * (2 * np.abs(x[r, :vocab]).max() + freq[r] * history + pres[r] + np.abs(val[r, :biases]).sum())
        assert np.all(np.abs(got[fine] - want[fine]) <= big)
