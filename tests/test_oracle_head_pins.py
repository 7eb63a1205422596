"""Pins of the oracle over the vocabulary: torch's own definitions in fp64, reverse-mode differentiation, closed forms."""
import math

import pytest
import torch

import oracle
from head_cases import rows

FINITE = ("plain", "peaked", "equal", "masked", "few", "one", "ties", "zeros")


@pytest.mark.parametrize("vocab,tau", [(1, 1.0), (2, 0.5), (7, 2.0), (300, 1.0), (1000, 0.7)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_log_probabilities_and_entropy(vocab, tau, dtype):
    z = rows(3, FINITE, vocab, dtype)
    T, n = len(FINITE), min(5, vocab)
    tgt = torch.randint(0, vocab, (T,), generator=torch.Generator().manual_seed(1)).int()
    tgt[0] = -1
    tgt[1] = vocab
    got = oracle.token_logprobs(z, tau, tgt, n)
    tau = float(torch.tensor(tau))
    lp = torch.log_softmax(z.double() / tau, 1)
    want = lp.gather(1, tgt.long().clamp(0, vocab - 1)[:, None])[:, 0]
    want[:2] = 0.0
    assert torch.allclose(got["logprob"], want, rtol=1e-12, atol=1e-13)
    assert torch.allclose(got["entropy"], torch.special.entr(lp.exp()).sum(1), rtol=1e-11, atol=1e-12)
    order = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :n]
    assert torch.equal(got["top_idx"].long(), order)
    assert torch.allclose(got["top_logprob"], lp.gather(1, order), rtol=1e-12, atol=1e-13)
    lse = got["stats"][:, 0] / tau + torch.log1p(got["stats"][:, 1])
    assert torch.allclose(lse, torch.logsumexp(z.double() / tau, 1), rtol=1e-13)


def test_rest_keeps_what_the_sum_loses():
    z = torch.tensor([[0.0, -60.0, -61.0]])
    got = oracle.token_logprobs(z, 1.0, torch.tensor([0], dtype=torch.int32), 0)
    assert got["logprob"].item() == pytest.approx(-(math.exp(-60) + math.exp(-61)), rel=1e-14)


def test_rows_without_a_distribution():
    z = rows(5, ("empty", "nan", "inf", "plain"), 9, torch.float32)
    tgt = torch.zeros(4, dtype=torch.int32)
    got = oracle.token_logprobs(z, 1.0, tgt, 3)
    assert got["logprob"][0] == -math.inf and got["entropy"][0] == 0.0 and got["stats"][0].tolist() == [-math.inf, -1.0]
    assert got["top_idx"][0].tolist() == [0, 1, 2]
    assert torch.isnan(got["logprob"][1:3]).all() and torch.isnan(got["entropy"][1:3]).all()
    g = oracle.token_logprobs_grad(z, 1.0, tgt, torch.ones(4), torch.ones(4))
    assert (g[0] == 0).all() and torch.isnan(g[1:3]).all() and torch.isfinite(g[3]).all()
    loss, _ = oracle.distill(z, 1.0, torch.tensor([[1, 2]] * 4, dtype=torch.int32), torch.zeros(4, 2))
    assert loss[0] == math.inf and torch.isnan(loss[1:3]).all()


@pytest.mark.parametrize("tau", [0.6, 1.0, 2.0])
def test_gradient_is_autograds(tau):
    T, V = 6, 23
    z = rows(7, ("plain", "peaked", "equal", "ties", "plain", "plain"), V, torch.float32).contiguous()
    g = torch.Generator().manual_seed(2)
    tgt = torch.randint(0, V, (T,), generator=g).int()
    tgt[4] = -100
    dl, dh = torch.randn(T, generator=g), torch.randn(T, generator=g)
    got = oracle.token_logprobs_grad(z, tau, tgt, dl, dh)
    x = z.double().requires_grad_()
    lp = torch.log_softmax(x / float(torch.tensor(tau)), 1)
    chosen = lp.gather(1, tgt.long().clamp(0)[:, None])[:, 0] * (tgt >= 0)
    (chosen * dl.double() + torch.special.entr(lp.exp()).sum(1) * dh.double()).sum().backward()
    assert torch.allclose(got, x.grad, rtol=1e-10, atol=1e-13)
    assert got.sum(1).abs().max() < 1e-12             # a softmax gradient has no component along the ones


@pytest.mark.parametrize("with_lse", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_distillation_is_kl_div_and_its_gradient(with_lse, tau):
    T, V, K = 5, 31, 6
    z = rows(9, ("plain", "peaked", "equal", "plain", "ties"), V, torch.float32).contiguous()
    g = torch.Generator().manual_seed(3)
    full = 2.0 * torch.randn(T, V, generator=g)
    vals, idx = torch.topk(full, K, 1)
    idx = idx.int()
    idx[1, 4:] = -1                                    # a shorter list
    idx[2, 5] = V
    idx[3, 5] = idx[3, 0]                              # an id twice
    vals[4, 3] = -math.inf
    lse = torch.logsumexp(full / tau, 1) if with_lse else None
    there = (idx >= 0) & (idx < V) & (vals > -math.inf)
    t = torch.where(there, vals, -math.inf).double() / tau
    log_q = t - lse.double()[:, None] if with_lse else torch.log_softmax(t, 1)
    dense_q = torch.zeros(T, V, dtype=torch.float64).scatter_add_(1, idx.long().clamp(0, V - 1), torch.where(there, log_q.exp(), 0.0))
    x = z.double().requires_grad_()
    lp = torch.log_softmax(x / tau, 1)
    want = (torch.where(there, log_q.exp() * log_q, 0.0)).sum(1) - (dense_q * lp).sum(1)
    loss, stats = oracle.distill(z, tau, idx, vals, lse)
    assert torch.allclose(loss, want, rtol=1e-11, atol=1e-12)
    if not with_lse:                                   # rows without an id twice: kl_div of the two distributions
        kl = torch.nn.functional.kl_div(lp, dense_q, reduction="none").sum(1)
        keep = torch.tensor([0, 1, 2, 4])
        assert torch.allclose(loss[keep], kl[keep], rtol=1e-11, atol=1e-12)
    d = torch.randn(T, generator=g)
    (want * d.double()).sum().backward()
    got = oracle.distill_grad(z, tau, idx, vals, d, lse)
    assert torch.allclose(got, x.grad, rtol=1e-10, atol=1e-13)


def test_gradient_is_the_difference_quotient():
    V, tau = 11, 1.0
    z = rows(13, ("plain",), V, torch.float32).contiguous()
    tgt, idx, tl = torch.tensor([4], dtype=torch.int32), torch.tensor([[2, 7, 9]], dtype=torch.int32), torch.tensor([[1.0, 0.5, -1.0]])
    one = torch.ones(1)
    ga, gb = oracle.token_logprobs_grad(z, tau, tgt, one, one), oracle.distill_grad(z, tau, idx, tl, one)
    for v in range(V):
        hi, lo = z.clone(), z.clone()
        hi[0, v] += 2.0 ** -8
        lo[0, v] -= 2.0 ** -8
        step = float(hi[0, v].double() - lo[0, v].double())
        a, b = oracle.token_logprobs(hi, tau, tgt, 0), oracle.token_logprobs(lo, tau, tgt, 0)
        quot = float(a["logprob"] + a["entropy"] - b["logprob"] - b["entropy"]) / step
        assert quot == pytest.approx(float(ga[0, v]), abs=2e-5)       # the third derivative's share, 2^-16 / 6 times at most 4
        quot = float(oracle.distill(hi, tau, idx, tl)[0] - oracle.distill(lo, tau, idx, tl)[0]) / step
        assert quot == pytest.approx(float(gb[0, v]), abs=2e-5)


def test_an_empty_list_is_no_loss():
    z = rows(15, ("plain", "plain"), 8, torch.float32)
    idx = torch.full((2, 3), -1, dtype=torch.int32)
    loss, _ = oracle.distill(z, 1.0, idx, torch.zeros(2, 3))
    assert (loss == 0).all() and (oracle.distill_grad(z, 1.0, idx, torch.zeros(2, 3), torch.ones(2)) == 0).all()
