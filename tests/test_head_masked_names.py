"""A token that is masked by -inf and named all the same, as the target or by a teacher: its probability is 0, and what the
gradient's formula has besides the probability stays."""
import pytest
import torch

import oracle

TAU = 0.5
TARGETS = torch.tensor([1, 0], dtype=torch.int32)                       # the first is masked
D = torch.tensor([3.0, -2.0])
IDX = torch.tensor([[1, 2], [4, 0]], dtype=torch.int32)                 # 1 and 4 are masked in their rows
TEACHER = torch.tensor([[0.5, 0.5], [0.25, 0.25]])                      # shares of one half


def _logits(dtype):
    z = torch.tensor([[1.0, -torch.inf, 0.0, 0.5, -1.0], [2.0, 0.0, -0.5, 0.25, -torch.inf]])
    return z.to(dtype)


def _wanted(z):
    """Both gradients from their definition in fp64."""
    p = torch.softmax(z.double() / TAU, 1)
    at, t = torch.arange(2), TARGETS.long()
    ce = -D.double()[:, None] * p
    ce[at, t] = D.double() * (1.0 - p[at, t])
    kd = p.clone()
    for j in range(2):
        kd[at, IDX[:, j].long()] -= 0.5
    return ce / TAU, D.double()[:, None] * kd / TAU


def test_oracle():
    z = _logits(torch.float32)
    ce, kd = _wanted(z)
    assert ce[0, 1] == D[0].double() / TAU and kd[0, 1] == -0.5 * D[0].double() / TAU and kd[1, 4] == -0.5 * D[1].double() / TAU
    assert torch.allclose(oracle.token_logprobs_grad(z, TAU, TARGETS, D, None), ce, rtol=1e-14, atol=1e-15)
    assert torch.allclose(oracle.distill_grad(z, TAU, IDX, TEACHER, D), kd, rtol=1e-14, atol=1e-15)
    assert torch.isneginf(oracle.token_logprobs(z, TAU, TARGETS, 0)["logprob"][0])
    assert torch.isposinf(oracle.distill(z, TAU, IDX, TEACHER)[0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_kernels(dtype):
    import paper_2605_27081_amd as remoe

    dev = "cuda:0"
    z = _logits(dtype)
    ce, kd = _wanted(z)
    zd, desc = z.to(dev), remoe.HeadDesc(5, remoe.REMOE_F32 if dtype == torch.float32 else remoe.REMOE_BF16, TAU)
    ws = torch.empty(remoe.remoe_head_workspace_bytes(desc, 2), dtype=torch.uint8, device=dev)
    lp, loss, stats, out = torch.empty(2, device=dev), torch.empty(2, device=dev), torch.empty(2, 2, device=dev), torch.empty_like(zd)
    tgt, d, idx, teacher = (t.to(dev) for t in (TARGETS, D, IDX, TEACHER))
    remoe.remoe_token_logprobs(desc, zd, tgt, lp, None, None, None, stats, ws)
    assert torch.isneginf(lp[0]) and torch.isfinite(lp[1])
    # sums of five exponentials: a step of each (exponent's argument below 16, exponential, quotient), and the type's rounding
    half = 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    for want, call in ((ce, lambda: remoe.remoe_token_logprobs_backward(desc, zd, stats, tgt, d, None, None, out)),
                       (kd, lambda: remoe.remoe_distill_backward(desc, zd, stats, idx, teacher, None, d, out))):
        call()
        got = out.cpu().double()
        assert ((got - want).abs() <= half * want.abs() + 64 * 2.0 ** -24 * D.double().abs()[:, None] / TAU).all()
        assert torch.equal(got == 0.0, want == 0.0)
    assert out[0, 1] == -0.5 * D[0] / TAU                                # shares of one half: no rounding
    remoe.remoe_distill_forward(desc, zd, idx, teacher, None, loss, None, ws)
    assert torch.isposinf(loss).all()


def _spoilt(dtype):
    return torch.tensor([[1.0, torch.nan, 0.0], [torch.inf, 0.0, 1.0], [1.0, 0.0, -1.0]]).to(dtype)


IGNORED = torch.tensor([-100, 3, -1], dtype=torch.int32)                # positions to be ignored, in rows with NaN, with +inf, without


def test_oracle_of_ignored_positions_in_spoilt_rows():
    z = _spoilt(torch.float32)
    assert torch.equal(oracle.token_logprobs(z, 1.0, IGNORED, 0)["logprob"], torch.zeros(3, dtype=torch.float64))
    grad = oracle.token_logprobs_grad(z, 1.0, IGNORED, torch.ones(3), None)
    assert torch.isnan(grad[:2]).all() and (grad[2] == 0.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ignored_positions_in_spoilt_rows(dtype):
    import paper_2605_27081_amd as remoe

    dev = "cuda:0"
    zd, desc = _spoilt(dtype).to(dev), remoe.HeadDesc(3, remoe.REMOE_F32 if dtype == torch.float32 else remoe.REMOE_BF16, 1.0)
    ws = torch.empty(remoe.remoe_head_workspace_bytes(desc, 3), dtype=torch.uint8, device=dev)
    lp, stats, out, tgt = torch.empty(3, device=dev), torch.empty(3, 2, device=dev), torch.empty_like(zd), IGNORED.to(dev)
    remoe.remoe_token_logprobs(desc, zd, tgt, lp, None, None, None, stats, ws)
    remoe.remoe_token_logprobs_backward(desc, zd, stats, tgt, torch.ones(3, device=dev), None, None, out)
    assert (lp == 0.0).all() and torch.isnan(out[:2]).all() and (out[2] == 0.0).all()
