"""Rows over the vocabulary that are cut into parts, the only ones with a workspace and a second launch."""
import math

import pytest
import torch

import oracle
from head_cases import STEP, SUM_TOL, close, rows
from test_gpu_head import BF16, DEV, _check_logprobs, _check_stats, _distill, _logprobs, _teacher

pytestmark = pytest.mark.gpu


def _repeated(z, T):
    """The rows of z again and again, on the device."""
    zd = torch.empty(T, z.shape[1], dtype=z.dtype, device=DEV)
    for t in range(T):
        zd[t].copy_(z[t] if t < z.shape[0] else zd[t % z.shape[0]])
    return zd


def _check_repeated(zd, z, tau, tgt, n, K):
    """All rows against the first of their kind and alignment, bit for bit, and those against the oracle; guard bytes behind the
    workspaces.  (The order of a row's sums depends on where in 16 bytes the row begins, so on the row's number modulo 8.)"""
    T, R = zd.shape[0], z.shape[0]
    firsts = min(T, math.lcm(R, 8))
    kind, again = torch.arange(T) % R, torch.arange(T) % firsts
    got = _logprobs(zd, tau, tgt[kind].contiguous(), n)
    idx, tl, _ = _teacher(7, z, K)
    loss, stats = _distill(zd, tau, idx[kind].contiguous(), tl[kind].contiguous(), None)
    for k, v in {**got, "loss": loss, "teacher's stats": stats}.items():
        bits = v.view(torch.int32)
        assert torch.equal(bits, bits[again.to(DEV)]), k
    head = kind[:firsts]
    _check_logprobs({k: v[:firsts] for k, v in got.items()}, z[head], tau, tgt[head].contiguous(), n)
    _check_losses(loss[:firsts], stats[:firsts], z[head], tau, idx[head], tl[head])


def _check_losses(loss, stats, z, tau, idx, tl):
    want, st = oracle.distill(z, tau, idx, tl, None)
    _check_stats(stats, st)
    # ln p in fp64 from an fp32 sum: its error once, as the list's shares add up to 1 (or to nothing); the result's rounding
    share = (st[:, 1] / (1.0 + st[:, 1])).abs().nan_to_num(0.0)
    close(loss, want, SUM_TOL * share + 2 * STEP * want.abs().nan_to_num(0, 0, 0) + 1e-12, "loss")


@pytest.mark.parametrize("n", [1, 20])
def test_more_rows_than_have_the_threads_of_few(n):
    """257 rows of 2,097,153: parts are aligned to fewer threads than those of 256 rows, so there are more of them."""
    z = rows(n, ("plain", "masked", "ties"), 2097153, BF16)
    print(f"257 rows of 2,097,153, {n} alternatives", flush=True)
    _check_repeated(_repeated(z, 257), z, 1.0, torch.tensor([5, 2097152, 1000000], dtype=torch.int32), n, 9)
