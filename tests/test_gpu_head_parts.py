"""Rows over the vocabulary that are cut into parts, the only ones with a workspace and a second launch."""
import math

import pytest
import torch

import oracle
import paper_2605_27081_amd as remoe
from head_cases import KINDS, STEP, SUM_TOL, close, rows
from test_gpu_head import (BF16, DEV, F32, _check_logprobs, _check_stats, _desc, _distill, _logprobs, _out, _targets, _teacher, _to_device,
                           _training_buffers, _training_step)

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
        if v is not None:
            bits = v.view(torch.int32)
            assert torch.equal(bits, bits[again.to(DEV)]), k
    head = kind[:firsts]
    _check_logprobs({k: None if v is None else v[:firsts] for k, v in got.items()}, z[head], tau, tgt[head].contiguous(), n)
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


# 98,304 logits are the fewest that are cut, V / 2048 rows the most
@pytest.mark.parametrize("T,V,dtype", [(1, 98304, BF16), (16, 100003, BF16), (16, 100003, F32), (48, 98304, BF16), (48, 98304, F32), (48, 100003, BF16)])
def test_every_kind_of_row_in_parts(T, V, dtype):
    print(f"rows in parts T={T} V={V} {dtype}", flush=True)
    z = rows(V + T, [KINDS[t % len(KINDS)] for t in range(T)], V, dtype)
    tgt = _targets(T, z)
    for tau, n in ((1.0, 0), (0.7, 20), (1.0, 64)):
        _check_logprobs(_logprobs(_to_device(z), tau, tgt, n), z, tau, tgt, n)
    idx, tl, _ = _teacher(T, z, 30)
    _check_losses(*_distill(_to_device(z), 1.0, idx, tl, None), z, 1.0, idx, tl)


@pytest.mark.parametrize("T,V,dtype", [(129, 262147, BF16), (129, 262147, F32), (130, 262145, BF16), (260, 262147, BF16), (260, 262145, F32),
                                       (257, 600001, BF16)])
def test_parts_by_length_alone(T, V, dtype):
    """More than V / 2048 rows, each longer than a part."""
    z = rows(T, ("plain", "masked", "ties"), V, dtype)
    print(f"parts by length T={T} V={V} {dtype}", flush=True)
    tgt = torch.tensor([V - 1, 0, V // 2], dtype=torch.int32)
    for n in (0, 20):
        _check_repeated(_repeated(z, T), z, 1.0, tgt, n, 40)


@pytest.mark.parametrize("V", [262143, 262144])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_longest_rows_of_one_workgroup(V, dtype):
    """260 rows of them have 256 threads, each with 32 times 32 logits."""
    z = rows(V, ("plain", "masked", "ties"), V, dtype)
    z[0, -1] = 30.0
    print(f"longest uncut rows V={V} {dtype}", flush=True)
    _check_repeated(_repeated(z, 260), z, 1.0, torch.tensor([V - 1, 0, V // 2], dtype=torch.int32), 20, 40)


def test_captured_and_replayed_in_parts():
    """The four calls in two graphs that share their workspaces, replayed in turn on new logits; whatever a workspace holds before a
    call is of no account."""
    T, V, K, n = 5, 100003, 12, 20
    z = rows(31, ("plain", "masked", "ties", "few", "peaked"), V, BF16)
    zd, tgt = _to_device(z), _targets(5, z).to(DEV)
    idx, tl, _ = _teacher(6, z, K)
    idx, tl = idx.to(DEV), tl.to(DEV)
    eager, ce, kd = _training_buffers(z, K, n)
    both = [_training_buffers(z, K, n)[0] for _ in range(2)]
    both[1]["ws"], both[1]["ws2"] = both[0]["ws"], both[0]["ws2"]
    graphs = []
    for bufs in both:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            _training_step(zd, tgt, idx, tl, bufs, ce, kd, T)
        torch.cuda.current_stream().wait_stream(side)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            _training_step(zd, tgt, idx, tl, bufs, ce, kd, T)
    for i in range(4):
        zd.copy_(rows(40 + i, ("masked", "plain", "empty", "ties", "peaked"), V, BF16))
        for bufs, garbage in ((eager, 0x00), (both[0], (0xFF, 0x7F, 0x00, 0x80)[i])):
            for k in ("ws", "ws2"):
                bufs[k].fill_(garbage)
        _training_step(zd, tgt, idx, tl, eager, ce, kd, T)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for bufs in both:
            for k in ("lp", "h", "ti", "tl", "st", "kd", "st2", "dz"):
                assert torch.equal(eager[k].view(torch.int16), bufs[k].view(torch.int16)), (i, k)


def test_two_streams_and_repeats_in_parts():
    """The same calls on two streams at once, each with one workspace for all of its calls, give the bits of a call alone."""
    T, V, n = 3, 151937, 33
    z = rows(51, ("plain", "ties", "masked"), V, BF16)
    zd, tgt = _to_device(z), _targets(7, z)
    idx, tl, _ = _teacher(3, z, 20)
    first, loss = _logprobs(zd, 1.0, tgt, n), _distill(zd, 1.0, idx, tl, None)[0]
    desc, tgt, idx, tl = _desc(V, BF16, 1.0), tgt.to(DEV), idx.to(DEV), tl.to(DEV)
    streams, runs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    spaces = [torch.full((remoe.remoe_head_workspace_bytes(desc, T, n),), 0xFF, dtype=torch.uint8, device=DEV) for _ in streams]
    made = [[(_out(T), _out(T), _out(T, n, dtype=torch.int32), _out(T, n), _out(T, 2), _out(T)) for _ in range(4)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(4):
        for s, ws, outs in zip(streams, spaces, made):
            with torch.cuda.stream(s):
                remoe.remoe_token_logprobs(desc, zd, tgt, *outs[i][:5], ws)
                remoe.remoe_distill_forward(desc, zd, idx, tl, None, outs[i][5], None, ws)
            runs.append(outs[i])
    torch.cuda.synchronize()
    for out in runs:
        for got, want in zip(out, (*first.values(), loss)):
            assert torch.equal(got.view(torch.int32), want.view(torch.int32))
