"""The calls over the vocabulary refuse what they cannot do before anything is launched.  Host calls only: the addresses
below are numbers that no refused call looks behind."""
import ctypes

import pytest

import paper_2605_27081_amd as remoe
from paper_2605_27081_amd import build as hip_build

A, B = 0x10000000, 0x20000000              # aligned "addresses" far apart
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not hip_build.is_built():
        hip_build.build()
    return remoe.load_library()


def _desc(vocab=100, dtype=1, tau=1.0):
    return ctypes.byref(remoe.HeadDesc(vocab, dtype, tau))


def _logprobs(lib, desc=None, logits=A, T=4, ld=100, targets=B, top_n=0, lp=B, ent=None, ti=None, tl=None, stats=B, ws=B, ws_bytes=BIG):
    return lib.remoe_token_logprobs(desc or _desc(), logits, T, ld, targets, top_n, lp, ent, ti, tl, stats, ws, ws_bytes, None)


def _logprobs_backward(lib, desc=None, logits=A, T=4, ld=100, stats=B, targets=B, dl=B, ent=None, dent=None, acc=0, dz=B, ld_d=100):
    return lib.remoe_token_logprobs_backward(desc or _desc(), logits, T, ld, stats, targets, dl, ent, dent, acc, dz, ld_d, None)


def _distill(lib, desc=None, logits=A, T=4, ld=100, idx=B, tl=B, td=0, lse=None, k=8, loss=B, stats=B, ws=B, ws_bytes=BIG):
    return lib.remoe_distill_forward(desc or _desc(), logits, T, ld, idx, tl, td, lse, k, loss, stats, ws, ws_bytes, None)


def _distill_backward(lib, desc=None, logits=A, T=4, ld=100, stats=B, idx=B, tl=B, td=0, lse=None, k=8, dl=B, acc=0, dz=B, ld_d=100):
    return lib.remoe_distill_backward(desc or _desc(), logits, T, ld, stats, idx, tl, td, lse, k, dl, acc, dz, ld_d, None)


CALLS = (_logprobs, _logprobs_backward, _distill, _distill_backward)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("desc,word", [((0, 1, 1.0), "vocab"), ((-5, 1, 1.0), "vocab"), (((1 << 24) + 1, 1, 1.0), "vocab"), ((100, 2, 1.0), "dtype"),
                                       ((100, 1, 0.0), "temperature"), ((100, 1, -1.0), "temperature"), ((100, 1, float("nan")), "temperature"),
                                       ((100, 1, float("inf")), "temperature"), ((100, 1, 1e-8), "temperature"),
                                       ((100, 1, 1.1e6), "temperature")])
def test_descriptors(lib, call, desc, word):
    assert call(lib, desc=_desc(*desc)) == -1 and word in remoe.remoe_last_error()
    assert lib.remoe_head_workspace_bytes(_desc(*desc), 4, 0) == 0 and word in remoe.remoe_last_error()


@pytest.mark.parametrize("call", CALLS)
def test_rows(lib, call):
    assert call(lib, logits=None) == -1 and "logits" in remoe.remoe_last_error()
    assert call(lib, ld=99) == -1 and "stride" in remoe.remoe_last_error()
    assert call(lib, ld=(1 << 32) + 1) == -1 and "stride" in remoe.remoe_last_error()
    assert call(lib, logits=A + 1) == -1 and "aligned" in remoe.remoe_last_error()
    assert call(lib, T=-1) == -1 and "n_tokens" in remoe.remoe_last_error()
    assert call(lib, T=(1 << 22) + 1) == -1 and "n_tokens" in remoe.remoe_last_error()
    assert call(lib, T=0) == 0                         # nothing to do, nothing is looked at
    assert call(lib, desc=_desc(100, 0), logits=A + 2) == -1 and "aligned" in remoe.remoe_last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(top_n=65, ti=B, tl=B), "top_n"), (dict(top_n=-1), "top_n"), (dict(targets=None), "targets"), (dict(lp=None), "targets"),
    (dict(top_n=3), "top_n"), (dict(top_n=3, ti=B), "top_n"), (dict(tl=B), "top_n"), (dict(targets=None, lp=None, stats=None), "no output"),
    (dict(stats=B + 2), "aligned"), (dict(targets=B + 1), "aligned")])
def test_log_probability_arguments(lib, kw, word):
    assert _logprobs(lib, **kw) == -1 and word in remoe.remoe_last_error()


def test_more_alternatives_than_tokens(lib):
    assert _logprobs(lib, desc=_desc(5), ld=5, top_n=6, ti=B, tl=B) == -1 and "top_n" in remoe.remoe_last_error()
    assert lib.remoe_head_workspace_bytes(_desc(5), 1, 6) == 0


@pytest.mark.parametrize("call", (_logprobs, _distill))
def test_workspaces(lib, call):
    for kw in (dict(ws=None), dict(ws=B + 128), dict(ws_bytes=0)):
        assert call(lib, **kw) == -3 and "workspace" in remoe.remoe_last_error()


@pytest.mark.parametrize("kw,word", [(dict(targets=None), "targets"), (dict(dl=None), "targets"), (dict(ent=B), "entropy"), (dict(dent=B), "entropy"),
                                     (dict(targets=None, dl=None), "neither"), (dict(dl=B + 2), "aligned")])
def test_gradient_arguments(lib, kw, word):
    assert _logprobs_backward(lib, **kw) == -1 and word in remoe.remoe_last_error()


@pytest.mark.parametrize("call", (_logprobs_backward, _distill_backward))
def test_gradient_rows(lib, call):
    assert call(lib, stats=None) == -1 and "stats" in remoe.remoe_last_error()
    assert call(lib, dz=None) == -1 and "dlogits" in remoe.remoe_last_error()
    assert call(lib, ld_d=99) == -1 and "stride" in remoe.remoe_last_error()
    assert call(lib, acc=2) == -1 and "accumulate" in remoe.remoe_last_error()
    assert call(lib, dz=A, acc=1) == -1 and "accumulate" in remoe.remoe_last_error()
    assert call(lib, dz=A + 2) == -1 and "overlaps" in remoe.remoe_last_error()
    assert call(lib, dz=A, ld=100, ld_d=120) == -1 and "overlaps" in remoe.remoe_last_error()
    assert call(lib, dz=A + 2 * (3 * 100 + 99)) == -1 and "overlaps" in remoe.remoe_last_error()      # the last value


@pytest.mark.parametrize("call", (_distill, _distill_backward))
def test_teachers(lib, call):
    for kw, word in [(dict(k=0), "top_k"), (dict(k=257), "top_k"), (dict(td=2), "teacher_dtype"), (dict(idx=None), "teacher"), (dict(tl=None), "teacher"),
                     (dict(tl=B + 2), "aligned"), (dict(lse=B + 2), "aligned")]:
        assert call(lib, **kw) == -1 and word in remoe.remoe_last_error()


def test_distillation_outputs(lib):
    assert _distill(lib, loss=None) == -1 and "out_loss" in remoe.remoe_last_error()
    assert _distill_backward(lib, dl=None) == -1 and "d_loss" in remoe.remoe_last_error()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("vocab", [1, 255, 8192, 32000, 151936, 262145, 1 << 24])
def test_workspace_never_shrinks_with_more_tokens(lib, dtype, vocab):
    for n in sorted({0, 1, min(20, vocab), min(64, vocab)}):
        last = 0
        for t in [*range(0, 3000), *range(3000, 1 << 22, 99991), 1 << 22]:
            size = lib.remoe_head_workspace_bytes(_desc(vocab, dtype), t, n)
            assert size >= max(last, 1), (t, n)
            last = size


def test_the_binding_refuses_host_tensors(lib):
    import torch
    z = torch.zeros(2, 100, dtype=torch.bfloat16)
    with pytest.raises(remoe.RemoeError, match="device"):
        remoe.remoe_token_logprobs(remoe.HeadDesc(100, 1, 1.0), z, None, None, None, None, None, None, z)


def test_more_rows_than_a_launch_counts(lib):
    # 2^22 rows that are each cut into 64 parts: refused in front of the launch, whatever the addresses
    d = _desc(1 << 24)
    for call, kw in ((_logprobs, {}), (_distill, {})):
        assert call(lib, desc=d, T=1 << 22, ld=1 << 24, **kw) == -2 and "launch" in remoe.remoe_last_error()
