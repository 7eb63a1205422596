"""How the forward calls over the vocabulary deal out their rows, and that the workspace remoe_head_workspace_bytes asks for
holds what the launch puts there.  Host arithmetic: the plan's header built with the host's compiler, against the library."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_2605_27081_amd as remoe
from paper_2605_27081_amd import build as hip_build

SHIM = """
#include "head_plan.h"
extern "C" void plan(int dtype, int vocab, int64_t rows, int top_n, int k, int64_t *out)
{
    const remoe::HeadCut c = remoe::head_cut(dtype, vocab, rows, top_n, k);
    out[0] = c.threads; out[1] = c.parts; out[2] = c.len; out[3] = (int64_t)remoe::head_keys_at(rows * c.parts);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cc").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fPIC", "-shared", "-I", hip_build.CSRC, "-I", os.path.join(hip_build.ROOT, "include"),
                    "-o", str(d / "plan.so"), str(d / "plan.cc")], check=True)
    lib, out = ctypes.CDLL(str(d / "plan.so")), (ctypes.c_int64 * 4)()
    lib.plan.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_void_p]
    lib.plan.restype = None

    def call(dtype, vocab, rows, top_n=0, k=0):
        lib.plan(dtype, vocab, rows, top_n, k, ctypes.byref(out))
        return tuple(out)
    return call


@pytest.fixture(scope="module")
def lib():
    if not hip_build.is_built():
        hip_build.build()
    return remoe.load_library()


def _written(plan, dtype, vocab, rows, top_n):
    """Bytes of the workspace up to the last one that the launch writes: 12 a part, and behind them 8 a part and alternative."""
    _, parts, _, keys_at = plan(dtype, vocab, rows, top_n)
    if parts == 1:
        return 0
    assert keys_at % 8 == 0 and keys_at >= 12 * rows * parts
    return keys_at + 8 * rows * parts * top_n if top_n else 12 * rows * parts


def _vocabularies():
    rng = random.Random(5)
    fixed = [1, 5, 98303, 98304, 98305, 151936, 262144, 262145, 524288, 600000, 2097151, 2097152, 2097153, 3000000, 16257002, 1 << 24]
    return fixed + [rng.randrange(1 << 18, 1 << 24) for _ in range(300)] + [int(2 ** rng.uniform(0, 24)) for _ in range(100)]


def _rows(vocab):
    few = vocab // 2048
    return sorted({t for t in (1, 2, 255, 256, 257, 300, few - 1, few, few + 1, 4 * few, 4 * few + 1, 1000, 1024, 1 << 22) if 1 <= t <= 1 << 22})


@pytest.mark.parametrize("dtype", [0, 1])
def test_the_workspace_holds_every_part(plan, lib, dtype):
    for vocab in _vocabularies():
        desc = ctypes.byref(remoe.HeadDesc(vocab, dtype, 1.0))
        for rows in _rows(vocab):
            for n in sorted({0, 1, min(20, vocab), min(64, vocab)}):
                asked, written = lib.remoe_head_workspace_bytes(desc, rows, n), _written(plan, dtype, vocab, rows, n)
                assert written <= asked, f"{rows} rows of {vocab}, {n} alternatives: {written} bytes written, {asked} asked for"


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_part_is_one_that_the_kernels_take(plan, dtype):
    per = 8 if dtype else 4
    for vocab in _vocabularies():
        for rows in _rows(vocab):
            for n, k in ((0, 0), (min(64, vocab), 0), (0, 1), (0, 65), (0, 256)):
                threads, parts, length, _ = plan(dtype, vocab, rows, n, k)
                assert threads in (64, 128, 256, 512) and threads >= k
                assert 1 <= parts <= 64 and (parts - 1) * length < vocab <= parts * length and length % (threads * per) == 0
                longest = min(length, vocab)
                assert longest <= threads * 32 * 32 and longest <= threads * threads * per       # bits of a mask; a thread a piece of the owner's
                assert 4 * threads * (-(-longest // (threads * 32)) + 1) <= 40960                # LDS: four workgroups a compute unit


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("vocab", [98304, 600000, 2097153, 3000000, 16257002])
def test_the_workspace_never_shrinks_where_rows_are_dealt_out_otherwise(lib, vocab, dtype):
    few = vocab // 2048
    last = 0
    for t in sorted({*range(0, 600), *range(max(0, few - 20), few + 20), *range(few, 10 * few, 7), 1 << 20, 1 << 22}):
        size = lib.remoe_head_workspace_bytes(ctypes.byref(remoe.HeadDesc(vocab, dtype, 1.0)), t, 64)
        assert size >= last, t
        last = size
