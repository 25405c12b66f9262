"""Which sequence a unit of a ragged batch belongs to, where offsets do not ascend or lie outside the tensors: the rule that the kernels
use, compiled for the host; and what they write by it."""
import ctypes as C
import os
import subprocess

import pytest
import torch

import kv_ref as R
from paper_2307_09782_b200 import binding

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2307_09782_b200", "csrc")


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("units")
    (d / "t.cpp").write_text('''
#include "kv_index.h"
extern "C" int sequence(long long u, int B, int size, int extra, const long long* cu, long long rows, int start, int step) {
  return zq::kv::unit_sequence(u, B, size, extra, [&](int b) { return cu[b]; }, rows, start, step);
}
extern "C" long long base(long long row, long long b, int size, int extra) { return zq::kv::unit_base(row, b, size, extra); }
''')
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "t.cpp"), "-o", str(d / "t.so")], check=True)
    L = C.CDLL(str(d / "t.so"))
    L.sequence.argtypes = [C.c_longlong, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_longlong, C.c_int, C.c_int]
    L.base.restype, L.base.argtypes = C.c_longlong, [C.c_longlong, C.c_longlong, C.c_int, C.c_int]
    return L


FALLING = [[0, 1000, 0, 10], [0, 2000, 500, 600], [-7, 40, 20, 30, 25, 60], [5, 5, 5, 2, 9], [0, 3, 3, 90, 1, 90], [999, 1000, 1001, 1002, 0, 50]]


@pytest.mark.parametrize("cu", FALLING)
@pytest.mark.parametrize("size,extra", [(16, 2), (16, 1), (64, 2), (128, 1)])
def test_first_owner_whatever_the_threads_order(rule, cu, size, extra):
    """The smallest of what the threads find is what one alone finds; a sequence without rows of the tensors owns nothing."""
    B, rows = len(cu) - 1, 1000
    arr = (C.c_longlong * len(cu))(*cu)
    for u in range(rule.base(rows, B, size, extra)):
        alone = rule.sequence(u, B, size, extra, arr, rows, 0, 1)
        for step in (2, 3, 256):
            found = [rule.sequence(u, B, size, extra, arr, rows, t, step) for t in range(min(step, 8))]
            assert alone == min([b for b in found if b >= 0], default=-1)
        owners = [b for b in range(B) if 0 <= cu[b] < cu[b + 1] <= rows
                  and rule.base(cu[b], b, size, extra) <= u < rule.base(cu[b + 1], b + 1, size, extra)]
        assert alone == min(owners, default=-1)


@pytest.mark.gpu
@pytest.mark.parametrize("cu,written", [([0, 1000, 0, 10], [0]), ([0, 2000, 500, 600], [2]), ([0, 40, 20, 30, 25, 60], [0, 2, 4])])
def test_writes_where_offsets_fall(cu, written):
    """The first owner's new tokens; nothing of sequences that have none; the same every time.  (In the last batch the sequences that
    share rows have units of their own: all are written.)"""
    B, H, D, page = len(cu) - 1, 2, 64, 16
    lens = [max(n, 1) + 5 for n in (cu[b + 1] - cu[b] for b in range(B))]
    codes, scale, table, lens, _ = R.batch(lens, [0] * B, H, D, page)
    k, v = R.heads(1000, H, D, 3), R.heads(1000, H, D, 4)
    expect = codes, scale
    for b in written:
        expect = R.write(*expect, k, v, table[b:b + 1], [lens[b]], cu[b:b + 2], "none")
    for _ in range(10):
        c, s = codes.clone(), scale.clone()
        binding.kv_cache_write(binding.Fp8KvCache(c, s), k, v, table, R.ints(lens), cu=R.ints(cu))
        assert torch.equal(c, expect[0]) and torch.equal(s.nan_to_num(nan=-1.0), expect[1].nan_to_num(nan=-1.0))
