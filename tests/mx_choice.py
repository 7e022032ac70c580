"""How the library cuts a call on a cache in 4 bits (csrc/kernel_choice.hpp, plain C++), so that a test can make sure that its cases run on
the kernels that they are about."""
import ctypes
import functools
import os
import subprocess
import tempfile

from paged_choice import COMPUTE_UNITS, CSRC

SOURCE = """
#include "kernel_choice.hpp"
extern "C" int plan(int cu, int hq, int hkv, int64_t batch, int64_t total_q, int64_t len_q, int64_t len_k) {
    const pec::MxPlan p = pec::mx_plan(cu, hq, hkv, batch, total_q, len_q, len_k);
    return p.nt | p.waves << 4 | (p.units ? 1 : 0) << 8 | (p.list ? 1 : 0) << 9;
}
"""


@functools.lru_cache(maxsize=1)
def _lib():
    d = tempfile.mkdtemp(prefix="mx_choice_")
    src, out = os.path.join(d, "c.cpp"), os.path.join(d, "c.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, "-o", out, src])
    lib = ctypes.CDLL(out)
    i64 = ctypes.c_int64
    lib.plan.argtypes = [ctypes.c_int] * 3 + [i64] * 4
    return lib


def path(hq, hkv, seqs, hints, page, table_len, spare_rows=0, room=False):
    """"units NT WAVES" or "spans NT"; "list" where the keys of all sequences go to the workspace (if there is `room`); "beside" where
    sequences with few rows and those with many are launched apart."""
    total = sum(n for n, _ in seqs) + spare_rows
    len_q = min(hints[0], total) if hints[0] else total
    len_k = min(hints[1], table_len * page) if hints[1] else table_len * page
    g = hq // hkv
    if len_q > max(1, (16 if g <= 16 else 32 if g <= 32 else 64) // g) and len(seqs) - -(-total // len_q) > 2:
        return "beside"
    p = _lib().plan(COMPUTE_UNITS, hq, hkv, len(seqs), total, len_q, len_k)
    if room and p >> 9 & 1:
        return "list"
    return "units %d %d" % (p & 15, p >> 4 & 15) if p >> 8 & 1 and page >= 16 else "spans %d" % (p & 15)
