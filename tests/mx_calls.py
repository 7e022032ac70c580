"""How the library takes a whole call on a cache in 4 bits apart (mx_call of csrc/kernel_choice.hpp, plain C++): what its sequences with few
rows and those with many run on.  ("beside" of mx_choice.path says no more than that a call may have both.)"""
import ctypes
import functools
import os
import subprocess
import tempfile

from paged_choice import COMPUTE_UNITS, CSRC

SOURCE = """
#include "kernel_choice.hpp"
extern "C" int call(int cu, int hq, int hkv, int64_t batch, int64_t total_q, int64_t max_len_q, int64_t len_k, int64_t room) {
    const int64_t pages = room > 0 && total_q * (hq / hkv) > pec::kPagedFewRows ? room / 64 + batch : 0;
    const pec::MxCall c = pec::mx_call(cu, hq, hkv, batch, total_q, max_len_q, len_k, pages);
    return (c.apart ? 1 : 0) | (c.many.list ? 2 : 0) | (c.many.units ? 4 : 0) | c.many.nt << 3 | c.few_q << 8;
}
"""


@functools.lru_cache(maxsize=1)
def _lib():
    d = tempfile.mkdtemp(prefix="mx_calls_")
    src, out = os.path.join(d, "c.cpp"), os.path.join(d, "c.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, "-o", out, src])
    lib = ctypes.CDLL(out)
    lib.call.argtypes = [ctypes.c_int] * 3 + [ctypes.c_int64] * 5
    return lib


def way(hq, hkv, seqs, hints, page, table_len, room=0, spare_rows=0):
    """"list", "units NT" or "spans NT" (NT row tiles of 16 to a unit), of a call whose sequences with few rows are launched by themselves
    behind "steps, ".  room: keys that the workspace was made for."""
    total = sum(n for n, _ in seqs) + spare_rows
    len_k = min(hints[1], table_len * page) if hints[1] else table_len * page
    c = _lib().call(COMPUTE_UNITS, hq, hkv, len(seqs), total, hints[0], len_k, room)
    many = "list" if c & 2 else "%s %d" % ("units" if c & 4 and page >= 16 else "spans", c >> 3 & 31)
    return ("steps, " if c & 1 else "") + many
