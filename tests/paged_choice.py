"""How the library cuts a paged call of given sizes (csrc/kernel_choice.hpp, plain C++), so that a test can make sure that its
cases run on the kernels that they are about."""
import ctypes
import functools
import os
import subprocess
import tempfile

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_15104_amd", "csrc")
COMPUTE_UNITS = 256
SOURCE = """
#include "kernel_choice.hpp"
extern "C" int cut(int cu, int hq, int hkv, int64_t batch, int64_t total_q, int64_t len_q, int64_t len_k) {
    const pec::PagedCut c = pec::paged_cut(cu, hq, hkv, batch, total_q, len_q, len_k);
    return (c.units ? 1 : 0) | (c.steps ? 2 : 0) | (c.list ? 4 : 0) | c.nt << 4 | c.few_rows << 8 | c.unit_waves << 16;
}
extern "C" int parts(int cu, int64_t tokens, int64_t quads) { return pec::norm_rope_parts(cu, tokens, quads); }
"""


@functools.lru_cache(maxsize=1)
def _lib():
    d = tempfile.mkdtemp(prefix="paged_choice_")
    src, out = os.path.join(d, "c.cpp"), os.path.join(d, "c.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I" + CSRC, "-o", out, src])
    lib = ctypes.CDLL(out)
    i64 = ctypes.c_int64
    lib.cut.argtypes = [ctypes.c_int] * 3 + [i64] * 4
    lib.parts.argtypes = [ctypes.c_int, i64, i64]
    return lib


def path(hq, hkv, seqs, hints, page, table_len, spare_rows=0):
    """("units", wavefronts) or (which of "steps nt" and "list" run) for sequences [(new, all)] and the caller's hints."""
    total = sum(n for n, _ in seqs) + spare_rows
    len_q = min(hints[0], total) if hints[0] else total
    len_k = min(hints[1], table_len * page) if hints[1] else table_len * page
    c = _lib().cut(COMPUTE_UNITS, hq, hkv, len(seqs), total, len_q, len_k)
    if c & 1:
        return "units %d" % (c >> 16)
    return " + ".join((["steps %d" % (c >> 4 & 15)] if c & 2 else []) + (["list"] if c & 4 else []))


def parts(tokens, quads):
    return _lib().parts(COMPUTE_UNITS, tokens, quads)
