"""csrc/kv_schedule.cuh: counts of keys and key blocks of a sequence, compiled for the host from
the kernels' own source, up to the longest sequence that a call takes.  No GPU."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2608_02474_gb300", "csrc")
SHIMS = """
#include <algorithm>
#include <climits>
#include <cstdint>
#include "extents.h"
using std::max;
using std::min;
#define ECHO_DEV inline
static inline uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }
"""
WRAP = """
extern "C" {
int most_keys() { return kMostKeys; }
// key blocks of tile t of a sequence of `len` tokens whose last `rows` are this call's
int blocks(int len, int rows, int cap, int tile, int shift, int causal_block, int t, int *keys) {
    int32_t row0[2] = {0, rows};
    KvWork w;
    w.b.len = &len;
    w.b.row0 = row0;
    w.b.n_seqs = 1;
    w.b.n_rows = rows;
    w.group = 1;
    w.causal_block = causal_block;
    w.by_group = KvDiv(1);
    w.by_tile = KvDiv(tile);
    w.by_block = KvDiv(causal_block > 0 ? causal_block : 1);
    w.tile = tile;
    w.cap = cap;
    w.block_shift = shift;
    KvSeq s;
    s.load(w, 0);
    *keys = s.keys(w, t);
    return s.blocks(w, t);
}
}
"""


def source(name):
    return open(os.path.join(CSRC, name)).read()


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no C++ compiler")
    pages, schedule = source("kv_pages.cuh"), source("kv_schedule.cuh")
    batch = re.search(r"struct KvBatch \{.*?\n\};", pages, re.S).group(0)
    own = schedule[schedule.index("struct KvDiv {"):schedule.index("// One piece of an item")]
    d = tmp_path_factory.mktemp("schedule")
    (d / "w.cpp").write_text(SHIMS + batch + own + WRAP)
    # -fwrapv: sums that pass 31 bits wrap, as on the device
    subprocess.run([cxx, "-std=c++17", "-O1", "-fwrapv", "-shared", "-fPIC", "-I" + CSRC, str(d / "w.cpp"), "-o",
                    str(d / "w.so")], check=True)
    return ctypes.CDLL(str(d / "w.so"))


def shifts():
    """log2 of the keys of the few-row kernels' blocks."""
    return sorted(int(n) for n in re.findall(r"[?:] (\d+)", re.search(r"BSHIFT = [^;]*", source("kv_decode.cu")).group(0)))


def test_block_sizes():
    assert shifts() == [6, 7, 8]
    assert "BN = 128;" in source("kv_chunk.cu")


@pytest.mark.parametrize("shift", [6, 7, 8])
@pytest.mark.parametrize("cb", [0, 1, 1560])
def test_blocks_of_any_length(lib, shift, cb):
    """As many blocks as cover the keys, for lengths around the blocks' borders and up to the most that
    a sequence may have; a table may cover more."""
    most = lib.most_keys()
    assert most == 2 ** 31 - 128
    keys = ctypes.c_int()
    lens = [0, 1, 63, 64, 65, 127, 128, 129, 255, 256, 257, 31200, 2 ** 30 + 1]
    lens += [most - k for k in (0, 1, 126, 127, 128, 129, 255, 256, 257, 512)]
    for n in lens + [2 ** 31 - 1]:
        for rows in (1, 40):
            for t in range(-(-rows // 16)):
                got = lib.blocks(n, rows, most, 16, shift, cb, t, ctypes.byref(keys))
                p = n - rows + min(16 * (t + 1), rows) - 1
                want = min(n, most) if cb == 0 else 0 if p < 0 else min(n, most, (p // cb + 1) * cb)
                assert keys.value == want and got == -(-want // 2 ** shift), (n, rows, t)


def test_the_rule_for_blocks_of_256_keys():
    """As test_gpu_int4_division.py, which widens tables to it, has it."""
    rule = re.search(r"if \(tile == 8 && ([^\n]*)\)\n\s*return launch<FORM, D, 1, true>", source("kv_decode.cu")).group(1)
    assert rule.replace("(double)", "").startswith("a.batch->n_seqs * a.pool->H * keys >= 2.0 * echo::num_sms() * 16 * 256")
