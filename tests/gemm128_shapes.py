"""Shapes of the products with a scale per 128 for every kernel, tile and cut along K that the library chooses among
(csrc/gemm128_choice.h), and that choice itself, compiled for the host.

Rows end inside a tile, k inside a block and features inside a tile of each; few128's cuts are uneven, with one tile of rows
and with several, many128's tiles fewer and more than the CTA pairs that the device holds, with few blocks along K and with more than
its rings have slots."""
import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

from paper_2606_13898_gb300 import build

SMS = 152

# kernel, columns, cut: rows, k, n
PLAIN = {
    ("few", 16, 1): [(1, 144, 11344), (18, 144, 5648)],
    ("few", 16, 2): [(1, 272, 144), (17, 272, 144)],
    ("few", 16, 4): [(1, 528, 144), (17, 528, 144)],
    ("few", 16, 8): [(1, 1040, 144), (17, 1040, 144)],
    ("few", 32, 1): [(18, 288, 13840), (964, 144, 288)],
    ("few", 32, 2): [(18, 416, 10800), (526, 272, 144)],
    ("few", 32, 4): [(19, 1312, 3904), (542, 832, 144)],
    ("few", 32, 8): [(18, 2656, 2096), (284, 2592, 160)],
    ("few", 64, 1): [(34, 864, 15952)],
    ("few", 64, 2): [(35, 976, 11440), (165, 1440, 2784)],
    ("few", 64, 4): [(34, 1824, 5776), (1155, 1216, 144)],
    ("few", 64, 8): [(34, 5056, 2384), (632, 4768, 160)],
    ("few", 128, 1): [(72, 4032, 9824), (268, 4128, 4944)],
    ("few", 128, 2): [(66, 2400, 5344), (2396, 2272, 160)],
    ("few", 128, 4): [(98, 1312, 4080), (1636, 1360, 160)],
    ("few", 128, 8): [(98, 3872, 1520), (755, 4448, 160)],
    ("many", 128, 1): [(1030, 16, 144), (528, 288, 9632), (1375, 1168, 160), (4879, 1184, 800)],
    ("many", 192, 1): [(66, 16, 13008), (533, 272, 13280), (67, 1168, 10288), (258, 1184, 9824)],
    ("many", 256, 1): [(264, 16, 7344), (769, 416, 12528), (258, 1184, 7568), (514, 1216, 10032), (777, 1168, 4400)],
}
GATED = {  # to 16 or 32 bits
    ("few", 16, 1): [(1, 144, 9504), (18, 144, 4944)],
    ("few", 16, 2): [(1, 272, 144), (17, 272, 144)],
    ("few", 16, 4): [(1, 528, 144), (17, 528, 144)],
    ("few", 16, 8): [(1, 1040, 144), (17, 1040, 144)],
    ("few", 32, 1): [(18, 288, 12640), (34, 144, 12976)],
    ("few", 32, 2): [(18, 688, 6448), (514, 1264, 160)],
    ("few", 32, 4): [(18, 1328, 3424), (447, 1312, 160)],
    ("few", 32, 8): [(18, 3744, 1312), (130, 4752, 160)],
    ("few", 64, 1): [(38, 432, 13296), (67, 2208, 5104)],
    ("few", 64, 2): [(35, 1216, 5456), (68, 4256, 2528)],
    ("few", 64, 4): [(34, 2368, 3008), (578, 2912, 160)],
    ("few", 64, 8): [(36, 6384, 1056), (261, 6336, 160)],
    ("few", 128, 1): [(67, 3312, 10704), (264, 3424, 5680)],
    ("few", 128, 2): [(67, 5808, 6288), (267, 6880, 2464)],
    ("few", 128, 4): [(67, 7088, 3312), (1590, 7504, 160)],
    ("few", 128, 8): [(66, 11920, 1632)],
    ("many", 128, 1): [(514, 16, 144), (66, 288, 11056), (67, 1168, 10288), (18, 1312, 4784)],
    ("many", 256, 1): [(34, 560, 7904), (275, 800, 12224), (258, 1184, 7568), (34, 1200, 8752)],
}
CODES = {  # gated, to codes
    ("few", 16, 1): [(1, 144, 9504), (18, 144, 4944)],
    ("few", 16, 2): [(1, 272, 144), (17, 272, 144)],
    ("few", 16, 4): [(1, 528, 144), (17, 528, 144)],
    ("few", 16, 8): [(1, 1040, 144), (17, 1040, 144)],
    ("few", 32, 1): [(18, 288, 12640), (780, 144, 288)],
    ("few", 32, 2): [(18, 688, 6448), (526, 272, 144)],
    ("few", 32, 4): [(18, 1328, 3424), (542, 832, 144)],
    ("few", 32, 8): [(18, 3744, 1312), (130, 4752, 160)],
    ("few", 64, 1): [(38, 432, 13296), (67, 2208, 5104)],
    ("few", 64, 2): [(35, 1216, 5456), (1068, 720, 160)],
    ("few", 64, 4): [(34, 2368, 3008), (1035, 864, 144)],
    ("few", 64, 8): [(36, 6384, 1056), (261, 6336, 160)],
    ("few", 128, 1): [(66, 720, 13456), (263, 672, 5072)],
    ("few", 128, 2): [(67, 5808, 6288), (2357, 6384, 160)],
    ("few", 128, 4): [(68, 2336, 4128), (2082, 2064, 144)],
    ("few", 128, 8): [(66, 11920, 1632)],
    ("many", 256, 1): [(1030, 16, 144), (82, 16, 13296), (257, 272, 9808), (130, 1200, 9936), (34, 1200, 8752)],
}

SOURCE = r"""
#include "gemm128_choice.h"
extern "C" void choice(int gated, int codes, int rows, int k, int n, int num_sms, int* out) {
  const int kblocks = (k + 127) / 128;
  const hilo::Gemm128Choice c = gated ? hilo::gemm128_choice<true>(rows, n, kblocks, codes, num_sms)
                                      : hilo::gemm128_choice<false>(rows, n, kblocks, codes, num_sms);
  out[0] = c.many;
  out[1] = c.nt;
  out[2] = c.split;
}
"""


@functools.lru_cache(None)
def _library():
    cxx = shutil.which("g++")
    assert cxx, "no C++ compiler"
    with tempfile.TemporaryDirectory() as d:
        src, lib = os.path.join(d, "choice.cpp"), os.path.join(d, "choice.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", build.CSRC, src, "-o", lib], check=True)
        return ctypes.CDLL(lib)


def choice(rows, k, n, gated=False, codes=False, num_sms=SMS):
    """(kernel, columns, cut) of a call."""
    out = (ctypes.c_int * 3)()
    _library().choice(int(gated), int(codes), rows, k, n, num_sms, out)
    return ("many" if out[0] else "few", out[1], out[2])


def flat(table):
    return [(*kind, *shape) for kind, shapes in table.items() for shape in shapes]
