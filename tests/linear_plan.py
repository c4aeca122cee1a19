"""The division of the integer products (cf_linear_plan.h) compiled for the host and called through ctypes."""
import collections
import ctypes
import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
_SRC = os.path.join(_HERE, "native", "linear_plan_host.cpp")
_LIB = os.path.join(_HERE, "native", "liblinear_plan_host.so")
_DEPENDS = [_SRC, os.path.join(_HERE, "..", "paper_2508_18850_amd", "csrc", "cf_linear_plan.h")]
_lib = None

Way = collections.namedtuple("Way", "rows cols tiles")


def load():
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB) or any(os.path.getmtime(_LIB) < os.path.getmtime(f) for f in _DEPENDS):
            part = "%s.%d" % (_LIB, os.getpid())
            subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-shared", "-fPIC", "-o", part, _SRC], check=True)
            os.replace(part, _LIB)
        _lib = ctypes.CDLL(_LIB)
    return _lib


def _sizes(way):
    s = (ctypes.c_int * 3)()
    load().lp_sizes(way, s)
    return Way(s[0], s[1], bool(s[2]))


def ways():
    return [_sizes(i) for i in range(load().lp_ways())]


def way_of(rows, n_out, cus=256):
    return _sizes(load().lp_way(n_out, rows, cus))


def stream_blocks(row_blocks, col_blocks):
    """(row block, output block) of every workgroup of a launch."""
    n = load().lp_stream_grid(row_blocks, col_blocks)
    m, k = (ctypes.c_int * n)(), (ctypes.c_int * n)()
    load().lp_stream_blocks(row_blocks, col_blocks, m, k)
    return list(zip(m, k))


# Products of many rows with few outputs, with the way that the rule gives them: blocks of outputs that are no multiple of eight, one block, less than one.
NARROW = [(300, 1376, 136, Way(16, 16, False)), (2001, 208, 8, Way(16, 16, False)), (1000, 1376, 72, Way(16, 32, False)), (1000, 1376, 136, Way(32, 32, False)),
          (2050, 2064, 72, Way(32, 32, False)), (4100, 1376, 72, Way(64, 32, False)), (8200, 496, 24, Way(64, 32, False)), (4100, 1376, 136, Way(64, 64, False)),
          (1000, 1376, 520, Way(64, 64, False)), (8200, 208, 136, Way(128, 64, True))]

# Products that are divided into tiles, likewise: rows, sums and outputs that end inside a tile.
TILED = [(1000, 1376, 2056, Way(64, 64, True)), (500, 1376, 6152, Way(128, 64, True)), (3000, 1376, 1800, Way(256, 128, True)), (2049, 1376, 4104, Way(256, 256, True)),
         (4100, 2064, 10248, Way(256, 256, True))]
