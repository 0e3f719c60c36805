"""Shapes that between them take every tile of the microscaled product, and the library's own choice
of a tile (csrc/mx_tiles.h, compiled by itself)."""
import ctypes
import os
import subprocess

from paper_2509_24416_gb300 import build

SOURCE = """
#include "mx_tiles.h"
extern "C" int dense(int M, int N, int K, int sms) {
  const clq::mx::TileShape t = clq::mx::pick_tile(M, 1, N, K, sms, false);
  return 10 * t.nt + t.cg;
}
extern "C" int grouped(int T, int k, int E, int N, int K, int sms) {
  const clq::mx::TileShape t = clq::mx::pick_grouped_tile(T, k, E, N, K, sms);
  return 10 * t.nt + t.cg;
}
"""

# M, K, N, (rows, CTAs) of the tile on 152 SMs.  Among them, for the tiles of 256 rows: last tiles of
# 64, 128, 192 and 256 columns, one and several tiles a CTA or pair, one K step and many, outputs
# whose rows are 16-byte aligned and not.
DENSE = [
    (20, 8192, 140, (32, 1)), (600, 288, 129, (64, 1)), (6000, 288, 257, (128, 1)), (8000, 96, 129, (128, 2)),
    (2741, 96, 3001, (128, 2)),
    (8023, 96, 4147, (256, 1)), (8023, 96, 4152, (256, 1)), (5249, 1056, 2616, (256, 1)), (4000, 4608, 1152, (256, 1)),
    (6000, 288, 3001, (256, 2)), (2000, 1184, 4096, (256, 2)), (4000, 1184, 2049, (256, 2)), (4673, 1184, 4096, (256, 2))]

# T, k, E, N, K, tile on 152 SMs; N the product's channels.
GROUPED = [
    (20, 2, 16, 256, 256, (32, 1)), (300, 2, 4, 544, 256, (128, 1)), (3000, 2, 8, 256, 288, (128, 1)),
    (2000, 2, 3, 2048, 544, (256, 2)), (1000, 4, 16, 2048, 544, (256, 2)), (3500, 2, 4, 1088, 1024, (256, 2)),
    (4100, 2, 3, 928, 1056, (256, 2))]


def library(folder):
    so = os.path.join(str(folder), "mx_tiles.so")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", build.CSRC, "-x", "c++", "-", "-o", so],
                       input=SOURCE, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return ctypes.CDLL(so)


def dense(lib, M, N, K, sms=152):
    return divmod(lib.dense(M, N, K, sms), 10)


def grouped(lib, T, k, E, N, K, sms=152):
    return divmod(lib.grouped(T, k, E, N, K, sms), 10)
