"""The choice of kernel and shape of the 8-bit head (csrc/choose.h, plain host arithmetic), compiled with g++ for the CPU tests.  Not
collected by pytest."""
from __future__ import annotations

import ctypes as C
import os
import subprocess
import tempfile
from collections import namedtuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_ABI = r"""
#include "choose.h"
using namespace nanospec;
extern "C" {
int c_few_supported(int M, int d) { return few_supported(M, d); }
int c_few_rounds(int M, int d) { return few_rounds(M, d); }
void c_few_plan(int M, int d, int batch, int cap, int* o) {
  const FewPlan f = few_plan(M, d, batch, cap, few_rounds(M, d));
  o[0] = f.KS; o[1] = f.slices; o[2] = f.log_groups; o[3] = f.waves; o[4] = f.log_parts; o[5] = f.seg; o[6] = f.lds;
}
int c_i8_shape(int M, int d, int batch, int cap, int dense) { return i8_shape(M, d, batch, cap, dense != 0); }
int c_policy_fuses(int rows, int V) { return policy_fuses(rows, V); }
}
"""

Few = namedtuple("Few", "KS slices log_groups waves log_parts seg lds")


def _load():
    with tempfile.TemporaryDirectory() as tmp:
        src, so = os.path.join(tmp, "choose.cpp"), os.path.join(tmp, "choose.so")
        with open(src, "w") as f:
            f.write(_ABI)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2605_26444_amd", "csrc"), "-o", so, src],
                       check=True)
        return C.CDLL(so)


_lib = _load()


def few_supported(M, d):
    return bool(_lib.c_few_supported(M, d))


def few_rounds(M, d):
    return bool(_lib.c_few_rounds(M, d))


def few_plan(M, d, batch, cap):
    o = (C.c_int * 7)()
    _lib.c_few_plan(M, d, batch, cap, o)
    return Few(*o)


def i8_shape(M, d, batch, cap, dense=False):
    return _lib.c_i8_shape(M, d, batch, cap, int(dense))


def policy_fuses(rows, V):
    return bool(_lib.c_policy_fuses(rows, V))
