"""The launch rules of the packed products (csrc/qf_matvec_plan.h), compiled for the host and called
through ctypes: which form of the kernel a call takes and how its launches are cut."""
import collections
import ctypes
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FMT = {"nvfp4": 1, "mxfp4": 2, "q4k": 3}
COPY = ("cached", "streamed", "words")
ROWS = ("all", "small", "twice")
CUS = 256                                                          # MI355X
SOURCE = r"""
#include "qf_matvec_plan.h"
extern "C" void plan(int fmt, int grouped, int64_t E, int64_t N, int64_t K, int64_t R, int64_t cus, int64_t* out) {
  const qf::MatvecPlan p = qf::matvec_plan(fmt, grouped != 0, E, N, K, R, cus);
  const int64_t v[9] = {p.nt, p.copy, p.rows, p.xmax, p.xrows, p.waves, p.tiles, p.items, p.per_launch};
  for (int i = 0; i < 9; ++i) out[i] = v[i];
}
"""
Plan = collections.namedtuple("Plan", "tiles_each copy rows xmax xrows waves tiles items per_launch")


class Rules:
    def __init__(self, folder):
        src, lib = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC",
                        "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2609_39223_amd", "csrc"),
                        src, "-o", lib], check=True)
        self.lib = ctypes.CDLL(lib)

    def plan(self, fmt, grouped, E, N, K, R):
        out, i = (ctypes.c_int64 * 9)(), ctypes.c_int64
        self.lib.plan(FMT[fmt], int(grouped), i(E), i(N), i(K), i(R), i(CUS), out)
        v = list(out)
        return Plan(v[0], COPY[v[1]], ROWS[v[2]], *v[3:])
