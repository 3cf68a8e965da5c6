"""How a call of decode attention over caches in 4 or 8 bits is divided: the planner, built
for the host, and the shapes that tests run because of their divisions."""
import ctypes
import os
import subprocess

import paper_2512_00722_amd as spec

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(spec.__file__)))
SOURCE = """
#include "quant_plan.h"
extern "C" void plan(const int* x, int* o) {
  spec::QuantDims d{};
  d.n_layers = x[0]; d.B = x[1]; d.L_cap = x[2]; d.H_kv = x[3]; d.G = x[4]; d.bits = x[5];
  d.H_q = d.G * d.H_kv;
  d.window = x[6] < d.L_cap ? x[6] : d.L_cap;
  d.n_sink = x[7] < d.L_cap ? x[7] : d.L_cap;
  d.k_max = x[8];
  const spec::QuantPlan p = spec::plan_of(d, d.k_max > 0);
  const int heads = spec::group_heads(d.G);
  o[0] = p.nh; o[1] = p.w; o[2] = p.ub_log2; o[3] = p.n_split; o[4] = p.deal;
  o[5] = heads <= 4 ? 4 : heads <= 8 ? 8 : 16;
}
"""


class Planner:
    def __init__(self, folder):
        src, lib = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        hip = os.path.join(os.path.dirname(os.path.dirname(
            os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"))), "include")
        subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-shared", "-fPIC",
                        "-D__HIP_PLATFORM_AMD__", "-isystem", hip,
                        "-I" + os.path.join(ROOT, "paper_2512_00722_amd", "csrc"),
                        "-I" + os.path.join(ROOT, "include"), src, "-o", lib], check=True)
        self.lib = ctypes.CDLL(lib)

    def __call__(self, n, B, L, H_kv, G, bits, window=None, n_sink=0, k_max=0):
        """nh, w, ub_log2, n_split, deal, columns of a call over whole caches (window None),
        a window, or selected rows (k_max)."""
        x = (ctypes.c_int * 9)(n, B, L, H_kv, G, bits, L if window is None else window, n_sink,
                               k_max)
        o = (ctypes.c_int * 6)()
        self.lib.plan(x, o)
        return tuple(o)


def divisions(plan, bits, selected):
    """What a kernel does differently: where a launch's wavefronts stand, and which code."""
    nh, w, ub, n_split, deal, columns = plan
    return {("divided", bits, selected, nh, w, ub, n_split > 1, bool(deal)),
            ("columns", bits, selected, nh, w, columns)}


# layers, sequences, capacity, KV heads, query heads of each, bits, which tokens and how many
# (a window's, or selected ones), sinks: the smallest that were found for the divisions that the
# shapes of test_quant_plans_gpu.py do not have
CASES = [
    (1, 1, 1, 2, 4, 4, "all", 0, 0), (1, 1, 723, 2, 2, 4, "all", 0, 0),
    (1, 1, 928, 4, 17, 4, "all", 0, 0), (1, 2, 2270, 4, 17, 4, "all", 0, 0),
    (1, 2, 2574, 4, 1, 4, "window", 662, 0), (1, 4, 794, 16, 17, 4, "all", 0, 0),
    (1, 26, 18963, 3, 20, 4, "window", 13297, 0), (2, 1, 943, 8, 17, 4, "all", 0, 0),
    (2, 2, 516, 16, 17, 4, "all", 0, 0), (2, 2, 1859, 8, 17, 4, "all", 0, 0),
    (3, 4, 38084, 1, 5, 4, "all", 0, 0), (3, 5, 2390, 3, 20, 4, "all", 0, 0),
    (4, 2, 3025, 1, 17, 4, "all", 0, 0), (6, 1, 62195, 3, 20, 4, "all", 0, 0),
    (7, 2, 198, 2, 17, 4, "all", 0, 0), (20, 2, 1, 16, 17, 4, "window", 1, 0),
    (33, 2, 3574, 3, 20, 4, "all", 0, 0), (1, 1, 1, 2, 2, 4, "selected", 1, 0),
    (1, 1, 1289, 16, 17, 4, "selected", 1229, 0), (1, 2, 1369, 8, 17, 4, "selected", 1092, 0),
    (1, 2, 1783, 2, 1, 4, "selected", 1752, 0), (1, 2, 7249, 4, 17, 4, "selected", 1334, 0),
    (1, 3, 678, 4, 1, 4, "selected", 669, 0), (1, 6, 9170, 8, 17, 4, "selected", 3911, 0),
    (1, 10, 4169, 4, 17, 4, "selected", 2670, 0), (1, 10, 4760, 1, 17, 4, "selected", 4274, 0),
    (2, 2, 4126, 16, 17, 4, "selected", 1860, 0), (2, 19, 1, 16, 17, 4, "selected", 1, 0),
    (3, 7, 62108, 3, 20, 4, "selected", 61575, 0), (3, 26, 457, 16, 1, 4, "selected", 415, 0),
    (5, 1, 529, 4, 17, 4, "selected", 426, 0), (5, 4, 35271, 1, 8, 4, "selected", 26412, 0),
    (16, 3, 5754, 3, 20, 4, "selected", 1623, 0), (27, 3, 5901, 3, 20, 4, "selected", 4177, 0),
    (1, 5, 3049, 1, 17, 8, "all", 0, 0), (1, 14, 39892, 1, 17, 8, "all", 0, 0),
    (2, 1, 787, 8, 17, 8, "all", 0, 0), (2, 7, 1918, 4, 17, 8, "all", 0, 0),
    (2, 7, 6583, 1, 17, 8, "all", 0, 0), (3, 1, 129810, 4, 3, 8, "all", 0, 0),
    (3, 5, 19434, 2, 17, 8, "all", 0, 0), (7, 2, 10084, 2, 17, 8, "all", 0, 0),
    (12, 1, 23124, 6, 3, 8, "all", 0, 0), (1, 1, 562, 2, 20, 8, "selected", 542, 0),
    (2, 30, 69086, 1, 5, 8, "selected", 43794, 0), (3, 2, 22259, 1, 17, 8, "selected", 5685, 0),
    (3, 19, 36237, 2, 4, 8, "selected", 18738, 0), (4, 1, 69204, 6, 48, 8, "selected", 56413, 0),
    (4, 5, 3700, 4, 3, 8, "selected", 3008, 0), (5, 1, 50648, 3, 17, 8, "selected", 13519, 0),
    (5, 21, 3451, 4, 32, 8, "selected", 2432, 0), (21, 1, 17626, 6, 20, 8, "selected", 15327, 0),
    (23, 5, 7658, 4, 4, 8, "selected", 3791, 0),
]


def arguments(case):
    """What Planner takes of a case."""
    *shape, kind, tokens, n_sink = case
    return shape, {"all": {}, "window": dict(window=tokens, n_sink=n_sink),
                   "selected": dict(k_max=tokens)}[kind]
