"""The drawing kernels (csrc/sample.hip) compiled for the CPU and run there, wavefront by wavefront (tests/workgroup_on_cpu.h)."""
import ctypes as C
import os
import subprocess

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCE = os.path.join(os.path.dirname(HERE), "paper_2505_07203_amd", "csrc", "sample.hip")

ENTRY = r"""
extern "C" long sample_bytes(long rows, int V, int k, int p) { return (long)po::sample_scratch(rows, V, k, p); }
// order: the wavefronts of a workgroup, in the order in which they run from barrier to barrier; -> 0, or the fault
extern "C" int sample(const float* z, long ld, int rows, int V, const float* u, const float* t, const int* k, const float* p,
                      const float* mp, int* tokens, float* logprobs, void* scratch, const int* order) {
    on_cpu::wave_order.assign(order, order + 16);
    on_cpu::fault = 0;
    po::launch_sample(z, ld, rows, V, u, t, k, p, mp, tokens, logprobs, scratch, nullptr);
    return on_cpu::fault;
}
"""


def build(folder):
    with open(SOURCE) as f:
        text = f.read()
    for old, new in (('#include "po_internal.h"', '#include "workgroup_on_cpu.h"'), ('asm volatile("s_waitcnt vmcnt(0)" ::: "memory");', "")):
        assert text.count(old) == 1, old
        text = text.replace(old, new)
    src, lib = os.path.join(folder, "sample.cpp"), os.path.join(folder, "libsample_on_cpu.so")
    with open(src, "w") as f:
        f.write(text + ENTRY)
    subprocess.run(["g++", "-std=c++17", "-O2", "-ffp-contract=off", "-shared", "-fPIC", "-Wno-attributes", "-I", HERE, src, "-o", lib], check=True)
    return C.CDLL(lib)


ORDERS = {"ascending": list(range(16)), "descending": list(range(15, -1, -1)), "inside out": [7, 8, 6, 9, 5, 10, 4, 11, 3, 12, 2, 13, 1, 14, 0, 15]}


def sample(lib, z, u, t=None, k=None, p=None, mp=None, order="ascending"):
    """-> tokens, log-probs of the rows of z"""
    z = np.ascontiguousarray(z, dtype=np.float32)
    rows, V = z.shape
    arrays = [None if a is None else np.ascontiguousarray(a, dtype=ty) for a, ty in ((u, np.float32), (t, np.float32), (k, np.int32), (p, np.float32), (mp, np.float32))]
    ptr = lambda a: None if a is None else C.c_void_p(a.ctypes.data)
    lib.sample_bytes.restype = C.c_long
    scratch = np.full(lib.sample_bytes(C.c_long(rows), V, int(k is not None), int(p is not None)) + 256, 0xff, dtype=np.uint8)
    base = C.c_void_p((scratch.ctypes.data + 255) // 256 * 256)
    tokens, lp = np.full(rows, -7, dtype=np.int32), np.full(rows, 7.0, dtype=np.float32)
    waves = np.array(ORDERS[order], dtype=np.int32)
    fault = lib.sample(ptr(z), C.c_long(V), rows, V, *[ptr(a) for a in arrays], ptr(tokens), ptr(lp), base, ptr(waves))
    assert fault == 0, f"threads of a workgroup meet at different barriers, one of them in line {fault}"
    return tokens, lp
