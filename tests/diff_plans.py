"""Which kernels a differential attention call takes, as api.cpp decides it: the host code, built for the CPU with
launchers that note what they are given.  Pointers are never dereferenced."""

import ctypes
import os
import subprocess

from paper_2505_22918_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2505_22918_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

NOTES = r"""
#include <hip/hip_runtime_api.h>
#include <algorithm>
#include <chrono>
#include "heads.h"
#include "rettention.h"
namespace rt {
int seen[8];
int64_t blocks;
hipError_t launch_rope(const RopeArgs& a, hipStream_t) {
    seen[0] = a.vec, seen[1] = a.groups, blocks = rope_blocks(a);
    return hipSuccess;
}
hipError_t launch_diff(const DiffArgs& a, int, hipStream_t) {
    seen[0] = a.by_keys, seen[1] = a.split, seen[2] = a.by_len;
    return hipSuccess;
}
hipError_t launch_diff_backward(const DiffArgs& a, int, hipStream_t) {
    seen[0] = a.two, seen[1] = a.split_k, seen[2] = a.split_q, seen[3] = a.short_rows, seen[4] = a.by_len;
    return hipSuccess;
}
}  // namespace rt
extern "C" const int* rt_seen() { return rt::seen; }
extern "C" int64_t rt_blocks() { return rt::blocks; }
template <class F>
static double least(F&& f) {
    double best = 1e30;
    for (int i = 0; i < 400; ++i) {
        const auto t = std::chrono::steady_clock::now();
        for (int j = 0; j < 10; ++j) f();
        best = std::min(best, std::chrono::duration<double, std::micro>(std::chrono::steady_clock::now() - t).count() / 10);
    }
    return best;
}
// microseconds of the host: a question for the workspace, and the call itself
extern "C" void rt_times(rt_diff_dims d, int backward, double* us) {
    auto at = [](int64_t i) { return (void*)((i + 1) << 40); };
    auto f = [&](int64_t i) { return (float*)at(i); };
    int64_t n;
    us[0] = least([&] { backward ? rt_attn_diff_backward_workspace(d, &n) : rt_attn_diff_workspace(d, &n); });
    us[1] = least([&] {
        backward ? rt_attn_diff_backward(at(0), at(1), at(2), f(3), 1, nullptr, at(5), at(6), f(7), f(8), at(9), d, at(10), at(11),
                                         at(12), f(13), at(14), (int64_t)1 << 40, nullptr)
                 : rt_attn_diff(at(0), at(1), at(2), f(3), 1, nullptr, d, at(5), at(6), f(7), f(8), at(9), (int64_t)1 << 40, nullptr);
    });
}
"""


def build(folder):
    src, out = os.path.join(folder, "notes.cpp"), os.path.join(folder, "librettention_notes.so")
    with open(src, "w") as f:
        f.write(NOTES)
    cmd = ["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(CSRC, "api.cpp"),
           os.path.join(HERE, "sanitize", "launch_stubs.cpp"), os.path.join(HERE, "sanitize", "train_stubs.cpp"), src, "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    lib = ctypes.CDLL(out)
    for name, (res_type, args) in _lib._SIGS.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res_type, args
    lib.rt_seen.restype = ctypes.POINTER(ctypes.c_int)
    lib.rt_blocks.restype = ctypes.c_int64
    lib.rt_times.restype, lib.rt_times.argtypes = None, [_lib.RtDiffDims, ctypes.c_int, ctypes.POINTER(ctypes.c_double)]
    return lib


def at(i):
    """An address for tensor i, a terabyte from the others."""
    return (i + 1) << 40


def forward(lib, B, H, Tq, Tk, D, lens, stats=True):
    """(kernel, keys in parts, samples taken by their keys): tile, keys or few; see attn_diff.hip."""
    dims = _lib.RtDiffDims(B, H, Tq, Tk, D)
    more = [at(i) if stats else None for i in (6, 7, 8)]
    assert lib.rt_attn_diff(at(0), at(1), at(2), at(3), 1, at(4) if lens else None, dims, at(5), *more, at(9), 1 << 40, None) == 0
    by_keys, split, by_len = lib.rt_seen()[:3]
    return ("few" if Tq <= 16 else "keys") if by_keys else "tile", split > 1, bool(by_len)


def backward(lib, B, H, Tq, Tk, D, lens):
    """(waves of a tile, which walks are in parts, row values in the same launch, samples taken by their keys)."""
    dims = _lib.RtDiffDims(B, H, Tq, Tk, D)
    status = lib.rt_attn_diff_backward(at(0), at(1), at(2), at(3), H, at(4) if lens else None, at(5), at(6), at(7), at(8), at(9), dims,
                                       at(10), at(11), at(12), at(13), at(14), 1 << 40, None)
    assert status == 0
    two, split_k, split_q, short, by_len = lib.rt_seen()[:5]
    return 8 if two else 4, ("k" if split_k > 1 else "") + ("q" if split_q > 1 else ""), bool(short), bool(by_len)
