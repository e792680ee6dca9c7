"""C-ABI refusals of rotary positions and differential attention, found on the host before anything is enqueued (no GPU
needed), and the same under AddressSanitizer and UndefinedBehaviorSanitizer with stand-ins for the launchers."""

import ctypes
import os
import subprocess
import sys

import pytest

from paper_2505_22918_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FAKE = 0x7F0000000000  # 16-byte aligned, never dereferenced
AT = {n: FAKE + i * 0x1000000 for i, n in enumerate(("x", "y", "pos", "freq", "axis", "q", "k", "v", "lam", "lens", "o", "o2",
                                                       "m", "l", "do", "dq", "dk", "dv", "dlam", "ws"))}
BIG = 1 << 23


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def _rope(lib, fn="rt_rope", xs=(0, 64 * 5, 64), ys=(0, 64 * 5, 64), amplitude=1.0, B=1, H=3, T=5, D=64, type=0, rotated=64,
          layout=0, axes=1, position_type=1, per_sample=0, **kw):
    a = {n: AT[n] for n in ("x", "y", "pos", "freq", "axis")}
    a.update(kw)
    strides = [_lib.Strides(*s) for s in (xs, ys)]
    dims = _lib.RtRopeDims(B, H, T, D, type, rotated, layout, axes, position_type, per_sample)
    return getattr(lib, fn)(a["x"], strides[0], a["pos"], a["freq"], a["axis"], amplitude, dims, a["y"], strides[1], None)


@pytest.mark.parametrize("fn", ["rt_rope", "rt_rope_backward"])
def test_rope_refusals(lib, fn):
    bad = [dict(B=-1), dict(T=-1), dict(D=1, rotated=2), dict(rotated=63), dict(rotated=0), dict(rotated=66), dict(axes=0),
           dict(amplitude=float("nan")), dict(amplitude=float("inf")), dict(x=None), dict(y=None), dict(pos=None), dict(freq=None),
           dict(axes=2, axis=None), dict(x=AT["x"] + 1), dict(pos=AT["pos"] + 4), dict(freq=AT["freq"] + 4),
           dict(axes=2, axis=AT["axis"] + 2), dict(xs=(0, -320, 64)), dict(ys=(0, 320, 32)),
           dict(ys=(0, 0, 64)), dict(y=AT["pos"]), dict(y=AT["freq"]), dict(y=AT["axis"], axes=2), dict(y=AT["x"] + 128),
           dict(y=AT["x"], xs=(0, 640, 64)), dict(T=1 << 30, D=64), dict(B=1 << 20, H=1 << 20, T=1, ys=(64 << 20, 64, 0))]
    for kw in bad:
        assert _rope(lib, fn, **kw) == _lib.RT_EINVAL, kw
        assert lib.rt_last_error()
    for kw in (dict(type=3), dict(layout=2), dict(position_type=3), dict(D=16385), dict(axes=17)):
        assert _rope(lib, fn, **kw) == _lib.RT_EUNSUPPORTED, kw
    # too many workgroups of one launch
    assert _rope(lib, fn, T=1 << 25, D=127, ys=(0, 127 << 25, 127)) == _lib.RT_EINVAL
    # nothing to do: the arguments behind the shape are not looked at
    for n in ("B", "H", "T"):
        assert _rope(lib, fn, **{n: 0}, x=None, pos=None) == _lib.RT_OK


def _dims(B=1, H=2, Tq=40, Tk=50, D=64):
    return _lib.RtDiffDims(B, H, Tq, Tk, D)


def _fwd(lib, dims=None, n_lam=2, nbytes=BIG, **kw):
    a = {n: AT[n] for n in ("q", "k", "v", "lam", "lens", "o", "o2", "m", "l", "ws")}
    a.update(kw)
    return lib.rt_attn_diff(a["q"], a["k"], a["v"], a["lam"], n_lam, a["lens"], dims or _dims(), a["o"], a["o2"], a["m"], a["l"],
                            a["ws"], nbytes, None)


def _bwd(lib, dims=None, n_lam=2, nbytes=BIG, **kw):
    a = {n: AT[n] for n in ("q", "k", "v", "lam", "lens", "o", "o2", "m", "l", "do", "dq", "dk", "dv", "dlam", "ws")}
    a.update(kw)
    return lib.rt_attn_diff_backward(a["q"], a["k"], a["v"], a["lam"], n_lam, a["lens"], a["o"], a["o2"], a["m"], a["l"], a["do"],
                                     dims or _dims(), a["dq"], a["dk"], a["dv"], a["dlam"], a["ws"], nbytes, None)


SPLIT = _dims(Tq=1, Tk=4096)  # few rows over many keys: parts of them, in the workspace


@pytest.mark.parametrize("name", ["q", "k", "v", "lam", "o", "o2", "m", "l", "ws", "do", "dq", "dk", "dv", "dlam"])
def test_differential_attention_needs_every_tensor(lib, name):
    odd = AT[name] + 2
    if name not in ("do", "dq", "dk", "dv", "dlam"):
        assert _fwd(lib, SPLIT, **{name: None}) == _lib.RT_EINVAL
        assert _fwd(lib, SPLIT, **{name: odd}) == _lib.RT_EINVAL
        assert "aligned" in lib.rt_last_error().decode()
    assert _bwd(lib, **{name: None}) == _lib.RT_EINVAL
    assert _bwd(lib, **{name: odd}) == _lib.RT_EINVAL
    assert "aligned" in lib.rt_last_error().decode()


def test_differential_attention_refuses_shapes_and_overlaps(lib):
    for call in (_fwd, _bwd):
        assert call(lib, _dims(D=80)) == _lib.RT_EUNSUPPORTED
        assert call(lib, _dims(B=-1)) == _lib.RT_EINVAL
        assert call(lib, _dims(Tk=-1)) == _lib.RT_EINVAL
        assert call(lib, n_lam=3) == _lib.RT_EINVAL
        assert call(lib, n_lam=0) == _lib.RT_EINVAL
        assert call(lib, lens=AT["lens"] + 2) == _lib.RT_EINVAL
        assert call(lib, _dims(Tk=1 << 23)) == _lib.RT_EINVAL
        assert call(lib, _dims(Tq=1 << 23)) == _lib.RT_EINVAL
        assert call(lib, _dims(B=1 << 12, H=1 << 11), n_lam=1) == _lib.RT_EINVAL
        assert call(lib, _dims(B=1 << 10, H=1 << 9, Tq=1024), n_lam=1) == _lib.RT_EINVAL
    for out in ("o", "o2", "m", "l"):
        for at in ("q", "k", "v", "lam", "lens"):
            assert _fwd(lib, **{out: AT[at]}) == _lib.RT_EINVAL
            assert "overlaps" in lib.rt_last_error().decode()
    assert _fwd(lib, o=AT["o2"]) == _lib.RT_EINVAL
    assert _fwd(lib, SPLIT, ws=AT["k"]) == _lib.RT_EINVAL
    assert _fwd(lib, SPLIT, ws=AT["o"]) == _lib.RT_EINVAL
    assert _fwd(lib, o2=None) == _lib.RT_EINVAL
    assert _fwd(lib, m=None, l=None) == _lib.RT_EINVAL
    for out in ("dq", "dk", "dv", "dlam", "ws"):
        for at in ("q", "k", "v", "lam", "lens", "o", "o2", "m", "l", "do"):
            assert _bwd(lib, **{out: AT[at]}) == _lib.RT_EINVAL
            assert "overlaps" in lib.rt_last_error().decode()
    assert _bwd(lib, dq=AT["dk"]) == _lib.RT_EINVAL
    assert _bwd(lib, ws=AT["dv"]) == _lib.RT_EINVAL


@pytest.mark.parametrize("dims", [_dims(), SPLIT, _dims(2, 15, 17776, 17776), _dims(4, 8, 4096, 226, 72), _dims(1, 1, 0, 9), _dims(1, 1, 9, 0),
                                  _dims(1, 1, 64, 4096, 72), _dims(8, 15, 1, 8192)])
def test_workspaces_are_checked_to_the_byte(lib, dims):
    need = ctypes.c_int64(-1)
    for name, call in (("rt_attn_diff", _fwd), ("rt_attn_diff_backward", _bwd)):
        size = getattr(lib, name + "_workspace")
        assert size(dims, ctypes.byref(need)) == _lib.RT_OK and need.value >= 16
        if need.value > 16 and need.value < 1 << 24:
            assert call(lib, dims, n_lam=1, nbytes=need.value - 1) == _lib.RT_ECAPACITY
        assert size(dims, None) == _lib.RT_EINVAL
        assert size(_dims(D=65), ctypes.byref(need)) == _lib.RT_EUNSUPPORTED


def test_nothing_to_do(lib):
    for d in (_dims(B=0), _dims(H=0), _dims(Tq=0)):
        assert _fwd(lib, d, q=None, o=None) == _lib.RT_OK
    assert _bwd(lib, _dims(H=0), n_lam=0, lam=None, dlam=None, q=None) == _lib.RT_OK


STUBS = r"""
#include <hip/hip_runtime_api.h>
#include <cstdio>
#include <cstdlib>
#include "heads.h"
#define EXPECT(c) do { if (!(c)) { std::fprintf(stderr, "launch stub: expectation failed: %s\n", #c); std::abort(); } } while (0)
namespace rt {
hipError_t launch_rope(const RopeArgs& a, hipStream_t) {
    EXPECT(a.x && a.y && a.positions && a.freq && a.B > 0 && a.H > 0 && a.T > 0 && a.pairs > 0 && 2 * a.pairs <= a.D);
    EXPECT((a.vec == 1 || a.vec == 4 || a.vec == 8) && a.D % a.vec == 0 && (!a.half || a.pairs % a.vec == 0));
    EXPECT(a.each >= 1 && a.groups >= 1 && (int64_t)a.each * a.groups >= a.H && (int64_t)a.each * (a.groups - 1) < a.H);
    EXPECT(rope_blocks(a) > 0 && rope_blocks(a) < (1 << 24));
    return hipSuccess;
}
hipError_t launch_diff(const DiffArgs& a, int D, hipStream_t) {
    EXPECT((D == 64 || D == 72) && a.q && a.lam && a.o && a.Tq > 0 && a.n_bh > 0 && a.n_bh % a.H == 0);
    EXPECT(a.split >= 1 && (a.split == 1 || a.part));
    EXPECT((a.o2 && a.row_max && a.row_sum) || (!a.o2 && !a.row_max && !a.row_sum));
    return hipSuccess;
}
hipError_t launch_diff_backward(const DiffArgs& a, int D, hipStream_t) {
    EXPECT((D == 64 || D == 72) && a.lam && a.d_lam && a.T64 >= a.Tq && a.T64 < a.Tq + 64 && a.T64 % 64 == 0);
    EXPECT(a.split_k >= 1 && a.split_q >= 1 && a.part_k >= a.row_vals && a.part_q >= a.part_k);
    return hipSuccess;
}
}  // namespace rt
"""


def test_accepted_calls_reach_the_launchers_sound(tmp_path):
    """The refusals above and accepted calls against a sanitizer build of the host code."""
    sys.path.insert(0, os.path.join(HERE, "sanitize"))
    import build as sbuild
    from test_sanitize import _runtime

    asan = _runtime("libasan.so")
    if asan is None or os.environ.get("LD_PRELOAD"):
        pytest.skip("no AddressSanitizer runtime, or a preload is already set")
    (tmp_path / "stubs.cpp").write_text(STUBS)
    lib = str(tmp_path / "librettention_asan.so")
    cmd = sbuild.command(lib)
    cmd[-2:-2] = [str(tmp_path / "stubs.cpp"), os.path.join(HERE, "sanitize", "train_stubs.cpp")]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    env = dict(os.environ, LD_PRELOAD=asan, RT_LIB_PATH=lib, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", PYTHONPATH=ROOT + os.pathsep + HERE)
    code = """
import itertools
import test_heads_abi as t
from paper_2505_22918_amd import _lib
lib = _lib.load()
t.test_rope_refusals(lib, "rt_rope")
t.test_differential_attention_refuses_shapes_and_overlaps(lib)
t.test_nothing_to_do(lib)
for ty, lay, D, T, H, axes, pos in itertools.product(range(3), range(2), (2, 64, 67, 72, 16384), (1, 5, 17776), (1, 3, 60), (1, 3), range(3)):
    if T == 17776 and D == 16384:
        continue
    for rot in {2, D // 2 * 2, D // 4 * 2 or 2}:
        s = (H * T * D, T * D, D)
        far = t.FAKE + (1 << 42)
        assert t._rope(lib, "rt_rope", s, s, 1.0, 2, H, T, D, ty, rot, lay, axes, pos, 1, y=far) == 0, lib.rt_last_error()
        assert t._rope(lib, "rt_rope_backward", s, s, 0.5, 2, H, T, D, ty, rot, lay, axes, pos, 0, x=far, y=far) == 0, lib.rt_last_error()
huge = {n: t.FAKE + (i << 40) for i, n in enumerate(t.AT)}
for B, H, Tq, Tk, D in itertools.product((1, 3), (1, 15), (1, 33, 4000, 17776), (0, 1, 226, 8192), (64, 72)):
    for n in {1, H}:
        a = {k: huge[k] for k in ("q", "k", "v", "lam", "lens", "o", "o2", "m", "l", "ws")}
        d = _lib.RtDiffDims(B, H, Tq, Tk, D)
        assert t._fwd(lib, d, n, 1 << 40, **a) == 0, lib.rt_last_error()
        assert t._fwd(lib, d, n, 1 << 40, **dict(a, o2=None, m=None, l=None, lens=None)) == 0, lib.rt_last_error()
        a.update({k: huge[k] for k in ("do", "dq", "dk", "dv", "dlam")})
        assert t._bwd(lib, d, n, 1 << 40, **a) == 0, lib.rt_last_error()
print("sound")
"""
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "sound" in out.stdout, out.stdout[-2000:] + out.stderr[-3000:]
