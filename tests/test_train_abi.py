"""C-ABI refusals of the training calls, found on the host before anything is enqueued (no GPU needed), and the same
under AddressSanitizer and UndefinedBehaviorSanitizer with stand-ins for the launchers."""

import ctypes
import os
import subprocess
import sys

import pytest

from paper_2505_22918_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
FAKE = 0x7F0000000000  # 16-byte aligned, never dereferenced
Q, K, V, O, DO, DQ, DK, DV, WS = (FAKE + i * 0x100000 for i in range(9))
M, L, RHO, DRHO = (FAKE + 0x1000000 + i * 0x100000 for i in range(4))
RP, CI, TRP, TCI = (FAKE + 0x2000000 + i * 0x100000 for i in range(4))
BIG = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def _dims(B=1, H=2, T=256, D=64):
    return _lib.RtDims(B, H, T, D)


def _bsr(rp=RP, ci=CI, block=64, n=4, nnz=8, masks=0):
    return _lib.RtBsr(rp, ci, block, n, nnz, masks)


def _t(**kw):
    return _bsr(**{"rp": TRP, "ci": TCI, **kw})


def _full(lib, dims=None, nbytes=BIG, **kw):
    a = dict(q=Q, k=K, v=V, o=O, m=M, l=L, do=DO, dq=DQ, dk=DK, dv=DV, ws=WS)
    a.update(kw)
    return lib.rt_attn_full_backward(a["q"], a["k"], a["v"], a["o"], a["m"], a["l"], a["do"], dims or _dims(), a["dq"],
                                     a["dk"], a["dv"], a["ws"], nbytes, None)


def _sparse(lib, dims=None, mask=None, t=None, rho=RHO, delta=0.0, drho=DRHO, nbytes=BIG, **kw):
    a = dict(q=Q, k=K, v=V, o=O, m=M, l=L, do=DO, dq=DQ, dk=DK, dv=DV, ws=WS)
    a.update(kw)
    mask, t = (ctypes.byref(x) if x is not None else None for x in (_bsr() if mask is None else mask,
                                                                     _t() if t is None else t))
    return lib.rt_attn_sparse_backward(a["q"], a["k"], a["v"], a["o"], a["m"], a["l"], a["do"], dims or _dims(), mask, t,
                                       rho, delta, a["dq"], a["dk"], a["dv"], drho, a["ws"], nbytes, None)


@pytest.mark.parametrize("name", ["q", "k", "v", "o", "m", "l", "do", "dq", "dk", "dv", "ws"])
def test_gradient_calls_need_every_tensor(lib, name):
    assert _full(lib, **{name: None}) == _lib.RT_EINVAL
    assert _sparse(lib, **{name: None}) == _lib.RT_EINVAL
    assert _full(lib, **{name: Q + 2 if name not in "ml" else M + 2}) == _lib.RT_EINVAL
    assert "aligned" in lib.rt_last_error().decode()


def test_gradient_calls_refuse_shapes_and_overlaps(lib):
    for call in (_full, _sparse):
        assert call(lib, dims=_dims(D=80)) == _lib.RT_EUNSUPPORTED
        assert call(lib, dims=_dims(B=-1)) == _lib.RT_EINVAL
        assert call(lib, nbytes=256 * 2 * 8 - 1) == _lib.RT_ECAPACITY
        for out in ("dq", "dk", "dv", "ws"):
            for at in (Q, V + 16, O, DO, M, L):
                assert call(lib, **{out: at & ~15}) == _lib.RT_EINVAL
                assert "overlaps" in lib.rt_last_error().decode()
        assert call(lib, dq=DK) == _lib.RT_EINVAL
        assert call(lib, ws=DV) == _lib.RT_EINVAL
    # heads past the 32-bit offsets of one buffer
    assert _full(lib, dims=_dims(T=1 << 24)) == _lib.RT_EINVAL
    # nothing to do: the arguments behind the shape are not looked at
    assert _full(lib, dims=_dims(T=0), q=None) == _lib.RT_OK


def test_sparse_gradient_refusals(lib):
    assert _sparse(lib, mask=_bsr(n=5)) == _lib.RT_EINVAL
    assert _sparse(lib, mask=_bsr(block=48)) == _lib.RT_EUNSUPPORTED
    assert _sparse(lib, mask=_bsr(masks=3)) == _lib.RT_EINVAL
    assert _sparse(lib, t=_t(n=5)) == _lib.RT_EINVAL
    assert _sparse(lib, t=_t(block=32)) == _lib.RT_EINVAL
    assert _sparse(lib, t=_t(masks=2)) == _lib.RT_EINVAL
    assert _sparse(lib, t=_t(nnz=7)) == _lib.RT_ECAPACITY
    assert _sparse(lib, t=_t(rp=None)) == _lib.RT_EINVAL
    assert _sparse(lib, delta=float("nan")) == _lib.RT_EINVAL
    assert _sparse(lib, delta=float("inf")) == _lib.RT_EINVAL
    assert _sparse(lib, rho=None) == _lib.RT_EINVAL  # d_rho without rho
    assert _sparse(lib, drho=RHO) == _lib.RT_EINVAL
    assert _sparse(lib, drho=DQ) == _lib.RT_EINVAL
    assert _sparse(lib, dq=CI) == _lib.RT_EINVAL
    assert _sparse(lib, dv=TCI) == _lib.RT_EINVAL
    assert lib.rt_attn_sparse_backward(Q, K, V, O, M, L, DO, _dims(), None, ctypes.byref(_t()), None, 0.0, DQ, DK, DV,
                                       None, WS, BIG, None) == _lib.RT_EINVAL
    assert lib.rt_attn_sparse_backward(Q, K, V, O, M, L, DO, _dims(), ctypes.byref(_bsr()), None, None, 0.0, DQ, DK, DV,
                                       None, WS, BIG, None) == _lib.RT_EINVAL


def test_workspace_sizes(lib):
    n = ctypes.c_int64(-1)
    assert lib.rt_attn_full_backward_workspace(_dims(), ctypes.byref(n)) == _lib.RT_OK and n.value >= 256 * 2 * 8
    assert lib.rt_attn_sparse_backward_workspace(_dims(), ctypes.byref(_bsr()), 0, ctypes.byref(n)) == _lib.RT_OK
    assert n.value >= 256 * 2 * 8
    assert lib.rt_attn_full_backward_workspace(_dims(D=80), ctypes.byref(n)) == _lib.RT_EUNSUPPORTED
    assert lib.rt_attn_full_backward_workspace(_dims(), None) == _lib.RT_EINVAL
    assert lib.rt_attn_sparse_backward_workspace(_dims(), ctypes.byref(_bsr(n=3)), 0, ctypes.byref(n)) == _lib.RT_EINVAL
    assert lib.rt_attn_sparse_backward_workspace(_dims(), ctypes.byref(_bsr()), 7, ctypes.byref(n)) == _lib.RT_ECAPACITY
    assert lib.rt_index_transpose_size(ctypes.byref(_bsr()), 8, ctypes.byref(n)) == _lib.RT_OK and n.value >= 8 + 4 * 4
    assert lib.rt_index_transpose_size(ctypes.byref(_bsr()), -1, ctypes.byref(n)) == _lib.RT_EINVAL
    assert lib.rt_index_transpose_size(None, 8, ctypes.byref(n)) == _lib.RT_EINVAL
    assert lib.rt_index_transpose_size(ctypes.byref(_bsr()), 8, None) == _lib.RT_EINVAL


def test_transpose_refusals(lib):
    def call(mask, T=256, t=None):
        return lib.rt_index_transpose(ctypes.byref(mask) if mask is not None else None, T,
                                      ctypes.byref(t if t is not None else _t()), None)

    assert call(None) == _lib.RT_EINVAL
    assert call(_bsr(), T=300) == _lib.RT_EINVAL
    assert call(_bsr(block=16)) == _lib.RT_EUNSUPPORTED
    assert call(_bsr(), t=_t(nnz=7)) == _lib.RT_ECAPACITY
    assert call(_bsr(), t=_t(rp=RP)) == _lib.RT_EINVAL
    assert call(_bsr(), t=_t(ci=CI + 8)) == _lib.RT_EINVAL
    assert call(_bsr(), t=_t(ci=TRP)) == _lib.RT_EINVAL
    assert call(_bsr(rp=None)) == _lib.RT_EINVAL


X, Y, W8, B8, MEAN, RSTD, DX, DW, DB = (FAKE + 0x3000000 + i * 0x100000 for i in range(9))


def _nd(n0=2, n1=3, n2=5, W=64, t=0, wt=2, sets=1):
    return _lib.RtNormDims(n0, n1, n2, W, t, wt, sets)


def _s(n1=3, n2=5, W=64):
    return _lib.Strides(n1 * n2 * W, n2 * W, W)


def _norm(lib, dims=None, xs=None, ys=None, eps=1e-5, **kw):
    a = dict(x=X, w=W8, b=B8, y=Y, mean=MEAN, rstd=RSTD)
    a.update(kw)
    return lib.rt_layer_norm(a["x"], xs or _s(), a["w"], a["b"], dims or _nd(), eps, a["y"], ys or _s(), a["mean"],
                             a["rstd"], None)


def _norm_bwd(lib, dims=None, dys=None, xs=None, dxs=None, nbytes=BIG, **kw):
    a = dict(dy=Y, x=X, mean=MEAN, rstd=RSTD, w=W8, dx=DX, dw=DW, db=DB, ws=WS)
    a.update(kw)
    return lib.rt_layer_norm_backward(a["dy"], dys or _s(), a["x"], xs or _s(), a["mean"], a["rstd"], a["w"],
                                      dims or _nd(), a["dx"], dxs or _s(), a["dw"], a["db"], a["ws"], nbytes, None)


def test_norm_refusals(lib):
    for call in (_norm, _norm_bwd):
        assert call(lib, dims=_nd(W=0)) == _lib.RT_EINVAL
        assert call(lib, dims=_nd(W=16385)) == _lib.RT_EUNSUPPORTED
        assert call(lib, dims=_nd(n1=-1)) == _lib.RT_EINVAL
        assert call(lib, dims=_nd(t=3)) == _lib.RT_EUNSUPPORTED
        assert call(lib, dims=_nd(t=0, wt=1)) == _lib.RT_EUNSUPPORTED
        assert call(lib, dims=_nd(sets=3)) == _lib.RT_EINVAL
        assert call(lib, dims=_nd(n0=70000, sets=70000)) == _lib.RT_EUNSUPPORTED
        assert call(lib, dims=_nd(n0=1 << 16, n1=1 << 15)) == _lib.RT_EINVAL
        assert call(lib, x=None) == _lib.RT_EINVAL
        assert call(lib, x=X + 1) == _lib.RT_EINVAL
        assert call(lib, xs=_lib.Strides(-64, 64, 64)) == _lib.RT_EINVAL
        assert call(lib, xs=_lib.Strides(1 << 62, 64, 64)) == _lib.RT_EINVAL
        assert call(lib, w=W8 + 2) == _lib.RT_EINVAL
    for eps in (-1e-5, float("nan"), float("inf")):
        assert _norm(lib, eps=eps) == _lib.RT_EINVAL
    # rows of an output that share memory, spans that overlap
    for s in (_lib.Strides(0, 320, 64), _lib.Strides(960, 320, 63), _lib.Strides(64, 64, 64), _lib.Strides(500, 320, 64)):
        assert _norm(lib, ys=s) == _lib.RT_EINVAL
        assert "share memory" in lib.rt_last_error().decode()
        assert _norm_bwd(lib, dxs=s) == _lib.RT_EINVAL
    assert _norm(lib, y=X) == _lib.RT_EINVAL
    assert _norm(lib, y=X + 30 * 64 * 2 - 16) == _lib.RT_EINVAL
    assert _norm(lib, mean=X) == _lib.RT_EINVAL
    assert _norm(lib, mean=RSTD) == _lib.RT_EINVAL
    assert _norm(lib, y=W8) == _lib.RT_EINVAL
    assert _norm_bwd(lib, dx=Y) == _lib.RT_EINVAL
    assert _norm_bwd(lib, dw=DB) == _lib.RT_EINVAL
    assert _norm_bwd(lib, ws=DW) == _lib.RT_EINVAL
    assert _norm_bwd(lib, mean=None) == _lib.RT_EINVAL
    assert _norm_bwd(lib, ws=None) == _lib.RT_EINVAL
    assert _norm_bwd(lib, nbytes=100) == _lib.RT_ECAPACITY
    n = ctypes.c_int64()
    assert lib.rt_layer_norm_backward_workspace(_nd(W=0), ctypes.byref(n)) == _lib.RT_EINVAL
    assert lib.rt_layer_norm_backward_workspace(_nd(), None) == _lib.RT_EINVAL
    assert _norm(lib, dims=_nd(n1=0)) == _lib.RT_OK


def test_valid_calls_reach_the_launchers(lib):
    """Only against the stand-ins, which launch nothing."""
    if not os.environ.get("RT_LIB_PATH"):
        pytest.skip("launches kernels on made-up pointers with the real library")
    assert _full(lib) == _lib.RT_OK and _sparse(lib) == _lib.RT_OK
    assert _sparse(lib, rho=None, drho=None) == _lib.RT_OK
    for n in (0, 1, 2):
        assert _sparse(lib, mask=_bsr(masks=n), t=_t(masks=n)) == _lib.RT_OK
    assert lib.rt_index_transpose(ctypes.byref(_bsr(masks=7)), 256, ctypes.byref(_t(masks=7)), None) == _lib.RT_OK
    assert _norm(lib) == _lib.RT_OK and _norm_bwd(lib) == _lib.RT_OK
    assert _norm(lib, dims=_nd(sets=2), mean=None, rstd=None, w=None, b=None) == _lib.RT_OK
    assert _norm(lib, ys=_lib.Strides(64, 128, 384)) == _lib.RT_OK
    assert _norm_bwd(lib, dims=_nd(n2=0), x=None) == _lib.RT_OK


@pytest.mark.skipif(bool(os.environ.get("LD_PRELOAD")),
                    reason="a preload is already set here; the sanitizer runtime is not stacked on it")
def test_these_tests_pass_under_asan_and_ubsan(tmp_path):
    sys.path.insert(0, os.path.join(HERE, "sanitize"))
    import build as sbuild

    asan = subprocess.run(["g++", "-print-file-name=libasan.so"], capture_output=True, text=True).stdout.strip()
    if not (os.path.isabs(asan) and os.path.exists(asan)):
        pytest.skip("host compiler has no AddressSanitizer runtime")
    out = str(tmp_path / "librettention_asan.so")
    cmd = sbuild.command(out)
    cmd.insert(cmd.index("-o"), os.path.join(HERE, "sanitize", "train_stubs.cpp"))
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    reports = tmp_path / "report"
    env = dict(os.environ, LD_PRELOAD=asan, RT_LIB_PATH=out,
               ASAN_OPTIONS=f"detect_leaks=0:halt_on_error=1:log_path={reports}",
               UBSAN_OPTIONS=f"halt_on_error=1:print_stacktrace=1:log_path={reports}")
    res = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "not gpu", "tests/test_train_abi.py"],
                         cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    written = sorted(p.name for p in tmp_path.glob("report*"))
    assert not written, "sanitizer reports: " + " ".join((tmp_path / n).read_text()[:2000] for n in written)
    assert res.returncode == 0 and " passed" in res.stdout, res.stdout[-4000:] + res.stderr[-4000:]
