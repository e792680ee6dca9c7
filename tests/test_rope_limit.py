"""The largest calls of rotary positions that one launch takes (CPU): as the header states it, for every layout and width of
an access."""

import itertools

import pytest

import diff_plans
from paper_2505_22918_amd import _lib


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return diff_plans.build(str(tmp_path_factory.mktemp("rope_limit")))


def _call(lib, B, H, T, D, type, rotated, half, shift=0):
    """y [B, H, T, D] contiguous, `shift` elements past a 16-byte boundary; x one row for all, as y."""
    size = 4 if type == _lib.RT_F32 else 2
    dims = _lib.RtRopeDims(B, H, T, D, type, rotated, half, 1, _lib.RT_POS_I32, 0)
    at = diff_plans.at
    return lib.rt_rope(at(0) + shift * size, _lib.Strides(0, 0, 0), at(1), at(2), None, 1.0, dims, at(8) + shift * size,
                       _lib.Strides(H * T * D, T * D, D), None)


def _threads(D, type, rotated, half, shift):
    """v and n of the header: elements of an access, threads of a token."""
    v = next(v for v in (8, 4, 1) if v == 1 or (v * (4 if type == _lib.RT_F32 else 2) <= 16 and D % v == 0 and shift % v == 0
                                                and not (half and rotated // 2 % v)))
    return v, D // v if v > 1 and not half else rotated // 2 // v + (D - rotated) // v


WIDTHS = [(64, 64, 0), (64, 64, 4), (64, 64, 1), (64, 48, 0), (72, 72, 0), (72, 48, 0), (72, 24, 0), (66, 66, 0), (127, 126, 0), (8, 8, 0), (2, 2, 0), (128, 2, 0)]


@pytest.mark.parametrize("type", range(3))
@pytest.mark.parametrize("half", range(2))
@pytest.mark.parametrize("D,rotated,shift", WIDTHS)
def test_the_largest_calls(lib, D, rotated, shift, half, type):
    v, n = _threads(D, type, rotated, half, shift)
    seen = 0
    for B, H in itertools.product((1, 3, 100, 70001, (1 << 24) - 1, 1 << 24), (1, 5)):
        # the most tokens by the header's rule, and one more
        T = ((1 << 24) - 1) // B * 256 // n
        for t in (T, T + 1):
            if not 0 < t < (1 << 32) // D or t >= 1 << 31 or B * H * t * D >= 1 << 38:
                continue
            fits = B * -(-t * n // 256) < 1 << 24
            assert _call(lib, B, H, t, D, type, rotated, half, shift) == (_lib.RT_OK if fits else _lib.RT_EINVAL), (B, H, t)
            if fits:
                assert lib.rt_seen()[0] == v and lib.rt_blocks() < 1 << 24
                seen += lib.rt_blocks() > 1 << 23
    assert seen
