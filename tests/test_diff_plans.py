"""Which plan a call of differential attention takes (CPU): the sizes of the GPU tests reach every kernel that is compiled,
with a rule that goes by sizes alone and may be fitted anew."""

import ctypes
import itertools

import pytest

import diff_plans
from paper_2505_22918_amd import _lib
import test_gpu_attn_diff as sizes
import test_gpu_attn_diff_plans as plans


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return diff_plans.build(str(tmp_path_factory.mktemp("diff_plans")))


@pytest.mark.parametrize("case", plans.CASES + [(*c[:5], None, *c[5:]) for c in plans.RAMPS], ids=lambda c: "-".join(str(x) for x in c[:5]))
def test_sizes_take_the_plan_that_they_are_for(lib, case):
    *dims, lens, kernel, parts, waves, walks = case
    by_len = lens is not None and dims[0] > 1
    for stats in (False, True):
        assert diff_plans.forward(lib, *dims, lens is not None, stats) == (kernel, parts, by_len)
    assert diff_plans.backward(lib, *dims, lens is not None) == (waves, walks, False, by_len)


def test_every_kernel_is_reached(lib):
    """Each instance of diff_fwd, diff_few and diff_bwd, for both widths: test_sizes and test_plans call each size with and
    without statistics."""
    calls = [(*s, D, False) for s in sizes.SIZES for D in (64, 72)] + [(*c[:5], c[5] is not None) for c in plans.CASES]
    fwd, bwd = set(), set()
    for c in calls:
        fwd.add((c[4],) + diff_plans.forward(lib, *c)[:2])
        bwd.add((c[4],) + diff_plans.backward(lib, *c)[:3])
    assert fwd == set(itertools.product((64, 72), ("tile", "keys", "few"), (False, True)))
    walks = set(itertools.product((64, 72), (4, 8), ("", "k", "q", "kq"), (False,)))
    assert bwd == walks | set(itertools.product((64, 72), (4, 8), ("",), (True,)))


@pytest.mark.parametrize("backward,dims", [(1, (1, 1, 4096, 4096, 64)), (1, (4, 8, 4096, 226, 72)), (1, (5, 3, 2734, 1175, 64)), (0, (1, 1, 4096, 4096, 64))])
def test_a_call_makes_its_plans_once(lib, backward, dims):
    """The search for a plan is most of the host's work (microseconds).  A question for the workspace makes two, with numbers
    of keys and without; a call needs no third."""
    us = (ctypes.c_double * 2)()
    lib.rt_times(_lib.RtDiffDims(*dims), backward, us)
    print(f"workspace {us[0]:.2f} us, call {us[1]:.2f}")
    # a third search would be half as much again; the checks of 14 tensors are a few tenths of a microsecond
    assert us[1] <= 1.25 * us[0] + 0.2
