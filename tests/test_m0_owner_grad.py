"""M0 has one owner in the gradients' device code too: its LDS DMAs set it in their own inline-assembly blocks, and
nothing else in the compiled code may name or read it (see test_m0_owner.py)."""

import os

import pytest

from paper_2505_22918_amd import build
from test_m0_owner import _device_asm, _instructions, check_m0


@pytest.mark.skipif(not os.path.exists(build.hipcc()), reason="hipcc not installed")
@pytest.mark.parametrize("src", build.GRAD_SOURCES)
def test_m0_is_written_only_by_the_dma_blocks(tmp_path, src):
    assert check_m0(_instructions(_device_asm(src, str(tmp_path / (src + ".s")))), src) > 0
