"""bench.py's HBM traffic goes by a hash of the fused kernel's sources: the committed summary is of these."""

import bench


def test_committed_traffic_is_of_the_sources():
    assert bench.measured_traffic("cogvideox_2b") is not None
