"""CPU: the benchmark's timed loops leave the garbage collector as they found it."""
import gc

import pytest

import bench


@pytest.mark.parametrize("on", [True, False])
@pytest.mark.parametrize("fails", [True, False])
def test_without_collection(on, fails):
    was = gc.isenabled()
    try:
        (gc.enable if on else gc.disable)()
        try:
            with bench.without_collection():
                assert not gc.isenabled()
                if fails:
                    raise RuntimeError("a call failed")
        except RuntimeError:
            assert fails
        assert gc.isenabled() == on
    finally:
        (gc.enable if was else gc.disable)()
