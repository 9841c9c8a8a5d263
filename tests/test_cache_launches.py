"""Launches of libcpcache's selection and attention on the host."""

import shutil

import pytest

from test_native_sanitizers import _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_launches_under_sanitizers(tmp_path):
    """Host C++: the workgroups of random batches and of the largest ones, each
    launched once, and the grids' limits (tests/native/cache_launches.cpp)."""
    assert _build_and_run(tmp_path, "cache_launches.cpp", ["cache_plan.cpp"]).startswith("ok")
