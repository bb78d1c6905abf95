"""The cache's GPU tests once more on the bounds-checking build, whose kernels check the indices they write to and report through
dev_status (the tests assert that it stays 0)."""
import os
import sys

import pytest

from test_gpu_bounds_check import ROOT, checked_lib, run_child  # noqa: F401

pytestmark = pytest.mark.gpu


def test_the_cache_on_the_checked_build(checked_lib):  # noqa: F811
    r = run_child([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider", os.path.join("tests", "test_gpu_cache.py"),
                   "-k", "histories or few_rows or chunks or selection or clip"], checked_lib)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
