"""The sanitized build has the host code of the operators in it, not the entry points' alone: a read past the end of a set's arrays, which
the driver makes the library commit, is reported."""
import os
import subprocess

import pytest

from paper_2409_12210_amd import build as modse_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if not all(os.path.exists(os.path.join(modse_build.CSRC, s.replace(".hip", ".o"))) for s in modse_build.SOURCES):
        modse_build.build(verbose=False)
    return modse_build.build_host_sanitized(str(tmp_path_factory.mktemp("san")), os.path.join(ROOT, "tests", "host_overread_driver.c"))


@pytest.mark.parametrize("which,where", [("rows", "ortho_layout"), ("cols", "ortho_layout"), ("coeffs", "modse_orthogonalize"), ("none", None)])
def test_a_read_past_the_arrays_is_reported(driver, which, where):
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=0:abort_on_error=0")
    r = subprocess.run([driver, which], capture_output=True, text=True, env=env, timeout=300)
    report = r.stdout + r.stderr
    if where is None:
        assert r.returncode == 0 and "AddressSanitizer" not in report, report
    else:
        assert "heap-buffer-overflow" in report and where in report, report


def test_every_source_of_the_operators_is_in_the_sanitized_build():
    assert {"ops_api.hip", "norm.hip", "logprobs.hip", "ortho.hip"} <= set(modse_build.HOST_SOURCES)
