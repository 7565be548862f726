"""The argument checks of the operators at both ends of a model under AddressSanitizer and UndefinedBehaviorSanitizer (host code only,
nothing is launched)."""
import os
import subprocess

from paper_2409_12210_amd import build as modse_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_argument_checks_of_the_operators_are_clean_under_sanitizers(tmp_path):
    if not all(os.path.exists(os.path.join(modse_build.CSRC, s.replace(".hip", ".o"))) for s in modse_build.SOURCES):
        modse_build.build(verbose=False)
    exe = modse_build.build_host_sanitized(str(tmp_path), os.path.join(ROOT, "tests", "host_ends_driver.c"))
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=0:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    report = r.stdout + r.stderr
    assert "AddressSanitizer" not in report and "runtime error" not in report, report
    assert r.returncode == 0 and "all checks passed" in r.stdout, report


def test_every_source_of_the_operators_is_in_the_sanitized_build():
    assert {"ops_api.hip", "embed.hip", "head.hip", "dropout.hip"} <= set(modse_build.HOST_SOURCES)
