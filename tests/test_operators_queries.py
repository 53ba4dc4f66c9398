"""The workspace queries of the training operators, at sizes that no call takes, and their checks under sanitizers (CPU)."""
import os
import subprocess
import sys

import pytest

from paper_2609_27193_amd.build_lib import SANITIZED_LIB, sanitizer_runtime
from tests.conftest import ROOT


@pytest.mark.parametrize("query,sizes", [("lc_embedding_backward_workspace", (5000, 0)), ("lc_embedding_backward_workspace", (2049, 0)),
                                         ("lc_embedding_backward_workspace", (1 << 31, 0)), ("lc_embedding_backward_workspace", (0, 0)),
                                         ("lc_embedding_backward_workspace", ((1 << 31) + 1, 8)), ("lc_embedding_backward_workspace", (5000, (1 << 30) + 1)),
                                         ("lc_embedding_backward_workspace", ((1 << 64) - 1, (1 << 64) - 1)),
                                         ("lc_norm_backward_workspace", (5000, 0)), ("lc_norm_backward_workspace", (0, 0)),
                                         ("lc_norm_backward_workspace", ((1 << 64) - 1, (1 << 64) - 1)),
                                         ("lc_linear_wgrad_workspace", (5000, 0, 8)), ("lc_linear_wgrad_workspace", (5000, 8, 0)),
                                         ("lc_linear_wgrad_workspace", (0, 0, 0)), ("lc_linear_wgrad_workspace", ((1 << 64) - 1,) * 3)])
def test_nothing_is_needed_beyond_the_limits(query, sizes):
    """In a child process: a query must not end the program."""
    r = subprocess.run([sys.executable, "-c", f"from paper_2609_27193_amd import layercheck as LC; print(LC.{query}{sizes})"],
                       cwd=ROOT, capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.split()[-1] == "0", (r.returncode, r.stdout, r.stderr)


@pytest.mark.parametrize("n,cols", [(1 << 31, 1 << 30), (1 << 31, 1), (2049, 1 << 30)])
def test_the_largest_sizes_have_one(n, cols):
    from paper_2609_27193_amd import layercheck as LC
    assert LC.lc_embedding_backward_workspace(n, cols) >= 8 * n
    assert LC.lc_norm_backward_workspace(n, cols) >= 8 * cols


def test_checks_and_queries_under_host_sanitizers():
    rt = sanitizer_runtime()
    if not os.path.exists(SANITIZED_LIB) or not rt:
        pytest.skip("the host-sanitized library is built by __graft_entry__.build()")
    env = dict(os.environ, LD_PRELOAD=rt, LAYERCHECK_LIB=SANITIZED_LIB, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "-m", "not gpu", "-k", "not sanitizers",
                        "tests/test_operators_abi.py", "tests/test_operators_apart.py", "tests/test_operators_queries.py"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "ERROR: AddressSanitizer" not in tail and "runtime error:" not in tail, tail
