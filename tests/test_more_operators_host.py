"""What the host code of the residual norm, of the Newton-Schulz steps and of the mixed optimizer step asks of HIP, on the
stand-in for its host calls, and their checks of arguments under the host sanitizers (CPU)."""
import math
import os
import subprocess
import sys

import pytest

from paper_2609_27193_amd.build_lib import GRID_CAPPED_LIB, LIB, SANITIZED_LIB, sanitizer_runtime
from tests.test_host_calls import DEVICE, ROOT, hip, standin  # noqa: F401 (a fixture)


def in_child(standin, lib, scenario):  # noqa: F811
    env = dict(os.environ, LD_PRELOAD=standin, HIP_STANDIN=standin, LAYERCHECK_LIB=lib)
    r = subprocess.run([sys.executable, "-c", f"import tests.test_more_operators_host as t; t.{scenario}()"], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]


# ---- in the child ----------------------------------------------------------------------------------------------------------


def calls(h):
    """(name, call, the kernels that it launches in order)."""
    from paper_2609_27193_amd import layercheck as LC
    B, F = LC.LC_DT_BF16, LC.LC_DT_F32
    at = h.standin_alloc(1 << 20, DEVICE)
    apart = iter(range(1 << 33, 1 << 50, 1 << 33))  # never read: any addresses that lie apart
    M = lambda rows, cols, dt=B: LC.matrix(at + next(apart), rows, cols, dt)  # noqa: E731
    K = lambda rows, cols: LC.saved_act(at + next(apart), at + next(apart), rows, cols)  # noqa: E731
    V = lambda: at + next(apart)  # noqa: E731
    out = []
    norm = LC.norm_params(LC.LC_NORM_LAYER, V(), V(), F, 1e-5)
    for dim in (7, 8, 4096, 16384, 16385):
        kind = "long" if dim in (7, 16385) else "fwd_k"
        out.append((f"residual norm {dim}", lambda dim=dim: LC.lc_residual_norm_forward(norm, M(5, dim), M(5, dim), M(5, dim), M(5, dim),
                                                                                         saved=K(5, dim), y_saved=K(5, dim)), [kind]))

        def back(dim=dim, dx=True, dw=True):
            need = LC.lc_norm_backward_workspace(5, dim)
            LC.lc_residual_norm_backward(norm, M(5, dim), M(5, dim), V(), M(5, dim) if dx else None, None, V() if dw else 0, 0, F, V(),
                                         need, saved=K(5, dim))
        kind = "long" if kind == "long" else "bwd_k"
        out.append((f"gradient {dim}", back, [kind, "join"]))
        out.append((f"dx {dim}", lambda back=back: back(dw=False), [kind]))
    for n, rows, cols, steps, dt, joins in [(1, 1, 1, 1, B, False), (2, 64, 900, 5, F, True), (1, 600, 400, 3, B, False), (1, 128, 16384, 2, F, True),
                                            (64, 2048, 2048, 1, B, False)]:
        def go(n=n, rows=rows, cols=cols, steps=steps, dt=dt):
            need = LC.lc_orthogonalize_workspace(n, rows, cols, dt)
            LC.lc_orthogonalize(LC.orthogonalize_params(steps), [M(rows, cols) for _ in range(n)],
                                [M(rows, cols, dt) for _ in range(n)], V(), need)
        kernels = ["norm", "load"] + ["product"] * (3 * steps)
        if joins:
            kernels = ["norm", "load"] + ["product", "join", "product", "product"] * steps
        if n == 64:  # 16 at once
            kernels = kernels * 4
        out.append((f"orthogonalize {n} {rows} {cols}", go, kernels))
    return LC, out


def launches():
    h = hip()
    LC, todo = calls(h)
    for name, call, kernels in todo:
        h.standin_clear()
        call()
        got = h.words()
        assert len(got) == len(kernels) and all(k in g for k, g in zip(kernels, got)), (name, got)


def failures():
    h = hip()
    LC, todo = calls(h)
    for name, call, kernels in todo:
        for fail in range(1, len(kernels) + 1):  # every launch of the call fails once: nothing follows it
            h.standin_clear()
            h.standin_fail_launch(fail)
            try:
                call()
                raise AssertionError(name)
            except LC.LCError as e:
                assert e.code == LC.LC_ERR_HIP, name
            assert len(h.words()) == fail, (name, fail, h.words())
        h.standin_clear()
        h.standin_stale_error()  # a call of the program that failed before
        call()
        assert len(h.words()) == len(kernels), name


# ---- the tests ---------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("lib", [LIB, GRID_CAPPED_LIB], ids=["built", "grid-capped"])
def test_calls_launch_kernels_and_ask_for_nothing_else(standin, lib):  # noqa: F811
    """No allocation, copy, query or wait: a call may be captured into a graph."""
    in_child(standin, lib, "launches")


def test_a_failed_launch_ends_the_call_and_a_stale_error_does_not(standin):  # noqa: F811
    in_child(standin, LIB, "failures")


def test_checks_of_arguments_under_host_sanitizers():
    rt = sanitizer_runtime()
    if not os.path.exists(SANITIZED_LIB) or not rt:
        pytest.skip("the host-sanitized library is built by __graft_entry__.build()")
    env = dict(os.environ, LD_PRELOAD=rt, LAYERCHECK_LIB=SANITIZED_LIB,
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "-m", "not gpu",
                        "tests/test_more_operators_abi.py"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    tail = (r.stdout + r.stderr)[-4000:]
    assert r.returncode == 0, tail
    assert "ERROR: AddressSanitizer" not in tail and "runtime error:" not in tail, tail


def test_loads_to_lds_have_their_offset_where_bounds_are_checked():
    """As test_buffer_bounds.py, of the loads whose scalar offset is the fifth argument."""
    from tests.test_buffer_bounds import CSRC, arguments
    found = 0
    for path in sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".hip", ".h"))):
        text = open(path).read()
        assert text.count("buffer_load_lds") == text.count("#define LC_BUFFER_LOAD_LDS __builtin_amdgcn_raw_ptr_buffer_load_lds"), path
        for at in (i + len("LC_BUFFER_LOAD_LDS(") for i in range(len(text)) if text.startswith("LC_BUFFER_LOAD_LDS(", i)):
            args = arguments(text, at)
            assert len(args) == 7 and args[4:6] == ["0", "0"], (os.path.basename(path), args)
            found += 1
    assert found == 1


def test_workspace_of_any_shape():
    """Holds X twice and A twice in 16 bits, or in two planes of them, both sides padded to 64, for the matrices at once; a matrix needs the same
    turned; more of them never need less, nor two planes less than one."""
    from paper_2609_27193_amd import layercheck as LC
    pad = lambda n: -(-n // 64) * 64  # noqa: E731
    for rows, cols in [(1, 1), (1, 65536), (65536, 1), (63, 65), (1000, 1000), (4096, 14336), (65536, 65536)]:
        m, n = pad(min(rows, cols)), pad(max(rows, cols))
        last = 0
        for count in (1, 2, 3, 17, 64):
            one, two = (LC.lc_orthogonalize_workspace(count, rows, cols, dt) for dt in (LC.LC_DT_BF16, LC.LC_DT_F32))
            assert one == LC.lc_orthogonalize_workspace(count, cols, rows, LC.LC_DT_BF16)
            at_once = min(count, max(1, 1024 // math.ceil(m / 256) ** 2))
            planes = 2 if min(rows, cols) < 384 else 1
            assert one >= at_once * planes * (4 * m * n + 4 * m * m) and two >= at_once * (8 * m * n + 8 * m * m)
            assert one >= last
            last = one
