"""What the training operators' host code asks of HIP (CPU): launches alone, which ones, and what an error does.  A child
process makes the calls on the preloaded stand-in for the HIP host calls, which runs no kernel and writes the calls down."""
import os
import subprocess
import sys

import pytest

from paper_2609_27193_amd.build_lib import GRID_CAPPED_LIB, LIB
from tests.test_host_calls import DEVICE, ROOT, hip, standin  # noqa: F401 (a fixture)


def in_child(standin, lib, scenario):  # noqa: F811
    env = dict(os.environ, LD_PRELOAD=standin, HIP_STANDIN=standin, LAYERCHECK_LIB=lib)
    r = subprocess.run([sys.executable, "-c", f"import tests.test_operators_host as t; t.{scenario}()"], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]


# ---- in the child ----------------------------------------------------------------------------------------------------------


def calls(h):
    """(name, call, the kernels that it launches in order)."""
    from paper_2609_27193_amd import layercheck as LC
    B, F = LC.LC_DT_BF16, LC.LC_DT_F32
    at = h.standin_alloc(1 << 20, DEVICE)
    apart = iter(range(1 << 30, 1 << 45, 1 << 28))  # never read: any addresses that lie apart
    M = lambda rows, cols, dt=B: LC.matrix(at + next(apart), rows, cols, dt)  # noqa: E731
    K = lambda rows, cols: LC.saved_act(at + next(apart), at + next(apart), rows, cols)  # noqa: E731
    V = lambda: at + next(apart)  # noqa: E731
    out = [("embedding", lambda: LC.lc_embedding_forward(M(99, 64), V(), 2, 7, M(7, 64)), ["embed_fwd"])]
    for n, vocab, kernels in [(7, 99, ["direct"]), (2048, 99, ["direct"]), (2049, 99, ["rank", "sum", "join"]),
                              (4096, 99, ["rank", "sum", "join"]), (4097, 99, ["block_sort", "sum", "join"]), (8192, 1 << 18, ["block_sort", "sum", "join"]),
                              (16384, 1 << 20, ["block_sort", "sum", "join"]), (16385, 1 << 20, ["count", "scatter"] * 3 + ["sum", "join"]),
                              (8193, 512, ["count", "scatter"] * 2 + ["sum", "join"]),
                              (8193, 511, ["count", "scatter", "sum", "join"]),
                              (8193, 1 << 18, ["count", "scatter"] * 3 + ["sum", "join"])]:
        def go(n=n, vocab=vocab):
            need = LC.lc_embedding_backward_workspace(n, 64)
            LC.lc_embedding_backward(M(n, 64), V(), 2, n, M(vocab, 64), V(), need)
        out.append((f"embedding gradient {n} {vocab}", go, kernels))
    norm = LC.norm_params(LC.LC_NORM_LAYER, V(), V(), F, 1e-5)
    for dim, kind in [(7, "long"), (8, "fwd_k"), (16384, "fwd_k"), (16385, "long")]:
        out.append((f"norm {dim}", lambda dim=dim: LC.lc_norm_forward(norm, M(5, dim), M(5, dim), saved=K(5, dim)), [kind]))
        bwd = "bwd_long" if kind == "long" else "bwd_k"
        def back(dim=dim, dx=True, dw=True):
            need = LC.lc_norm_backward_workspace(5, dim)
            LC.lc_norm_backward(norm, M(5, dim), V(), M(5, dim) if dx else None, V() if dw else 0, 0, F, V(), need, saved=K(5, dim))
        out.append((f"norm gradient {dim}", back, [bwd, "join"]))
        out.append((f"dx {dim}", lambda back=back: back(dw=False), [bwd]))
        out.append((f"dw {dim}", lambda back=back: back(dx=False), [bwd, "join"]))
    out.append(("save", lambda: LC.lc_act_save(M(5, 40), K(5, 40)), ["save"]))
    out.append(("load", lambda: LC.lc_act_load(K(5, 40), M(5, 40)), ["load"]))
    for rows, n, k, dt, bias, kernels in [(4096, 4096, 4096, B, False, ["big"]), (8192, 1024, 4096, B, False, ["big", "join"]),
                                          (4096, 4096, 4096, B, True, ["sums_k", "sums_join", "big"]),
                                          (4096, 4095, 4097, B, False, ["big", "join"]), (64, 100, 256, B, True, ["wgrad_kernel"]),
                                          (64, 256, 256, F, False, ["wgrad_kernel"]),
                                          (4096, 256, 256, F, True, ["wgrad_kernel", "join"])]:
        def go(rows=rows, n=n, k=k, dt=dt, bias=bias):
            need = LC.lc_linear_wgrad_workspace(rows, n, k)
            LC.lc_linear_wgrad(M(rows, n, dt), K(rows, k), M(n, k, dt), V(), need, dbias=V() if bias else 0)
        out.append((f"wgrad {rows} {n} {k}", go, kernels))
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
