"""Which kernels the weight gradient's cut sends the GPU tests' sizes to (CPU): a change of its estimate must not take them
off the paths that they are there for."""
import os
import subprocess
import sys

from paper_2609_27193_amd.build_lib import LIB
from tests.test_host_calls import DEVICE, ROOT, hip, standin  # noqa: F401 (a fixture)
from tests.wgrad_cases import ALIGNED, RAGGED, SMALL


def routes():
    from paper_2609_27193_amd import layercheck as LC
    h = hip()
    at = h.standin_alloc(1 << 20, DEVICE)
    a = [at + (i + 1 << 38) for i in range(6)]  # never read
    for dtype, (rows, n, k), kernels in [(LC.LC_DT_BF16, *c) for c in ALIGNED + RAGGED + SMALL] + [(LC.LC_DT_F32, *c) for c in SMALL]:
        h.standin_clear()
        LC.lc_linear_wgrad(LC.matrix(a[0], rows, n, dtype), LC.saved_act(a[1], a[2], rows, k),
                           LC.matrix(a[3], n, k, LC.LC_DT_F32), a[4], LC.lc_linear_wgrad_workspace(rows, n, k))
        got = h.words()
        assert len(got) == len(kernels) and all(w in g for w, g in zip(kernels, got)), ((rows, n, k), got)


def test_sizes_take_the_kernels_that_they_test(standin):  # noqa: F811
    env = dict(os.environ, LD_PRELOAD=standin, HIP_STANDIN=standin, LAYERCHECK_LIB=LIB)
    r = subprocess.run([sys.executable, "-c", "import tests.test_wgrad_routes as t; t.routes()"], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
