"""Replays the GPU tests of the expert rows and of the MXFP4 products of a few rows on the CPU execution model, as
tests/test_host_model_replay.py does for the other operators."""
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
MODEL_DIR = os.path.join(HERE, "host_model")
LIB = os.path.join(MODEL_DIR, "_build", "libmxfp8_hostmodel.so")


@pytest.fixture(scope="module")
def hostmodel_lib(request):
    proc = getattr(request.config, "_hostmodel_shared_build", None)   # started by conftest.py when collection ended
    if proc is None:
        res = subprocess.run([os.path.join(MODEL_DIR, "build.sh"), "--shared", LIB], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-4000:]
    else:
        if proc.returncode is None:
            proc.communicate()
        assert proc.returncode == 0
    return LIB


@pytest.mark.parametrize("file,at_least", [("test_gpu_experts.py", 90), ("test_gpu_fp4_gemv.py", 70)])
def test_gpu_tests_pass_on_the_host_model(hostmodel_lib, file, at_least):
    env = dict(os.environ, MXFP8_HOSTMODEL_LIB=hostmodel_lib, PYTHONPATH=os.pathsep.join([MODEL_DIR, ROOT, os.environ.get("PYTHONPATH", "")]))
    for var in ("OMP_NUM_THREADS", "OPENBLAS_NUM_THREADS", "MKL_NUM_THREADS"):
        env[var] = "2"
    res = subprocess.run([sys.executable, "-m", "pytest", "-p", "no:cacheprovider", "-p", "replay_plugin", "-q", "-x", "-m", "gpu", "-k", "not full_size",
                          os.path.join(HERE, file)], capture_output=True, text=True, cwd=ROOT, env=env, timeout=2400)
    out = res.stdout + res.stderr
    assert res.returncode == 0, out[-3000:]
    m = re.search(r"(\d+) passed", out)
    assert m and int(m.group(1)) >= at_least, out[-3000:]
