"""The tests of the paged attention's number formats once more on forms that a call can take (the switch is read once, so each form runs in a process of its own)."""
import os
import subprocess
import sys

import pytest

import paper_2608_03537_b200 as cf

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(cluster, **more):
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_gpu_kv_extremes.py"), "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider"], cwd=ROOT,
                       env=dict(os.environ, COMFUSE_ATTENTION_CLUSTER=str(cluster), PYTHONPATH=ROOT, **more), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:]


@pytest.mark.parametrize("cluster", [0, 1, 4, 16])
def test_form(cluster, cuda_device):
    _run(cluster)


def test_checked_build(cuda_device):
    _run(0, COMFUSE_LIB=os.path.join(os.path.dirname(cf.__file__), "libcomfuse_checked.so"))
