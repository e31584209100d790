"""Every test of the paged attention once more on each form that a call can take: equal shares and a second kernel, and clusters of each size (the switch is read once, so each form runs in a
process of its own)."""
import os
import subprocess
import sys

import pytest

import paper_2608_03537_b200 as cf

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(cluster, **more):
    env = dict(os.environ, COMFUSE_ATTENTION_CLUSTER=str(cluster), PYTHONPATH=ROOT, **more)
    # (the refusals ask for a workspace, which clusters do without)
    pick = ["-k", "not refusals"] if cluster else []
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_gpu_paged_attention.py"), "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", *pick], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:]


@pytest.mark.parametrize("cluster", [0, 1, 2, 4, 8, 16])
def test_form(cluster, cuda_device):
    _run(cluster)


@pytest.mark.parametrize("cluster", [0, 4])
def test_checked_build(cluster, cuda_device):
    """The bounds predicates hold on every call of the tests (each ends with a clear device status)."""
    _run(cluster, COMFUSE_LIB=os.path.join(os.path.dirname(cf.__file__), "libcomfuse_checked.so"))
