"""The calls for sequences that share blocks in the checked build of the library, whose copies are held against the extent of the pools
and whose waits can be told to give up after a few polls."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(*args):
    import paper_2509_19729_b200.build as b

    b.build(checked=True)
    env = dict(os.environ, AMOEBA_BINDING_BUILD="checked", PYTHONPATH=os.pathsep.join([ROOT, os.path.join(ROOT, "tests")]))
    r = subprocess.run([sys.executable, *args], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    return r.stdout


def test_waits_that_run_out():
    assert "gave up and came back" in run(os.path.join(ROOT, "tests", "give_up_sharing_check.py"))


def test_copies_stay_inside_their_pools():
    assert " passed" in run("-m", "pytest", "tests/test_gpu_sharing.py", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider", "-k", "copies")
