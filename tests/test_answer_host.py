"""The host code of the last stage's operators around calls that fail, with a
stand-in for the HIP runtime (hip_host.cpp) and no GPU."""
import json
import os
import subprocess
import sys

import pytest

from paper_2608_19147_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask(question, *arguments): what host_stage.py answers."""
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2608_19147_amd import build

        build.build()
    so = str(tmp_path_factory.mktemp("host") / "hip_host.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", os.path.join(HERE, "hip_host.cpp"), "-o", so], check=True)

    def run(*args):
        env = {**os.environ, "LD_PRELOAD": so, "STAGE_PERSISTENT": "0", "OPENBLAS_NUM_THREADS": "1"}
        r = subprocess.run([sys.executable, os.path.join(HERE, "host_stage.py"), *args], env=env, capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        return json.loads(r.stdout)

    return run


CALLS = ["product", "product_passes", "product_one_pass", "sample", "top1_mx4", "sample_mx4", "sample_int4"]


@pytest.mark.parametrize("name", CALLS)
def test_nothing_behind_a_failed_launch(ask, name):
    """The launch that fails is a call's last one: what would come next reads what it did not write."""
    seen = ask("order", name)
    assert seen
    for q in seen:
        assert q["queued"] == q["at"] - 1, q


@pytest.mark.parametrize("name", CALLS)
def test_order_behind_a_failed_call(ask, name):
    """A call whose second or later launch fails has queued work that uses the stage's workspace: the next call, on another
    stream, waits for it."""
    seen = ask("order", name)
    assert seen
    for q in seen:
        assert q["rc"] == -5 and q["rc2"] == 0 and q["ordered"], q


@pytest.mark.parametrize("name", CALLS + ["top1_int4"])
@pytest.mark.parametrize("capture", [0, 1])
def test_no_host_memory(ask, name, capture):
    """A host allocation that fails is STAGE_E_OOM, and no exception leaves the call; the last status is that of the call
    with memory."""
    got = ask("allocations", name, str(capture))
    assert got[:-1] == [-4] * (len(got) - 1)
    assert got[-1] == (-7 if capture and name != "top1_int4" else 0)


@pytest.mark.parametrize("name", ["top1_mx4", "sample_mx4", "sample_int4"])
def test_logits_workspace(ask, name):
    """Logits rows are allocated for calls that give none, and only for those."""
    most, logits = ask("largest_allocation", name)
    assert most == logits
    most, logits = ask("largest_allocation", name + "_logits")
    assert most < logits


@pytest.mark.parametrize("name", ["head", "matrix"])
def test_weights_without_memory(ask, name):
    """MXFP4 weights that do not fit leave nothing allocated and no error behind, and the call can be made again."""
    got = ask("weights_without_memory", name)
    assert len(got) >= 5 and got[-1][0] == 0
    assert [tuple(g) for g in got[:-1]] == [(-4, 0, 0)] * (len(got) - 1)
