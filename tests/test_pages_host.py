"""The paged cache's host code with a stand-in for the HIP runtime (hip_host.cpp):
refusals, calls whose launches or allocations fail, captures."""
import json
import os
import subprocess
import sys

import pytest

from paper_2608_19147_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask(question, *arguments): what host_pages.py answers."""
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2608_19147_amd import build

        build.build()
    so = str(tmp_path_factory.mktemp("host") / "hip_host.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", os.path.join(HERE, "hip_host.cpp"), "-o", so], check=True)

    def run(*args):
        env = {**os.environ, "LD_PRELOAD": so, "STAGE_PERSISTENT": "0", "OPENBLAS_NUM_THREADS": "1"}
        r = subprocess.run([sys.executable, os.path.join(HERE, "host_pages.py"), *args], env=env, capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        return json.loads(r.stdout)

    return run


CALLS = ["fork", "fork_keep", "append", "compact", "read", "plan", "forward"]


def test_refusals(ask):
    for i, (want, got, same) in enumerate(ask("refusals")):
        assert got == want and same, i


@pytest.mark.parametrize("name", CALLS)
def test_failed_launch(ask, name):
    """A launch that fails ends the call with STAGE_E_HIP, leaves the sequences and the free pages as they were, and the next call
    on another stream waits behind what had been queued."""
    seen = ask("failing", name, "launch")
    assert seen
    for q in seen:
        assert q["rc"] == -5 and q["rc2"] == 0 and q["ordered"] and q["queued"] == q["at"] - 1, q
        assert q["same"] or name == "forward", q                 # (a forward may have replaced a shared last page by its copy)


@pytest.mark.parametrize("name", CALLS)
def test_no_host_memory(ask, name):
    """A host allocation that fails is STAGE_E_OOM, no exception leaves the call, and nothing has changed."""
    seen = ask("failing", name, "memory")
    assert seen
    for q in seen:
        assert q["rc"] == -4 and q["rc2"] == 0 and (q["same"] or name == "forward"), q


def test_no_device_memory(ask):
    plan, again, pool = ask("device_memory")
    assert plan == [-4, True] and again[0] == 0 and pool == [-4, True]


def test_capture(ask):
    for name, (rc, same, launches) in ask("captured_status").items():
        assert rc == -7 and same and launches == 0, name


def test_workspace(ask):
    assert ask("workspace") == [True, -1, -1, -1, 0]


def test_lost_rows(ask):
    """A step whose sequences have lost rows that it covers has no plan: its rows may be another sequence's by then."""
    kept = {"nothing", "a fork", "a fork cut", "rows behind it", "another step", "no row dropped", "planned again"}
    for name, write, attend in ask("lost_rows"):
        assert [write, attend] == ([0, 0] if name in kept else [-1, -1]), name


def test_overlapping_outputs(ask):
    got = ask("overlaps")
    assert got["allowed"] == [0] * 6 and got["refused"] == [-1] * 9, got
