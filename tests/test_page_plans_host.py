"""Plans of the paged cache whose sequences get other pages, on the stand-in for the
HIP runtime (hip_host.cpp): a step answers as long as its pages are its sequences'."""
import json
import os
import subprocess
import sys

import pytest

from paper_2608_19147_amd import _lib

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """ask(question, *arguments): what host_page_plans.py answers."""
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2608_19147_amd import build

        build.build()
    so = str(tmp_path_factory.mktemp("host") / "hip_host.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", os.path.join(HERE, "hip_host.cpp"), "-o", so], check=True)

    def run(*args):
        env = {**os.environ, "LD_PRELOAD": so, "STAGE_PERSISTENT": "0", "OPENBLAS_NUM_THREADS": "1"}
        r = subprocess.run([sys.executable, os.path.join(HERE, "host_page_plans.py"), *args], env=env, capture_output=True, text=True,
                           timeout=120)
        assert r.returncode == 0, r.stderr
        return json.loads(r.stdout)

    return run


def _check(got, replaced):
    """[same pages, write, attend] of each case: those named had a page of the plan replaced, and its step has no plan."""
    for name, (same, write, attend) in got.items():
        assert same == (name not in replaced), name
        assert [write, attend] == ([0, 0] if same else [-1, -1]), name


def test_compaction(ask):
    """The old pages of a compaction may be another sequence's next: a plan with rows in one of them is withdrawn."""
    _check(ask("compacted"), {"in its last page, into new pages", "in its last page, in place of a shared one"})


def test_copies(ask):
    """So is one with rows in a shared last page that is replaced by a copy."""
    got = ask("copied")
    _check(got, {name for name in got if "last page" in name})


def test_shared_rows(ask):
    """Nothing writes into a page while it is shared: the rows of a fork stay as they were when it was made."""
    got = ask("shared")
    assert got == {"a page before them": [0, 0, 0, 0], "a page of them": [-1, 0, 0, 0], "all": [-1, 0, 0, 0]}


@pytest.mark.parametrize("rows", [1 << 20, 1 << 21])
def test_longest_prompts(ask, rows):
    """Costs of splits are computed wide enough for the most rows behind millions of keys (4096 splits of 2^19 query vectors pass 2^31).
    A split's partial results cost a 16th of a step a query vector, over 512 places; S splits save at most half of the longest one's
    steps, as the last ones leave places empty: S 2^19 / (16 512) <= steps / 2.  A partial result is 64 + 2 floats."""
    plan, size, each = ask("long_prompt", str(rows))
    steps = (rows + 8192) // 32
    assert [plan, size] == [0, 0] and each / (4 * 66) <= steps / 128


def test_freed_steps(ask):
    """A step's end waits for nothing (a collected one would end a capture that is under way): the pool keeps its memory for the next."""
    got = ask("freed_steps")
    assert all(a == [-1, -1, 0, 0, 0] for a in got["answers"])
    assert got["waits"] == [0] * 22 and got["live"] == 0
    assert got["both"] == [0, 0, -1, -1] and got["held"] == [0, 0] and not got["again"]
