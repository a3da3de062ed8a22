"""Run as a program under tests/hip_host.cpp's stand-in for the HIP runtime, like
host_pages.py: what becomes of a step's plan when its sequences get other pages, as JSON."""
import json
import sys

import numpy as np

from host_pages import PAGE, Pool, array, fork, lib, pages, plan, request, use


def _drop(n, *rows):
    return array((~np.isin(np.arange(n), rows)).astype(np.uint8))


def _fill(p, left):
    """Takes pages until `left` are free."""
    while p.free() > left:
        p.seq(1)


def _after(change, n_pages=40):
    """A plan of 5 rows behind 40 of a sequence, and `change`: the pages of its 45 rows before and after, and what the step
    answers then (write, attend)."""
    p = Pool(n_pages)
    q, step = p.seq(40), p.step()
    assert plan(step, [request(q, 5)]) == 0
    assert lib.kv_seq_append(q, p.rows, p.rows, 25, None) == 0   # 70 rows, 5 pages
    covered = lambda: pages(q)[: -(-45 // PAGE)]
    before = covered()
    assert change(p, q) == 0
    got = [before == covered(), *use(step, p)]
    assert lib.kv_step_free(step) == 0 and lib.kv_pages_free(p.h) == 0
    return got


def compacted():
    def in_place(p, q):
        _fill(p, 1)
        return lib.kv_seq_compact(q, _drop(70, 46), None)

    def in_place_shared(p, q):
        assert fork([q], 1, [48])[0] == 0
        return in_place(p, q)

    return {
        "in its last page, into new pages": _after(lambda p, q: lib.kv_seq_compact(q, _drop(70, 46), None)),
        "in its last page, its tail alone": _after(lambda p, q: lib.kv_seq_compact(q, _drop(70, *range(46, 70)), None)),
        "in its last page, in place": _after(in_place),
        "in its last page, in place of a shared one": _after(in_place_shared),
        "behind its pages": _after(lambda p, q: lib.kv_seq_compact(q, _drop(70, 48), None)),
    }


if __name__ == "__main__":
    print(json.dumps(globals()[sys.argv[1]](*sys.argv[2:])))
