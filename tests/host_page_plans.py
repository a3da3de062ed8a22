"""Run as a program under tests/hip_host.cpp's stand-in for the HIP runtime, like
host_pages.py: what becomes of a step's plan when its sequences get other pages, as JSON."""
import ctypes
import json
import sys

import numpy as np

from host_stage import quant
from host_pages import H, PAGE, Pool, _lib, array, fork, host, length, lib, pages, plan, request, use


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


def copied():
    """A shared last page is replaced by a copy before rows are added to it."""
    def shared(add, cut):
        def change(p, q):
            rc, (kid,) = fork([q], 1, [64])                      # four whole pages, of which q's rows up to `cut` stay
            assert rc == 0 and lib.kv_seq_truncate(q, cut) == 0
            assert add(p, q) == 0
            assert cut == 64 or pages(kid)[cut // PAGE] != pages(q)[cut // PAGE]
            return lib.kv_seq_free(kid)
        return change

    def load(p, q):
        state = ctypes.c_void_p()
        assert lib.kv_state_alloc(p.st, 1, 64, ctypes.byref(state)) == 0
        rows = array(np.zeros((1, 2, 8, 64), np.uint16))
        assert lib.kv_append(state, rows, rows, 8, 0, None) == 0
        rc = lib.kv_seq_load(q, state, 0, 1, 3, None)
        assert lib.kv_state_free(state) == 0
        return rc

    def forward(p, q, fail=False):
        x, y, pos = (array(np.zeros((64, H), np.uint16)), array(np.zeros((64, H), np.uint16)), array(np.zeros(64, np.int32)))
        reqs = (_lib.KVStepRequest * 1)(request(q, 2, pos))
        n = len(pages(q))
        last, rows = pages(q)[-1], length(q)
        if fail:                                                 # behind the plan and its copy
            host.host_start(4, 0, 0)
        rc = lib.stage_forward_paged(p.st, reqs, 1, x, y, None)
        host.host_start(0, 0, 0)
        if fail:
            assert rc == -5 and length(q) == rows and len(pages(q)) == n and pages(q)[-1] != last
        return 0 if fail else rc

    ways = {
        "append": lambda p, q: lib.kv_seq_append(q, p.rows, p.rows, 2, None),
        "load": load,
        "another step's plan": lambda p, q: plan(p.step(), [request(q, 2)]),
        "forward": forward,
        "a forward that fails": lambda p, q: forward(p, q, True),
    }
    out = {f"{name}, in its last page": _after(shared(f, 45)) for name, f in ways.items()}
    out.update({f"{name}, in the next page": _after(shared(f, 50)) for name, f in ways.items()})
    out["append, nothing shared"] = _after(shared(ways["append"], 64))
    return out


def shared():
    """What a step answers (write, attend) while a fork shares a page of its new rows, and once it does no more."""
    out = {}
    for name, rows in (("a page before them", 32), ("a page of them", 48), ("all", 64)):
        p = Pool()
        q, step = p.seq(40), p.step()
        assert plan(step, [request(q, 24)]) == 0
        rc, (kid,) = fork([q], 1, [rows])
        assert rc == 0
        got = [*use(step, p)]
        assert lib.kv_seq_free(kid) == 0
        out[name] = [*got, *use(step, p)]
    return out


def long_prompt(rows):
    """Statuses of a plan of 8192 rows of 64 heads on one kv head behind `rows` keys, and the bytes of its workspace by row and head."""
    n, D = 8192, 64
    dims = {"wq": (64 * D, H), "wk": (D, H), "wv": (D, H), "wo": (H, 64 * D), "wg": (688, H), "wu": (688, H), "wd": (H, 688)}
    layer = _lib.LayerWeights(attn_norm=array(np.zeros(H, np.uint16)), ffn_norm=array(np.zeros(H, np.uint16)),
                              **{name: quant(*d) for name, d in dims.items()})
    cfg = _lib.StageConfig(n_layers=1, hidden=H, n_q_heads=64, n_kv_heads=1, head_dim=D, ffn=688, group_size=128, rms_eps=1e-5,
                           act_dtype=_lib.DTYPE_BF16, kv_dtype=_lib.DTYPE_BF16, rope_theta=10000.0, max_positions=64, rope_cos_sin=None)
    st, pool, q, step = (ctypes.c_void_p() for _ in range(4))
    assert lib.stage_create(ctypes.byref(cfg), ctypes.byref(layer), 0, None, ctypes.byref(st)) == 0, lib.stage_last_error()
    count = (int(rows) + n) // 256 + 2
    k, v, x = (array(np.zeros(count * 256 * D + 8, np.uint16)) // 16 * 16 + 16 for _ in range(3))
    assert lib.kv_pages_create(st, count, 256, k, v, None, 1, ctypes.byref(pool)) == 0
    assert lib.kv_seq_create(pool, ctypes.byref(q)) == 0 and lib.kv_step_create(pool, ctypes.byref(step)) == 0
    assert lib.kv_seq_append(q, x, x, int(rows), None) == 0, lib.stage_last_error()
    got = plan(step, [request(q, n)])
    size = ctypes.c_int64()
    return [got, lib.kv_step_workspace(step, ctypes.byref(size)), size.value / (n * 64)]


def freed_steps():
    """Frees of steps and sequences: whether one waited for the device; device allocations of 20 steps made, planned and freed one
    after the other beyond the first's; what a new one answers before it has a plan, and after."""
    host.host_syncs.restype = ctypes.c_long
    p = Pool()
    q = p.seq(40)

    def one():
        step = p.step()
        none = [*use(step, p), plan(step, [request(q, 1)]), *use(step, p)]
        before = host.host_syncs()
        assert lib.kv_step_free(step) == 0
        return none, host.host_syncs() - before

    first = one()
    live = host.host_live()
    rest = [one() for _ in range(20)]
    live = host.host_live() - live
    two = p.step(), p.step()                                     # at the same time: each its own
    assert plan(two[0], [request(q, 1)]) == 0
    both = [*use(two[0], p), *use(two[1], p)]
    # a step that a graph holds is not another's
    host.host_start(0, 0, 1)
    held = use(two[0], p)
    host.host_start(0, 0, 0)
    assert lib.kv_step_free(two[0]) == 0
    third = p.step()
    again = third.value == two[0].value
    before = host.host_syncs()
    assert lib.kv_seq_free(q) == 0
    waits = host.host_syncs() - before
    assert lib.kv_pages_free(p.h) == 0
    return dict(answers=[first[0], *[r[0] for r in rest]], waits=[first[1], waits, *[r[1] for r in rest]], live=live, both=both, held=held,
                again=again)


if __name__ == "__main__":
    print(json.dumps(globals()[sys.argv[1]](*sys.argv[2:])))
