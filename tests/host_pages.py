"""Run as a program under tests/hip_host.cpp's stand-in for the HIP runtime, like
host_stage.py: answers one question about the host code of the paged cache, as JSON."""
import ctypes
import json
import sys

import numpy as np

from host_stage import H, KEEP, _lib, array, host, lib, make_stage, notes

PAGE = 16


class Pool:
    """A pool of a one-layer stage (2 kv heads of 64) with its sequences and steps."""

    def __init__(self, n_pages=40, axes=1, pair_axis=None):
        self.st = make_stage()
        self.k, self.v = (array(np.zeros(n_pages * 2 * PAGE * 64 + 8, np.uint16)) // 16 * 16 + 16 for _ in range(2))
        self.h = ctypes.c_void_p()
        rc = lib.kv_pages_create(self.st, n_pages, PAGE, self.k, self.v, pair_axis, axes, ctypes.byref(self.h))
        assert rc == 0, lib.stage_last_error()
        self.rows = array(np.zeros(1 << 20, np.uint16)) // 16 * 16 + 16

    def seq(self, n=0):
        q = ctypes.c_void_p()
        assert lib.kv_seq_create(self.h, ctypes.byref(q)) == 0
        if n:
            assert lib.kv_seq_append(q, self.rows, self.rows, n, None) == 0, lib.stage_last_error()
        return q

    def step(self):
        s = ctypes.c_void_p()
        assert lib.kv_step_create(self.h, ctypes.byref(s)) == 0
        return s

    def free(self):
        n = ctypes.c_int()
        assert lib.kv_pages_available(self.h, ctypes.byref(n)) == 0
        return n.value


def length(q):
    n = ctypes.c_int()
    assert lib.kv_seq_length(q, ctypes.byref(n)) == 0
    return n.value


def pages(q):
    n = ctypes.c_int()
    out = (ctypes.c_int32 * 4096)()
    assert lib.kv_seq_pages(q, out, 4096, ctypes.byref(n)) == 0
    return list(out[: n.value])


def fork(q, n, lengths=None, keep=None, stream=None):
    hs = (ctypes.c_void_p * n)(*[x.value for x in q])
    out = (ctypes.c_void_p * n)()
    lens = None if lengths is None else (ctypes.c_int32 * n)(*lengths)
    kp = None if keep is None else (ctypes.c_void_p * n)(*[None if k is None else array(k) for k in keep])
    rc = lib.kv_seq_fork(hs, lens, kp, n, out, stream)
    return rc, [ctypes.c_void_p(h) for h in out]


def request(q, n, positions=None, mask=None, mask_rows=None):
    return _lib.KVStepRequest(seq=q, n_tokens=n, positions=positions, attention_mask=mask, attention_mask_rows=mask_rows)


def plan(step, reqs, stream=None):
    return lib.kv_step_plan(step, (_lib.KVStepRequest * len(reqs))(*reqs), len(reqs), stream)


def calls(p):
    """Each call of the paged cache that does device work, with one sequence of 40 rows whose last page is shared, as functions
    of the stream; and what must not have changed where they fail."""
    q = p.seq(40)
    rc, (kid,) = fork([q], 1)
    assert rc == 0
    assert lib.kv_seq_truncate(kid, 20) == 0                     # its last page is q's too
    step = p.step()
    state = lambda: (p.free(), length(q), pages(q), length(kid), pages(kid))
    keep = array((np.arange(40) % 3 != 1).astype(np.uint8))
    kept = array((np.arange(20) % 3 != 1).astype(np.uint8))
    pos = array(np.zeros(64, np.int32))
    hid = array(np.zeros((64, H), np.uint16)), array(np.zeros((64, H), np.uint16))
    many = (_lib.KVStepRequest * 2)(request(kid, 3, pos), request(q, 5, pos))
    table = {
        "fork": lambda s: lib.kv_seq_fork((ctypes.c_void_p * 2)(q, q), (ctypes.c_int32 * 2)(37, 3), None, 2, (ctypes.c_void_p * 2)(), s),
        "fork_keep": lambda s: lib.kv_seq_fork((ctypes.c_void_p * 1)(q), None, (ctypes.c_void_p * 1)(keep), 1, (ctypes.c_void_p * 1)(), s),
        "append": lambda s: lib.kv_seq_append(kid, p.rows, p.rows, 30, s),
        "compact": lambda s: lib.kv_seq_compact(kid, kept, s),
        "read": lambda s: lib.kv_seq_read(q, 0, 3, 30, p.rows, p.rows, s),
        "plan": lambda s: lib.kv_step_plan(step, many, 2, s),
        "forward": lambda s: lib.stage_forward_paged(p.st, many, 2, hid[0], hid[1], s),
    }
    return table, state


def failing(name, kind):
    """Per launch (kind 'launch') or host allocation ('memory') that fails: the status, whether anything changed, and for
    launches whether the next call on another stream waits behind what was queued."""
    out = []
    for at in range(1, 80):
        p = Pool()
        table, state = calls(p)
        before = state()
        host.host_start(at if kind == "launch" else 0, at if kind == "memory" else 0, 0)
        rc = table[name](1)
        got = notes()
        host.host_start(0, 0, 0)
        if rc == 0:
            break
        same = state() == before
        rc2 = lib.kv_seq_append(p.seq(), p.rows, p.rows, 1, 2)
        after = notes()
        launched = [i for i, n in enumerate(got) if n[0] == "L"]
        first = [n[0] for n in after].index("L")
        waits = [n[2] for n in after[:first] if n[0] == "W" and n[1] == "2"]
        behind = [n[2] for n in got[launched[-1] + 1:] if n[0] == "R"] if launched else []
        out.append(dict(at=at, rc=rc, same=same, rc2=rc2, queued=len(launched), ordered=not launched or any(b in waits for b in behind)))
    return out


def captured_status():
    out = {}
    for name in ("fork", "fork_keep", "append", "compact", "read", "plan", "forward"):
        p = Pool()
        table, state = calls(p)
        before = state()
        host.host_start(0, 0, 1)
        out[name] = [table[name](1), state() == before, len([n for n in notes() if n[0] == "L"])]
        host.host_start(0, 0, 0)
    return out


def device_memory():
    """A plan whose metadata finds no device or pinned memory, and a pool whose axis table does."""
    out = []
    p = Pool()
    table, state = calls(p)
    before = state()
    host.host_fail_malloc(1)
    out.append([table["plan"](1), state() == before])
    host.host_fail_malloc(0)
    out.append([table["plan"](1), state() == before])
    h = ctypes.c_void_p()
    live = host.host_live()
    host.host_fail_malloc(1)
    rc = lib.kv_pages_create(p.st, 4, PAGE, p.k, p.v, array(np.zeros(32, np.uint8)), 1, ctypes.byref(h))
    host.host_fail_malloc(0)
    out.append([rc, host.host_live() == live and not h.value])
    return out


def refusals():
    """Statuses of calls that must be refused, and whether they left everything as it was."""
    p, other = Pool(), Pool()
    q, r = p.seq(20), other.seq(20)
    big = p.seq()
    step, empty = p.step(), p.step()
    pos = array(np.zeros(64, np.int32))
    far, neg = array(np.full(64, 64, np.int32)), array(np.full(64, -1, np.int32))
    out = (ctypes.c_void_p * 4)()
    x = p.rows
    hid = array(np.zeros((65, H), np.uint16)), array(np.zeros((65, H), np.uint16))
    h = ctypes.c_void_p()
    n32 = ctypes.c_int()
    i64 = ctypes.c_int64()
    assert plan(step, [request(q, 2)]) == 0
    before = lambda: (p.free(), length(q), pages(q), length(big))
    was = before()
    Q, R = 4 * 64, 2 * 64
    got = []

    def create(st=p.st, n=4, rows=16, k=p.k, v=p.v, axis=None, axes=1, to=ctypes.byref(h)):
        return lib.kv_pages_create(st, n, rows, k, v, axis, axes, to)

    def fwd(reqs, st=p.st, a=hid[0], b=hid[1], n=None):
        return lib.stage_forward_paged(st, (_lib.KVStepRequest * len(reqs))(*reqs), len(reqs) if n is None else n, a, b, None)

    def write(s=step, layer=0, a=x, lda=Q, b=x, ldb=R, c=x, ldc=R, dt=2, o=x, ldo=Q, odt=2):
        return lib.kv_step_write(s, layer, a, lda, b, ldb, c, ldc, dt, o, ldo, odt, None)

    def attend(s=step, layer=0, a=x, dt=2, ld=Q, o=x, odt=2, ldo=Q, scale=0.0, ws=None, n=0):
        return lib.kv_step_attend(s, layer, a, dt, ld, o, odt, ldo, scale, ws, n, None)

    arr = lambda *a: (ctypes.c_void_p * len(a))(*[getattr(v, "value", v) for v in a])
    one = array(np.ones(64, np.uint8))
    none = array(np.zeros(64, np.uint8))
    for code, f in [
        (-1, lambda: create(st=None)), (-1, lambda: create(k=None)), (-1, lambda: create(v=None)), (-1, lambda: create(to=None)),
        (-1, lambda: create(k=p.k + 8)), (-7, lambda: create(rows=8)), (-7, lambda: create(rows=48)), (-7, lambda: create(rows=512)),
        (-3, lambda: create(n=0)), (-3, lambda: create(n=1 << 27)), (-3, lambda: create(axes=0)), (-3, lambda: create(axes=5)),
        (-1, lambda: create(axes=2)), (-1, lambda: create(axis=array(np.full(32, 2, np.uint8)), axes=2)),
        (-1, lambda: lib.kv_pages_free(None)), (-1, lambda: lib.kv_pages_available(None, ctypes.byref(n32))),
        (-1, lambda: lib.kv_seq_create(None, ctypes.byref(h))), (-1, lambda: lib.kv_seq_create(p.h, None)), (-1, lambda: lib.kv_seq_free(None)),
        (-1, lambda: lib.kv_seq_length(None, ctypes.byref(n32))), (-1, lambda: lib.kv_seq_pages(q, None, 0, None)),
        (-1, lambda: lib.kv_seq_fork(None, None, None, 1, out, None)), (-1, lambda: lib.kv_seq_fork(arr(q), None, None, 0, out, None)),
        (-1, lambda: lib.kv_seq_fork(arr(q, None), None, None, 2, out, None)), (-6, lambda: lib.kv_seq_fork(arr(q, r), None, None, 2, out, None)),
        (-1, lambda: lib.kv_seq_fork(arr(q), (ctypes.c_int32 * 1)(23), None, 1, out, None)),
        (-1, lambda: lib.kv_seq_fork(arr(q), (ctypes.c_int32 * 1)(-1), None, 1, out, None)),
        (-3, lambda: fork([q] * 39, 39)[0]),
        (-1, lambda: lib.kv_seq_compact(None, one, None)), (-1, lambda: lib.kv_seq_compact(q, None, None)),
        (-1, lambda: lib.kv_seq_truncate(None, 0)), (-1, lambda: lib.kv_seq_truncate(q, 23)), (-1, lambda: lib.kv_seq_truncate(q, -1)),
        (-1, lambda: lib.kv_seq_append(None, x, x, 1, None)), (-1, lambda: lib.kv_seq_append(q, None, x, 1, None)),
        (-1, lambda: lib.kv_seq_append(q, x, x, 0, None)), (-1, lambda: lib.kv_seq_append(q, x + 2, x, 1, None)),
        (-3, lambda: lib.kv_seq_append(q, x, x, 16 * 40, None)), (-3, lambda: lib.kv_seq_append(q, x, x, 2 ** 31 - 1, None)),
        (-1, lambda: lib.kv_seq_load(q, None, 0, 0, 1, None)),
        (-1, lambda: lib.kv_seq_read(None, 0, 0, 1, x, x, None)), (-1, lambda: lib.kv_seq_read(q, 1, 0, 1, x, x, None)),
        (-1, lambda: lib.kv_seq_read(q, 0, 20, 3, x, x, None)), (-1, lambda: lib.kv_seq_read(q, 0, -1, 1, x, x, None)),
        (-1, lambda: lib.kv_seq_read(q, 0, 1, -1, x, x, None)), (-1, lambda: lib.kv_seq_read(q, 0, 2 ** 31 - 1, 1, x, x, None)),
        (-1, lambda: lib.kv_step_create(None, ctypes.byref(h))), (-1, lambda: lib.kv_step_free(None)),
        (-1, lambda: lib.kv_step_plan(None, None, 1, None)), (-1, lambda: plan(step, [])), (-1, lambda: plan(step, [request(None, 1)])),
        (-1, lambda: plan(step, [request(q, 0)])), (-6, lambda: plan(step, [request(r, 1)])), (-6, lambda: plan(step, [request(q, 1), request(q, 1)])),
        (-3, lambda: plan(step, [request(q, 8193)])), (-3, lambda: plan(step, [request(q, 619)])), (-3, lambda: plan(step, [request(q, 1, far)])),
        (-3, lambda: plan(step, [request(q, 1, neg)])), (-1, lambda: plan(step, [request(q, 1, pos), request(big, 1)])),
        (-1, lambda: write(s=None)), (-1, lambda: write(s=empty)), (-1, lambda: write(layer=1)), (-1, lambda: write(layer=-1)),
        (-1, lambda: write(dt=3)), (-1, lambda: write(odt=-1)), (-1, lambda: write(a=None)), (-1, lambda: write(o=None)),
        (-2, lambda: write(lda=Q - 1)), (-2, lambda: write(ldb=R - 1)), (-2, lambda: write(ldc=0)), (-2, lambda: write(ldo=-5)), (-1, lambda: write(odt=0)), (-1, lambda: write(ldo=Q + 1)),
        (-1, lambda: attend(s=None)), (-1, lambda: attend(s=empty)), (-1, lambda: attend(layer=1)), (-1, lambda: attend(dt=1)),
        (-1, lambda: attend(odt=4)), (-1, lambda: attend(scale=-1.0)), (-1, lambda: attend(scale=float("nan"))),
        (-1, lambda: attend(scale=float("inf"))), (-2, lambda: attend(ld=Q - 1)), (-2, lambda: attend(ldo=Q - 1)), (-1, lambda: attend(a=None)),
        (-1, lambda: lib.kv_step_workspace(empty, ctypes.byref(i64))), (-1, lambda: lib.kv_step_workspace(step, None)),
        (-1, lambda: fwd([request(q, 1)])), (-1, lambda: fwd([request(q, 1, pos)], n=0)), (-1, lambda: fwd([request(q, 1, pos)], a=None)),
        (-1, lambda: fwd([request(None, 1, pos)])), (-6, lambda: fwd([request(r, 1, pos)])), (-6, lambda: fwd([request(q, 1, pos), request(r, 1, pos)])),
        (-3, lambda: fwd([request(q, 65, array(np.zeros(65, np.int32)))])), (-1, lambda: fwd([request(q, 1, pos)], b=hid[0])),
        (-1, lambda: fwd([request(q, 1, pos, mask=none)])), (-1, lambda: fwd([request(q, 2, pos, mask_rows=array(np.r_[np.ones(24, np.uint8), np.zeros(24, np.uint8)]))])),
        (-3, lambda: fwd([request(q, 1, far)])),
    ]:
        got.append([code, f(), before() == was])
    return got


def lost_rows():
    """What a step answers once its sequences have lost rows: [case, write's status, attend's]."""
    out = []
    keep = lambda n, drop: array((np.arange(n) != drop).astype(np.uint8))
    other = {}
    for name, change in (
            ("nothing", lambda p, q: 0),
            ("a fork", lambda p, q: fork([q], 1)[0]),
            ("a fork cut", lambda p, q: lib.kv_seq_truncate(fork([q], 1)[1][0], 3)),
            ("rows behind it", lambda p, q: lib.kv_seq_append(q, p.rows, p.rows, 9, None) or lib.kv_seq_truncate(q, 45)),
            ("another step", lambda p, q: plan(other["step"], [request(q, 4)])),
            ("no row dropped", lambda p, q: lib.kv_seq_compact(q, keep(45, -1), None)),
            ("cut", lambda p, q: lib.kv_seq_truncate(q, 44)),
            ("cut and refilled", lambda p, q: lib.kv_seq_truncate(q, 40) or lib.kv_seq_append(q, p.rows, p.rows, 5, None)),
            ("compacted", lambda p, q: lib.kv_seq_compact(q, keep(45, 7), None)),
            ("freed", lambda p, q: lib.kv_seq_free(q))):
        p = Pool()
        q, r, step = p.seq(40), p.seq(3), p.step()
        other["step"] = p.step()
        assert plan(step, [request(q, 5), request(r, 2)]) == 0
        assert change(p, q) == 0, name
        out.append([name, *use(step, p)])
        if name == "cut":                                        # planned again, it has a plan; and the other sequence is free of it
            assert plan(step, [request(r, 2)]) == 0 and lib.kv_seq_free(q) == 0
            out.append(["planned again", *use(step, p)])
        assert lib.kv_step_free(step) == 0 and lib.kv_seq_free(r) == 0 and lib.kv_pages_free(p.h) == 0, name
    return out


def use(step, p, q_out=None, ld=4 * 64):
    big = p.rows
    w = lib.kv_step_write(step, 0, big, ld, big + (1 << 18), 128, big + (1 << 19), 128, 2, q_out or big + (3 << 18), ld, 2, None)
    a = lib.kv_step_attend(step, 0, big, 2, ld, big + (3 << 18), 2, ld, 0.0, big + (1 << 20), 1 << 19, None)
    return w, a


def overlaps():
    """Statuses of writes and attentions whose output shares memory with an input, or lies between its rows."""
    p = Pool()
    step = p.step()
    assert plan(step, [request(p.seq(20), 3)]) == 0
    b, far, ws, W = p.rows, p.rows + (1 << 19), p.rows + (1 << 20), 4 * 64
    write = lambda q, k, v, out, ld=W, ldo=W: lib.kv_step_write(step, 0, q, ld, k, ld, v, ld, 2, out, ldo, 2, None)
    attend = lambda q, out, ld=W, ldo=W: lib.kv_step_attend(step, 0, q, 2, ld, out, 2, ldo, 0.0, ws, 1 << 19, None)
    k, v = far, far + (1 << 16)
    return {
        "allowed": [write(b, k, v, b), write(b, b + 2 * W, b + 2 * W + 256, b, 2 * W, 2 * W), write(b, k, v, b + 2 * W, 2 * W, 2 * W),
                    write(b, k, v, b + 2 * 3 * W), attend(b, b + 2 * 3 * W), attend(b, b + 2 * W, 2 * W, 2 * W)],
        "refused": [write(b, k, v, b + 2), write(b, k, v, k), write(b, k, v, v + 2), write(b, k, v, b + 2 * W, 2 * W, 3 * W),
                    attend(b, b), attend(b, b + 2), attend(b, b + 2 * W), attend(b, b - 2, 2 * W, 2 * W), attend(b, b + 2 * W, 2 * W, 3 * W)],
    }


def workspace():
    """A step with partial results refuses a workspace that is missing, too small or not aligned."""
    p = Pool(200)
    q = p.seq(2000)
    step = p.step()
    assert plan(step, [request(q, 1)]) == 0
    n = ctypes.c_int64()
    assert lib.kv_step_workspace(step, ctypes.byref(n)) == 0
    call = lambda ws, size: lib.kv_step_attend(step, 0, p.rows, 2, 256, p.rows + 512, 2, 256, 0.0, ws, size, None)
    return [n.value > 0, call(None, n.value), call(p.rows, n.value - 1), call(p.rows + 4, n.value), call(p.rows, n.value)]


if __name__ == "__main__":
    print(json.dumps(globals()[sys.argv[1]](*sys.argv[2:])))
