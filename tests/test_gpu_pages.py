"""The paged cache on the GPU against plain 64-bit forms: attention of sequences that
share pages, the write of rotated rows, forks, compaction, and runs of them together."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref
from paper_2608_19147_amd import PagedRequest, StageError

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stages():
    made = {}

    def get(**kw):
        key = tuple(sorted(kw.items()))
        if key not in made:
            made[key] = ref.make_stage(**kw)
        return made[key]

    yield get
    for s in made.values():
        s.close()


def _q(stage, M, seed, dtype=None, scale=1.3, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = stage.shape.n_q_heads * stage.shape.head_dim
    return (torch.randn((M, w + pad), device="cuda", generator=g) * scale).to(dtype or stage.kv_dtype)[:, :w]


def _check_attend(stage, step, seqs, q, P, n, masks=None, mask_rows=None, layer=0, scale=None, **kw):
    """One layer's attention of a planned step against the rows that the sequences hold."""
    D, Hq = stage.shape.head_dim, stage.shape.n_q_heads
    out = step.attend(layer, q, scale=scale, **kw)
    row = 0
    for i, s in enumerate(seqs):
        k, v = s.read(layer)
        see = ref.sees(P[i], n[i], None if masks is None else masks[i], None if mask_rows is None else mask_rows[i])
        qi = q[row:row + n[i]].reshape(n[i], Hq, D)
        o, a, s_abs, s_top = ref.attend(qi, k, v, see, scale or 1 / math.sqrt(D))
        bound = ref.attend_bound(o, a, s_abs, s_top, P[i] + n[i], D, stage.kv_dtype, q.dtype, out.dtype)
        err = (out[row:row + n[i]].reshape(n[i], Hq, D).double() - o).abs()
        assert torch.isfinite(out[row:row + n[i]]).all()
        assert (err <= bound).all(), (i, float((err / bound).max()))
        row += n[i]
    return out


def _batch(stage, page, prefixes, own, n, seed=0):
    """Sequences over a common tree of prefixes: prefixes[i] names the rows of each level that sequence i begins with; own rows
    and n new ones behind them.  Returns (pool, seqs, P)."""
    levels = {}
    need = 0
    for ps in prefixes:
        for d in range(len(ps)):
            key = ps[: d + 1]
            if key not in levels:
                levels[key] = None
                need += -(-ps[d][1] // page) + 2
    need += sum(-(-(o + m) // page) + 2 for o, m in zip(own, n))
    pool = stage.new_pages(need, page)
    pool.k.fill_(float("nan"))                                   # what nobody wrote may hold anything
    pool.v.fill_(float("nan"))
    base = pool.new_sequence()
    for key in sorted(levels, key=len):
        parent = base if len(key) == 1 else levels[key[:-1]]
        levels[key] = pool.fork([parent])[0]
        if key[-1][1]:
            at = seed + 7 * len(key) + key[-1][0]
            levels[key].append(ref.rows(stage, key[-1][1], 100 + at, 1.1), ref.rows(stage, key[-1][1], 200 + at))
    seqs = pool.fork([levels[ps] if ps else base for ps in prefixes])
    for i, s in enumerate(seqs):
        if own[i]:
            s.append(ref.rows(stage, own[i], 300 + seed + i), ref.rows(stage, own[i], 400 + seed + i))
    return pool, seqs, [s.length for s in seqs]


def _write_raw(stage, step, M, seed, layer=0):
    """New rows of K and V, not turned."""
    w = stage.shape.n_kv_heads * stage.shape.head_dim
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn((M, w), device="cuda", generator=g).to(stage.kv_dtype) for _ in range(2))
    q = _q(stage, M, seed + 1)
    step.write(layer, q, k, v)


SHAPES = [dict(Hq=4, Hkv=2, D=64, kv="bf16"), dict(Hq=8, Hkv=1, D=128, kv="f16"), dict(Hq=14, Hkv=2, D=128, kv="bf16"),
          dict(Hq=16, Hkv=16, D=64, kv="f16"), dict(Hq=32, Hkv=2, D=64, kv="bf16")]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("past,n", [(0, 1), (1, 1), (15, 1), (31, 2), (63, 1), (64, 3), (255, 1), (700, 5), (1023, 1), (95, 40)])
def test_attend_one(stages, shape, page, past, n):
    """One sequence: lengths around the ends of pages, steps and splits."""
    st = stages(**shape)
    pool, seqs, P = _batch(st, page, [()], [past], [n])
    step = pool.new_step()
    step.plan([PagedRequest(seqs[0], n)])
    _write_raw(st, step, n, 5)
    _check_attend(st, step, seqs, _q(st, n, 9), P, [n])
    pool.free()


def _tree(n, T, seed):
    """Masks of n new rows behind T - n others, each with one of those before it for its parent."""
    r = np.random.default_rng(seed)
    rows = np.ones((n, T), np.uint8)
    rows[:, T - n:] = 0
    for i in range(n):
        rows[i, T - n + i] = 1
        if i:
            p = int(r.integers(max(0, i - 4), i))
            rows[i, T - n:] |= rows[p, T - n:]
    return rows


def _holes(T, n, seed, share=0.1):
    m = (np.random.default_rng(seed).random(T) >= share).astype(np.uint8)
    m[T - n:] = 1
    return m


# a level is (name, rows); sequences that name the same levels share them
A, B, C = (0, 512), (1, 300), (2, 129)
BATCHES = {
    "same prefix": ([(A,)] * 9, [0, 1, 15, 16, 17, 64, 200, 300, 5], [1] * 9),
    "two levels": ([(A, B), (A, B), (A, C), (A, C), (A,), (A, B, C), (A, B, C)], [3, 40, 0, 70, 9, 1, 0], [1, 2, 3, 1, 5, 4, 1]),
    "nothing shared": ([(), (), ()], [600, 17, 0], [3, 1, 7]),
    "many": ([(B,)] * 40, [i % 7 for i in range(40)], [1] * 40),
    "prompts": ([(A,), (A,), (A, B)], [10, 0, 33], [70, 200, 1]),
    "short prefix": ([((3, 20),)] * 4, [1, 2, 3, 4], [1] * 4),
    "ends with the prefix": ([((4, 256),), ((4, 256),), ((4, 256), (5, 256))], [0, 0, 0], [1, 2, 1]),
}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("batch", list(BATCHES))
@pytest.mark.parametrize("mask", ["none", "holes", "tree"])
def test_attend_shared(stages, shape, page, batch, mask):
    st = stages(**shape)
    prefixes, own, n = BATCHES[batch]
    pool, seqs, P = _batch(st, page, prefixes, own, n)
    step = pool.new_step()
    masks = None if mask == "none" else [_holes(p + m, m, i) for i, (p, m) in enumerate(zip(P, n))]
    rows = [_tree(m, p + m, i) for i, (p, m) in enumerate(zip(P, n))] if mask == "tree" else None
    step.plan([PagedRequest(q, m, mask=masks and masks[i], mask_rows=rows and rows[i]) for i, (q, m) in enumerate(zip(seqs, n))])
    _write_raw(st, step, sum(n), 6)
    _check_attend(st, step, seqs, _q(st, sum(n), 10), P, n, masks, rows)
    pool.free()


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("q_dtype", ["kv", "f32"])
@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_attend_types(stages, kv, q_dtype, out, D):
    """Query and output types; rows inside wider ones at odd strides; a scale of its own."""
    st = stages(Hq=12, Hkv=2, D=D, kv=kv)
    prefixes, own, n = BATCHES["two levels"]
    n = [20 if m == 5 else m for m in n]
    pool, seqs, P = _batch(st, 32, prefixes, own, n)
    step = pool.new_step()
    step.plan([PagedRequest(q, m) for q, m in zip(seqs, n)])
    M = sum(n)
    _write_raw(st, step, M, 7)
    q = _q(st, M, 11, None if q_dtype == "kv" else torch.float32, pad=3)
    wide = torch.full((M, 12 * D + 5), 77.0, dtype=ref.TORCH[out], device="cuda")
    got = _check_attend(st, step, seqs, q, P, n, scale=0.05, out=wide[:, :12 * D])
    assert got.data_ptr() == wide.data_ptr() and (wide[:, 12 * D:] == 77.0).all()
    pool.free()


@pytest.mark.parametrize("kv", ["bf16", "f16"])
def test_attend_fp32_of_any_size(stages, kv):
    """fp32 queries far from 1 (beyond fp16's range) keep their bits: the scores are the scale's business."""
    st = stages(Hq=4, Hkv=2, D=64, kv=kv)
    pool, seqs, P = _batch(st, 64, [()], [300], [2])
    step = pool.new_step()
    step.plan([PagedRequest(seqs[0], 2)])
    _write_raw(st, step, 2, 8)
    q = _q(st, 2, 12, torch.float32)
    for power in (-100, -30, 20, 60):
        _check_attend(st, step, seqs, q * 2.0 ** power, P, [2], scale=0.1 * 2.0 ** -power)
    pool.free()


def test_rows_that_see_nothing(stages):
    """A row whose masks leave nothing gives zeros, beside rows that see something."""
    for kv, D in (("bf16", 128), ("f16", 64)):
        st = stages(Hq=4, Hkv=2, D=D, kv=kv)
        pool, seqs, P = _batch(st, 16, [(A,), (A,), (A,)], [30, 0, 5], [3, 1, 2])
        n = [3, 1, 2]
        masks = [np.zeros(P[0] + 3, np.uint8), None, np.ones(P[2] + 2, np.uint8)]
        rows = np.ones((2, P[2] + 2), np.uint8)
        rows[1] = 0
        step = pool.new_step()
        step.plan([PagedRequest(seqs[0], 3, mask=masks[0]), PagedRequest(seqs[1], 1), PagedRequest(seqs[2], 2, mask=masks[2], mask_rows=rows)])
        _write_raw(st, step, 6, 8)
        out = _check_attend(st, step, seqs, _q(st, 6, 13), P, n, masks, [None, None, rows])
        assert (out[:3] == 0).all() and (out[5] == 0).all() and (out[4] != 0).any()
        pool.free()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("kv,D,n", [("bf16", 128, 5), ("f16", 64, 5), ("bf16", 64, 30), ("f16", 128, 70)])
def test_what_is_not_seen(stages, bad, kv, D, n):
    """Rows with no numbers that a query does not see (later tokens, other branches of a tree, hidden rows of a shared prefix)
    reach it in no way; those that it sees do."""
    st = stages(Hq=4, Hkv=2, D=D, kv=kv)
    pool, seqs, P = _batch(st, 16, [(A,), (A,)], [40, 7], [n, n])
    masks, rows = [], []
    for i in range(2):
        m = np.ones(P[i] + n, np.uint8)
        m[[3, 140, P[i] - 1]] = 0                                # hidden rows, shared and own, hold no numbers
        w = np.tril(np.ones((n, P[i] + n), np.uint8), P[i])
        w[:, P[i] + 2] = 0                                       # one new row only the last new one sees, beside itself
        w[[2, n - 1], P[i] + 2] = 1
        masks.append(m)
        rows.append(w)
    step = pool.new_step()
    step.plan([PagedRequest(q, n, mask=m, mask_rows=w) for q, m, w in zip(seqs, masks, rows)])
    _write_raw(st, step, 2 * n, 9)
    table = [s.pages for s in seqs]

    def put(i, j, what):
        for t in what:
            t[0, table[i][j // 16], :, j % 16] = bad
    for i in range(2):
        for j in (3, 140, P[i] - 1):
            put(i, j, (pool.k, pool.v))
        put(i, P[i] + 2, (pool.v,))
    out = step.attend(0, _q(st, 2 * n, 14)).view(2, n, 4, D)
    for i in range(2):
        k, v = seqs[i].read(0)
        see = ref.sees(P[i], n, masks[i], rows[i])
        o, a, s_abs, s_top = ref.attend(_q(st, 2 * n, 14)[i * n:(i + 1) * n].reshape(n, 4, D), k, torch.nan_to_num(v.double(), 0, 0, 0), see, 1 / math.sqrt(D))
        clean = [r for r in range(n) if r not in (2, n - 1)]
        bound = ref.attend_bound(o, a, s_abs, s_top, P[i] + n, D, st.kv_dtype, st.kv_dtype, st.kv_dtype)
        assert ((out[i].double() - o).abs()[clean] <= bound[clean]).all()
        for r in (2, n - 1):
            assert torch.isnan(out[i, r]).all() if math.isnan(bad) else (out[i, r].double() == bad).all()
    pool.free()


def test_long_cache(stages):
    """Offsets of one layer's pages past 32 bits of bytes, and partial results of many splits."""
    st = stages(Hq=16, Hkv=8, D=128, kv="bf16")
    pool = st.new_pages(4800, 256)                               # 2.5 GB of K
    filler = pool.new_sequence()
    r = ref.rows(st, 65536, 1)
    for _ in range(17):
        filler.append(r, r)                                      # the first 4352 pages
    a = pool.new_sequence()
    a.append(ref.rows(st, 70001, 2), ref.rows(st, 70001, 3))
    assert min(a.pages) >= 4352 and (min(a.pages) * 8 * 256 * 128 * 2) > 2 ** 31
    step = pool.new_step()
    step.plan([PagedRequest(a, 1)])
    _write_raw(st, step, 1, 4)
    _check_attend(st, step, [a], _q(st, 1, 5, scale=0.5), [70001], [1])
    pool.free()


@pytest.mark.parametrize("kv", ["bf16", "f16"])
@pytest.mark.parametrize("x", ["f32", "kv"])
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 2), (128, 10, 2), (128, 64, 8)])
@pytest.mark.parametrize("axes", [0, 1, 3])
@pytest.mark.parametrize("n,page,pad", [([1], 16, 0), ([3, 1, 18], 16, 3), ([130, 7], 64, 1)])
def test_write(stages, kv, x, D, Hq, Hkv, axes, n, page, pad):
    """Rows turned (by one axis, by three, not at all) and stored; nothing else in the pages changes."""
    st = stages(Hq=Hq, Hkv=Hkv, D=D, kv=kv)
    r = np.random.default_rng(3)
    axis = r.integers(0, 3, D // 2).astype(np.uint8) if axes == 3 else None
    if axis is not None:
        axis[:3] = (0, 1, 2)
    pool = st.new_pages(64, page, pair_axis=axis)
    assert pool.n_axes == max(1, axes)
    past = [5 * i + 2 for i in range(len(n))]
    seqs = [pool.new_sequence() for _ in n]
    for i, s in enumerate(seqs):
        s.append(ref.rows(st, past[i], 20 + i), ref.rows(st, past[i], 30 + i))
    before = (pool.k.clone(), pool.v.clone())
    pos = [r.integers(0, 4096, (max(1, axes), m)).astype(np.int32) for m in n]
    step = pool.new_step()
    step.plan([PagedRequest(s, m, positions=pos[i] if axes else None) for i, (s, m) in enumerate(zip(seqs, n))])
    M, g = sum(n), torch.Generator(device="cuda").manual_seed(4)
    dt = torch.float32 if x == "f32" else st.kv_dtype
    wide = torch.randn((M, (Hq + 2 * Hkv) * D + pad), device="cuda", generator=g).to(dt)
    q, k, v = wide[:, :Hq * D], wide[:, Hq * D:(Hq + Hkv) * D], wide[:, (Hq + Hkv) * D:(Hq + 2 * Hkv) * D]
    qo = step.write(0, q, k, v)
    at = np.concatenate(pos, 1) if axes else np.zeros((1, M))
    wq, wk = ref.turned(q.reshape(M, Hq, D), at, axis), ref.turned(k.reshape(M, Hkv, D), at, axis)

    def near(got, want, src):
        # two products and a sum in fp32 of values and of cos and sin rounded to fp32, then one rounding
        pair = (src.double() ** 2).reshape(len(src), -1, 2, D // 2).sum(2).sqrt().repeat(1, 1, 2)
        bound = 6 * 2.0 ** -24 * pair * (1 + ref.HALF_STEP[got.dtype]) + want.abs() * ref.HALF_STEP[got.dtype] + ref.TINY[got.dtype]
        assert ((got.double() - want).abs() <= bound).all()

    near(qo.view(M, Hq, D), wq, q.reshape(M, Hq, D))
    row = 0
    for i, s in enumerate(seqs):
        gk, gv = s.read(0, past[i], n[i])
        near(gk.transpose(0, 1), wk[row:row + n[i]], k.reshape(M, Hkv, D)[row:row + n[i]])
        assert torch.equal(gv.transpose(0, 1), v.reshape(M, Hkv, D)[row:row + n[i]].to(st.kv_dtype))
        for j in range(past[i], past[i] + n[i]):
            for t in (pool.k, pool.v):
                t[0, s.pages[j // page], :, j % page] = 0
        row += n[i]
    assert torch.equal(pool.k, before[0]) and torch.equal(pool.v, before[1])   # (new pages start as zeros)
    # into q itself, and in fp32
    if x == "f32":
        want = step.write(0, q.clone(), k, v, q_out=torch.empty((M, Hq * D), device="cuda"))
        same = q.clone()
        assert step.write(0, same, k, v, q_out=same) is same and torch.equal(same, want)
    pool.free()


# ------------------------------------------------------------------ forks, compaction, truncation

class Mirror:
    """Sequences of a pool and what their rows have to be: K and V [L, Hkv, n, D] each."""

    def __init__(self, stage, pool):
        self.stage, self.pool, self.live, self.seed = stage, pool, [], 1000

    def rows(self, n):
        self.seed += 2
        return [ref.rows(self.stage, n, self.seed + j) for j in range(2)]

    def new(self):
        sh = self.stage.shape
        empty = torch.empty((sh.n_layers, sh.n_kv_heads, 0, sh.head_dim), dtype=self.stage.kv_dtype, device="cuda")
        self.live.append([self.pool.new_sequence(), [empty, empty]])

    def check(self):
        used = set()
        for s, kv in self.live:
            assert s.length == kv[0].shape[2]
            pages = s.pages
            used |= set(pages)
            assert len(set(pages)) == len(pages) == -(-s.length // self.pool.page_rows)
            for l in range(self.stage.shape.n_layers):
                got = s.read(l)
                assert torch.equal(got[0], kv[0][l]) and torch.equal(got[1], kv[1][l])
        assert self.pool.free_pages == self.pool.n_pages - len(used)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("D,kv", [(64, "f16"), (128, "bf16")])
@pytest.mark.parametrize("seed", range(4))
def test_sequences_against_a_mirror(stages, page, D, kv, seed):
    """Random appends, forks (some with masks or lengths), compactions, truncations, steps and frees: every sequence keeps its own
    rows, and pages are neither lost nor shared beyond their sequences."""
    st = stages(L=2, Hq=4, Hkv=2, D=D, kv=kv)
    pool = st.new_pages(160, page)
    r = np.random.default_rng(seed)
    m = Mirror(st, pool)
    m.new()
    for turn in range(60):
        what = r.choice(["append", "fork", "fork", "mask", "compact", "cut", "free", "step", "new"])
        if not m.live or what == "new":
            m.new()
        at = int(r.integers(len(m.live)))
        s, kv_ = m.live[at]
        n = s.length
        if what == "append":
            more = m.rows(int(r.integers(1, 5 * page if n < 400 else 5)))
            s.append(*more)
            m.live[at][1] = [torch.cat(x, 2) for x in zip(kv_, more)]
        elif what in ("fork", "mask") and len(m.live) < 8:
            at2 = int(r.integers(len(m.live)))
            src = [at, at, at2]                                  # the same sequence twice
            lens = [int(r.integers(0, m.live[i][0].length + 1)) for i in src] if r.random() < 0.5 else None
            got = [m.live[i][0].length if lens is None else lens[j] for j, i in enumerate(src)]
            keep = None
            if what == "mask":
                keep = [(r.random(g) >= r.choice([0.0, 0.02, 0.5, 1.0])).astype(np.uint8) for g in got]
                keep[1] = None
            kids = pool.fork([m.live[i][0] for i in src], lengths=lens, keep=keep)
            for j, (kid, i) in enumerate(zip(kids, src)):
                sel = torch.arange(got[j], device="cuda")
                if keep is not None and keep[j] is not None:
                    sel = sel[torch.from_numpy(keep[j]).cuda().bool()]
                m.live.append([kid, [x[:, :, sel] for x in m.live[i][1]]])
        elif what == "compact" and n:
            keep = (r.random(n) >= r.choice([0.01, 0.4, 1.0])).astype(np.uint8)
            if r.random() < 0.3:
                keep[: n // 2] = 1
            assert s.compact(keep) == keep.sum()
            sel = torch.from_numpy(keep).cuda().bool()
            m.live[at][1] = [x[:, :, sel] for x in kv_]
        elif what == "cut":
            to = int(r.integers(0, n + 1))
            s.truncate(to)
            m.live[at][1] = [x[:, :, :to] for x in kv_]
        elif what == "free":
            s.free()
            m.live.pop(at)
        elif what == "step":
            pick = sorted(set(int(i) for i in r.integers(0, len(m.live), 3)))
            new = [int(r.integers(1, 20)) for _ in pick]
            step = pool.new_step()
            step.plan([PagedRequest(m.live[i][0], k) for i, k in zip(pick, new)])
            M = sum(new)
            q = _q(st, M, turn)
            both = [torch.empty((2, 2, M, D), dtype=st.kv_dtype, device="cuda") for _ in range(2)]   # [L, Hkv, M, D]
            for l in range(2):
                flat = [_q(st, M, turn + 50 * l + 7 * j)[:, :2 * D] for j in range(2)]
                step.write(l, q, *flat)
                for b, f in zip(both, flat):
                    b[l] = f.reshape(M, 2, D).transpose(0, 1)
            row = 0
            for i, k in zip(pick, new):
                m.live[i][1] = [torch.cat([x, b[:, :, row:row + k]], 2) for x, b in zip(m.live[i][1], both)]
                row += k
        m.check()
    for s, _ in m.live:
        s.free()
    assert pool.free_pages == 160
    pool.free()


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("n,drop", [(1500, 0.3), (1500, 0.001), (700, 0.9)])
@pytest.mark.parametrize("shared", [0, 100, 1400])
@pytest.mark.parametrize("full", [False, True])
def test_compact_long(stages, page, n, drop, shared, full):
    """Compaction of many rows, into new pages and (in a pool that has none left) in place; sharers keep theirs."""
    st = stages(L=2, Hq=4, Hkv=2, D=64, kv="f16")
    shared = min(shared, n)
    pool = st.new_pages(2 * -(-n // page) + 4 if not full else -(-n // page) + (-(-shared // page) if shared else 0) + 2, page)
    s = pool.new_sequence()
    k, v = ref.rows(st, n, 1), ref.rows(st, n, 2)
    s.append(k, v)
    other = pool.fork([s], [shared])[0]
    rest = pool.new_sequence()
    if full and pool.free_pages - -(-shared // page) > 0:
        fill = (pool.free_pages - -(-shared // page)) * page
        r = ref.rows(st, fill, 3)
        rest.append(r, r)
    keep = (np.random.default_rng(5).random(n) >= drop).astype(np.uint8)
    sel = torch.from_numpy(keep).cuda().bool()
    assert s.compact(keep) == keep.sum()
    for l in range(2):
        got = s.read(l)
        assert torch.equal(got[0], k[l][:, sel]) and torch.equal(got[1], v[l][:, sel])
        got = other.read(l)
        assert torch.equal(got[0], k[l][:, :shared]) and torch.equal(got[1], v[l][:, :shared])
    pool.free()


def test_lowest_pages_first(stages):
    st = stages(Hq=4, Hkv=2, D=64, kv="bf16")
    pool = st.new_pages(200, 16)
    r = ref.rows(st, 16 * 70, 1)
    a, b = pool.new_sequence(), pool.new_sequence()
    a.append(r, r)
    b.append(r, r)
    assert a.pages == list(range(70)) and b.pages == list(range(70, 140))
    a.truncate(33)
    c = pool.fork([b], keep=[np.r_[np.zeros(1, np.uint8), np.ones(16 * 70 - 1, np.uint8)]])[0]
    assert c.pages == list(range(3, 70)) + [140, 141, 142]
    pool.free()


def test_parent_goes_on_behind_its_forks(stages):
    """A sequence that is truncated into a page that it shares, and goes on, writes to a copy of it."""
    st = stages(Hq=4, Hkv=2, D=64, kv="bf16")
    pool = st.new_pages(20, 16)
    a = pool.new_sequence()
    k, v = ref.rows(st, 64, 1), ref.rows(st, 64, 2)
    a.append(k, v)
    b = pool.fork([a])[0]
    assert b.pages == a.pages
    a.truncate(40)
    more = ref.rows(st, 3, 3)
    a.append(more, more)
    assert a.pages[:2] == b.pages[:2] and a.pages[2] != b.pages[2]
    assert torch.equal(b.read(0)[0], k[0]) and torch.equal(a.read(0)[0], torch.cat([k[0][:, :40], more[0]], 1))
    b.truncate(42)                                               # now the other way, and by a step
    step = pool.new_step()
    c = pool.fork([b], [32])[0]
    step.plan([PagedRequest(b, 2), PagedRequest(c, 1)])
    _write_raw(st, step, 3, 4)
    _check_attend(st, step, [b, c], _q(st, 3, 5), [42, 32], [2, 1])
    assert torch.equal(b.read(0, 0, 42)[1], v[0][:, :42])
    pool.free()


def test_load_from_a_state(stages):
    """Rows of a KV state's slot as the slot sees them, through its beam table."""
    from paper_2608_19147_amd import Request
    st = stages(L=2, Hq=4, Hkv=2, D=64, kv="bf16")
    state = st.new_state(3, 64)
    k, v = (torch.cat([ref.rows(st, 20, 10 * j + b)[:, None] for b in range(3)], 1) for j in (1, 2))
    state.append(k, v)
    x = torch.randn((3, 256), device="cuda").to(torch.bfloat16)
    st.forward([Request(state, np.full((3, 1), 20, np.int32), np.ones((3, 21), np.uint8), np.array([2, 0, 0], np.int32))], x)
    pool = st.new_pages(12, 16)
    for slot in range(3):
        s = pool.new_sequence()
        s.load(state, slot, 0, 7)
        s.load(state, slot, 7)
        assert s.length == 21
        for l in range(2):
            want = state.read(l, slot, 0, 21)
            assert all(torch.equal(a, b) for a, b in zip(s.read(l), want))
    pool.free()
    state.free()


# ------------------------------------------------------------------ the forward over sequences

@pytest.fixture(scope="module", params=[128, 64])
def pair(request):
    """A stage of the matrix-core products, and one of another group size, which has none."""
    import dataclasses
    import synth
    from gpu_cases import Pair
    p = Pair(dataclasses.replace(synth.TINY, group_size=request.param), 77)
    yield p
    p.close()


def _twin(pair, rows_k, rows_v, cap=400):
    """A KV state and the oracle's with the given rows [L, Hkv, n, D]."""
    import oracle
    g = pair.gpu.new_state(1, cap)
    o = oracle.OracleState(pair.shape, 1, cap)
    if rows_k.shape[2]:
        g.append(rows_k[:, None].contiguous(), rows_v[:, None].contiguous())
        o.append(rows_k[:, None].double().cpu().numpy(), rows_v[:, None].double().cpu().numpy())
    return g, o


@pytest.mark.parametrize("n", [[1, 1, 1], [3, 1, 5], [20, 17, 9]])
@pytest.mark.parametrize("page", [16, 64])
def test_forward_over_shared_pages(pair, n, page):
    """Requests that share a prefix, through the stage: as stage_forward of states that hold the prefix each (to rounding), and as
    the oracle; twice in turn, so that the second forward reads what the first wrote.  One request hides rows, one is a tree."""
    import oracle
    from gpu_cases import TOL_STAGE, Request, host, rel_err
    import synth
    st = pair.gpu
    pool = st.new_pages(60, page)
    base = pool.new_sequence()
    k, v = ref.rows(st, 200, 5, 0.7), ref.rows(st, 200, 6)
    base.append(k, v)
    seqs = pool.fork([base] * 3)
    mine = [(ref.rows(st, m, 10 + m, 0.7), ref.rows(st, m, 20 + m)) for m in (1, 40, 13)]
    states, oracles = [], []
    for s, (a, b) in zip(seqs, mine):
        s.append(a, b)
        g, o = _twin(pair, torch.cat([k, a], 2), torch.cat([v, b], 2))
        states.append(g)
        oracles.append(o)
    for turn in range(2):
        P = [s.length for s in seqs]
        pos = [np.arange(p, p + m, dtype=np.int32) for p, m in zip(P, n)]
        masks = [np.ones(P[0] + n[0], np.uint8), _holes(P[1] + n[1], n[1], 3), None]
        rows = [None, None, _tree(n[2], P[2] + n[2], 4)]
        x = synth.make_hidden(pair.shape, sum(n), 0, 3 + turn).cuda()
        got = st.forward_paged([PagedRequest(s, m, positions=p, mask=mk, mask_rows=w) for s, m, p, mk, w in zip(seqs, n, pos, masks, rows)], x)
        same = st.forward([Request(g, p[None], None if mk is None else mk[None], None, None if w is None else w[None])
                           for g, p, mk, w in zip(states, pos, masks, rows)], x)
        row = 0
        for i in range(3):
            a, b = got[row:row + n[i]], same[row:row + n[i]]
            see = ref.sees(P[i], n[i], masks[i], rows[i]).astype(np.uint8)
            want = oracle.forward(pair.orc, oracles[i], host(x[row:row + n[i]]), pos[i][None], None, None, see[None])
            assert rel_err(host(a), want) <= TOL_STAGE
            assert rel_err(host(a), want) <= 1.5 * rel_err(host(b), want) + 1e-3
            row += n[i]
    for i in range(3):
        assert seqs[i].length == states[i].length
        for l in range(pair.shape.n_layers):
            a, b = seqs[i].read(l), states[i].read(l, 0, 0, states[i].length)
            assert all(rel_err(host(x), host(y)) <= TOL_STAGE for x, y in zip(a, b))
    pool.free()
    for g in states:
        g.free()


def test_forward_generates_from_forks(pair):
    """One prompt prefilled into a state, loaded into pages, forked, decoded by several requests at once, one of them with its
    rejected rows cut or compacted away: each goes on as a state of its own would."""
    from gpu_cases import TOL_STAGE, Request, host, rel_err
    import synth
    st = pair.gpu
    prompt = synth.make_hidden(pair.shape, 90, 0, 8).cuda()
    states = [st.new_state(1, 200) for _ in range(3)]
    for g in states:
        if pair.shape.group_size == 128:
            st.prefill(g, np.arange(90), prompt)
        else:                                                    # no prefill there
            for at in (0, 45):
                pos = np.arange(at, at + 45, dtype=np.int32)[None]
                st.forward([Request(g, pos, np.ones((1, at + 45), np.uint8))], prompt[at:at + 45].contiguous())
    pool = st.new_pages(40, 16)
    base = pool.new_sequence()
    base.load(states[0])
    seqs = pool.fork([base] * 3)
    base.free()
    for turn in range(4):
        x = synth.make_hidden(pair.shape, 3 * 4, 0, 20 + turn).cuda()
        P = [s.length for s in seqs]
        got = st.forward_paged([PagedRequest(s, 4, positions=np.arange(p, p + 4)) for s, p in zip(seqs, P)], x)
        for i, g in enumerate(states):
            want = st.forward([Request(g, np.arange(P[i], P[i] + 4, dtype=np.int32)[None], np.ones((1, P[i] + 4), np.uint8))], x[4 * i:4 * i + 4])
            assert rel_err(host(got[4 * i:4 * i + 4]), host(want)) <= TOL_STAGE
        keep = np.ones(P[1] + 4, np.uint8)
        keep[P[1] + 1:P[1] + 3] = 0                              # the second and third new rows were rejected
        seqs[1].compact(keep)
        states[1].compact(keep[None])
        seqs[2].truncate(P[2] + 1)
        states[2].truncate(P[2] + 1)
        assert [s.length for s in seqs] == [g.length for g in states]
    pool.free()
    for g in states:
        g.free()


def test_forward_refused(pair):
    st = pair.gpu
    pool, other = st.new_pages(4, 16), st.new_pages(4, 16)
    a, b, c = pool.new_sequence(), pool.new_sequence(), other.new_sequence()
    x = torch.zeros((2, pair.shape.hidden), dtype=st.act_dtype, device="cuda")
    pos = np.zeros(1, np.int32)
    for reqs, code in (([PagedRequest(a, 1), PagedRequest(b, 1)], -1),                                    # no positions
                       ([PagedRequest(a, 1, pos), PagedRequest(a, 1, pos)], -6),                          # twice
                       ([PagedRequest(a, 1, pos), PagedRequest(c, 1, pos)], -6),                          # another pool
                       ([PagedRequest(a, 1, pos), PagedRequest(b, 1, pos + 10 ** 6)], -3),                # position
                       ([PagedRequest(a, 1, pos), PagedRequest(b, 1, pos, mask=np.zeros(1, np.uint8))], -1)):
        with pytest.raises(StageError) as e:
            st.forward_paged(reqs, x)
        assert e.value.code == code and a.length == b.length == c.length == 0 and pool.free_pages == 4
    with pytest.raises(StageError) as e:
        st.forward_paged([PagedRequest(a, 65, np.arange(65))], torch.zeros((65, pair.shape.hidden), dtype=st.act_dtype, device="cuda"))
    assert e.value.code == -3
    with pytest.raises(ValueError):
        st.forward_paged([PagedRequest(a, 1, pos)], x)
    with pytest.raises(StageError) as e:                         # hidden rows overlap
        st.forward_paged([PagedRequest(a, 1, pos), PagedRequest(b, 1, pos)], x, hidden_out=x)
    assert e.value.code == -1
    small = st.new_pages(1, 16)
    d, f = small.new_sequence(), small.new_sequence()
    with pytest.raises(StageError) as e:
        st.forward_paged([PagedRequest(d, 1, pos), PagedRequest(f, 1, pos)], x)
    assert e.value.code == -3 and small.free_pages == 1 and d.length == 0
    for p in (pool, other, small):
        p.free()


# ------------------------------------------------------------------ streams, graphs

def test_graphs_of_a_step(stages):
    """Two graphs of a step's write and attention on two streams at once, and eager calls in between: every replay gives the eager
    result for the queries that stand there then."""
    st = stages(Hq=8, Hkv=2, D=128, kv="bf16")
    prefixes, own, n = BATCHES["same prefix"]
    pool, seqs, P = _batch(st, 16, prefixes, own, n)
    step = pool.new_step()
    step.plan([PagedRequest(q, m, positions=np.arange(p, p + m)) for q, m, p in zip(seqs, n, P)])
    M = sum(n)
    g = torch.Generator(device="cuda").manual_seed(1)
    xs = [torch.randn((M, 8 * 128), device="cuda", generator=g).to(torch.bfloat16) for _ in range(8)]
    kv = torch.randn((M, 2 * 128), device="cuda", generator=g).to(torch.bfloat16)
    eager = [step.attend(0, step.write(0, x, kv, kv)) for x in xs]
    held = []
    for j in range(2):
        s = torch.cuda.Stream()
        x = xs[0].clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = step.attend(0, step.write(0, x, kv, kv))
        held.append((s, x, graph, out))
    for i in range(0, 8, 2):
        for j, (s, x, graph, out) in enumerate(held):
            with torch.cuda.stream(s):
                x.copy_(xs[i + j])
                graph.replay()
        again = step.attend(0, step.write(0, xs[i], kv, kv))
        torch.cuda.synchronize()
        assert torch.equal(again, eager[i])
        for j, (s, x, graph, out) in enumerate(held):
            assert torch.equal(out, eager[i + j])
    with pytest.raises(StageError) as e:                         # the graphs hold this plan
        step.plan([PagedRequest(seqs[0], 1)])
    assert e.value.code == -7
    step.free()                                                  # they hold it still
    other = pool.new_step()
    other.plan([PagedRequest(seqs[0], 1)])
    s, x, graph, out = held[0]
    with torch.cuda.stream(s):
        x.copy_(xs[5])
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, eager[5])
    del held, graph
    pool.free()


def test_capture_refused(stages):
    st = stages(Hq=4, Hkv=2, D=64, kv="bf16")
    pool = st.new_pages(8, 16)
    a = pool.new_sequence()
    r = ref.rows(st, 20, 1)
    a.append(r, r)
    step = pool.new_step()
    calls = [lambda: pool.fork([a]), lambda: a.append(r, r), lambda: a.compact(np.zeros(20, np.uint8)), lambda: a.read(0),
             lambda: step.plan([PagedRequest(a, 1)])]
    for call in calls:
        graph, codes = torch.cuda.CUDAGraph(), []
        with torch.cuda.graph(graph):
            torch.zeros(1, device="cuda")
            try:
                call()
            except StageError as e:
                codes.append(e.code)
        assert codes == [-7]
    assert a.length == 20 and pool.free_pages == 6
    pool.free()


def test_calls_on_other_streams(stages):
    """A sequence appended on one stream, forked on a second, stepped on a third and read on a fourth: in the order of the calls."""
    st = stages(L=2, Hq=4, Hkv=2, D=128, kv="f16")
    streams = [torch.cuda.Stream() for _ in range(4)]
    k, v = ref.rows(st, 3000, 1), ref.rows(st, 3000, 2)
    new = [_q(st, 4, 20 + i)[:, :2 * 128] for i in range(2)]
    q = _q(st, 4, 30)
    torch.cuda.synchronize()
    for _ in range(3):
        pool = st.new_pages(2 * 190, 16)
        a = pool.new_sequence()
        a.append(k, v, stream=streams[0])
        b = pool.fork([a], keep=[np.arange(3000) % 3 != 0], stream=streams[1])[0]
        step = pool.new_step()
        step.plan([PagedRequest(a, 3), PagedRequest(b, 1)], stream=streams[2])
        step.write(1, q, *new, stream=streams[3])
        out = step.attend(1, q, stream=streams[0])
        got = b.read(1, stream=streams[1])
        for s in streams:
            s.synchronize()
        want = torch.arange(3000, device="cuda") % 3 != 0
        assert torch.equal(got[0], torch.cat([k[1][:, want], new[0][3:].view(1, 2, 128).transpose(0, 1)], 1))
        assert torch.equal(out, step.attend(1, q))
        pool.free()


def test_binding_refusals(stages):
    st = stages(Hq=4, Hkv=2, D=64, kv="bf16")
    pool, other = st.new_pages(8, 16), st.new_pages(2, 16)
    a = pool.new_sequence()
    step = pool.new_step()
    q, k = _q(st, 2, 1), _q(st, 2, 2)[:, :128]
    with pytest.raises(ValueError):
        step.write(0, q, k, k)                                   # no plan: no rows
    with pytest.raises(ValueError):
        step.plan([PagedRequest(other.new_sequence(), 1)])
    with pytest.raises(ValueError):
        step.plan([PagedRequest(a, 2, mask=np.ones(3, np.uint8))])
    with pytest.raises(ValueError):
        step.plan([PagedRequest(a, 2, mask_rows=np.ones((1, 2), np.uint8))])
    with pytest.raises(ValueError):
        step.plan([PagedRequest(a, 2, positions=np.zeros((3, 2), np.int32))])
    with pytest.raises(StageError) as e:
        step.plan([PagedRequest(a, 8 * 16 + 1)])
    assert e.value.code == -3 and a.length == 0 and pool.free_pages == 8
    with pytest.raises(StageError) as e:
        step.plan([PagedRequest(a, 0)])
    assert e.value.code == -1
    with pytest.raises(StageError) as e:
        step.plan([])
    assert e.value.code == -1
    step.plan([PagedRequest(a, 2)])
    for bad in (q[:1], q.half(), q.double(), q.t(), q.cpu(), _q(st, 2, 1).repeat(1, 2)):
        with pytest.raises(ValueError):
            step.attend(0, bad)
    for layer in (-1, 1):
        with pytest.raises(StageError):
            step.attend(layer, q)
        with pytest.raises(StageError):
            step.write(layer, q, k, k)
    with pytest.raises(ValueError):
        step.attend(0, q, scale=0.0)
    with pytest.raises(StageError):
        step.attend(0, q, scale=math.inf)
    with pytest.raises(ValueError):
        step.write(0, q, k.float(), k)
    with pytest.raises(ValueError):
        step.write(0, q, k, _q(st, 2, 2)[:, :64])
    with pytest.raises(ValueError):
        pool.fork([a], lengths=[1, 2])
    with pytest.raises(StageError):
        pool.fork([a], lengths=[3])
    with pytest.raises(ValueError):
        pool.fork([a], keep=[np.ones(1, np.uint8)])
    with pytest.raises(ValueError):
        a.append(ref.rows(st, 1, 1), ref.rows(st, 2, 1))
    with pytest.raises(ValueError):
        a.append(ref.rows(st, 1, 1).float(), ref.rows(st, 1, 1).float())
    for args in ((0, 0, 3), (0, -1, 1), (1, 0, 1), (0, 2, 1)):
        with pytest.raises(StageError):
            a.read(*args)
    with pytest.raises(StageError):
        a.truncate(3)
    with pytest.raises(ValueError):
        a.compact(np.ones(3, np.uint8))
    a.free()
    with pytest.raises(ValueError):
        pool.fork([a])
    with pytest.raises(ValueError):
        st.new_pages(4, 48)
    with pytest.raises(ValueError):
        st.new_pages(4, 16, pair_axis=np.full(32, 4))
    with pytest.raises(ValueError):
        st.new_pages(4, 16, pair_axis=np.zeros(31))
    pool.free()
    other.free()
