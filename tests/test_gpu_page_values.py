"""Attention over pages whose values are no numbers where rows see them, against what
the definition gives: an infinity times a weight is that infinity, wherever it lies."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref
from paper_2608_19147_amd import PagedRequest

pytestmark = pytest.mark.gpu

W = dict(Hq=4, Hkv=2)


def _attend(kv, D, q_dtype, n, P, put, peak, masked=False, copies=1):
    """One step of `copies` sequences that share P rows and have n new ones each; put(v) changes rows of V [T, D] of kv head 1 (all new
    rows are alike).  With `peak` one row draws nearly all weight of every query.  (out, 64-bit o, bound, sees) of the first."""
    st = ref.make_stage(kv=kv, D=D, **W)
    pool = st.new_pages((P + 16) // 16 + copies * (n // 16 + 3), 16)
    base = pool.new_sequence()
    g = torch.Generator(device="cuda").manual_seed(n + P)
    k, v = (torch.randn((1, 2, P, D), device="cuda", generator=g).to(st.kv_dtype) for _ in range(2))
    if peak:
        k[..., 0] = 0
        k[..., P // 2, 0] = 4
    base.append(k, v)
    seqs = pool.fork([base] * copies)
    M = n * copies
    mask = None
    if masked:
        mask = np.ones(P + n, np.uint8)
        mask[P // 3] = 0
    step = pool.new_step()
    step.plan([PagedRequest(s, n, mask=mask) for s in seqs])
    q = torch.randn((M, 4 * D), device="cuda", generator=g).to(q_dtype)
    if peak:
        q[:, ::D] = 8.0
    new = [torch.randn((n, 2 * D), device="cuda", generator=g).to(st.kv_dtype).repeat(copies, 1) for _ in range(2)]
    if peak:
        new[0][:, ::D] = 0
    step.write(0, q[:, :4 * D].to(st.kv_dtype), *new)
    for s in seqs:                                               # shared rows are changed more than once, to the same
        table = s.pages
        rows = torch.cat([pool.v[0, p, 1] for p in table])[: P + n]
        put(rows)
        for t, p in enumerate(table):
            part = rows[16 * t: 16 * (t + 1)]
            pool.v[0, p, 1, : len(part)] = part
    scale = 1.0 if peak else 1 / math.sqrt(D)
    out = step.attend(0, q, scale=scale)[:n].view(n, 4, D).double()
    kk, vv = seqs[0].read(0)
    see = ref.sees(P, n, mask)
    clean = torch.where(torch.isfinite(vv), vv, 0)
    o, a, s_abs, s_top = ref.attend(q[:n].view(n, 4, D), kk, clean, see, scale)
    bound = ref.attend_bound(o, a, s_abs, s_top, P + n, D, st.kv_dtype, q_dtype, q_dtype)
    # what is no number and is seen: one infinity stays, two signs or a NaN are NaN
    bad = torch.where(torch.isfinite(vv), 0, vv).double()[1]     # of kv head 1: query heads 2 and 3
    for i in range(n):
        seen = bad[torch.from_numpy(see[i]).cuda()]
        o[i, 2:] = o[i, 2:] + seen.sum(0)
    pool.free()
    st.close()
    return out, o, bound


def _check(out, o, bound):
    finite = torch.isfinite(o)
    assert torch.isnan(out[torch.isnan(o)]).all()
    inf = torch.isinf(o)
    assert (out[inf] == o[inf]).all(), out[inf & (out != o)]
    err = (out - o).abs()
    assert torch.isfinite(out[finite]).all() and (err[finite] <= bound[finite]).all()


CASES = [("bf16", 128, torch.bfloat16), ("f16", 64, torch.float16), ("bf16", 64, torch.float32), ("f16", 128, torch.float32)]


@pytest.mark.parametrize("kv,D,q_dtype", CASES)
@pytest.mark.parametrize("n,P", [(1, 700), (1, 40), (5, 333), (10, 95), (30, 260), (70, 1000), (150, 64)])
@pytest.mark.parametrize("peak", [False, True])
def test_infinite_rows_that_are_seen(kv, D, q_dtype, n, P, peak):
    """Infinities at the start, within and at the end of the rows that all see, in steps of 16 and 32 keys that are whole and in the
    last one; among them one under a weight that 16 bits do not hold (e^-32 of the largest)."""
    for j in (0, 17, P // 2 + 1, P - 1, P):                      # (row P is the first new one: the last that every new row sees)
        def put(v):
            v[j, 0] = math.inf
            v[j, 3] = -math.inf
            v[j, D // 2 + 1] = math.inf
        _check(*_attend(kv, D, q_dtype, n, P, put, peak))


@pytest.mark.parametrize("kv,D,q_dtype", CASES)
@pytest.mark.parametrize("n,P", [(1, 700), (10, 95), (30, 260), (150, 64)])
@pytest.mark.parametrize("masked", [False, True])
def test_signs_and_nans(kv, D, q_dtype, n, P, masked):
    """Infinities of both signs in one dim, NaN beside infinity, and a hidden row (where there is a mask) that holds them."""
    def put(v):
        v[5, 1] = math.inf
        v[P - 2, 1] = -math.inf
        v[5, 2] = math.nan
        v[P - 2, 4] = math.inf
        v[P + n - 1, 6] = -math.inf
        v[P // 3 if masked else P - 1, 7] = math.inf
    _check(*_attend(kv, D, q_dtype, n, P, put, False, masked))


@pytest.mark.parametrize("kv,D,q_dtype", CASES)
@pytest.mark.parametrize("copies,n", [(16, 1), (5, 5), (3, 40)])
def test_shared_rows(kv, D, q_dtype, copies, n):
    """An infinite row of a run that several sequences share, and one of the last of their own."""
    def put(v):
        v[100, 9] = math.inf
        v[-1, 10] = -math.inf
    _check(*_attend(kv, D, q_dtype, n, 800, put, True, copies=copies))


@pytest.mark.parametrize("kv,D", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("n", [1, 10, 40])
@pytest.mark.parametrize("size", [0.0, 1e-40, 1e-30])
@pytest.mark.parametrize("scale", [1e-9, 1e-44, None])
def test_smallest_scores(kv, D, n, size, scale):
    """Queries and scales whose scores all round to zero: the mean of what a row sees (their product is no fp32 number above zero)."""
    st = ref.make_stage(kv=kv, D=D, **W)
    pool = st.new_pages(40, 16)
    s = pool.new_sequence()
    s.append(ref.rows(st, 300, 1), ref.rows(st, 300, 2))
    step = pool.new_step()
    step.plan([PagedRequest(s, n)])
    g = torch.Generator(device="cuda").manual_seed(3)
    new = [torch.randn((n, 2 * D), device="cuda", generator=g).to(st.kv_dtype) for _ in range(2)]
    q = torch.randn((n, 4 * D), device="cuda", generator=g) * size
    step.write(0, q.to(st.kv_dtype), *new)
    out = step.attend(0, q, scale=scale).view(n, 4, D).double()
    k, v = s.read(0)
    o, a, s_abs, s_top = ref.attend(q.view(n, 4, D), k, v, ref.sees(300, n), scale or 1 / math.sqrt(D))
    bound = ref.attend_bound(o, a, s_abs, s_top, 300 + n, D, st.kv_dtype, torch.float32, torch.float32)
    assert ((out - o).abs() <= bound).all()
    pool.free()
    st.close()


@pytest.mark.parametrize("kv,D,q_dtype", CASES)
@pytest.mark.parametrize("copies,n", [(1, 1), (12, 1), (5, 5), (3, 40), (1, 150)])
def test_queries_that_are_no_numbers(kv, D, q_dtype, copies, n):
    """A row whose query holds NaN (a padded one, say) is NaN in that head; the others are as without it, bit for bit, an infinite
    value among the rows that they see too."""
    for infinite in (False, True):
        st = ref.make_stage(kv=kv, D=D, **W)
        pool = st.new_pages(80 + 12 * copies, 16)
        base = pool.new_sequence()
        base.append(ref.rows(st, 700, 1), ref.rows(st, 700, 2))
        if infinite:
            pool.v[0, base.pages[5], :, 3, 7] = math.inf
        seqs = pool.fork([base] * copies)
        step = pool.new_step()
        step.plan([PagedRequest(s, n) for s in seqs])
        g = torch.Generator(device="cuda").manual_seed(n)
        M = n * copies
        q = torch.randn((M, 4 * D), device="cuda", generator=g).to(q_dtype)
        new = [torch.randn((M, 2 * D), device="cuda", generator=g).to(st.kv_dtype) for _ in range(2)]
        step.write(0, q.to(st.kv_dtype), *new)
        clean = step.attend(0, q)
        bad = q.clone()
        bad[M // 2, D + 1] = math.nan
        out = step.attend(0, bad)
        assert torch.isnan(out[M // 2, D:2 * D]).all()
        out[M // 2, D:2 * D] = clean[M // 2, D:2 * D]
        assert torch.equal(out, clean)
        assert torch.isinf(clean).sum() == (4 * M if infinite else 0)
        pool.free()
        st.close()
