"""Steps whose sequences get other pages, on the GPU: a call that is answered leaves
every other sequence's rows as they were."""
import numpy as np
import pytest
import torch

import pages_ref as ref
from paper_2608_19147_amd import PagedRequest, StageError

pytestmark = pytest.mark.gpu

PAGE, SHAPE = 16, dict(L=2, Hq=4, Hkv=2, D=64, kv="bf16")


@pytest.fixture(scope="module")
def st():
    s = ref.make_stage(**SHAPE)
    yield s
    s.close()


def _all(seqs):
    return [tuple(x.clone() for x in s.read(l)) for s in seqs for l in range(2)]


def _same(a, b):
    return all(torch.equal(x, y) for p, q in zip(a, b) for x, y in zip(p, q))


def _step(st, pool, seq, n):
    step = pool.new_step()
    step.plan([PagedRequest(seq, n)])
    return step, [torch.full((n, w), 3.0, dtype=st.kv_dtype, device="cuda") for w in (256, 128, 128)]


def _write(step, rows):
    for l in range(2):
        step.write(l, *rows)


CHANGES = {
    "compacted": lambda st, pool, q: q.compact((np.arange(70) != 46).astype(np.uint8)),
    "compacted behind": lambda st, pool, q: q.compact((np.arange(70) != 48).astype(np.uint8)),
    "appended to a shared page": lambda st, pool, q: (pool.fork([q], [64]), q.truncate(45), q.append(ref.rows(st, 2, 7), ref.rows(st, 2, 8))),
    "planned on a shared page": lambda st, pool, q: (pool.fork([q], [64]), q.truncate(45), _write(*_step(st, pool, q, 2))),
    "cut": lambda st, pool, q: q.truncate(44),
}


@pytest.mark.parametrize("change", CHANGES)
def test_old_plans(st, change):
    """A plan of 5 rows behind 40, its sequence changed, and the free pages taken by others: its step is refused where one of its
    pages is no more its sequence's, and answers with the sequence's own rows where they are."""
    pool = st.new_pages(24, PAGE)
    q = pool.new_sequence()
    q.append(ref.rows(st, 40, 1), ref.rows(st, 40, 2))
    step, rows = _step(st, pool, q, 5)
    _write(step, rows)
    q.append(ref.rows(st, 25, 3), ref.rows(st, 25, 4))
    held = CHANGES[change](st, pool, q)
    others = [s for s in (held[0] if isinstance(held, tuple) else [])]
    while pool.free_pages:
        s = pool.new_sequence()
        s.append(ref.rows(st, PAGE, 50 + pool.free_pages), ref.rows(st, PAGE, 90 + pool.free_pages))
        others.append(s)
    was = _all(others)
    query = torch.randn((5, 256), device="cuda").to(st.kv_dtype)
    if change == "compacted behind":
        assert q.length == 69
        _write(step, rows)
        k, v = q.read(0)
        o, a, s_abs, s_top = ref.attend(query.view(5, 4, 64), k[:, :45], v[:, :45], ref.sees(40, 5), 0.125)
        bound = ref.attend_bound(o, a, s_abs, s_top, 45, 64, st.kv_dtype, st.kv_dtype, st.kv_dtype)
        assert ((step.attend(0, query).view(5, 4, 64).double() - o).abs() <= bound).all()
    else:
        with pytest.raises(StageError):
            step.write(0, *rows)
        with pytest.raises(StageError):
            step.attend(0, query)
    assert _same(was, _all(others))
    pool.free()


def test_rows_that_a_fork_shares(st):
    """A write into rows of a page that a fork shares is refused; once the fork has gone, it is answered."""
    pool = st.new_pages(24, PAGE)
    q = pool.new_sequence()
    q.append(ref.rows(st, 40, 1), ref.rows(st, 40, 2))
    step, rows = _step(st, pool, q, 8)
    _write(step, rows)
    kid = pool.fork([q])[0]
    was = _all([kid, q])
    with pytest.raises(StageError):
        step.write(0, rows[0], rows[1] + 1, rows[2])
    assert _same(was, _all([kid, q]))
    kid.free()
    step.write(0, rows[0], rows[1] + 1, rows[2])
    assert (q.read(0)[0][:, 40:] == 4).all()
    pool.free()


def test_steps_one_after_the_other(st):
    """Steps that take over the memory of freed ones while their work is queued, on two streams: each answers with its own plan."""
    pool = st.new_pages(200, PAGE)
    q = pool.new_sequence()
    q.append(ref.rows(st, 1000, 1), ref.rows(st, 1000, 2))
    seqs = pool.fork([q] * 12, [80 * (i + 1) for i in range(12)])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    query = torch.randn((1, 256), device="cuda").to(st.kv_dtype)
    rows = [torch.full((1, 128), 0.5, dtype=st.kv_dtype, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i, s in enumerate(seqs):
        stream = streams[i % 2]
        step = pool.new_step()
        step.plan([PagedRequest(s, 1)], stream=stream)
        step.write(0, query, *rows, stream=stream)
        outs.append(step.attend(0, query, stream=stream, out_dtype=torch.float32))
        step.free()
    torch.cuda.synchronize()
    for s, out in zip(seqs, outs):
        k, v = s.read(0)
        T = s.length
        o, a, s_abs, s_top = ref.attend(query.view(1, 4, 64), k, v, ref.sees(T - 1, 1), 0.125)
        bound = ref.attend_bound(o, a, s_abs, s_top, T, 64, st.kv_dtype, st.kv_dtype, torch.float32)
        assert ((out.view(1, 4, 64).double() - o).abs() <= bound).all()
    pool.free()
