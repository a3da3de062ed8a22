"""How many bits of a probability reach a row's result over pages: they follow from its
own request, not from what is batched with it."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref
from paper_2608_19147_amd import PagedRequest
from test_gpu_pages import A, _batch, _q, _write_raw

pytestmark = pytest.mark.gpu


def _bound(o, a, v_sum, s_abs, T, D, kv):
    """As ref.attend_bound for outputs in fp32, with a probability in two terms of kv: its relative error is the square of a half
    step; fp16's terms end at 2^-24 (half a step of that a probability, whose sum is at least 1)."""
    u = 2.0 ** -24
    p = ref.HALF_STEP[kv] ** 2 + 2 * ((D + 8) * u * s_abs[..., None] + 8 * u) + (4 * (T / 32) + 128) * u
    return a * p + (2.0 ** -25 * v_sum if kv == torch.float16 else 0.0) + o.abs() * u + 2.0 ** -126


def _check(st, out, seqs, q, P, n, see, skip=()):
    D, Hq = st.shape.head_dim, st.shape.n_q_heads
    row, worst = 0, 0.0
    for i, s in enumerate(seqs):
        k, v = s.read(0)
        if i not in skip:
            qi = q[row:row + n[i]].reshape(n[i], Hq, D)
            o, a, s_abs, _ = ref.attend(qi, k, v, see[i], 1 / math.sqrt(D))
            v_sum = v.double().abs().sum(1).repeat_interleave(Hq // v.shape[0], 0)[None]
            err = (out[row:row + n[i]].reshape(n[i], Hq, D).double() - o).abs()
            worst = max(worst, float((err / _bound(o, a, v_sum, s_abs, P[i] + n[i], D, st.kv_dtype)).max()))
        row += n[i]
    assert worst <= 1, worst


@pytest.mark.parametrize("shape", [dict(Hq=8, Hkv=2, D=128, kv="bf16"), dict(Hq=8, Hkv=2, D=64, kv="f16"), dict(Hq=16, Hkv=2, D=64, kv="bf16")])
@pytest.mark.parametrize("copies,n", [(1, 1), (20, 1), (64, 1), (1, 5), (7, 5), (3, 15), (12, 8)])
@pytest.mark.parametrize("mate", [0, 300])
def test_two_terms(shape, copies, n, mate):
    """Requests of up to 128 query vectors a kv head, alone, among sharers and beside a prompt: probabilities in two terms."""
    st = ref.make_stage(**shape)
    own = [11 + 3 * i for i in range(copies)] + ([40] if mate else [])
    news = [n] * copies + ([mate] if mate else [])
    pool, seqs, P = _batch(st, 16, [(A,)] * len(news), own, news)
    M = sum(news)
    masks = [None] * len(news)
    if n == 15:
        masks[0] = np.ones(P[0] + n, np.uint8)
        masks[0][[2, 30, 77]] = 0
    step = pool.new_step()
    step.plan([PagedRequest(s, m, mask=k) for s, m, k in zip(seqs, news, masks)])
    _write_raw(st, step, M, 5)
    q = _q(st, M, 6)
    out = step.attend(0, q, out_dtype=torch.float32)
    _check(st, out, seqs, q, P, news, [ref.sees(P[i], news[i], masks[i]) for i in range(len(news))], skip=(copies,) if mate else ())
    pool.free()
    st.close()
