"""Sampling against its 64-bit form: the token has to be the same wherever no cut
and no draw of the 64-bit form comes within 1e-9 of the kept weight of another
outcome (the kernel's sums are exact to 2^-36 a token and 2^-50 a bin, and leave
out at most 1.4e-8 of the weight at its far end, which no u or top_p reaches);
p within fp32's rounding and those 1.4e-8."""
import numpy as np
import pytest
import torch

import synth
from answer_ref import sample
from gpu_cases import Pair
from paper_2608_19147_amd import Sampling, StageError

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
MIX = [(1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.0), (1.0, 0, 0.95, 0.0), (0.9, 0, 1.0, 0.05), (0.0, 5, 0.5, 0.5), (1.3, 1000, 0.98, 0.02),
       (0.6, 20, 0.95, 0.01), (1.0, 1, 1.0, 0.0), (5.0, 0, 0.999, 0.0), (0.05, 0, 1.0, 0.0), (1000.0, 0, 1.0, 0.0), (1.0, 3000, 1.0, 0.0),
       (1.0, 0, 1e-6, 0.0), (1.0, 0, 1.0, 1.0), (2.0, 70000, 0.9999, 1e-5), (1.0, 1 << 30, 1.0, 1e-30), (1e-3, 0, 0.5, 0.0)]


@pytest.fixture(scope="module")
def stage():
    p = Pair(synth.TINY, 330, with_oracle=False)
    yield p.gpu
    p.close()


def _logits(M, V, seed, spread=2.0):
    r = np.random.default_rng([seed, M, V])
    z = r.standard_normal((M, V)) * spread - 3
    for m in range(M):
        z[m, r.integers(0, V, min(V, 12))] += r.random(min(V, 12)) * 10
    return z


def _check(stage, z, params, u, near_ok=0):
    """z: CPU tensor [M, V] or a view of one.  At most near_ok rows may be too near a border to be told."""
    z = z if isinstance(z, torch.Tensor) else torch.from_numpy(np.asarray(z)).float()
    M = z.shape[0]
    d = z.cuda() if z._base is None else z._base.cuda().as_strided(z.shape, z.stride(), z.storage_offset())
    u = np.asarray(u, np.float32)
    tok, p = stage.sample(d, [Sampling(*q) for q in params], torch.from_numpy(u).cuda())
    tok, p = tok.cpu().numpy(), p.cpu().numpy().astype(np.float64)
    near = 0
    for m in range(M):
        t, q, gap = sample(z[m].double().numpy(), *params[m], u[m])
        if gap < 1e-9:
            near += 1
            continue
        assert tok[m] == t, (m, params[m], u[m], tok[m], t)
        assert abs(p[m] - q) <= q * (2.0 ** -24 + 3e-8), (m, params[m], p[m], q)
    assert near <= near_ok
    return tok, p


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 1000, 1025, 4097, 50257, 128256])
def test_sample(stage, V, dtype):
    M = len(MIX)
    u = np.random.default_rng(V).random(M)
    _check(stage, torch.from_numpy(_logits(M, V, 1)).to(DT[dtype]), MIX, u, near_ok=1)


@pytest.mark.parametrize("V", [8191, 8192, 8193, 16384, 16391, 24576, 24577])
def test_sample_slices(stage, V):
    """Around the ends of the slices that are counted apart, and of the rows that one workgroup holds; at last equal logits,
    which fill one bin of every slice."""
    M = len(MIX)
    u = np.random.default_rng(V + 1).random(M)
    _check(stage, torch.from_numpy(_logits(M, V, 11)).float(), MIX, u, near_ok=1)
    _check(stage, torch.from_numpy(_logits(M, V, 12, spread=0.3)).bfloat16(), MIX, u, near_ok=1)
    us = [0.0, 0.5, 1 - 2.0 ** -24]
    tok, p = stage.sample(torch.full((3, V), -1.5, device="cuda"), Sampling(), torch.tensor(us, dtype=torch.float32, device="cuda"))
    assert tok.tolist() == [int(u * V) for u in us]
    assert (p.double() - 1.0 / V).abs().max().item() <= 2.0 ** -24 / V


@pytest.mark.parametrize("spread", [0.01, 0.3, 8.0, 100.0])
def test_spreads(stage, spread):
    """From almost equal logits (every token in few bins) to ones far apart."""
    M = len(MIX)
    u = np.random.default_rng(7).random(M)
    z = np.random.default_rng([8, int(spread * 100)]).standard_normal((M, 30011)) * spread
    _check(stage, z, MIX, u, near_ok=1)


@pytest.mark.parametrize("V", [5, 2048, 2049, 100000])
def test_equal_logits(stage, V):
    """All equal: u and top_p count tokens, exactly, and the lowest indices come first."""
    us = [0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 1.0 / 3]
    params = [(1.0, 0, 1.0, 0.0), (1.0, 0, 0.5, 0.0), (2.0, V // 2 + 1, 1.0, 0.0), (1.0, 0, 1.0, 1.0)]
    rows = [(q, u) for q in params for u in us]
    z = np.full((len(rows), V), 1.3)
    tok, _ = _check(stage, z, [q for q, _ in rows], [u for _, u in rows])
    for (q, u), t in zip(rows, tok):
        kept = int(np.ceil(0.5 * V)) if q[2] == 0.5 else q[1] or V
        assert t == int(np.float32(u) * float(kept))


def test_two_levels(stage):
    """Many equal tokens at two heights: the place is found by index within a height."""
    z = np.full((6, 60000), 0.7)
    z[:, 1000:31000] = 1.2
    u = [0.0, 0.3, 0.6, 0.9, 0.999, 0.7]
    _check(stage, z, [(1.0, 0, 1.0, 0.0)] * 3 + [(0.5, 45000, 0.95, 0.0), (1.0, 45000, 1.0, 0.0), (1.0, 0, 1.0, 0.61)], u)


def test_masked(stage):
    """-inf and NaN are never drawn, +inf ranks as the largest number, -0 equals 0; a row with nothing to draw gives -1."""
    inf, nan = np.inf, np.nan
    low = float(np.finfo(np.float32).min)
    z = np.full((9, 300), -inf)
    z[1] = nan
    z[2, 77] = -5.0
    z[3, [10, 250]] = inf
    z[3, 20] = 3.0
    z[4, ::2] = np.random.default_rng(3).standard_normal(150)
    z[4, 1::2] = nan
    z[5] = low
    z[6] = low
    z[6, 123] = 1.0
    z[7, 5], z[7, 9] = -0.0, 0.0
    z[8, 40], z[8, 41] = 3e38, -3e38
    for u in (0.0, 0.5, 0.99):
        tok, p = _check(stage, z, [(1.0, 0, 1.0, 0.0)] * 9, [u] * 9)
        assert tok[0] == -1 and tok[1] == -1 and p[0] == 0 and p[1] == 0
        assert tok[2] == 77 and p[2] == 1
        assert tok[3] == (10 if u < 0.5 else 250) and p[3] == 0.5
        assert tok[4] % 2 == 0
        assert tok[5] == int(u * 300) or abs(u * 300 - round(u * 300)) < 1e-4
        assert tok[6] == 123
        assert tok[7] == (5 if u < 0.5 else 9)
        assert tok[8] == 40


@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 8), (8, 0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(stage, dtype, offset, pad):
    V = 5003
    wide = torch.from_numpy(_logits(9, V + offset + pad, 4)).to(DT[dtype])
    wide[:, :offset] = 50.0                                  # what is beside the rows would win
    wide[:, offset + V:] = 50.0
    _check(stage, wide[:, offset:offset + V], MIX[:9], np.random.default_rng(5).random(9), near_ok=1)


def test_u_outside(stage):
    """u below 0 counts as 0, u of 1 and more as the largest number below 1, NaN as 0."""
    z = torch.from_numpy(_logits(1, 500, 6)).float().repeat(5, 1).cuda()
    tok, _ = stage.sample(z, Sampling(), torch.tensor([0.0, -1.0, 1 - 2.0 ** -24, 7.0, float("nan")], device="cuda"))
    tok = tok.tolist()
    assert tok[0] == tok[1] == tok[4] and tok[2] == tok[3]


@pytest.mark.parametrize("M", [1, 2, 63, 64])
def test_rows_are_independent(stage, M):
    """A row's token and probability, bit for bit, whatever rows come with it and however often it is asked."""
    z = torch.from_numpy(_logits(64, 40007, 9)).float().cuda()[:M]
    u = torch.from_numpy(np.random.default_rng(10).random(64).astype(np.float32)).cuda()[:M]
    params = [Sampling(*MIX[i % len(MIX)]) for i in range(M)]
    tok, p = stage.sample(z, params, u)
    again = stage.sample(z, params, u)
    assert torch.equal(tok, again[0]) and torch.equal(p, again[1])
    for m in {0, M // 2, M - 1}:
        t1, p1 = stage.sample(z[m:m + 1], params[m], u[m:m + 1].clone())
        assert torch.equal(t1, tok[m:m + 1]) and torch.equal(p1, p[m:m + 1])


def test_frequencies(stage):
    """Draws at 4096 evenly spread u land on each token in proportion to its weight, to one draw."""
    z = torch.tensor([[0.0, 1.0, -1.0, 2.0, 0.5]])
    n, got = 4096, np.zeros(5)
    for s in range(0, n, 64):
        u = ((torch.arange(s, s + 64) + 0.5) / n).float()
        tok, _ = stage.sample(z.repeat(64, 1).cuda(), Sampling(0.8), u.cuda())
        got += np.bincount(tok.cpu().numpy(), minlength=5)
    w = np.exp(z[0].double().numpy() / float(np.float32(0.8)))
    assert (np.abs(got - n * w / w.sum()) <= 1.0).all()


def test_streams(stage):
    """Calls on several streams at once give what they give alone."""
    zs = [torch.from_numpy(_logits(m, v, 20 + m)).float().cuda() for m, v in ((64, 128256), (1, 999), (20, 50257), (3, 128256))]
    us = [torch.from_numpy(np.random.default_rng(m.shape[0]).random(m.shape[0]).astype(np.float32)).cuda() for m in zs]
    ps = [[Sampling(*MIX[i % len(MIX)]) for i in range(z.shape[0])] for z in zs]
    want = [stage.sample(*a) for a in zip(zs, ps, us)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in zs]
    for _ in range(5):
        got = [stage.sample(*a, stream=s) for a, s in zip(zip(zs, ps, us), streams)]
        torch.cuda.synchronize()
        for (a, b), (c, d) in zip(got, want):
            assert torch.equal(a, c) and torch.equal(b, d)


def test_refusals(stage):
    z, u = torch.zeros((2, 10), device="cuda"), torch.zeros(2, device="cuda")
    for q in (Sampling(-1.0), Sampling(1e-4), Sampling(float("nan")), Sampling(1.0, -1), Sampling(1.0, 0, 0.0), Sampling(1.0, 0, 1.5),
              Sampling(1.0, 0, 1.0, -0.1), Sampling(1.0, 0, 1.0, 2.0), Sampling(1.0, 0, float("nan"))):
        with pytest.raises(StageError) as ei:
            stage.sample(z, [Sampling(), q], u)
        assert ei.value.code == -1 and "row 1" in str(ei.value)
    with pytest.raises(StageError) as ei:
        stage.sample(torch.zeros((65, 10), device="cuda"), Sampling(), torch.zeros(65, device="cuda"))
    assert ei.value.code == -3
    for bad in (lambda: stage.sample(z.cpu(), Sampling(), u), lambda: stage.sample(z.double(), Sampling(), u),
                lambda: stage.sample(z.t(), Sampling(), torch.zeros(10, device="cuda")), lambda: stage.sample(z, Sampling(), u.double()),
                lambda: stage.sample(z, [Sampling()], u), lambda: stage.sample(z, Sampling(), u[:1]), lambda: stage.sample(z[:0], Sampling(), u[:0])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(StageError) as ei:
        stage.head_sample(torch.zeros((1, synth.TINY.hidden), dtype=stage.act_dtype, device="cuda"), Sampling(), u[:1])
    assert ei.value.code == -1


def test_head_sample_int4():
    """stage_head_sample through the INT4 head: the tokens that stage_sample draws from the logits that came with them."""
    shape = synth.TINY
    p = Pair(shape, 340, with_oracle=False)
    p.gpu.attach_head(*synth.make_head(shape, 1000, 340))
    M = len(MIX)
    x = synth.make_hidden(shape, M, 341).cuda()
    u = np.random.default_rng(342).random(M).astype(np.float32)
    ud = torch.from_numpy(u).cuda()
    tok, pr, lg = p.gpu.head_sample(x, [Sampling(*q) for q in MIX], ud, with_logits=True)
    tok2, pr2, none = p.gpu.head_sample(x, [Sampling(*q) for q in MIX], ud)
    assert none is None and torch.equal(tok, tok2) and torch.equal(pr, pr2)
    _, _, _, lg2 = p.gpu.head_top1(x, with_logits=True)
    assert torch.equal(lg, lg2)
    got, _ = _check(p.gpu, lg.cpu(), MIX, u, near_ok=1)
    assert np.array_equal(got, tok.cpu().numpy())
    p.close()


def test_largest_vocabulary(stage):
    """2^20 tokens: every slice, and equal logits in all of them."""
    V = 1 << 20
    M = 6
    u = np.random.default_rng(71).random(M)
    _check(stage, torch.from_numpy(_logits(M, V, 72)).float(), MIX[:M], u, near_ok=1)
    us = [0.0, 0.3125, 1 - 2.0 ** -20]
    tok, p = stage.sample(torch.zeros((3, V), device="cuda", dtype=torch.bfloat16), Sampling(), torch.tensor(us, device="cuda"))
    assert tok.tolist() == [int(v * V) for v in us] and p.tolist() == [2.0 ** -20] * 3


def test_other_device_refused(stage, monkeypatch):
    """Tensors on a device that is not the stage's (the stage is made to say that its own is another)."""
    z, u = torch.zeros((1, 10), device="cuda"), torch.zeros(1, device="cuda")
    t = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    codes, scales = stage.mx4_quantize(torch.ones((2, 32), device="cuda"))
    mat = stage.mx4_matrix(codes, scales, 32)
    monkeypatch.setattr(stage, "device_index", stage.device_index + 1)
    for call in (lambda: stage.sample(z, Sampling(), u), lambda: stage.tree_accept(t, t, t), lambda: stage.mx4_quantize(z),
                 lambda: stage.mx4_dequantize(codes, scales, 32), lambda: stage.mx4_matrix(codes, scales, 32),
                 lambda: mat.product(torch.ones((1, 32), device="cuda"), 4),
                 lambda: stage.head_sample(torch.zeros((1, synth.TINY.hidden), dtype=stage.act_dtype, device="cuda"), Sampling(), u)):
        with pytest.raises(ValueError, match="the stage is on"):
            call()
    mat.free()


def test_capture(stage):
    """A row that one workgroup holds is sampled in a graph, with the logits and u of each replay; longer rows, which use
    the stage's workspace, refuse."""
    M, V = 5, 20000
    params = [Sampling(*q) for q in MIX[:M]]
    z, u = torch.zeros((M, V), device="cuda"), torch.zeros(M, device="cuda")
    wide = torch.from_numpy(_logits(2, 30000, 80)).float().cuda()
    stage.sample(z, params, u)
    stage.sample(wide, Sampling(), u[:2].clone())
    u2 = torch.zeros(2, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tok, p = stage.sample(z, params, u)
        with pytest.raises(StageError) as ei:
            stage.sample(wide, Sampling(), u2)
        assert ei.value.code == -7
    for i in range(3):
        z.copy_(torch.from_numpy(_logits(M, V, 81 + i)).float())
        u.copy_(torch.from_numpy(np.random.default_rng(90 + i).random(M).astype(np.float32)))
        stage.sample(wide, Sampling(), u2)
        g.replay()
        eager = stage.sample(z, params, u)
        torch.cuda.synchronize()
        assert torch.equal(tok, eager[0]) and torch.equal(p, eager[1])
