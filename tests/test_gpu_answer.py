"""The last stage's operators where their bits, their loops and their order are
easily lost: small elements beside large ones, runs of equal logits, large norm
weights, borders between bins, and calls that follow a call that failed."""
import numpy as np
import pytest
import torch

import synth
from answer_ref import BLOCK, mx4_pack, sample
from gpu_cases import Pair
from paper_2608_19147_amd import Sampling

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def stage():
    p = Pair(synth.TINY, 350, with_oracle=False)
    yield p.gpu
    p.close()


@pytest.mark.parametrize("m,n,k", [(1, 500, 512), (16, 500, 4096), (64, 4096, 4096), (130, 500, 4096), (520, 1024, 1024)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16, torch.float32])
def test_small_elements_keep_their_bits(stage, m, n, k, out):
    """Each output is one element of x, 2^-8 below its block's largest: within 2^-18 of that one and a rounding of the
    output type, whatever that type is."""
    r = np.random.default_rng([351, m, k])
    x = torch.from_numpy((1 + r.integers(0, 128, (m, k)) / 128) * r.choice((-1.0, 1.0), (m, k)))
    x[:, ::BLOCK] *= 256
    x = x.to(torch.bfloat16)                                  # every value is one
    at = (1 + np.arange(n) * 37) % k
    codes = np.zeros((n, k), np.uint8)
    codes[np.arange(n), at] = 2                               # 1.0
    mat = stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.full((n, k // BLOCK), 127, dtype=torch.uint8), k)
    got = mat.product(x.cuda(), out_dtype=out).double().cpu().numpy()
    mat.free()
    ref = x.double().numpy()[:, at]
    top = np.abs(x.double().numpy()).reshape(m, -1, BLOCK).max(2)[:, at // BLOCK]
    tol = 2.0 ** -18 * top
    tol += (np.abs(ref) + tol) * torch.finfo(out).eps / 2
    assert (np.abs(got - ref) <= tol).all()


def _drawn(stage, z, rows, near_ok=0):
    """Rows (params, u) drawn from the one logits row z, each against the 64-bit form, unless that comes within 1e-9 of
    another outcome."""
    d = z.cuda()[None].repeat(len(rows), 1)
    tok, p = stage.sample(d, [Sampling(*q) for q, _ in rows], torch.tensor([u for _, u in rows], device="cuda"))
    near = 0
    for (q, u), t, pr in zip(rows, tok.tolist(), p.tolist()):
        rt, rp, gap = sample(z.double().numpy(), *q, u)
        if gap < 1e-9:
            near += 1
            continue
        assert t == rt, (q, u, t, rt)
        assert abs(pr - rp) <= rp * (2.0 ** -24 + 3e-8)
    assert near <= near_ok


@pytest.mark.parametrize("V", [30000, 262144, 262145, 1 << 20])
@pytest.mark.parametrize("n", [257, 300, 1024, 8192])
@pytest.mark.parametrize("rest", [-np.inf, -12.0])
def test_runs_of_equal_logits(stage, V, n, rest):
    """More equal neighbours than are ranked at once, at the row's start, across a power of two and at its end, beside
    nothing and beside many lower tokens."""
    rows = [((1.0, 0, 1.0, 0.0), 0.0), ((1.0, 0, 1.0, 0.0), 0.4375), ((1.0, 0, 1.0, 0.0), 0.9990234375), ((1.0, n // 2 + 1, 1.0, 0.0), 0.8125),
            ((1.0, 0, 0.5, 0.0), 0.9375), ((0.7, n + 5, 0.2531, 0.5), 0.5625)]
    for at in (0, 16384 - n // 3, V - n):
        z = torch.full((V,), rest)
        z[at:at + n] = 1.5
        _drawn(stage, z, rows, near_ok=1)


@pytest.mark.parametrize("power", [15, -13])
def test_head_norm_weight_range(power):
    """A final norm weight times a power of two gives the logits times that power, bit for bit: the normalized rows have no
    largest or smallest value that it could meet."""
    shape = synth.TINY
    fn, _ = synth.make_head(shape, 64, 352)
    x = synth.make_hidden(shape, 20, 353).cuda()
    w = torch.from_numpy(np.random.default_rng(354).standard_normal((1003, shape.hidden)) * 0.02).float().cuda()
    logits = []
    for s in (0, power):
        scaled = fn * 2.0 ** s
        assert torch.equal(scaled.double(), fn.double() * 2.0 ** s)
        p = Pair(shape, 355, with_oracle=False)
        p.gpu.attach_head_mx4(scaled.cuda(), *p.gpu.mx4_quantize(w))
        tok, pr, _, lg = p.gpu.head_top1(x, with_logits=True)
        assert torch.equal(tok.long(), lg.argmax(1)) and bool((pr > 0).all())
        logits.append(lg.double() * 2.0 ** -s)
        p.close()
    assert torch.equal(*logits)


U_NEAR = 1 - 2.0 ** -12


def _border_row(seed, at, V=1000):
    """A logits row whose first 100 tokens in rank, in bins 0 to 21 of 1/32, hold U_NEAR of its weight to within some units
    in the last place of a double (`at`, 0 to 63, moves it by them), with empty bins behind them.  Every logit is exact:
    a multiple of 2^-17."""
    r = np.random.default_rng([356, seed])
    weight = lambda b, f: np.rint(2.0 ** 36 * np.exp((f - 0.5) / 32)) * np.exp(-b / 32)  # noqa: E731
    bins, part = np.sort(r.integers(0, 22, 100)), r.integers(0, 4096, 100) / 4096
    bins[0] = 0
    ahead = weight(bins, part).sum()
    left, f, tail = ahead * (1 - U_NEAR) / U_NEAR + (at - 32) * 0.5 * np.spacing(ahead), 4095 / 4096, []
    for b in range(300, 1024):
        n = int(left / weight(b, f))
        left -= n * weight(b, f)
        tail += [b] * n
    x = np.concatenate([-np.sort(bins - part), f - np.array(tail)])
    z = np.full(V, -np.inf)
    z[:len(x)] = x / 32
    return z


@pytest.mark.parametrize("V", [1000, 30000])
def test_draw_between_bins(stage, V):
    """A draw at the border between two bins that have empty ones in between, one unit in the last place after the other: the
    last token ahead of it or the first behind, never none."""
    for seed in range(24):
        z = np.stack([_border_row(seed, at, V) for at in range(64)])
        assert np.array_equal(z, z.astype(np.float32))
        tok, p = stage.sample(torch.from_numpy(z).float().cuda(), Sampling(), torch.full((64,), U_NEAR, device="cuda"))
        for row, t, q in zip(z, tok.tolist(), p.tolist()):
            assert t in (99, 100)
            w = np.exp(row - row[0])
            assert abs(q - w[t] / w.sum()) <= q * (2.0 ** -24 + 3e-8)


def test_head_row_without_a_token():
    """A hidden row with a NaN or an infinity has no token through an MXFP4 head: -1, probability 0, from both calls; the
    rows beside it have theirs."""
    shape = synth.TINY
    p = Pair(shape, 357, with_oracle=False)
    fn, _ = synth.make_head(shape, 64, 357)
    w = torch.from_numpy(np.random.default_rng(358).standard_normal((1003, shape.hidden)) * 0.02).float().cuda()
    p.gpu.attach_head_mx4(fn.cuda(), *p.gpu.mx4_quantize(w))
    x = synth.make_hidden(shape, 4, 359)
    want = [t.tolist() for t in p.gpu.head_top1(x.cuda())[:3]]
    x[1, 7], x[2, 0] = float("nan"), float("inf")
    tok, pr, top, lg = p.gpu.head_top1(x.cuda(), with_logits=True)
    assert bool(torch.isnan(lg[1:3]).all())
    assert tok.tolist() == [want[0][0], -1, -1, want[0][3]] and pr.tolist() == [want[1][0], 0.0, 0.0, want[1][3]]
    assert top.tolist() == [want[2][0], -np.inf, -np.inf, want[2][3]]
    tok, pr, _ = p.gpu.head_sample(x.cuda(), Sampling(), torch.full((4,), 0.5, device="cuda"))
    assert tok[1:3].tolist() == [-1, -1] and pr[1:3].tolist() == [0.0, 0.0] and min(tok[0].item(), tok[3].item()) >= 0
    p.close()


def test_head_rows_alike():
    """A row's logits through an MXFP4 head, bit for bit, whether it comes alone, in a verify or among 64 rows (K is long
    enough here for the rows' number to matter to how a product splits it)."""
    shape = synth.StageShape("alike", 16, n_layers=1, hidden=1024, n_q_heads=2, n_kv_heads=1, head_dim=128, ffn=512)
    p = Pair(shape, 360, with_oracle=False)
    fn, _ = synth.make_head(shape, 64, 360)
    w = torch.from_numpy(np.random.default_rng(361).standard_normal((1000, shape.hidden)) * 0.02).float().cuda()
    p.gpu.attach_head_mx4(fn.cuda(), *p.gpu.mx4_quantize(w))
    x = synth.make_hidden(shape, 64, 362).cuda()
    u = torch.from_numpy(np.random.default_rng(363).random(64).astype(np.float32)).cuda()
    tok, pr, lg = p.gpu.head_sample(x, Sampling(0.9, 0, 0.95), u, with_logits=True)
    for a, b in ((0, 1), (7, 27), (20, 53), (63, 64)):
        t, q, z = p.gpu.head_sample(x[a:b].clone(), Sampling(0.9, 0, 0.95), u[a:b].clone(), with_logits=True)
        assert torch.equal(z, lg[a:b]) and torch.equal(t, tok[a:b]) and torch.equal(q, pr[a:b])
    p.close()


@pytest.mark.parametrize("value", [0.0, float(np.finfo(np.float32).min), float(np.finfo(np.float32).max), -1e-45])
def test_equal_extremes_by_index(stage, value):
    """300 equal logits at the ends of the range, some -inf ones between them: u of them by count, exactly."""
    z = torch.full((400,), -np.inf)
    at = np.sort(np.random.default_rng(364).permutation(400)[:300])
    z[torch.from_numpy(at)] = value
    us = np.array([0.0, 1 / 300, 0.1, 1 / 3, 0.5, 0.7, 0.99, 1 - 2.0 ** -24], np.float32)
    tok, p = stage.sample(z.cuda()[None].repeat(len(us), 1), Sampling(), torch.from_numpy(us).cuda())
    assert tok.tolist() == [at[int(float(u) * 300)] for u in us]
    assert (p.double() - 1 / 300).abs().max().item() <= 2.0 ** -24 / 300


@pytest.mark.parametrize("V", [4, 11, 36, 700, 9000, 30000, 128256])
def test_few_kept(stage, V):
    """Few tokens kept by top_k, cut by top_p (and min_p) over bins that lie apart: the bins in which the cuts and the draw
    can fall lie within each other."""
    r = np.random.default_rng([365, V])
    for _ in range(6):
        z = torch.from_numpy(r.standard_normal(V) * np.exp(r.uniform(-2, 2))).float()
        rows = [((float(r.choice([0.3, 0.7, 1.0, 1.5])), int(r.choice([2, 2, 3, 5, 8])), float(r.choice([0.5, 0.9, 0.95, 0.999])),
                  float(r.choice([0, 0, 0.01, 0.05]))), float(np.float32(r.random()))) for _ in range(64)]
        _drawn(stage, z, rows, near_ok=1)


@pytest.mark.parametrize("V", [20, 9000, 30000])
@pytest.mark.parametrize("scale", [1e3, 1e12, 1e30, 3e38])
def test_large_logits(stage, V, scale):
    """Logits far beyond the numbers that have fractions, some of them equal: the first ones share the weight by count, at
    every temperature."""
    r = np.random.default_rng([366, V])
    z = r.standard_normal(V).clip(-1, 0.8)
    z[r.permutation(V)[: V // 4]] = 0.9
    z = torch.from_numpy((z * scale).astype(np.float32))
    first = np.flatnonzero(z.numpy() == z.numpy().max())
    rows = [(t, p, m, float(np.float32(u))) for t in (1e-3, 0.3, 0.7, 1.0, 30.0) for p, m in ((1.0, 0.0), (0.5, 0.0), (1.0, 1.0)) for u in (0.0, 0.3, 0.99)]
    if scale < 1e4:
        rows = [q for q in rows if q[0] < 0.5]                # so that the other tokens weigh nothing
    tok, p = stage.sample(z.cuda()[None].repeat(len(rows), 1), [Sampling(t, 0, q, m) for t, q, m, _ in rows], torch.tensor([u for *_, u in rows], device="cuda"))
    for (t, q, m, u), got, pr in zip(rows, tok.tolist(), p.tolist()):
        kept = int(np.ceil(q * len(first)))
        assert got == first[int(u * kept)] and abs(pr - 1 / kept) <= 2.0 ** -24 / kept, (t, q, m, u, got, pr)


def test_infinite_logits(stage):
    """+inf ranks as the largest finite number, however that is scaled."""
    for dtype in (torch.float16, torch.bfloat16, torch.float32):
        z = torch.zeros((15, 300), dtype=dtype)
        z[:, 7::10] = np.inf
        ts = [1e-3, 0.3, 0.7, 1.5, 30.0]
        us = [0.0, 0.41, 0.97]
        tok, p = stage.sample(z.cuda(), [Sampling(t) for t in ts for _ in us], torch.tensor(us * 5, device="cuda"))
        assert tok.tolist() == [7 + 10 * int(float(np.float32(u)) * 30) for u in us] * 5
        assert (p.double() - 1 / 30).abs().max().item() <= 2.0 ** -24 / 30


@pytest.mark.parametrize("spread", [0.5, 50.0, 5000.0])
def test_min_p_one(stage, spread):
    """min_p 1 keeps the first token (and its equals) at every temperature."""
    r = np.random.default_rng([367, int(spread)])
    for V in (30, 9000, 40000):
        z = torch.from_numpy(r.standard_normal((40, V)) * spread).half()
        ts = [(1e-3, 0.3, 0.7, 1.1, 30.0)[i % 5] for i in range(40)]
        tok, p = stage.sample(z.cuda(), [Sampling(t, 0, 1.0, 1.0) for t in ts], torch.full((40,), 0.5, device="cuda"))
        for row, t, q in zip(z.double().numpy(), tok.tolist(), p.tolist()):
            first = np.flatnonzero(row == row.max())
            assert t == first[len(first) // 2] and abs(q - 1 / len(first)) <= 2.0 ** -24
