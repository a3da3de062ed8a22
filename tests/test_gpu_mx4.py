"""MXFP4 rounding, products and the MXFP4 head against their 64-bit forms.

Codes and scale bytes are whole numbers and have to be equal; values are exact
or one rounding of the output type away.  A product may differ by
  * what the activation's terms leave: 2^-18 of the largest magnitude of the
    element's block (2^-14 for bf16 rows with 16-bit results, 0 at act_bits 4),
    times |w|;
  * the fp32 sums: one group of 8 products and one addition a step, each at most
    2^-23 of the sum of magnitudes so far: 2^-23 (terms k / 8 + 8) sum |x w|
    (the 8 covers sums of parts of k);
  * the rounding of the result: half a step, eps / 2, or half the smallest
    subnormal of fp16."""
import numpy as np
import pytest
import torch

import oracle
import synth
from answer_ref import BLOCK, mx4_encode, mx4_pack, mx4_values
from gpu_cases import Pair, host
from paper_2608_19147_amd import Sampling, StageError

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def stage():
    p = Pair(synth.TINY, 300, with_oracle=False)
    yield p.gpu
    p.close()


def _rows(m, k, seed, dtype, wide=1.0):
    r = np.random.default_rng([seed, m, k])
    x = r.standard_normal((m, k)) * np.exp2(r.integers(-3, 4, (m, k)) * wide)
    return torch.from_numpy(x).to(DT[dtype])


def _edge_rows(dtype):
    """Ties between neighbouring codes, saturation, zeros, signs, subnormals and non-finite values, one kind a block."""
    top = 6.0
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    x = np.zeros((8, 70))
    x[0, :32] = [top] + ties + [-t for t in ties] + [0.0] * 17
    x[0, 32:64] = np.linspace(-7.99, 7.99, 32)
    x[1, :32] = 0.0
    x[1, 32:64] = -0.0
    x[2, :32] = np.nan
    x[2, 40] = np.inf
    x[3, 5] = -np.inf
    x[3, 32:64] = 1.0
    tiny = float(torch.finfo(DT[dtype]).tiny)
    x[4, :32] = tiny * np.linspace(0, 1, 32)
    x[4, 32:64] = tiny * np.arange(32)
    x[5] = float(torch.finfo(DT[dtype]).max) * np.linspace(-1, 1, 70)
    x[6, ::3] = 2.0 ** -14
    x[7, 64:] = [4.0, 7.0, 7.5, -7.0, 0.3, -0.2]
    return torch.from_numpy(x).to(DT[dtype])


def _check_quantize(stage, x):
    """x: a CPU tensor [m, k], or a view of one; the device copy keeps its strides."""
    base = x if x._base is None else x._base
    d = base.cuda()
    d = d if x._base is None else d.as_strided(x.shape, x.stride(), x.storage_offset())
    codes, scales = stage.mx4_quantize(d)
    c, s = mx4_encode(x.double().numpy())
    assert np.array_equal(scales.cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), mx4_pack(c))
    return codes, scales, c, s


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,k", [(1, 1), (1, 2), (3, 31), (2, 32), (5, 33), (4, 64), (1, 257), (7, 693), (2, 4096), (130, 72)])
def test_quantize(stage, dtype, m, k):
    _check_quantize(stage, _rows(m, k, 1, dtype))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_quantize_edges(stage, dtype):
    _check_quantize(stage, _edge_rows(dtype))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 5), (8, 8), (4, 4)])
def test_quantize_strides(stage, dtype, offset, pad):
    """Rows inside wider ones, at every alignment of their start."""
    wide = _rows(6, 200 + offset + pad, 2, dtype)
    _check_quantize(stage, wide[:, offset:offset + 200])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_dequantize_every_code(stage, dtype):
    """All 256 scale bytes with all 16 codes, and ragged rows."""
    codes = np.tile(np.arange(16, dtype=np.uint8), (256, 4))[:, :63]
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 2, 1)
    out = stage.mx4_dequantize(torch.from_numpy(mx4_pack(codes)).cuda(), torch.from_numpy(scales).cuda(), 63, DT[dtype]).cpu()
    with np.errstate(over="ignore"):
        ref = torch.from_numpy(mx4_values(codes, scales)).float().to(DT[dtype])      # every value is exact in fp32, or past it
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    ok = ~torch.isnan(ref)
    assert torch.equal(out[ok], ref[ok])


@pytest.mark.parametrize("dtype,m,k", [("bf16", 1030, 16389), ("f16", 1030, 16389), ("f32", 1030, 8197)])
def test_round_trip_large(stage, dtype, m, k):
    """More values than the caches hold, odd rows: those of single rows on their own."""
    g = torch.Generator(device="cuda").manual_seed(k)
    x = torch.randn((m, k), device="cuda", generator=g).to(DT[dtype])
    codes, scales = stage.mx4_quantize(x)
    out = stage.mx4_dequantize(codes, scales, k, DT[dtype])
    for r in (0, 1, m // 2, m - 1):
        c, s, _, _ = _check_quantize(stage, x[r:r + 1].cpu())
        assert torch.equal(codes[r:r + 1].cpu(), c.cpu()) and torch.equal(scales[r:r + 1].cpu(), s.cpu())
        assert torch.equal(out[r:r + 1].cpu(), stage.mx4_dequantize(c.cuda(), s.cuda(), k, DT[dtype]).cpu())


@pytest.mark.parametrize("m,k", [(1, 1), (3, 40), (2, 4096), (33, 129)])
def test_round_trip(stage, m, k):
    x = _rows(m, k, 3, "bf16")
    codes, scales, c, s = _check_quantize(stage, x)
    out = stage.mx4_dequantize(codes, scales, k, torch.bfloat16)
    assert np.array_equal(out.double().cpu().numpy(), mx4_values(c, s))


def _weights(n, k, seed):
    r = np.random.default_rng([seed, n, k])
    codes = r.integers(0, 16, (n, k)).astype(np.uint8)
    scales = r.integers(110, 124, (n, -(-k // BLOCK))).astype(np.uint8)
    return codes, scales


def _product(x, codes, scales, act, out_dtype):
    """(reference, tolerance) float64 of a product."""
    w = mx4_values(codes, scales)
    xd = x.double().numpy()
    k = xd.shape[1]
    if act == 4:
        xd = mx4_values(*mx4_encode(xd))
    nb = -(-k // BLOCK)
    top = np.abs(np.pad(xd, ((0, 0), (0, nb * BLOCK - k)))).reshape(len(xd), nb, BLOCK).max(2)
    terms = 1 if act == 4 else 2 if x.dtype == torch.bfloat16 and out_dtype != torch.float32 else 3
    left = 0.0 if act == 4 else 2.0 ** -14 if terms == 2 else 2.0 ** -18
    ref = xd @ w.T
    tol = left * np.repeat(top, BLOCK, 1)[:, :k] @ np.abs(w).T + 2.0 ** -23 * (terms * k / 8 + 8) * (np.abs(xd) @ np.abs(w).T)
    f = torch.finfo(out_dtype)
    return ref, tol + (np.abs(ref) + tol) * f.eps / 2 + f.tiny * f.eps / 2


def _check_product(stage, m, n, k, dtype, act, out, seed=4, pad=0):
    codes, scales = _weights(n, k, seed)
    x = _rows(m, k + pad, seed + 1, dtype)[:, :k]
    mat = stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.from_numpy(scales), k)
    d = x._base.cuda()[:, :k] if pad else x.contiguous().cuda()
    got = mat.product(d, act, DT[out]).double().cpu().numpy()
    ref, tol = _product(x, codes, scales, act, DT[out])
    err = np.abs(got - ref)
    print(f"m {m} n {n} k {k} {dtype} act {act} -> {out}: worst error {np.max(err / tol):.3f} of the tolerance")
    assert (err <= tol).all()
    mat.free()


SIZES = [(1, 1, 1), (1, 64, 32), (1, 200, 693), (2, 65, 33), (5, 130, 257), (15, 63, 512), (16, 257, 1024), (17, 64, 255), (31, 1001, 64),
         (32, 96, 2048), (33, 129, 300), (64, 500, 688), (65, 70, 256), (130, 260, 320), (257, 513, 96), (300, 1030, 1100)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype,act,out", [("bf16", 16, "bf16"), ("bf16", 16, "f32"), ("f16", 16, "f16"), ("f16", 16, "f32"),
                                           ("bf16", 4, "bf16"), ("f32", 4, "f32"), ("f16", 4, "bf16")])
def test_product(stage, m, n, k, dtype, act, out):
    _check_product(stage, m, n, k, dtype, act, out)


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (8, 512, 14336), (20, 8192, 4096), (64, 4096, 4096), (200, 1024, 8192), (512, 2048, 1024)])
@pytest.mark.parametrize("dtype,act,out", [("bf16", 16, "bf16"), ("f16", 16, "f32"), ("bf16", 4, "f16")])
def test_product_large(stage, m, n, k, dtype, act, out):
    _check_product(stage, m, n, k, dtype, act, out)


# Row tiles of every size, K whole and split, with the short and the long form of the loop.
TILES = {"bf16": [(1521, 20251, 65), (1459, 64, 14310), (237, 24956, 1092), (132, 26514, 2033), (1160, 1679, 4147)],
         "f16": [(622, 24412, 66), (1755, 68, 9007), (131, 27946, 1752), (651, 9662, 796), (1672, 261, 10981)],
         "4 bits": [(1526, 9690, 65), (1157, 118, 13128), (568, 7255, 2176), (76, 11101, 12573), (1803, 7009, 2326)]}


@pytest.mark.parametrize("kind,m,n,k", [(kind, *size) for kind, sizes in TILES.items() for size in sizes])
def test_product_tiles(stage, kind, m, n, k):
    """Every output against 64 bits, on the device for its speed; rows of x and of the result inside wider ones."""
    act, dtype, out = (4, torch.bfloat16, torch.bfloat16) if kind == "4 bits" else (16, DT[kind], DT[kind])
    g = torch.Generator(device="cuda").manual_seed(m * 7 + k)
    nb = -(-k // BLOCK)
    codes = torch.randint(0, 16, (n, k), device="cuda", generator=g, dtype=torch.uint8)
    scales = torch.randint(110, 124, (n, nb), device="cuda", generator=g, dtype=torch.uint8)
    even = torch.nn.functional.pad(codes, (0, k % 2))
    mat = stage.mx4_matrix(even[:, 0::2] | even[:, 1::2] << 4, scales, k)
    x = (torch.randn((m, k + 3), device="cuda", generator=g) * torch.exp2(torch.randint(-3, 4, (m, k + 3), device="cuda", generator=g))).to(dtype)
    x = x[:, :k]
    got = mat.product(x, act, out).double()
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    w = torch.cat([grid, -grid])[codes.int()] * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, 1)[:, :k]
    xd = x.double() if act == 16 else stage.mx4_dequantize(*stage.mx4_quantize(x), k, torch.float32).double()
    top = torch.nn.functional.pad(xd.abs(), (0, nb * BLOCK - k)).view(m, nb, BLOCK).amax(2).repeat_interleave(BLOCK, 1)[:, :k]
    terms, left = {"bf16": (2, 2.0 ** -14), "f16": (3, 2.0 ** -18), "4 bits": (1, 0.0)}[kind]
    wt = w.t().contiguous()
    ref = xd @ wt
    tol = (left * top + 2.0 ** -23 * (terms * k / 8 + 8) * xd.abs()) @ wt.abs_()
    f = torch.finfo(out)
    tol += (ref.abs() + tol) * (f.eps / 2) + f.tiny * f.eps / 2
    worst = float(((got - ref).abs() / tol).max())
    print(f"{kind} m {m} n {n} k {k}: worst error {worst:.3f} of the tolerance")
    assert worst <= 1.0
    mat.free()


@pytest.mark.parametrize("m", [20, 64])
def test_capture_without_workspace(stage, m):
    """Up to 64 rows are captured also where an eager call takes the stage's workspace, and need none of it on replay."""
    n, k = 4200, 4100
    codes, scales = _weights(n, k, 23)
    mat = stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.from_numpy(scales), k)
    x = _rows(m, k, 24, "bf16").cuda()
    mat.product(x)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o = mat.product(x)
    for i in range(3):
        new = _rows(m, k, 25 + i, "bf16")
        x.copy_(new)
        eager = mat.product(x).double().cpu().numpy()
        g.replay()
        mat.product(x.flip(0))
        torch.cuda.synchronize()
        ref, tol = _product(new, codes, scales, 16, torch.bfloat16)
        assert (np.abs(o.double().cpu().numpy() - ref) <= tol).all()
        assert (np.abs(eager - ref) <= tol).all()
    mat.free()


def test_product_passes(stage):
    """More rows than one pass takes: rows of the second pass equal the same rows on their own."""
    codes, scales = _weights(96, 160, 9)
    mat = stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)).cuda(), torch.from_numpy(scales).cuda(), 160)
    x = _rows(2100, 160, 9, "bf16")
    got = mat.product(x.cuda(), 16, torch.float32).double().cpu().numpy()
    ref, tol = _product(x, codes, scales, 16, torch.float32)
    assert (np.abs(got - ref) <= tol).all()
    mat.free()


@pytest.mark.parametrize("m", [1, 7, 40, 200])
@pytest.mark.parametrize("act", [16, 4])
def test_product_strides(stage, m, act):
    """Rows inside wider ones on both sides; what lies between and behind stays."""
    n, k = 75, 100
    codes, scales = _weights(n, k, 11)
    mat = stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.from_numpy(scales), k)
    wide = _rows(m, k + 5, 12, "f16")
    for out_dtype in (torch.float32, torch.float16):
        out = torch.full((m + 1, n + 6), 7.0, dtype=out_dtype, device="cuda")
        mat.product(wide.cuda()[:, 3:3 + k], act, out=out[:m, 2:2 + n])
        got = out.double().cpu().numpy()
        ref, tol = _product(wide[:, 3:3 + k], codes, scales, act, out_dtype)
        assert (np.abs(got[:m, 2:2 + n] - ref) <= tol).all()
        got[:m, 2:2 + n] = 7.0
        assert (got == 7.0).all()
    mat.free()


@pytest.mark.parametrize("m", [3, 40, 140])
@pytest.mark.parametrize("act", [16, 4])
def test_product_nonfinite(stage, m, act):
    """A row with a NaN or an infinity and a column with a NaN scale are NaN, the others as without them."""
    n, k = 70, 96
    codes, scales = _weights(n, k, 13)
    scales[5, 1] = 255
    mat = stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.from_numpy(scales), k)
    x = _rows(m, k, 14, "bf16")
    x[0, 40] = float("nan")
    x[2, 95] = float("inf")
    got = mat.product(x.cuda(), act, torch.float32).double().cpu().numpy()
    bad = np.zeros((m, n), bool)
    bad[[0, 2]] = True
    bad[:, 5] = True
    assert (np.isnan(got) == bad).all()
    x[[0, 2]] = 0.0
    scales[5, 1] = 120
    ref, tol = _product(x, codes, scales, act, torch.float32)
    assert (np.abs(got - ref) <= tol)[~bad].all()
    mat.free()


@pytest.mark.parametrize("act", [16, 4])
def test_product_scales(stage, act):
    """Activations and weights from the smallest to the largest powers of two; rows of zeros."""
    n, k = 64, 64
    codes, _ = _weights(n, k, 15)
    for e in (-100, -60, 0, 60, 100):
        scales = np.full((n, 2), 127 - e, np.uint8)
        x = (_rows(4, k, 16, "bf16").double() * 2.0 ** e).to(torch.bfloat16)
        x[3] = 0.0
        mat = stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.from_numpy(scales), k)
        got = mat.product(x.cuda(), act, torch.float32).double().cpu().numpy()
        ref, tol = _product(x, codes, scales, act, torch.float32)
        assert (np.abs(got - ref) <= tol).all() and (got[3] == 0).all()
        mat.free()


def test_product_streams(stage):
    """Products on two streams share the stage's workspace: each waits for the one before it."""
    codes, scales = _weights(640, 512, 17)
    mat = stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.from_numpy(scales), 512)
    xs = [_rows(m, 512, 18 + m, "f16").cuda() for m in (64, 3, 200, 17, 1, 90)]
    want = [mat.product(x, 16, torch.float32) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [mat.product(x, 16, torch.float32, stream=streams[i % 2]) for i, x in enumerate(xs)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    mat.free()


def test_product_order(stage):
    """Long products, split and not, on the default stream and two others in turn: each waits for the whole of the one before
    it, also where that took several passes or a sampling call came between."""
    mats = []
    for n, k in ((4096, 4096), (520, 8200), (8192, 700)):
        codes, scales = _weights(n, k, 27)
        mats.append(stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.from_numpy(scales), k))
    calls = [(mats[i % 3], _rows(m, mats[i % 3].k, 28 + i, "bf16").cuda()) for i, m in enumerate((1500, 300, 2500, 65, 2000, 700, 2100, 1000))]
    z = torch.from_numpy(np.random.default_rng(29).standard_normal((20, 60000))).float().cuda()
    u = torch.full((20,), 0.4, device="cuda")
    want = [mat.product(x) for mat, x in calls]
    tok, p = stage.sample(z, Sampling(), u)
    torch.cuda.synchronize()
    streams = [None, torch.cuda.Stream(), torch.cuda.Stream()]
    for r in range(4):
        got = []
        for i, (mat, x) in enumerate(calls):
            got.append(mat.product(x, stream=streams[(i + r) % 3]))
            if i % 3 == 1:
                t2, p2 = stage.sample(z, Sampling(), u, stream=streams[(i + r + 1) % 3])
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert torch.equal(t2, tok) and torch.equal(p2, p)
    for mat in mats:
        mat.free()


def test_capture(stage):
    """Rounding and products of few rows use no memory of the stage and can be captured; a larger product refuses and
    leaves the capture whole."""
    codes, scales = _weights(64, 64, 19)
    mat = stage.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.from_numpy(scales), 64)
    x, many = _rows(9, 64, 20, "bf16").cuda(), _rows(65, 64, 20, "bf16").cuda()
    mat.product(x)
    mat.product(many)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c, s = stage.mx4_quantize(x)
        v = stage.mx4_dequantize(c, s, 64, torch.bfloat16)
        o = mat.product(x, out_dtype=torch.float32)
        with pytest.raises(StageError) as ei:
            mat.product(many)
        assert ei.value.code == -7
    for i in range(3):
        x.copy_(_rows(9, 64, 21 + i, "bf16"))
        mat.product(many)
        g.replay()
        eager = mat.product(x, out_dtype=torch.float32)
        torch.cuda.synchronize()
        ref = mx4_values(*mx4_encode(x.double().cpu().numpy()))
        assert np.array_equal(v.double().cpu().numpy(), ref)
        assert torch.equal(o, eager)
    mat.free()


def _mx4_head(stage, shape, vocab, seed):
    fn, _ = synth.make_head(shape, vocab, seed)
    w = torch.from_numpy(np.random.default_rng(seed).standard_normal((vocab, shape.hidden)) * 0.02).float().cuda()
    codes, scales = stage.mx4_quantize(w)
    unpacked = np.stack([codes.cpu().numpy() & 15, codes.cpu().numpy() >> 4], -1).reshape(vocab, -1)[:, : shape.hidden]
    return fn, codes, scales, mx4_values(unpacked, scales.cpu().numpy())


@pytest.mark.parametrize("M", [1, 5, 64])
def test_head_mx4(M):
    """stage_head_top1 and stage_head_sample through an MXFP4 head: logits against 64 bits, the token and its
    probability those of the logits that came with it."""
    shape = synth.TINY
    p = Pair(shape, 310, with_oracle=False)
    vocab = 1003
    fn, codes, scales, w = _mx4_head(p.gpu, shape, vocab, 311)
    p.gpu.attach_head_mx4(fn.cuda(), codes, scales)
    x = synth.make_hidden(shape, M, 312, M)
    tok, pr, mx, lg = p.gpu.head_top1(x.cuda(), with_logits=True)
    tok2, pr2, lg2 = p.gpu.head_sample(x.cuda(), Sampling(0.0), torch.zeros(M, device="cuda"), with_logits=True)
    xd = host(x)
    h = xd / np.sqrt((xd ** 2).mean(1, keepdims=True) + shape.rms_eps) * host(fn)
    # the normalized row is rounded to fp16 (2^-11 of each value; the fp32 norm adds less than 2^-21), then the product
    ref = h @ w.T
    tol = (np.abs(h) * (2.0 ** -11 + 2.0 ** -21) + 2.0 ** -25) @ np.abs(w).T + 2.0 ** -18 * np.abs(h).max(1, keepdims=True) * np.abs(w).sum(1) \
        + 2.0 ** -23 * (3 * shape.hidden / 8 + 8) * (np.abs(h) @ np.abs(w).T)
    assert (np.abs(host(lg) - ref) <= tol).all()
    assert torch.equal(lg, lg2)
    gi, gp, gmx = oracle.top1(lg.double().cpu().numpy())
    assert np.array_equal(tok.cpu().numpy(), gi) and np.array_equal(tok2.cpu().numpy(), gi)
    assert np.array_equal(mx.cpu().numpy(), gmx.astype(np.float32))
    assert np.max(np.abs(pr.cpu().numpy() - gp) / gp) <= 2.0 ** -22
    assert (pr2.cpu().numpy() == 1).all()
    for f in (lambda: p.gpu.attach_head_mx4(fn.cuda(), codes, scales), lambda: p.gpu.attach_head(*synth.make_head(shape, 64, 1))):
        with pytest.raises(StageError) as ei:
            f()
        assert ei.value.code == -7
    p.close()


def test_matrix_freed_with_its_stage():
    p = Pair(synth.TINY, 320, with_oracle=False)
    codes, scales = _weights(64, 64, 22)
    mat = p.gpu.mx4_matrix(torch.from_numpy(mx4_pack(codes)), torch.from_numpy(scales), 64)
    p.close()
    assert mat.handle is None
