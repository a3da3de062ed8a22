"""The last stage's operators where their bits, their loops and their order are
easily lost: small elements beside large ones, runs of equal logits, large norm
weights, borders between bins, and calls that follow a call that failed."""
import numpy as np
import pytest
import torch

import synth
from answer_ref import BLOCK, mx4_pack
from gpu_cases import Pair

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
