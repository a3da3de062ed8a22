"""Plain fp64 forms of the paged cache's operators, and a stage, pool and mirror of
its sequences for the tests."""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

from paper_2608_19147_amd import Stage

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}   # relative, of one rounding
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}     # absolute, below the normal range
THETA = 10000.0


def make_stage(L=1, Hq=4, Hkv=2, D=64, kv="bf16", max_positions=4096) -> Stage:
    g = torch.Generator().manual_seed(1)
    H, F = 256, 688
    dims = {"wq": (Hq * D, H), "wk": (Hkv * D, H), "wv": (Hkv * D, H), "wo": (H, Hq * D), "wg": (F, H), "wu": (F, H), "wd": (H, F)}
    mats = {name: SimpleNamespace(q=torch.randint(0, 256, (n, k // 2), generator=g, dtype=torch.uint8).numpy(),
                                  scales=np.full((n, -(-k // 128)), 0.002, np.float16), n=n, k=k) for name, (n, k) in dims.items()}
    shape = SimpleNamespace(n_layers=L, hidden=H, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=D, ffn=F, group_size=128, rms_eps=1e-5,
                            rope_theta=THETA, act_dtype=kv, kv_dtype=kv, max_positions=max_positions)
    norm = torch.ones(H, dtype=TORCH[kv])
    return Stage(shape, [SimpleNamespace(attn_norm=norm, ffn_norm=norm, mats=mats)] * L)


def rows(stage, n, seed, scale=1.0):
    """K or V rows [L, Hkv, n, D] in the KV dtype, on the device."""
    sh = stage.shape
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((sh.n_layers, sh.n_kv_heads, n, sh.head_dim), device="cuda", generator=g) * scale).to(stage.kv_dtype)


def sees(P, n, mask=None, mask_rows=None) -> np.ndarray:
    s = np.arange(P + n)[None, :] <= P + np.arange(n)[:, None]
    if mask is not None:
        s = s & (np.asarray(mask)[None, :] != 0)
    if mask_rows is not None:
        s = s & (np.asarray(mask_rows) != 0)
    return s


def attend(q, k, v, see, scale):
    """fp64 attention of q [n, Hq, D] over k, v [Hkv, T, D]: (o, bound) with o [n, Hq, D] and the weighted mean of |v| [n, Hq, D],
    the largest scale sum |q k| over the seen rows [n, Hq], and of max |q| sum |k|."""
    q, k, v = q.double(), k.double(), v.double()
    n, Hq, D = q.shape
    gs = Hq // k.shape[0]
    see = torch.from_numpy(np.ascontiguousarray(see)).to(q.device)
    o, a = torch.zeros_like(q), torch.zeros_like(q)
    s_abs, s_top = (torch.zeros((n, Hq), dtype=torch.float64, device=q.device) for _ in range(2))
    for h in range(Hq):
        kh, vh, qh = k[h // gs], v[h // gs], q[:, h]
        kh = torch.where(see.any(0)[:, None], kh, 0.0)               # what no row sees may hold anything
        z = torch.where(see, scale * (qh @ kh.t()), -math.inf)
        top = z.amax(1, keepdim=True)
        w = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
        tot = w.sum(1, keepdim=True)
        w = w / torch.where(tot == 0, 1.0, tot)
        vs = torch.where(see.any(0)[:, None], vh, 0.0)
        o[:, h], a[:, h] = w @ vs, w @ vs.abs()
        s_abs[:, h] = torch.where(see, scale * (qh.abs() @ kh.abs().t()), 0.0).amax(1)
        s_top[:, h] = torch.where(see, scale * qh.abs().amax(1, keepdim=True) * kh.abs().sum(1)[None], 0.0).amax(1)
    return o, a, s_abs, s_top


def attend_bound(o, a, s_abs, s_top, T, D, kv, q_dtype, out_dtype, parts=64):
    """How far a result may be from 64 bits.  A probability's relative error is that of its exponent (the score's sum of D
    products and its scaling, in fp32; a query in fp32 enters as two terms of kv, within the square of a half step of it, or in
    fp16 of 2^-25 of the largest), of exp2 (2 steps), and of its own term: one of kv at worst, which the sum does not
    share; the output then is off by that times the weighted mean of |v|.  Sums of T terms are taken in groups of 32 and
    joined in at most `parts` partial results; the last rounding is that of the output."""
    u = 2.0 ** -24
    score = (D + 8) * u * s_abs
    if q_dtype == torch.float32:
        score = score + (HALF_STEP[kv] ** 2 * s_abs + 2.0 ** -25 * s_top if kv == torch.float16 else 2 * HALF_STEP[kv] ** 2 * s_abs)
    p = HALF_STEP[kv] + 2 * (score[..., None] + 8 * u) + (4 * (T / 32) + 64 + parts) * u
    return a * p + o.abs() * HALF_STEP[out_dtype] + TINY[out_dtype] + 2.0 ** -126


def turned(x, positions, pair_axis=None):
    """Rows x [M, H, D] in fp64 with pair (i, i + D/2) turned by positions [axes, M]."""
    x = x.double()
    D = x.shape[-1]
    pos = np.atleast_2d(np.asarray(positions, np.float64))
    axis = np.zeros(D // 2, int) if pair_axis is None else np.asarray(pair_axis, int)
    ang = torch.from_numpy(pos[axis].T * THETA ** (-2.0 * np.arange(D // 2) / D)).to(x.device)[:, None]
    a, b = x[..., : D // 2], x[..., D // 2:]
    return torch.cat([a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()], -1)
