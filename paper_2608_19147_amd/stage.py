"""Python binding of libstage: argument marshalling only.

Every step of the forward runs in the HIP kernels of libstage.so; torch is used
for device buffers (``data_ptr``) and for the current HIP stream.
"""
from __future__ import annotations

import atexit
import ctypes
import struct
import weakref
from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np
import torch

from . import _lib
from ._lib import check

# The current stream's handle of a device: by a name that torch keeps to itself, which makes no objects, where it is there.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)

MATRIX_NAMES = ("wq", "wk", "wv", "wo", "wg", "wu", "wd")
_DT = {"f16": _lib.DTYPE_F16, "bf16": _lib.DTYPE_BF16}
_TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}


_DT_OF = {torch.float32: _lib.DTYPE_F32, torch.float16: _lib.DTYPE_F16, torch.bfloat16: _lib.DTYPE_BF16}

_LIVE_STATES: "weakref.WeakSet[KVState]" = weakref.WeakSet()
_LIVE_MATRICES: "weakref.WeakSet[Mx4Matrix]" = weakref.WeakSet()
_LIVE_POOLS: "weakref.WeakSet[PagePool]" = weakref.WeakSet()
_LIVE_STAGES: "weakref.WeakSet[Stage]" = weakref.WeakSet()


def close_all() -> None:
    """Free every live KV state, MXFP4 matrix and page pool, then every live stage.  Registered with
    atexit, so the library's device synchronizations and frees run while the
    interpreter and the HIP runtime are both still whole, rather than from
    ``__del__`` during interpreter shutdown."""
    for kv in list(_LIVE_STATES):
        kv.free()
    for m in list(_LIVE_MATRICES):
        m.free()
    for pool in list(_LIVE_POOLS):
        pool.free()
    for st in list(_LIVE_STAGES):
        st.close()


atexit.register(close_all)


def _stream_ptr(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _ptr(a) -> int:
    if isinstance(a, torch.Tensor):
        return a.data_ptr()
    return a.ctypes.data


def _rows(t: torch.Tensor, name: str) -> int:
    """The row stride of a device [m, k] tensor of a float type whose rows are contiguous."""
    if t.dim() != 2 or not t.is_cuda or t.dtype not in _DT_OF:
        raise ValueError(f"{name} must be a device [rows, columns] tensor in float32, float16 or bfloat16")
    m, k = t.shape
    if m < 1 or k < 1:
        raise ValueError(f"{name} is empty")
    ld, step = t.stride()
    if k > 1 and step != 1 or m > 1 and ld < k:
        raise ValueError(f"{name}'s rows must be contiguous and must not overlap")
    return max(ld, k)


def _on(stage, stream, device):
    """(stream handle, maker of tensors) of a call on the tensors' ``device``, which
    has to be the stage's: the results come from the pool of the stream that writes
    them, so that a later use of their memory is ordered behind it."""
    if device.index != stage.device_index:
        raise ValueError(f"the stage is on cuda:{stage.device_index}, the tensors on {device}")
    if stream is None:
        return _raw_stream(device.index), torch.empty
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")

    def empty(shape, dtype, device):
        with torch.cuda.stream(stream):
            return torch.empty(shape, dtype=dtype, device=device)

    return int(stream.cuda_stream), empty


def _count(n, name: str) -> int:
    """n as the C calls take it: ctypes would narrow it to some other number."""
    n = int(n)
    if not -2 ** 31 <= n < 2 ** 31:
        raise ValueError(f"{name} {n} is out of range")
    return n


def _int32(a, name: str) -> np.ndarray:
    """Whole numbers as a contiguous int32 array; others, and those that it does not hold, are refused."""
    if not (isinstance(a, np.ndarray) and a.dtype == np.int32):
        a = np.asarray(a)
        with np.errstate(invalid="ignore"):
            b = a.astype(np.int32)
        if (a != b).any():
            raise ValueError(f"{name} must be whole numbers below 2^31")
        a = b
    return np.ascontiguousarray(a)


def _mask8(a) -> np.ndarray:
    """A mask as contiguous uint8: what is not zero stays so."""
    if not (isinstance(a, np.ndarray) and a.dtype == np.uint8):
        a = np.asarray(a) != 0
    return np.ascontiguousarray(a, dtype=np.uint8)


def _weights_on(stage, stream, t: torch.Tensor) -> int:
    """The stream handle of a call that packs weights from ``t``, on the stage's device or on the host."""
    return _on(stage, stream, t.device if t.is_cuda else torch.device("cuda", stage.device_index))[0]


class Stage:
    """One pipeline stage on the current GPU.

    ``shape`` provides n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn,
    group_size, rms_eps, rope_theta, act_dtype ('f16'|'bf16'), kv_dtype,
    max_positions.  ``layers[l]`` provides ``attn_norm``/``ffn_norm`` (torch
    tensors in the act dtype) and ``mats[name]`` with ``q`` (uint8 [N, K/2]),
    ``scales`` (float16 [N, K/G]), ``n``, ``k`` — host numpy arrays or device
    torch tensors (``on_device=True``).
    """

    device_index = 0

    def __init__(self, shape, layers: Sequence, on_device: bool = False, stream=None):
        self.lib = _lib.load()
        self.shape = shape
        cfg = _lib.StageConfig(
            n_layers=shape.n_layers, hidden=shape.hidden, n_q_heads=shape.n_q_heads,
            n_kv_heads=shape.n_kv_heads, head_dim=shape.head_dim, ffn=shape.ffn,
            group_size=shape.group_size, rms_eps=shape.rms_eps, act_dtype=_DT[shape.act_dtype],
            kv_dtype=_DT[shape.kv_dtype], rope_theta=shape.rope_theta,
            max_positions=shape.max_positions, rope_cos_sin=None)
        arr = (_lib.LayerWeights * shape.n_layers)()
        keep = []
        for l, lay in enumerate(layers):
            an = lay.attn_norm.contiguous()
            fn = lay.ffn_norm.contiguous()
            if not on_device:
                an, fn = an.cpu(), fn.cpu()
            keep += [an, fn]
            arr[l].attn_norm = an.data_ptr()
            arr[l].ffn_norm = fn.data_ptr()
            for name in MATRIX_NAMES:
                m = lay.mats[name]
                q, s = m.q, m.scales
                if not on_device:
                    q = np.ascontiguousarray(q, dtype=np.uint8)
                    s = np.ascontiguousarray(s).view(np.uint16)
                keep += [q, s]
                setattr(arr[l], name, _lib.QuantMatrix(q=_ptr(q), scales=_ptr(s), n=m.n, k=m.k))
        h = ctypes.c_void_p()
        self.device_index = torch.cuda.current_device()
        check(self.lib.stage_create(ctypes.byref(cfg), arr, int(on_device), ctypes.c_void_p(_stream_ptr(stream)),
                                    ctypes.byref(h)))
        self.handle = h
        self.act_dtype = _TORCH[shape.act_dtype]
        self.kv_dtype = _TORCH[shape.kv_dtype]
        _LIVE_STAGES.add(self)

    # ------------------------------------------------------------------
    def close(self) -> None:
        """Free the stage's device memory (its KV states, matrices and page pools first)."""
        if getattr(self, "handle", None):
            for kv in list(_LIVE_STATES):
                if kv.stage is self:
                    kv.free()
            for m in list(_LIVE_MATRICES):
                if m.stage is self:
                    m.free()
            for pool in list(_LIVE_POOLS):
                if pool.stage is self:
                    pool.free()
            check(self.lib.stage_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def weight_bytes(self) -> int:
        return int(self.lib.stage_weight_bytes(self.handle))

    def profile(self, kernel_class: Optional[str]) -> None:
        """Bracket every launch of one kernel class ('qkv', 'attn', 'oproj',
        'gateup', 'down') with hipEvents on the launch stream; None stops."""
        check(self.lib.stage_profile_enable(self.handle, -1 if kernel_class is None else _lib.KERNEL_CLASSES[kernel_class]))

    def profile_read(self):
        """(launches, total_ms) recorded since profile() or the last read."""
        n = ctypes.c_int()
        ms = ctypes.c_double()
        check(self.lib.stage_profile_read(self.handle, ctypes.byref(n), ctypes.byref(ms)))
        return n.value, ms.value

    def profile_read_each(self, capacity: int = 65536) -> np.ndarray:
        """Each recorded launch's duration in ms (launch order) since profile()
        or the last read."""
        out = np.zeros(capacity, np.float32)
        n = ctypes.c_int()
        check(self.lib.stage_profile_read_each(self.handle, ctypes.c_void_p(out.ctypes.data), capacity, ctypes.byref(n)))
        return out[: min(n.value, capacity)].copy()

    def debug_attn_arm(self, layer: int, max_keys: int) -> None:
        """Record `layer`'s rotated queries and visible scores in later forwards
        (per-layer kernels); layer = -1 disarms."""
        check(self.lib.stage_debug_attn_arm(self.handle, layer, max_keys))
        if layer >= 0:
            self._dbg_cap = max(getattr(self, "_dbg_cap", 0), max_keys)   # the library's buffers only grow

    def debug_attn_read(self):
        """(q [M, Hq, D], logits [M, Hq, max_keys]) of the last armed forward;
        keys a row does not see are NaN."""
        sh = self.shape
        q = np.empty(64 * sh.n_q_heads * sh.head_dim, np.float32)
        rows, keys = ctypes.c_int(), ctypes.c_int()
        lg = np.empty(64 * sh.n_q_heads * self._dbg_cap, np.float32)
        check(self.lib.stage_debug_attn_read(self.handle, q.ctypes.data, lg.ctypes.data, ctypes.byref(rows), ctypes.byref(keys)))
        m, k = rows.value, keys.value
        return (q[: m * sh.n_q_heads * sh.head_dim].reshape(m, sh.n_q_heads, sh.head_dim),
                lg[: m * sh.n_q_heads * k].reshape(m, sh.n_q_heads, k))

    def device_status(self) -> None:
        """Wait for the device; raise StageError (STAGE_E_DEVICE) once if a
        single-launch forward of this stage gave up waiting on another
        workgroup or an embedding gather met an id outside its table."""
        check(self.lib.stage_device_status(self.handle))

    def phase_trace(self) -> np.ndarray:
        """[workgroups, layers, 40] device real-time stamps (100 MHz) and exchange
        pass counts of the last single-launch forward (needs STAGE_PS_TRACE=1 at
        creation)."""
        per = 40                                   # entries per workgroup and layer
        n = torch.cuda.get_device_properties(0).multi_processor_count * self.shape.n_layers * per
        out = np.empty(n, dtype=np.uint64)
        nwg = ctypes.c_int()
        check(self.lib.stage_debug_phase_trace(self.handle, out.ctypes.data, n, ctypes.byref(nwg)))
        return out[: nwg.value * self.shape.n_layers * per].reshape(nwg.value, self.shape.n_layers, per)

    def attach_head(self, final_norm: torch.Tensor, lm_head, on_device: bool = False, stream=None) -> None:
        """Final RMSNorm weight [H] (act dtype) and INT4 LM head (``q`` uint8
        [vocab, H/2], ``scales`` float16 [vocab, H/G], ``n``, ``k``)."""
        fn = final_norm.contiguous()
        q, s = lm_head.q, lm_head.scales
        if not on_device:
            fn = fn.cpu()
            q = np.ascontiguousarray(q, dtype=np.uint8)
            s = np.ascontiguousarray(s).view(np.uint16)
        qm = _lib.QuantMatrix(q=_ptr(q), scales=_ptr(s), n=lm_head.n, k=lm_head.k)
        check(self.lib.stage_head_attach(self.handle, ctypes.c_void_p(fn.data_ptr()), ctypes.byref(qm), int(on_device),
                                         ctypes.c_void_p(_stream_ptr(stream))))
        self.vocab = int(lm_head.n)

    def head_top1(self, hidden: torch.Tensor, with_logits: bool = False, stream=None):
        """(token int32 [M], p_max fp32 [M], max logit fp32 [M], logits fp32
        [M, vocab] or None) on the device for the rows of ``hidden``."""
        M = int(hidden.shape[0])
        tok = torch.empty(M, dtype=torch.int32, device=hidden.device)
        p = torch.empty(M, dtype=torch.float32, device=hidden.device)
        lg = torch.empty(M, dtype=torch.float32, device=hidden.device)
        full = torch.empty((M, self.vocab), dtype=torch.float32, device=hidden.device) if with_logits else None
        check(self.lib.stage_head_top1(self.handle, ctypes.c_void_p(hidden.contiguous().data_ptr()), M,
                                       ctypes.c_void_p(tok.data_ptr()), ctypes.c_void_p(p.data_ptr()),
                                       ctypes.c_void_p(lg.data_ptr()),
                                       ctypes.c_void_p(full.data_ptr() if full is not None else None),
                                       ctypes.c_void_p(_stream_ptr(stream))))
        return tok, p, lg, full

    def attach_head_mx4(self, final_norm: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, stream=None) -> None:
        """Final RMSNorm weight [H] (act dtype) and an MXFP4 LM head: codes uint8
        [vocab, ceil(H/2)], scales uint8 [vocab, ceil(H/32)], all on the host or
        all on the device."""
        on_dev = _check_mx4(codes, scales, self.shape.hidden)
        sp = _weights_on(self, stream, codes)
        if tuple(final_norm.shape) != (self.shape.hidden,) or final_norm.dtype != self.act_dtype or not final_norm.is_contiguous():
            raise ValueError("final_norm must be a contiguous [hidden] tensor in the activation dtype")
        if final_norm.device != codes.device:
            raise ValueError("final_norm, codes and scales must be on one device")
        check(self.lib.stage_head_attach_mx4(self.handle, final_norm.data_ptr(), codes.data_ptr(), scales.data_ptr(),
                                             codes.shape[0], on_dev, sp))
        self.vocab = int(codes.shape[0])

    def head_sample(self, hidden: torch.Tensor, params, u: torch.Tensor, with_logits: bool = False, stream=None):
        """(token int32 [M], p fp32 [M], logits fp32 [M, vocab] or None): one token
        drawn per row of ``hidden`` through the attached head; ``params`` and ``u``
        as in ``sample``."""
        if hidden.dim() != 2 or hidden.shape[1] != self.shape.hidden or hidden.dtype != self.act_dtype or not hidden.is_cuda \
                or not hidden.is_contiguous():
            raise ValueError("hidden must be a contiguous device [M, hidden] tensor in the activation dtype")
        M, dev = hidden.shape[0], hidden.device
        packed = _sampling(params, M)
        _check_u(u, M, dev)
        sp, empty = _on(self, stream, dev)
        tok, p = empty(M, dtype=torch.int32, device=dev), empty(M, dtype=torch.float32, device=dev)
        full = empty((M, getattr(self, "vocab", 1)), dtype=torch.float32, device=dev) if with_logits else None
        check(self.lib.stage_head_sample(self.handle, hidden.data_ptr(), M, packed, u.data_ptr(), tok.data_ptr(), p.data_ptr(),
                                         full.data_ptr() if full is not None else None, sp))
        return tok, p, full

    def sample(self, logits: torch.Tensor, params, u: torch.Tensor, stream=None):
        """(token int32 [M], p fp32 [M]): one token drawn per row of ``logits``
        [M, vocab] (float32, float16 or bfloat16; rows may be part of wider ones)
        by ``params`` (a ``Sampling``, or one per row) and ``u`` fp32 [M] in [0, 1)."""
        ld = _rows(logits, "logits")
        M, V = logits.shape
        dev = logits.device
        packed = _sampling(params, M)
        _check_u(u, M, dev)
        sp, empty = _on(self, stream, dev)
        tok, p = empty(M, dtype=torch.int32, device=dev), empty(M, dtype=torch.float32, device=dev)
        check(self.lib.stage_sample(self.handle, logits.data_ptr(), _DT_OF[logits.dtype], ld, M, V, packed, u.data_ptr(),
                                    tok.data_ptr(), p.data_ptr(), sp))
        return tok, p

    def tree_accept(self, parents: torch.Tensor, tokens: torch.Tensor, sampled: torch.Tensor, stream=None):
        """(count int32 [S], path int32 [S, n], next int32 [S], keep uint8 [S, n]) of
        the walk of S drafted trees of n nodes: device int32 [S, n] parents (before
        their children; node 0 is the root), drafted tokens and the tokens sampled
        at the nodes.  ``path`` holds the walked nodes, then -1; ``keep`` marks them;
        ``next`` is the token sampled at the last one."""
        if parents.dim() != 2 or not parents.is_cuda:
            raise ValueError("parents must be a device [slots, nodes] tensor")
        shape, dev = parents.shape, parents.device
        for t, name in ((parents, "parents"), (tokens, "tokens"), (sampled, "sampled")):
            if t.dtype != torch.int32 or t.device != dev or t.shape != shape or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} on {dev}")
        S, n = shape
        sp, empty = _on(self, stream, dev)
        count, path = empty(S, dtype=torch.int32, device=dev), empty((S, n), dtype=torch.int32, device=dev)
        nxt, keep = empty(S, dtype=torch.int32, device=dev), empty((S, n), dtype=torch.uint8, device=dev)
        check(self.lib.stage_tree_accept(self.handle, parents.data_ptr(), tokens.data_ptr(), sampled.data_ptr(), S, n,
                                         count.data_ptr(), path.data_ptr(), nxt.data_ptr(), keep.data_ptr(), sp))
        return count, path, nxt, keep

    def mx4_quantize(self, x: torch.Tensor, stream=None):
        """(codes uint8 [m, ceil(k/2)], scales uint8 [m, ceil(k/32)]): the rows of a
        device [m, k] tensor (float32, float16 or bfloat16) in MXFP4."""
        ld = _rows(x, "x")
        m, k = x.shape
        dev = x.device
        sp, empty = _on(self, stream, dev)
        codes = empty((m, (k + 1) // 2), dtype=torch.uint8, device=dev)
        scales = empty((m, (k + 31) // 32), dtype=torch.uint8, device=dev)
        check(self.lib.stage_mx4_quantize(self.handle, x.data_ptr(), _DT_OF[x.dtype], ld, m, k, codes.data_ptr(),
                                          scales.data_ptr(), sp))
        return codes, scales

    def mx4_dequantize(self, codes: torch.Tensor, scales: torch.Tensor, k: int, out_dtype=torch.float32, stream=None) -> torch.Tensor:
        """The values [m, k] that device codes and scales stand for."""
        if not _check_mx4(codes, scales, k):
            raise ValueError("codes and scales must be device tensors")
        if out_dtype not in _DT_OF:
            raise ValueError("out_dtype must be float32, float16 or bfloat16")
        m, dev = codes.shape[0], codes.device
        sp, empty = _on(self, stream, dev)
        out = empty((m, k), dtype=out_dtype, device=dev)
        check(self.lib.stage_mx4_dequantize(self.handle, codes.data_ptr(), scales.data_ptr(), m, k, out.data_ptr(),
                                            _DT_OF[out_dtype], k, sp))
        return out

    def mx4_matrix(self, codes: torch.Tensor, scales: torch.Tensor, k: int, stream=None) -> "Mx4Matrix":
        """A weight matrix [n, k] in MXFP4 for products, packed once: codes uint8
        [n, ceil(k/2)] and scales uint8 [n, ceil(k/32)], on the host or the device."""
        return Mx4Matrix(self, codes, scales, k, stream)

    def attach_embedding(self, table: torch.Tensor, on_device: bool = False, stream=None) -> None:
        """Token embedding table [vocab, H] in the act dtype (first-stage role)."""
        t = table.contiguous() if on_device else table.detach().cpu().contiguous()
        if t.dim() != 2 or t.shape[1] != self.shape.hidden or t.element_size() != 2:
            raise ValueError("embedding table must be [vocab, hidden] with 2-byte elements")
        check(self.lib.stage_embed_attach(self.handle, ctypes.c_void_p(t.data_ptr()), int(t.shape[0]), int(on_device),
                                          ctypes.c_void_p(_stream_ptr(stream))))
        self.embed_vocab = int(t.shape[0])

    def embed(self, ids: torch.Tensor, hidden_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Hidden rows [n, H] (device, act dtype) = table[ids] for device int32 ids [n]."""
        if ids.dtype != torch.int32 or not ids.is_cuda:
            raise ValueError("ids must be a device int32 tensor")
        ids = ids.contiguous()
        n = int(ids.numel())
        if hidden_out is None:
            hidden_out = torch.empty((n, self.shape.hidden), dtype=self.act_dtype, device=ids.device)
        check(self.lib.stage_embed(self.handle, ctypes.c_void_p(ids.data_ptr()), n, ctypes.c_void_p(hidden_out.data_ptr()),
                                   ctypes.c_void_p(_stream_ptr(stream))))
        return hidden_out

    def prefill(self, state: "KVState", positions, hidden_in: torch.Tensor, past_mask=None,
                hidden_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Prompt rows hidden_in [n, H] (device, act dtype) of a one-slot state;
        positions [n]; past_mask [P] or None."""
        if hidden_out is None:
            hidden_out = torch.empty_like(hidden_in)
        pos = np.ascontiguousarray(positions, dtype=np.int32).reshape(-1)
        pm = None if past_mask is None else np.ascontiguousarray(past_mask, dtype=np.uint8).reshape(-1)
        check(self.lib.stage_prefill(self.handle, state.handle, int(pos.size), ctypes.c_void_p(pos.ctypes.data),
                                     ctypes.c_void_p(pm.ctypes.data if pm is not None else None),
                                     ctypes.c_void_p(hidden_in.data_ptr()), ctypes.c_void_p(hidden_out.data_ptr()),
                                     ctypes.c_void_p(_stream_ptr(stream))))
        return hidden_out

    def new_state(self, n_slots: int, capacity: int) -> "KVState":
        return KVState(self, n_slots, capacity)

    def new_pages(self, n_pages: int, page_rows: int = 64, pair_axis=None) -> "PagePool":
        """A pool of ``n_pages`` pages of ``page_rows`` (16, 32, 64, 128 or 256) cache
        rows for sequences that share pages.  ``pair_axis`` [head_dim / 2] names the
        axis of positions that turns each rotary pair (None: one axis)."""
        return PagePool(self, n_pages, page_rows, pair_axis)

    def forward_paged(self, requests: Sequence["PagedRequest"], hidden_in: torch.Tensor, hidden_out: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
        """``forward`` over sequences of one pool: hidden_in [M, H] (device, act dtype),
        rows request-major.  Positions are required; every new row must see a row."""
        for t, name in ((hidden_in, "hidden_in"), (hidden_out, "hidden_out")):
            if t is not None and (t.dim() != 2 or t.shape[1] != self.shape.hidden or t.dtype != self.act_dtype or not t.is_cuda
                                  or not t.is_contiguous()):
                raise ValueError(f"{name} must be a contiguous device [M, hidden] tensor in the activation dtype")
        M = sum(int(r.n_tokens) for r in requests)
        if hidden_in.shape[0] != M or hidden_out is not None and hidden_out.shape[0] != M:
            raise ValueError(f"the requests have {M} rows")
        if hidden_out is not None and hidden_out.device != hidden_in.device:
            raise ValueError("hidden_in and hidden_out must be on one device")
        sp, empty = _on(self, stream, hidden_in.device)
        arr, keep = _step_requests(requests)
        if hidden_out is None:
            hidden_out = empty(hidden_in.shape, dtype=self.act_dtype, device=hidden_in.device)
        check(self.lib.stage_forward_paged(self.handle, arr, len(requests), hidden_in.data_ptr(), hidden_out.data_ptr(), sp))
        return hidden_out

    def debug_dequant(self, layer: int, which: str, row_layout: bool = False) -> np.ndarray:
        """The matrix as the kernels decode it (tiled layout, or the row layout
        of the persistent kernel)."""
        n, k = self.shape.matrix_shapes()[which]
        out = np.empty((n, k), dtype=np.float32)
        code = MATRIX_NAMES.index(which) + (8 if row_layout else 0)
        check(self.lib.stage_debug_dequant(self.handle, layer, code, out.ctypes.data))
        return out

    def forward(self, requests: Sequence["Request"], hidden_in: torch.Tensor,
                hidden_out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """hidden_in: device [M, H] in the act dtype, rows request-major, then slot, then token."""
        if hidden_out is None:
            hidden_out = torch.empty_like(hidden_in)
        arr = (_lib.StageRequest * len(requests))()
        keep = []
        for i, r in enumerate(requests):
            pos = np.ascontiguousarray(r.positions, dtype=np.int32)
            mask = None if r.mask is None else np.ascontiguousarray(r.mask, dtype=np.uint8)
            rows = None if r.mask_rows is None else np.ascontiguousarray(r.mask_rows, dtype=np.uint8)
            keep += [pos, mask, rows]
            beam = None
            if r.beam_idx is not None:
                beam = np.ascontiguousarray(r.beam_idx, dtype=np.int32)
                keep.append(beam)
            arr[i].state = r.state.handle
            arr[i].n_tokens = int(r.n_tokens)
            arr[i].positions = pos.ctypes.data
            arr[i].beam_idx = beam.ctypes.data if beam is not None else None
            arr[i].attention_mask = mask.ctypes.data if mask is not None else None
            arr[i].attention_mask_rows = rows.ctypes.data if rows is not None else None
            src = mask if mask is not None else rows
            arr[i].mask_len = int(src.shape[-1]) if src is not None and src.ndim else 0
        check(self.lib.stage_forward(self.handle, arr, len(requests), ctypes.c_void_p(hidden_in.data_ptr()),
                                     ctypes.c_void_p(hidden_out.data_ptr()), ctypes.c_void_p(_stream_ptr(stream))))
        return hidden_out


def _check_mx4(codes: torch.Tensor, scales: torch.Tensor, k: int) -> int:
    """1 if the MXFP4 pair of rows of k is on the device, 0 on the host."""
    ok = codes.dtype == torch.uint8 and scales.dtype == torch.uint8 and codes.dim() == 2 and scales.dim() == 2 and k >= 1 \
        and tuple(codes.shape) == (scales.shape[0], (k + 1) // 2) and scales.shape[1] == (k + 31) // 32 and codes.shape[0] >= 1
    if not ok:
        raise ValueError(f"codes and scales must be uint8 [rows, {(k + 1) // 2}] and [rows, {(k + 31) // 32}]")
    if codes.device != scales.device or not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError("codes and scales must be contiguous and on one device")
    return int(codes.is_cuda)


def _check_u(u: torch.Tensor, M: int, device) -> None:
    if u.dtype != torch.float32 or tuple(u.shape) != (M,) or u.device != device or not u.is_contiguous():
        raise ValueError(f"u must be a contiguous float32 [{M}] tensor on {device}")


@dataclass(frozen=True)
class Sampling:
    """How a row's token is drawn: weights exp((logit - max) / temperature) over
    the tokens ranked highest logit first (lowest index first among equals), of
    which top_k keeps the first (0: all), top_p the shortest run that holds its
    share of their weight (1: all), min_p those of at least min_p of the largest
    weight (0: all).  Temperature 0 takes the first."""

    temperature: float = 1.0
    top_k: int = 0
    top_p: float = 1.0
    min_p: float = 0.0

    def __post_init__(self):
        # the C struct StageSampling, made once for every call that takes this object
        object.__setattr__(self, "packed", struct.pack("=fiff", self.temperature, self.top_k, self.top_p, self.min_p))


def _sampling(params, M: int) -> bytes:
    if isinstance(params, Sampling):
        return params.packed * M
    if len(params) != M:
        raise ValueError(f"{len(params)} sampling parameters for {M} rows")
    return b"".join([q.packed for q in params])


class Mx4Matrix:
    """A weight matrix W [n, k] in MXFP4, packed for products (``Stage.mx4_matrix``)."""

    def __init__(self, stage: Stage, codes: torch.Tensor, scales: torch.Tensor, k: int, stream=None):
        on_dev = _check_mx4(codes, scales, k)
        sp = _weights_on(stage, stream, codes)
        self.stage, self.lib = stage, stage.lib
        self.n, self.k = int(codes.shape[0]), int(k)
        h = ctypes.c_void_p()
        check(self.lib.stage_mx4_create(stage.handle, codes.data_ptr(), scales.data_ptr(), self.n, self.k, on_dev,
                                        sp, ctypes.byref(h)))
        self.handle = h
        _LIVE_MATRICES.add(self)

    def free(self) -> None:
        if getattr(self, "handle", None):
            check(self.lib.stage_mx4_free(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def product(self, x: torch.Tensor, act_bits: int = 16, out_dtype: Optional[torch.dtype] = None,
                out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """x W^T [m, n] of device rows x [m, k]: 16-bit rows to within 2^-18 of the
        largest magnitude of each block of 32 (``act_bits`` 16), or rounded to MXFP4
        first (4, also float32 rows), in ``out_dtype`` (x's by default) or into
        ``out`` [m, n], whose rows may be part of wider ones and must not overlap x."""
        ldx = _rows(x, "x")
        m, k = x.shape
        if k != self.k:
            raise ValueError(f"x has {k} columns, the matrix {self.k}")
        dev = x.device
        sp, empty = _on(self.stage, stream, dev)
        if out is None:
            out_dtype = out_dtype or x.dtype
            if out_dtype not in _DT_OF:
                raise ValueError("out_dtype must be float32, float16 or bfloat16")
            out, ldo = empty((m, self.n), dtype=out_dtype, device=dev), self.n
        else:
            if tuple(out.shape) != (m, self.n) or out.device != dev or out_dtype not in (None, out.dtype):
                raise ValueError(f"out must be a [{m}, {self.n}] tensor on {dev}")
            ldo = _rows(out, "out")
        check(self.lib.stage_mx4_product(self.handle, x.data_ptr(), _DT_OF[x.dtype], ldx, m, act_bits, out.data_ptr(),
                                         _DT_OF[out.dtype], ldo, sp))
        return out


@dataclass
class Request:
    """One request of a forward: positions [S, n] int32, mask [S, P+n] uint8
    (nonzero = visible) or None, beam_idx [S] int32 or None, mask_rows
    [S, n, P+n] uint8 (one key mask per query row) or None."""

    state: "KVState"
    positions: np.ndarray
    mask: Optional[np.ndarray]
    beam_idx: Optional[np.ndarray] = None
    mask_rows: Optional[np.ndarray] = None

    @property
    def n_tokens(self) -> int:
        return int(np.asarray(self.positions).shape[-1])


class KVState:
    def __init__(self, stage: Stage, n_slots: int, capacity: int):
        self.stage = stage
        self.lib = stage.lib
        self.n_slots = n_slots
        self.capacity = capacity
        h = ctypes.c_void_p()
        check(self.lib.kv_state_alloc(stage.handle, n_slots, capacity, ctypes.byref(h)))
        self.handle = h
        _LIVE_STATES.add(self)

    def free(self) -> None:
        if getattr(self, "handle", None):
            check(self.lib.kv_state_free(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    @property
    def length(self) -> int:
        n = ctypes.c_int()
        check(self.lib.kv_length(self.handle, ctypes.byref(n)))
        return n.value

    def reset(self) -> None:
        check(self.lib.kv_state_reset(self.handle))

    def truncate(self, new_len: int) -> None:
        check(self.lib.kv_truncate(self.handle, int(new_len)))

    def append(self, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """k, v: [L][S][Hkv][n][D] in the KV dtype (host or device)."""
        k = k.contiguous()
        v = v.contiguous()
        on_dev = int(k.is_cuda)
        check(self.lib.kv_append(self.handle, ctypes.c_void_p(k.data_ptr()), ctypes.c_void_p(v.data_ptr()),
                                 int(k.shape[3]), on_dev, ctypes.c_void_p(_stream_ptr(stream))))

    def _keep(self, keep):
        if keep is None:
            return None, None
        keep = np.ascontiguousarray(keep, dtype=np.uint8)
        if keep.shape != (self.n_slots, self.length):
            raise ValueError(f"keep mask shape {keep.shape} != {(self.n_slots, self.length)}")
        return keep, ctypes.c_void_p(keep.ctypes.data)

    def compact(self, keep=None, stream=None) -> np.ndarray:
        """Remove the rows keep [S, P] (nonzero = keep; None = all) drops, in
        place.  Returns each slot's kept count; P becomes their maximum."""
        keep, kp = self._keep(keep)
        lens = np.zeros(self.n_slots, np.int32)
        check(self.lib.kv_compact(self.handle, kp, ctypes.c_void_p(lens.ctypes.data),
                                  ctypes.c_void_p(_stream_ptr(stream))))
        return lens

    def capture_size(self, keep=None) -> int:
        keep, kp = self._keep(keep)
        n = ctypes.c_int64()
        check(self.lib.kv_capture_size(self.handle, kp, ctypes.byref(n)))
        return n.value

    def capture(self, keep=None, on_device: bool = True, stream=None):
        """Serialized kept rows: a device uint8 tensor, or a host numpy array."""
        keep_arr, kp = self._keep(keep)
        n = self.capture_size(keep_arr)
        if on_device:
            blob = torch.empty(n, dtype=torch.uint8, device="cuda")
            ptr = blob.data_ptr()
        else:
            blob = np.empty(n, dtype=np.uint8)
            ptr = blob.ctypes.data
        check(self.lib.kv_capture(self.handle, kp, ctypes.c_void_p(ptr), n, int(on_device),
                                  ctypes.c_void_p(_stream_ptr(stream))))
        return blob

    def capture_noalloc(self, keep=None, stream=None) -> np.ndarray:
        """kv_capture into a host blob through the library's fixed device
        staging array (no device allocation)."""
        keep_arr, kp = self._keep(keep)
        blob = np.empty(self.capture_size(keep_arr), dtype=np.uint8)
        check(self.lib.kv_capture_noalloc(self.handle, kp, ctypes.c_void_p(blob.ctypes.data), blob.size,
                                          ctypes.c_void_p(_stream_ptr(stream))))
        return blob

    def restore(self, blob, stream=None) -> np.ndarray:
        """Install a captured state (device tensor or host array); returns each
        slot's captured count."""
        lens = np.zeros(self.n_slots, np.int32)
        if isinstance(blob, torch.Tensor) and blob.is_cuda:
            ptr, n, dev = blob.data_ptr(), blob.numel() * blob.element_size(), 1
        else:
            blob = np.ascontiguousarray(blob)
            ptr, n, dev = blob.ctypes.data, blob.nbytes, 0
        check(self.lib.kv_restore(self.handle, ctypes.c_void_p(ptr), int(n), dev, ctypes.c_void_p(lens.ctypes.data),
                                  ctypes.c_void_p(_stream_ptr(stream))))
        return lens

    def read(self, layer: int, slot: int, start: int, count: int, stream=None):
        """Rows [start, start+count) of one layer and slot as the slot sees them: K, V [Hkv, count, D]."""
        sh = self.stage.shape
        k = torch.empty((sh.n_kv_heads, count, sh.head_dim), dtype=self.stage.kv_dtype, device="cuda")
        v = torch.empty_like(k)
        check(self.lib.kv_read(self.handle, layer, slot, start, count, ctypes.c_void_p(k.data_ptr()),
                               ctypes.c_void_p(v.data_ptr()), 1, ctypes.c_void_p(_stream_ptr(stream))))
        return k, v


class PagePool:
    """Pages of cache rows for every layer of a stage, and the sequences that hold
    them (``Stage.new_pages``).  ``k`` and ``v`` are the pages [n_layers, n_pages,
    n_kv_heads, page_rows, head_dim]; they start as zeros, and free ones are handed
    out lowest first."""

    def __init__(self, stage: Stage, n_pages: int, page_rows: int, pair_axis=None):
        sh = stage.shape
        axis = None
        if pair_axis is not None:
            axis = np.asarray(pair_axis)
            if axis.shape != (sh.head_dim // 2,) or ((axis < 0) | (axis >= _lib.MAX_AXES)).any() or (axis != axis.astype(np.uint8)).any():
                raise ValueError(f"pair_axis must name an axis below {_lib.MAX_AXES} for each of {sh.head_dim // 2} pairs")
            axis = np.ascontiguousarray(axis, dtype=np.uint8)
        if n_pages < 1 or page_rows not in (16, 32, 64, 128, 256):
            raise ValueError("n_pages must be positive and page_rows 16, 32, 64, 128 or 256")
        self.stage, self.lib = stage, stage.lib
        self.n_pages, self.page_rows = int(n_pages), int(page_rows)
        self.n_axes = 1 if axis is None else int(axis.max()) + 1
        dev = torch.device("cuda", stage.device_index)
        shape = (sh.n_layers, self.n_pages, sh.n_kv_heads, self.page_rows, sh.head_dim)
        self.k = torch.zeros(shape, dtype=stage.kv_dtype, device=dev)
        self.v = torch.zeros(shape, dtype=stage.kv_dtype, device=dev)
        # the zeros are there before any stream's first call on the pool
        torch.cuda.current_stream(dev).synchronize()
        h = ctypes.c_void_p()
        check(self.lib.kv_pages_create(stage.handle, self.n_pages, self.page_rows, self.k.data_ptr(), self.v.data_ptr(),
                                       None if axis is None else axis.ctypes.data, self.n_axes, ctypes.byref(h)))
        self.handle = h
        _LIVE_POOLS.add(self)

    def free(self) -> None:
        """Free the pool, and its sequences and steps with it."""
        if getattr(self, "handle", None):
            check(self.lib.kv_pages_free(self.handle))
            self.handle = None
            self.k = self.v = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    @property
    def free_pages(self) -> int:
        n = ctypes.c_int()
        check(self.lib.kv_pages_available(self.handle, ctypes.byref(n)))
        return n.value

    def new_sequence(self) -> "PagedSequence":
        h = ctypes.c_void_p()
        check(self.lib.kv_seq_create(self.handle, ctypes.byref(h)))
        return PagedSequence(self, h.value)

    def new_step(self) -> "PagedStep":
        return PagedStep(self)

    def fork(self, seqs: Sequence["PagedSequence"], lengths=None, keep=None, stream=None) -> List["PagedSequence"]:
        """One new sequence per entry of ``seqs`` (which may repeat): its first
        ``lengths[i]`` rows (all by default), of them those that ``keep[i]`` (uint8,
        nonzero = kept; None: all) keeps.  Whole pages ahead of the first row left out
        are shared, the other rows copied."""
        n = len(seqs)
        if lengths is not None and len(lengths) != n or keep is not None and len(keep) != n:
            raise ValueError(f"lengths and keep must have {n} entries")
        if self.handle is None:
            raise ValueError("the pool has been freed")
        handles = []
        for q in seqs:
            if q.pool is not self or q._handle is None:
                q._check(self)
            handles.append(q._handle)
        lens = None if lengths is None else _int32(lengths, "lengths")
        masks, kp = None, None
        if keep is not None:
            masks = [None if k is None else _mask8(k) for k in keep]
            for i, m in enumerate(masks):
                if m is not None and m.shape != (int(lens[i]) if lens is not None else seqs[i].length,):
                    raise ValueError(f"keep[{i}] must have one entry per row")
            kp = (ctypes.c_void_p * n)(*[None if m is None else m.ctypes.data for m in masks])
        out = (ctypes.c_void_p * n)()
        check(self.lib.kv_seq_fork((ctypes.c_void_p * n)(*handles), None if lens is None else lens.ctypes.data, kp, n,
                                   out, _pool_stream(self.stage, stream)))
        return [PagedSequence(self, h) for h in out]


def _pool_stream(stage: Stage, stream) -> int:
    return _on(stage, stream, torch.device("cuda", stage.device_index))[0]


class PagedSequence:
    """A sequence of cache rows in a pool's pages (``PagePool.new_sequence``, ``PagePool.fork``)."""

    __slots__ = ("pool", "_handle")                              # a fork makes many at once

    def __init__(self, pool: PagePool, handle: int):
        self.pool, self._handle = pool, handle

    @property
    def handle(self) -> int:
        if self._handle is None or self.pool.handle is None:
            raise ValueError("the sequence has been freed")
        return self._handle

    @property
    def lib(self):
        return self.pool.lib

    def _check(self, pool: PagePool) -> None:
        if self.pool is not pool:
            raise ValueError("the sequence belongs to another pool")
        self.handle                                              # raises if it has been freed

    def free(self) -> None:
        """Give back the pages that no other sequence holds."""
        h = self._handle
        if h is not None:
            self._handle = None
            if self.pool.handle is not None:
                check(self.pool.lib.kv_seq_free(h))

    def __del__(self):
        try:
            if self._handle is not None:
                self.free()
        except Exception:
            pass

    @property
    def length(self) -> int:
        n = ctypes.c_int()
        check(self.lib.kv_seq_length(self.handle, ctypes.byref(n)))
        return n.value

    @property
    def pages(self) -> List[int]:
        """The page of each ``page_rows`` rows."""
        n = ctypes.c_int()
        check(self.lib.kv_seq_pages(self.handle, None, 0, ctypes.byref(n)))
        out = np.empty(n.value, np.int32)
        check(self.lib.kv_seq_pages(self.handle, out.ctypes.data, n.value, ctypes.byref(n)))
        return out.tolist()

    def truncate(self, new_len: int) -> None:
        check(self.lib.kv_seq_truncate(self.handle, _count(new_len, "length")))

    def compact(self, keep, stream=None) -> int:
        """Drop the rows that ``keep`` (uint8 [length], nonzero = kept) does not keep
        and close the others up.  Returns the new length."""
        keep = _mask8(keep)
        if keep.shape != (self.length,):
            raise ValueError(f"keep must have {self.length} entries")
        check(self.lib.kv_seq_compact(self.handle, keep.ctypes.data, _pool_stream(self.pool.stage, stream)))
        return self.length

    def append(self, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
        """Append rows k, v [L][Hkv][n][D] (device, KV dtype; K after rotary)."""
        st = self.pool.stage
        sh = st.shape
        for t, name in ((k, "k"), (v, "v")):
            if t.dim() != 4 or t.dtype != st.kv_dtype or not t.is_cuda or t.shape[2] < 1 \
                    or (t.shape[0], t.shape[1], t.shape[3]) != (sh.n_layers, sh.n_kv_heads, sh.head_dim):
                raise ValueError(f"{name} must be a device [layers, kv heads, rows, head_dim] tensor in the KV dtype")
        if k.shape != v.shape or k.device != v.device:
            raise ValueError("k and v must be alike")
        sp, _ = _on(st, stream, k.device)
        k, v = (t if t.is_contiguous() and t.data_ptr() % 16 == 0 else _copy_on(t, stream) for t in (k, v))
        check(self.lib.kv_seq_append(self.handle, k.data_ptr(), v.data_ptr(), int(k.shape[2]), sp))

    def load(self, state: "KVState", slot: int = 0, start: int = 0, count: Optional[int] = None, stream=None) -> None:
        """Append rows [start, start + count) of a slot of a KV state, as the slot sees them."""
        if count is None:
            count = state.length - start
        check(self.lib.kv_seq_load(self.handle, state.handle, _count(slot, "slot"), _count(start, "start"), _count(count, "count"),
                                   _pool_stream(self.pool.stage, stream)))

    def read(self, layer: int, start: int = 0, count: Optional[int] = None, stream=None):
        """Rows [start, start + count) of one layer: K, V [Hkv, count, D]."""
        st = self.pool.stage
        if count is None:
            count = self.length - start
        if count < 0:
            raise ValueError("count must not be negative")
        dev = torch.device("cuda", st.device_index)
        sp, empty = _on(st, stream, dev)
        k, v = (empty((st.shape.n_kv_heads, count, st.shape.head_dim), dtype=st.kv_dtype, device=dev) for _ in range(2))
        check(self.lib.kv_seq_read(self.handle, _count(layer, "layer"), _count(start, "start"), _count(count, "count"), k.data_ptr() or 16,
                                   v.data_ptr() or 16, sp))
        return k, v


def _copy_on(t: torch.Tensor, stream) -> torch.Tensor:
    """A contiguous copy made on ``stream`` (None: the current one), where the call that takes it runs."""
    if stream is None:
        return t.clone(memory_format=torch.contiguous_format)
    with torch.cuda.stream(stream):
        return t.clone(memory_format=torch.contiguous_format)


@dataclass
class PagedRequest:
    """One sequence of a step and its ``n_tokens`` new rows: positions int32
    [n_tokens] or [n_axes, n_tokens] (None: rows are not turned), mask [P + n_tokens]
    uint8 (nonzero = visible) or None, mask_rows [n_tokens, P + n_tokens] uint8 (one
    mask per new row) or None.  New row i sees row j iff j <= P + i and both masks
    keep j."""

    seq: PagedSequence
    n_tokens: int
    positions: Optional[np.ndarray] = None
    mask: Optional[np.ndarray] = None
    mask_rows: Optional[np.ndarray] = None


def _step_requests(requests: Sequence[PagedRequest]):
    """The C array of a step's requests, and what has to live as long as its call."""
    arr = (_lib.KVStepRequest * len(requests))()
    keep = []

    def put(a, shape, name):
        if a is None:
            return None
        a = _int32(a, name) if name == "positions" else _mask8(a)
        if a.shape != shape and a.size == int(np.prod(shape)) and len(shape) == 2 and shape[0] == 1:
            a = a.reshape(shape)
        if a.shape != shape:
            raise ValueError(f"{name} must be {list(shape)}, is {list(a.shape)}")
        keep.append(a)
        return a.ctypes.data

    for c, r in zip(arr, requests):
        r.seq._check(r.seq.pool)
        n = _count(r.n_tokens, "n_tokens")
        T = r.seq.length + n
        c.seq, c.n_tokens = r.seq.handle, n
        c.positions = put(r.positions, (r.seq.pool.n_axes, n), "positions")
        c.attention_mask = put(r.mask, (T,), "mask")
        c.attention_mask_rows = put(r.mask_rows, (n, T), "mask_rows")
    return arr, keep


class PagedStep:
    """A batch of sequences with new rows each (``PagePool.new_step``): ``plan`` makes
    room for them, then every layer's rows are written (``write``) and attend
    (``attend``).  Rows are request-major."""

    def __init__(self, pool: PagePool):
        self.pool, self.lib = pool, pool.lib
        sh = pool.stage.shape
        self._nq, self._nk = sh.n_q_heads * sh.head_dim, sh.n_kv_heads * sh.head_dim
        h = ctypes.c_void_p()
        self._handle = None
        check(self.lib.kv_step_create(pool.handle, ctypes.byref(h)))
        self._handle = h.value
        self.rows = self._ws = 0

    @property
    def handle(self):
        if self._handle is None or self.pool.handle is None:
            raise ValueError("the step has been freed")
        return self._handle

    def free(self) -> None:
        h, self._handle = self._handle, None
        if h is not None and self.pool.handle is not None:
            check(self.lib.kv_step_free(h))

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def plan(self, requests: Sequence[PagedRequest], stream=None) -> None:
        """Make room for the new rows of each request's sequence, whose length grows by
        them, and lay out the step.  The plan stands until one of the sequences loses
        rows that it covers, or has a page of them replaced (``compact``, or rows added
        to a shared last page)."""
        for r in requests:
            r.seq._check(self.pool)
        arr, keep = _step_requests(requests)
        check(self.lib.kv_step_plan(self.handle, arr, len(requests), _pool_stream(self.pool.stage, stream)))
        ws = ctypes.c_int64()
        check(self.lib.kv_step_workspace(self.handle, ctypes.byref(ws)))
        self.rows, self._ws = sum(int(r.n_tokens) for r in requests), ws.value

    def _in(self, t: torch.Tensor, width: int, name: str, device=None) -> int:
        ld = _rows(t, name)
        if t.shape[0] != self.rows or t.shape[1] != width or device is not None and t.device != device:
            raise ValueError(f"{name} must be [{self.rows}, {width}]" + ("" if device is None else f" on {device}"))
        return ld

    def write(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, q_out: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
        """Turn q [M, Hq D] and k [M, Hkv D] by the rows' positions, store k and v [M,
        Hkv D] in their rows of the pages, and return q (in the KV dtype, or in
        ``q_out``).  Rows may be parts of wider ones; all of one dtype.  Refused while a
        fork shares a page of the step's new rows."""
        st, dev = self.pool.stage, q.device
        ldq, ldk, ldv = self._in(q, self._nq, "q"), self._in(k, self._nk, "k", dev), self._in(v, self._nk, "v", dev)
        if q.dtype != k.dtype or q.dtype != v.dtype:
            raise ValueError("q, k and v must have one dtype")
        sp, empty = _on(st, stream, dev)
        if q_out is None:
            q_out, ldo = empty((self.rows, self._nq), dtype=st.kv_dtype, device=dev), self._nq
        else:
            ldo = self._in(q_out, self._nq, "q_out", dev)
        check(self.lib.kv_step_write(self.handle, _count(layer, "layer"), q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, _DT_OF[q.dtype],
                                     q_out.data_ptr(), ldo, _DT_OF[q_out.dtype], sp))
        return q_out

    def attend(self, layer: int, q: torch.Tensor, scale: Optional[float] = None, out_dtype: Optional[torch.dtype] = None,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention [M, Hq D] of the turned queries q [M, Hq D] (KV dtype or float32)
        over the rows that they see (``scale`` 1/sqrt(head_dim) by default), in
        ``out_dtype`` (q's by default) or into ``out``; a row that sees none gives
        zeros."""
        st, dev = self.pool.stage, q.device
        ldq = self._in(q, self._nq, "q")
        if q.dtype != torch.float32 and q.dtype != st.kv_dtype:
            raise ValueError("q must be float32 or in the KV dtype")
        if scale is not None and not scale > 0:
            raise ValueError("scale must be positive")
        sp, empty = _on(st, stream, dev)
        if out is None:
            out_dtype = out_dtype or q.dtype
            if out_dtype not in _DT_OF:
                raise ValueError("out_dtype must be float32, float16 or bfloat16")
            out, ldo = empty((self.rows, self._nq), dtype=out_dtype, device=dev), self._nq
        else:
            if out_dtype not in (None, out.dtype):
                raise ValueError("out has another dtype")
            ldo = self._in(out, self._nq, "out", dev)
        room = empty(self._ws, dtype=torch.uint8, device=dev) if self._ws else None
        check(self.lib.kv_step_attend(self.handle, _count(layer, "layer"), q.data_ptr(), _DT_OF[q.dtype], ldq, out.data_ptr(), _DT_OF[out.dtype], ldo,
                                      scale or 0.0, room.data_ptr() if room is not None else None, self._ws, sp))
        return out
