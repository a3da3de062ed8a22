"""Run as a program under tests/hip_host.cpp's stand-in for the HIP runtime: makes a
tiny stage and answers one question about its host code, as JSON.  Without torch,
which would take the stand-in for its own runtime."""
import ctypes
import importlib.util
import json
import os
import struct
import sys

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("_lib", os.path.join(ROOT, "paper_2608_19147_amd", "_lib.py"))
_lib = importlib.util.module_from_spec(spec)
sys.modules["_lib"] = _lib
spec.loader.exec_module(_lib)

H, VOCAB = 256, 30000
lib = _lib.load()
host = ctypes.CDLL(os.environ["LD_PRELOAD"])
host.host_start.argtypes = [ctypes.c_int, ctypes.c_long, ctypes.c_int]
host.host_notes.restype = ctypes.c_char_p
host.host_largest_malloc.restype = ctypes.c_longlong
host.host_fail_malloc.argtypes = [ctypes.c_long]
host.host_live.restype = ctypes.c_long
KEEP = []


def array(a):
    KEEP.append(a)
    return a.ctypes.data


def quant(n, k):
    return _lib.QuantMatrix(q=array(np.zeros((n, k // 2), np.uint8)), scales=array(np.zeros((n, -(-k // 128)), np.float16)), n=n, k=k)


def make_stage():
    dims = {"wq": (256, H), "wk": (128, H), "wv": (128, H), "wo": (H, 256), "wg": (688, H), "wu": (688, H), "wd": (H, 688)}
    layer = _lib.LayerWeights(attn_norm=array(np.zeros(H, np.uint16)), ffn_norm=array(np.zeros(H, np.uint16)),
                              **{name: quant(n, k) for name, (n, k) in dims.items()})
    cfg = _lib.StageConfig(n_layers=1, hidden=H, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn=688, group_size=128, rms_eps=1e-5,
                           act_dtype=_lib.DTYPE_BF16, kv_dtype=_lib.DTYPE_BF16, rope_theta=10000.0, max_positions=64, rope_cos_sin=None)
    h = ctypes.c_void_p()
    assert lib.stage_create(ctypes.byref(cfg), ctypes.byref(layer), 0, None, ctypes.byref(h)) == 0, lib.stage_last_error()
    return h


def mx4(n, k):
    return array(np.zeros((n, (k + 1) // 2), np.uint8)), array(np.zeros((n, (k + 31) // 32), np.uint8))


def attach(st, kind):
    norm = array(np.zeros(H, np.uint16))
    if kind == "mx4":
        rc = lib.stage_head_attach_mx4(st, norm, *mx4(VOCAB, H), VOCAB, 0, None)
    else:
        rc = lib.stage_head_attach(st, norm, ctypes.byref(quant(VOCAB, H)), 0, None)
    assert rc == 0, lib.stage_last_error()


def call(st, name):
    """The named call as a function of its stream; returns the status."""
    room = array(np.zeros(1 << 22, np.float32))               # stands for every device array
    params = struct.pack("=fiff", 1.0, 0, 1.0, 0.0) * 64
    if name.startswith("product"):
        m, n, k = {"product": (300, 4096, 4096), "product_passes": (2100, 520, 8200), "product_one_pass": (2000, 4096, 512)}[name]
        h = ctypes.c_void_p()
        assert lib.stage_mx4_create(st, *mx4(n, k), n, k, 0, None, ctypes.byref(h)) == 0
        return lambda s: lib.stage_mx4_product(h, room, _lib.DTYPE_BF16, k, m, 16, room, _lib.DTYPE_F32, n, s)
    if name == "sample":
        return lambda s: lib.stage_sample(st, room, _lib.DTYPE_F32, VOCAB, 20, VOCAB, params, room, room, room, s)
    attach(st, "int4" if "int4" in name else "mx4")
    if "top1" in name:
        return lambda s: lib.stage_head_top1(st, room, 20, room, room, None, room if "logits" in name else None, s)
    return lambda s: lib.stage_head_sample(st, room, 20, params, room, room, room, room if "logits" in name else None, s)


def notes():
    return [line.split() for line in host.host_notes().decode().splitlines()]


def order(name):
    """Per launch that fails: is the next call on another stream ordered behind those that had been queued?"""
    out = []
    for at in range(2, 40):
        st = make_stage()
        f = call(st, name)
        host.host_start(at, 0, 0)
        rc = f(1)
        got = notes()
        if rc == 0:
            break
        host.host_start(0, 0, 0)
        rc2 = f(2)
        after = notes()
        recorded = [i for i, n in enumerate(got) if n[0] == "R" and n[1] == "1"]
        launched = [i for i, n in enumerate(got) if n[0] == "L"]
        first = [n[0] for n in after].index("L")
        waits = [n[2] for n in after[:first] if n[0] == "W" and n[1] == "2"]
        out.append(dict(at=at, rc=rc, rc2=rc2, queued=len(launched),
                        ordered=bool(recorded and recorded[-1] > launched[-1] and got[recorded[-1]][2] in waits)))
        lib.stage_destroy(st)
    return out


def allocations(name, capture):
    """Statuses of the call while its first, second, ... host allocation fails, up to the one that needs no more."""
    out = []
    for n in range(1, 40):
        st = make_stage()
        f = call(st, name)
        host.host_start(0, n, int(capture))
        rc = f(1)
        host.host_start(0, 0, 0)
        out.append(rc)
        lib.stage_destroy(st)
        if rc != -4:
            break
    return out


def largest_allocation(name):
    """Bytes of the largest device allocation that the stage's first such call makes, beside a [64][VOCAB] array of logits."""
    st = make_stage()
    f = call(st, name)
    host.host_start(0, 0, 0)
    assert f(1) == 0
    return host.host_largest_malloc(), 64 * VOCAB * 4


def weights_without_memory(name):
    """Per device allocation that fails while weights are packed: the status, and what the failed call leaves allocated; at
    last those of the call with memory."""
    out = []
    norm, (codes, scales) = array(np.zeros(H, np.uint16)), mx4(VOCAB, H)
    h = ctypes.c_void_p()
    st = make_stage()
    for n in range(1, 20):
        host.host_start(0, 0, 0)
        had = host.host_live()
        host.host_fail_malloc(n)
        if name == "head":
            rc = lib.stage_head_attach_mx4(st, norm, codes, scales, VOCAB, 0, None)
        else:
            rc = lib.stage_mx4_create(st, codes, scales, VOCAB, H, 0, None, ctypes.byref(h))
        host.host_fail_malloc(0)
        out.append((rc, host.host_live() - had, host.host_last_error()))
        if rc == 0:
            break
    return out


if __name__ == "__main__":
    print(json.dumps(globals()[sys.argv[1]](*sys.argv[2:])))
