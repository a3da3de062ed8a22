"""The last stage's operators without a GPU: refusals that come before any device
work, the drafted tree's bookkeeping, and the binding's argument forms."""
import ctypes
import os
import struct
import subprocess
import sys
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2608_19147_amd import Sampling, _lib
from paper_2608_19147_amd.driver import VerifyDriver

F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2608_19147_amd import build

        build.build()
    return _lib.load()


BUF = ctypes.create_string_buffer(1 << 16)                 # stands for handles and arrays whose contents a refusal never uses
P = ctypes.addressof(BUF)


def _params(*q):
    return b"".join(struct.pack("=fiff", *v) for v in q)


GOOD = (1.0, 0, 1.0, 0.0)


@pytest.mark.parametrize("args,code", [
    ((None, P, F32, 8, 1, 8, _params(GOOD), P, P, P), -1),
    ((P, None, F32, 8, 1, 8, _params(GOOD), P, P, P), -1),
    ((P, P, F32, 8, 1, 8, None, P, P, P), -1),
    ((P, P, F32, 8, 1, 8, _params(GOOD), None, P, P), -1),
    ((P, P, 3, 8, 1, 8, _params(GOOD), P, P, P), -1),
    ((P, P, F32, 8, 0, 8, _params(GOOD), P, P, P), -3),
    ((P, P, F32, 8, 65, 8, _params(*[GOOD] * 65), P, P, P), -3),
    ((P, P, F32, 8, 1, 0, _params(GOOD), P, P, P), -2),
    ((P, P, F32, 1 << 21, 1, (1 << 20) + 1, _params(GOOD), P, P, P), -3),
    ((P, P, F32, 7, 1, 8, _params(GOOD), P, P, P), -2),
    ((P, P, F32, 8, 2, 8, _params(GOOD, (-0.5, 0, 1.0, 0.0)), P, P, P), -1),
    ((P, P, F32, 8, 1, 8, _params((1.0, -1, 1.0, 0.0)), P, P, P), -1),
    ((P, P, F32, 8, 1, 8, _params((1.0, 0, 0.0, 0.0)), P, P, P), -1),
    ((P, P, F32, 8, 1, 8, _params((1.0, 0, 1.0, float("nan"))), P, P, P), -1),
    ((P, P, F32, 8, 1, 8, _params((float("inf"), 0, 1.0, 0.0)), P, P, P), -1),
])
def test_sample_refused(lib, args, code):
    assert lib.stage_sample(*args, None) == code
    assert lib.stage_last_error()


@pytest.mark.parametrize("args,code", [
    ((None, P, F32, 8, 1, 8, P, P), -1), ((P, P, 5, 8, 1, 8, P, P), -1), ((P, P, F32, 8, 0, 8, P, P), -1), ((P, P, F32, 8, 1, 0, P, P), -1),
    ((P, P, F32, 7, 1, 8, P, P), -2), ((P, P, F32, 1 << 25, 1, 1 << 25, P, P), -3), ((P, P, F32, 1 << 20, 1 << 20, 1 << 20, P, P), -3),
])
def test_quantize_refused(lib, args, code):
    assert lib.stage_mx4_quantize(*args, None) == code
    s, x, dt, ld, m, k, c, sc = args
    assert lib.stage_mx4_dequantize(s, c, sc, m, k, x, dt, ld, None) == code


def test_matrix_refused(lib):
    h = ctypes.c_void_p()
    assert lib.stage_mx4_create(None, P, P, 4, 4, 0, None, ctypes.byref(h)) == -1
    assert lib.stage_mx4_create(P, P, None, 4, 4, 0, None, ctypes.byref(h)) == -1
    assert lib.stage_mx4_create(P, P, P, 0, 4, 0, None, ctypes.byref(h)) == -1
    assert lib.stage_mx4_create(P, P, P, 1 << 20, 1 << 20, 0, None, ctypes.byref(h)) == -3
    assert lib.stage_mx4_free(None) == -1
    ok = dict(x=P, dt=BF16, ldx=64, m=1, act=16, out=P, odt=F32, ldo=64)   # a zeroed matrix has n = k = 0

    def call(w=P, **kw):
        a = {**ok, **kw}
        return lib.stage_mx4_product(w, a["x"], a["dt"], a["ldx"], a["m"], a["act"], a["out"], a["odt"], a["ldo"], None)

    assert call(None) == -1 and call(x=None) == -1 and call(out=None) == -1
    assert call(dt=9) == -1 and call(odt=-1) == -1 and call(act=8) == -1
    assert call(dt=F32) == -7
    assert call(m=0) == -3 and call(m=_lib.MAX_PREFILL + 1) == -3
    assert call(ldx=-1) == -2 and call(ldo=-1) == -2


def test_head_refused(lib):
    assert lib.stage_head_attach_mx4(None, P, P, P, 8, 0, None) == -1
    assert lib.stage_head_attach_mx4(P, P, P, P, 0, 0, None) == -2
    assert lib.stage_head_attach_mx4(P, P, P, P, (1 << 20) + 1, 0, None) == -3
    assert lib.stage_head_sample(P, P, 1, _params(GOOD), P, P, P, None, None) == -1 and b"no head" in lib.stage_last_error()


def test_tree_refused(lib):
    good = [P, P, P, P, 1, 4, P, P, P, P]
    for i in (0, 1, 2, 3, 6, 7, 8, 9):
        assert lib.stage_tree_accept(*[None if j == i else a for j, a in enumerate(good)], None) == -1
    assert lib.stage_tree_accept(P, P, P, P, 0, 4, P, P, P, P, None) == -1
    assert lib.stage_tree_accept(P, P, P, P, 1, 0, P, P, P, P, None) == -3
    assert lib.stage_tree_accept(P, P, P, P, 1, 65, P, P, P, P, None) == -3


def test_sampling_struct():
    q = Sampling(0.5, 7, 0.25, 0.125)
    assert struct.unpack("=fiff", q.packed) == (0.5, 7, 0.25, 0.125)
    assert q == Sampling(0.5, 7, 0.25, 0.125) and hash(q) == hash(Sampling(0.5, 7, 0.25, 0.125))


def test_tree_inputs():
    """Positions are the valid rows plus the depth; a node sees the valid rows, its ancestors and itself."""
    d = VerifyDriver(2, 3)
    d.valid[1, 1] = 0
    parents = np.array([[-1, 0, 0, 1, 3], [-1, 0, 1, 2, 0]])
    pos, rows, beam = d.tree_inputs(parents)
    assert beam is None and rows.shape == (2, 5, 8) and rows.dtype == np.uint8
    assert pos.tolist() == [[3, 4, 4, 5, 6], [2, 3, 4, 5, 3]]
    for b in range(2):
        for i in range(5):
            see, j = set(), i
            while True:
                see.add(j)
                if j == 0:
                    break
                j = int(parents[b, j])
            assert set(np.flatnonzero(rows[b, i, 3:])) == see
            assert (rows[b, i, :3] == d.valid[b]).all()
    kept = d.accept_tree(np.array([[1, 0, 1, 0, 0], [1, 1, 1, 0, 0]], np.uint8))
    assert kept.tolist() == [2, 3]
    assert d.valid.tolist() == [[1, 1, 1, 1, 0, 1, 0, 0], [1, 0, 1, 1, 1, 1, 0, 0]]
    pos, _, beam = d.tree_inputs(np.array([[-1], [-1]]), np.array([1, 1]))
    assert pos.tolist() == [[5], [5]] and beam.tolist() == [1, 1]


def test_largest_launches(lib):
    """Sizes whose launch would not fit are refused before anything is read."""
    assert lib.stage_tree_accept(P, P, P, P, (1 << 24) + 1, 4, P, P, P, P, None) == -3
    assert lib.stage_mx4_quantize(P, P, F32, 1 << 18, 1 << 17, 1 << 18, P, P, None) == -3
    assert lib.stage_mx4_dequantize(P, P, P, 1 << 18, 1 << 17, P, F32, 1 << 17, None) == -3


def test_tree_inputs_refused():
    d = VerifyDriver(1, 2)
    for bad in (np.array([[-1, 1]]), np.array([[-1, 0, 2]]), np.array([[-1, -1]]), np.zeros((2, 3), int), np.zeros((1, 0), int)):
        with pytest.raises(ValueError):
            d.tree_inputs(bad)
    with pytest.raises(ValueError):
        d.accept_tree(np.ones((2, 2)))


def test_chain_is_step_inputs():
    """A chain as a tree has the positions and the visible rows of a linear verify."""
    d = VerifyDriver(2, 4)
    d.valid[0, 2] = 0
    pos, mask, _ = d.step_inputs(3)
    tpos, rows, _ = d.tree_inputs(np.array([[-1, 0, 1]] * 2))
    assert (pos == tpos).all()
    tri = np.tril(np.ones((3, 3), np.uint8))
    assert (rows == mask[:, None] * np.concatenate([np.ones((3, 4), np.uint8), tri], 1)[None]).all()


def test_import_without_cuda_names():
    """The package, its driver and its binding import with a torch that has no streams, as CPU builds of it have none."""
    code = ("import torch\ndel torch._C._cuda_getCurrentRawStream\n"
            "import paper_2608_19147_amd.stage as s, paper_2608_19147_amd.driver\nassert callable(s._raw_stream)")
    subprocess.run([sys.executable, "-c", code], check=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


class _Lib:
    """Takes every call of the binding and notes its arguments."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


def test_weights_go_by_the_stage_device(monkeypatch):
    """MXFP4 weights are packed on the current stream of the stage's device, whatever device is current, or on a stream of
    that device; a stream of another one is refused."""
    from paper_2608_19147_amd import Mx4Matrix, Stage, stage as binding

    monkeypatch.setattr(binding, "_raw_stream", lambda index: 1000 + index)
    st = Stage.__new__(Stage)
    st.lib, st.handle, st.device_index = _Lib(), None, 3
    st.shape, st.act_dtype = SimpleNamespace(hidden=64), torch.float16
    codes, scales, norm = torch.zeros((5, 32), dtype=torch.uint8), torch.zeros((5, 2), dtype=torch.uint8), torch.ones(64, dtype=torch.float16)
    makers = (lambda **kw: Mx4Matrix(st, codes, scales, 64, **kw), lambda **kw: st.attach_head_mx4(norm, codes, scales, **kw))
    for make in makers:
        make()
        assert st.lib.calls[-1][1][6] == 1003
        make(stream=SimpleNamespace(device=torch.device("cuda", 3), cuda_stream=77))
        assert st.lib.calls[-1][1][6] == 77
        with pytest.raises(ValueError, match="stream"):
            make(stream=SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=77))


@pytest.mark.parametrize("parents,beam", [([[-1, 1], [-1, 0]], [1, 0]), ([[-1, 0]], [1, 0]), ([[-1, 0], [-1, 0]], [0]), ([[-1, 0], [-1, 0]], [0, 2])])
def test_refused_tree_leaves_the_slots(parents, beam):
    """A tree or an order of the slots that is refused has not reordered them: the call can be made again."""
    d = VerifyDriver(2, 3)
    d.valid[0, 2] = 0
    was = d.valid.copy()
    with pytest.raises((ValueError, IndexError)):
        d.tree_inputs(np.array(parents), np.array(beam))
    assert np.array_equal(d.valid, was) and d.n_slots == 2
    pos, _, _ = d.tree_inputs(np.array([[-1, 0]] * 2), np.array([1, 0]))
    assert pos.tolist() == [[3, 4], [2, 3]]


def test_kept_nodes_are_those_of_the_tree():
    """The nodes recorded are those of the last forward's tree: another number of them would shift every later mask."""
    d = VerifyDriver(2, 3)
    d.tree_inputs(np.array([[-1, 0, 1]] * 2))
    for n in (2, 4):
        with pytest.raises(ValueError):
            d.accept_tree(np.ones((2, n), np.uint8))
    assert d.physical_len == 3
    assert d.accept_tree(np.array([[1, 1, 0], [1, 0, 0]], np.uint8)).tolist() == [2, 1]
    assert d.physical_len == 6
