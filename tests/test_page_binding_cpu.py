"""The paged cache's binding without a GPU: values that the C types do not hold are
refused, not narrowed to others; any value that is not zero is one in a mask."""
import ctypes
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2608_19147_amd import PagedRequest, PagedSequence, PagePool, _lib, stage as binding


class Lib:
    """Stands for the library: notes what its calls get and succeeds."""

    def __init__(self):
        self.got = []

    def __getattr__(self, name):
        def call(*args):
            self.got.append((name, args))
            if name == "kv_seq_length":
                args[1]._obj.value = 40
            if name == "kv_seq_fork":
                self.lengths = list((ctypes.c_int32 * args[3]).from_address(args[1])) if args[1] else None
                self.keep = [bytes((ctypes.c_uint8 * 40).from_address(p)) if p else None for p in args[2]] if args[2] else None
            if name == "kv_seq_compact":
                self.keep = bytes((ctypes.c_uint8 * 40).from_address(args[1]))
            return 0
        return call


@pytest.fixture
def seq(monkeypatch):
    monkeypatch.setattr(binding, "_pool_stream", lambda stage, stream: 0)
    pool = PagePool.__new__(PagePool)
    pool.stage, pool.lib, pool.handle, pool.n_axes = SimpleNamespace(device_index=0), Lib(), 1, 1
    s = PagedSequence(pool, 7)
    yield s
    s._handle = pool.handle = None


def _ints(p, n):
    return list((ctypes.c_int32 * n).from_address(p))


@pytest.mark.parametrize("positions", [[0, 2 ** 32 + 5], [0, 2 ** 31], [0, -2 ** 31 - 1], [0.0, 0.5], [0.0, float("nan")]])
def test_positions_refused(seq, positions):
    for a in (np.array(positions), torch.tensor(positions)):
        with pytest.raises(ValueError):
            binding._step_requests([PagedRequest(seq, 2, positions=a)])


@pytest.mark.parametrize("dtype", [np.int32, np.int64, np.uint8, np.float64])
def test_positions_taken(seq, dtype):
    arr, keep = binding._step_requests([PagedRequest(seq, 2, positions=np.array([3, 5], dtype))])
    assert _ints(arr[0].positions, 2) == [3, 5]


@pytest.mark.parametrize("dtype,value", [(np.int64, 256), (np.int64, -1), (np.float32, 0.25), (bool, True), (np.uint8, 7), (np.int8, -128)])
def test_masks(seq, dtype, value):
    """What is not zero keeps its row, whatever type it has."""
    mask = np.zeros(42, dtype)
    mask[::3] = value
    arr, keep = binding._step_requests([PagedRequest(seq, 2, mask=mask, mask_rows=np.stack([mask, 0 * mask]).astype(dtype))])
    want = [i % 3 == 0 for i in range(42)]
    got = (ctypes.c_uint8 * 42).from_address(arr[0].attention_mask)
    rows = (ctypes.c_uint8 * 84).from_address(arr[0].attention_mask_rows)
    assert [x != 0 for x in got] == want and [x != 0 for x in rows] == want + [False] * 42
    lib = seq.pool.lib
    for kid in seq.pool.fork([seq, seq], keep=[mask[:40], None]):
        kid._handle = None
    assert [x != 0 for x in lib.keep[0]] == want[:40] and lib.keep[1] is None
    seq.compact(mask[:40])
    assert [x != 0 for x in lib.keep] == want[:40]


@pytest.mark.parametrize("n", [2 ** 32 + 1, 2 ** 31])
def test_counts_refused(seq, n):
    for call in (lambda: binding._step_requests([PagedRequest(seq, n)]), lambda: seq.pool.fork([seq], lengths=[n]),
                 lambda: seq.truncate(n), lambda: seq.load(SimpleNamespace(handle=1, length=n + 3), 0, n, 1),
                 lambda: seq.load(SimpleNamespace(handle=1, length=3), n, 0, 1), lambda: seq.load(SimpleNamespace(handle=1, length=3), 0, 0, n)):
        with pytest.raises(ValueError):
            call()
    assert [name for name, _ in seq.pool.lib.got if name != "kv_seq_length"] == []


def test_lengths_taken(seq):
    for lengths in ([3], np.array([3], np.int64), (np.int32(3),)):
        for kid in seq.pool.fork([seq], lengths=lengths):
            kid._handle = None
        assert seq.pool.lib.lengths == [3]
