"""A handle has one owner, however it or a module around it is copied: on the CPU, with the library replaced."""
import copy
import io
import pickle

import pytest

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
from paper_2603_27462_amd import binding  # noqa: E402
from paper_2603_27462_amd.linear import RsrGatedMlp, RsrInt4Linear  # noqa: E402


class _Library:
    freed = []

    def rsr_destroy(self, ptr):
        self.freed.append(ptr)


def _handle(Q, scales, group, zeros=None):
    _handle.ptr += 1
    h = rsr.Handle(_handle.ptr, Q.shape[0], Q.shape[1], 0, rsr.RSR_INT4)
    h.device = Q.device
    return h


@pytest.fixture
def freed(monkeypatch):
    monkeypatch.setattr(binding, "load_library", _Library)
    monkeypatch.setattr(binding, "rsr_preprocess_int4", _handle)
    _Library.freed, _handle.ptr = [], 1000
    return lambda: list(_Library.freed)


def _layer(rows, cols):
    return RsrInt4Linear(torch.ones((rows, cols), dtype=torch.int8), torch.ones((rows, 1)), cols)


def test_copies_of_a_handle(freed):
    h = _handle(torch.ones((4, 64), dtype=torch.int8), None, 64)
    copies = [copy.copy(h), copy.deepcopy(h)]
    del h
    assert freed() == []
    rsr.rsr_destroy(copies.pop())
    assert freed() == [1001]
    del copies
    assert freed() == [1001]


def test_copies_of_modules(freed):
    block = RsrGatedMlp(_layer(8, 4), _layer(8, 4), _layer(4, 8))
    other = copy.deepcopy(torch.nn.Sequential(block, _layer(4, 4)))
    assert other[0] is not block and other[0].gate.handle is block.gate.handle
    del block
    assert freed() == [] and other[1].handle.ptr == 1004
    del other
    assert sorted(freed()) == [1001, 1002, 1003, 1004]


def test_not_pickled(freed):
    layer = _layer(8, 4)
    for write in (lambda: pickle.dumps(layer.handle), lambda: torch.save(layer, io.BytesIO()), lambda: torch.save(layer.handle, io.BytesIO())):
        with pytest.raises(TypeError, match="not pickled"):
            write()
    assert freed() == []
