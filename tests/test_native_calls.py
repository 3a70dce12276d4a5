"""The native calls for new results are used all together or not at all."""
import pytest

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
from paper_2603_27462_amd import binding  # noqa: E402


class _Used(Exception):
    pass


def _used(*args):
    raise _Used


def test_those_of_4_bit_weights_follow_the_product(monkeypatch):
    rsr.load_library()
    product = binding._product
    assert product is not None, "not built"
    # a library loaded under another torch turns all of them off
    monkeypatch.setattr(binding, "_product", product)
    monkeypatch.setattr(binding, "_int4", binding._int4)
    monkeypatch.setattr(binding, "_gated", binding._gated)
    with monkeypatch.context() as other:
        other.setattr(binding._build, "torch_tag", lambda: "another torch", raising=False)
        with pytest.warns(UserWarning, match="another torch"):
            binding._load_call(rsr.load_library())
    assert binding._product is None
    h, x = rsr.Handle(0, 4, 64, 0, rsr.RSR_INT4), torch.zeros(64)
    h.device = torch.device("cuda", 0)
    if binding._int4 is not None:
        monkeypatch.setattr(binding, "_int4", _used)
        monkeypatch.setattr(binding, "_gated", _used)
    for call in (lambda: rsr.rsr_int4_matvec(h, x), lambda: rsr.rsr_gated(h, h, x)):
        with pytest.raises(TypeError):              # refused by the path through ctypes
            call()
    # and where the product's is there again, so are they
    binding._product = product
    monkeypatch.setattr(binding, "_int4", binding._int4 and _used)
    monkeypatch.setattr(binding, "_gated", binding._gated and _used)
    for call in (lambda: rsr.rsr_int4_matvec(h, x), lambda: rsr.rsr_gated(h, h, x)):
        with pytest.raises(_Used):
            call()
