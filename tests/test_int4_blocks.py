"""Which layers make a feed-forward block: said when it is made, on the CPU as on the GPU."""
import types

import pytest

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
from paper_2603_27462_amd import binding  # noqa: E402
from paper_2603_27462_amd.linear import RsrGatedMlp, RsrInt4Linear  # noqa: E402


def _layer(rows, cols, group, device="cpu"):
    n = -(-cols // group)
    return RsrInt4Linear(torch.ones((rows, cols), dtype=torch.int8, device=device), torch.ones((rows, n), device=device), group)


# columns, groups of gate and up, whether they go together
PAIRS = [(320, 64, 64, True), (320, 64, 192, True), (320, 128, 256, True), (320, 128, 320, True), (320, 32, 96, True),
         (320, 1000, 128, True), (320, 64, 128, False), (320, 32, 64, False), (320, 32, 1000, False), (320, 64, 256, False)]


@pytest.mark.parametrize("cols,one,other,fit", PAIRS)
def test_groups(monkeypatch, cols, one, other, fit):
    monkeypatch.setattr(binding, "rsr_preprocess_int4",
                        lambda Q, s, group, zeros=None: types.SimpleNamespace(device=Q.device, rows=Q.shape[0], cols=Q.shape[1]))
    gate, up, down = _layer(4, cols, one), _layer(4, cols, other), _layer(cols, 4, 32)
    if fit:
        RsrGatedMlp(gate, up, down)
        up.handle.device = torch.device("meta")
        with pytest.raises(ValueError, match="device"):
            RsrGatedMlp(gate, up, down)
    else:
        with pytest.raises(ValueError, match="groups"):
            RsrGatedMlp(gate, up, down)


@pytest.mark.gpu
@pytest.mark.parametrize("cols,one,other,fit", PAIRS)
def test_as_the_library_has_it(cols, one, other, fit):
    gate, up = _layer(4, cols, one, "cuda:0"), _layer(4, cols, other, "cuda:0")
    x = torch.ones((2, cols), device="cuda:0")
    if fit:
        block = RsrGatedMlp(gate, up, _layer(cols, 4, 32, "cuda:0"), "relu2")
        assert torch.equal(block(x), torch.full((2, cols), 4.0 * cols ** 3, device="cuda:0"))
    else:
        with pytest.raises(rsr.RsrError) as e:
            rsr.rsr_gated(gate.handle, up.handle, x)
        assert e.value.code == 3
