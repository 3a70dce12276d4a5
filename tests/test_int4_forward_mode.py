"""Forward-mode derivatives through layers of 4-bit weights are refused, not dropped: on the CPU, with the products replaced."""
import pytest

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
from torch.autograd import forward_ad  # noqa: E402

from paper_2603_27462_amd import binding  # noqa: E402
from paper_2603_27462_amd.linear import RsrGatedMlp, RsrInt4Linear  # noqa: E402


class _Weight:
    def __init__(self, codes, scales, group, zeros=None):
        self.rows, self.cols = codes.shape
        self.matrix = codes.float() * scales.repeat_interleave(group, dim=1)[:, :self.cols]
        self.device = scales.device


def _matvec(h, v, transposed=False, scale=1.0, dtype=None, out=None, stream=None):
    return (v.float() @ (h.matrix if transposed else h.matrix.t())).to(dtype or torch.float32)


def _gated(gate, up, v, act="silu", dtype=None, out=None, pre=None, stream=None):
    a, b = v.float() @ gate.matrix.t(), v.float() @ up.matrix.t()
    if pre is not None:
        pre.copy_(torch.stack((a, b), dim=1))
    return (torch.relu(a) ** 2 * b).to(dtype or torch.float32)


def _gated_backward(gate, up, pre, dout, act="silu", dtype=None, **rest):
    a, b = torch.relu(pre[:, 0]), pre[:, 1]
    da, db = 2 * dout * b * a, dout * a * a
    return (da @ gate.matrix + db @ up.matrix).to(dtype or torch.float32), torch.stack((da, db), dim=1)


@pytest.fixture
def layers(monkeypatch):
    monkeypatch.setattr(binding, "rsr_preprocess_int4", _Weight)
    monkeypatch.setattr(binding, "rsr_int4_matvec", _matvec)
    monkeypatch.setattr(binding, "rsr_gated", _gated)
    monkeypatch.setattr(binding, "rsr_gated_backward", _gated_backward)
    g = torch.Generator().manual_seed(1)

    def layer(rows, cols):
        codes = torch.randint(-8, 8, (rows, cols), generator=g, dtype=torch.int8)
        return RsrInt4Linear(codes, torch.ones((rows, 1)), cols)

    linear = layer(5, 6)
    return linear, RsrGatedMlp(layer(7, 6), layer(7, 6), layer(6, 7), "relu2")


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("requires_grad", [False, True])
def test_dual_tensors_are_refused(layers, which, requires_grad):
    layer = layers[which]
    x = torch.randn((3, 6), requires_grad=requires_grad)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones((3, 6)))
        with pytest.raises(NotImplementedError, match="reverse mode"):
            layer(dual)
        with torch.no_grad(), pytest.raises(NotImplementedError, match="reverse mode"):
            layer(dual)
        plain = layer(x)                            # inside a level, without a tangent
        assert forward_ad.unpack_dual(plain).tangent is None and plain.requires_grad == requires_grad
    with pytest.raises(RuntimeError):
        torch.func.jvp(layer, (x.detach(),), (torch.ones((3, 6)),))


def test_reverse_mode_as_before(layers):
    for layer in layers:
        x = torch.randn((3, 6), requires_grad=True)
        y = layer(x)
        with torch.no_grad():
            assert torch.equal(layer(x), y) and not layer(x).requires_grad
        y.sum().backward()
        assert x.grad.shape == x.shape
    linear, x = layers[0], torch.randn((3, 6), requires_grad=True)
    linear(x).sum().backward()                      # sums of five whole numbers
    assert torch.equal(x.grad, linear.handle.matrix.sum(dim=0).expand(3, -1))
