"""A forward and backward pass through RsrInt4Linear and RsrGatedMlp, captured together and replayed with new inputs."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
from paper_2603_27462_amd.linear import RsrGatedMlp, RsrInt4Linear  # noqa: E402

DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _layer(rows, cols, group, seed, dtype):
    g = _gen(seed)
    Q = torch.randint(-8, 8, (rows, cols), generator=g, device=DEV, dtype=torch.int8)
    s = ((0.5 + torch.rand((rows, -(-cols // group)), generator=g, device=DEV)) / (5 * cols ** 0.5)).to(torch.bfloat16)
    return RsrInt4Linear(Q, s, group, dtype=dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 5, 200])
def test_forward_and_backward_in_a_graph(tokens, dtype):
    proj = _layer(320, 320, 32, 1, dtype)
    block = RsrGatedMlp(_layer(700, 320, 64, 2, dtype), _layer(700, 320, 64, 3, dtype), _layer(320, 700, 128, 4, dtype))
    x = torch.randn((tokens, 320), generator=_gen(5), device=DEV).to(dtype).requires_grad_()
    dy = torch.randn((tokens, 320), generator=_gen(6), device=DEV).to(dtype)

    def step():
        y = block(proj(x))
        return y.detach(), torch.autograd.grad(y, x, dy)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                      # (its graph is gone before the capture)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = step()
    for turn in range(4):
        with torch.no_grad():
            x.copy_(torch.randn((tokens, 320), generator=_gen(10 + turn), device=DEV))
            dy.copy_(torch.randn((tokens, 320), generator=_gen(20 + turn), device=DEV))
        y.fill_(float("nan"))
        dx.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), dx.clone()
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
