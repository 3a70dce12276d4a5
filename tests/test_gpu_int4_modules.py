"""RsrInt4Linear and RsrGatedMlp: the functions' results, their gradients through autograd, and a block as it is used, at decode, for a
prompt, in a training step and in a graph, against float64."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
from paper_2603_27462_amd import binding  # noqa: E402
from paper_2603_27462_amd.linear import RsrGatedMlp, RsrInt4Linear  # noqa: E402

DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _layer(out_features, in_features, group, seed, dtype=torch.float32, zeros=False):
    """a layer whose rows have about unit norm, and its matrix in 64 bits"""
    g = _gen(seed)
    n = -(-in_features // group)
    Q = torch.randint(-8, 8, (out_features, in_features), generator=g, device=DEV, dtype=torch.int8)
    s = ((0.5 + torch.rand((out_features, n), generator=g, device=DEV)) / (5 * in_features ** 0.5)).to(torch.bfloat16)
    z = torch.randint(-2, 3, (out_features, n), generator=g, device=DEV, dtype=torch.int8) if zeros else None
    M = Q.double() - (0 if z is None else z.double().repeat_interleave(group, dim=1)[:, :in_features])
    M *= s.double().repeat_interleave(group, dim=1)[:, :in_features]
    return RsrInt4Linear(Q, s, group, zeros=z, dtype=dtype), M


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(300,), (1, 300), (2, 3, 300), (0, 300), (4, 0, 300), (70, 300)])
def test_linear(shape, dtype):
    layer, M = _layer(200, 300, 64, 1, dtype, zeros=True)
    x = torch.randn(shape, generator=_gen(2), device=DEV).to(dtype).requires_grad_()
    y = layer(x)
    assert y.shape == (*shape[:-1], 200) and y.dtype == dtype
    with torch.no_grad():
        assert torch.equal(layer(x), y)
    dy = torch.randn(y.shape, generator=_gen(3), device=DEV).to(dtype)
    y.backward(dy)
    assert x.grad.shape == x.shape and x.grad.dtype == dtype
    if y.numel():
        half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
        # sums of 300 and 200 products of at most 24 |s x| (codes, zero points and the offset of 8), rounded once each
        want, size = x.detach().double() @ M.t(), x.detach().double().abs() @ M.abs().clamp(min=24 * 1.5 / (5 * 300 ** 0.5)).t()
        assert bool(((y.double() - want).abs() <= 300 * 2.0 ** -24 * size + half * want.abs()).all())
        want, size = dy.double() @ M, dy.double().abs() @ M.abs().clamp(min=24 * 1.5 / (5 * 300 ** 0.5))
        bound = 232 * 2.0 ** -24 * size + half * want.abs()
        if dtype == torch.bfloat16:
            bound += 2.0 ** -8 * (dy.double().abs() @ M.abs()) * (1 + half)     # dy, scaled, is rounded
        assert bool(((x.grad.double() - want).abs() <= bound).all())


def test_inner_strides_and_gradients_that_are_views():
    layer, M = _layer(64, 96, 32, 4)
    x = torch.randn((96, 7), generator=_gen(5), device=DEV, requires_grad=True)
    y = layer(x.t())
    assert torch.equal(y, layer(x.t().contiguous()))
    y.sum().backward()                              # an expanded gradient: all strides zero
    want = M.sum(dim=0)[:, None].expand(96, 7)
    assert bool(((x.grad.double() - want).abs() <= 96 * 2.0 ** -24 * 24 * 1.5 / (5 * 96 ** 0.5) * 64).all())


def test_native_calls_leave_what_is_not_plain():
    rsr.load_library()
    assert binding._int4 is not None and binding._gated is not None, "not built"
    layer, _ = _layer(64, 96, 32, 4)
    h, x = layer.handle, torch.randn((5, 96), device=DEV)
    want = torch.empty((5, 64), device=DEV)
    rsr.rsr_int4_matvec(h, x, out=want)
    assert torch.equal(binding._int4(h.ptr, 64, 96, x, False, 1.0, False), want)
    assert torch.equal(binding._gated(h.ptr, h.ptr, 64, 96, x, 2, False), rsr.rsr_gated(h, h, x, 2, out=torch.empty_like(want)))
    assert torch.equal(binding._int4(h.ptr, 64, 96, torch.nn.Parameter(x), False, 1.0, False), want)    # (as plain as any)
    for v in (x.cpu(), x.double(), x[:, :95], x.t(), x[:0], x[None], None):
        assert binding._int4(h.ptr, 64, 96, v, False, 1.0, False) is None
        assert binding._gated(h.ptr, h.ptr, 64, 96, v, 0, False) is None
    for args in ((), (h.ptr, 64, 96, x, False, "one", False), (0, 64, 96, x, False, 1.0, False)):
        assert binding._int4(*args) is None
    assert binding._gated(h.ptr, h.ptr, 64, 96, x, 7, False) is None
    with pytest.raises(TypeError):
        rsr.rsr_int4_matvec(h, x, dtype=torch.float16)


def _block(hidden=320, ffn=700, group=64, dtype=torch.float32, seed=10):
    gate, Mg = _layer(ffn, hidden, group, seed, zeros=True)
    up, Mu = _layer(ffn, hidden, group, seed + 1)
    down, Md = _layer(hidden, ffn, 128, seed + 2, dtype)
    return gate, up, down, (Mg, Mu, Md)


def _plain(x, matrices, act):
    Mg, Mu, Md = matrices
    a, b = x @ Mg.t(), x @ Mu.t()
    f = {"silu": lambda: a * torch.sigmoid(a), "relu2": lambda: torch.relu(a) ** 2,
         "gelu": lambda: a * torch.sigmoid((8 / torch.pi) ** 0.5 * (a + 0.044715 * a ** 3))}[act]()
    return (f * b) @ Md.t()


@pytest.mark.parametrize("act", ["silu", "gelu", "relu2"])
@pytest.mark.parametrize("tokens", [1, 4, 30, 200])
def test_block_float32(act, tokens):
    """Float32 throughout: within 2^-14 of the largest value, far more than a few hundred roundings of 2^-24 amount to."""
    gate, up, down, matrices = _block()
    block = RsrGatedMlp(gate, up, down, act)
    x = torch.randn((tokens, 320), generator=_gen(1), device=DEV, requires_grad=True)
    y = block(x)
    x64 = x.detach().double().requires_grad_()
    y64 = _plain(x64, matrices, act)
    assert bool(((y.double() - y64).abs() <= 2.0 ** -14 * y64.abs().max()).all())
    dy = torch.randn(y.shape, generator=_gen(2), device=DEV)
    y.backward(dy)
    y64.backward(dy.double())
    assert bool(((x.grad.double() - x64.grad).abs() <= 2.0 ** -14 * x64.grad.abs().max()).all())
    with torch.no_grad():
        assert torch.equal(block(x), y)


@pytest.mark.parametrize("tokens", [3, 150])
def test_block_bf16(tokens):
    """bf16 in, between and out: every value is rounded a handful of times, 2^-8 each; 16 such of the largest value."""
    gate, up, down, matrices = _block(dtype=torch.bfloat16)
    block = RsrGatedMlp(gate, up, down)
    x = torch.randn((tokens, 320), generator=_gen(3), device=DEV).bfloat16().requires_grad_()
    y = block(x)
    assert y.dtype == torch.bfloat16
    x64 = x.detach().double().requires_grad_()
    y64 = _plain(x64, matrices, "silu")
    assert bool(((y.double() - y64).abs() <= 2.0 ** -4 * y64.abs().max()).all())
    y.backward(torch.ones_like(y))
    y64.sum().backward()
    assert x.grad.dtype == torch.bfloat16
    assert bool(((x.grad.double() - x64.grad).abs() <= 2.0 ** -4 * x64.grad.abs().max()).all())


def test_backward_twice_and_no_second_derivative():
    gate, up, down, _ = _block()
    block = RsrGatedMlp(gate, up, down)
    x = torch.randn((5, 320), generator=_gen(4), device=DEV, requires_grad=True)
    y = block(x).square().sum()
    first, = torch.autograd.grad(y, x, retain_graph=True)
    second, = torch.autograd.grad(y, x, retain_graph=True)
    assert torch.equal(first, second)               # nothing that was kept is overwritten
    g, = torch.autograd.grad(y, x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_training_beside_the_block():
    """An adapter before the block learns through it: its gradient against float64."""
    gate, up, down, matrices = _block()
    block = RsrGatedMlp(gate, up, down)
    A = (0.05 * torch.randn((320, 320), generator=_gen(5), device=DEV)).requires_grad_()
    x = torch.randn((40, 320), generator=_gen(6), device=DEV)
    loss = block(x + x @ A).square().mean()
    loss.backward()
    A64 = A.detach().double().requires_grad_()
    _plain(x.double() + x.double() @ A64, matrices, "silu").square().mean().backward()
    assert bool(((A.grad.double() - A64.grad).abs() <= 2.0 ** -12 * A64.grad.abs().max()).all())


def test_decode_in_a_graph():
    """A decode step of two blocks, captured and replayed with new inputs, against the eager one."""
    blocks = []
    for seed in (10, 20):
        gate, up, down, _ = _block(dtype=torch.bfloat16, seed=seed)
        blocks.append(RsrGatedMlp(gate, up, down))
    x = torch.randn((1, 320), generator=_gen(7), device=DEV).bfloat16()

    def step():
        y = x
        for b in blocks:
            y = y + b(y)
        return y

    with torch.no_grad():
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        for turn in range(4):
            x.copy_(torch.randn((1, 320), generator=_gen(30 + turn), device=DEV).bfloat16())
            want = step()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_blocks_that_do_not_fit():
    gate, up, down, _ = _block()
    with pytest.raises(ValueError):
        RsrGatedMlp(gate, down, up)
    with pytest.raises(ValueError):
        RsrGatedMlp(gate, up, down, "relu")
    with pytest.raises(ValueError):
        RsrGatedMlp(gate, up, down)(torch.zeros((2, 319), device=DEV))
    with pytest.raises(TypeError):
        down(torch.zeros((2, 700), device=DEV, dtype=torch.float16))


def test_tokens_in_one_place():
    """one token, expanded to several, and a gradient that is the same for all tokens"""
    layer, M = _layer(64, 96, 32, 30)
    token = torch.randn(96, generator=_gen(31), device=DEV, requires_grad=True)
    w = torch.randn(64, generator=_gen(32), device=DEV)
    y = layer(token.expand(5, 96))
    want = layer(token.detach().expand(5, 96).contiguous())
    assert torch.equal(y, want)
    (y.sum(dim=0) * w).sum().backward()
    size = w.double().abs() @ M.abs().clamp(min=24 * 1.5 / (5 * 96 ** 0.5))
    # five gradients of sums of 64 products, rounded, and their sum
    assert bool(((token.grad.double() - 5 * (w.double() @ M)).abs() <= 5 * (96 + 6) * 2.0 ** -24 * size).all())
    block = RsrGatedMlp(*_block()[:3])
    x = torch.randn(3, 320, generator=_gen(33), device=DEV, requires_grad=True)
    block(x).sum(dim=0).pow(2).sum().backward()
    got, x.grad = x.grad, None
    y = block(x)
    y.backward((2 * y.detach().sum(dim=0)).expand(3, -1).contiguous())
    assert torch.equal(got, x.grad)
    overlapping = torch.randn(200, generator=_gen(34), device=DEV).as_strided((4, 96), (32, 1))
    assert torch.equal(layer(overlapping), layer(overlapping.clone()))
