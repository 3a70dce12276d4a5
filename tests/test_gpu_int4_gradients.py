"""Input gradients in bf16 through 4-bit weights: rounded once, in the result.

Vectors are small whole numbers and scales bf16 with all of their eight bits, in steps of 2^-7, so that a scaled vector needs more
bits than a bf16 has while every partial sum, in any order, is a float32: sums of n products are below 2^17 (checked on the result;
terms have either sign).  Results have to be the exact ones, rounded to nearest even."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
DEV = "cuda:0"
BF16 = torch.bfloat16

# rows, cols, group, batch, zeros
SIZES = [(1, 1, 32, 1, True), (40, 300, 32, 5, True), (100, 500, 128, 16, False), (2050, 130, 64, 16, True), (2100, 260, 32, 3, False),
         (333, 700, 96, 40, True), (500, 2000, 128, 33, False), (1001, 8000, 128, 200, True), (1000, 8003, 128, 400, False),
         (300, 14000, 64, 600, True), (257, 4000, 32, 300, True)]


def _weight(rows, cols, group, zeros, seed):
    """codes, scales, zeros, and the matrix in 64 bits"""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = -(-cols // group)
    Q = torch.randint(-8, 8, (rows, cols), generator=g, device=DEV, dtype=torch.int8)
    s = 1.0 + torch.randint(0, 128, (rows, n), generator=g, device=DEV) / 128.0
    z = torch.randint(-8, 8, (rows, n), generator=g, device=DEV, dtype=torch.int8) if zeros else None
    M = Q.double()
    if zeros:
        M -= z.double().repeat_interleave(group, dim=1)[:, :cols]
    return Q, s, z, M * s.double().repeat_interleave(group, dim=1)[:, :cols]


def _whole(shape, most, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV).float()


@pytest.mark.parametrize("rows,cols,group,batch,zeros", SIZES)
def test_gradients_are_rounded_once(rows, cols, group, batch, zeros):
    Q, s, z, M = _weight(rows, cols, group, zeros, rows)
    h = rsr.rsr_preprocess_int4(Q, s, group, zeros=z)
    y = _whole((batch, rows), 7, 2).to(BF16)
    want = y.double() @ M
    assert want.abs().max() < 2 ** 17
    got = rsr.rsr_int4_matvec(h, y, transposed=True, dtype=BF16)
    assert torch.equal(got, want.to(BF16))


@pytest.mark.parametrize("rows,cols,group,batch,zeros", SIZES)
def test_gradients_of_the_gated_block_are_rounded_once(rows, cols, group, batch, zeros):
    """relu2 of whole numbers: da = 2 dh b a and db = dh a^2 are whole too, up to 16."""
    Qg, sg, zg, Mg = _weight(rows, cols, group, zeros, rows)
    Qu, su, zu, Mu = _weight(rows, cols, group, not zeros, rows + 1)
    gate, up = rsr.rsr_preprocess_int4(Qg, sg, group, zeros=zg), rsr.rsr_preprocess_int4(Qu, su, group, zeros=zu)
    pre, dh = _whole((batch, 2, rows), 2, 3), _whole((batch, rows), 2, 4).to(BF16)
    dv, dpre = rsr.rsr_gated_backward(gate, up, pre, dh, "relu2", dtype=BF16)
    a, b, d = torch.relu(pre[:, 0]), pre[:, 1], dh.float()
    assert torch.equal(dpre, torch.stack((2 * d * b * a, d * a * a), dim=1))
    want = dpre[:, 0].double() @ Mg + dpre[:, 1].double() @ Mu
    assert want.abs().max() < 2 ** 17
    assert torch.equal(dv, want.to(BF16))


@pytest.mark.parametrize("batch", [3, 40, 300])
def test_float32_scales_keep_sixteen_bits(batch):
    """Scales of 24 bits: a scaled vector is off by 2^-16 of itself at most, sums of 60 products by 92 roundings (see
    test_gpu_int4.py), the result by half a step, 2^-8."""
    rows, cols, group = 60, 3000, 128
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    Q = torch.randint(-8, 8, (rows, cols), generator=g, device=DEV, dtype=torch.int8)
    s = torch.randn((rows, -(-cols // group)), generator=g, device=DEV)
    wide = s.double().repeat_interleave(group, dim=1)[:, :cols]
    M, T = Q.double() * wide, (Q.double() + 16.0) * wide.abs()
    y = torch.randn((batch, rows), generator=g, device=DEV).to(BF16)
    got = rsr.rsr_int4_matvec(rsr.rsr_preprocess_int4(Q, s, group), y, transposed=True, dtype=BF16).double()
    want, size = y.double() @ M, y.double().abs()
    bound = (2.0 ** -16 + (rows + 32) * 2.0 ** -24) * (size @ T) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    assert bool(((got - want).abs() <= bound).all())
