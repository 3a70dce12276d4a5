"""4-bit weights with group scales: products, input gradients and the gated block against their definitions in 64 bits.

Exact cases: whole-numbered vectors and scales that are powers of two (or, where nothing is rounded below float32, such
with a factor 1 + 2^-8), so that every partial sum in any order is a float32 and results have to be equal, and for
a bf16 result the exact one rounded to nearest even.

Tolerances of the others, from the formulas.  A product adds s_g (sum u x - (8 + z) sum x) over its groups: with T = sum
s (u + 8 + z) |x| and at most P additions on a path to the result (128 in a group, one per group, 32 at the joins) its
error is at most P 2^-24 T; the transpose adds over the rows, P = rows + 32.  A vector that is scaled and rounded to bf16 adds
2^-8 sum |M| |v|, a bf16 result 2^-8 of itself.  Activations: exp and the reciprocal are exact to a few units in the last
place and the exponent t (silu: a, gelu: sqrt(8/pi) (a + 0.044715 a^3), five roundings) is off by a few 2^-24 |t|, which is
its relative error in exp(t): act, its derivative and what they are multiplied with are within 2^-20 (1 + |t|) of the
factors beside them."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _weight(rows, cols, group, zeros, seed, exact=None):
    """codes, scales, zeros; exact: "pow2" or "wide" (see above), None: any float32 scales, "bf16": any bf16 ones"""
    g = _gen(seed)
    n = -(-cols // group)
    Q = torch.randint(-8, 8, (rows, cols), generator=g, device=DEV, dtype=torch.int8)
    if exact in ("pow2", "wide"):
        s = torch.exp2(torch.randint(-1, 2, (rows, n), generator=g, device=DEV).float())
        s = torch.where(torch.rand((rows, n), generator=g, device=DEV) < 0.3, -s, s)
        if exact == "wide":
            s = s * (1.0 + 2.0 ** -8)
    else:
        s = torch.randn((rows, n), generator=g, device=DEV) / 16
        if exact == "bf16":
            s = s.to(BF16).float()
    z = torch.randint(-8, 8, (rows, n), generator=g, device=DEV, dtype=torch.int8) if zeros else None
    return Q, s, z


def _wide(x, group, cols):
    return x.double().repeat_interleave(group, dim=1)[:, :cols]


def _matrix(w, group):
    """M, and the sizes of the terms that the kernels add, in 64 bits"""
    Q, s, z = w
    cols = Q.shape[1]
    s, z = _wide(s, group, cols), 0.0 if z is None else _wide(z, group, cols)
    q = Q.double()
    return (q - z) * s, (q + 8.0 + 8.0 + z) * s.abs()


def _handle(w, group):
    return rsr.rsr_preprocess_int4(w[0], w[1], group, zeros=w[2])


def _vectors(batch, length, dtype, seed, pad, whole):
    """[batch][length] inside a buffer with `pad` NaNs between the vectors"""
    g = _gen(seed)
    buf = torch.full((batch, length + pad), float("nan"), device=DEV, dtype=dtype)
    x = torch.randint(-4, 5, (batch, length), generator=g, device=DEV).float() if whole else \
        torch.randn((batch, length), generator=g, device=DEV)
    buf[:, :length] = x.to(dtype)
    return buf[:, :length]


def _out(batch, length, dtype, pad):
    buf = torch.full((batch, length + pad), -77.0, device=DEV, dtype=dtype)
    return buf, buf[:, :length]


# sizes on both sides of tiles, groups, row groups and vectors per workgroup
SIZES = [
    # rows, cols, group, batch, vectors, result, zeros, scales, pad
    (1, 1, 32, 1, BF16, F32, False, "pow2", 0), (1, 33, 32, 2, F32, F32, True, "wide", 1),
    (15, 31, 64, 1, F32, BF16, True, "pow2", 0), (16, 256, 128, 4, BF16, BF16, False, "wide", 0),
    (17, 257, 96, 3, BF16, F32, True, "pow2", 1), (33, 511, 1000, 5, F32, F32, False, "wide", 3),
    (100, 300, 256, 16, BF16, F32, True, "wide", 1), (64, 640, 32, 17, BF16, BF16, False, "pow2", 8),
    (129, 129, 64, 33, F32, F32, True, "wide", 1), (640, 2560, 128, 1, BF16, F32, False, "pow2", 0),
    (640, 2560, 64, 4, F32, F32, True, "wide", 0), (1001, 2999, 32, 3, F32, F32, True, "wide", 1),
    (500, 4111, 128, 1, F32, BF16, False, "wide", 0), (2100, 777, 64, 2, BF16, BF16, True, "pow2", 2),
    (48, 9000, 128, 7, BF16, F32, False, "pow2", 0), (300, 1111, 32, 12, F32, F32, True, "wide", 1),
    (257, 1300, 64, 40, BF16, F32, True, "wide", 4), (130, 2048, 128, 64, F32, BF16, False, "pow2", 0),
    (1030, 513, 128, 129, BF16, BF16, True, "pow2", 8), (1200, 1024, 32, 100, F32, F32, False, "wide", 0),
    (2048, 700, 64, 300, BF16, F32, False, "pow2", 4), (2500, 900, 128, 260, F32, F32, True, "wide", 3),
    (4096, 512, 128, 513, BF16, BF16, False, "wide", 0), (4100, 320, 32, 520, BF16, F32, True, "pow2", 1),
]


@pytest.mark.parametrize("rows,cols,group,batch,dtype,result,zeros,scales,pad", SIZES)
def test_products_exact(rows, cols, group, batch, dtype, result, zeros, scales, pad):
    w = _weight(rows, cols, group, zeros, rows + cols, scales)
    M, _ = _matrix(w, group)
    h = _handle(w, group)
    assert (h.rows, h.cols, h.kind) == (rows, cols, rsr.RSR_INT4)
    v = _vectors(batch, cols, dtype, batch, pad, True)
    buf, out = _out(batch, rows, result, 3)
    rsr.rsr_int4_matvec(h, v, scale=-0.5, out=out)
    want = -0.5 * (v.double() @ M.t())
    assert want.abs().max() < 2 ** 15               # (in units of 2^-9: a float32)
    assert torch.equal(out, want.to(result))
    assert bool((buf[:, rows:] == -77.0).all())
    if result == F32:
        assert torch.equal(rsr.rsr_matvec_ex(h, v, scale=-0.5), out)
        one = rsr.rsr_matvec_ex(h, v[0], scale=-0.5)
        assert one.shape == (rows,) and torch.equal(one, out[0])
        if dtype == F32:
            assert torch.equal(rsr.rsr_matvec(h, v[0]), -2.0 * out[0])


@pytest.mark.parametrize("rows,cols,group,batch,dtype,result,zeros,scales,pad", SIZES)
def test_transposed_exact(rows, cols, group, batch, dtype, result, zeros, scales, pad):
    if dtype == BF16 and result == BF16:
        scales = "pow2"                             # (the scaled vector is rounded to bf16)
    w = _weight(rows, cols, group, zeros, 2 * rows + cols, scales)
    M, _ = _matrix(w, group)
    h = _handle(w, group)
    v = _vectors(batch, rows, dtype, batch + 1, pad, True)
    buf, out = _out(batch, cols, result, 3)
    rsr.rsr_int4_matvec(h, v, transposed=True, scale=-0.5, out=out)
    want = -0.5 * (v.double() @ M)
    assert want.abs().max() < 2 ** 15
    assert torch.equal(out, want.to(result))
    assert bool((buf[:, cols:] == -77.0).all())
    one = rsr.rsr_int4_matvec(h, v[0], transposed=True, scale=-0.5, dtype=result)
    assert one.shape == (cols,) and torch.equal(one, out[0])


def test_transposed_float32_scales_in_a_bf16_product():
    """A handle of float32 scales in the product that rounds the scaled vector: the odd scales meet zeros."""
    rows, cols, group = 200, 640, 64
    w = _weight(rows, cols, group, True, 5, "pow2")
    w[1][7::16] *= 1.0 + 2.0 ** -20
    v = _vectors(150, rows, BF16, 6, 0, True)
    v[:, 7::16] = 0.0
    M, _ = _matrix(w, group)
    h = _handle(w, group)
    for n in (1, 20, 150):
        got = rsr.rsr_int4_matvec(h, v[:n], transposed=True, dtype=BF16)
        assert torch.equal(got, (v[:n].double() @ M).to(BF16))


@pytest.mark.parametrize("rows,cols,group,batch,dtype,result,zeros,scales", [
    (640, 2560, 128, 1, F32, F32, False, None), (640, 2560, 64, 3, BF16, F32, True, "bf16"), (1001, 2999, 32, 5, F32, F32, True, None),
    (96, 14336, 128, 1, BF16, F32, True, "bf16"), (300, 5000, 96, 16, F32, BF16, True, None), (512, 1500, 128, 50, BF16, BF16, False, "bf16"),
    (1111, 2222, 64, 128, F32, F32, False, None), (2048, 1024, 128, 400, BF16, F32, True, None), (700, 1800, 3000, 333, BF16, BF16, True, None)])
def test_products_and_gradients_close(rows, cols, group, batch, dtype, result, zeros, scales):
    w = _weight(rows, cols, group, zeros, cols, scales)
    M, T = _matrix(w, group)
    h = _handle(w, group)
    half = 2.0 ** -8 if result == BF16 else 2.0 ** -24
    x = _vectors(batch, cols, dtype, 1, 0, False)
    got, want = rsr.rsr_int4_matvec(h, x, dtype=result).double(), x.double() @ M.t()
    bound = (160 + cols / 32) * 2.0 ** -24 * (x.double().abs() @ T.t()) * (1 + half) + half * want.abs()
    assert bool(((got - want).abs() <= bound).all())
    y = _vectors(batch, rows, dtype, 2, 0, False)
    got, want = rsr.rsr_int4_matvec(h, y, transposed=True, dtype=result).double(), y.double() @ M
    bound = (rows + 32) * 2.0 ** -24 * (y.double().abs() @ T)
    if dtype == BF16 and result == BF16:
        bound += 2.0 ** -8 * (y.double().abs() @ M.abs())
    bound = bound * (1 + half) + half * want.abs()
    assert bool(((got - want).abs() <= bound).all())


def test_every_bit_of_a_float32_vector():
    """One element per vector that needs all three bf16 planes: results are its products with one column."""
    rows, cols, group = 40, 700, 32
    w = _weight(rows, cols, group, False, 9, "pow2")
    M, _ = _matrix(w, group)
    h = _handle(w, group)
    for batch in (1, 3, 20, 140):
        x = torch.zeros((batch, cols), device=DEV)
        at = torch.randint(0, cols, (batch,), generator=_gen(batch), device=DEV)
        x[torch.arange(batch, device=DEV), at] = 1.0 + torch.randint(0, 1 << 23, (batch,), generator=_gen(3), device=DEV) * 2.0 ** -23
        # u x - 8 x: each has four more bits than a float32 and is rounded once, the difference is theirs
        got, want = rsr.rsr_matvec_ex(h, x).double(), x.double() @ M.t()
        assert bool(((got - want).abs() <= 3 * 2.0 ** -24 * 32 * M.abs().max() / 7).all())
        y = torch.zeros((batch, rows), device=DEV)
        y[torch.arange(batch, device=DEV), at % rows] = 1.0 + torch.randint(0, 1 << 23, (batch,), generator=_gen(4), device=DEV) * 2.0 ** -23
        got, want = rsr.rsr_int4_matvec(h, y, transposed=True).double(), y.double() @ M
        assert bool(((got - want).abs() <= 3 * 2.0 ** -24 * 32 * M.abs().max() / 7).all())


# ---- the gated block --------------------------------------------------------------------------------
def _act(name, a):
    """act(a) and its derivative in 64 bits"""
    a = a.double()
    if name == "silu":
        p = torch.sigmoid(a)
        return a * p, p + a * p * torch.sigmoid(-a)
    if name == "gelu":
        # 0.5 (1 + tanh(t / 2)) = sigmoid(t); 1 + tanh(t / 2) has nothing left below 2^-53, the sigmoid has
        t = _exponent(name, a)
        p, dt = torch.sigmoid(t), (8.0 / torch.pi) ** 0.5 * (1 + 3 * 0.044715 * a * a)
        return a * p, p + a * p * torch.sigmoid(-t) * dt
    return torch.relu(a) ** 2, 2 * torch.relu(a)


def _exponent(name, a):
    a = a.double()
    return (8.0 / torch.pi) ** 0.5 * (a + 0.044715 * a ** 3) if name == "gelu" else a


@pytest.mark.parametrize("act", ["silu", "gelu", "relu2"])
@pytest.mark.parametrize("rows,cols,group,batch,dtype,result,zeros,pad", [
    (1, 1, 32, 1, F32, F32, False, 0), (17, 257, 64, 2, BF16, BF16, True, 1), (640, 300, 128, 1, BF16, F32, False, 0),
    (333, 1111, 32, 4, F32, F32, True, 1), (500, 640, 96, 13, BF16, BF16, True, 8), (200, 1000, 64, 33, F32, BF16, False, 3),
    (1030, 513, 128, 140, BF16, BF16, True, 3), (2050, 400, 32, 300, F32, F32, False, 0), (3000, 256, 64, 520, BF16, F32, True, 0)])
def test_gated(rows, cols, group, batch, dtype, result, zeros, pad, act):
    # one side with float32 scales and one with bf16, one with zero points and one without
    wg, wu = _weight(rows, cols, group, zeros, 1, "pow2"), _weight(rows, cols, group, not zeros, 2, "wide")
    gate, up = _handle(wg, group), _handle(wu, group)
    x = _vectors(batch, cols, dtype, 3, pad, True)
    a, b = (0.125 * (x.double() @ _matrix(w, group)[0].t()) for w in (wg, wu))
    x = x * 0.125                                   # (activations near their bends)
    if pad:
        x = torch.nn.functional.pad(x, (0, pad), value=float("nan"))[:, :cols]
    buf, out = _out(batch, rows, result, 3)
    pre = torch.full((batch, 2, rows), -77.0, device=DEV)
    rsr.rsr_gated(gate, up, x, act, out=out, pre=pre)
    assert torch.equal(pre, torch.stack((a, b), dim=1).float())
    f, _ = _act(act, a)
    half = 2.0 ** -8 if result == BF16 else 2.0 ** -24
    want = f * b
    size = 2.0 ** -20 * (1 + _exponent(act, a).abs())
    # (a sigmoid below 2^-126, the smallest normal float32, is zero: off by 2^-126 at most, times |a b|; so is a result)
    assert bool(((out.double() - want).abs() <= size * want.abs() * (1 + half) + half * want.abs()
                 + 2.0 ** -126 * (1 + (a * b).abs())).all())
    assert bool((buf[:, rows:] == -77.0).all())
    assert torch.equal(rsr.rsr_gated(gate, up, x, act, dtype=result), out)      # without `pre`
    one = rsr.rsr_gated(gate, up, x[0], act, dtype=result)
    assert one.shape == (rows,) and torch.equal(one, out[0])    # (a and b are exact)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu2"])
@pytest.mark.parametrize("rows,cols,group,batch,dtype,result,zeros", [
    (1, 1, 32, 1, F32, F32, True), (33, 300, 64, 3, BF16, BF16, False), (640, 257, 128, 1, BF16, F32, True), (300, 1001, 32, 20, F32, F32, False),
    (777, 640, 96, 50, BF16, BF16, True), (520, 1030, 128, 140, F32, BF16, False), (400, 2100, 32, 300, BF16, BF16, True),
    (1200, 1500, 64, 260, F32, F32, True)])
def test_gated_backward(rows, cols, group, batch, dtype, result, zeros, act):
    wg, wu = _weight(rows, cols, group, zeros, 4, "bf16"), _weight(rows, cols, group, not zeros, 5, None)
    gate, up = _handle(wg, group), _handle(wu, group)
    g = _gen(6)
    pre = 3 * torch.randn((batch, 2, rows), generator=g, device=DEV)
    dh = _vectors(batch, rows, dtype, 7, 3, False)
    a, b, d = pre[:, 0].double(), pre[:, 1].double(), dh.double()
    f, slope = _act(act, a)
    da, db = d * b * slope, d * f
    kept = pre.clone()
    dv, dpre = rsr.rsr_gated_backward(gate, up, pre, dh, act, dtype=result)
    assert torch.equal(pre, kept) and dv.dtype == result and dv.shape == (batch, cols)
    size = 2.0 ** -20 * (1 + _exponent(act, a).abs())
    # (the two terms of the derivative may cancel: they are at most 1 + |a| dt/da / 4 each)
    terms = 1 + slope.abs() + (a.abs() if act != "gelu" else a.abs() * (1 + a * a).clamp(max=260.0)) / 4
    assert bool(((dpre[:, 0].double() - da).abs() <= size * (d * b).abs() * terms + 2.0 ** -126).all())
    assert bool(((dpre[:, 1].double() - db).abs() <= size * d.abs() * f.abs() + 2.0 ** -126 * (1 + (a * d).abs())).all())
    # dv of the dpre that was written
    (Mg, Tg), (Mu, Tu) = _matrix(wg, group), _matrix(wu, group)
    da, db = dpre[:, 0].double(), dpre[:, 1].double()
    want = da @ Mg + db @ Mu
    half = 2.0 ** -8 if result == BF16 else 2.0 ** -24
    bound = (2 * rows + 64) * 2.0 ** -24 * (da.abs() @ Tg + db.abs() @ Tu)
    if result == BF16:
        bound += 2.0 ** -8 * (da.abs() @ Mg.abs() + db.abs() @ Mu.abs())
    assert bool(((dv.double() - want).abs() <= bound * (1 + half) + half * want.abs()).all())
    # in place, and without dv
    none, again = rsr.rsr_gated_backward(gate, up, kept, dh, act, dpre=kept, need_dv=False)
    assert none is None and again is kept and torch.equal(kept, dpre)


def test_gradients_against_differences():
    """The block's input gradient against central differences of its forward pass in float32."""
    rows, cols, group, batch = 60, 96, 32, 3
    wg, wu = _weight(rows, cols, group, True, 11), _weight(rows, cols, group, False, 12)
    gate, up = _handle(wg, group), _handle(wu, group)
    x = torch.randn((batch, cols), generator=_gen(13), device=DEV)
    dh = torch.randn((batch, rows), generator=_gen(14), device=DEV)
    step = 2.0 ** -6
    for act in ("silu", "gelu", "relu2"):
        pre = torch.empty((batch, 2, rows), device=DEV)
        rsr.rsr_gated(gate, up, x, act, pre=pre)
        dv, _ = rsr.rsr_gated_backward(gate, up, pre, dh, act)
        # all 96 coordinates as one batch
        xs = x[:, None, :] + step * torch.eye(cols, device=DEV)
        ys = x[:, None, :] - step * torch.eye(cols, device=DEV)
        f = [rsr.rsr_gated(gate, up, t.reshape(-1, cols), act).reshape(batch, cols, rows).double() for t in (xs, ys)]
        diff = ((f[0] - f[1]) * dh.double()[:, None, :]).sum(dim=2) / (2 * step)
        # rounding: 2^-20 of the values over 2 steps; curvature: step^2 / 6 of a third derivative of order |M|^3
        size = (f[0].abs() * dh.double().abs()[:, None, :]).sum(dim=2)
        weight = (_matrix(wg, group)[0].abs().amax() + _matrix(wu, group)[0].abs().amax()) ** 3 * dh.double().abs().sum(dim=1, keepdim=True)
        assert bool(((dv.double() - diff).abs() <= 2.0 ** -20 * size / step + step ** 2 / 6 * 8 * (1 + pre.abs().amax()) * weight).all())


# ---- the calls around it ------------------------------------------------------------------------------
def _pair(rows=200, cols=640, group=64, seed=20):
    wg, wu = _weight(rows, cols, group, True, seed, "pow2"), _weight(rows, cols, group, False, seed + 1, "pow2")
    return wg, wu, _handle(wg, group), _handle(wu, group)


@pytest.mark.parametrize("batch", [1, 3, 20, 150])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_infinities_and_nan_stay_in_their_vector(batch, dtype):
    wg, wu, gate, up = _pair()
    for length, transposed in ((640, False), (200, True)):
        x = _vectors(batch, length, dtype, 1, 0, True)
        clean = rsr.rsr_int4_matvec(gate, x, transposed=transposed)
        for bad in (float("inf"), float("-inf"), float("nan")):
            y = x.clone()
            y[0, length // 2] = bad
            got = rsr.rsr_int4_matvec(gate, y, transposed=transposed)
            assert not bool(got[0].isfinite().any()) and torch.equal(got[1:], clean[1:])
    x = _vectors(batch, 640, dtype, 2, 0, True)
    clean, y = rsr.rsr_gated(gate, up, x, "silu"), x.clone()
    y[-1, 0] = float("nan")
    got = rsr.rsr_gated(gate, up, y, "silu")
    assert bool(got[-1].isnan().all()) and torch.equal(got[:-1], clean[:-1])


def test_activations_at_their_ends():
    """Products from far below to far above: nothing becomes NaN, and relu2 passes NaN on."""
    rows, cols = 64, 32
    Q = torch.full((rows, cols), 1, dtype=torch.int8, device=DEV)
    s = torch.ones((rows, 1), device=DEV)
    gate, up = rsr.rsr_preprocess_int4(Q, s, 32), rsr.rsr_preprocess_int4(Q, s, 32)
    x = torch.zeros((10, cols), device=DEV)
    x[:, 0] = torch.tensor([-1e30, -1e4, -100.0, -20.0, -0.0, 0.0, 20.0, 100.0, 1e4, 1e10], device=DEV)
    for act in ("silu", "gelu", "relu2"):
        pre = torch.empty((10, 2, rows), device=DEV)
        h = rsr.rsr_gated(gate, up, x, act, pre=pre)
        f, slope = _act(act, x[:, :1])
        assert not bool(h.isnan().any())
        assert torch.allclose(h.double(), (f * x[:, :1]).expand(-1, rows), rtol=2.0 ** -12, atol=1e-30)
        _, dpre = rsr.rsr_gated_backward(gate, up, pre, torch.ones((10, rows), device=DEV), act)
        want = (x[:, :1].double() * torch.nan_to_num(slope)).expand(-1, rows)
        inner = x[:, 0].abs() <= 100
        assert not bool(dpre.isnan().any())
        assert torch.allclose(dpre[inner, 0].double(), want[inner], rtol=2.0 ** -12, atol=1e-6)


@pytest.mark.parametrize("batch", [1, 4, 40, 200])
def test_captured_and_replayed(batch):
    wg, wu, gate, up = _pair()
    x = _vectors(batch, 640, BF16, 1, 0, True)
    dh = _vectors(batch, 200, BF16, 2, 0, True)
    pre, h = torch.empty((batch, 2, 200), device=DEV), torch.empty((batch, 200), device=DEV, dtype=BF16)
    dpre, dv = torch.empty_like(pre), torch.empty((batch, 640), device=DEV, dtype=BF16)
    y, dx = torch.empty((batch, 200), device=DEV), torch.empty((batch, 640), device=DEV)

    def step():
        rsr.rsr_int4_matvec(gate, x, out=y)
        rsr.rsr_int4_matvec(up, dh, transposed=True, out=dx)
        rsr.rsr_gated(gate, up, x, "silu", out=h, pre=pre)
        rsr.rsr_gated_backward(gate, up, pre, dh, "silu", dv=dv, dpre=dpre)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        x.copy_(_vectors(batch, 640, BF16, 10 + turn, 0, True))
        dh.copy_(_vectors(batch, 200, BF16, 20 + turn, 0, True))
        for t in (pre, h, dpre, dv, y, dx):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (pre, h, dpre, dv, y, dx)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (pre, h, dpre, dv, y, dx)))


def test_streams():
    """The current stream is used, and a stream given."""
    wg, wu, gate, up = _pair()
    M = _matrix(wg, 64)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        v = torch.zeros((2, 640), device=DEV)
        for _ in range(200):
            v += 1
        got = rsr.rsr_int4_matvec(gate, v)
    side.synchronize()
    assert torch.equal(got.double(), 200.0 * M.sum(dim=1).expand(2, -1))
    out = torch.empty((2, 200), device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        v.zero_()
        for _ in range(100):
            v += 1
    rsr.rsr_int4_matvec(gate, v, out=out, stream=side)
    side.synchronize()
    assert torch.equal(out.double(), 100.0 * M.sum(dim=1).expand(2, -1))


def test_no_vectors_and_one():
    wg, wu, gate, up = _pair()
    none = torch.empty((0, 640), device=DEV, dtype=BF16)
    assert rsr.rsr_int4_matvec(gate, none).shape == (0, 200)
    assert rsr.rsr_int4_matvec(gate, none[:, :200], transposed=True, dtype=BF16).shape == (0, 640)
    pre = torch.empty((0, 2, 200), device=DEV)
    assert rsr.rsr_gated(gate, up, none, pre=pre).shape == (0, 200)
    dv, dpre = rsr.rsr_gated_backward(gate, up, pre, none[:, :200])
    assert dv.shape == (0, 640) and dpre.shape == (0, 2, 200)
    x = _vectors(1, 640, F32, 1, 0, True)
    pre = torch.empty((1, 2, 200), device=DEV)
    one = rsr.rsr_gated(gate, up, x[0], "silu", pre=pre)
    assert one.shape == (200,) and torch.equal(one, rsr.rsr_gated(gate, up, x, "silu")[0])
    dv, _ = rsr.rsr_gated_backward(gate, up, pre, one, "silu")
    assert dv.shape == (640,)


def test_same_bits_every_time():
    w = _weight(700, 1500, 64, True, 30)
    h = _handle(w, 64)
    for batch in (1, 4, 30, 250):
        for dtype in (F32, BF16):
            x, y = _vectors(batch, 1500, dtype, 1, 1, False), _vectors(batch, 700, dtype, 2, 1, False)
            for _ in range(3):
                assert torch.equal(rsr.rsr_int4_matvec(h, x), rsr.rsr_int4_matvec(h, x))
                a = rsr.rsr_int4_matvec(h, y, transposed=True, dtype=dtype)
                assert torch.equal(a, rsr.rsr_int4_matvec(h, y, transposed=True, dtype=dtype))


def test_values_out_of_range():
    Q, s, z = _weight(50, 300, 32, True, 1)
    for at, value in (((0, 0), 8), ((49, 299), -9), ((20, 150), 127), ((31, 31), -128)):
        bad = Q.clone()
        bad[at] = value
        with pytest.raises(rsr.RsrError) as e:
            rsr.rsr_preprocess_int4(bad, s, 32, zeros=z)
        assert e.value.code == 2
    for value in (float("inf"), float("-inf"), float("nan")):
        bad = s.clone()
        bad[49, 9] = value
        with pytest.raises(rsr.RsrError) as e:
            rsr.rsr_preprocess_int4(Q, bad, 32, zeros=z)
        assert e.value.code == 2
    for value in (8, -9):
        bad = z.clone()
        bad[49, 9] = value
        with pytest.raises(rsr.RsrError) as e:
            rsr.rsr_preprocess_int4(Q, s, 32, zeros=bad)
        assert e.value.code == 2
    assert rsr.rsr_preprocess_int4(Q, s, 32, zeros=z).rows == 50


def test_refusals():
    wg, wu, gate, up = _pair()
    lib = rsr.load_library()
    x, out = torch.zeros((4, 640), device=DEV), torch.zeros((4, 200), device=DEV)
    p, q = x.data_ptr(), out.data_ptr()

    def code(*args):
        return lib.rsr_int4_matvec(gate.ptr, *args, None)

    assert code(0, p, 2, 1.0, q, 0, 4, 640, 200) == 1           # types
    assert code(0, p, 0, 1.0, q, -1, 4, 640, 200) == 1
    assert code(0, p, 0, 1.0, q, 0, -1, 640, 200) == 1          # number and distances of vectors
    assert code(0, p, 0, 1.0, q, 0, 4, 639, 200) == 1
    assert code(0, p, 0, 1.0, q, 0, 4, 640, 199) == 1
    assert code(1, q, 0, 1.0, p, 0, 4, 199, 640) == 1
    assert code(0, p, 0, 1.0, q, 0, (1 << 24) + 1, 640, 200) == 3
    assert code(0, None, 0, 1.0, q, 0, 4, 640, 200) == 1
    assert code(0, p, 0, 1.0, None, 0, 4, 640, 200) == 1
    assert code(0, p, 0, 1.0, q, 0, 0, 0, 0) == 0
    assert lib.rsr_gated(gate.ptr, up.ptr, p, 0, 3, q, 0, None, 4, 640, 200, None) == 1
    other = _pair(rows=201)[2]
    wide = _pair(group=32)[2]
    for pair, want in (((gate, other), 1), ((gate, wide), 3)):
        with pytest.raises(rsr.RsrError) as e:
            rsr.rsr_gated(*pair, x)
        assert e.value.code == want
    assert torch.equal(rsr.rsr_gated(gate, gate, x), out)       # the same handle twice
    for call in (lambda: rsr.rsr_serialize(gate), lambda: rsr.rsr_preprocess_into(gate, wg[0])):
        with pytest.raises(rsr.RsrError) as e:
            call()
        assert e.value.code == 3
    for call in (lambda: rsr.rsr_get_perm(gate), lambda: rsr.rsr_get_packed(gate), lambda: rsr.rsr_launch_shape(gate)):
        with pytest.raises(rsr.RsrError) as e:
            call()
        assert e.value.code == 1
    assert rsr.rsr_algorithmic_bytes(gate, rsr.RSR_BF16, 2) > 200 * 640 // 2
    assert rsr.rsr_kernel_name(gate).startswith("k_int4")
    for v in (x.cpu(), x[:, :639], x.half(), x.t(), x[None], x[0, 0]):
        with pytest.raises(TypeError):
            rsr.rsr_int4_matvec(gate, v)
        with pytest.raises(TypeError):
            rsr.rsr_gated(gate, up, v)
    for bad in (out[:3], out[:, :199], out.half(), out.cpu()):
        with pytest.raises(TypeError):
            rsr.rsr_int4_matvec(gate, x, out=bad)
    with pytest.raises(TypeError):
        rsr.rsr_gated(gate, up, x, pre=torch.empty((4, 200, 2), device=DEV))
    with pytest.raises(TypeError):
        rsr.rsr_gated_backward(gate, up, torch.empty((3, 2, 200), device=DEV), out)
    with pytest.raises(ValueError):
        rsr.rsr_gated(gate, up, x, "relu")
    rsr.rsr_destroy(up)
    with pytest.raises(rsr.RsrError):
        rsr.rsr_gated(gate, up, x)


def test_offsets_beyond_32_bits():
    """Vectors and results 2^31 elements apart."""
    wg, wu, gate, up = _pair()
    far = 1 << 31
    buf = torch.empty(far + 640, device=DEV, dtype=BF16)
    res = torch.empty(far + 640, device=DEV, dtype=BF16)
    x = buf.as_strided((2, 640), (far, 1))
    x.copy_(_vectors(2, 640, BF16, 1, 0, True))
    out = res.as_strided((2, 200), (far, 1))
    rsr.rsr_int4_matvec(gate, x, out=out)
    assert torch.equal(out, (x.double() @ _matrix(wg, 64)[0].t()).to(BF16))
    rsr.rsr_gated(gate, up, x, "relu2", out=out)
    assert torch.equal(out, rsr.rsr_gated(gate, up, x.contiguous(), "relu2", dtype=BF16))
    y, dx = buf.as_strided((2, 200), (far, 1)), res.as_strided((2, 640), (far, 1))
    rsr.rsr_int4_matvec(gate, y, transposed=True, out=dx)
    assert torch.equal(dx, (y.double() @ _matrix(wg, 64)[0]).to(BF16))


def test_codes_beyond_32_bits():
    """9 * 2^30 entries: 4.5 GiB of codes.  The rows at both ends against one vector of ones."""
    rows, cols = 9 << 17, 1 << 13
    g = _gen(40)
    Q = torch.randint(-8, 8, (rows, cols), generator=g, device=DEV, dtype=torch.int8)
    s = torch.ones((rows, 1), device=DEV)
    h = rsr.rsr_preprocess_int4(Q, s, cols)
    x = torch.ones(cols, device=DEV, dtype=BF16)
    got = rsr.rsr_matvec_ex(h, x)
    want = torch.cat([Q[at:at + 65536].sum(dim=1, dtype=torch.int32) for at in range(0, rows, 65536)]).float()
    assert torch.equal(got, want)
    y = torch.zeros(rows, device=DEV)
    y[5] = y[rows // 2] = y[-3] = 1.0
    assert torch.equal(rsr.rsr_int4_matvec(h, y, transposed=True), (Q[5].float() + Q[rows // 2] + Q[-3]))


@pytest.mark.parametrize("rows,cols", [((1 << 24) - 5, 33), (70, (1 << 24) - 300)])
def test_the_largest_sizes(rows, cols):
    """Row and column counts at the limits, with vectors for every kernel: several launches where one does not hold them."""
    g = _gen(50)
    Q = torch.randint(-8, 8, (rows, cols), generator=g, device=DEV, dtype=torch.int8)
    s = torch.ones((rows, 1), device=DEV)
    h = rsr.rsr_preprocess_int4(Q, s, cols)
    tall = rows > cols
    for batch in (1, 4, 20, 90):
        # one element in each vector: products are columns, or rows, of Q
        at = torch.randint(0, cols if tall else rows, (batch,), generator=g, device=DEV)
        x = torch.zeros((batch, cols if tall else rows), device=DEV, dtype=BF16)
        x[torch.arange(batch, device=DEV), at] = 1.0
        got = rsr.rsr_int4_matvec(h, x, transposed=not tall, dtype=BF16)
        for n in range(batch):
            assert torch.equal(got[n], (Q[:, at[n]] if tall else Q[at[n]]).to(BF16))


def test_many_vectors():
    """More vectors than a grid has in one direction, and than one launch of the activation's gradient."""
    wg, wu, gate, up = _pair(rows=40, cols=33, group=32)
    batch = 66000
    x, dh = _vectors(batch, 33, BF16, 1, 0, True), _vectors(batch, 40, BF16, 2, 0, True)
    assert torch.equal(rsr.rsr_int4_matvec(gate, x, dtype=BF16), (x.double() @ _matrix(wg, 32)[0].t()).to(BF16))
    assert torch.equal(rsr.rsr_int4_matvec(gate, dh, transposed=True, dtype=BF16), (dh.double() @ _matrix(wg, 32)[0]).to(BF16))
    pre = torch.empty((batch, 2, 40), device=DEV)
    h = rsr.rsr_gated(gate, up, x, "relu2", pre=pre)
    assert torch.equal(h[-100:], rsr.rsr_gated(gate, up, x[-100:], "relu2"))
    dv, dpre = rsr.rsr_gated_backward(gate, up, pre, dh, "relu2")
    assert torch.equal(dpre[-3:, 1], dh[-3:].float() * torch.relu(pre[-3:, 0]) ** 2)
    assert torch.equal(dpre[:3, 1], dh[:3].float() * torch.relu(pre[:3, 0]) ** 2)


@pytest.mark.parametrize("group", [300, 1 << 31, (1 << 63) - 1])
def test_one_scale_per_row(group):
    w = _weight(70, 300, 300, True, 90)
    h = _handle(w, 300) if group == 300 else rsr.rsr_preprocess_int4(w[0], w[1], group, zeros=w[2])
    M, sizes = _matrix(w, 300)
    v = torch.randint(-3, 4, (3, 300), generator=_gen(91), device=DEV).float()
    got = rsr.rsr_int4_matvec(h, v).double()
    assert bool(((got - v.double() @ M.t()).abs() <= 300 * 2.0 ** -24 * (v.double().abs() @ sizes.t())).all())
