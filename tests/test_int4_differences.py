"""The gated block's input gradient against differences of its definition in 64 bits, with a bound that a missing term breaks.

The central difference of the float64 block at a step of h = 2^-20 is off from its derivative by 2^-53 / h of the terms it subtracts
and, where relu2 has its bend within a step, by h |dh b| M^2 (the other curvatures are below h^2: nothing).  The float32 gradient
is off by what its parts are: with P = 160 additions on a path (see test_gpu_int4.py), e(a) = P 2^-24 sum |x| s (u + 8 + z) in each
product, da = dh b act'(a) therefore by |dh| (e(b) |act'| + |b| |act''| e(a)) and 2^-20 (1 + |t|) of its factors, db = dh act(a) by
|dh| |act'| e(a) and the same of itself, and the last sums by (2 rows + 64) 2^-24 of their terms.  |act''| is at most 2."""
import pytest

torch = pytest.importorskip("torch")
ACTS = ["silu", "gelu", "relu2"]
ROWS, COLS, BATCH, GROUP = 60, 96, 3, 32


def _exponent(name, a):
    return (8.0 / torch.pi) ** 0.5 * (a + 0.044715 * a ** 3) if name == "gelu" else a


def _act(name, a):
    """act(a) and its derivative"""
    if name == "relu2":
        return torch.relu(a) ** 2, 2 * torch.relu(a)
    t = _exponent(name, a)
    p = torch.sigmoid(t)
    dt = 1.0 if name == "silu" else (8.0 / torch.pi) ** 0.5 * (1 + 3 * 0.044715 * a * a)
    return a * p, p + a * p * torch.sigmoid(-t) * dt


def _case(seed):
    """x, dh, and for gate and up codes, scales, zero points, M and s (u + 8 + z), all made on the CPU"""
    g = torch.Generator().manual_seed(seed)
    weights = []
    for zeros in (True, False):
        Q = torch.randint(-8, 8, (ROWS, COLS), generator=g, dtype=torch.int8)
        s = torch.randn((ROWS, COLS // GROUP), generator=g) / 16
        z = torch.randint(-8, 8, s.shape, generator=g, dtype=torch.int8) if zeros else None
        wide = [0.0 if t is None else t.double().repeat_interleave(GROUP, dim=1) for t in (s, z)]
        weights.append((Q, s, z, (Q.double() - wide[1]) * wide[0], (Q.double() + 16.0 + wide[1]) * wide[0].abs()))
    return torch.randn((BATCH, COLS), generator=g), torch.randn((BATCH, ROWS), generator=g), weights


def _differences(x, dh, Mg, Mu, act, step=2.0 ** -20):
    """the gradient of sum(dh * block(x)) and how far it may be off, in 64 bits"""
    x, dh = x.double(), dh.double()
    sides = []
    for sign in (1, -1):
        t = (x[:, None, :] + sign * step * torch.eye(COLS, dtype=torch.float64)).reshape(-1, COLS)
        f, _ = _act(act, t @ Mg.t())
        sides.append((f * (t @ Mu.t())).reshape(BATCH, COLS, ROWS))
    diff = ((sides[0] - sides[1]) * dh[:, None, :]).sum(dim=2) / (2 * step)
    terms = (sides[0].abs() * dh.abs()[:, None, :]).sum(dim=2)
    off = (COLS + 2 * ROWS) * 2.0 ** -53 / step * terms
    if act == "relu2":
        off = off + step * (dh * (x @ Mu.t())).abs() @ (Mg * Mg)
    return diff, off


def _excess(dv, x, dh, weights, act):
    """the largest error of dv over its bound"""
    (_, _, _, Mg, Tg), (_, _, _, Mu, Tu) = weights
    diff, off = _differences(x, dh, Mg, Mu, act)
    x, d = x.double(), dh.double()
    a, b = x @ Mg.t(), x @ Mu.t()
    ea, eb = (160 * 2.0 ** -24 * (x.abs() @ T.t()) for T in (Tg, Tu))
    f, slope = _act(act, a)
    size = 2.0 ** -20 * (1 + _exponent(act, a).abs())
    # (the two terms of the derivative may cancel: they are at most 1 + |a| dt/da / 4 each)
    parts = 1 + slope.abs() + (a.abs() if act != "gelu" else a.abs() * (1 + a * a)) / 4
    da = d.abs() * (eb * (slope.abs() + size * parts) + b.abs() * (2 * ea + size * parts))
    db = d.abs() * (slope.abs() * ea + ea * ea + size * f.abs())
    last = (2 * ROWS + 64) * 2.0 ** -24 * ((d * b * slope).abs() @ Tg + (d * f).abs() @ Tu)
    bound = off + da @ Mg.abs() + db @ Mu.abs() + last
    return float(((dv.double() - diff).abs() / bound).max())


def _gradient(x, dh, Mg, Mu, act, drop=None):
    """the formula in 64 bits, rounded to float32; drop: a part that is left out"""
    x, d = x.double(), dh.double()
    a, b = x @ Mg.t(), x @ Mu.t()
    f, slope = _act(act, a)
    if drop == "slope":
        slope = slope * (1 - 2.0 ** -5)
    if drop == "second" and act != "relu2":
        slope = torch.sigmoid(_exponent(act, a))
    da, db = d * b * slope, d * f
    dv = (0 if drop == "gate" else da @ Mg) + (0 if drop == "up" else db @ Mu)
    return (dv * (1 + 2.0 ** -6) if drop == "percent" else dv).float()


@pytest.mark.parametrize("act", ACTS)
def test_the_bound_tells_mistakes(act):
    """On the CPU: the formula is within the bound, and with any part left out, or off by a few per cent, it is not."""
    for seed in range(3):
        x, dh, weights = _case(seed)
        Mg, Mu = weights[0][3], weights[1][3]
        assert _excess(_gradient(x, dh, Mg, Mu, act), x, dh, weights, act) < 1
        for drop in ("gate", "up", "slope", "percent") + (("second",) if act != "relu2" else ()):
            assert _excess(_gradient(x, dh, Mg, Mu, act, drop), x, dh, weights, act) > 2, drop
        assert _excess(torch.zeros_like(x), x, dh, weights, act) > 2


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(act):
    rsr = pytest.importorskip("paper_2603_27462_amd")
    for seed in range(3):
        x, dh, weights = _case(seed)
        gate, up = (rsr.rsr_preprocess_int4(Q.cuda(), s.cuda(), GROUP, zeros=None if z is None else z.cuda())
                    for Q, s, z, _, _ in weights)
        pre = torch.empty((BATCH, 2, ROWS), device="cuda")
        rsr.rsr_gated(gate, up, x.cuda(), act, pre=pre)
        dv, _ = rsr.rsr_gated_backward(gate, up, pre, dh.cuda(), act)
        assert _excess(dv.cpu(), x, dh, weights, act) < 1
