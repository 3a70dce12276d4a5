"""Products with 4-bit weights and group scales, their input gradients, and the gated feed-forward block.

A weight matrix is M[r][c] = scales[r][c // group] * (codes[r][c] - zeros[r][c // group]) with codes and zeros from
-8 to 7 (no zeros: 0).  A case is a dict of plain values; `path` says which operator it is:

  product   y = x M^T, float32 (rsr_matvec_ex on an int4 handle)
  gradient  dx = dy M in the type of dy (rsr_int4_matvec, transposed)
  gated     h = act(x Mg^T) * (x Mu^T) in the type of x (rsr_gated)
  train     the same with what its backward pass needs kept, and that pass: h, dx and the gradients of both
            projections' results, float32 (rsr_gated, rsr_gated_backward)

Layer shapes are those of bench.py and perf/cases.py: the 2B-class set (2560, 640, 6912) and the 8B-class set (4096,
14336); draw() spreads the same work over the sizes around them.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # the smallest layer of the 2B-class set, one token: nearly all latency
        dict(name="product_640x2560", path="product", rows=640, cols=2560, batch=1, dtype="bf16", group=128, scales="bf16", zeros=False),
        # the headline shape, one token through a down projection
        dict(name="product_down", path="product", rows=4096, cols=14336, batch=1, dtype="bf16", group=128, scales="bf16", zeros=False),
        # a few float32 vectors on a matrix that fits no tile, small groups, zero points, float32 scales
        dict(name="product_ragged", path="product", rows=1001, cols=2999, batch=3, dtype="f32", group=32, scales="f32", zeros=True),
        # sixteen sequences decode together through the widest layer; zero points and half-precision scales
        dict(name="product_batch16", path="product", rows=14336, cols=4096, batch=16, dtype="bf16", group=64, scales="f16", zeros=True),
        # a long prompt through the largest layer
        dict(name="product_prompt", path="product", rows=4096, cols=14336, batch=2048, dtype="bf16", group=128, scales="bf16", zeros=False),
        # the gradient of a few tokens, small groups
        dict(name="gradient_few", path="gradient", rows=2560, cols=6912, batch=8, dtype="bf16", group=32, scales="bf16", zeros=False),
        # the gradient of a long sequence through the largest layer
        dict(name="gradient_2048", path="gradient", rows=4096, cols=14336, batch=2048, dtype="bf16", group=128, scales="bf16", zeros=False),
        # one token through gate and up of the 2B-class set
        dict(name="gated_decode", path="gated", rows=6912, cols=2560, batch=1, dtype="bf16", group=128, scales="bf16", zeros=False, act="silu"),
        # eight sequences through gate and up of the 8B-class set
        dict(name="gated_batch8", path="gated", rows=14336, cols=4096, batch=8, dtype="bf16", group=64, scales="bf16", zeros=False, act="gelu"),
        # a prompt through the same
        dict(name="gated_prompt", path="gated", rows=14336, cols=4096, batch=512, dtype="bf16", group=128, scales="bf16", zeros=True, act="silu"),
        # a training step of a small block in float32: odd sizes, zero points, float32 scales
        dict(name="train_ragged", path="train", rows=1001, cols=2999, batch=37, dtype="f32", group=32, scales="f32", zeros=True, act="relu2"),
        # a training step of the 2B-class block
        dict(name="train_1024", path="train", rows=6912, cols=2560, batch=1024, dtype="bf16", group=128, scales="bf16", zeros=False, act="silu"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    path = rng.choice(["product", "product", "gradient", "gated", "train"])
    rows, cols = _log_uniform(rng, 300, 14336), _log_uniform(rng, 300, 14336)
    if rows * cols > 4096 * 14336:
        rows = 4096 * 14336 // cols
    if rng.random() < 0.5:                       # a model's sizes are whole multiples more often than not
        rows, cols = 64 * max(1, rows // 64), 64 * max(1, cols // 64)
    most = 1024 if path == "train" else 2048
    batch = rng.choice([1, rng.randint(2, 16), _log_uniform(rng, 17, most)])
    case = dict(path=path, rows=rows, cols=cols, batch=batch, dtype=rng.choice(["bf16", "bf16", "f32"]),
                group=rng.choice([32, 64, 96, 128, 256, cols]), scales=rng.choice(["bf16", "f16", "f32"]), zeros=rng.random() < 0.4)
    if case["dtype"] == "f32":                   # a float32 product is several of bf16
        case["batch"] = min(batch, 512)
    if path in ("gated", "train"):
        case["act"] = rng.choice(["silu", "gelu", "relu2"])
    return case


# ------------------------------------------------------------------------------ inputs
def _weight(g, case):
    """Codes as a quantiser leaves them (bell-shaped, every value met), scales that differ by group, such that a row of M has
    about unit norm."""
    rows, cols, group = case["rows"], case["cols"], min(case["group"], case["cols"])
    n = -(-cols // group)
    codes = torch.randn((rows, cols), generator=g, device="cuda").mul_(3.0).round_().clamp_(-8, 7).to(torch.int8)
    scales = (0.5 + torch.rand((rows, n), generator=g, device="cuda")) / (3.0 * math.sqrt(cols))
    scales = scales.to(DTYPES[case["scales"]])
    zeros = torch.randint(-3, 4, (rows, n), generator=g, device="cuda", dtype=torch.int8) if case["zeros"] else None
    return codes, scales, zeros


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    count = 2 if case["path"] in ("gated", "train") else 1
    state = {"weights": [_weight(g, case) for _ in range(count)]}
    dtype = DTYPES[case["dtype"]]
    if case["path"] != "gradient":
        state["x"] = torch.randn((case["batch"], case["cols"]), generator=g, device="cuda").to(dtype)
    if case["path"] in ("gradient", "train"):
        state["dy"] = torch.randn((case["batch"], case["rows"]), generator=g, device="cuda").to(dtype)
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    state.update(path=case["path"], group=case["group"], act=case.get("act"))
    if own:
        import paper_2603_27462_amd as rsr
        state["handles"] = [rsr.rsr_preprocess_int4(q, s, case["group"], zeros=z) for q, s, z in state["weights"]]
    return state


# ------------------------------------------------------------------------------ plain form
def _matrix(weight, group):
    codes, scales, zeros = weight
    cols = codes.shape[1]
    wide = scales.float().repeat_interleave(min(group, cols), dim=1)[:, :cols]
    if zeros is None:
        return codes.float() * wide
    return (codes.float() - zeros.float().repeat_interleave(min(group, cols), dim=1)[:, :cols]) * wide


def _act(name, a):
    """act(a) and its derivative."""
    if name == "silu":
        s = torch.sigmoid(a)
        return a * s, s * (1.0 + a * (1.0 - s))
    if name == "gelu":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (a + 0.044715 * a * a * a))
        return 0.5 * a * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * a * a)
    r = torch.relu(a)
    return r * r, 2.0 * r


def run(state):
    path = state["path"]
    if own:
        import paper_2603_27462_amd as rsr
        handles, act = state["handles"], state["act"]
        if path == "product":
            return rsr.rsr_matvec_ex(handles[0], state["x"])
        if path == "gradient":
            return rsr.rsr_int4_matvec(handles[0], state["dy"], transposed=True, dtype=state["dy"].dtype)
        x = state["x"]
        if path == "gated":
            return rsr.rsr_gated(handles[0], handles[1], x, act, dtype=x.dtype)
        pre = torch.empty((x.shape[0], 2, handles[0].rows), dtype=torch.float32, device=x.device)
        h = rsr.rsr_gated(handles[0], handles[1], x, act, dtype=x.dtype, pre=pre)
        dx, dpre = rsr.rsr_gated_backward(handles[0], handles[1], pre, state["dy"], act, dtype=x.dtype)
        return h, dx, dpre
    M = [_matrix(w, state["group"]) for w in state["weights"]]
    if path == "product":
        return state["x"].float() @ M[0].t()
    if path == "gradient":
        dy = state["dy"]
        return (dy.float() @ M[0]).to(dy.dtype)
    x = state["x"]
    a, b = x.float() @ M[0].t(), x.float() @ M[1].t()
    f, slope = _act(state["act"], a)
    h = (f * b).to(x.dtype)
    if path == "gated":
        return h
    dh = state["dy"].float()
    da, db = dh * b * slope, dh * f
    return h, (da @ M[0] + db @ M[1]).to(x.dtype), torch.stack((da, db), dim=1)


# ------------------------------------------------------------------------------ what it costs, and what it is
def work(case):
    rows, cols, batch, path = case["rows"], case["cols"], case["batch"], case["path"]
    item = 4 if case["dtype"] == "f32" else 2
    groups = rows * -(-cols // min(case["group"], cols))
    weight = rows * cols / 2 + groups * ((4 if case["scales"] == "f32" else 2) + (0.5 if case["zeros"] else 0))
    x, y = batch * cols * item, batch * rows * item
    flops = 2.0 * rows * cols * batch
    if path == "product":
        return {"bytes": weight + x + batch * rows * 4, "flops": flops}
    if path == "gradient":
        return {"bytes": weight + x + y, "flops": flops}
    if path == "gated":
        return {"bytes": 2 * weight + x + y, "flops": 2 * flops}
    # forward and backward: the incoming gradient too, and the gradients of both projections' results
    return {"bytes": 2 * weight + 2 * x + 2 * y + 2 * batch * rows * 4, "flops": 4 * flops}


def exact(case, seed):
    """The definition in 64 bits, group by group."""
    state, group = _inputs(case, seed), min(case["group"], case["cols"])

    def project(x, weight):
        codes, scales, zeros = weight
        y = torch.zeros((x.shape[0], codes.shape[0]), dtype=torch.float64, device=x.device)
        for at in range(0, codes.shape[1], group):
            q = codes[:, at:at + group].double()
            if zeros is not None:
                q -= zeros[:, at // group, None]
            y += (x[:, at:at + group] @ q.t()) * scales[:, at // group].double()
        return y

    def back(dy, weight):
        codes, scales, zeros = weight
        parts = []
        for at in range(0, codes.shape[1], group):
            q = codes[:, at:at + group].double()
            if zeros is not None:
                q -= zeros[:, at // group, None]
            parts.append((dy * scales[:, at // group].double()) @ q)
        return torch.cat(parts, dim=1)

    if case["path"] == "product":
        return project(state["x"].double(), state["weights"][0])
    dy = state["dy"].double() if "dy" in state else None
    if case["path"] == "gradient":
        return back(dy, state["weights"][0])
    a, b = (project(state["x"].double(), w) for w in state["weights"])
    act = case["act"]
    if act == "silu":
        f = a / (1.0 + torch.exp(-a))
        slope = (1.0 + torch.exp(-a) * (1.0 + a)) / (1.0 + torch.exp(-a)) ** 2
    elif act == "gelu":
        # 0.5 (1 + tanh(z)) = 1 / (1 + exp(-2 z))
        z = math.sqrt(2.0 / math.pi) * (a + 0.044715 * a ** 3)
        p = 1.0 / (1.0 + torch.exp(-2.0 * z))
        f = a * p
        slope = p + a * 2.0 * p * (1.0 - p) * math.sqrt(2.0 / math.pi) * (1.0 + 0.134145 * a ** 2)
    else:
        f, slope = torch.where(a > 0, a * a, 0.0), torch.where(a > 0, 2.0 * a, 0.0)
    if case["path"] == "gated":
        return f * b
    da, db = dy * b * slope, dy * f
    return f * b, back(da, state["weights"][0]) + back(db, state["weights"][1]), torch.stack((da, db), dim=1)
