"""Every kernel on 4-bit weights, asked for by its name and compared with the definition in 64 bits.

The cases below name all kernels that the built library has (checked on the CPU), at sizes that end inside tiles, groups of rows and
vectors, with enough columns (or rows, transposed) for the waves' loops to run several times.  Vectors are small whole numbers, scales
1 to 2 in steps of 2^-7, and every sum stays below 2^17: any partial sum in any order is a float32, and results have to be equal."""
import os
import re

import pytest

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"
NAMES = {F32: "float", BF16: "unsigned short"}
CODES = {F32: rsr.RSR_F32, BF16: rsr.RSR_BF16}
PER_TILE = {32: 8, 64: 4, 128: 2}


def _forward():
    """(kernel, rows, cols, group, batch, type of the vectors, number of matrices, zero points)"""
    cases = []
    for group, per in PER_TILE.items():
        for dtype in (F32, BF16):
            for n in (1, 2):
                def case(kernel, numbers, rows, cols, batch, zeros):
                    cases.append(("%s<%s, %s>" % (kernel, NAMES[dtype], numbers), rows, cols, group, batch, dtype, n, zeros))

                case("k_int4_few", "1, %d, %d" % (per, n), 51, 20011, 1, True)
                case("k_int4_few", "4, %d, %d" % (per, n), 51, 20011, 3, False)
                case("k_int4_few", "4, %d, %d" % (per, n), 3001, 1300, 4, True)
                split = "%%d, %d, %d, %%d, %%d" % (per, n)
                if dtype == BF16:
                    case("k_int4_split", split % (1, 1, 16), 100, 9001, 9, True)
                    case("k_int4_split", split % (2, 1, 8), 100, 4111, 45, True)
                    case("k_int4_split", split % (2, 2, 8), 8209, 4111, 29, False)
                case("k_int4_split", split % (1, 1, 8), 100, 4095 if dtype == BF16 else 4111, 13, False)
                case("k_int4_split", split % (1, 2, 8), 8209, 4111, 11, True)
                for zeros in (False, True):
                    case("k_int4_tile", "%d, %d, %s" % (per, n, "true" if zeros else "false"), 2099 if n == 1 else 1051, 777, 789, zeros)
    return cases


def _transposed():
    """(kernel, rows, cols, group, batch, type of the vectors, of the results, number of matrices, zero points)"""
    cases = []
    for dtype, result, n in ((BF16, F32, 1), (BF16, BF16, 1), (F32, F32, 1), (F32, BF16, 1), (F32, F32, 2), (F32, BF16, 2)):
        planes = 2 if result == BF16 and (dtype == BF16 or n == 2) else 3
        for group in PER_TILE:
            def case(kernel, numbers, rows, cols, batch, zeros):
                cases.append(("%s<%s, %s, %s>" % (kernel, NAMES[dtype], NAMES[result], numbers), rows, cols, group, batch, dtype, result, n, zeros))

            split = "%d, %d, %%d, %%d" % (planes, 2 if group == 32 else 1)
            case("k_int4_back_split", split % (16, 8), 777, 333, 13, True)
            case("k_int4_back_split", split % (32, 8), 777, 333, 45, False)
            if dtype == BF16 and result == BF16:
                case("k_int4_back_split", split % (16, 16), 3001, 333, 9, True)
            if group == 128 and planes == 3:
                case("k_int4_back_tile", "3, 1, 64, 2", 1001, 8003, 200, True)
                case("k_int4_back_tile", "3, 1, 64, 2", 1024, 8064, 256, False)
            if group == 128 and planes == 2:
                case("k_int4_back_tile", "2, 1, 128, 2", 1001, 8003, 200, True)
                case("k_int4_back_tile", "2, 1, 128, 2", 1024, 8064, 256, False)
                case("k_int4_back_tile", "2, 1, 64, 1", 1001, 8003, 397, False)
                case("k_int4_back_tile", "2, 1, 64, 1", 1024, 8064, 448, True)
            if group == 64 and planes == 2:
                case("k_int4_back_tile", "2, 2, 32, 1", 301, 14003, 597, True)
                case("k_int4_back_tile", "2, 2, 32, 1", 320, 14080, 640, False)
    return cases


def test_the_cases_name_every_kernel():
    """(on the CPU: the names of the kernels are in the built library)"""
    lib = rsr.load_library()._name
    found = set()
    with open(os.path.abspath(lib), "rb") as f:
        for kernel, args in re.findall(rb"\d+(k_int4_(?:few|split|tile|back_split|back_tile))I((?:[tf]|L[ib]\d+E)+)E", f.read()):
            numbers = [{"t": "unsigned short", "f": "float"}.get(a, a) for a in re.findall(r"[tf]|L[ib]\d+(?=E)", args.decode())]
            numbers = [a if a[0] != "L" else ("true" if a == "Lb1" else "false") if a[1] == "b" else a[2:] for a in numbers]
            found.add("%s<%s>" % (kernel.decode(), ", ".join(numbers)))
    named = {c[0] for c in _forward()} | {c[0] for c in _transposed()}
    # (a float32 product into bf16 of one matrix keeps all bits, of two 16: the types alone do not say which)
    assert found == named, (sorted(found - named), sorted(named - found))


# ---- on the GPU ---------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _weight(rows, cols, group, zeros, seed):
    """a handle, and its matrix in 64 bits"""
    g = _gen(seed)
    n = -(-cols // group)
    Q = torch.randint(-8, 8, (rows, cols), generator=g, device=DEV, dtype=torch.int8)
    s = 1.0 + torch.randint(0, 128, (rows, n), generator=g, device=DEV) / 128.0
    z = torch.randint(-8, 8, (rows, n), generator=g, device=DEV, dtype=torch.int8) if zeros else None
    M = Q.double()
    if zeros:
        M -= z.double().repeat_interleave(group, dim=1)[:, :cols]
    M *= s.double().repeat_interleave(group, dim=1)[:, :cols]
    return rsr.rsr_preprocess_int4(Q, s, group, zeros=z), M


def _whole(batch, length, most, dtype, seed):
    """whole numbers, with NaN behind every vector"""
    buf = torch.full((batch, length + 3), float("nan"), device=DEV, dtype=dtype)
    buf[:, :length] = torch.randint(-most, most + 1, (batch, length), generator=_gen(seed), device=DEV).to(dtype)
    return buf[:, :length]


def _guarded(batch, length, dtype):
    buf = torch.full((batch, length + 5), -77.0, device=DEV, dtype=dtype)
    return buf, buf[:, :length]


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,rows,cols,group,batch,dtype,n,zeros", _forward())
def test_forward(kernel, rows, cols, group, batch, dtype, n, zeros):
    h, M = _weight(rows, cols, group, zeros, 1)
    x = _whole(batch, cols, 3, dtype, 3)
    a = x.double() @ M.t()
    assert a.abs().max() < 2 ** 17
    a = a.float()
    if n == 1:
        assert rsr.rsr_int4_kernel_name(h, v_dtype=CODES[dtype], batch=batch) == kernel
        assert rsr.rsr_batch_kernel_name(h, CODES[dtype], batch) == kernel
        for result in (F32, BF16):
            buf, out = _guarded(batch, rows, result)
            rsr.rsr_int4_matvec(h, x, scale=-2.0, out=out)
            assert torch.equal(out, (-2.0 * a).to(result)) and bool((buf[:, rows:] == -77.0).all())
        return
    up, Mu = _weight(rows, cols, group, False, 2)       # (zero points on one side, or none)
    b = x.double() @ Mu.t()
    assert b.abs().max() < 2 ** 17
    b = b.float()
    assert rsr.rsr_int4_kernel_name(h, up, v_dtype=CODES[dtype], batch=batch) == kernel
    for result in (F32, BF16):
        buf, out = _guarded(batch, rows, result)
        pre = torch.full((batch, 2, rows), -77.0, device=DEV)
        rsr.rsr_gated(h, up, x, "relu2", out=out, pre=pre)
        assert torch.equal(pre, torch.stack((a, b), dim=1))
        r = torch.relu(a)
        # (two roundings of products, as here)
        assert torch.equal(out, (r * r * b).to(result)) and bool((buf[:, rows:] == -77.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,rows,cols,group,batch,dtype,result,n,zeros", _transposed())
def test_transposed(kernel, rows, cols, group, batch, dtype, result, n, zeros):
    h, M = _weight(rows, cols, group, zeros, 4)
    buf, out = _guarded(batch, cols, result)
    if n == 1:
        assert rsr.rsr_int4_kernel_name(h, None, True, CODES[dtype], CODES[result], batch) == kernel
        y = _whole(batch, rows, 7, dtype, 5)
        want = -2.0 * (y.double() @ M)
        rsr.rsr_int4_matvec(h, y, transposed=True, scale=-2.0, out=out)
    else:
        up, Mu = _weight(rows, cols, group, not zeros, 6)
        assert rsr.rsr_int4_kernel_name(h, up, True, rsr.RSR_F32, CODES[result], batch) == kernel
        # relu2 of whole numbers: da = 2 dh b a and db = dh a^2 are whole too, up to 16
        pre = _whole(batch, 2 * rows, 2, F32, 7).reshape(batch, 2, rows).contiguous()
        dh = _whole(batch, rows, 2, BF16, 8)
        _, dpre = rsr.rsr_gated_backward(h, up, pre, dh, "relu2", dv=out)
        a, d = torch.relu(pre[:, 0]), dh.float()
        assert torch.equal(dpre, torch.stack((2 * d * pre[:, 1] * a, d * a * a), dim=1))
        want = dpre[:, 0].double() @ M + dpre[:, 1].double() @ Mu
    assert want.abs().max() < 2 ** 17
    assert torch.equal(out, want.to(result)) and bool((buf[:, cols:] == -77.0).all())


@pytest.mark.gpu
def test_names_that_are_refused():
    h, _ = _weight(16, 64, 64, False, 1)
    other, _ = _weight(17, 64, 64, False, 1)
    ternary = rsr.rsr_preprocess(torch.ones((16, 64), dtype=torch.int8, device=DEV), 4, rsr.RSR_TERNARY_FUSED)
    for args, code in (((ternary,), 1), ((h, other), 1), ((h, ternary), 1), ((h, None, False, 2), 1), ((h, None, True, 0, 2), 1),
                       ((h, None, False, 0, 0, 0), 1), ((h, h, True, rsr.RSR_BF16), 1), ((h, None, False, 0, 0, (1 << 24) + 1), 3)):
        with pytest.raises(rsr.RsrError) as e:
            rsr.rsr_int4_kernel_name(*args)
        assert e.value.code == code
    assert rsr.rsr_int4_kernel_name(h, batch=1 << 24).startswith("k_int4_")
