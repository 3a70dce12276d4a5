"""What the entries on 4-bit weights refuse before any device call: on the CPU."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")

EINVAL, EUNSUPPORTED = 1, 3
SOME = ctypes.c_void_p(4096)            # a pointer that nothing may follow


def _preprocess(Q=SOME, scales=SOME, zeros=None, rows=4, cols=64, group=32):
    lib = rsr.load_library()
    assert not lib.rsr_preprocess_int4(Q, scales, zeros, rows, cols, group)
    return lib.rsr_last_error()


@pytest.mark.parametrize("args", [dict(Q=None), dict(scales=None), dict(rows=0), dict(cols=0), dict(rows=-3), dict(group=0),
                                  dict(group=-32)])
def test_preprocess_invalid(args):
    assert _preprocess(**args) == EINVAL


@pytest.mark.parametrize("args", [dict(group=31), dict(group=48), dict(rows=(1 << 24) + 1), dict(rows=(1 << 30) + 1), dict(cols=(1 << 24) + 1),
                                  dict(cols=1 << 40)])
def test_preprocess_beyond_the_limits(args):
    assert _preprocess(**args) == EUNSUPPORTED


def test_products_without_a_handle():
    lib = rsr.load_library()
    junk = ctypes.create_string_buffer(4096)            # not a handle: its magic is wrong
    for h in (None, ctypes.addressof(junk)):
        assert lib.rsr_int4_matvec(h, 0, SOME, 0, 1.0, SOME, 0, 1, 64, 64, None) == EINVAL
        assert lib.rsr_gated(h, h, SOME, 0, 0, SOME, 0, None, 1, 64, 64, None) == EINVAL
        assert lib.rsr_gated_backward(h, h, SOME, SOME, 0, 0, SOME, None, 0, 1, 64, 64, None) == EINVAL
        assert lib.rsr_last_error() == EINVAL


def test_other_kinds_do_not_become_int4():
    lib = rsr.load_library()
    assert not lib.rsr_preprocess(SOME, 4, 64, 4, rsr.RSR_INT4) and lib.rsr_last_error() == EINVAL


def test_binding_refuses_what_is_not_on_a_gpu():
    Q, s = torch.zeros((4, 64), dtype=torch.int8), torch.ones((4, 2))
    with pytest.raises(TypeError):
        rsr.rsr_preprocess_int4(Q, s, 32)
    other = rsr.Handle(0, 4, 64, 4, rsr.RSR_TERNARY_FUSED)
    with pytest.raises(TypeError, match="int4 handle"):
        rsr.rsr_int4_matvec(other, torch.zeros(64))
    with pytest.raises(TypeError, match="int4 handle"):
        rsr.rsr_gated(other, other, torch.zeros(64))
    h = rsr.Handle(0, 4, 64, 0, rsr.RSR_INT4)
    h.device = torch.device("cuda", 0)
    for v in (torch.zeros(64), torch.zeros((2, 63)), None):
        with pytest.raises(TypeError):
            rsr.rsr_int4_matvec(h, v)
        with pytest.raises(TypeError):
            rsr.rsr_gated(h, h, v)
        with pytest.raises(TypeError):
            rsr.rsr_gated_backward(h, h, None, v)


def test_activations_by_name_and_number():
    from paper_2603_27462_amd import binding
    assert [binding._act_code(a) for a in ("silu", "gelu", "relu2", 0, 1, 2)] == [0, 1, 2, 0, 1, 2]
    for bad in ("relu", 3, -1, None):
        with pytest.raises(ValueError):
            binding._act_code(bad)
