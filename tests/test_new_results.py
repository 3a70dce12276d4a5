"""Results that a call makes for a stream of the caller's are allocated on that stream."""
import contextlib

import pytest

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
from paper_2603_27462_amd import binding  # noqa: E402


class _Library:
    """every function succeeds"""

    def __getattr__(self, name):
        return lambda *args: 0


def test_allocated_on_the_stream_given(monkeypatch):
    """On the CPU, with torch's streams replaced: which one is current when a result is allocated."""
    class Stream:
        cuda_stream = 7

    current, seen, kept = ["outer"], [], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: kept.append(stream))
    monkeypatch.setattr(torch, "empty", lambda *args, **kw: seen.append(current[-1]) or empty(*args, **kw))
    monkeypatch.setattr(binding, "load_library", _Library)
    monkeypatch.setattr(binding, "_current_device", lambda: None)
    h = rsr.Handle(0, 4, 64, 0, rsr.RSR_INT4)
    h.device = torch.device("cpu")
    x, dh, pre = torch.zeros((3, 64)), torch.zeros((3, 4)), torch.zeros((3, 2, 4))
    side = Stream()
    assert rsr.rsr_int4_matvec(h, x, stream=side).shape == (3, 4)
    assert rsr.rsr_gated(h, h, x, stream=side).shape == (3, 4)
    dv, dpre = rsr.rsr_gated_backward(h, h, pre, dh, stream=side)
    assert dv.shape == (3, 64) and dpre.shape == (3, 2, 4)
    assert seen == [side] * 4 and kept == ["outer"] * 4
    given = empty((3, 4))
    assert rsr.rsr_int4_matvec(h, x, out=given, stream=side) is given and len(seen) == 4


@pytest.mark.gpu
def test_results_on_a_side_stream(monkeypatch):
    """Every product with a stream given, its result made by the call: allocated there, and right."""
    dev = "cuda:0"
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    M = torch.randint(-1, 2, (40, 64), generator=g, dtype=torch.int8, device=dev)
    h, two = rsr.rsr_preprocess(M, 4, rsr.RSR_TERNARY_FUSED), rsr.rsr_preprocess_stacked([M, M], 4, rsr.RSR_TERNARY_FUSED)
    h4 = rsr.rsr_preprocess_int4(M, torch.ones((40, 1), device=dev), 64)
    x, dh, pre = torch.ones((3, 64), device=dev), torch.ones((3, 40), device=dev), torch.ones((3, 2, 40), device=dev)
    sums = M.sum(dim=1, dtype=torch.float32)
    torch.cuda.synchronize()
    side, seen, empty = torch.cuda.Stream(), [], torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: seen.append(torch.cuda.current_stream()) or empty(*a, **k))
    raw = torch.cuda.ExternalStream(side.cuda_stream)
    outs = [rsr.rsr_matvec(h, x[0], stream=side), rsr.rsr_matvec_ex(h, x[0], stream=raw), *rsr.rsr_matvec_stacked(two, x[0], stream=side),
            rsr.rsr_int4_matvec(h4, x[0], stream=side)]
    batches = [rsr.rsr_matvec_ex(h, x, stream=side), rsr.rsr_int4_matvec(h4, x, stream=side)]
    gated = rsr.rsr_gated(h4, h4, x, "relu2", stream=side)
    dv, dpre = rsr.rsr_gated_backward(h4, h4, pre, dh, "relu2", stream=side)
    side.synchronize()
    assert len(seen) == 10 and all(s.cuda_stream == side.cuda_stream for s in seen)
    assert all(torch.equal(o, sums) for o in outs) and all(torch.equal(o, sums.expand(3, -1)) for o in batches)
    assert torch.equal(gated, (torch.relu(sums) ** 2 * sums).expand(3, -1))
    assert torch.equal(dpre, torch.stack((2 * dh, dh), dim=1)) and torch.equal(dv, 3 * M.sum(dim=0, dtype=torch.float32).expand(3, -1))
