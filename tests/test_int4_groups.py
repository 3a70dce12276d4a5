"""One scale per row, said with a number of any size."""
import contextlib

import pytest

torch = pytest.importorskip("torch")
rsr = pytest.importorskip("paper_2603_27462_amd")
from paper_2603_27462_amd import binding  # noqa: E402

# (as 64-bit integers: negative, 0, 32, 2^63 - 1 and 32 again)
GROUPS = [301, 1 << 63, 1 << 64, (1 << 64) + 32, (1 << 64) + (1 << 63) - 1, (1 << 200) + 32]


@pytest.mark.parametrize("group", GROUPS + [300])
def test_what_the_library_is_told(monkeypatch, group):
    """On the CPU: the group that is passed on never asks for more scales than one per row."""
    told = []

    class OnGpu(torch.Tensor):
        is_cuda = True

    class Library:
        def rsr_preprocess_int4(self, Q, scales, zeros, rows, cols, group):
            told.append((rows, cols, group))
            return 1

    class Stream:
        def synchronize(self):
            pass

    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(torch.cuda, "device", lambda device: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    Q = torch.zeros((4, 300), dtype=torch.int8).as_subclass(OnGpu)
    h = rsr.rsr_preprocess_int4(Q, torch.ones((4, 1)), group)
    h.ptr = 0                                       # (not the library's)
    assert told == [(4, 300, 300)]


@pytest.mark.gpu
@pytest.mark.parametrize("group", GROUPS)
def test_one_scale_per_row(group):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(3)
    Q = torch.randint(-8, 8, (70, 300), generator=g, device="cuda:0", dtype=torch.int8)
    s = torch.exp2(torch.randint(-1, 2, (70, 1), generator=g, device="cuda:0").float())
    z = torch.randint(-8, 8, (70, 1), generator=g, device="cuda:0", dtype=torch.int8)
    v = torch.randint(-3, 4, (3, 300), generator=g, device="cuda:0").float()
    got = rsr.rsr_int4_matvec(rsr.rsr_preprocess_int4(Q, s, group, zeros=z), v)
    assert torch.equal(got, (v.double() @ ((Q.double() - z) * s).t()).float())
