"""The sequence student refuses tensors that its operators would read beyond their end, before anything is launched (no GPU)."""
import pytest
import torch

from paper_1807_02037_amd import sequence_student
from paper_1807_02037_amd.sequence_student import SequenceStudent


@pytest.fixture
def on_gpu(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))


def student():
    s = SequenceStudent.__new__(SequenceStudent)                   # the sizes alone
    s.rows, s.seqs, s.width, s.classes, s.top, s.slots = 6, 2, 16, 30, 3, 4
    s.state = torch.zeros(4, 16)
    return s


GOOD = dict(tokens=((6,), torch.int64), offsets=((3,), torch.int32), t=((6, 3), torch.float32), ids=((6, 3), torch.int32))


@pytest.mark.parametrize("what,shape,dtype", [("tokens", (5,), torch.int64), ("tokens", (6,), torch.int32), ("offsets", (2,), torch.int32), ("offsets", (3,), torch.int64),
                                              ("t", (6, 2), torch.float32), ("t", (6, 3), torch.bfloat16), ("ids", (6, 3), torch.int64)])
def test_step_refuses(what, shape, dtype, on_gpu):
    args = {k: torch.zeros(*s, dtype=d) for k, (s, d) in GOOD.items()}
    args[what] = torch.zeros(*shape, dtype=dtype)
    with pytest.raises(ValueError, match=what + ":"):
        student().step(**args)


@pytest.mark.parametrize("what,kw", [("tokens", dict(tokens=torch.zeros(3, dtype=torch.int32))), ("slots", dict(slots=torch.zeros(2, dtype=torch.int32))),
                                     ("slots", dict(slots=torch.zeros(3, dtype=torch.int64))), ("into", dict(into=torch.zeros(3, 16))), ("into", dict(into=torch.zeros(4, 16).half()))])
def test_read_refuses(what, kw, on_gpu):
    args = {**dict(tokens=torch.zeros(3, dtype=torch.int64), slots=torch.zeros(3, dtype=torch.int32)), **kw}
    with pytest.raises(ValueError, match=what + ":"):
        student().read(**args)


@pytest.mark.parametrize("what,shape,dtype", [("p", (2, 3, 9), torch.float32), ("p", (2, 4, 9), torch.float64), ("drafted", (2, 3), torch.int64), ("u", (2, 2), torch.float32),
                                              ("v", (3,), torch.float32)])
def test_verify_refuses(what, shape, dtype, on_gpu):
    good = dict(p=torch.zeros(2, 4, 9), q=torch.zeros(2, 3, 9), drafted=torch.zeros(2, 3, dtype=torch.int32), u=torch.zeros(2, 3), v=torch.zeros(2))
    with pytest.raises(ValueError, match=what + ":"):
        sequence_student.verify(**{**good, what: torch.zeros(*shape, dtype=dtype)})


def test_widths_of_whole_groups():
    with pytest.raises(ValueError, match="width"):
        SequenceStudent(8, 1, 30, 10, 2)
