"""The student refuses tensors that its layers would read beyond their end, before anything is launched (no GPU)."""
import pytest
import torch

from paper_1807_02037_amd.student import Student


def student():
    s = Student.__new__(Student)                                    # the sizes alone
    s.rows, s.width, s.top = 6, 16, 3
    return s


GOOD = dict(x=((6, 16), torch.bfloat16), t=((6, 3), torch.float32), ids=((6, 3), torch.int32), weight=((6,), torch.float32))


@pytest.mark.parametrize("what,shape,dtype", [("t", (5, 3), torch.float32), ("t", (6, 3), torch.bfloat16), ("ids", (6, 2), torch.int32), ("ids", (6, 3), torch.int64),
                                              ("weight", (6,), torch.float64), ("weight", (1,), torch.float32)])
def test_step_refuses(what, shape, dtype, monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    args = {k: torch.zeros(*s, dtype=d) for k, (s, d) in GOOD.items()}
    args[what] = torch.zeros(*shape, dtype=dtype)
    with pytest.raises(ValueError, match=what + ":"):
        student().step(**args)


@pytest.mark.parametrize("call,rows", [("logits", 6), ("answer", 1)])
def test_features_refused(call, rows, monkeypatch):
    with pytest.raises(ValueError, match="on cpu"):
        getattr(student(), call)(torch.zeros(rows, 16, dtype=torch.bfloat16))
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    for bad in (torch.zeros(rows + 1, 16, dtype=torch.bfloat16), torch.zeros(rows, 8, dtype=torch.bfloat16), torch.zeros(rows, 16), torch.zeros(16, dtype=torch.bfloat16),
                torch.zeros(rows, 32, dtype=torch.bfloat16)[:, ::2]):
        with pytest.raises(ValueError, match="x:"):
            getattr(student(), call)(bad)
