"""Drafting and answering of the sequence student on the host, with its reads replaced (no GPU)."""
import pytest
import torch

from paper_1807_02037_amd.sequence_student import SequenceStudent, verify


class Reads(SequenceStudent):
    """A student whose read adds 1 to the states and prefers the class behind the token's; the read number `fails` does not come back."""

    def __init__(self, slots=2, classes=7, fails=None):
        self.slots, self.classes, self.width, self.fails, self.reads = slots, classes, 4, fails, 0
        self.state = torch.zeros(slots, 4)

    def read(self, tokens, slots, into=None):
        self.reads += 1
        if self.reads == self.fails:
            raise RuntimeError("no answer")
        into = self.state if into is None else into
        into += 1
        return torch.nn.functional.one_hot((tokens + 1) % self.classes, self.classes) * 50.0


def test_drafting_leaves_the_states():
    s = Reads()
    state = s.state
    drafted, probs = s.draft(torch.tensor([0, 5]), 3, torch.full((2, 3), 0.5))
    assert drafted.tolist() == [[1, 2, 3], [6, 0, 1]] and probs.shape == (2, 3, 7)
    assert s.state is state and not state.any()


def test_drafting_leaves_the_states_after_an_error():
    s = Reads(fails=2)
    state = s.state
    with pytest.raises(RuntimeError, match="no answer"):
        s.draft(torch.tensor([0, 5]), 3, torch.full((2, 3), 0.5))
    assert s.state is state and not state.any()


@pytest.mark.parametrize("shape,dtype", [((3,), torch.int32), ((2,), torch.int64), ((2, 1), torch.int32)])
def test_verify_refuses_counts(shape, dtype, monkeypatch):
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    with pytest.raises(ValueError, match="counts:"):
        verify(torch.zeros(2, 4, 9), torch.zeros(2, 3, 9), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3), torch.zeros(2), torch.zeros(*shape, dtype=dtype))


def test_no_drafts():
    drafted, probs = Reads().draft(torch.tensor([0, 5]), 0, torch.empty(2, 0))
    assert drafted.shape == (2, 0) and drafted.dtype == torch.int64 and probs.shape == (2, 0, 7) and probs.dtype == torch.float32


@pytest.mark.parametrize("shape", [(1, 3), (2, 2), (2, 4), (3, 3)])
def test_random_numbers_of_another_size(shape):
    """One row would be the same numbers for every request."""
    with pytest.raises(ValueError, match="u:"):
        Reads().draft(torch.tensor([0, 5]), 3, torch.full(shape, 0.5))
