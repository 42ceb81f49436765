"""The sequence student's verification with fewer drafts of some requests, and its answers at their ends, on the GPU."""
import pytest

import test_gpu_verify as V

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,d,c", [(6, 4, 300), (300, 3, 20000)])
def test_requests_with_fewer_drafts(b, d, c):
    import torch
    from paper_1807_02037_amd.sequence_student import verify
    p, q, t, n, u, v = V.make(3, b, d, c)
    args = [torch.as_tensor(x).cuda() for x in (p, q, t.astype("int32"), u, v)]
    for counts in (None, torch.as_tensor(n, dtype=torch.int32).cuda()):
        got = verify(*args, counts)
        want = V.rule(p.astype(float), q.astype(float), t, None if counts is None else n, u.astype(float), v.astype(float))
        assert (got[0].cpu().numpy() == want[0]).all() and (got[1].cpu().numpy() == want[1]).all()


def models(torch, b=3):
    from paper_1807_02037_amd.sequence_student import SequenceStudent
    return [SequenceStudent(32, 1, 64, 120, 4, slots=b, seed=1) for _ in range(2)], torch.Generator(device="cuda").manual_seed(3)


def test_answers_without_drafts_and_without_length():
    import torch
    from paper_1807_02037_amd.sequence_student import answer
    (student, teacher), gen = models(torch)
    first = torch.randint(120, (3,), generator=gen, device="cuda")
    answers, accepted = answer(student, teacher, first, 5, 0, gen)
    assert [len(a) for a in answers] == [5, 5, 5] and accepted == 0 and all(0 <= t < 120 for a in answers for t in a)
    assert torch.equal(student.state, teacher.state) and student.state.any()
    assert answer(student, teacher, first, 0, 4, gen) == ([[], [], []], 0)


def test_no_class_to_take():
    """Logits that are not finite: an error, not tokens that are no class."""
    import torch
    from paper_1807_02037_amd.sequence_student import answer
    (student, teacher), gen = models(torch)
    teacher.weights["wh"][3] = float("nan")
    with pytest.raises(ValueError, match="no class"):
        answer(student, teacher, torch.randint(120, (3,), generator=gen, device="cuda"), 5, 2, gen)


def test_no_tokens():
    import torch
    (student, _), _ = models(torch)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    for _ in range(2):
        assert student.read(none, none.int()).shape == (0, 120) and not student.state.any()
        student.quantise()
