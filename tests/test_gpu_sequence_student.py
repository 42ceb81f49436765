"""The sequence operators used together: gradients of a whole step against fp64, single tokens like their rows of a batch, in 8 bits too, drafts and their verification with the states that they leave."""
import numpy as np
import pytest

import layer_oracle as O
import sequence_oracle as S

pytestmark = pytest.mark.gpu


def forward(s, tokens, offsets):
    w, p = {k: O.f64(v) for k, v in s.weights.items()}, {k: O.f64(v) for k, v in s.params.items()}
    e = O.f64(s.embed[tokens])
    xgo = e @ w["wp"] + p["bp"]
    x, g, o = np.split(xgo, 3, axis=1)
    return w, p, e, x, g, o


def close(got, want, roundings, name):
    # tensors between are rounded to bf16, 2^-8 of a value each: norms against norms
    assert np.linalg.norm(O.f64(got) - want) <= roundings * 2.0 ** -8 * np.linalg.norm(want), name


def test_step_against_fp64():
    import torch
    from paper_1807_02037_amd.sequence_student import SequenceStudent, batches
    rows, seqs, width, classes, top = 150, 5, 72, 203, 9
    teacher, s = SequenceStudent(rows, seqs, width, classes, top, seed=5), SequenceStudent(rows, seqs, width, classes, top, seed=6)
    tokens, offsets, t, ids = next(batches(teacher, rows, seqs, classes, top, torch.Generator(device="cuda").manual_seed(1)))
    loss = s.step(tokens, offsets, t, ids).item()
    w, p, e, x, g, o = forward(s, tokens, offsets)
    borders, zero = S.spans(rows, seqs, offsets.cpu().numpy()), np.zeros((seqs, width))
    h = S.recur(x, g, o, "silu", borders, zero)["y"][0]
    (n, _), (mean, _), (rstd, _) = S.group_norm_fwd(h, rows, 1, s.GROUPS, p["gamma"], p["beta"], "none", 1e-5, torch.bfloat16)
    r = n @ w["wd"] + p["bd"] + e
    z = r @ w["wh"]
    want, _, _, dz = O.distill(z, O.f64(t), ids.cpu().numpy(), np.ones(rows), 2.0, 1 / rows)
    assert abs(loss - want) <= 12 * 2.0 ** -8 * abs(want)
    dr = dz @ w["wh"].T
    dn = dr @ w["wd"].T
    (dh, _), (dgamma, _), (dbeta, _) = S.group_norm_bwd(dn, h, rows, 1, s.GROUPS, p["gamma"], p["beta"], mean, rstd, "none", torch.bfloat16)
    back = S.recur(x, g, o, "silu", borders, zero, dh, zero)
    dxgo = np.concatenate([back[k][0] for k in ("dx", "dg", "do")], 1)
    grads = {"wh": r.T @ dz, "wd": n.T @ dr, "bd": dr.sum(0), "gamma": dgamma, "beta": dbeta, "wp": e.T @ dxgo, "bp": dxgo.sum(0)}
    # at most twelve in a row: x, g, o, h, n, r, z, dz, dr, dn, dh, dxgo
    for k, v in grads.items():
        close(s.grads[k], v, 12, k)


def test_tokens_one_by_one_like_a_batch():
    import torch
    from paper_1807_02037_amd.sequence_student import SequenceStudent
    rows, seqs, width, classes = 64, 2, 96, 301
    s = SequenceStudent(rows, seqs, width, classes, 4, slots=3, seed=3)
    tokens = torch.randint(classes, (rows,), device="cuda")
    offsets = torch.tensor([0, 24, 64], dtype=torch.int32, device="cuda")
    z = s.logits(tokens, offsets).clone()
    # sequence 0 in slot 2, one token at a time; sequence 1 in slot 0, in runs of several tokens
    one = torch.cat([s.read(tokens[i:i + 1], torch.tensor([2], dtype=torch.int32, device="cuda")) for i in range(24)])
    runs = torch.cat([s.read(tokens[i:i + 8].contiguous(), torch.zeros(8, dtype=torch.int32, device="cuda")) for i in range(24, 64, 8)])
    # sums in another order may round x, g, o, h, n, r and z to either side
    close(torch.cat([one, runs]), O.f64(z), 7, "bf16")
    assert not s.state[1].any()
    # in 8 bits: three layers whose rows and weights are off by half a step of their largest, 1/254 of it; a normal row's largest is 3 of its root mean square here, and errors of many terms
    # add as the root of their squares: 3 / (254 sqrt 3) of a product for each operand, 1 % for both, of which the normalisation and the gates pass no more than they get
    s.state.zero_()
    s.quantise()
    q = torch.cat([s.read(tokens[:24].contiguous(), torch.full((24,), 2, dtype=torch.int32, device="cuda")),
                   s.read(tokens[24:].contiguous(), torch.zeros(40, dtype=torch.int32, device="cuda"))])
    assert np.linalg.norm(O.f64(q) - O.f64(z)) <= 0.06 * np.linalg.norm(O.f64(z))


def test_drafts_and_their_verification():
    """Whatever is accepted: the answers are as long as they say, tokens are classes, and the states of both models are those of their answers read from the start."""
    import torch
    from paper_1807_02037_amd.sequence_student import SequenceStudent, answer
    b, width, classes = 3, 64, 120
    teacher, student = SequenceStudent(32, 1, width, classes, 4, slots=b, seed=1), SequenceStudent(32, 1, width, classes, 4, slots=b, seed=1)
    student.quantise()                                             # the same weights in 8 bits: most drafts pass
    gen = torch.Generator(device="cuda").manual_seed(3)
    first = torch.randint(classes, (b,), generator=gen, device="cuda")
    answers, accepted = answer(student, teacher, first, 20, 4, gen)
    assert 2.0 < accepted <= 4.0 and min(map(len, answers)) >= 20
    assert all(0 <= t < classes for a in answers for t in a)
    for m in (teacher, student):
        fresh = SequenceStudent(32, 1, width, classes, 4, slots=b, seed=1)
        fresh.q8 = m.q8
        for i, a in enumerate(answers):
            read = torch.tensor([first[i].item()] + a[:-1], device="cuda")         # the last token has not been read yet
            fresh.read(read, torch.full((len(read),), i, dtype=torch.int32, device="cuda"))
        # x and g rounded to bf16 on either side
        assert np.linalg.norm(O.f64(fresh.state) - O.f64(m.state)) <= 2 * 2.0 ** -8 * np.linalg.norm(O.f64(m.state))


def test_training_runs():
    from paper_1807_02037_amd.sequence_student import train
    student, teacher, losses = train(steps=3, rows=256, seqs=4, width=64, classes=200, top=8, slots=2)
    assert np.isfinite(losses).all()
    assert all(v.isfinite().all() for v in student.grads.values())
