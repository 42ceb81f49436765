"""The language-model layers used together: gradients of a whole step against fp64, the loss falls in training, one position answers like its row of a batch."""
import numpy as np
import pytest

import layer_oracle as O

pytestmark = pytest.mark.gpu


def test_step_against_fp64():
    import torch
    from paper_1807_02037_amd.student import Student, teacher_top
    rows, width, classes, top = 70, 72, 203, 9
    for keep in (True, False):
        teacher, s = Student(rows, width, 160, classes, top, seed=5), Student(rows, width, 136, classes, top, seed=6, keep=keep)
        tokens = torch.randint(classes, (rows, 2), device="cuda")
        t, ids = teacher_top(teacher, tokens, top)
        weight = torch.rand(rows, device="cuda")
        x = s.features(tokens)
        loss = s.step(x, t, ids, weight).item()
        xx, w = O.f64(x), {k: O.f64(v) for k, v in s.weights.items()}
        g, u = xx @ w["wg"], xx @ w["wu"]
        a, slope = O.act("silu", g)
        h = a * u
        y = h @ w["wd"] + xx
        z = y @ w["wh"]
        want, _, _, dz = O.distill(z, O.f64(t), ids.cpu().numpy(), O.f64(weight), 2.0, 1 / rows)
        dy = dz @ w["wh"].T
        dh = dy @ w["wd"].T
        grads = {"wh": y.T @ dz, "wd": h.T @ dy, "wg": xx.T @ (dh * u * slope), "wu": xx.T @ (dh * a)}
        # every tensor between is rounded to bf16, 2^-8 of a value: nine of them at most (h, y, z, dz, dy, dh, g, u, dg) in a row, norms against norms
        assert abs(loss - want) <= 9 * 2.0 ** -8 * abs(want)
        for k, v in grads.items():
            assert np.linalg.norm(O.f64(s.grads[k]) - v) <= 9 * 2.0 ** -8 * np.linalg.norm(v), k
        assert np.linalg.norm(O.f64(s.dbias) - dy.sum(0)) <= 9 * 2.0 ** -8 * np.linalg.norm(dy.sum(0))


def test_training_lowers_the_loss():
    from paper_1807_02037_amd.student import train
    losses = train(steps=40, rows=512, width=128, classes=600, top=16, lr=2.0)
    assert np.isfinite(losses).all()
    assert np.mean(losses[-5:]) < 0.8 * np.mean(losses[:5]), losses[::8]


def test_one_position_answers_like_its_row():
    import torch
    from paper_1807_02037_amd.student import Student
    s = Student(33, 256, 512, 1003, 8, seed=3)
    x = s.features(torch.randint(1003, (33, 2), device="cuda"))
    z = s.logits(x).clone()
    for i in (0, 17, 32):
        one = s.answer(x[i:i + 1].contiguous())
        # sums of 32 bits in another order, and h, y and z each rounded to bf16 on either side of a border
        off = np.linalg.norm(O.f64(one[0]) - O.f64(z[i])) / np.linalg.norm(O.f64(z[i]))
        assert off <= 3 * 2.0 ** -8
