"""A small student of a language model, trained by distillation: the language-model layers of the library used together.

    python -m paper_1807_02037_amd.student [--steps 60] [--width 256] [--classes 2000]

A position's features x (fixed embeddings of its last two tokens) pass a gated feed-forward block with a residual sum and a head over the
vocabulary; the loss is the distillation from a teacher's top logits.  Everything but the embedding lookup and the update of the weights
runs in liblms.so:

    h = silu(x wg) * (x wu)        lms_gated_fwd
    y = h wd + bd + x              lms_linear_fwd with bias and residual
    z = y wh                       lms_linear_fwd
    loss, dz                       lms_distill_loss_grad, dz over z
    dy, dwh; dh, dwd, dbd; dwg, dwu    lms_linear_bwd twice, lms_gated_bwd

`answer` is the same forward pass for one position, as a program that answers token by token calls it."""
import argparse

import torch

from . import _lib as A
from . import api as L


def _bf16(*shape, scale, gen):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(torch.bfloat16)


def _expect(what, t, shape, dtype):
    """The layers take addresses: a tensor of another size, type or place would be read beyond its end."""
    if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{what}: a contiguous {dtype} tensor of {shape} on the GPU is needed, not {t.dtype} {tuple(t.shape)} on {t.device}")


class Student:
    """Weights, the buffers of a batch of `rows` positions, and the calls on them.  keep: the forward pass keeps g and u for the backward pass (else it computes
    them again)."""

    def __init__(self, rows, width, hidden, classes, top, temperature=2.0, seed=0, keep=True):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rows, self.width, self.hidden, self.classes, self.top, self.keep = rows, width, hidden, classes, top, keep
        self.embed = _bf16(classes, width, scale=0.7, gen=gen)
        self.weights = {"wg": _bf16(width, hidden, scale=width ** -0.5, gen=gen), "wu": _bf16(width, hidden, scale=width ** -0.5, gen=gen),
                        "wd": _bf16(hidden, width, scale=hidden ** -0.5, gen=gen), "wh": _bf16(width, classes, scale=width ** -0.5, gen=gen)}
        self.bias = torch.zeros(width, device="cuda")
        self.grads = {k: torch.empty(v.shape, device="cuda") for k, v in self.weights.items()}
        self.dbias = torch.empty_like(self.bias)
        self.gated, self.down, self.head = self._descs(rows)
        self.loss_desc = L.distill_desc(rows, classes, top, temperature=temperature, scale=1.0 / rows)

        def act(cols):
            return torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
        self.g, self.u, self.h = (act(hidden) if keep else None), (act(hidden) if keep else None), act(hidden)
        self.y, self.z, self.dy, self.dh = act(width), act(classes), act(width), act(hidden)
        self.loss = torch.empty(1, device="cuda")
        need = [L.gated_workspace_bytes(self.gated, w) for w in (A.GATED_FWD, A.GATED_BWD if keep else A.GATED_BWD_RECOMPUTE)]
        need += [L.linear_workspace_bytes(d, w) for d in (self.down, self.head) for w in (A.LINEAR_FWD, A.LINEAR_BWD)]
        need.append(L.distill_workspace_bytes(self.loss_desc, A.DISTILL_LOSS_GRAD))
        one = self._descs(1)
        need += [L.gated_workspace_bytes(one[0], A.GATED_FWD)] + [L.linear_workspace_bytes(d, A.LINEAR_FWD) for d in one[1:]]
        self.ws = torch.empty(max(need) + 16, dtype=torch.uint8, device="cuda")

    def _descs(self, rows):
        return (L.gated_desc(rows, self.hidden, self.width, act=A.ACT_SILU), L.linear_desc(rows, self.width, self.hidden),
                L.linear_desc(rows, self.classes, self.width))

    def features(self, tokens):
        """tokens: (rows, 2) class numbers."""
        e = self.embed[tokens]
        return (e[:, 0] + e[:, 1].roll(1, dims=1)).contiguous()

    def _forward(self, descs, x, h, g, u, y, z, stream):
        w, ws = self.weights, self.ws.data_ptr()
        ptr = [None if t is None else t.data_ptr() for t in (x, h, g, u, y, z)]
        L.gated_fwd(descs[0], ptr[0], w["wg"].data_ptr(), w["wu"].data_ptr(), ptr[1], ptr[2], ptr[3], ws, stream)
        L.linear_fwd(descs[1], ptr[1], w["wd"].data_ptr(), self.bias.data_ptr(), ptr[0], ptr[4], None, ws, stream)
        L.linear_fwd(descs[2], ptr[4], w["wh"].data_ptr(), None, None, ptr[5], None, ws, stream)

    def logits(self, x):
        """Logits of the batch (the student's own buffer)."""
        _expect("x", x, (self.rows, self.width), torch.bfloat16)
        self._forward((self.gated, self.down, self.head), x, self.h, self.g, self.u, self.y, self.z, torch.cuda.current_stream().cuda_stream)
        return self.z

    def answer(self, x):
        """Logits of one position: x is (1, width)."""
        _expect("x", x, (1, self.width), torch.bfloat16)
        h, y, z = (torch.empty(1, c, dtype=torch.bfloat16, device="cuda") for c in (self.hidden, self.width, self.classes))
        self._forward(self._descs(1), x, h, None, None, y, z, torch.cuda.current_stream().cuda_stream)
        return z

    def step(self, x, t, ids, weight=None):
        """Forward, loss and gradients of a batch; t, ids: the teacher's top logits and their classes.  Returns the loss (a tensor, not waited for)."""
        _expect("t", t, (self.rows, self.top), torch.float32)
        _expect("ids", ids, (self.rows, self.top), torch.int32)
        if weight is not None:
            _expect("weight", weight, (self.rows,), torch.float32)
        s, w, g, ws = torch.cuda.current_stream().cuda_stream, self.weights, self.grads, self.ws.data_ptr()
        self.logits(x)
        L.distill_loss_grad(self.loss_desc, self.z.data_ptr(), t.data_ptr(), ids.data_ptr(), None if weight is None else weight.data_ptr(),
                            self.loss.data_ptr(), self.z.data_ptr(), ws, s)
        L.linear_bwd(self.head, self.z.data_ptr(), self.y.data_ptr(), w["wh"].data_ptr(), None, self.dy.data_ptr(), g["wh"].data_ptr(), None, ws, s)
        L.linear_bwd(self.down, self.dy.data_ptr(), self.h.data_ptr(), w["wd"].data_ptr(), None, self.dh.data_ptr(), g["wd"].data_ptr(),
                     self.dbias.data_ptr(), ws, s)
        L.gated_bwd(self.gated, self.dh.data_ptr(), x.data_ptr(), w["wg"].data_ptr(), w["wu"].data_ptr(), self.g.data_ptr() if self.keep else None,
                    self.u.data_ptr() if self.keep else None, None, g["wg"].data_ptr(), g["wu"].data_ptr(), ws, s)
        return self.loss

    def update(self, lr):
        for k, v in self.weights.items():
            v.copy_(v.float() - lr * self.grads[k])
        self.bias -= lr * self.dbias


def teacher_top(teacher, tokens, top):
    """The top logits of a teacher (here a student of other weights) and their classes."""
    t, ids = torch.topk(teacher.logits(teacher.features(tokens)).float() * 3.0, top, dim=1)
    return t.contiguous(), ids.int().contiguous()


def train(steps=60, rows=1024, width=256, classes=2000, top=32, lr=6.0, seed=0):
    """Trains a student on a synthetic teacher; returns the losses."""
    teacher = Student(rows, width, 4 * width, classes, top, seed=seed + 1)
    student = Student(rows, width, 2 * width, classes, top, seed=seed)
    student.embed = teacher.embed
    gen = torch.Generator(device="cuda").manual_seed(seed + 2)
    losses = []
    for _ in range(steps):
        tokens = torch.randint(classes, (rows, 2), generator=gen, device="cuda")
        t, ids = teacher_top(teacher, tokens, top)
        losses.append(student.step(student.features(tokens), t, ids).clone())
        student.update(lr)
    return [v.item() for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--rows", type=int, default=1024)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--classes", type=int, default=2000)
    ap.add_argument("--lr", type=float, default=6.0)
    a = ap.parse_args()
    losses = train(a.steps, a.rows, a.width, a.classes, lr=a.lr)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {i:4d}  loss {losses[i]:.4f}")
    print(f"step {len(losses) - 1:4d}  loss {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
