"""Timed operators of a language model's training and serving: the linear layer with its epilogue, the gated feed-forward
projection and the distillation loss, each with its backward pass.

`run` computes them in plain torch operations in 32 bits, or, with `own` set, through the framework's entry points.

  linear    y = act(x w + b) + r, keeping pre = x w + b for the backward pass;
            backward: dz = dy act'(pre), dx = dz w^T, dw = x^T dz, db = sum over rows of dz
  gated     h = act(x wg) * (x wu), keeping g = x wg and u = x wu, or not;
            backward: dg = dh u act'(g), du = dh act(g), dx = dg wg^T + du wu^T, dwg = x^T dg, dwu = x^T du;
            where g and u were not kept they are computed again
  distill   p = softmax(t / T) over the teacher's top logits of a row, q = softmax(z / T) over all classes,
            loss = scale * sum over rows of weight * T^2 * sum_j p_j (log p_j - log q[id_j]);
            dz = scale * weight * T * (q - p) for the rows that have a teacher entry, else 0

Weights lie as (inputs, outputs).  Weight gradients are fp32 where the gradient that enters the product is a tensor of the
storage type as it is (no activation), else of the storage type; bias gradients are fp32."""
import math

import torch

own = False

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
MAX_FLOPS = 2.2e12
MAX_BYTES = 1.0e9
SQRT_HALF = math.sqrt(0.5)
TANH_A, TANH_B = math.sqrt(2.0 / math.pi), 0.044715


# ------------------------------------------------------------------ cases
def _linear(name, way, m, k, n, act, bias, res, dtype="bf16", pad=0):
    """way: "fwd", "train" (forward that keeps pre) or "bwd".  pad: elements between the end of a row and the next one."""
    return {"name": name, "op": "linear", "way": way, "m": m, "k": k, "n": n, "act": act, "bias": bias, "res": res, "dtype": dtype, "pad": pad}


def _gated(name, way, m, k, f, act, kept, dtype="bf16"):
    """way: "fwd" or "bwd".  kept: g and u are written by the forward pass and read by the backward pass."""
    return {"name": name, "op": "gated", "way": way, "m": m, "k": k, "f": f, "act": act, "kept": kept, "dtype": dtype}


def _distill(name, way, rows, classes, k, temperature, ragged, masked, dtype="bf16"):
    """way: "fwd" (loss, per-row losses, log-sum-exp), "bwd" (from these), "step" (loss and gradient together).
    ragged: rows with fewer than k teacher entries, some with none, and rows of weight 0; masked: columns of -inf at the end."""
    return {"name": name, "op": "distill", "way": way, "rows": rows, "classes": classes, "k": k, "temperature": temperature, "ragged": ragged,
            "masked": masked, "dtype": dtype}


def listed():
    return [
        # output projection of one token while answering: the weights are read once, latency counts
        _linear("linear_token", "fwd", 1, 4096, 4096, "none", True, True),
        # widening projection of a few requests answered together
        _linear("linear_requests", "fwd", 24, 2048, 8192, "gelu", True, False),
        # closing projection of a feed-forward block over a long batch of training tokens, with the residual sum
        _linear("linear_long", "fwd", 8192, 8192, 4096, "none", True, True),
        # its kind with an activation, backward: data, weight and bias gradient
        _linear("linear_long_bwd", "bwd", 8192, 4096, 4096, "gelu_tanh", True, False),
        # a short ragged batch through a small layer, backward, weight gradients in 32 bits
        _linear("linear_ragged_bwd", "bwd", 1003, 520, 776, "none", True, False, pad=8),
        # the 32-bit type that a program checks itself in
        _linear("linear_fp32", "train", 1000, 1024, 1000, "silu", True, True, dtype="fp32"),
        # gated block, one token
        _gated("gated_token", "fwd", 1, 4096, 8192, "silu", False),
        # gated block, training, forward and backward
        _gated("gated_long", "fwd", 8192, 4096, 8192, "silu", True),
        _gated("gated_long_bwd", "bwd", 8192, 4096, 8192, "silu", True),
        # a ragged batch of a small model that does not keep g and u
        _gated("gated_ragged_bwd", "bwd", 1531, 1032, 2056, "gelu", False),
        # loss and gradient over a large vocabulary, as a training step takes them
        _distill("distill_step", "step", 4096, 50304, 64, 2.0, True, False),
        # validation loss of a short text over an odd vocabulary, 32 bits
        _distill("distill_odd", "fwd", 301, 32003, 20, 1.0, True, True, dtype="fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths of layers: mostly multiples of 64, or of 8, now and then any number."""
    step = rng.choice((64, 64, 64, 8, 8, 1))
    return max(lo, _log_int(rng, lo, hi) // step * step)


def draw(rng):
    op = rng.choice(("linear", "gated", "distill"))
    while True:
        dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
        if op == "linear":
            few = rng.random() < 0.3                                # a few tokens being answered
            case = _linear("", "fwd" if few else rng.choice(("fwd", "train", "bwd", "bwd")), _log_int(rng, 1, 64) if few else _log_int(rng, 16, 16384),
                           _width(rng, 64, 8192), _width(rng, 64, 16384), rng.choice(ACTS), rng.random() < 0.6, rng.random() < 0.5, dtype,
                           rng.choice((0, 0, 0, 8, 3)))
        elif op == "gated":
            few = rng.random() < 0.3
            case = _gated("", "fwd" if few else rng.choice(("fwd", "bwd", "bwd")), _log_int(rng, 1, 64) if few else _log_int(rng, 16, 16384),
                          _width(rng, 64, 8192), _width(rng, 64, 16384), rng.choice(ACTS[1:]), not few and rng.random() < 0.6, dtype)
        else:
            classes = _log_int(rng, 100, 200000)
            case = _distill("", rng.choice(("fwd", "bwd", "step", "step")), _log_int(rng, 1, 8192), classes, min(classes // 2, _log_int(rng, 1, 256)),
                            rng.choice((1.0, 2.0, 0.7, 4.0)), rng.random() < 0.7, rng.random() < 0.3, dtype)
        w = work(case)
        if w["flops"] <= (MAX_FLOPS if dtype == "bf16" else MAX_FLOPS / 16) and w["bytes"] <= MAX_BYTES:
            del case["name"]
            return case


def _products(case):
    """Matrix products of m x k x (n or f) in one pass."""
    if case["op"] == "linear":
        return 2 if case["way"] == "bwd" else 1
    return 2 if case["way"] == "fwd" else 4 if case["kept"] else 6


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "distill":
        rows, classes, k = case["rows"], case["classes"], case["k"]
        passes = 1 if case["way"] == "fwd" else 2                   # the logits in, their gradient out
        return {"bytes": passes * rows * classes * e + rows * (8 * k + 12), "flops": (4 if case["way"] == "fwd" else 8) * rows * classes}
    m, k = case["m"], case["k"]
    n = case["n"] if case["op"] == "linear" else case["f"]
    flops = 2.0 * m * k * n * _products(case)
    if case["op"] == "linear":
        if case["way"] == "bwd":
            out = 4 if case["act"] == "none" else e
            size = 2 * m * k * e + m * n * e * (1 if case["act"] == "none" else 2) + k * n * (e + out) + 4 * n * case["bias"]
        else:
            size = m * k * e + k * n * e + 4 * n * case["bias"] + m * n * e * (1 + case["res"] + (case["way"] == "train"))
    elif case["way"] == "fwd":
        size = m * k * e + 2 * k * n * e + m * n * e * (3 if case["kept"] else 1)
    else:
        size = 2 * m * k * e + 4 * k * n * e + m * n * e * (3 if case["kept"] else 1)
    return {"bytes": int(size), "flops": int(flops)}


# ------------------------------------------------------------------ inputs
def _rows(gen, rows, cols, pad, dtype, scale=1.0):
    """A matrix whose rows lie cols + pad elements apart."""
    t = torch.randn(rows, cols + pad, generator=gen, device="cuda", dtype=torch.float32)
    return t.mul_(scale).to(dtype)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    st = dict(case)
    if case["op"] == "distill":
        rows, classes, k = case["rows"], case["classes"], case["k"]
        z = torch.randn(rows, classes, generator=gen, device="cuda").mul_(2.0)
        valid = classes - classes // 16 if case["masked"] else classes
        z[:, valid:] = -math.inf
        # one class of each of k runs of classes, so that no class comes twice; the teacher mostly agrees with the student
        run_ = valid // k
        ids = torch.arange(k, device="cuda")[None, :] * run_ + torch.randint(run_, (rows, k), generator=gen, device="cuda")
        t = z.gather(1, ids) + torch.randn(rows, k, generator=gen, device="cuda") + 1.0
        weight = torch.rand(rows, generator=gen, device="cuda") + 0.5
        if case["ragged"]:
            left = torch.randint(k + 1, (rows, 1), generator=gen, device="cuda")
            full = torch.rand(rows, 1, generator=gen, device="cuda") < 0.5
            ids = torch.where(full | (torch.arange(k, device="cuda")[None, :] < left), ids, torch.full_like(ids, -1))
            weight = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.2, torch.zeros_like(weight), weight)
        z = z.to(dtype)
        st.update(z=z, ids=ids.to(torch.int32).contiguous(), t=t.contiguous(), weight=weight, scale=1.0 / rows)
        if case["way"] == "bwd":
            # what the forward pass left
            st["lse"] = torch.cat([torch.logsumexp(c.double() / case["temperature"], 1) for c in z.split(512)]).float()
        return st
    m, k = case["m"], case["k"]
    if case["op"] == "linear":
        n, pad = case["n"], case["pad"]
        st["x"] = _rows(gen, m, k, pad, dtype)
        st["w"] = _rows(gen, k, n, 0, dtype, k ** -0.5)
        if case["way"] == "bwd":
            st["dy"] = _rows(gen, m, n, pad, dtype)
            st["pre"] = None if case["act"] == "none" else _rows(gen, m, n, pad, dtype)
        else:
            st["bias"] = torch.randn(n, generator=gen, device="cuda").mul_(0.5) if case["bias"] else None
            st["res"] = _rows(gen, m, n, pad, dtype) if case["res"] else None
        return st
    f = case["f"]
    st["x"] = _rows(gen, m, k, 0, dtype)
    st["wg"] = _rows(gen, k, f, 0, dtype, k ** -0.5)
    st["wu"] = _rows(gen, k, f, 0, dtype, k ** -0.5)
    if case["way"] == "bwd":
        st["dh"] = _rows(gen, m, f, 0, dtype)
        st["g"] = _rows(gen, m, f, 0, dtype) if case["kept"] else None
        st["u"] = _rows(gen, m, f, 0, dtype) if case["kept"] else None
    return st


# ------------------------------------------------------------------ plain form
def _act(name, v):
    if name == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * SQRT_HALF))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(TANH_A * (v + TANH_B * v * v * v)))
    return v


def _act_grad(name, v):
    if name == "relu":
        return (v > 0).to(v.dtype)
    if name == "silu":
        s = 1 / (1 + torch.exp(-v))
        return s * (1 + v * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(v * SQRT_HALF)) + v * torch.exp(-0.5 * v * v) * (1 / math.sqrt(2 * math.pi))
    if name == "gelu_tanh":
        th = torch.tanh(TANH_A * (v + TANH_B * v * v * v))
        return 0.5 * (1 + th) + 0.5 * v * (1 - th * th) * TANH_A * (1 + 3 * TANH_B * v * v)
    return torch.ones_like(v)


def _plain_linear(st):
    x, w, kind = st["x"].float(), st["w"].float(), st["x"].dtype
    if st["way"] == "bwd":
        dy = st["dy"].float()
        dz = dy if st["pre"] is None else dy * _act_grad(st["act"], st["pre"].float())
        out = {"dx": (dz @ w.T).to(kind), "dw": (x.T @ dz).to(torch.float32 if st["act"] == "none" else kind)}
        if st["bias"]:
            out["db"] = dz.sum(0, dtype=torch.float64).float()
        return out
    pre = x @ w
    if st["bias"] is not None:
        pre = pre + st["bias"]
    y = _act(st["act"], pre)
    if st["res"] is not None:
        y = y + st["res"].float()
    return {"y": y.to(kind), "pre": pre.to(kind)} if st["way"] == "train" else {"y": y.to(kind)}


def _plain_gated(st):
    x, wg, wu, kind = st["x"].float(), st["wg"].float(), st["wu"].float(), st["x"].dtype
    if st["way"] == "fwd":
        g, u = x @ wg, x @ wu
        h = (_act(st["act"], g) * u).to(kind)
        return {"h": h, "g": g.to(kind), "u": u.to(kind)} if st["kept"] else {"h": h}
    g, u = (st["g"].float(), st["u"].float()) if st["kept"] else (x @ wg, x @ wu)
    dh = st["dh"].float()
    dg, du = dh * u * _act_grad(st["act"], g), dh * _act(st["act"], g)
    return {"dx": (dg @ wg.T + du @ wu.T).to(kind), "dwg": (x.T @ dg).to(kind), "dwu": (x.T @ du).to(kind)}


def _plain_distill(st):
    temp, ids = st["temperature"], st["ids"].long()
    there = ids >= 0
    at = ids.clamp(min=0)
    t = torch.where(there, st["t"] / temp, torch.full_like(st["t"], -math.inf))
    some = there.any(1)
    top = torch.where(some, t.amax(1), torch.zeros_like(st["weight"]))[:, None]
    p = torch.where(there, torch.exp(t - top), torch.zeros_like(t))
    total = p.sum(1, keepdim=True)
    total = torch.where(total > 0, total, torch.ones_like(total))
    log_p = torch.where(there, t - top - torch.log(total), torch.zeros_like(t))
    p = p / total
    s = st["z"].float() / temp
    if st["way"] == "bwd":
        lse = st["lse"]
    else:
        high = s.amax(1)
        lse = high + torch.log(torch.exp(s - high[:, None]).sum(1))
        log_q = torch.where(there, s.gather(1, at) - lse[:, None], torch.zeros_like(t))
        row = temp * temp * (p * (log_p - log_q)).sum(1)
        loss = (st["scale"] * (st["weight"] * row).sum(dtype=torch.float64)).float().reshape(1)
        if st["way"] == "fwd":
            return {"loss": loss, "row_loss": row, "lse": lse}
    dz = torch.exp(s - lse[:, None]) * some[:, None]
    dz.scatter_add_(1, at, -p)
    dz = (dz * (st["scale"] * temp * st["weight"])[:, None]).to(st["z"].dtype)
    return {"dz": dz} if st["way"] == "bwd" else {"loss": loss, "dz": dz}


# ------------------------------------------------------------------ the framework's operators
def _like(t, rows, cols, dtype=None):
    """An output whose rows lie as far apart as those of t."""
    pad = t.stride(0) - t.shape[1] if t.shape[0] > 1 else 0
    return torch.empty(rows, cols + pad, dtype=dtype or t.dtype, device="cuda")[:, :cols]


def _ptr(t):
    return None if t is None else t.data_ptr()


def _own_buffers(st):
    """What a program sets up once: descriptor, outputs, workspace."""
    import paper_1807_02037_amd as L
    A = L.abi
    dt = A.BF16 if st["dtype"] == "bf16" else A.F32
    b = {"L": L}
    if st["op"] == "distill":
        z, rows = st["z"], st["rows"]
        b["desc"] = L.distill_desc(rows, st["classes"], st["k"], temperature=st["temperature"], scale=st["scale"], dtype=dt)
        which = {"fwd": A.DISTILL_FWD, "bwd": A.DISTILL_BWD, "step": A.DISTILL_LOSS_GRAD}[st["way"]]
        need = L.distill_workspace_bytes(b["desc"], which)
        if st["way"] != "bwd":
            b["loss"] = torch.empty(1, device="cuda")
        if st["way"] == "fwd":
            b["row_loss"], b["lse"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        else:
            b["dz"] = torch.empty_like(z)
    else:
        act = {"none": A.ACT_NONE, "relu": A.ACT_RELU, "silu": A.ACT_SILU, "gelu": A.ACT_GELU, "gelu_tanh": A.ACT_GELU_TANH}[st["act"]]
        m, k, x, kind = st["m"], st["k"], st["x"], st["x"].dtype
        if st["op"] == "linear":
            n, pad = st["n"], st["pad"]
            b["desc"] = L.linear_desc(m, n, k, act=act, dtype=dt, wgrad_dtype=A.F32 if st["act"] == "none" else dt, ldx=k + pad, ldy=n + pad, ldr=n + pad)
            need = L.linear_workspace_bytes(b["desc"], A.LINEAR_BWD if st["way"] == "bwd" else A.LINEAR_FWD)
            if st["way"] == "bwd":
                b["dx"] = torch.empty(m, k + pad, dtype=kind, device="cuda")[:, :k]
                b["dw"] = torch.empty(k, n, dtype=torch.float32 if st["act"] == "none" else kind, device="cuda")
                b["db"] = torch.empty(n, device="cuda") if st["bias"] else None
            else:
                b["y"] = torch.empty(m, n + pad, dtype=kind, device="cuda")[:, :n]
                b["pre"] = torch.empty(m, n + pad, dtype=kind, device="cuda")[:, :n] if st["way"] == "train" else None
        else:
            f = st["f"]
            b["desc"] = L.gated_desc(m, f, k, act=act, dtype=dt, wgrad_dtype=dt)
            need = L.gated_workspace_bytes(b["desc"], A.GATED_FWD if st["way"] == "fwd" else A.GATED_BWD if st["kept"] else A.GATED_BWD_RECOMPUTE)
            if st["way"] == "fwd":
                b["h"] = torch.empty(m, f, dtype=kind, device="cuda")
                b["g"] = torch.empty_like(b["h"]) if st["kept"] else None
                b["u"] = torch.empty_like(b["h"]) if st["kept"] else None
            else:
                b["dx"] = torch.empty(m, k, dtype=kind, device="cuda")
                b["dwg"], b["dwu"] = torch.empty(k, f, dtype=kind, device="cuda"), torch.empty(k, f, dtype=kind, device="cuda")
    b["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return b


def _own_run(st):
    b = st.get("buffers")
    if b is None:
        b = st["buffers"] = _own_buffers(st)
    L, d, ws, stream = b["L"], b["desc"], b["ws"].data_ptr(), torch.cuda.current_stream().cuda_stream
    if st["op"] == "linear":
        if st["way"] == "bwd":
            L.linear_bwd(d, _ptr(st["dy"]), _ptr(st["x"]), _ptr(st["w"]), _ptr(st["pre"]), _ptr(b["dx"]), _ptr(b["dw"]), _ptr(b["db"]), ws, stream)
            return {"dx": b["dx"], "dw": b["dw"], "db": b["db"]} if st["bias"] else {"dx": b["dx"], "dw": b["dw"]}
        L.linear_fwd(d, _ptr(st["x"]), _ptr(st["w"]), _ptr(st["bias"]), _ptr(st["res"]), _ptr(b["y"]), _ptr(b["pre"]), ws, stream)
        return {"y": b["y"], "pre": b["pre"]} if st["way"] == "train" else {"y": b["y"]}
    if st["op"] == "gated":
        if st["way"] == "fwd":
            L.gated_fwd(d, _ptr(st["x"]), _ptr(st["wg"]), _ptr(st["wu"]), _ptr(b["h"]), _ptr(b["g"]), _ptr(b["u"]), ws, stream)
            return {"h": b["h"], "g": b["g"], "u": b["u"]} if st["kept"] else {"h": b["h"]}
        L.gated_bwd(d, _ptr(st["dh"]), _ptr(st["x"]), _ptr(st["wg"]), _ptr(st["wu"]), _ptr(st["g"]), _ptr(st["u"]), _ptr(b["dx"]), _ptr(b["dwg"]),
                    _ptr(b["dwu"]), ws, stream)
        return {"dx": b["dx"], "dwg": b["dwg"], "dwu": b["dwu"]}
    z, t, ids, weight = (_ptr(st[n]) for n in ("z", "t", "ids", "weight"))
    if st["way"] == "fwd":
        L.distill_fwd(d, z, t, ids, weight, _ptr(b["loss"]), _ptr(b["row_loss"]), _ptr(b["lse"]), ws, stream)
        return {"loss": b["loss"], "row_loss": b["row_loss"], "lse": b["lse"]}
    if st["way"] == "bwd":
        L.distill_bwd(d, z, t, ids, weight, _ptr(st["lse"]), _ptr(b["dz"]), ws, stream)
        return {"dz": b["dz"]}
    L.distill_loss_grad(d, z, t, ids, weight, _ptr(b["loss"]), _ptr(b["dz"]), ws, stream)
    return {"loss": b["loss"], "dz": b["dz"]}


def run(state):
    if own:
        return _own_run(state)
    return {"linear": _plain_linear, "gated": _plain_gated, "distill": _plain_distill}[state["op"]](state)


# ------------------------------------------------------------------ in 64 bits, from the definitions
def _exact_act(name, v):
    """(act(v), act'(v))"""
    if name == "none":
        return v, torch.ones_like(v)
    if name == "relu":
        return v.clamp(min=0), torch.where(v > 0, 1.0, 0.0).double()
    if name == "silu":
        s = torch.sigmoid(v)
        return v * s, s + v * s * torch.sigmoid(-v)
    if name == "gelu":
        cdf = torch.special.ndtr(v)
        return v * cdf, cdf + v * torch.exp(-v.square() / 2) / math.sqrt(2 * math.pi)
    inner = math.sqrt(2 / math.pi) * (v + 0.044715 * v.pow(3))
    s = torch.sigmoid(2 * inner)                                    # (1 + tanh(inner)) / 2
    return v * s, s + 2 * v * s * torch.sigmoid(-2 * inner) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v.square())


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["op"]
    if kind == "linear":
        x, w = st["x"].double(), st["w"].double()
        if case["way"] == "bwd":
            dz = st["dy"].double()
            if case["act"] != "none":
                dz = dz * _exact_act(case["act"], st["pre"].double())[1]
            out = {"dx": torch.mm(dz, w.t()), "dw": torch.mm(x.t(), dz)}
            if case["bias"]:
                out["db"] = dz.sum(dim=0)
            return out
        pre = torch.mm(x, w)
        if st["bias"] is not None:
            pre += st["bias"].double()
        y = _exact_act(case["act"], pre)[0]
        if st["res"] is not None:
            y = y + st["res"].double()
        return {"y": y, "pre": pre} if case["way"] == "train" else {"y": y}
    if kind == "gated":
        x, wg, wu = st["x"].double(), st["wg"].double(), st["wu"].double()
        g, u = (st["g"].double(), st["u"].double()) if case["way"] == "bwd" and case["kept"] else (torch.mm(x, wg), torch.mm(x, wu))
        a, slope = _exact_act(case["act"], g)
        if case["way"] == "fwd":
            return {"h": a * u, "g": g, "u": u} if case["kept"] else {"h": a * u}
        dh = st["dh"].double()
        dg, du = dh * slope * u, dh * a
        return {"dx": torch.mm(dg, wg.t()) + torch.mm(du, wu.t()), "dwg": torch.mm(x.t(), dg), "dwu": torch.mm(x.t(), du)}
    temp, scale, rows, losses, stats, grads = case["temperature"], st["scale"], case["rows"], [], [], []
    for r in range(0, rows, 1024):
        ids = st["ids"][r:r + 1024].long()
        none = ids < 0
        teacher = (st["t"][r:r + 1024].double() / temp).masked_fill(none, -math.inf)
        logp = torch.log_softmax(teacher, dim=1).masked_fill(none, 0.0)
        p = torch.softmax(teacher, dim=1).masked_fill(none, 0.0)    # rows without an entry: all masked
        z = st["z"][r:r + 1024].double() / temp
        lse = torch.logsumexp(z, dim=1, keepdim=True)
        cross = z.gather(1, ids.clamp_min(0)).masked_fill(none, 0.0)
        has = (~none).any(dim=1)
        losses.append(temp ** 2 * ((p * (logp - cross)).sum(dim=1) + lse[:, 0] * has))
        stats.append(lse[:, 0])
        if case["way"] != "fwd":
            target = torch.zeros_like(z).scatter_add_(1, ids.clamp_min(0), p)
            grads.append((scale * temp * st["weight"][r:r + 1024].double() * has)[:, None] * (torch.softmax(z, dim=1) - target))
    row = torch.cat(losses)
    loss = (scale * torch.dot(st["weight"].double(), row)).reshape(1)
    if case["way"] == "fwd":
        return {"loss": loss, "row_loss": row, "lse": torch.cat(stats)}
    return {"dz": torch.cat(grads)} if case["way"] == "bwd" else {"loss": loss, "dz": torch.cat(grads)}
