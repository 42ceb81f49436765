"""Timed operators of a student that reads sequences and answers: the gated recurrence, group normalisation with an activation,
the linear layer in 8-bit integers and the verification of drafted tokens.

`run` computes them in plain torch operations, or, with `own` set, through the framework's entry points.

  recur     a = sigmoid(g); h_t = a_t h_{t-1} + (1 - a_t) x_t within a sequence, from its initial state h0; y_t = h_t act(o_t), or h_t;
            backward, from dy and the gradient `dlast` of the last states: dh_t = dy_t act(o_t) + a_{t+1} dh_{t+1},
            dx = (1 - a) dh, dg = dh (h_{t-1} - x) a (1 - a), do = dy h act'(o), dh0 = a dh of the first position
  norm      over a sample's positions and a group's channels: xhat = (x - mean) / sqrt(variance + eps), y = act(gamma xhat + beta);
            backward: dv = dy act'(gamma xhat + beta), dgamma = sum dv xhat, dbeta = sum dv,
            dx = (gamma dv - mean(gamma dv) - xhat mean(gamma dv xhat)) / sqrt(variance + eps)
  q8        xq = rint(127 x / max |row of x|), ties to even, sx = max |row| / 127; weights wq, sw alike, by column, quantised before;
            y = act((xq wq) sx sw + bias) + r
  verify    a request's drafted tokens t_i are accepted while u_i q_i(t_i) < p_i(t_i); the next token is drawn from max(p_i - q_i, 0)
            at the first that is not (from p_i where that is nowhere above 0), from p behind the last draft where all are:
            the first class whose running sum is above v times the whole"""
import math

import torch

own = False

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
MAX_FLOPS = 5.6e11
MAX_BYTES = 1.9e9
EPS = 1e-5


# ------------------------------------------------------------------ cases
def _recur(name, way, rows, channels, seqs, packed, act, dtype="bf16", pad=0):
    """way: "fwd" (as a training step takes it: it leaves what the backward pass needs), "bwd", "step" (one token of each request, states in slots).
    packed: sequences of different lengths one after the other, some empty, with rows behind the last; else of one length.  act: of the output gate, None: no gate."""
    return {"name": name, "op": "recur", "way": way, "rows": rows, "channels": channels, "seqs": seqs, "packed": packed, "act": act, "dtype": dtype, "pad": pad}


def _norm(name, way, samples, positions, channels, groups, act, affine, dtype="bf16", pad=0):
    """way: "fwd" (leaves mean and 1 / deviation) or "bwd".  affine: gamma and beta, and their gradients."""
    return {"name": name, "op": "norm", "way": way, "samples": samples, "positions": positions, "channels": channels, "groups": groups, "act": act,
            "affine": affine, "dtype": dtype, "pad": pad}


def _q8(name, m, k, n, act, bias, res, dtype="bf16", pad=0):
    return {"name": name, "op": "q8", "way": "fwd", "m": m, "k": k, "n": n, "act": act, "bias": bias, "res": res, "dtype": dtype, "pad": pad}


def _verify(name, requests, drafts, classes, ragged):
    """ragged: requests with fewer drafts than `drafts`, some with none."""
    return {"name": name, "op": "verify", "way": "fwd", "requests": requests, "drafts": drafts, "classes": classes, "ragged": ragged, "dtype": "fp32"}


def listed():
    return [
        # the next token of a few dozen requests, states in a pool of slots: latency counts
        _recur("recur_step", "step", 48, 4096, 64, False, "silu"),
        # a training batch of long sequences, forward and backward
        _recur("recur_long", "fwd", 32768, 4096, 8, False, "silu"),
        _recur("recur_long_bwd", "bwd", 32768, 4096, 8, False, "silu"),
        # packed sequences of a small model, odd sizes, in the 32-bit type that a program checks itself in
        _recur("recur_packed_bwd", "bwd", 5003, 1033, 37, True, None, dtype="fp32", pad=3),
        # tokens of a training batch, each normalised over groups of its channels
        _norm("norm_tokens_bwd", "bwd", 8192, 1, 4096, 32, "none", True),
        # first level of a volume network, one sample
        _norm("norm_volume", "fwd", 1, 128 * 128 * 128, 64, 8, "relu", True),
        # late level of an image network, a batch, backward
        _norm("norm_image_bwd", "bwd", 64, 14 * 14, 1024, 32, "silu", True),
        # output projection of one token while answering
        _q8("q8_token", 1, 4096, 4096, "none", True, True),
        # widening projection of a few requests answered together
        _q8("q8_requests", 24, 2048, 8192, "gelu", True, False),
        # a long prompt through a closing projection, with the residual sum
        _q8("q8_long", 8192, 8192, 4096, "none", True, True),
        # one request's drafts over an odd vocabulary
        _verify("verify_one", 1, 4, 32003, False),
        # a batch of requests with fewer and more drafts
        _verify("verify_batch", 128, 5, 50304, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths of layers: mostly multiples of 64, or of 8, now and then any number."""
    step = rng.choice((64, 64, 64, 8, 8, 1))
    return max(lo, _log_int(rng, lo, hi) // step * step)


def draw(rng):
    op = rng.choice(("recur", "recur", "norm", "norm", "q8", "verify"))
    while True:
        dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
        if op == "recur":
            way = rng.choice(("fwd", "bwd", "bwd", "step"))
            act = rng.choice((None, "none", "silu", "silu", "gelu", "relu", "gelu_tanh"))
            channels, pad = _width(rng, 16, 8192), rng.choice((0, 0, 0, 8, 3))
            if way == "step":
                rows = _log_int(rng, 1, 512)
                case = _recur("", way, rows, channels, rows + rng.randrange(0, 64), False, act, dtype, pad)
            elif rng.random() < 0.5:
                case = _recur("", way, _log_int(rng, 8, 65536), channels, _log_int(rng, 1, 512), True, act, dtype, pad)
            else:
                seqs, length = _log_int(rng, 1, 64), _log_int(rng, 1, 32768)
                case = _recur("", way, seqs * length, channels, seqs, False, act, dtype, pad)
        elif op == "norm":
            way, act, affine, pad = rng.choice(("fwd", "bwd", "bwd")), rng.choice(ACTS), rng.random() < 0.8, rng.choice((0, 0, 0, 8, 3))
            groups = rng.choice((1, 2, 4, 8, 16, 32))
            if rng.random() < 0.4:                                  # tokens
                case = _norm("", way, _log_int(rng, 1, 32768), 1, groups * max(1, _width(rng, 64, 8192) // groups), groups, act, affine, dtype, pad)
            else:                                                   # images and volumes
                case = _norm("", way, _log_int(rng, 1, 128), _log_int(rng, 4, 300000), groups * max(1, _width(rng, 16, 2048) // groups), groups, act, affine, dtype, pad)
        elif op == "q8":
            few = rng.random() < 0.5                                # a few tokens being answered
            case = _q8("", _log_int(rng, 1, 64) if few else _log_int(rng, 16, 16384), _width(rng, 64, 8192), _width(rng, 64, 16384), rng.choice(ACTS),
                       rng.random() < 0.6, rng.random() < 0.5, dtype, rng.choice((0, 0, 0, 8, 3)))
        else:
            case = _verify("", _log_int(rng, 1, 256), rng.randrange(1, 9), _log_int(rng, 100, 130000), rng.random() < 0.7)
            if case["requests"] * (case["drafts"] + 1) * case["classes"] > 1.5e8:
                continue
        w = work(case)
        if w["flops"] <= (MAX_FLOPS if dtype == "bf16" else MAX_FLOPS / 4) and w["bytes"] <= MAX_BYTES:
            del case["name"]
            return case


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "recur":
        n = case["rows"] * case["channels"]
        gate = case["act"] is not None
        if case["way"] == "step":
            return {"bytes": n * (e * (3 + gate) + 8) + 4 * case["rows"], "flops": 20 * n}
        states = 8 * case["seqs"] * case["channels"]
        if case["way"] == "fwd":
            return {"bytes": n * e * (3 + gate) + states, "flops": 20 * n}
        return {"bytes": n * e * (5 + 2 * gate) + states + states // 2, "flops": 40 * n}
    if case["op"] == "norm":
        n = case["samples"] * case["positions"] * case["channels"]
        stats, par = 8 * case["samples"] * case["groups"], 8 * case["channels"] * case["affine"]
        return {"bytes": n * e * (2 if case["way"] == "fwd" else 3) + stats + par * (1 if case["way"] == "fwd" else 2), "flops": (10 if case["way"] == "fwd" else 25) * n}
    if case["op"] == "q8":
        m, k, n = case["m"], case["k"], case["n"]
        return {"bytes": m * k * e + k * n + 4 * n * (1 + case["bias"]) + m * n * e * (1 + case["res"]), "flops": 2 * m * k * n}
    b, d, c = case["requests"], case["drafts"], case["classes"]
    return {"bytes": b * (8 * c + 16 * d + 4 * d + 16), "flops": 4 * b * c}


# ------------------------------------------------------------------ inputs
def _rows(gen, rows, cols, pad, dtype, scale=1.0):
    """A matrix whose rows lie cols + pad elements apart."""
    t = torch.randn(rows, cols + pad, generator=gen, device="cuda", dtype=torch.float32)
    return t.mul_(scale).to(dtype)[:, :cols]


def _offsets(rows, seqs, gen):
    """Borders of sequences of different lengths: some empty, and a few rows behind the last."""
    used = rows - rows // 50
    cuts = torch.randint(used + 1, (seqs - 1,), generator=gen, device="cuda")
    cuts = torch.where(torch.rand(seqs - 1, generator=gen, device="cuda") < 0.1, cuts.roll(1), cuts)       # the same border twice: an empty sequence
    ends = torch.tensor([0, used], device="cuda")
    return torch.cat([ends[:1], cuts.sort().values, ends[1:]]).to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    st = dict(case)
    if case["op"] == "recur":
        rows, c, pad = case["rows"], case["channels"], case["pad"]
        st["x"] = _rows(gen, rows, c, pad, dtype)
        st["g"] = _rows(gen, rows, c, pad, dtype).add_(2.0)         # gates near 0.9: a state is remembered for some ten positions, in some channels for hundreds
        st["o"] = None if case["act"] is None else _rows(gen, rows, c, pad, dtype)
        if case["way"] == "step":
            st["slots"] = torch.randperm(case["seqs"], generator=gen, device="cuda")[:rows].to(torch.int32).contiguous()
            st["state"] = torch.randn(case["seqs"], c, generator=gen, device="cuda").mul_(0.3)
            st["next"] = st["state"].clone()
            return _ready(st)
        st["offsets"] = _offsets(rows, case["seqs"], gen) if case["packed"] else None
        st["h0"] = torch.randn(case["seqs"], c, generator=gen, device="cuda").mul_(0.3)
        if case["way"] == "bwd":
            st["dy"] = _rows(gen, rows, c, pad, dtype)
            st["dlast"] = torch.randn(case["seqs"], c, generator=gen, device="cuda")
        return _ready(st)
    if case["op"] == "norm":
        rows, c, pad = case["samples"] * case["positions"], case["channels"], case["pad"]
        shift = torch.randn(c, generator=gen, device="cuda")
        x = torch.randn(rows, c + pad, generator=gen, device="cuda")
        x[:, :c].add_(shift)
        st["x"] = x.to(dtype)[:, :c]
        del x
        st["gamma"] = torch.randn(c, generator=gen, device="cuda").mul_(0.2).add_(1.0) if case["affine"] else None
        st["beta"] = torch.randn(c, generator=gen, device="cuda").mul_(0.2) if case["affine"] else None
        if case["way"] == "bwd":
            st["dy"] = _rows(gen, rows, c, pad, dtype)
            # what the forward pass left
            st["mean"], st["rstd"] = _norm_stats(st)
        return _ready(st)
    if case["op"] == "q8":
        m, k, n, pad = case["m"], case["k"], case["n"], case["pad"]
        st["x"] = _rows(gen, m, k, pad, dtype)
        st["w"] = _rows(gen, k, n, 0, dtype, k ** -0.5)
        # the quantised weights that a program keeps
        st["wq"], st["sw"] = _quantise(st["w"].T)
        st["wq"] = st["wq"].T.to(torch.int8).contiguous()
        st["bias"] = torch.randn(n, generator=gen, device="cuda").mul_(0.5) if case["bias"] else None
        st["res"] = _rows(gen, m, n, pad, dtype) if case["res"] else None
        return _ready(st)
    b, d, c = case["requests"], case["drafts"], case["classes"]
    # a student that mostly agrees with its teacher, logits of a spread as of trained models
    z = torch.randn(b, d + 1, c, generator=gen, device="cuda").mul_(3.0)
    st["p"] = torch.softmax(z, dim=2)
    z = z[:, :d] + torch.randn(b, d, c, generator=gen, device="cuda").mul_(0.7)
    st["q"] = torch.softmax(z, dim=2)
    # tokens drawn from the student's distribution: the largest of z - log(-log(u))
    noise = torch.rand(b, d, c, generator=gen, device="cuda").clamp_(1e-7, 1 - 1e-7)
    st["drafted"] = (z - torch.log(-torch.log(noise))).argmax(2).to(torch.int32).contiguous()
    st["counts"] = torch.randint(d + 1, (b,), generator=gen, device="cuda").to(torch.int32) if case["ragged"] else None
    st["u"] = torch.rand(b, d, generator=gen, device="cuda")
    st["v"] = torch.rand(b, generator=gen, device="cuda")
    return _ready(st)


def _norm_stats(st):
    """Mean and 1 / deviation of each sample's groups."""
    n, s, c, g = st["samples"], st["positions"], st["channels"], st["groups"]
    mean, rstd = [], []
    for x in st["x"].split(max(1, (1 << 25) // (s * c)) * s):
        v = x.reshape(-1, s, g, c // g).double()
        var, m = torch.var_mean(v, dim=(1, 3), correction=0)
        mean.append(m.float())
        rstd.append((1.0 / torch.sqrt(var + EPS)).float())
    return torch.cat(mean), torch.cat(rstd)


# ------------------------------------------------------------------ plain form
def _act(name, v):
    if name == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if name == "silu":
        return v / (1 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    return v


def _slope(name, v):
    if name == "relu":
        return (v > 0).to(v.dtype)
    if name == "silu":
        s = 1 / (1 + torch.exp(-v))
        return s * (1 + v * (1 - s))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1 / math.sqrt(2 * math.pi))
    if name == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (v + 0.044715 * v * v * v))
        return 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * a * (1 + 3 * 0.044715 * v * v)
    return torch.ones_like(v)


def _running(a, b):
    """h_t = a_t h_{t-1} + b_t over the rows, by doubling the distance; a is 0 where a sequence begins."""
    reach = 1
    while reach < a.shape[0]:
        b = torch.cat([b[:reach], torch.addcmul(b[reach:], a[reach:], b[:-reach])])
        a = torch.cat([a[:reach], a[reach:] * a[:-reach]])
        reach *= 2
    return b


def _layout(st):
    """Rows in use, the first row of each sequence that has one, and that sequence."""
    rows, seqs = st["rows"], st["seqs"]
    if st["offsets"] is None:
        each = rows // seqs
        return rows, torch.arange(seqs, device="cuda") * each, torch.arange(seqs, device="cuda") * each + each - 1, torch.arange(seqs, device="cuda")
    off = st["offsets"].long()
    full = (off[1:] > off[:-1]).nonzero().flatten()
    return rows - rows // 50, off[:-1][full], off[1:][full] - 1, full


def _plain_recur(st):
    kind, act = st["x"].dtype, st["act"]
    if st["way"] == "step":
        at = st["slots"].long()
        a = 1 / (1 + torch.exp(-st["g"].float()))
        h = a * st["state"][at] + (1 - a) * st["x"].float()
        y = h if act is None else h * _act(act, st["o"].float())
        new = st["state"].clone()
        new[at] = h
        return {"y": y.to(kind), "state": new}
    used, first, last, seq = _layout(st)
    x, g = st["x"][:used].float(), st["g"][:used].float()
    o = None if act is None else st["o"][:used].float()
    a, rest = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    b = rest * x
    b[first] += a[first] * st["h0"][seq]
    cut = a.clone()
    cut[first] = 0
    h = _running(cut, b)
    if st["way"] == "fwd":
        out = h if o is None else h * _act(act, o)
        states = st["h0"].clone()
        states[seq] = h[last]
        return {"y": out.to(kind), "last": states}
    dy = st["dy"][:used].float()
    e = dy if o is None else dy * _act(act, o)
    e = e.clone()
    e[last] += st["dlast"][seq]
    # backwards in time: dh_t = e_t + a_{t+1} dh_{t+1}
    step = torch.cat([cut[1:], torch.zeros_like(cut[:1])]).flip(0)
    dh = _running(step, e.flip(0)).flip(0)
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[first] = st["h0"][seq]
    dh0 = st["dlast"].clone()
    dh0[seq] = a[first] * dh[first]
    out = {"dx": (rest * dh).to(kind), "dg": (dh * (before - x) * a * rest).to(kind), "dh0": dh0}
    if o is not None:
        out["do"] = (dy * h * _slope(act, o)).to(kind)
    return out


def _plain_norm(st):
    n, s, c, g, kind = st["samples"], st["positions"], st["channels"], st["groups"], st["x"].dtype
    x = st["x"].float().reshape(n, s, g, c // g)
    gamma = 1.0 if st["gamma"] is None else st["gamma"].reshape(g, c // g)
    beta = 0.0 if st["beta"] is None else st["beta"].reshape(g, c // g)
    if st["way"] == "fwd":
        mean = x.mean(dim=(1, 3), keepdim=True)
        d = x - mean
        rstd = 1 / torch.sqrt((d * d).mean(dim=(1, 3), keepdim=True) + EPS)
        y = _act(st["act"], d * rstd * gamma + beta)
        return {"y": y.reshape(n * s, c).to(kind), "mean": mean.reshape(n, g), "rstd": rstd.reshape(n, g)}
    rstd = st["rstd"].reshape(n, 1, g, 1)
    hat = (x - st["mean"].reshape(n, 1, g, 1)) * rstd
    dv = st["dy"].float().reshape(n, s, g, c // g)
    if st["act"] != "none":
        dv = dv * _slope(st["act"], hat * gamma + beta)
    u = dv * gamma
    dx = rstd * (u - u.mean(dim=(1, 3), keepdim=True) - hat * (u * hat).mean(dim=(1, 3), keepdim=True))
    out = {"dx": dx.reshape(n * s, c).to(kind)}
    if st["affine"]:
        out["dgamma"] = (dv * hat).sum(dim=(0, 1), dtype=torch.float64).float().reshape(c)
        out["dbeta"] = dv.sum(dim=(0, 1), dtype=torch.float64).float().reshape(c)
    return out


def _quantise(x):
    """Rows as whole numbers from -127 to 127, and what one of them stands for.  In 64 bits: a value half way between two goes to the even one."""
    most = x.abs().amax(1, keepdim=True).double()
    q = torch.round(x.double() * 127 / torch.where(most > 0, most, torch.ones_like(most)))
    return q, (most / 127).float()[:, 0]


def _plain_q8(st):
    xq, sx = _quantise(st["x"])
    y = (xq.float() @ st["wq"].float()) * sx[:, None] * st["sw"]
    if st["bias"] is not None:
        y = y + st["bias"]
    y = _act(st["act"], y)
    if st["res"] is not None:
        y = y + st["res"].float()
    return {"y": y.to(st["x"].dtype)}


def _plain_verify(st):
    b, d, c = st["requests"], st["drafts"], st["classes"]
    t = st["drafted"].long()[:, :, None]
    counts = torch.full((b,), d, device="cuda") if st["counts"] is None else st["counts"].long()
    at = torch.arange(d, device="cuda")[None, :]
    good = st["u"].double() * st["q"].gather(2, t)[:, :, 0].double() < st["p"][:, :d].gather(2, t)[:, :, 0].double()
    accepted = (good & (at < counts[:, None])).long().cumprod(1).sum(1)
    rows = torch.arange(b, device="cuda")
    p = st["p"][rows, accepted].double()
    q = torch.where((accepted < counts)[:, None], st["q"][rows, accepted.clamp(max=d - 1)].double(), torch.zeros_like(p))
    r = torch.clamp(p - q, min=0)
    r = torch.where(r.sum(1, keepdim=True) > 0, r, p)
    run_ = r.cumsum(1)
    token = (run_ > st["v"].double()[:, None] * run_[:, -1:]).long().argmax(1)
    tokens = torch.where(at < accepted[:, None], t[:, :, 0], torch.full_like(t[:, :, 0], -1))
    tokens = torch.cat([tokens, torch.full_like(tokens[:, :1], -1)], dim=1).scatter(1, accepted[:, None], token[:, None])
    return {"accepted": accepted.to(torch.int32), "tokens": tokens.to(torch.int32)}


# ------------------------------------------------------------------ the framework's operators
def _ptr(t):
    return None if t is None else t.data_ptr()


def _ready(st):
    if own:
        st["buffers"] = _own_buffers(st)
    return st


def _own_buffers(st):
    """What a program sets up once: descriptor, outputs, workspace, quantised weights, and for a backward pass what the forward pass kept."""
    import paper_1807_02037_amd as L
    A = L.abi
    dt = A.BF16 if st["dtype"] == "bf16" else A.F32
    acts = {None: A.ACT_NONE, "none": A.ACT_NONE, "relu": A.ACT_RELU, "silu": A.ACT_SILU, "gelu": A.ACT_GELU, "gelu_tanh": A.ACT_GELU_TANH}
    b = {"L": L}
    stream = torch.cuda.current_stream().cuda_stream

    def space(need):
        return torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    if st["op"] == "recur":
        rows, c, pad, seqs, kind = st["rows"], st["channels"], st["pad"], st["seqs"], st["x"].dtype

        def out():
            return torch.empty(rows, c + pad, dtype=kind, device="cuda")[:, :c]
        b["desc"] = d = L.recur_desc(rows, c, seqs, act=acts[st["act"]], dtype=dt, ldx=c + pad, ldy=c + pad)
        if st["way"] == "step":
            b["y"] = out()
            return b
        b["kept"] = space(L.recur_kept_bytes(d))
        b["ws"] = space(max(L.recur_workspace_bytes(d, A.RECUR_FWD), L.recur_workspace_bytes(d, A.RECUR_BWD)))
        b["y"], b["last"] = out(), torch.empty(seqs, c, device="cuda")
        if st["way"] == "bwd":
            L.recur_fwd(d, _ptr(st["x"]), _ptr(st["g"]), _ptr(st["o"]), _ptr(st["offsets"]), _ptr(st["h0"]), _ptr(b["y"]), _ptr(b["last"]), _ptr(b["kept"]),
                        _ptr(b["ws"]), stream)
            b["y"] = None
            b["dx"], b["dg"], b["do"], b["dh0"] = out(), out(), None if st["o"] is None else out(), torch.empty(seqs, c, device="cuda")
        return b
    if st["op"] == "norm":
        n, s, c, g, pad = st["samples"], st["positions"], st["channels"], st["groups"], st["pad"]
        b["desc"] = d = L.group_norm_desc(n, s, c, g, act=acts[st["act"]], dtype=dt, eps=EPS, ldx=c + pad, ldy=c + pad)
        b["ws"] = space(L.group_norm_workspace_bytes(d, A.GROUP_NORM_FWD if st["way"] == "fwd" else A.GROUP_NORM_BWD))
        b["out"] = torch.empty(n * s, c + pad, dtype=st["x"].dtype, device="cuda")[:, :c]
        if st["way"] == "fwd":
            b["mean"], b["rstd"] = torch.empty(n, g, device="cuda"), torch.empty(n, g, device="cuda")
        else:
            b["dgamma"], b["dbeta"] = (torch.empty(c, device="cuda"), torch.empty(c, device="cuda")) if st["affine"] else (None, None)
        return b
    if st["op"] == "q8":
        m, k, n, pad = st["m"], st["k"], st["n"], st["pad"]
        b["desc"] = d = L.linear_q8_desc(m, n, k, act=acts[st["act"]], dtype=dt, ldx=k + pad, ldy=n + pad, ldr=n + pad)
        b["wq"], b["sw"] = space(L.linear_q8_weight_bytes(d)), torch.empty(n, device="cuda")
        L.linear_q8_weight(d, _ptr(st["w"]), _ptr(b["wq"]), _ptr(b["sw"]), stream)
        b["ws"] = space(L.linear_q8_workspace_bytes(d))
        b["y"] = torch.empty(m, n + pad, dtype=st["x"].dtype, device="cuda")[:, :n]
        return b
    b["desc"] = d = L.verify_desc(st["requests"], st["drafts"], st["classes"])
    b["ws"] = space(L.verify_workspace_bytes(d))
    b["accepted"] = torch.empty(st["requests"], dtype=torch.int32, device="cuda")
    b["tokens"] = torch.empty(st["requests"], st["drafts"] + 1, dtype=torch.int32, device="cuda")
    return b


def _own_run(st):
    b = st.get("buffers")
    if b is None:
        b = st["buffers"] = _own_buffers(st)
    L, d, ws, stream = b["L"], b["desc"], _ptr(b.get("ws")), torch.cuda.current_stream().cuda_stream
    if st["op"] == "recur":
        x, g, o = _ptr(st["x"]), _ptr(st["g"]), _ptr(st["o"])
        if st["way"] == "step":
            # the old states stay, for drafts that may be taken back
            L.recur_step(d, x, g, o, _ptr(st["slots"]), _ptr(st["state"]), _ptr(st["next"]), _ptr(b["y"]), stream)
            return {"y": b["y"], "state": st["next"]}
        off, h0, kept = _ptr(st["offsets"]), _ptr(st["h0"]), _ptr(b["kept"])
        used = st["rows"] if st["offsets"] is None else st["rows"] - st["rows"] // 50
        if st["way"] == "fwd":
            L.recur_fwd(d, x, g, o, off, h0, _ptr(b["y"]), _ptr(b["last"]), kept, ws, stream)
            return {"y": b["y"][:used], "last": b["last"]}
        L.recur_bwd(d, _ptr(st["dy"]), x, g, o, off, h0, kept, _ptr(st["dlast"]), _ptr(b["dx"]), _ptr(b["dg"]), _ptr(b["do"]), _ptr(b["dh0"]), ws, stream)
        out = {"dx": b["dx"][:used], "dg": b["dg"][:used], "dh0": b["dh0"]}
        if st["o"] is not None:
            out["do"] = b["do"][:used]
        return out
    if st["op"] == "norm":
        x, gamma, beta = _ptr(st["x"]), _ptr(st["gamma"]), _ptr(st["beta"])
        if st["way"] == "fwd":
            L.group_norm_fwd(d, x, gamma, beta, _ptr(b["out"]), _ptr(b["mean"]), _ptr(b["rstd"]), ws, stream)
            return {"y": b["out"], "mean": b["mean"], "rstd": b["rstd"]}
        L.group_norm_bwd(d, _ptr(st["dy"]), x, gamma, beta, _ptr(st["mean"]), _ptr(st["rstd"]), _ptr(b["out"]), _ptr(b["dgamma"]), _ptr(b["dbeta"]), ws, stream)
        return {"dx": b["out"], "dgamma": b["dgamma"], "dbeta": b["dbeta"]} if st["affine"] else {"dx": b["out"]}
    if st["op"] == "q8":
        L.linear_q8_fwd(d, _ptr(st["x"]), _ptr(b["wq"]), _ptr(b["sw"]), _ptr(st["bias"]), _ptr(st["res"]), _ptr(b["y"]), ws, stream)
        return {"y": b["y"]}
    L.verify(d, _ptr(st["p"]), _ptr(st["q"]), _ptr(st["drafted"]), _ptr(st["counts"]), _ptr(st["u"]), _ptr(st["v"]), _ptr(b["accepted"]), _ptr(b["tokens"]), ws,
             stream)
    return {"accepted": b["accepted"], "tokens": b["tokens"]}


def run(st):
    if own:
        return _own_run(st)
    return {"recur": _plain_recur, "norm": _plain_norm, "q8": _plain_q8, "verify": _plain_verify}[st["op"]](st)


# ------------------------------------------------------------------ from the definition, in 64 bits
def exact(case, seed):
    """The outputs of `run`, the recurrence position by position, everything else with torch's own operators in 64 bits."""
    if case["op"] == "verify":
        return None                                                 # whole numbers
    st = prepare(case, seed)
    F = torch.nn.functional
    acts = {None: torch.ones_like, "none": lambda v: v, "relu": torch.relu, "silu": F.silu, "gelu": F.gelu, "gelu_tanh": lambda v: F.gelu(v, approximate="tanh")}
    if case["op"] == "recur":
        return _exact_recur(st, acts[case["act"]])
    if case["op"] == "q8":
        x = st["x"].double()
        top = x.abs().amax(dim=1)
        xq = torch.round(x * 127 / top.clamp_min(1e-300)[:, None])
        y = torch.mm(xq, st["wq"].double()) * (top / 127)[:, None] * (st["w"].double().abs().amax(dim=0) / 127)
        y = acts[case["act"]](y if st["bias"] is None else y + st["bias"].double())
        return {"y": y if st["res"] is None else y + st["res"].double()}
    n, s, c, g = case["samples"], case["positions"], case["channels"], case["groups"]
    gamma = torch.ones(c, device="cuda").double() if st["gamma"] is None else st["gamma"].double()
    beta = torch.zeros(c, device="cuda").double() if st["beta"] is None else st["beta"].double()
    parts = {}
    # a few samples at a time; gradients by torch's automatic differentiation
    each = max(1, (1 << 26) // (s * c))
    for i in range(0, n, each):
        m = min(each, n - i)
        x = st["x"][i * s:(i + m) * s].double().reshape(m, s, g, c // g)
        ga, be = gamma.clone().requires_grad_(), beta.clone().requires_grad_()
        var, mean = torch.var_mean(x, dim=(1, 3), correction=0, keepdim=True)
        rstd = torch.rsqrt(var + EPS)
        if case["way"] == "fwd":
            v = ((x - mean) * rstd).reshape(m * s, c) * gamma + beta
            got = {"y": acts[case["act"]](v), "mean": mean.reshape(m, g), "rstd": rstd.reshape(m, g)}
        else:
            hat = ((x - mean) * rstd).reshape(m * s, c).requires_grad_()
            y = acts[case["act"]](hat * ga + be)
            dhat, dga, dbe = torch.autograd.grad(y, (hat, ga, be), st["dy"][i * s:(i + m) * s].double())
            dhat, hat = dhat.reshape(m, s, g, c // g), hat.detach().reshape(m, s, g, c // g)
            dx = rstd * (dhat - dhat.mean((1, 3), keepdim=True) - hat * (dhat * hat).mean((1, 3), keepdim=True))
            got = {"dx": dx.reshape(m * s, c)}
            if st["affine"]:
                got["dgamma"], got["dbeta"] = dga, dbe
        for name, t in got.items():
            parts.setdefault(name, []).append(t)
    return {name: sum(t) if name in ("dgamma", "dbeta") else torch.cat(t) for name, t in parts.items()}


def _exact_recur(st, act):
    x, g = st["x"].double(), st["g"].double()
    gate = torch.ones_like(x) if st["o"] is None else act(st["o"].double())
    a = torch.sigmoid(g)
    if st["way"] == "step":
        state = st["state"].double()
        at = st["slots"].long()
        h = torch.lerp(x, state[at], a)
        state[at] = h
        return {"y": h * gate, "state": state}
    seqs = st["seqs"]
    if st["offsets"] is None:
        off = torch.arange(seqs + 1) * (st["rows"] // seqs)
    else:
        off = st["offsets"].cpu().long()
    used, length = int(off[-1]), (off[1:] - off[:-1])
    order = length.argsort(descending=True)                        # the longest first: those that have a position t are the first of them
    begin = off[:-1][order].cuda()
    many = [int((length > t).sum()) for t in range(int(length.max()))]
    state = st["h0"].double()[order.cuda()]
    h, before = torch.empty_like(x), torch.empty_like(x)
    for t, m in enumerate(many):
        at = begin[:m] + t
        before[at] = state[:m]
        state[:m] = torch.lerp(x[at], state[:m], a[at])
        h[at] = state[:m]
    back = order.argsort().cuda()
    if st["way"] == "fwd":
        return {"y": (h * gate)[:used], "last": state[back]}
    dy = st["dy"].double()
    e = dy * gate
    carry, dh = st["dlast"].double()[order.cuda()], torch.empty_like(x)
    for t in range(len(many) - 1, -1, -1):
        at = begin[:many[t]] + t
        dh[at] = e[at] + carry[:many[t]]
        carry[:many[t]] = a[at] * dh[at]
    out = {"dx": (torch.sigmoid(-g) * dh)[:used], "dg": (dh * (before - x) * a * torch.sigmoid(-g))[:used], "dh0": carry[back]}
    if st["o"] is not None:
        o = st["o"].double().requires_grad_()
        out["do"] = torch.autograd.grad(act(o), o, dy * h)[0][:used]
    return out
