"""The operators at the entrance and the end of a sparse expert layer, as cases that can be timed and checked.

Learned node embeddings are looked up by id and scaled; rows are normalised by their root mean square, with
the residual's addition before it and, for serving, a result in 8 bits with a scale for 32 values; and for
few rows, as a request brings them, all the chosen experts of a layer are one call: up and gate product,
activation, down product and the weighted sum of a row's experts.  Each case is one pass through one of the
three operators, with what a user's program would have in hand prepared beforehand.  The sizes are those of
the workloads that ``graphgen`` names (169,343 nodes; 2,449,029 nodes of 100 features; the typed graph of
1.9M, 736k and 8.7k nodes) or generic ones.

Kinds of case:
  embed    rows of a table by ids, times a scale; (train) and the table's gradient
  norm     root-mean-square norm, with a residual or not; (train) the gradients; (quant) the result in 8 bits
  experts  the chosen experts of few rows, with weights in 4 bits or bf16

Definitions.  Embedding: out[r] = scale * table[ids[r]]; ids outside the table are padding: a row of zeros
that reaches no gradient.  Norm: total = x + residual, rounded to the type of x; rstd = 1 / sqrt(mean over
the row of total^2 + eps); out = total * rstd * weight.  8 bits: E4M3 values under E8M0 scales
2^(floor(log2 max|x|) - 8) of 32 neighbouring values, to nearest, ties to even, saturating at 448 (OCP
microscaling formats, 2023).  Experts: h = act(w1 x), or gated act(g) * u where g and u are the first and
the second half of w1 x, out[r] = sum over the row's choices j (idx[r, j] >= 0) of weight[r, j] * w2 h.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-5


def listed():
    return [
        # serving: the embeddings of the few nodes that a request names; latency counts
        dict(name="embed-48", kind="embed", n=48, v=169343, f=128, dtype="bf16", ids="i64",
             spread="even", padding=0.0, train=False),
        # training on a mini-batch: sampled node ids, popular nodes many times, padded to a whole batch
        dict(name="embed-train-190k", kind="embed", n=190001, v=169343, f=256, dtype="f32", ids="i64",
             spread="popular", padding=0.05, train=True),
        # training on a large node table, as many lookups as the typed graph has nodes of one type
        dict(name="embed-train-1.9M", kind="embed", n=1900000, v=2449029, f=100, dtype="bf16", ids="i32",
             spread="popular", padding=0.0, train=True),
        # serving: before the experts of a handful of rows, the result in 8 bits; latency counts
        dict(name="norm-8bit-16", kind="norm", n=16, f=4096, dtype="bf16", residual=True, quant=True,
             train=False),
        # the hidden layer of a node table in training, with the residual stream
        dict(name="norm-train-169k", kind="norm", n=169343, f=256, dtype="bf16", residual=True,
             quant=False, train=True),
        # input features of full-graph training: rows of an odd number of bytes in lines
        dict(name="norm-train-2.4M", kind="norm", n=2449029, f=100, dtype="f32", residual=False,
             quant=False, train=True),
        # a large prompt or batch before 8-bit products
        dict(name="norm-8bit-65k", kind="norm", n=65537, f=4096, dtype="bf16", residual=True, quant=True,
             train=False),
        # one row, two of 8 experts, 4-bit weights: the single step of a served sequence
        dict(name="experts-1", kind="experts", n=1, experts=8, k=2, f=2048, h=4096, fo=2048, w="mx4",
             x="bf16", out="bf16", act="silu", gated=True, masked=False),
        # a few rows with odd sizes, in training's types, some rows without any choice
        dict(name="experts-7-odd", kind="experts", n=7, experts=16, k=2, f=1001, h=517, fo=999, w="bf16",
             x="f32", out="f32", act="relu", gated=False, masked=True),
        # a small batch of requests, 8 of 64 experts each, rows in 8 bits from the norm
        dict(name="experts-16", kind="experts", n=16, experts=64, k=8, f=2048, h=1024, fo=2048, w="mx4",
             x="mx8", out="bf16", act="silu", gated=True, masked=False),
        # a batch of requests, weights as they were trained
        dict(name="experts-64", kind="experts", n=64, experts=64, k=4, f=2048, h=1024, fo=2048, w="bf16",
             x="bf16", out="bf16", act="gelu", gated=True, masked=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed", "norm", "norm", "norm", "experts", "experts", "experts"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "embed":
        f = _log(rng, 1, 1024)
        return dict(kind=kind, n=_log(rng, 1, min(1900000, (1 << 27) // f)),
                    v=_log(rng, 2, min(2449029, (1 << 27) // f)), f=f, dtype=dtype,
                    ids=rng.choice(["i32", "i64"]), spread=rng.choice(["even", "popular", "popular"]),
                    padding=rng.choice([0.0, 0.05, 0.3]), train=rng.random() < 0.7)
    if kind == "norm":
        f = _log(rng, 1, 16384)
        quant = rng.random() < 0.4
        return dict(kind=kind, n=_log(rng, 1, min(2449029, (1 << 27) // f)), f=f, dtype=dtype,
                    residual=rng.random() < 0.6, quant=quant, train=not quant and rng.random() < 0.7)
    experts, f, h, fo = _log(rng, 1, 64), _log(rng, 30, 4096), _log(rng, 20, 4096), _log(rng, 16, 4096)
    gated = rng.random() < 0.6
    experts = max(1, min(experts, (1 << 28) // (h * (f * (1 + gated) + fo))))
    return dict(kind=kind, n=_log(rng, 1, 64), experts=experts,
                k=min(experts, rng.choice([1, 2, 2, 4, 6, 8])), f=f, h=h, fo=fo,
                w=rng.choice(["mx4", "mx4", "bf16"]), x=rng.choice(["f32", "bf16", "bf16", "mx8"]),
                out=dtype, act=rng.choice(["relu", "silu", "gelu"]), gated=gated,
                masked=rng.random() < 0.4)


# ---- inputs ----------------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + stream)
    return g


def _randn(seed, stream, *shape):
    return torch.randn(*shape, generator=_gen(seed, stream), device=DEV)


def _rand(seed, stream, *shape, dtype=torch.float32):
    return torch.rand(*shape, generator=_gen(seed, stream), device=DEV, dtype=dtype)


def _ids(c, seed):
    """Even: every row alike.  Popular: the logarithm of the rank is even, so that a node is the more
    often named the lower its number, the first by some 5 to 20 percent of all."""
    u = _rand(seed, 1, c["n"], dtype=torch.float64)
    ids = u * c["v"] if c["spread"] == "even" else torch.exp(u * math.log(c["v"] + 1)) - 1
    ids = ids.long().clamp(max=c["v"] - 1)
    if c["padding"]:
        ids = torch.where(_rand(seed, 2, c["n"]) < c["padding"], -1, ids)
    return ids.to(torch.int32 if c["ids"] == "i32" else torch.int64)


def _rows(seed, stream, n, f, dtype):
    """Rows whose sizes lie a power of two or so apart, with a channel that sticks out."""
    x = _randn(seed, stream, n, f).mul_(torch.exp2(_randn(seed, stream + 1, n, 1)))
    x[:, f // 3] *= 8
    return x.to(DT[dtype])


def _codes8(seed, stream, n, f):
    """Rows in 8 bits: E4M3 codes (none of them NaN) and scale bytes, filled up to whole blocks."""
    kb = -(-f // 32)
    v = (100.0 * _randn(seed, stream, n, kb * 32)).clamp(-448, 448)
    v[:, f:] = 0
    codes = v.to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, torch.randint(118, 122, (n, kb), generator=_gen(seed, stream + 1), device=DEV,
                                dtype=torch.uint8)


def _codes4(seed, stream, e, rows, k):
    """4-bit weights in the format's own layout: two codes a byte, the lower nibble first, rows filled up
    to whole blocks of 32."""
    kb = -(-k // 32)
    codes = torch.randint(0, 256, (e, rows, kb * 16), generator=_gen(seed, stream), device=DEV,
                          dtype=torch.uint8)
    if k % 32:
        at = torch.arange(kb * 32, device=DEV).view(-1, 2) < k
        codes &= (at[:, 0] * 15 + at[:, 1] * 240).to(torch.uint8)
    scales = torch.randint(119, 122, (e, rows, kb), generator=_gen(seed, stream + 1), device=DEV,
                           dtype=torch.uint8)
    return codes, scales


def prepare(case, seed):
    c, s = dict(case), {"case": dict(case)}
    kind, n, f = c["kind"], c["n"], c["f"]
    if kind == "embed":
        s["table"] = _randn(seed, 3, c["v"], f).mul_(f ** -0.5).to(DT[c["dtype"]])
        s["ids"] = _ids(c, seed)
        s["scale"] = f ** 0.5
        if c["train"]:
            s["dout"] = _randn(seed, 4, n, f).to(DT[c["dtype"]])
    elif kind == "norm":
        s["x"] = _rows(seed, 1, n, f, c["dtype"])
        s["residual"] = _rows(seed, 3, n, f, c["dtype"]) if c["residual"] else None
        s["weight"] = 1.0 + 0.2 * _randn(seed, 5, f)
        if c["train"]:
            s["dout"] = _randn(seed, 6, n, f).to(DT[c["dtype"]])
            s["dtotal"] = _randn(seed, 7, n, f).to(DT[c["dtype"]]) if c["residual"] else None
    elif kind == "experts":
        e, h, fo, rows1 = c["experts"], c["h"], c["fo"], c["h"] * (1 + c["gated"])
        if c["w"] == "mx4":
            s["w1"], s["w2"] = _codes4(seed, 1, e, rows1, f), _codes4(seed, 3, e, fo, h)
        else:
            s["w1"] = (_randn(seed, 1, e, rows1, f) * f ** -0.5).to(torch.bfloat16)
            s["w2"] = (_randn(seed, 3, e, fo, h) * h ** -0.5).to(torch.bfloat16)
        s["x"] = _codes8(seed, 5, n, f) if c["x"] == "mx8" else _randn(seed, 5, n, f).to(DT[c["x"]])
        # a router's choices: the largest of normal logits, their softmax weights
        top, idx = (1.5 * _randn(seed, 7, n, e)).topk(c["k"], dim=1)
        weight = torch.softmax(top, 1)
        if c["masked"]:  # rows that take no part have no choice
            off = (_rand(seed, 8, n, 1) < 0.2) & (torch.arange(n, device=DEV)[:, None] > 0)
            idx, weight = torch.where(off, -1, idx), torch.where(off, 0.0, weight)
        s["idx"], s["weight"] = idx.to(torch.int32).contiguous(), weight.contiguous()
    else:
        raise ValueError(kind)
    return s


# ---- plain forms -----------------------------------------------------------------------------

def _embed(s):
    c = s["case"]
    ids = s["ids"].long()
    inside = (ids >= 0) & (ids < c["v"])
    at = torch.where(inside, ids, 0)
    part = inside[:, None].float()
    r = dict(out=(s["table"][at].float() * s["scale"] * part).to(DT[c["dtype"]]))
    if c["train"]:
        d = torch.zeros(c["v"], c["f"], device=DEV)
        d.index_add_(0, at, s["dout"].float() * (part * s["scale"]))
        r["dtable"] = d.to(DT[c["dtype"]])
    return r


def _fp8(x):
    """The values that rows of x stand for once they are held in 8 bits, in fp32."""
    n, k = x.shape
    kb = -(-k // 32)
    v = torch.zeros(n, kb * 32, device=DEV)
    v[:, :k] = x
    v = v.view(n, kb, 32)
    e = (torch.frexp(v.abs().amax(2, keepdim=True))[1] - 9).clamp(min=-127)
    a = torch.ldexp(v, -e).clamp(-448, 448).to(torch.float8_e4m3fn).float()
    return torch.ldexp(a, e).view(n, kb * 32)[:, :k]


def _norm(s):
    c, dt = s["case"], DT[s["case"]["dtype"]]
    total, r = s["x"], {}
    if s["residual"] is not None:
        total = (s["x"].float() + s["residual"].float()).to(dt)
        r["total"] = total
    t = total.float()
    rstd = 1 / torch.sqrt((t * t).mean(1, keepdim=True) + EPS)
    xhat = t * rstd
    out = xhat * s["weight"]
    if c["quant"]:
        r["values"] = _fp8(out).to(dt)
        return r
    r["out"], r["rstd"] = out.to(dt), rstd[:, 0]
    if c["train"]:
        d = s["dout"].float()
        r["dweight"] = (d * xhat).sum(0)
        g = d * s["weight"]
        dx = (g - xhat * (g * xhat).mean(1, keepdim=True)) * rstd
        if s["dtotal"] is not None:
            dx = dx + s["dtotal"].float()
        r["dx"] = dx.to(dt)
    return r


def _values4(codes, scales, k):
    """[..., k] fp32 of packed 4-bit codes and scale exponents."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    lead, nb = codes.shape[:-1], scales.shape[-1]
    v = table[torch.stack([codes & 15, codes >> 4], -1).view(*lead, nb, 32).int()]
    return torch.ldexp(v, scales.int()[..., None] - 127).view(*lead, nb * 32)[..., :k]


def _weights(w, at, k):
    """[len(at) or all, rows, k] fp32 of an expert's weights."""
    if isinstance(w, tuple):
        codes, scales = w
        return _values4(codes if at is None else codes[at], scales if at is None else scales[at], k)
    return (w if at is None else w[at]).float()


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z * 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))


def _experts(s):
    c = s["case"]
    n, k, e, f, h = c["n"], c["k"], c["experts"], c["f"], c["h"]
    if c["x"] == "mx8":
        x = s["x"][0].view(torch.float8_e4m3fn).float().view(n, -1, 32)
        x = torch.ldexp(x, s["x"][1].int()[..., None] - 127).view(n, -1)[:, :f]
    else:
        x = s["x"].float()
    idx = s["idx"].long()
    weight = torch.where(idx >= 0, s["weight"], 0.0)
    idx = idx.clamp(min=0)
    if n * k < e:  # the weights of every choice
        at = idx.view(-1)
        z = (_weights(s["w1"], at, f) @ x.repeat_interleave(k, 0)[:, :, None])[:, :, 0]
    else:          # all experts, and a row's share in each
        at = None
        z = torch.matmul(x[None], _weights(s["w1"], None, f).transpose(1, 2).contiguous())
        share = torch.zeros(n, e, device=DEV).scatter_add_(1, idx, weight)
    z = _act(z[..., :h], c["act"]) * z[..., h:] if c["gated"] else _act(z, c["act"])
    if at is not None:
        y = (_weights(s["w2"], at, h) @ z[:, :, None])[:, :, 0].view(n, k, -1)
        out = (y * weight[:, :, None]).sum(1)
    else:
        z = z * share.t()[:, :, None]
        out = torch.matmul(z, _weights(s["w2"], None, h).transpose(1, 2).contiguous()).sum(0)
    return dict(out=out.to(DT[c["out"]]))


# ---- the framework's operators ----------------------------------------------------------------

def _own(s):
    import paper_2507_16991_amd as mp

    c = s["case"]
    kind = c["kind"]
    if kind == "embed":
        r = dict(out=mp.embed(s["ids"], s["table"], scale=s["scale"]))
        if c["train"]:
            r["dtable"] = mp.embed_backward(s["ids"], s["dout"], c["v"], scale=s["scale"])
        return r
    if kind == "norm":
        if c["quant"]:
            codes, scales, values, total = mp.rms_norm_mx8(
                s["x"], s["weight"], residual=s["residual"], eps=EPS, want_values=True)
            return dict(values=values, total=total) if s["residual"] is not None else dict(values=values)
        out, total, rstd = mp.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        r = dict(out=out, rstd=rstd)
        if s["residual"] is not None:
            r["total"] = total
        if c["train"]:
            r["dx"], r["dweight"] = mp.rms_norm_backward(total, s["dout"], rstd, s["weight"],
                                                         dtotal=s["dtotal"])
        return r
    return dict(out=mp.expert_mlp(s["x"], s["idx"], s["weight"], s["w1"], s["w2"], act=c["act"],
                                  gated=c["gated"], out_dtype=DT[c["out"]]))


def run(state):
    if own:
        return _own(state)
    return {"embed": _embed, "norm": _norm, "experts": _experts}[state["case"]["kind"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    c = case
    kind, n, f = c["kind"], c["n"], c["f"]
    if kind == "embed":
        b = BYTES[c["dtype"]]
        # each row of the table that is named at all is read once
        named = min(n, c["v"])
        if c["spread"] == "popular":  # 1 - (1 - p)^n over ranks of probability about 1 / (rank log v)
            at = np.exp(np.linspace(0.0, math.log(c["v"]), 4097))
            p = np.minimum(1.0, 1.0 / (at * math.log(c["v"] + 1)))
            named = float(np.trapezoid(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-9))), at))
        bytes_ = n * (8 if c["ids"] == "i64" else 4) + (named + n) * f * b
        if c["train"]:
            bytes_ += n * (8 if c["ids"] == "i64" else 4) + (n + c["v"]) * f * b
        return {"bytes": bytes_, "flops": n * f * (3 if c["train"] else 1)}
    if kind == "norm":
        b = BYTES[c["dtype"]]
        passes = 2 + 2 * c["residual"]                 # x, out; residual, total
        if c["train"]:
            passes += 3 + c["residual"]                # total, dout, dx; dtotal
        extra = n * -(-f // 32) * 33 if c["quant"] else 0  # codes and scales beside the values
        return {"bytes": n * f * b * passes + extra + 4 * f * (3 if c["train"] else 1)
                + (8 * n if c["train"] else 4 * n), "flops": n * f * (14 if c["train"] else 5)}
    k, e, h, fo, rows1 = c["k"], c["experts"], c["h"], c["fo"], c["h"] * (1 + c["gated"])
    live = n * (0.8 if c["masked"] else 1.0)
    used = e * (1 - (1 - k / e) ** live)  # experts that some row chose
    if c["w"] == "mx4":
        weights = rows1 * -(-f // 32) * 17 + fo * -(-h // 32) * 17
    else:
        weights = 2 * (rows1 * f + fo * h)
    x = -(-f // 32) * 33 if c["x"] == "mx8" else f * BYTES[c["x"]]
    return {"bytes": used * weights + n * (x + 8 * k + fo * BYTES[c["out"]]),
            "flops": 2.0 * live * k * (rows1 * f + fo * h)}


# ---- the definitions in 64 bits -----------------------------------------------------------------

def _exact_embed(s):
    c = s["case"]
    ids = s["ids"].to(torch.int64)
    ok = (ids > -1) & (ids < c["v"])
    out = torch.zeros(c["n"], c["f"], dtype=torch.float64, device=DEV)
    out[ok] = s["table"].index_select(0, ids[ok]).double().mul_(s["scale"])
    r = dict(out=out)
    if c["train"]:
        d = torch.zeros(c["v"], c["f"], dtype=torch.float64, device=DEV)
        d.index_put_((ids[ok],), s["dout"][ok].double(), accumulate=True)
        r["dtable"] = d.mul_(s["scale"])
    return r


def _exact_fp8(y):
    """By halfway points: a step of the format between powers of two is an eighth of the lower one."""
    n, k = y.shape
    v = torch.nn.functional.pad(y, (0, -k % 32)).view(n, -1, 32)
    top = v.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -119))) - 8)
    scale = torch.where(top / scale >= 512, scale * 2, torch.where(top / scale < 256, scale / 2, scale))
    scale = scale.clamp(min=2.0 ** -127)
    a = (v / scale).abs()
    low = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))))
    step = torch.where(a < 2.0 ** -6, 2.0 ** -6, low) / 8
    q = (a / step).round() * step
    return (torch.copysign(q.clamp(max=448.0), v) * scale).view(n, -1)[:, :k]


def _exact_norm(s):
    c = s["case"]
    x, w, r = s["x"].double(), s["weight"].double(), {}
    if s["residual"] is not None:
        r["total"] = x.add(s["residual"].double())
        # the norm is that of the sum as it is stored
        x = r["total"].to(DT[c["dtype"]]).double()
    rstd = (x.square().sum(1) / c["f"] + EPS).rsqrt()
    y = x * rstd[:, None]
    if c["quant"]:
        r["values"] = _exact_fp8(y * w)
        return r
    r["out"], r["rstd"] = y * w, rstd
    if c["train"]:
        d = s["dout"].double()
        r["dweight"] = torch.sum(d * y, 0)
        d = d * w
        dot = (d * x).sum(1) * rstd.pow(3) / c["f"]
        dx = d * rstd[:, None] - x * dot[:, None]
        r["dx"] = dx if s["dtotal"] is None else dx + s["dtotal"].double()
    return r


def _exact_weights(w, k):
    if not isinstance(w, tuple):
        return w.double()
    codes, scales = w
    b = torch.stack((codes % 16, codes // 16), -1).view(*codes.shape[:-1], -1).short()
    exponent, mantissa = b % 8 // 2, b % 2
    v = torch.where(exponent > 0, (2.0 + mantissa) * torch.exp2(exponent - 2.0), mantissa / 2.0).double()
    v *= 1 - 2 * (b // 8)
    v = v.view(*scales.shape, 32) * torch.exp2(scales.double() - 127).unsqueeze(-1)
    return v.view(*codes.shape[:-1], -1)[..., :k]


def _exact_experts(s, e, x):
    """What expert e adds to the rows, and to which."""
    c = s["case"]
    at, j = (s["idx"] == e).nonzero(as_tuple=True)
    pick = lambda w: tuple(t[e] for t in w) if isinstance(w, tuple) else w[e]  # noqa: E731
    z = x[at] @ _exact_weights(pick(s["w1"]), c["f"]).t().contiguous()
    g = z[:, :c["h"]]
    if c["act"] == "relu":
        g = g.relu()
    elif c["act"] == "silu":
        g = g * g.sigmoid()
    else:
        g = g * 0.5 * torch.erfc(g / -2 ** 0.5)
    if c["gated"]:
        g = g * z[:, c["h"]:]
    y = g @ _exact_weights(pick(s["w2"]), c["h"]).t().contiguous()
    return at, y * s["weight"].double()[at, j][:, None]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "embed":
        return _exact_embed(s)
    if case["kind"] == "norm":
        return _exact_norm(s)
    if case["x"] == "mx8":
        code, scale = s["x"][0].long(), s["x"][1]
        exponent, mantissa = code % 128 // 8, code % 8
        x = torch.where(exponent > 0, (8.0 + mantissa) * torch.exp2(exponent - 10.0), mantissa / 512.0)
        x = (x * (1 - 2 * (code // 128))).double().view(*scale.shape, 32)
        x = (x * torch.exp2(scale.double() - 127).unsqueeze(-1)).view(case["n"], -1)[:, :case["f"]]
    else:
        x = s["x"].double()
    out = torch.zeros(case["n"], case["fo"], dtype=torch.float64, device=DEV)
    for e in range(case["experts"]):
        at, y = _exact_experts(s, e, x)
        out.index_add_(0, at, y)
    return dict(out=out)
