"""The operators of a sparse expert layer over node features, as cases that can be timed and checked.

Such a layer normalises the nodes of each graph (group norm with an activation, channels last, over
ragged segments of rows), lets a router choose k experts a node (with the per-expert counts, a balance
loss and its gradients), multiplies the nodes of each expert by the expert's weights (in training the
typed projections, for serving microscaled 4-bit floating point), and drops features, nodes or edges by
a counter-based generator.  Each case is one pass through one of the four operators, with what a user's
program would have in hand prepared beforehand.  The sizes are those of the workloads that ``graphgen``
names (2,708 nodes; 169,343; 2,449,029 nodes of 100 features and 124M edges; the typed graph of 1.9M,
736k and 8.7k nodes) or generic ones.

Kinds of case:
  norm      group norm with an activation over segments of rows, forward, or (train) with its gradients
  dropout   dropout of elements or rows, with a residual or not, keyed by position or by ids; forward,
            or (train) with the gradient
  route     softmax router: the k largest logits of a row, counts, balance and z loss; (train) gradient
  quantize  a table to 4-bit floating point with a power-of-two scale for 32 values of a row
  product   rows of segments times the segments' 4-bit weights, the rows quantised on the way

Definitions.  Group norm: mean and variance of a segment's rows and a group's channels; rows of an
empty segment do not exist, its mean and rstd are 0.  Dropout: word w of element e = id * F + f (or of
row e = id) is the (e % 8)-th 16-bit word of Philox4x32-10 (Salmon et al. 2011) with key = seed and
counter = (e / 8, offset); the element stays where w >= round(65536 p), times 65536 / (65536 -
round(65536 p)).  Router: see ``_route``.  4-bit: E2M1 values under E8M0 scales 2^(floor(log2 max|x|) -
2), to nearest, ties to even, saturating at 6 (OCP microscaling formats, 2023).
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
        # serving: the nodes of one small graph, between two layers; latency counts
        dict(name="norm-2.7k", kind="norm", n=2708, segments=1, lengths="even", groups=8, width=8,
             dtype="f32", act="silu", train=False),
        # training on a batch of molecules: thousands of graphs of about two dozen atoms
        dict(name="norm-train-190k", kind="norm", n=190001, segments=8192, lengths="ragged", groups=32,
             width=4, dtype="bf16", act="relu", train=True),
        # training on a batch of 1,024 large graphs of very different sizes, groups of 25 channels
        dict(name="norm-train-2.4M", kind="norm", n=2449029, segments=1024, lengths="skewed", groups=4,
             width=25, dtype="bf16", act="gelu", train=True),
        # the hidden layer of a small graph network in training
        dict(name="dropout-2.7k", kind="dropout", n=2708, f=64, dtype="f32", p=0.5, residual=False,
             ids=False, rows=False, train=True),
        # a residual branch of full-graph training
        dict(name="dropout-2.4M", kind="dropout", n=2449029, f=100, dtype="bf16", p=0.1, residual=True,
             ids=False, rows=False, train=True),
        # edges dropped from 124M weights in destination order, keyed by the edges' own numbers, so
        # that the transposed order drops the same ones
        dict(name="dropout-edges-124M", kind="dropout", n=123718280, f=1, dtype="f32", p=0.2,
             residual=False, ids=True, rows=False, train=False),
        # serving: a handful of rows choose 8 of 64 experts; latency counts
        dict(name="route-16", kind="route", n=16, experts=64, k=8, dtype="f32", masked=False,
             train=False),
        # training: a node table, a part of it padding, chooses 8 of 64 experts; both losses
        dict(name="route-train-169k", kind="route", n=169343, experts=64, k=8, dtype="bf16",
             masked=True, train=True),
        # the weights of 8 experts to 4 bits, and the values they stand for (for training with them)
        dict(name="quantize-32k", kind="quantize", n=32768, k=4096, dtype="bf16"),
        # serving: 8 rows with two experts each, out of 8
        dict(name="product-16", kind="product", n=16, types=8, lengths="ragged", k=2048, fo=4096,
             dtype="bf16", out="bf16"),
        # typed projections of the typed graph's node tables
        dict(name="product-2.6M", kind="product", n=2644700, types=3, lengths="typed", k=128, fo=128,
             dtype="bf16", out="bf16"),
        # experts' products of a large batch
        dict(name="product-65k", kind="product", n=65537, types=8, lengths="ragged", k=4096, fo=4096,
             dtype="bf16", out="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm", "dropout", "dropout", "route", "route", "quantize",
                       "product", "product", "product"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "norm":
        groups, width = _log(rng, 1, 32), _log(rng, 1, 40)
        n = _log(rng, 500, min(2449029, (1 << 28) // (groups * width)))
        return dict(kind=kind, n=n, segments=_log(rng, 1, max(1, min(20000, n // 10))),
                    lengths=rng.choice(["even", "ragged", "ragged", "skewed"]), groups=groups,
                    width=width, dtype=dtype, act=rng.choice(["none", "relu", "silu", "gelu"]),
                    train=rng.random() < 0.6)
    if kind == "dropout":
        f = 1 if rng.random() < 0.3 else _log(rng, 2, 512)
        n = _log(rng, 500, (1 << 26) if f == 1 else min(2449029, (1 << 28) // f))
        return dict(kind=kind, n=n, f=f, dtype=dtype, p=round(rng.uniform(0.02, 0.7), 3),
                    residual=rng.random() < 0.4, ids=rng.random() < 0.4,
                    rows=f > 1 and rng.random() < 0.3, train=rng.random() < 0.5)
    if kind == "route":
        experts = _log(rng, 4, 256)
        n = _log(rng, 1, min(1000000, (1 << 25) // experts))
        return dict(kind=kind, n=n, experts=experts, k=min(experts, rng.choice([1, 2, 2, 4, 6, 8])),
                    dtype=dtype, masked=rng.random() < 0.5, train=rng.random() < 0.6)
    if kind == "quantize":
        k = _log(rng, 30, 8192)
        return dict(kind=kind, n=_log(rng, 1, (1 << 27) // k), k=k, dtype=dtype)
    k, fo, types = _log(rng, 30, 4096), _log(rng, 16, 4096), _log(rng, 1, 64)
    n = _log(rng, 1, min(2000000, (1 << 39) // (k * fo), (1 << 28) // max(k, fo)))
    types = max(1, min(types, (1 << 27) // (k * fo)))
    return dict(kind=kind, n=n, types=types, lengths=rng.choice(["ragged", "even"]), k=k, fo=fo,
                dtype=dtype, out=rng.choice(["f32", "bf16"]))


# ---- inputs ----------------------------------------------------------------------------------

def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + stream)
    return g


def _randn(seed, stream, *shape):
    return torch.randn(*shape, generator=_gen(seed, stream), device=DEV)


def _rand(seed, stream, *shape):
    return torch.rand(*shape, generator=_gen(seed, stream), device=DEV)


def _offsets(c, parts, seed):
    """Offsets of `parts` consecutive segments of c["n"] rows, a list of ints: equal lengths; random
    borders (ragged, a few of them empty); half of the rows in one segment (skewed); the shares of the
    typed graph's node types."""
    n = c["n"]
    if c["lengths"] == "even":
        return [n * i // parts for i in range(parts + 1)]
    if c["lengths"] == "typed":
        return [0, 1900000 * n // 2644700, 2636000 * n // 2644700, n]
    r = np.random.default_rng([int(seed), 77])
    inner = np.sort(r.integers(0, n + 1, parts - 1))
    if c["lengths"] == "skewed":
        half = np.sort(r.integers(0, n // 2 + 1, parts - 1))
        at = int(r.integers(0, parts))
        inner = np.where(np.arange(parts - 1) >= at, half + (n - n // 2), half)
    return [0] + [int(v) for v in inner] + [n]


def _features(c, seed, stream, n, f):
    """Node features as aggregation leaves them: every channel with an offset and a spread of its own."""
    x = _randn(seed, stream, n, f)
    x.mul_(0.5 + _rand(seed, stream + 1, f)).add_(2.0 * _randn(seed, stream + 2, f))
    return x.to(DT[c["dtype"]])


def _scaled(c, seed, stream, n, k):
    """Rows whose scales lie a few powers of two apart, with an outlier here and there."""
    x = _randn(seed, stream, n, k)
    x.mul_(torch.exp2(2.0 * _randn(seed, stream + 1, n, 1)))
    x.mul_(torch.where(_rand(seed, stream + 2, n, k) < 0.001, 16.0, 1.0))
    return x.to(DT[c["dtype"]])


def prepare(case, seed):
    c, s = dict(case), {"case": dict(case)}
    kind, n = c["kind"], c["n"]
    if kind == "norm":
        f = c["groups"] * c["width"]
        s["ptr"] = torch.tensor(_offsets(c, c["segments"], seed), device=DEV, dtype=torch.int32)
        s["x"] = _features(c, seed, 1, n, f)
        s["weight"] = 1.0 + 0.1 * _randn(seed, 5, f)
        s["bias"] = 0.1 * _randn(seed, 6, f)
        if c["train"]:
            s["dout"] = _randn(seed, 7, n, f).to(DT[c["dtype"]])
    elif kind == "dropout":
        shape = (n, c["f"])
        s["x"] = _randn(seed, 1, *shape).to(DT[c["dtype"]])
        s["residual"] = _randn(seed, 2, *shape).to(DT[c["dtype"]]) if c["residual"] else None
        s["ids"] = (torch.randperm(n, generator=_gen(seed, 3), device=DEV).to(torch.int32)
                    if c["ids"] else None)
        s["dout"] = _randn(seed, 4, *shape).to(DT[c["dtype"]]) if c["train"] else None
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 * (int(seed) + 1) % (1 << 63), 1000 + int(seed)
    elif kind == "route":
        e = c["experts"]
        s["logits"] = (1.5 * _randn(seed, 1, n, e) + 0.5 * _randn(seed, 2, e)).to(DT[c["dtype"]])
        s["mask"] = None
        if c["masked"]:  # padding rows hold whatever was there before
            s["mask"] = _rand(seed, 3, n) < 0.9
            s["logits"][~s["mask"]] = float("nan")
        if c["train"]:
            s["dweight"] = _randn(seed, 4, n, c["k"])
            s["dloss"] = torch.tensor([0.01 * n, 0.001 * n], device=DEV)
    elif kind == "quantize":
        s["x"] = _scaled(c, seed, 1, n, c["k"])
    elif kind == "product":
        t, fo, k = c["types"], c["fo"], c["k"]
        s["offsets"] = _offsets(c, t, seed)
        s["seg"] = torch.tensor(s["offsets"], device=DEV, dtype=torch.int32)
        s["x"] = _scaled(c, seed, 1, n, k)
        # weights come in the format's own layout: two codes a byte, the lower nibble first, rows
        # filled up to whole blocks of 32
        kb = -(-k // 32)
        codes = torch.randint(0, 256, (t, fo, kb * 16), generator=_gen(seed, 4), device=DEV,
                              dtype=torch.uint8)
        if k % 32:
            at = torch.arange(kb * 32, device=DEV).view(-1, 2) < k
            codes &= (at[:, 0] * 15 + at[:, 1] * 240).to(torch.uint8)
        s["codes"] = codes
        s["scales"] = torch.randint(118, 124, (t, fo, kb), generator=_gen(seed, 5), device=DEV,
                                    dtype=torch.uint8)
    else:
        raise ValueError(kind)
    return s


# ---- plain forms -----------------------------------------------------------------------------

def _act(z, act):
    """act(z) and its derivative."""
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if act == "silu":
        g = 1 / (1 + torch.exp(-z))
        return z * g, g * (1 + z * (1 - g))
    if act == "gelu":
        g = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * g, g + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return z, torch.ones_like(z)


def _norm(s):
    c, ptr = s["case"], s["ptr"].long()
    n, g, w = c["n"], c["groups"], c["width"]
    lengths = ptr[1:] - ptr[:-1]
    at = torch.repeat_interleave(torch.arange(c["segments"], device=DEV), lengths, output_size=n)
    count = (lengths.clamp(min=1) * w).float()[:, None]

    def over(v):  # the mean over every segment's rows and a group's channels
        return torch.zeros(c["segments"], g, device=DEV).index_add_(0, at, v.sum(2)) / count

    x = s["x"].float().view(n, g, w)
    mean = over(x)
    d = x - mean[at][:, :, None]
    rstd = (lengths > 0).float()[:, None] / torch.sqrt(over(d * d) + EPS)
    xhat = (d * rstd[at][:, :, None]).view(n, g * w)
    out, slope = _act(xhat * s["weight"] + s["bias"], c["act"])
    r = dict(out=out.to(DT[c["dtype"]]), mean=mean, rstd=rstd)
    if c["train"]:
        da = s["dout"].float() * slope
        r["dweight"], r["dbias"] = (da * xhat).sum(0), da.sum(0)
        da = (da * s["weight"]).view(n, g, w)
        xhat = xhat.view(n, g, w)
        dx = da - over(da)[at][:, :, None] - xhat * over(da * xhat)[at][:, :, None]
        r["dx"] = (dx * rstd[at][:, :, None]).view(n, g * w).to(DT[c["dtype"]])
    return r


def _philox(block, seed, offset):
    """The four 32-bit words of Philox4x32-10 for the counters (block, offset), in int64."""
    low = 0xFFFFFFFF
    c0, c1 = block & low, block >> 32
    c2, c3 = torch.full_like(block, offset & low), torch.full_like(block, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        # int64 products wrap; their upper half is right after the mask
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _keep(s):
    """Which elements stay, [n, f] or [n, 1], and what those that stay are multiplied by."""
    c = s["case"]
    n, f = c["n"], 1 if c["rows"] else c["f"]
    limit = int(math.floor(65536 * c["p"] + 0.5))
    if s["ids"] is None:  # consecutive elements share a block
        words = _philox(torch.arange(-(-n * f // 8), device=DEV), s["seed"], s["offset"])
        words = torch.stack([h for w in words for h in (w & 65535, w >> 16)], 1).view(-1)[:n * f]
    else:
        e = (s["ids"].long()[:, None] * f + torch.arange(f, device=DEV)).view(-1)
        words = torch.stack(_philox(e >> 3, s["seed"], s["offset"]))
        words = words.gather(0, ((e >> 1) & 3)[None])[0] >> (16 * (e & 1)) & 65535
    return (words >= limit).view(n, f), 65536 / (65536 - limit)


def _dropout(s):
    c = s["case"]
    keep, scale = _keep(s)
    zero = torch.zeros((), device=DEV)
    out = torch.where(keep, s["x"].float() * scale, zero)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    r = dict(out=out.to(DT[c["dtype"]]))
    if s["dout"] is not None:
        r["dx"] = torch.where(keep, s["dout"].float() * scale, zero).to(DT[c["dtype"]])
    return r


def _route(s):
    """Of every row that takes part (mask, and a logit above -inf): the experts of its k largest logits
    (equal ones: the lower number first), their softmax weights among the k, and over all such rows the
    rows' number R, the choices c_e of every expert and the means P_e of the softmax over all experts.
    balance = experts * sum_e c_e / (sum c) * P_e; z = the mean of logsumexp^2."""
    c = s["case"]
    e, k = c["experts"], c["k"]
    l = s["logits"].float()
    if s["mask"] is not None:
        l = torch.where(s["mask"][:, None], l, torch.full((), -torch.inf, device=DEV))
    part = (l > -torch.inf).any(1)
    top, idx = torch.sort(l, dim=1, descending=True, stable=True)
    top, idx = top[:, :k], idx[:, :k]
    real = top > -torch.inf
    big = torch.where(part, top[:, 0], 0.0)[:, None]
    weight = torch.exp(top - big)
    weight = weight / weight.sum(1, keepdim=True).clamp(min=1e-30)
    p = torch.exp(l - big)
    total = p.sum(1, keepdim=True).clamp(min=1e-30)
    p = p / total
    rows = part.sum()
    chosen = torch.zeros(e + 1, dtype=torch.int32, device=DEV)
    chosen.index_add_(0, torch.where(real, idx, e).view(-1),
                      torch.ones(idx.numel(), dtype=torch.int32, device=DEV))
    chosen = chosen[:e]
    share = chosen.float() / chosen.sum().clamp(min=1)
    some = rows.clamp(min=1)
    balance = e * (share * (p.sum(0) / some)).sum()
    lse = torch.where(part, torch.log(total[:, 0]) + big[:, 0], 0.0)
    z = (lse * lse).sum() / some
    r = dict(idx=torch.where(real, idx, -1).int(), weight=weight, counts=torch.cat([chosen, rows[None].int()]),
             loss=torch.stack([balance, z]))
    if c["train"]:
        dw = torch.where(real, s["dweight"], 0.0)
        dtop = weight * (dw - (weight * dw).sum(1, keepdim=True))
        dp = s["dloss"][0] * e * share / some
        dl = p * (dp - (p * dp).sum(1, keepdim=True) + 2 * s["dloss"][1] * (lse / some)[:, None])
        dl = dl.scatter_add(1, idx, torch.where(real, dtop, 0.0))
        r["dlogits"] = torch.where(part[:, None], dl, 0.0).to(DT[c["dtype"]])
    return r


def _fp4(x):
    """The values that rows of x stand for once they are held in 4 bits, in fp32."""
    n, k = x.shape
    kb = -(-k // 32)
    v = torch.zeros(n, kb * 32, device=DEV)
    v[:, :k] = x
    v = v.view(n, kb, 32)
    e = (torch.frexp(v.abs().amax(2, keepdim=True))[1] - 3).clamp(min=-127)
    a = torch.ldexp(v, -e)
    step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(-6, 6)
    return torch.ldexp(a, e).view(n, kb * 32)[:, :k]


def _values(codes, scales, k):
    """[t, fo, k] fp32 of packed codes and scale exponents."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    t, fo, nb = codes.shape
    v = table[torch.stack([codes & 15, codes >> 4], 3).view(t, fo, -1, 32).int()]
    return torch.ldexp(v, scales.int()[..., None] - 127).view(t, fo, -1)[:, :, :k]


def _product(s):
    c, at = s["case"], s["offsets"]
    x, w = _fp4(s["x"].float()), _values(s["codes"], s["scales"], c["k"])
    out = [x[at[t]:at[t + 1]] @ w[t].t() for t in range(c["types"])]
    return dict(out=torch.cat(out).to(DT[c["out"]]))


def _quantize(s):
    return dict(values=_fp4(s["x"].float()).to(DT[s["case"]["dtype"]]))


# ---- the framework's operators ----------------------------------------------------------------

def _own(s):
    import paper_2507_16991_amd as mp

    c = s["case"]
    kind = c["kind"]
    if kind == "norm":
        out, mean, rstd = mp.group_norm(s["ptr"], s["x"], c["groups"], weight=s["weight"],
                                        bias=s["bias"], eps=EPS, act=c["act"])
        r = dict(out=out, mean=mean, rstd=rstd)
        if c["train"]:
            r["dx"], r["dweight"], r["dbias"] = mp.group_norm_backward(
                s["ptr"], s["x"], s["dout"], c["groups"], mean, rstd, weight=s["weight"],
                bias=s["bias"], act=c["act"])
        return r
    if kind == "dropout":
        key = dict(offset=s["offset"], ids=s["ids"], rows=c["rows"])
        r = dict(out=mp.dropout(s["x"], c["p"], s["seed"], residual=s["residual"], **key))
        if c["train"]:
            r["dx"] = mp.dropout_backward(s["dout"], c["p"], s["seed"], **key)
        return r
    if kind == "route":
        idx, weight, counts, loss = mp.route(s["logits"], c["k"], mask=s["mask"])
        r = dict(idx=idx, weight=weight, counts=counts, loss=loss)
        if c["train"]:
            r["dlogits"] = mp.route_backward(s["logits"], idx, weight, counts, dweight=s["dweight"],
                                             dloss=s["dloss"], mask=s["mask"])
        return r
    if kind == "quantize":
        codes, scales, values = mp.mx_quantize(s["x"], want_values=True)
        return dict(values=values)
    return dict(out=mp.mx_segment_matmul(s["seg"], s["x"], s["codes"], s["scales"],
                                         out_dtype=DT[c["out"]]))


def run(state):
    if own:
        return _own(state)
    return {"norm": _norm, "dropout": _dropout, "route": _route, "quantize": _quantize,
            "product": _product}[state["case"]["kind"]](state)


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    c = case
    kind, n = c["kind"], c["n"]
    if kind == "norm":
        f, g = c["groups"] * c["width"], c["groups"]
        small = 8 * f + 4 * (c["segments"] + 1) + 8 * c["segments"] * g + (8 * f if c["train"] else 0)
        return {"bytes": n * f * BYTES[c["dtype"]] * (4 if c["train"] else 2) + small,
                "flops": n * f * (30 if c["train"] else 12)}
    if kind == "dropout":
        passes = 2 + c["residual"] + (2 if c["train"] else 0)
        return {"bytes": n * c["f"] * BYTES[c["dtype"]] * passes + (4 * n if c["ids"] else 0),
                "flops": 2 * n * c["f"] * (2 if c["train"] else 1)}
    if kind == "route":
        e, k, b = c["experts"], c["k"], BYTES[c["dtype"]]
        return {"bytes": n * (e * b + 8 * k + c["masked"]) + 4 * e
                + (n * (e * b + 4 * k) if c["train"] else 0),
                "flops": n * e * (12 if c["train"] else 5)}
    kb = -(-c["k"] // 32)
    if kind == "quantize":  # the codes and scales are written besides the values
        return {"bytes": 2 * n * c["k"] * BYTES[c["dtype"]] + n * kb * 17, "flops": 4 * n * c["k"]}
    # weights of the segments that have rows
    t = c["types"]
    used = t if c["lengths"] != "ragged" else t * n / (n + t - 1)
    return {"bytes": n * c["k"] * BYTES[c["dtype"]] + used * c["fo"] * kb * 17
            + n * c["fo"] * BYTES[c["out"]], "flops": 2.0 * n * c["k"] * c["fo"]}


# ---- the definitions in 64 bits -----------------------------------------------------------------

def _exact_norm(s):
    """Segment by segment for a few of them, by differences of exact running sums otherwise."""
    c, n = s["case"], s["case"]["n"]
    g, w, ptr = c["groups"], c["width"], s["ptr"].long()
    wt, bs = s["weight"].double().view(g, w), s["bias"].double().view(g, w)
    lengths = ptr[1:] - ptr[:-1]
    slot = torch.searchsorted(ptr[1:].contiguous(), torch.arange(n, device=DEV), right=True)
    share = torch.where(lengths > 0, 1.0 / (lengths * w).double(), 0.0)

    def mean_of(v):  # [n, g] -> [segments, g]
        run = torch.zeros(n + 1, g, dtype=torch.float64, device=DEV)
        torch.cumsum(v, 0, out=run[1:])
        return (run[ptr[1:]] - run[ptr[:-1]]) * share[:, None]

    x = s["x"].double().reshape(n, g, w)
    mean = mean_of(x.sum(-1))
    x -= mean.index_select(0, slot).unsqueeze(-1)
    rstd = torch.where(lengths[:, None] > 0, (mean_of(x.pow(2).sum(-1)) + EPS).rsqrt(), 0.0)
    x *= rstd.index_select(0, slot).unsqueeze(-1)
    z = x * wt + bs
    act = c["act"]
    if act == "relu":
        out, slope = z.relu(), z.gt(0).double()
    elif act == "silu":
        q = z.sigmoid()
        out, slope = z * q, q + z * q * (1 - q)
    elif act == "gelu":
        q = 0.5 * torch.erfc(-z / 2 ** 0.5)
        out, slope = z * q, q + z * (z.square() / -2).exp() * (2 * math.pi) ** -0.5
    else:
        out, slope = z, torch.ones((), dtype=torch.float64, device=DEV)
    r = dict(out=out.reshape(n, g * w), mean=mean, rstd=rstd)
    del z, out
    if c["train"]:
        d = s["dout"].double().view(n, g, w) * slope
        del slope
        r["dbias"] = d.sum(0).view(-1)
        r["dweight"] = (d * x).sum(0).view(-1)
        d *= wt
        a, b = mean_of(d.sum(-1)), mean_of((d * x).sum(-1))
        d -= a.index_select(0, slot).unsqueeze(-1)
        x *= b.index_select(0, slot).unsqueeze(-1)
        d -= x
        d *= rstd.index_select(0, slot).unsqueeze(-1)
        r["dx"] = d.view(n, g * w)
    return r


def _exact_words(e, seed, offset):
    """The 16-bit random word of every element number e: Philox on pairs of 16-bit halves, whose
    products cannot overflow."""
    def times(v, m):  # upper and lower 32 bits of v * m
        a, b, h, l = v // 65536, v % 65536, m // 65536, m % 65536
        low = b * l
        mid = a * l + low // 65536
        mid2 = b * h + mid % 65536
        return a * h + mid // 65536 + mid2 // 65536, (mid2 % 65536) * 65536 + low % 65536

    block = e // 8
    x = [block % 2 ** 32, block // 2 ** 32, torch.tensor(offset % 2 ** 32, device=DEV),
         torch.tensor(offset // 2 ** 32, device=DEV)]
    for i in range(10):
        key = ((seed % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32)
        (h0, l0), (h2, l2) = times(x[0], 0xD2511F53), times(x[2], 0xCD9E8D57)
        x = [torch.bitwise_xor(torch.bitwise_xor(h2, x[1]), key[0]), l2,
             torch.bitwise_xor(torch.bitwise_xor(h0, x[3]), key[1]), l0]
    which = e % 8
    word = torch.where(which < 4, torch.where(which < 2, x[0], x[1]), torch.where(which < 6, x[2], x[3]))
    return torch.where(which % 2 == 0, word % 65536, word // 65536)


def _exact_dropout(s):
    c = s["case"]
    n, f = c["n"], 1 if c["rows"] else c["f"]
    limit = round(65536 * c["p"])
    stays = torch.empty(n, f, dtype=torch.bool, device=DEV)
    rows = max(1, (1 << 25) // f)
    for i in range(0, n, rows):  # a slice of the rows at a time: every element has a block here
        j = min(n, i + rows)
        who = torch.arange(i, j, device=DEV) if s["ids"] is None else s["ids"][i:j].long()
        e = who.view(-1, 1) * f + torch.arange(f, device=DEV)
        stays[i:j] = _exact_words(e, s["seed"], s["offset"]) >= limit
    factor = stays.double() / (1 - limit / 65536)
    out = s["x"].double() * factor
    if s["residual"] is not None:
        out += s["residual"].double()
    r = dict(out=out)
    if c["train"]:
        r["dx"] = s["dout"].double() * factor
    return r


def _exact_route(s):
    c = s["case"]
    n, e, k = c["n"], c["experts"], c["k"]
    l = s["logits"].double()
    live = torch.ones(n, dtype=torch.bool, device=DEV) if s["mask"] is None else s["mask"].clone()
    l = l.masked_fill(~live[:, None], 0.0)
    lse = torch.logsumexp(l, 1)
    p = (l - lse[:, None]).exp() * live[:, None]
    # the rank of a logit: how many are larger, or equal and before it
    left, rank = l.clone(), torch.full((n, e), e, device=DEV)
    for j in range(k):
        first = left.eq(left.amax(1, keepdim=True)).cumsum(1).lt(1)
        at = first.sum(1, keepdim=True)
        rank.scatter_(1, at, j)
        left.scatter_(1, at, -torch.inf)
    sel = (rank < k) & live[:, None]
    order = rank.argsort(1)[:, :k]
    pk = p.gather(1, order)
    weight = torch.where(live[:, None], pk / pk.sum(1, keepdim=True), 0.0)
    m = int(live.sum())
    chosen = sel.sum(0)
    share = chosen.double() / max(1, int(chosen.sum()))
    mean = p.sum(0) / max(m, 1)
    r = dict(idx=torch.where(live[:, None], order, -1).int(), weight=weight,
             counts=torch.cat([chosen.int(), torch.tensor([m], dtype=torch.int32, device=DEV)]),
             loss=torch.stack([e * share.dot(mean), (lse.square() * live).sum() / max(m, 1)]))
    if c["train"]:
        dw = s["dweight"].double()
        a = s["dloss"].double()
        # softmax over the chosen, softmax over all, and the square of logsumexp
        g = torch.zeros(n, e, dtype=torch.float64, device=DEV)
        g.scatter_(1, order, weight * dw - weight * (weight * dw).sum(1, keepdim=True))
        g += p * (a[0] * e / max(m, 1)) * (share - (p @ share)[:, None])
        g += p * (2 * a[1] / max(m, 1)) * lse[:, None]
        r["dlogits"] = torch.where(live[:, None], g, 0.0)
    return r


def _exact_fp4(x):
    """By the nearest of the sixteen values, on the CPU's definition of a power of two."""
    n, k = x.shape
    pad = -k % 32
    v = torch.nn.functional.pad(x.double(), (0, pad)).view(n, -1, 32)
    top = v.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -125))) - 2)
    scale = torch.where(top / scale >= 8, scale * 2, torch.where(top / scale < 4, scale / 2, scale))
    scale = scale.clamp(min=2.0 ** -127)
    a = v / scale
    m = a.abs()
    # halfway points between neighbours: those of an even lower neighbour belong to it
    val = 0.5 * ((m > 0.25).double() + (m >= 0.75).double() + (m > 1.25).double() + (m >= 1.75).double())
    val += (m > 2.5).double() + (m >= 3.5).double() + 2 * (m > 5).double()
    return (torch.copysign(val, a) * scale).view(n, -1)[:, :k]


def _exact_product(s):
    c, at = s["case"], s["offsets"]
    x = _exact_fp4(s["x"])
    out = torch.empty(c["n"], c["fo"], dtype=torch.float64, device=DEV)
    for t in range(c["types"]):
        if at[t] == at[t + 1]:
            continue
        codes = s["codes"][t].long()
        b = torch.stack((codes % 16, codes // 16), -1).view(c["fo"], -1)
        exponent, mantissa = b % 8 // 2, b % 2
        w = torch.where(exponent > 0, (2 + mantissa) * 2.0 ** (exponent - 2), mantissa / 2)
        w = w.double() * (1 - 2 * (b // 8))
        w = w.view(c["fo"], -1, 32) * torch.exp2(s["scales"][t].double() - 127).unsqueeze(-1)
        torch.matmul(x[at[t]:at[t + 1]], w.view(c["fo"], -1)[:, :c["k"]].t().contiguous(),
                     out=out[at[t]:at[t + 1]])
    return dict(out=out)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        return _exact_norm(s)
    if kind == "dropout":
        return _exact_dropout(s)
    if kind == "route":
        return _exact_route(s)
    if kind == "quantize":
        return dict(values=_exact_fp4(s["x"]))
    return _exact_product(s)
