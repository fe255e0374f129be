"""Performance cases of the way from a layer's last activations to the next token.

``add_norm`` adds the residual and divides each row by its root mean square,
``add_norm_int8`` gives that row in 8 bits with a scale, ``norm_grad`` is the
backward pass of the norm; ``quantise_rows`` gives any rows in 8 bits,
``project_int8`` multiplies rows and weights of 8 bits, with a scale for each
row and each channel; ``sample_logits`` picks the next token of each row by the
row's uniform number, among the likeliest under a temperature, a count, a share
of the probability and a floor.

``listed`` names the cases, ``draw`` gives more of the same ranges, ``prepare``
makes what a program holds before the call, ``run`` is the call (the plain form
in elementary torch operations where ``own`` is false), ``work`` what it cannot
do without and ``exact`` the result in 64 bits.

The definitions:
  * norm: h = x + residual, y = h * weight / sqrt(mean(h^2) + eps);
  * 8 bits: scale = max |y| / 127 of the row, q = y / scale, to the nearest
    whole number, halves to the even one;
  * product: out[m][n] = (sum over k of q[m][k] weight[n][k]) * scale[m] *
    weight_scale[n] + bias[n];
  * sampling: w = exp((x - max x) / temperature).  Tokens in the order of
    falling logits, equal ones by number: the first top_k of them stay, of
    those the fewest whose weights reach the share top_p, of those the ones of
    at least min_p times the largest weight.  The token is the first, by
    number, up to which the weights that stay sum to more than u times all of
    them; its probability is its share.  Without a temperature above 0 it is the
    first of the largest logits, with probability 1.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def _norm(N, D, dtype, weight, residual, bits8=False, name=None):
    return dict({"name": name} if name else {}, op="norm", N=N, D=D, dtype=dtype, weight=weight,
                residual=residual, bits8=bits8)


def _grad(N, D, dtype, weight, residual, name=None):
    return dict({"name": name} if name else {}, op="grad", N=N, D=D, dtype=dtype, weight=weight,
                residual=residual)


def _project(M, N, K, dtype, rows, bias, name=None):
    """``rows``: the activations come in ``dtype`` and are quantised on the way."""
    return dict({"name": name} if name else {}, op="project", M=M, N=N, K=K, dtype=dtype,
                rows=rows, bias=bias)


def _sample(B, V, dtype, top_k, top_p, min_p, name=None):
    """``top_k``: the largest of the rows' (0: none has one)."""
    return dict({"name": name} if name else {}, op="sample", B=B, V=V, dtype=dtype, top_k=top_k,
                top_p=top_p, min_p=min_p)


def listed():
    return [
        # a decoding step: one token of each of 64 sequences, for an 8-bit product
        _norm(64, 1024, "bf16", "bf16", True, True, name="norm8-decode"),
        # a training step's residual stream
        _norm(16_384, 4096, "bf16", "bf16", True, name="norm-train"),
        # a long prompt, rows that are no multiple of the vector
        _norm(8192, 5003, "f16", "f32", False, True, name="norm8-prompt"),
        # a small model's backward pass in 32 bits
        _grad(300, 1000, "f32", "f32", False, name="grad-small"),
        # a training step's backward pass, the residual's gradient on the way
        _grad(32_768, 2048, "bf16", "f32", True, name="grad-train"),
        # one token of one sequence through a square layer: latency
        _project(1, 4096, 4096, "bf16", True, False, name="project-one"),
        # an odd layer over a short prompt
        _project(333, 1003, 1001, "f16", False, True, name="project-odd"),
        # 64 sequences' logits: the table of words is read once
        _project(64, 100_000, 4096, "bf16", True, False, name="project-logits"),
        # a long prompt through a wide layer
        _project(8192, 8192, 4096, "bf16", True, False, name="project-prompt"),
        # one sequence's next token
        _sample(1, 32_768, "bf16", 50, True, False, name="sample-one"),
        # a serving batch, each row with its own settings
        _sample(256, 100_000, "bf16", 1000, True, True, name="sample-batch"),
        # a batch of 32-bit logits cut by probability alone
        _sample(64, 49_999, "f32", 0, True, False, name="sample-share"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly round, else anything."""
    d = _log(rng, lo, hi)
    return d // 64 * 64 if d >= 128 and rng.random() < 0.6 else d


def draw(rng):
    op = rng.choice(("norm", "grad", "project", "project", "sample", "sample"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    if op in ("norm", "grad"):
        D = _width(rng, 64, 8192)
        N = _log(rng, 1, min(32_768, 67_000_000 // D))
        weight, residual = rng.choice(("f32", dtype)), rng.random() < 0.6
        if op == "grad":
            return _grad(N, D, dtype, weight, residual)
        return _norm(N, D, dtype, weight, residual, rng.random() < 0.5)
    if op == "project":
        K = _width(rng, 64, 8192)
        N = _width(rng, 64, min(100_000, 410_000_000 // K))
        M = _log(rng, 1, min(8192, 67_000_000 // N, 270_000_000_000 // (N * K)))
        return _project(M, N, K, dtype, rng.random() < 0.5, rng.random() < 0.5)
    B = _log(rng, 1, 256)
    V = _log(rng, 300, min(131_072, 25_600_000 // B))
    return _sample(B, V, dtype, rng.choice((0, _log(rng, 1, min(V, 5000)))), rng.random() < 0.7,
                   rng.random() < 0.4)


def _normal(shape, sd, dtype, g):
    return (torch.randn(shape, device="cuda", generator=g) * sd).to(DTYPES[dtype])


def _uniform(shape, lo, hi, g):
    return torch.rand(shape, device="cuda", generator=g) * (hi - lo) + lo


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st = dict(case)
    if case["op"] in ("norm", "grad"):
        N, D, dtype = case["N"], case["D"], case["dtype"]
        st["x"] = _normal((N, D), 1.3, dtype, g)
        st["w"] = (1 + 0.2 * torch.randn(D, device="cuda", generator=g)).to(DTYPES[case["weight"]])
        if case["op"] == "grad":
            st["dy"] = _normal((N, D), 1e-2, dtype, g)
        if case["residual"]:
            st["res"] = _normal((N, D), 1e-2 if case["op"] == "grad" else 2.0, dtype, g)
    elif case["op"] == "project":
        M, N, K = case["M"], case["N"], case["K"]
        # a few channels are much larger than the others, as activations' are
        loud = 1 + 9 * (torch.rand(K, device="cuda", generator=g) < 0.01)
        x = torch.randn((M, K), device="cuda", generator=g) * loud
        if case["rows"]:
            st["x"] = x.to(DTYPES[case["dtype"]])
        else:
            top = x.abs().amax(1, keepdim=True)
            st["q"] = torch.round(x * (127 / top)).to(torch.int8)
            st["s"] = (top / 127).squeeze(1)
        w = torch.randn((N, K), device="cuda", generator=g)
        top = w.abs().amax(1, keepdim=True)
        st["qw"] = torch.round(w * (127 / top)).to(torch.int8)
        st["sw"] = (top / (127 * math.sqrt(K))).squeeze(1)
        if case["bias"]:
            st["b"] = torch.randn(N, device="cuda", generator=g) * 0.1
    else:
        _prepare_sample(st, g)
    return st


def _prepare_sample(st, g):
    B, V = st["B"], st["V"]
    # most tokens are unlikely, about twenty of each row are likely
    x = torch.randn((B, V), device="cuda", generator=g) * 2.2
    few = min(20, V)
    stretch = V // few
    at = torch.randint(0, stretch, (B, few), device="cuda", generator=g)
    x.scatter_(1, at + torch.arange(few, device="cuda") * stretch, _uniform((B, few), 4.0, 12.0, g))
    # a grammar or a bias has taken some out
    x[torch.rand((B, V), device="cuda", generator=g) < 0.05] = -math.inf
    x[:, V // 2] = x[:, V // 3]
    if B > 4:
        x[3] = -math.inf  # a row with nothing left
    st["logits"] = x.to(DTYPES[st["dtype"]])
    st["u"] = torch.rand(B, device="cuda", generator=g)
    t = _uniform((B,), 0.3, 1.4, g)
    st["temperature"] = torch.where(torch.rand(B, device="cuda", generator=g) < 0.1, 0.0, t)
    if st["top_k"]:
        k = torch.exp(_uniform((B,), 0.0, math.log(st["top_k"] + 1), g)).int()
        off = torch.rand(B, device="cuda", generator=g) < 0.1
        st["k"] = torch.where(off, torch.zeros_like(k), k.clamp(1, st["top_k"]))
    if st["top_p"]:
        p = _uniform((B,), 0.5, 1.0, g)
        st["p"] = torch.where(torch.rand(B, device="cuda", generator=g) < 0.15, 1.0, p)
    if st["min_p"]:
        m = torch.exp(_uniform((B,), math.log(1e-4), math.log(0.2), g))
        st["m"] = torch.where(torch.rand(B, device="cuda", generator=g) < 0.3, 0.0, m)


# ---- the framework's operators


def _run_own(st):
    import paper_1505_03851_amd as lda
    if st["op"] == "norm":
        if not st["bits8"]:
            return lda.add_norm(st["x"], st["w"], EPS, residual=st.get("res"))
        q, scale, *h = lda.add_norm_int8(st["x"], st["w"], EPS, residual=st.get("res"))
        return (_values(q, scale), scale, *h)
    if st["op"] == "grad":
        return lda.norm_grad(st["dy"], st["x"], st["w"], EPS, residual_grad=st.get("res"))
    if st["op"] == "project":
        q, scale = lda.quantise_rows(st["x"]) if st["rows"] else (st["q"], st["s"])
        return lda.project_int8(q, scale, st["qw"], st["sw"], bias=st.get("b"),
                                dtype=DTYPES[st["dtype"]])
    return lda.sample_logits(st["logits"], st["u"], temperature=st["temperature"],
                             top_k=st.get("k"), top_p=st.get("p"), min_p=st.get("m"))


def _values(q, scale):
    """What 8-bit rows stand for."""
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    return torch.mul(q, scale[:, None], out=out)


# ---- the plain forms: elementary operations in 32 bits, one rounding at the end


def _plain_bits(y):
    """(q as float, scale): whether a value is next to a half is decided in 64 bits."""
    top = y.abs().amax(1, keepdim=True)
    q = torch.round(y.double() * 127 / torch.where(top > 0, top, 1.0).double())
    return q.float(), (top / 127).squeeze(1)


def _plain_norm(st):
    dtype = DTYPES[st["dtype"]]
    h = st["x"].float()
    if st["residual"]:
        h = h + st["res"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * st["w"].float()
    if st["bits8"]:
        q, scale = _plain_bits(y)
        out = (_values(q, scale), scale)
        return (*out, h.to(dtype)) if st["residual"] else out
    return (y.to(dtype), h.to(dtype)) if st["residual"] else y.to(dtype)


def _plain_grad(st):
    h, dy = st["x"].float(), st["dy"].float()
    r = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    unit = h * r
    d = dy * st["w"].float()
    dx = r * (d - unit * (d * unit).mean(1, keepdim=True))
    if st["residual"]:
        dx = dx + st["res"].float()
    return dx.to(DTYPES[st["dtype"]]), (dy * unit).sum(0)


def _plain_project(st):
    q, scale = _plain_bits(st["x"].float()) if st["rows"] else (st["q"].float(), st["s"])
    y = q @ st["qw"].float().t()
    y = y * scale[:, None] * st["sw"]
    if st["bias"]:
        y = y + st["b"]
    return y.to(DTYPES[st["dtype"]])


def _plain_sample(st):
    x = st["logits"].double()
    B, V = x.shape
    t = st["temperature"].double()[:, None]
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    top = x[:, :1]
    w = torch.where(x == top, 1.0, torch.exp((x - top) / t))
    w = torch.where(x == -math.inf, 0.0, w)
    if "k" in st:
        k = st["k"][:, None]
        place = torch.arange(V, device="cuda")[None, :]
        w = torch.where((k <= 0) | (place < k), w, 0.0)
    if "p" in st:
        p = st["p"].double()[:, None]
        upto = torch.cumsum(w, 1)
        w = torch.where((p >= 1) | (upto - w < p * upto[:, -1:]), w, 0.0)
    if "m" in st:
        w = torch.where(w < st["m"].double()[:, None], 0.0, w)
    w = torch.zeros_like(w).scatter_(1, order, w)  # by number again
    upto = torch.cumsum(w, 1)
    total = upto[:, -1:]
    z = (upto <= st["u"].double()[:, None] * total).sum(1, keepdim=True).clamp_max(V - 1)
    z = torch.where(t > 0, z, order[:, :1])
    prob = torch.where(t > 0, w.gather(1, z) / total, 1.0)
    none = top == -math.inf
    return (torch.where(none, -1, z).int().squeeze(1),
            torch.where(none, 0.0, prob).float().squeeze(1))


def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "norm":
        return _plain_norm(st)
    if st["op"] == "grad":
        return _plain_grad(st)
    return _plain_project(st) if st["op"] == "project" else _plain_sample(st)


# ---- what a pass cannot do without


def work(case):
    if case["op"] in ("norm", "grad"):
        N, D, e = case["N"], case["D"], SIZE[case["dtype"]]
        b = SIZE[case["weight"]] * D + e * N * D
        if case["op"] == "grad":
            return {"bytes": b + e * N * D * (3 if case["residual"] else 2) + 4 * D,
                    "flops": 10 * N * D}
        b += 2 * e * N * D if case["residual"] else 0
        return {"bytes": b + (N * D + 4 * N if case["bits8"] else e * N * D), "flops": 5 * N * D}
    if case["op"] == "project":
        M, N, K, e = case["M"], case["N"], case["K"], SIZE[case["dtype"]]
        b = (e * M * K if case["rows"] else M * K + 4 * M) + N * K + 4 * N + e * M * N
        return {"bytes": b + (4 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    B, V = case["B"], case["V"]
    each = 16 + sum(4 for k in ("top_k", "top_p", "min_p") if case[k])
    return {"bytes": SIZE[case["dtype"]] * B * V + each * B, "flops": 4 * B * V}


# ---- the results in 64 bits


def _exact_bits(y):
    top = y.abs().max(dim=1).values
    step = top / 127
    return torch.round(127 * y / torch.where(top == 0, 1.0, top)[:, None]), step


def _exact_rows(case, st):
    h = st["x"].double()
    D = h.shape[1]
    if case["op"] == "norm" and case["residual"]:
        h = h + st["res"].double()
    size = torch.sqrt(h.square().sum(1) / D + EPS)
    unit = h / size[:, None]
    w = st["w"].double()
    if case["op"] == "grad":
        dy = st["dy"].double()
        along = (dy * w * unit).sum(1) / D
        dx = (dy * w - unit * along[:, None]) / size[:, None]
        if case["residual"]:
            dx += st["res"].double()
        return dx, torch.sum(dy.mul_(unit), dim=0)
    y = unit * w
    out = (y,)
    if case["bits8"]:
        q, step = _exact_bits(y)
        out = (q * step[:, None], step)
    if case["residual"]:
        out = (*out, h)
    return out if len(out) > 1 else out[0]


def _exact_sample(st):
    x = st["logits"].double().cpu().numpy()
    B, V = x.shape
    z, prob = np.full(B, -1, dtype=np.int32), np.zeros(B)

    def setting(name, b, off):
        return float(st[name][b]) if name in st else off

    for b in range(B):
        best = int(np.argmax(x[b]))
        if x[b, best] == -math.inf:
            continue
        t = setting("temperature", b, 1.0)
        if t == 0:
            z[b], prob[b] = best, 1.0
            continue
        w = np.exp((x[b] - x[b, best]) / t)
        order = np.argsort(-x[b], kind="stable")
        k = int(setting("k", b, 0))
        if k > 0:
            order = order[:k]
        p = setting("p", b, 1.0)
        if p < 1:
            sums = np.cumsum(w[order])
            order = order[:int(np.searchsorted(sums, p * sums[-1])) + 1]
        order = order[w[order] >= setting("m", b, 0.0)]
        stay = np.sort(order)
        sums = np.cumsum(w[stay])
        i = min(int(np.searchsorted(sums, float(st["u"][b]) * sums[-1], side="right")),
                len(stay) - 1)
        z[b], prob[b] = stay[i], w[stay[i]] / sums[-1]
    return torch.from_numpy(z), torch.from_numpy(prob)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("norm", "grad"):
        return _exact_rows(case, st)
    if case["op"] == "sample":
        return _exact_sample(st)
    q, step = _exact_bits(st["x"].double()) if case["rows"] else (st["q"].double(),
                                                                  st["s"].double())
    y = torch.mm(q, st["qw"].double().t()) * step[:, None] * st["sw"].double()
    return y + st["b"].double() if case["bias"] else y
