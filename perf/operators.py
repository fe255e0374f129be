"""Performance cases of the operators around a language model's tokens.

What a model of token sequences does with its tokens, first and last in every
step: ``embed`` looks their rows up in a table (scaled, and dropped out by the
counter-based generator), ``embed_grad`` sums the gradient back by sorted
tokens, ``dropout`` is the same generator over any activations (and over their
gradients: the operator is its own backward pass), ``penalise_logits`` applies
the penalties for repeated tokens, biases and grammar masks, and
``draw_logits`` draws the next token of every sequence from logits under those
rules, a temperature and a floor on the probability.

``listed`` names the cases, ``draw`` gives more of the same ranges, ``prepare``
makes what a program holds before the call, ``run`` is the call (the plain form
in elementary torch operations where ``own`` is false), ``work`` what it cannot
do without and ``exact`` the result in 64 bits.

The random numbers are Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC 2011)
under the key (seed mod 2**32, seed >> 32):
  * dropout: eight columns share the counter (col // 8, row, step, 1); column
    c takes half c % 2 (low first) of output word (c % 8) // 2 and is kept if
    it is at least q = round(65536 p); what is kept is multiplied by
    65536 / (65536 - q), the reciprocal of the probability of keeping it;
  * the draw: y = word 0 of the counter (i, position, 0, 2) for group i of
    1,024 tokens and (v, position, 0, 3) for token v, and the exponential
    variate -log(1 - (y + 1/2) / 2**32).  The row's group is the one with the
    smallest variate / (sum of weights), its token the one of that group with
    the smallest variate / weight.
"""
from __future__ import annotations

import functools
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
GROUP = 1024
M32 = 0xFFFFFFFF


def _embed(N, V, D, dtype, p=0.0, name=None):
    return dict({"name": name} if name else {}, op="embed", N=N, V=V, D=D, dtype=dtype, p=p)


def _grad(N, V, D, dtype, out, p=0.0, name=None):
    return dict({"name": name} if name else {}, op="embed_grad", N=N, V=V, D=D, dtype=dtype,
                out=out, p=p)


def _dropout(rows, D, dtype, p, name=None):
    return dict({"name": name} if name else {}, op="dropout", N=rows, D=D, dtype=dtype, p=p)


def _logits(op, B, V, dtype, history, bias, mask, min_p=False, name=None):
    """``history``: the longest sequence so far (0: no penalties); ``bias``:
    none, shared (one row for the batch) or rows."""
    return dict({"name": name} if name else {}, op=op, B=B, V=V, dtype=dtype, history=history,
                bias=bias, mask=mask, min_p=min_p)


def listed():
    return [
        # a decoding step's lookup: one token of each of 64 sequences
        _embed(64, 32_768, 1024, "bf16", name="embed-decode"),
        # a training step's lookup with embedding dropout
        _embed(16_384, 100_000, 4096, "bf16", p=0.1, name="embed-train"),
        # a small model's gradient, rows that are no multiple of the vector
        _grad(4096, 1024, 1000, "f32", "f32", name="grad-tiny"),
        # a training step's gradient into a 32-bit master gradient
        _grad(32_768, 50_000, 2048, "bf16", "f32", p=0.1, name="grad-train"),
        # the medium corpus in one pass: many tokens of frequent words
        _grad(1 << 20, 32_768, 256, "bf16", "bf16", name="grad-corpus1M"),
        # one sequence's activations, rows of an odd length
        _dropout(300, 1001, "f16", 0.2, name="dropout-small"),
        # a training step's activations (or their gradient)
        _dropout(32_768, 4096, "bf16", 0.1, name="dropout-train"),
        # one sequence's penalties: latency
        _logits("penalise", 1, 32_768, "f32", 512, "none", False, name="penalise-one"),
        # a serving batch under penalties, a bias and grammars
        _logits("penalise", 256, 100_000, "bf16", 4096, "shared", True, name="penalise-batch"),
        # one sequence's next token
        _logits("draw", 1, 32_768, "bf16", 512, "none", False, name="draw-one"),
        # a serving batch with everything on
        _logits("draw", 64, 100_000, "bf16", 8192, "shared", True, True, name="draw-batch"),
        # a wide batch of plain draws
        _logits("draw", 256, 49_999, "f32", 0, "none", False, name="draw-wide"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("embed", "embed_grad", "dropout", "penalise", "draw"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    e = SIZE[dtype]
    if op in ("embed", "embed_grad", "dropout"):
        p = rng.choice((0.0, 0.1, rng.uniform(0.01, 0.6)))
        D = _log(rng, 64, 8192)
        if rng.random() < 0.6:  # widths are mostly round
            D = 1 << max(6, D.bit_length() - 1)
        V = min(_log(rng, 1000, 100_000), 400_000_000 // (4 * D))
        N = _log(rng, 1, min(1 << 20, 130_000_000 // (e * D)))
        if op == "embed":
            return _embed(N, V, D, dtype, p)
        if op == "dropout":
            return _dropout(N, D, dtype, p or 0.3)
        return _grad(N, V, D, dtype, rng.choice(("f32", dtype)), p)
    B = _log(rng, 1, 256)
    V = _log(rng, 300, min(131_072, 25_000_000 // B))
    return _logits(op, B, V, dtype, rng.choice((0, _log(rng, 1, 8192))),
                   rng.choice(("none", "shared", "rows")), rng.random() < 0.5,
                   op == "draw" and rng.random() < 0.5)


def _zipf_ids(N, V, g):
    w = torch.arange(1, V + 1, dtype=torch.float64, device="cuda").reciprocal()
    cdf = (w / w.sum()).cumsum(0)
    ids = torch.searchsorted(cdf, torch.rand(N, dtype=torch.float64, device="cuda", generator=g))
    return ids.clamp_max(V - 1).int()


def _normal(shape, sd, dtype, g):
    return (torch.randn(shape, device="cuda", generator=g) * sd).to(DTYPES[dtype])


def _uniform(shape, lo, hi, g):
    return torch.rand(shape, device="cuda", generator=g) * (hi - lo) + lo


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st = dict(case, seed=seed * 0x9E3779B97F4A7C15 % (1 << 63), step=seed % 100_000)
    if case["op"] in ("embed", "embed_grad"):
        st["ids"] = _zipf_ids(case["N"], case["V"], g)
        st["scale"] = math.sqrt(case["D"])
    if case["op"] == "embed":
        st["table"] = _normal((case["V"], case["D"]), 0.02, case["dtype"], g)
    elif case["op"] == "embed_grad":
        st["grad"] = _normal((case["N"], case["D"]), 1e-3, case["dtype"], g)
    elif case["op"] == "dropout":
        st["x"] = _normal((case["N"], case["D"]), 1.0, case["dtype"], g)
    else:
        _prepare_logits(st, g)
    return st


def _places(B, V, few, g):
    """[B][few] distinct tokens of each row: one from each stretch of V // few."""
    stretch = V // few
    at = torch.randint(0, stretch, (B, few), device="cuda", generator=g)
    return at + torch.arange(few, device="cuda") * stretch


def _prepare_logits(st, g):
    B, V = st["B"], st["V"]
    # most tokens are unlikely, about twenty of each row are likely
    x = torch.randn((B, V), device="cuda", generator=g) * 2.2
    few = min(20, V)
    likely = _places(B, V, few, g)
    x.scatter_(1, likely, _uniform((B, few), 5.0, 14.0, g))
    st["logits"] = x.to(DTYPES[st["dtype"]])
    if st["history"]:
        cap = st["history"]
        h = _zipf_ids(B * cap, V, g).view(B, cap)
        again = torch.rand((B, cap), device="cuda", generator=g) < 0.02
        pick = torch.randint(0, few, (B, cap), device="cuda", generator=g)
        st["tokens"] = torch.where(again, likely.gather(1, pick).int(), h).contiguous()
        st["lengths"] = torch.randint((cap + 1) // 2, cap + 1, (B,), device="cuda", generator=g,
                                      dtype=torch.int32)
        st["prompt"] = (st["lengths"] * torch.rand(B, device="cuda", generator=g)).int()
        st["repetition"] = _uniform((B,), 1.0, 1.3, g)
        st["frequency"] = _uniform((B,), 0.0, 0.5, g)
        st["presence"] = _uniform((B,), 0.0, 0.5, g)
    if st["bias"] != "none":
        b = torch.zeros((1 if st["bias"] == "shared" else B, V), device="cuda")
        at = _places(b.shape[0], V, min(300, V), g)
        b.scatter_(1, at, _uniform(at.shape, -8.0, 4.0, g))
        b[:, :2] = -math.inf  # two tokens that are never wanted
        st["bias_rows"] = b[0].contiguous() if st["bias"] == "shared" else b
    if st["mask"]:
        # a row's grammar allows a share of the words, from all down to none
        share = torch.rand((B, 1), device="cuda", generator=g) ** 2
        share[::7] = 1.1
        if B > 4:
            share[3] = -1.0
        ok = torch.rand((B, V), device="cuda", generator=g) < share
        pad = torch.zeros((B, (V + 31) // 32 * 32), dtype=torch.int64, device="cuda")
        pad[:, :V] = ok
        bits = (pad.view(B, -1, 32) << torch.arange(32, device="cuda")).sum(2)
        st["mask_bits"] = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int()
    if st["op"] == "draw":
        st["seeds"] = torch.randint(0, (1 << 63) - 1, (B,), device="cuda", generator=g)
        st["position"] = torch.randint(0, 100_000, (B,), device="cuda", generator=g,
                                       dtype=torch.int32)
        t = _uniform((B,), 0.3, 1.4, g)
        st["temperature"] = torch.where(torch.rand(B, device="cuda", generator=g) < 0.15,
                                        torch.zeros_like(t), t)
        if st["min_p"]:
            m = _uniform((B,), 0.01, 0.2, g)
            st["floor"] = torch.where(torch.rand(B, device="cuda", generator=g) < 0.25,
                                      torch.zeros_like(m), m)


# ---- the framework's operators


def _rules(st):
    names = dict(history="tokens", lengths="lengths", prompt="prompt", repetition="repetition",
                 frequency="frequency", presence="presence", bias="bias_rows", mask="mask_bits")
    return {k: st[v] for k, v in names.items() if v in st}


def _run_own(st):
    import paper_1505_03851_amd as lda
    if st["op"] == "embed":
        return lda.embed(st["table"], st["ids"], scale=st["scale"], p=st["p"], seed=st["seed"],
                         step=st["step"])
    if st["op"] == "embed_grad":
        return lda.embed_grad(st["grad"], st["ids"], st["V"], scale=st["scale"], p=st["p"],
                              seed=st["seed"], step=st["step"], dtype=DTYPES[st["out"]])
    if st["op"] == "dropout":
        return lda.dropout(st["x"], st["p"], st["seed"], st["step"])
    if st["op"] == "penalise":
        return lda.penalise_logits(st["logits"], **_rules(st))
    return lda.draw_logits(st["logits"], st["seeds"], st["position"],
                           temperature=st["temperature"], min_p=st.get("floor"), **_rules(st))


# ---- the plain forms: elementary operations in 32 bits, one rounding at the end


def _philox(x0, x1, x2, x3, k0, k1):
    """The four output words; counters and keys are int64 tensors or numbers
    that broadcast (a 64-bit product wraps, its upper half is masked)."""
    def one(s, r):
        p0, p1 = s[0] * 0xD2511F53, s[2] * 0xCD9E8D57
        a, b = (k0 + r * 0x9E3779B9) & M32, (k1 + r * 0xBB67AE85) & M32
        return (((p1 >> 32) & M32) ^ s[1] ^ a, p1 & M32, ((p0 >> 32) & M32) ^ s[3] ^ b, p0 & M32)
    return functools.reduce(one, range(10), (x0, x1, x2, x3))


def _kept(rows, D, st):
    """[rows][D] truth values, and the factor of what is kept."""
    q = min(65535, round(65536 * st["p"]))
    row = torch.arange(rows, device="cuda")[:, None]
    col = torch.arange((D + 7) // 8, device="cuda")[None, :]
    zero = torch.zeros_like(row + col)
    w = torch.stack(_philox(col + zero, row + zero, zero + st["step"], zero + 1,
                            st["seed"] & M32, st["seed"] >> 32), 2)
    half = torch.stack((w & 0xFFFF, w >> 16), 3).view(rows, -1)[:, :D]
    return half >= q, 65536.0 / (65536 - q)


def _plain_rows(x, scale, st):
    """``x`` (32-bit rows) scaled and dropped out."""
    if not st["p"]:
        return x * scale
    keep, more = _kept(x.shape[0], x.shape[1], st)
    return torch.where(keep, x * (scale * more), 0.0)


def _plain_penalise(st):
    """The logits under the rules, float32 [B][V]."""
    x = st["logits"].float()
    B, V = x.shape
    if "tokens" in st:
        cap = st["tokens"].shape[1]
        at = torch.arange(cap, device="cuda")[None, :]
        there = at < st["lengths"][:, None]
        made = there & (at >= st["prompt"][:, None])
        cell = st["tokens"].long() + torch.arange(B, device="cuda")[:, None] * V
        count = [torch.zeros(B * V, dtype=torch.int32, device="cuda").index_add_(
            0, cell.view(-1), m.view(-1).int()).view(B, V) for m in (there, made)]
        r = st["repetition"][:, None]
        x = torch.where(count[0] > 0, torch.where(x > 0, x / r, x * r), x)
        x = x - st["frequency"][:, None] * count[1]
        x = x - torch.where(count[1] > 0, st["presence"][:, None], 0.0)
    if "bias_rows" in st:
        x = x + st["bias_rows"]
    if "mask_bits" in st:
        bit = torch.arange(V, device="cuda")
        ok = (st["mask_bits"][:, bit >> 5] >> (bit & 31)) & 1
        x = torch.where(ok == 1, x, -math.inf)
    return x


def _variates(index, st, domain):
    """-log(1 - u) of the counters (index, position, 0, domain), float32."""
    zero = torch.zeros_like(index)
    key = st["seeds"][:, None]
    y = _philox(index, zero + st["position"][:, None], zero, zero + domain, (key & M32) + zero,
                ((key >> 32) & M32) + zero)[0]
    u = (y.float() * 2.0 ** -32 + 2.0 ** -33).clamp_max(1 - 2.0 ** -24)
    return -torch.log1p(-u)


def _first(key):
    """The lowest index of each row's smallest value."""
    i = torch.arange(key.shape[1], device="cuda")[None, :]
    low = torch.where(key == key.amin(1, keepdim=True), i, key.shape[1] - 1)
    return low.amin(1, keepdim=True)


def _plain_draw(st):
    x = _plain_penalise(st)
    x = torch.where(torch.isnan(x), -math.inf, x)
    B, V = x.shape
    G = (V + GROUP - 1) // GROUP
    pad = torch.full((B, G * GROUP), -math.inf, device="cuda")
    pad[:, :V] = x
    top = pad.amax(1, keepdim=True)
    t = st["temperature"][:, None]
    if "floor" in st:
        keep = (pad == top) | ((pad - top) / t >= torch.log(st["floor"])[:, None])
        pad = torch.where(keep, pad, -math.inf)
    part = pad.view(B, G, GROUP)
    m = part.amax(2)
    w = torch.where(part == m[:, :, None], 1.0, torch.exp((part - m[:, :, None]) / t[:, :, None]))
    w = torch.where(part == -math.inf, 0.0, w)
    share = torch.where(m == top, 1.0, torch.exp((m - top) / t))
    share = torch.where(m == -math.inf, 0.0, share) * w.sum(2)
    zero = torch.zeros((B, 1), dtype=torch.int64, device="cuda")
    g = _first(_variates(torch.arange(G, device="cuda")[None, :] + zero, st, 2) / share)
    index = torch.arange(GROUP, device="cuda")[None, :] + g * GROUP
    mine = w.gather(1, g[:, :, None].expand(B, 1, GROUP)).squeeze(1)
    z = g * GROUP + _first(_variates(index, st, 3) / mine)
    z = torch.where(t > 0, z, _first(-pad))
    xz = pad.gather(1, z)
    prob = torch.where(xz == top, 1.0, torch.exp((xz - top) / t)) / share.sum(1, keepdim=True)
    prob = torch.where(t > 0, prob, 1.0)
    none = top == -math.inf
    return (torch.where(none, -1, z).int().squeeze(1),
            torch.where(none, 0.0, prob).squeeze(1))


def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "embed":
        return _plain_rows(st["table"][st["ids"].long()].float(), st["scale"], st).to(
            DTYPES[st["dtype"]])
    if st["op"] == "embed_grad":
        rows = _plain_rows(st["grad"].float(), st["scale"], st)
        total = torch.zeros((st["V"], st["D"]), device="cuda")
        return total.index_add_(0, st["ids"], rows).to(DTYPES[st["out"]])
    if st["op"] == "dropout":
        return _plain_rows(st["x"].float(), 1.0, st).to(st["x"].dtype)
    if st["op"] == "penalise":
        return _plain_penalise(st).to(st["logits"].dtype)
    return _plain_draw(st)


# ---- what a pass cannot do without


def work(case):
    if case["op"] == "dropout":
        n = case["N"] * case["D"]
        return {"bytes": 2 * SIZE[case["dtype"]] * n, "flops": n}
    if case["op"] in ("embed", "embed_grad"):
        N, V, D, e = case["N"], case["V"], case["D"], SIZE[case["dtype"]]
        if case["op"] == "embed_grad":
            return {"bytes": 4 * N + e * N * D + SIZE[case["out"]] * V * D, "flops": 2 * N * D}
        w = 1.0 / np.arange(1, V + 1, dtype=np.float64)
        used = float((1.0 - np.exp(N * np.log1p(-w / w.sum()))).sum())  # rows that occur
        return {"bytes": 4 * N + e * D * (used + N), "flops": N * D}
    B, V, e = case["B"], case["V"], SIZE[case["dtype"]]
    b = e * B * V
    if case["history"]:
        b += B * (20 + 3 * case["history"])  # three quarters of the longest, 4 bytes a token
    b += {"none": 0, "shared": 4 * V, "rows": 4 * B * V}[case["bias"]]
    if case["mask"]:
        b += B * ((V + 31) // 32 * 4)
    if case["op"] == "penalise":
        return {"bytes": b + e * B * V, "flops": 4 * B * V}
    return {"bytes": b + B * (24 + (4 if case["min_p"] else 0)), "flops": 8 * B * V}


# ---- the results in 64 bits


def _exact_philox(c0, c1, c2, c3, k0, k1):
    """Four uint64 arrays of 32-bit words, by numpy."""
    m, s = np.uint64(M32), np.uint64(32)
    x = [np.asarray(c).astype(np.uint64) for c in (c0, c1, c2, c3)]
    k0, k1 = np.asarray(k0).astype(np.uint64), np.asarray(k1).astype(np.uint64)
    for _ in range(10):
        lo, hi = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(hi >> s) ^ x[1] ^ k0, hi & m, (lo >> s) ^ x[3] ^ k1, lo & m]
        k0, k1 = (k0 + np.uint64(0x9E3779B9)) & m, (k1 + np.uint64(0xBB67AE85)) & m
    return x


def _exact_factor(rows, D, st):
    """float64 [rows][D]: what each element is multiplied by."""
    q = min(65535, int(math.floor(65536 * st["p"] + 0.5)))
    out = torch.ones((rows, D), dtype=torch.float64, device="cuda")
    if not q:
        return out
    cols = (D + 7) // 8
    step = max(1, (1 << 21) // cols)
    for r in range(0, rows, step):
        n = min(step, rows - r)
        words = _exact_philox(np.tile(np.arange(cols), (n, 1)), np.arange(r, r + n)[:, None],
                              st["step"], 1, st["seed"] & M32, st["seed"] >> 32)
        half = np.empty((n, cols, 8), dtype=np.uint16)
        for j, y in enumerate(words):
            half[:, :, 2 * j] = y & np.uint64(0xFFFF)
            half[:, :, 2 * j + 1] = y >> np.uint64(16)
        keep = torch.from_numpy(half.reshape(n, -1)[:, :D] >= q).cuda()
        out[r:r + n] = keep.double() * (65536.0 / (65536 - q))
    return out


def _exact_logits(st):
    x = st["logits"].double()
    B, V = x.shape
    for b in range(B):
        if "tokens" in st:
            n, first = int(st["lengths"][b]), int(st["prompt"][b])
            seq = st["tokens"][b, :n].long()
            seen = torch.bincount(seq, minlength=V) > 0
            made = torch.bincount(seq[first:], minlength=V).double()
            r, f, p = (st[k][b].double() for k in ("repetition", "frequency", "presence"))
            x[b] = torch.where(seen, torch.where(x[b] > 0, x[b] / r, x[b] * r), x[b])
            x[b] -= f * made + p * (made > 0)
        if "bias_rows" in st:
            rows = st["bias_rows"]
            x[b] += (rows if rows.dim() == 1 else rows[b]).double()
        if "mask_bits" in st:
            words = st["mask_bits"][b].cpu().numpy().view(np.uint8)
            ok = np.unpackbits(words, bitorder="little")[:V].astype(bool)
            x[b][torch.from_numpy(~ok).cuda()] = -math.inf
    return x


def _exact_draw(st):
    x = _exact_logits(st).cpu().numpy()
    B, V = x.shape
    z, prob = np.full(B, -1, dtype=np.int32), np.zeros(B)
    key = st["seeds"].cpu().numpy().astype(np.uint64)
    pos = st["position"].cpu().numpy()
    temp = st["temperature"].cpu().numpy().astype(np.float64)
    floor = st["floor"].cpu().numpy().astype(np.float64) if "floor" in st else np.zeros(B)

    def variates(index, b, domain):
        y = _exact_philox(index, int(pos[b]), 0, domain, key[b] & np.uint64(M32),
                          key[b] >> np.uint64(32))[0]
        return -np.log1p(-(y.astype(np.float64) + 0.5) * 2.0 ** -32)

    for b in range(B):
        top = x[b].max()
        if top == -math.inf:
            continue
        if temp[b] == 0:
            z[b], prob[b] = int(np.argmax(x[b])), 1.0
            continue
        w = np.exp((x[b] - top) / temp[b])
        w[w < floor[b]] = 0.0
        starts = np.arange(0, V, GROUP)
        mass = np.add.reduceat(w, starts)
        with np.errstate(divide="ignore"):
            g = int(np.argmin(variates(np.arange(len(starts)), b, 2) / mass))
            at = np.arange(g * GROUP, min(V, (g + 1) * GROUP))
            z[b] = at[int(np.argmin(variates(at, b, 3) / w[at]))]
        prob[b] = w[z[b]] / mass.sum()
    return torch.from_numpy(z), torch.from_numpy(prob)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "embed":
        x = st["table"][st["ids"].long()].double() * st["scale"]
        return x * _exact_factor(case["N"], case["D"], st)
    if case["op"] == "embed_grad":
        x = st["grad"].double() * _exact_factor(case["N"], case["D"], st) * st["scale"]
        out = torch.zeros((case["V"], case["D"]), dtype=torch.float64, device="cuda")
        return out.index_add_(0, st["ids"], x)
    if case["op"] == "dropout":
        return st["x"].double() * _exact_factor(case["N"], case["D"], st)
    return _exact_logits(st) if case["op"] == "penalise" else _exact_draw(st)
