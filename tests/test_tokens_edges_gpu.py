"""The token operators at the edges of their ranges, against the oracle in 64
bits or against the same call away from the edge.  Tolerances are those of
test_tokens_gpu.py."""
import numpy as np
import pytest

from oracle import tokens as ref
from test_tokens_gpu import EPS, TYPES, _close, _gpu, _lda, _np, _rounded, _torch_type

pytestmark = pytest.mark.gpu


# ---- the embedding's gradient: tables smaller than a sorting launch's shares


@pytest.mark.parametrize("dtype,V,D", [
    ("float32", 1, 1), ("float32", 4, 1), ("float32", 1, 4), ("float32", 2, 2), ("float32", 5, 1),
    ("bfloat16", 8, 1), ("bfloat16", 2, 4), ("bfloat16", 3, 3), ("float16", 1, 8), ("float16", 1, 1)])
@pytest.mark.parametrize("N", [200, 4096, 4097, 5000, 70_001])
def test_embed_grad_into_a_few_bytes(dtype, V, D, N):
    """Rows without tokens are zero, whatever the memory held."""
    import torch
    lda = _lda()
    g = np.random.default_rng([V, D, N])
    grad = _rounded(g.normal(0, 1, (N, D)), dtype)
    # no token of any word; of every word but the middle one; of every word
    every = g.integers(0, V, N).astype(np.int32)
    for ids in (np.full(N, -1, dtype=np.int32), np.where(every == V // 2, V, every).astype(np.int32),
                every):
        want, size, tokens = ref.embed_grad(grad, ids, V, 1.0)
        out = torch.full((V, D), 5.0, device="cuda", dtype=_torch_type(dtype))
        lda.embed_grad(_gpu(grad, dtype), _gpu(ids), V, out=out)
        _close(_np(out), want, (tokens[:, None] + 2) * EPS * size, dtype, (dtype, V, D, N))
        # rows apart: what lies between them is kept
        wide = torch.full((V, D + 3), 5.0, device="cuda", dtype=_torch_type(dtype))
        lda.embed_grad(_gpu(grad, dtype), _gpu(ids), V, out=wide[:, 1:1 + D])
        assert torch.equal(wide[:, 1:1 + D], out)
        assert bool((wide[:, 0] == 5).all()) and bool((wide[:, 1 + D:] == 5).all())


# ---- the draw: tokens of the history past the row's end


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 300, 16_000, 20_001, 32_769, 33_001, 49_999, 131_071])
def test_draw_ignores_history_past_the_row(dtype, V):
    """Ids in [V, the next multiple of 1,024) under a negative repetition, which
    turns -inf into +inf: no token of that number is drawn."""
    import torch
    lda = _lda()
    B = 12
    g = np.random.default_rng(V)
    x = _rounded(g.normal(0, 2, (B, V)), dtype)
    x[:, :max(0, V - 40)] = -np.inf  # the last group is drawn
    past = np.arange(V, (V + 1023) // 1024 * 1024 + 3, dtype=np.int32)
    history = _gpu(np.tile(past, (B, 1)))
    n = torch.full((B,), len(past), dtype=torch.int32, device="cuda")
    seed, pos = torch.arange(B, device="cuda"), torch.arange(B, dtype=torch.int32, device="cuda")
    t = torch.full((B,), 0.9, device="cuda")
    t[::5] = 0.0
    minus = torch.full((B,), -1.5, device="cuda")
    want = lda.draw_logits(_gpu(x, dtype), seed, pos, t)
    for prompt in (None, n):
        got = lda.draw_logits(_gpu(x, dtype), seed, pos, t, history=history, lengths=n,
                              prompt=prompt, repetition=minus)
        assert int(got[0].max()) < V and int(got[0].min()) >= 0, (dtype, V)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (dtype, V)


# ---- rules: a prompt below zero is an empty one


@pytest.mark.parametrize("V", [700, 40_000])
def test_prompt_below_zero(V):
    import torch
    lda = _lda()
    B, cap = 6, 9000
    g = np.random.default_rng(V)
    x = g.normal(0, 3, (B, V))
    h = g.integers(0, V, (B, cap)).astype(np.int32)
    n = np.full(B, cap, dtype=np.int32)
    f32 = lambda a: _gpu(np.full(B, a, dtype=np.float32))  # noqa: E731
    rules = dict(history=_gpu(h), lengths=_gpu(n), repetition=f32(1.2), frequency=f32(0.3),
                 presence=f32(0.4))
    seed, pos = torch.arange(B, device="cuda"), torch.arange(B, dtype=torch.int32, device="cuda")
    want = lda.penalise_logits(_gpu(x, "float32"), **rules)
    drawn = lda.draw_logits(_gpu(x, "float32"), seed, pos, **rules)
    exact, size = ref.penalise(_rounded(x, "float32"), h, n, None, *(
        _np(rules[k]) for k in ("repetition", "frequency", "presence")))
    _close(_np(want), exact, 6 * EPS * size, "float32")
    for p in (-1, -9000, -2 ** 31 + 9001, -2 ** 31 + 5000, -2 ** 31 + 3, -2 ** 31):
        prompt = torch.full((B,), p, dtype=torch.int32, device="cuda")
        got = lda.penalise_logits(_gpu(x, "float32"), prompt=prompt, **rules)
        assert torch.equal(got, want), p
        z = lda.draw_logits(_gpu(x, "float32"), seed, pos, prompt=prompt, **rules)
        assert torch.equal(z[0], drawn[0]) and torch.equal(z[1], drawn[1]), p


# ---- the embedding's gradient of very long rows


def _marked(D, at, dtype, rows=1):
    import torch
    x = torch.zeros(rows, D, dtype=_torch_type(dtype), device="cuda")
    for r in range(rows):
        for k, c in enumerate(at):
            x[r, c] = 1 + k + 16 * r
    return x


def _check_marks(row, at, times):
    import torch
    assert row[at].tolist() == [times * (1 + k) for k in range(len(at))]
    assert int(torch.count_nonzero(row)) == len(at)


def test_embed_grad_of_long_rows():
    """Columns past 4 GiB into a row, and past 2^31 - 512; without a sort and with
    one; more tiles than a launch has wavefronts."""
    import torch
    lda = _lda()
    D = 2 ** 31 - 1
    at = [0, 511, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 7, D - 600, D - 512, D - 9, D - 8, D - 1]
    grad = _marked(D, at, "float32", 2)
    out = torch.full((2, D), 7.0, device="cuda")
    lda.embed_grad(grad, torch.tensor([1, 1], dtype=torch.int32, device="cuda"), 2, out=out)
    assert out[1][at].tolist() == [2 * (1 + k) + 16 for k in range(len(at))]
    assert int(torch.count_nonzero(out)) == len(at)
    del grad, out
    torch.cuda.empty_cache()
    D = 2 ** 30 + 1003
    at = [0, 511, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 7, D - 513, D - 9, D - 8, D - 1]
    ids = torch.full((129,), -1, dtype=torch.int32, device="cuda")
    ids[10:100] = 0
    if torch.cuda.mem_get_info()[0] > lda.embed_grad_workspace_bytes(129, 1, D) + (20 << 30):
        out = lda.embed_grad(_marked(D, at, "float32").expand(129, D), ids, 1)
        _check_marks(out[0], at, 90.0)
        del out
        torch.cuda.empty_cache()
    D = 2 ** 28 + 9
    at = [0, 511, 2 ** 27, 2 ** 28, D - 1]
    out = lda.embed_grad(_marked(D, at, "float16").expand(128, D), ids[:128], 1)
    _check_marks(out[0], at, 90.0)
    del out
    torch.cuda.empty_cache()


# ---- the draw with a floor: the sums made again while other workgroups read


@pytest.mark.parametrize("dtype", TYPES)
def test_floor_of_long_rows(dtype):
    """Rows in three launches draw what the same rows draw in one (they are 32,768
    logits, and the same with -inf after them), whatever the workspace held, at
    temperatures that keep every group and at ones that keep few.  The shares are
    sums of the same weights: 64 eps."""
    import torch
    lda = _lda()
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    B, V, more = 96, 32_768, 20_000
    x = (torch.randn(B, V, device="cuda", generator=g) * 2).to(_torch_type(dtype))
    low = torch.full((B, more), -np.inf, device="cuda", dtype=x.dtype)
    seed, pos = torch.arange(B, device="cuda"), torch.arange(B, dtype=torch.int32, device="cuda")
    t = torch.linspace(0.2, 8.0, B, device="cuda")
    m = torch.full((B,), 0.02, device="cuda")
    m[::4] = 0.3
    want = lda.draw_logits(x, seed, pos, t, m)
    long = torch.cat([x, low], 1)
    ws = torch.empty(lda.draw_logits_workspace_bytes(B, V + more), dtype=torch.uint8, device="cuda")
    for held in (0x00, 0x7F, 0xFF):
        z, prob = lda.draw_logits(long, seed, pos, t, m, workspace=ws.fill_(held))
        assert torch.equal(z, want[0]), (dtype, held)
        assert float(((prob - want[1]).abs() / want[1]).max()) <= 64 * EPS, (dtype, held)


# ---- sizes past 32 bits, where the library counts in 32


def test_sizes_past_32_bits_are_refused():
    """V or D of 2^32 + a few, which 32 bits would take for a few.  The large
    tensors are views of a few numbers but for one row of logits."""
    import torch
    lda = _lda()
    many = 2 ** 32 + 5
    ids = torch.tensor([0, 4, 5], dtype=torch.int32, device="cuda")
    row = torch.zeros(1, 8, device="cuda")
    half = torch.zeros(1, many, dtype=torch.float16, device="cuda")
    i, s = ids[:1], torch.zeros(1, dtype=torch.int64, device="cuda")
    out = torch.zeros(many, 1, dtype=torch.float16, device="cuda")
    for call in (lambda: lda.embed(row.expand(many, 8), ids),
                 lambda: lda.embed(row.expand(2 ** 31, 8), ids),
                 lambda: lda.embed(half, i, out=torch.empty_like(half)),
                 lambda: lda.embed_grad(half, i, 1, out=torch.empty_like(half)),
                 lambda: lda.embed_grad(half[:, :1].expand(3, 1), ids, many, out=out),
                 lambda: lda.embed_grad(half[:, :1].expand(3, 1), ids, many),
                 lambda: lda.penalise_logits(half, out=torch.empty_like(half)),
                 lambda: lda.draw_logits(half, s, i)):
        with pytest.raises(lda.LdaError) as e:
            call()
        assert e.value.status == lda.STATUS["LDA_ERR_UNSUPPORTED"]


# ---- autograd


def _outs():
    """(name, a call that writes into the tensors it is given, those tensors)"""
    import torch
    lda = _lda()
    x = torch.randn(20, 40, device="cuda")
    i = torch.arange(20, dtype=torch.int32, device="cuda")
    y, G = torch.empty_like(x), torch.zeros(30, 40, device="cuda")
    z, prob = torch.empty_like(i), torch.empty(20, device="cuda")
    return {
        "embed": (lambda: lda.embed(x, i, out=y), [y]),
        "embed_grad": (lambda: lda.embed_grad(x, i, 30, out=G), [G]),
        "embed_grad, added": (lambda: lda.embed_grad(x, i, 30, out=G, accumulate=True), [G]),
        "dropout": (lambda: lda.dropout(x, 0.5, 1, out=y), [y]),
        "dropout in place": (lambda: lda.dropout(x, 0.5, 1, out=x), [x]),
        "penalise": (lambda: lda.penalise_logits(x, out=y), [y]),
        "penalise in place": (lambda: lda.penalise_logits(x, out=x), [x]),
        "draw": (lambda: lda.draw_logits(x, i.long(), i, out=(z, prob)), [z, prob]),
    }


@pytest.mark.parametrize("name", ["embed", "embed_grad", "embed_grad, added", "dropout",
                                  "dropout in place", "penalise", "penalise in place", "draw"])
def test_what_is_overwritten_is_marked(name):
    """A tensor that a call wrote into has another version, so that a backward
    pass that saved it says so and does not use the wrong values."""
    call, written = _outs()[name]
    before = [t._version for t in written]
    call()
    assert all(t._version > v for t, v in zip(written, before)), name


@pytest.mark.parametrize("op", ["dropout", "penalise_logits"])
def test_backward_through_an_overwritten_tensor_raises(op):
    import torch
    lda = _lda()
    x = torch.randn(20, 40, device="cuda", requires_grad=True)
    y = x.exp()  # its backward needs y
    with torch.no_grad():
        lda.dropout(y, 0.5, 1, out=y) if op == "dropout" else lda.penalise_logits(y, out=y)
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()


def test_no_gradient_is_lost_in_silence():
    """A call that would cut a tensor off from its gradient is refused; without
    gradients, and where the result has none (a draw), it runs."""
    import torch
    lda = _lda()
    x = torch.randn(20, 40, device="cuda")
    i = torch.arange(20, dtype=torch.int32, device="cuda")
    h, f, b = i[:, None].contiguous(), torch.ones(20, device="cuda"), torch.zeros(40, device="cuda")
    calls = []
    for t in (torch.nn.Parameter(x), x.clone().requires_grad_(), x.clone().requires_grad_() * 2):
        calls += [lambda t=t: lda.embed(t, i), lambda t=t: lda.embed_grad(t, i, 30),
                  lambda t=t: lda.dropout(t, 0.5, 1), lambda t=t: lda.penalise_logits(t),
                  lambda t=t: lda.embed(x, i, out=t), lambda t=t: lda.dropout(x, 0.5, 1, out=t),
                  lambda t=t: lda.embed_grad(x, i, 20, out=t),
                  lambda t=t: lda.penalise_logits(x, out=t)]
    need = f.clone().requires_grad_()
    calls += [lambda k=k: lda.penalise_logits(x, h, i, **{k: need})
              for k in ("repetition", "frequency", "presence")]
    calls.append(lambda: lda.penalise_logits(x, bias=b.clone().requires_grad_()))
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    z, prob = lda.draw_logits(x.clone().requires_grad_(), i.long(), i)
    z2, prob2 = lda.draw_logits(x, i.long(), i)
    assert torch.equal(z, z2) and torch.equal(prob, prob2) and not prob.requires_grad


# ---- one history for every row


@pytest.mark.parametrize("V", [900, 40_000])
def test_one_history_for_all_rows(V):
    import torch
    lda = _lda()
    B, cap = 7, 300
    g = np.random.default_rng(V)
    x = _gpu(g.normal(0, 3, (B, V)), "float32")
    h = _gpu(g.integers(0, V, (1, cap)).astype(np.int32))
    n = _gpu(g.integers(0, cap + 1, B).astype(np.int32))
    f = torch.full((B,), 0.7, device="cuda")
    seed, pos = torch.arange(B, device="cuda"), torch.arange(B, dtype=torch.int32, device="cuda")
    one = dict(history=h.expand(B, cap), lengths=n, frequency=f)
    each = dict(one, history=h.repeat(B, 1))
    assert torch.equal(lda.penalise_logits(x, **one), lda.penalise_logits(x, **each))
    for a, b in zip(lda.draw_logits(x, seed, pos, **one), lda.draw_logits(x, seed, pos, **each)):
        assert torch.equal(a, b)
    wide = torch.zeros(B * 3 + cap, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):  # rows that overlap
        lda.penalise_logits(x, history=wide.as_strided((B, cap), (3, 1)), lengths=n)


# ---- rules: an infinite penalty reaches the tokens it is for


@pytest.mark.parametrize("V", [900, 40_000])
def test_infinite_frequency(V):
    """A frequency of +inf takes the generated tokens out and leaves those of the
    prompt, and those not seen, as they are; -inf makes the generated ones +inf."""
    import torch
    lda = _lda()
    B, cap, first = 5, 400, 150
    g = np.random.default_rng(V)
    x = _rounded(g.normal(0, 3, (B, V)), "float32")
    h = g.integers(0, V, (B, cap)).astype(np.int32)
    n = np.full(B, cap, dtype=np.int32)
    made = np.zeros((B, V), dtype=bool)
    for b in range(B):
        made[b, h[b, first:]] = True
    seed, pos = torch.arange(B, device="cuda"), torch.arange(B, dtype=torch.int32, device="cuda")
    rules = dict(history=_gpu(h), lengths=_gpu(n), prompt=torch.full_like(pos, first))
    for sign in (1, -1):
        f = torch.full((B,), sign * np.inf, device="cuda")
        got = _np(lda.penalise_logits(_gpu(x, "float32"), frequency=f, **rules))
        assert np.array_equal(got, np.where(made, -sign * np.inf, x)), sign
        z, prob = lda.draw_logits(_gpu(x, "float32"), seed, pos, frequency=f, **rules)
        want = lda.draw_logits(_gpu(got, "float32"), seed, pos)
        assert torch.equal(z, want[0]) and torch.equal(prob, want[1]), sign


# ---- the gradient of a broadcast, larger than the caches if it were written out


@pytest.mark.parametrize("dtype,D,p", [("bfloat16", 1024, 0.0), ("float16", 1003, 0.1)])
def test_embed_grad_of_one_row_for_many(dtype, D, p):
    import torch
    lda = _lda()
    g = torch.Generator(device="cuda")
    g.manual_seed(D)
    N, V = (150 << 20) // (2 * D), 3000
    ids = torch.randint(-1, V + 1, (N,), device="cuda", generator=g, dtype=torch.int32)
    one = torch.randn(1, D, device="cuda", generator=g).to(_torch_type(dtype)).expand(N, D)
    got = lda.embed_grad(one, ids, V, 1.5, p, 3, 4)
    assert torch.equal(got, lda.embed_grad(one.contiguous(), ids, V, 1.5, p, 3, 4))
