"""What one operator of the way from a layer's last activations to the next token gives has to
equal, bit for bit, what another way to the same numbers gives."""
import numpy as np
import pytest

from test_layers_gpu import SIZES, _check, _norm_inputs
from test_tokens_gpu import TYPES, _gpu, _lda

pytestmark = pytest.mark.gpu


# ---- the norm's 8 bits: those of its rows in float


@pytest.mark.parametrize("N,D", [*SIZES, (2000, 600), (500, 3000), (100, 12_000), (60, 20_000)])
def test_norm_bits_are_those_of_its_rows(N, D):
    """The rows as add_norm gives them in float, put into 8 bits by quantise_rows, which decides
    every half exactly: of a million columns about fifteen are so near to one that a rounding on the
    way would move them."""
    import torch
    lda = _lda()
    for residual in (True, False):
        x, r, w = _norm_inputs(N, D, "float32", "float32", residual)
        args = _gpu(x, "float32"), _gpu(w, "float32"), 1e-5
        more = None if r is None else _gpu(r, "float32")
        y = lda.add_norm(*args, residual=more)
        want = lda.quantise_rows(y[0] if residual else y)
        got = lda.add_norm_int8(*args, residual=more)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [40, 700, 3000, 5003, 20_001])
def test_norm_bits_at_halves(dtype, D):
    """Rows of one magnitude under weights that are halves of the 127th part of the largest, so
    that nearly every column is next to a half; and 16-bit rows as the same rows in float."""
    import torch
    lda = _lda()
    g = np.random.default_rng(D)
    w = (g.integers(-127, 127, D) + 0.5).astype(np.float32)
    w[D // 3] = 127
    sign = g.choice([-1.0, 1.0], (12, D))
    x = sign * np.resize([1.0, 0.75, 1.25, 3.0, 0.1015625, 30.0], (12, 1))
    rows, weight = _gpu(x, dtype), _gpu(w)
    got = lda.add_norm_int8(rows, weight)
    want = lda.quantise_rows(lda.add_norm(rows.float(), weight))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert bool((got[0].abs().amax(1) == 127).all())


# ---- the norm's gradient, in place


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,D", [(1, 7), (3, 64), (5, 300), (33, 512), (2050, 1000), (31, 1024), (9, 1500),
                                 (4099, 2048), (7, 4096), (66, 5003), (9, 16_000), (5, 17_003)])
def test_norm_grad_over_its_inputs(dtype, N, D):
    """dx over the gradient, over h and over the residual's gradient: the bits of dx elsewhere."""
    lda = _lda()
    h, r, w = _norm_inputs(N, D, dtype, "float32")
    dy = _norm_inputs(N + 1, D, dtype, "float32")[0][:N]
    weight = _gpu(w, "float32")
    for residual in (True, False):
        def inputs():
            return _gpu(dy, dtype), _gpu(h, dtype), _gpu(r, dtype) if residual else None
        a, b, c = inputs()
        dx, dw = lda.norm_grad(a, b, weight, residual_grad=c)
        for i in range(3 if residual else 2):
            args = inputs()
            got = lda.norm_grad(args[0], args[1], weight, residual_grad=args[2], out=args[i])
            assert got[0] is args[i]
            _same(got[0], dx)
            _same(got[1], dw)


def _same(a, b):
    import torch
    assert torch.equal(torch.nan_to_num(a, 5.0, 6.0, 7.0), torch.nan_to_num(b, 5.0, 6.0, 7.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), "overflow"])
@pytest.mark.parametrize("N,D", [(1, 40), (5, 300), (6, 1024), (4097, 520), (3, 1400), (1027, 2000)])
def test_norm_grad_over_h_of_an_infinite_last_row(dtype, bad, N, D):
    """The last row's dx is infinite or NaN, by the residual's gradient or by its type's range, and
    written over h while other wavefronts, whose rows are past the last, load that row in place of
    theirs: the weight's gradient, which is finite, has no part in it."""
    import torch
    lda = _lda()
    h, r, w = _norm_inputs(N, D, dtype, "float32")
    dy = _norm_inputs(N + 1, D, dtype, "float32")[0][:N]
    weight = _gpu(w, "float32")
    largest = float(torch.finfo(_gpu(dy, dtype).dtype).max)

    def inputs():
        grad, rows, rest = _gpu(dy, dtype), _gpu(h, dtype), _gpu(r, dtype)
        rest[-1] = largest if bad == "overflow" else bad
        if bad == "overflow":  # s (grad weight - ...) of the largest's size on top of it
            grad[-1] = largest / 4 * torch.sign(weight)
            rows[-1] *= 2.0 ** -6
        return grad, rows, rest
    a, b, c = inputs()
    dx, dw = lda.norm_grad(a, b, weight, residual_grad=c)
    assert bad == "overflow" or bool(torch.isfinite(dw).all())
    assert not torch.isfinite(dx[-1]).all()
    for _ in range(10):
        grad, rows, rest = inputs()
        got = lda.norm_grad(grad, rows, weight, residual_grad=rest, out=rows)
        _same(got[0], dx)
        _same(got[1], dw)


# ---- the product: a scale of any layout


@pytest.mark.parametrize("T,B,N,K", [(2, 300, 1, 64), (300, 2, 1, 64), (64, 33, 1, 4096), (8, 70, 40, 200),
                                     (3, 700, 130, 512)])
def test_project_scale_of_any_layout(T, B, N, K):
    """Scales that are a transposed tensor, or every other column of one, against contiguous ones,
    at outputs of a scale's own size among others."""
    import torch
    lda = _lda()
    g = torch.Generator(device="cuda").manual_seed(T)
    q = torch.randint(-128, 128, (T, B, K), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-128, 128, (N, K), dtype=torch.int8, device="cuda", generator=g)
    ws = torch.rand(N, device="cuda", generator=g)
    scale = torch.rand(T, B, device="cuda", generator=g)
    want = lda.project_int8(q, scale, w, ws, dtype=torch.float32)
    wide = torch.stack([scale, -scale], 2).view(T, 2 * B)
    for view in (scale.t().contiguous().t(), wide[:, ::2]):
        assert not view.is_contiguous() or 1 in (T, B)
        for _ in range(20):
            assert torch.equal(lda.project_int8(q, view, w, ws, dtype=torch.float32), want)
        out = torch.empty_like(want)
        assert torch.equal(lda.project_int8(q, view, w, ws, out=out), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,K", [(7, 10), (50, 64), (1000, 130), (4096, 512), (300, 1024), (900, 2000),
                                 (5000, 2048), (17_000, 256)])
def test_project_row_alone_and_among_others(dtype, N, K):
    """Bit for bit, by the kernel for a few rows and by those of every tile, aligned or not."""
    import torch
    lda = _lda()
    g = torch.Generator(device="cuda").manual_seed(N)
    M = 2100
    q = torch.randint(-128, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
    w = torch.randint(-128, 128, (N, K), dtype=torch.int8, device="cuda", generator=g)
    s = torch.rand(M, device="cuda", generator=g) / 100
    ws = torch.rand(N, device="cuda", generator=g) / 100
    bias = torch.randn(N, device="cuda", generator=g)
    odd = torch.zeros(M, K + 1, dtype=torch.int8, device="cuda")[:, 1:]  # lines at any byte
    odd.copy_(q)
    for b in (bias, None):
        def product(rows, n):
            return lda.project_int8(rows[:n], s[:n], w, ws, bias=b, dtype=getattr(torch, dtype))
        want = product(q, M)
        for n in (1, 5, 16, 17, 40, 64, 100, 300, 700):
            assert torch.equal(product(q, n), want[:n]), n
            assert torch.equal(product(odd, n), want[:n]), n


# ---- sampling: what min_p cuts off


def _floors_next_to_a_weight(n):
    """(largest logits, next floats below, temperatures, floors): a weight of 2^-1 to 2^-6 and a float
    within 1e-10 to 4e-9 of it, above or below.  A logit is a float, 2^-25 to 2^-23 of the largest
    below it, so the logarithm of a weight, taken from the logit in double, is off by up to 6 2^-28
    of itself: less than that is next to nothing, and 1e-9 is not."""
    g = np.random.default_rng(3)
    tops = g.choice(np.float32([1e6, 3e5, -7e6, 1234567.0, 1e20, -2.5, 64.0]), 400_000)
    nexts = np.nextafter(tops, np.float32(-np.inf))
    apart = tops.astype(float) - nexts.astype(float)
    t = (apart / (g.uniform(1, 6, len(tops)) * np.log(2))).astype(np.float32)
    w = np.exp(-apart / t.astype(float))
    m = w.astype(np.float32)
    off = np.abs(m.astype(float) - w)
    take = np.nonzero((off > 1e-10) & (off < 4e-9))[0][:n]
    assert len(take) == n
    return tops[take], nexts[take], t[take], m[take]


@pytest.mark.parametrize("V", [700, 1500, 3000])
@pytest.mark.parametrize("share", [None, 0.97, 0.999999])
def test_sample_floors_next_to_a_weight(V, share):
    """Half of the floors are next above a weight, which goes, the others next below, which stays:
    among few tokens and many, alone and before the place where top_p ends."""
    B = 1200
    top, following, t, m = _floors_next_to_a_weight(B)
    g = np.random.default_rng(V)
    x = np.repeat(following[:, None], V, 1)
    for _ in range(2):  # the others one to three floats further down, with weights of their own
        x = np.where(g.random((B, V)) < 0.6, np.nextafter(x, np.float32(-np.inf)), x)
    x = np.where(g.random((B, V)) < 0.5, np.float32(-np.inf), x)
    x[:, V // 3], x[:, V // 2], x[:, 2 * V // 3] = top, following, following
    p = None if share is None else np.full(B, share, dtype=np.float32)
    _check(x.astype(float), g.random(B).astype(np.float32), t, None, p, m, what=(V, share))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_sample_floors_between_two_steps(dtype):
    """min_p is asked of a weight as it is, not of the whole multiple of 2^-46 that it is held as,
    whatever the row's length and so its way: a u of 1 takes the last token that stays.  Weights of
    10.6 and 10.4 steps (to 2^-20 of them in float) against floors on both sides of them."""
    import torch
    lda = _lda()
    x, m, want = [], [], []
    for steps, floor in ((10.6, 10.75), (10.6, 10.55), (10.4, 10.3), (10.4, 10.45), (0.75, 0.8),
                         (0.75, 0.7), (5.5, 5.5 - 2.0 ** -16), (5.5, 5.5 + 2.0 ** -16)):
        x.append(np.log(steps * 2.0 ** -46))
        m.append(floor * 2.0 ** -46)
        want.append(steps >= floor)
    if dtype == "bfloat16":  # (whole logits: weights of 17.9 and 6.58 steps)
        x = [-29.0, -29.0, -30.0, -30.0]
        w = np.exp(x)
        m = [w[0] * (1 + 2e-3), w[0] * (1 - 2e-3), w[2] * (1 + 2e-3), w[2] * (1 - 2e-3)]
        want = [False, True, False, True]
    B = len(x)
    for V in (3, 60, 200, 256, 257, 900, 1024, 1025, 3000, 20_000):
        rows = torch.full((B, V), -float("inf"), device="cuda")
        rows[:, 0] = 0.0
        rows[:, V // 2] = -1.0
        rows[:, V - 1] = torch.tensor(x, device="cuda")
        floor = torch.tensor(m, dtype=torch.float32, device="cuda")
        for k, p in ((None, None), (3, None), (700, None), (None, 1 - 2.0 ** -24), (3, 1 - 2.0 ** -24)):
            z, _ = lda.sample_logits(
                rows.to(getattr(torch, dtype)), torch.ones(B, device="cuda"), min_p=floor,
                top_k=None if k is None else torch.full((B,), k, dtype=torch.int32, device="cuda"),
                top_p=None if p is None else torch.full((B,), p, device="cuda"))
            last = [V - 1 if stays and p is None else V // 2 for stays in want]
            assert z.tolist() == last, (V, k, p)


# ---- sampling: a row is the same wherever its tokens are


@pytest.mark.parametrize("dtype", TYPES)
def test_sample_of_a_row_among_others(dtype):
    """200 logits alone, with nothing after them and between them, so that they are compared,
    sorted, cut by bins and found in other stretches: the same token and the same bits of its
    probability."""
    import torch
    lda = _lda()
    B, n = 400, 200
    g = torch.Generator(device="cuda").manual_seed(6)
    x = (torch.randn(B, n, device="cuda", generator=g) * 3).to(getattr(torch, dtype))

    def draw(low, high):
        return torch.rand(B, device="cuda", generator=g) * (high - low) + low
    u, t, p, m = draw(0, 1), draw(0.2, 3), draw(0.3, 1.1), 10 ** draw(-6, -0.3)
    k = torch.randint(0, n, (B,), dtype=torch.int32, device="cuda", generator=g)
    for rules in ({}, dict(top_p=p), dict(min_p=m), dict(top_k=k, top_p=p, min_p=m),
                  dict(top_p=p, min_p=m)):
        want = lda.sample_logits(x, u, temperature=t, **rules)
        for V, apart in ((257, 1), (1000, 1), (1000, 5), (2000, 1), (2000, 10), (40_000, 200),
                         (131_072, 600), (70_000, 3)):
            wide = torch.full((B, V), -float("inf"), dtype=x.dtype, device="cuda")
            first = (V - n * apart) // 2
            wide[:, first:first + n * apart:apart] = x
            z, prob = lda.sample_logits(wide, u, temperature=t, **rules)
            assert torch.equal((z - first) // apart, want[0]) and torch.equal(prob, want[1]), (V, rules)
