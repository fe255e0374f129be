"""The norm, its gradient, 8-bit rows and products, and the sampling, against the oracle
in 64 bits.

Tolerances, from the arithmetic (eps = 2^-24, half a unit of float; the outputs' half
units as in test_tokens_gpu):
  * norm: h is rounded once; the mean of D squares is summed in chains of at most c =
    8 ceil(D / 512) + 30 additions (a lane's columns, the tree over lanes, wavefronts), each eps;
    its root, the division and the reciprocal halve that and add 4; two products: |y| (c / 2 + 8)
    eps, then the output;
  * 8 bits: scale as y; q within 1/2 of 127 y / max |y|, whose error is 127 (c + 20) eps;
  * gradient: the terms of dx without their signs, times (2 c + 16) eps; those of dweight,
    added over N rows in chains of at most N / 256 + 80, times (that + c / 2 + 10) eps;
  * rows as given in 8 bits: exact, halves included; scale one division: eps;
  * product: the sum rounded to float, two products, the bias: 4 eps of the largest;
  * sampling: a weight is off by 2^-47 of the largest (rounding to whole multiples of 2^-46)
    and 2^-49 of itself; z must be the oracle's unless the oracle's sums decide by less than
    2^-46 V (S is at least 1).  Its probability: 2^-40 and the rounding to float.
"""
import numpy as np
import pytest

from oracle import layers as ref
from test_tokens_gpu import EPS, TYPES, UNIT, _close, _gpu, _lda, _np, _rounded, _torch_type, _wide

pytestmark = pytest.mark.gpu


def _chain(D):
    return 8 * -(-D // 512) + 30


# ---- the norm


SIZES = [(1, 1), (1, 7), (5, 8), (3, 64), (9, 65), (4, 511), (33, 512), (2, 513), (7, 1000),
         (130, 1024), (6, 1025), (3, 2048), (5, 2049), (17, 4096), (2, 4099), (3, 8192), (2, 8200),
         (1, 16_384), (2, 16_385), (1, 40_001), (700, 16_390), (5000, 33)]


def _norm_inputs(N, D, dtype, wt, residual=True):
    g = np.random.default_rng(N * 31 + D)
    x = _rounded(g.normal(0, 1.5, (N, D)), dtype)
    r = _rounded(g.normal(0, 2, (N, D)), dtype) if residual else None
    w = _rounded(1 + 0.3 * g.normal(0, 1, D), wt)
    return x, r, w


@pytest.mark.parametrize("dtype,wt", [("float32", "float32"), ("bfloat16", "bfloat16"),
                                      ("bfloat16", "float32"), ("float16", "float16"),
                                      ("float16", "float32")])
@pytest.mark.parametrize("N,D", SIZES)
def test_norm(dtype, wt, N, D):
    lda = _lda()
    for residual in (True, False):
        x, r, w = _norm_inputs(N, D, dtype, wt, residual)
        want, h = ref.norm(x, w, 1e-5, r)
        got = lda.add_norm(_gpu(x, dtype), _gpu(w, wt), 1e-5,
                           residual=None if r is None else _gpu(r, dtype))
        if residual:
            got, total = got
            _close(_np(total), h, np.abs(h) * EPS, dtype, "h")
        slack = np.abs(want) * (_chain(D) / 2 + 8) * EPS
        _close(_np(got), want, slack, dtype, (dtype, N, D))
        q, scale, *total = lda.add_norm_int8(_gpu(x, dtype), _gpu(w, wt), 1e-5,
                                             residual=None if r is None else _gpu(r, dtype))
        real, step = ref.quantise(want)
        assert q.dtype == _torch_type("int8") and len(total) == int(residual)
        assert np.abs(_np(scale) / step - 1).max() <= (_chain(D) / 2 + 10) * EPS
        assert np.abs(_np(q) - real).max() <= 0.5 + 127 * (_chain(D) + 20) * EPS
        if residual:
            _close(_np(total[0]), h, np.abs(h) * EPS, dtype, "h")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [37, 1500, 4097, 17_000])
def test_norm_rows_that_are_not_ordinary(dtype, D):
    import torch
    lda = _lda()
    N = 8
    x, _, w = _norm_inputs(N, D, dtype, dtype, False)
    x[1] = 0
    x[2, D // 2] = np.inf
    x[3, D - 1] = np.nan
    x[4] *= 2.0 ** -20
    x = _rounded(x, dtype)
    with np.errstate(invalid="ignore"):
        want, _ = ref.norm(x, w, 1e-6)
    got = _np(lda.add_norm(_gpu(x, dtype), _gpu(w, dtype)))
    assert not got[1].any() and np.isnan(got[3]).all() and np.isnan(got[2, D // 2])
    assert not np.delete(got[2], D // 2).any()
    rest = [0, 4, 5, 6, 7]
    _close(got[rest], want[rest], np.abs(want[rest]) * (_chain(D) / 2 + 8) * EPS, dtype)
    q, scale = lda.add_norm_int8(_gpu(x, dtype), _gpu(w, dtype))
    q, scale = _np(q), _np(scale)
    assert not q[[1, 2, 3]].any() and scale[1] == 0 and np.isnan(scale[[2, 3]]).all()
    assert (np.abs(q[rest]).max(1) == 127).all() and np.isfinite(scale[rest]).all()
    assert torch.isfinite(lda.add_norm(torch.zeros(2, D, device="cuda"), torch.ones(D, device="cuda"))).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,at", [(1, 1), (5, 3), (8, 0), (64, 7)])
@pytest.mark.parametrize("D", [203, 3001, 20_001])
def test_norm_rows_at_any_distance(dtype, pad, at, D):
    import torch
    lda = _lda()
    N = 9
    x, r, w = _norm_inputs(N, D, dtype, dtype)
    dense = _gpu(x, dtype), _gpu(r, dtype)
    weight = _gpu(w, dtype)
    want = lda.add_norm(dense[0], weight, residual=dense[1])
    xv, rv = _wide(x, dtype, pad, at)[0], _wide(r, dtype, pad + 3, at)[0]
    out, buf = _wide(np.zeros((N, D)), dtype, pad, at)
    total, buf2 = _wide(np.zeros((N, D)), dtype, pad + 1, at)
    y, h = lda.add_norm(xv, weight, residual=rv, out=out, sum_out=total)
    assert y is out and h is total and torch.equal(y, want[0]) and torch.equal(h, want[1])
    assert int(torch.isfinite(buf).sum()) == N * D == int(torch.isfinite(buf2).sum())
    wide = torch.full((N, D + pad), 99, dtype=torch.int8, device="cuda")
    scale = torch.empty(N, device="cuda")
    q, s, h = lda.add_norm_int8(xv, weight, residual=rv, out=(wide[:, :D], scale))
    plain = lda.add_norm_int8(dense[0], weight, residual=dense[1])
    assert torch.equal(q, plain[0]) and torch.equal(s, plain[1]) and torch.equal(h, want[1])
    assert bool((wide[:, D:] == 99).all())
    # in place: h over the residual, y over x
    y, h = lda.add_norm(xv, weight, residual=rv, out=xv, sum_out=rv)
    assert torch.equal(y, want[0]) and torch.equal(h, want[1])
    # one row for all of the residual
    one = dense[1][:1]
    a = lda.add_norm(dense[0], weight, residual=one.expand(N, D))
    b = lda.add_norm(dense[0], weight, residual=one.expand(N, D).contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_norm_shapes():
    import torch
    lda = _lda()
    x, r = torch.randn(2, 2, 3, 5, 96, device="cuda")
    w = torch.randn(96, device="cuda")
    y, h = lda.add_norm(x, w, residual=r)
    assert y.shape == h.shape == x.shape
    assert torch.equal(y.view(30, 96), lda.add_norm((x + r).view(30, 96), w))
    q, s = lda.add_norm_int8(x, w)
    assert q.shape == x.shape and s.shape == x.shape[:-1]
    flat = lda.add_norm_int8(x.view(30, 96), w)
    assert torch.equal(q.view(30, 96), flat[0]) and torch.equal(s.view(30), flat[1])
    dx, dw = lda.norm_grad(y, h, w, residual_grad=r)
    assert dx.shape == x.shape and dw.shape == w.shape
    v = torch.randn(96, device="cuda")
    assert torch.equal(lda.add_norm(v, w), lda.add_norm(v[None], w)[0])
    empty = torch.empty(0, 96, device="cuda")
    assert lda.add_norm(empty, w).shape == (0, 96)
    q, s = lda.quantise_rows(torch.empty(4, 0, 96, device="cuda"))
    assert q.shape == (4, 0, 96) and s.shape == (4, 0)
    dx, dw = lda.norm_grad(empty, empty, w)
    assert dx.shape == (0, 96) and not dw.any()
    keep = torch.ones(96, device="cuda")
    lda.norm_grad(empty, empty, w, weight_out=keep, accumulate=True)
    assert bool((keep == 1).all())
    y, h = lda.add_norm(x, w, sum_out=torch.empty_like(x))  # h without a residual is x
    assert torch.equal(h, x)


# ---- its gradient


@pytest.mark.parametrize("dtype,wt", [("float32", "float32"), ("bfloat16", "bfloat16"),
                                      ("bfloat16", "float32"), ("float16", "float16"),
                                      ("float16", "float32")])
@pytest.mark.parametrize("N,D", SIZES)
def test_norm_grad(dtype, wt, N, D):
    import torch
    lda = _lda()
    h, r, w = _norm_inputs(N, D, dtype, wt)
    g = np.random.default_rng(D)
    dy = _rounded(g.normal(0, 1, (N, D)), dtype)
    rest = ((N // 256 + 80) + _chain(D) / 2 + 10) * EPS
    for residual in (r, None):
        dx, dw, size, size_w = ref.norm_grad(dy, h, w, 1e-5, residual)
        args = _gpu(dy, dtype), _gpu(h, dtype), _gpu(w, wt), 1e-5
        more = None if residual is None else _gpu(residual, dtype)
        got, got_w = lda.norm_grad(*args, residual_grad=more)
        _close(_np(got), dx, size * (2 * _chain(D) + 16) * EPS, dtype, (dtype, N, D))
        _close(_np(got_w), dw, size_w * rest, "float32", "dweight")
        # added to what is there; and the same bits again
        before = torch.ones(D, device="cuda")
        again, total = lda.norm_grad(*args, residual_grad=more, weight_out=before, accumulate=True)
        assert total is before and torch.equal(again, got) and torch.equal(total, got_w + 1)
        # over the gradient itself
        place = args[0].clone()
        lda.norm_grad(place, *args[1:], residual_grad=more, out=place)
        assert torch.equal(place, got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,D", [(40, 203), (3000, 40), (9, 2900), (9, 17_003)])
def test_norm_grad_rows_at_any_distance(dtype, N, D):
    import torch
    lda = _lda()
    h, r, w = _norm_inputs(N, D, dtype, dtype)
    dy = _rounded(np.random.default_rng(3).normal(0, 1, (N, D)), dtype)
    weight = _gpu(w, dtype)
    want = lda.norm_grad(_gpu(dy, dtype), _gpu(h, dtype), weight, residual_grad=_gpu(r, dtype))
    out, buf = _wide(np.zeros((N, D)), dtype, 5, 3)
    space = torch.empty(lda.norm_grad_workspace_bytes(N, D), dtype=torch.uint8, device="cuda")
    got = lda.norm_grad(_wide(dy, dtype, 1, 1)[0], _wide(h, dtype, 7, 2)[0], weight,
                        residual_grad=_wide(r, dtype, 9, 4)[0], out=out, workspace=space)
    assert got[0] is out and torch.equal(out, want[0]) and torch.equal(got[1], want[1])
    assert int(torch.isfinite(buf).sum()) == N * D
    # the gradient of a broadcast: one row for all
    one = _gpu(dy[:1], dtype).expand(N, D)
    a = lda.norm_grad(one, _gpu(h, dtype), weight)
    b = lda.norm_grad(one.contiguous(), _gpu(h, dtype), weight)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_norm_grad_against_differences():
    """The float kernels' own gradient, against differences of the float kernels' loss: the
    second difference of a row's norm is about |dy| / |h|^2 per unit, so a step of 1e-2 leaves
    1e-4 of the terms, and sums of 50 rounded outputs over twice the step 50 eps 4 / 2e-2."""
    import torch
    lda = _lda()
    g = torch.Generator(device="cuda").manual_seed(5)

    def draw(*shape):
        return torch.randn(shape, device="cuda", generator=g)
    x, r, w, dy = draw(2, 25), draw(2, 25), draw(25), draw(2, 25)

    def loss(x, w):
        return float((lda.add_norm(x, w, residual=r)[0].double() * dy).sum())
    h = lda.add_norm(x, w, residual=r)[1]
    dx, dw = lda.norm_grad(dy, h, w)
    step = 1e-2
    for i, j in ((0, 0), (0, 13), (1, 24), (1, 5)):
        e = torch.zeros_like(x)
        e[i, j] = step
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * step) - float(dx[i, j])) < 2e-3
        assert abs((loss(x, w + e[i]) - loss(x, w - e[i])) / (2 * step) - float(dw[j])) < 2e-3


# ---- rows in 8 bits


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,D", SIZES)
def test_quantise(dtype, N, D):
    lda = _lda()
    g = np.random.default_rng(N + D)
    x = g.normal(0, 1, (N, D)) * 10.0 ** g.uniform(-3, 3, (N, 1))
    x = _rounded(np.clip(x, -6e4, 6e4), dtype)
    q, scale = lda.quantise_rows(_gpu(x, dtype))
    real, step = ref.quantise(x)
    assert np.array_equal(_np(q), np.rint(real))
    assert (np.abs(_np(scale) - step) <= step * EPS).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [300, 5000, 20_000])
def test_quantise_halves(dtype, D):
    """Every half there is: quotients are k + 1/2 exactly where the largest is 127 or 254 (times
    a power of two), and at x = max / 2; of the float row the digit next to a half decides."""
    lda = _lda()
    g = np.random.default_rng(D)
    x = np.zeros((6, D))
    x[0] = g.integers(-254, 255, D) / 2
    x[0, 3] = 127
    x[1] = g.integers(-127, 128, D) * 2.0 ** -9
    x[1, D - 1] = -127 * 2.0 ** -8
    x[2] = g.choice([1.0, -1.0, 0.5, 2.0], D) * 1.2890625
    x[3] = g.choice([1.0, -1.0, 0.5, 2.0], D) * 2.0 ** -14 * 1.6015625
    x[4] = (g.integers(-126, 127, D) + 0.5) * 1.109375 / 127
    x[4, 7] = 1.109375
    x[5] = np.nextafter((g.integers(-126, 127, D) + 0.5).astype(np.float32), np.float32(9)).astype(float)
    x[5, 0] = 127
    x = _rounded(x, dtype)
    q, scale = lda.quantise_rows(_gpu(x, dtype))
    real, step = ref.quantise(x)
    assert np.array_equal(_np(q), np.rint(real))
    assert (np.abs(_np(scale) - step) <= step * EPS).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_quantise_rows_that_are_not_ordinary(dtype):
    """Rows of zeros, of the smallest and the largest numbers, with NaN and infinities."""
    lda = _lda()
    g = np.random.default_rng(2)
    D = 700
    x = g.normal(0, 1, (9, D))
    x[0] = 0
    x[1, 5] = np.nan
    x[2, 699] = -np.inf
    x[3] *= 2.0 ** 120
    x[4] *= 2.0 ** -110
    x[5] *= 2.0 ** -126
    x[6] = 0
    x[6, 9] = 2.0 ** -133  # a subnormal number alone
    x[7] = -3.0e38
    x[8] = -0.0
    x = _rounded(x, dtype)
    q, scale = lda.quantise_rows(_gpu(x, dtype))
    real, step = ref.quantise(x)
    assert np.array_equal(_np(q), np.rint(real))
    got = _np(scale)
    assert np.array_equal(np.isnan(got), np.isnan(step))
    fine = np.isfinite(step)
    assert (np.abs(got - step)[fine] <= step[fine] * EPS + 2.0 ** -150).all()


def test_quantise_views():
    import torch
    lda = _lda()
    x = torch.randn(20, 333, device="cuda").bfloat16()
    want = lda.quantise_rows(x)
    buf = torch.full((20, 400), 99, dtype=torch.int8, device="cuda")
    scale = torch.empty(20, device="cuda")
    got = lda.quantise_rows(torch.cat([x, x], 1)[:, 333:], out=(buf[:, 11:344], scale))
    assert torch.equal(got[0], want[0]) and torch.equal(scale, want[1])
    assert int((buf == 99).sum()) >= 20 * 67 and bool((buf[:, :11] == 99).all())
    rows = lda.quantise_rows(x[:1].expand(5, 333))
    assert torch.equal(rows[0], want[0][:1].expand(5, 333))


# ---- the product


def _whole(g, shape, extremes=True):
    a = g.integers(-128, 128, shape).astype(np.int8)
    if extremes:
        a.flat[::7] = -128
        a.flat[::11] = 127
    return a


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 1), (1, 5, 3), (2, 16, 16), (1, 100, 64), (16, 17, 65), (17, 33, 127), (3, 1000, 128),
    (31, 64, 200), (32, 130, 1001), (33, 65, 63), (64, 64, 64), (65, 127, 129), (100, 300, 999),
    (128, 256, 512), (200, 1003, 77), (257, 255, 1024), (5, 4096, 4096), (513, 129, 2047),
    (1000, 7, 640), (7, 1000, 5000), (300, 520, 192), (1030, 1030, 320), (520, 776, 1000)])
def test_project(dtype, M, N, K):
    lda = _lda()
    g = np.random.default_rng(M + 3 * N + 7 * K)
    q, w = _whole(g, (M, K)), _whole(g, (N, K))
    s, ws = (g.uniform(0.5, 2, n).astype(np.float32) * 2.0 ** -10 for n in (M, N))
    b = g.normal(0, 1, N).astype(np.float32)
    for bias in (None, b):
        want, part = ref.project(q, s.astype(float), w, ws.astype(float),
                                 None if bias is None else bias.astype(float))
        got = lda.project_int8(_gpu(q), _gpu(s), _gpu(w), _gpu(ws),
                               bias=None if bias is None else _gpu(bias), dtype=_torch_type(dtype))
        slack = np.abs(part) * 4 * EPS + (0 if bias is None else np.abs(bias) * EPS)
        _close(_np(got), want, slack, dtype, (M, N, K))


@pytest.mark.parametrize("M,N", [(1, 3), (40, 20), (300, 260)])
def test_project_largest_sums(M, N):
    """All -128 at the longest K: 2^14 * 131,071 is the last sum in 32 bits."""
    import torch
    lda = _lda()
    K = 131_071
    q = torch.full((M, K), -128, dtype=torch.int8, device="cuda")
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    ones = torch.ones(max(M, N), device="cuda")
    got = lda.project_int8(q, ones[:M], w, ones[:N], dtype=torch.float32)
    assert bool((got == float(2 ** 14 * K)).all())
    w.fill_(127)
    got = lda.project_int8(q, ones[:M], w, ones[:N], dtype=torch.float32)
    assert bool((got.double() == float(np.float32(-128 * 127 * K))).all())
    with pytest.raises(Exception):
        lda.project_int8(torch.zeros(1, K + 1, dtype=torch.int8, device="cuda"), ones[:1],
                         torch.zeros(1, K + 1, dtype=torch.int8, device="cuda"), ones[:1])


@pytest.mark.parametrize("M,N,K", [(3, 70, 130), (70, 90, 257), (300, 300, 640), (1, 64, 4096)])
@pytest.mark.parametrize("pad,at", [(1, 1), (16, 0), (13, 5), (64, 16)])
def test_project_rows_at_any_distance(M, N, K, pad, at):
    import torch
    lda = _lda()
    g = np.random.default_rng(pad)
    q, w = _whole(g, (M, K)), _whole(g, (N, K))
    s, ws = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    want = lda.project_int8(_gpu(q), s, _gpu(w), ws)

    def wide(a):
        buf = torch.full((a.shape[0], a.shape[1] + pad), 77, dtype=torch.int8, device="cuda")
        view = buf[:, min(at, pad):min(at, pad) + a.shape[1]]
        view.copy_(_gpu(a))
        return view
    buf = torch.full((M + 1, N + pad), float("nan"), device="cuda", dtype=torch.bfloat16)
    out = buf[:M, 1:1 + N]
    assert lda.project_int8(wide(q), s, wide(w), ws, out=out) is out
    assert torch.equal(out, want) and int(torch.isfinite(buf).sum()) == M * N
    # one row for all
    one = _gpu(q[:1]).expand(M, K)
    assert torch.equal(lda.project_int8(one, s, _gpu(w), ws),
                       lda.project_int8(one.contiguous(), s, _gpu(w), ws))


def test_project_shapes_and_scales():
    import torch
    lda = _lda()
    q = torch.randint(-128, 128, (2, 3, 40), dtype=torch.int8, device="cuda")
    w = torch.randint(-128, 128, (9, 40), dtype=torch.int8, device="cuda")
    s, ws = torch.rand(2, 3, device="cuda"), torch.rand(9, device="cuda")
    s[0, 1] = float("nan")
    s[1, 2] = 0
    y = lda.project_int8(q, s, w, ws, dtype=torch.float32)
    assert y.shape == (2, 3, 9) and torch.isnan(y[0, 1]).all() and not y[1, 2].any()
    flat = lda.project_int8(q.view(6, 40), s.view(6), w, ws, dtype=torch.float32)
    assert torch.equal(torch.nan_to_num(y.view(6, 9)), torch.nan_to_num(flat))
    assert lda.project_int8(q[:0], s[:0], w, ws).shape == (0, 3, 9)
    assert y.dtype == torch.float32 and lda.project_int8(q, s, w, ws).dtype == torch.bfloat16


# ---- sampling


def _settings(B, g, V):
    """Rows of every kind of setting, in turn."""
    t = g.choice([1.0, 0.7, 1.3, 0.3, 5.0], B).astype(np.float32)
    k = np.where(g.random(B) < 0.5, 0, np.exp(g.uniform(0, np.log(V + 1), B))).astype(np.int32)
    p = np.where(g.random(B) < 0.4, 1.0, g.uniform(0, 1, B)).astype(np.float32)
    m = np.where(g.random(B) < 0.6, 0.0, 10.0 ** g.uniform(-5, 0, B)).astype(np.float32)
    return t, k, p, m


def _check(x, u, t=None, k=None, p=None, m=None, what="", view=None, dtype="float32"):
    import torch
    lda = _lda()
    B, V = x.shape
    logits = _gpu(x, dtype) if view is None else view
    z, prob = lda.sample_logits(logits, _gpu(u), *(None if a is None else _gpu(a)
                                                   for a in (t, k, p, m)))
    assert z.dtype == torch.int32 and prob.dtype == torch.float32
    z, prob = _np(z), _np(prob)
    near = 0
    for b in range(B):
        want, share, margin = ref.sample(
            x[b], float(u[b]), 1.0 if t is None else float(t[b]), 0 if k is None else int(k[b]),
            1.0 if p is None or np.isnan(p[b]) else float(p[b]),
            0.0 if m is None or np.isnan(m[b]) else float(m[b]))
        if margin <= V * 2.0 ** -46:
            near += 1
            continue
        assert z[b] == want, (what, b, z[b], want, margin)
        assert abs(prob[b] - share) <= share * (EPS + 2.0 ** -40) + 2.0 ** -46, (what, b)
    assert near <= B // 20 + 1, (what, near)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,V", [(1, 1), (3, 2), (5, 7), (40, 33), (64, 300), (20, 1024), (30, 2049),
                                 (9, 8191), (33, 10_000), (6, 32_768), (5, 50_001), (4, 131_072),
                                 (3, 131_073), (2, 400_003)])
def test_sample(dtype, B, V):
    g = np.random.default_rng(B + V)
    x = g.normal(0, 2.5, (B, V))
    x[:, g.integers(0, V, min(10, V))] += 6
    x = _rounded(x, dtype)
    u = g.random(B).astype(np.float32)
    t, k, p, m = _settings(B, g, V)
    args = dict(dtype=dtype, what=(dtype, B, V))
    _check(x, u, **args)
    _check(x, u, t, **args)
    _check(x, u, t, k, **args)
    _check(x, u, t, None, p, **args)
    _check(x, u, t, None, None, m, **args)
    _check(x, u, t, k, p, m, **args)
    _check(x, u, t, np.minimum(np.maximum(k, 1), 60), p, **args)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,V,values", [(20, 50, 2), (20, 5000, 3), (12, 40_000, 5), (16, 9000, 1),
                                        (6, 70_000, 1), (10, 30_000, 40)])
def test_sample_ties(dtype, B, V, values):
    """Few different logits: the cuts fall between equal ones, by number."""
    g = np.random.default_rng(V + values)
    x = _rounded(g.integers(0, values, (B, V)) * 0.5 - 1.0, dtype)
    x[g.random((B, V)) < 0.1] = -np.inf
    x[:, 0] = -1.0
    x[x == 0] = g.choice([0.0, -0.0], int((x == 0).sum()))
    u = g.random(B).astype(np.float32)
    t, k, p, m = _settings(B, g, V)
    for args in ((t, k), (t, None, p), (t, k, p), (t, k, p, m), (None, np.maximum(k, V // 3))):
        _check(x, u, *args, dtype=dtype, what=(dtype, V, values))


def test_sample_settings_at_their_limits():
    import torch
    lda = _lda()
    nan, inf = float("nan"), float("inf")
    g = np.random.default_rng(7)
    V = 3000
    row = g.normal(0, 2, V)
    row[17] = 9.0
    rows, u, t, k, p, m = [], [], [], [], [], []

    def add(x=row, at=0.6, heat=1.0, count=0, share=1.0, floor=0.0):
        for to, v in zip((rows, u, t, k, p, m), (x, at, heat, count, share, floor)):
            to.append(v)
    for at in (0.0, -0.0, 1e-30, 2.0 ** -24, 1 - 2.0 ** -24):
        add(at=at)
        add(at=at, count=5)
        add(at=at, share=0.9)
    for heat in (0.0, -1.0, 1e-45, 1e-30, 0.01, 1e4, 1e30, 3e38):
        add(heat=heat)
        add(heat=heat, count=7, share=0.5)
        add(heat=heat, share=0.999)
    for count in (-5, 0, 1, 2, V - 1, V, V + 1, 2 ** 31 - 1, -2 ** 31):
        add(count=count)
    for share in (0.0, -1.0, 1e-30, 1 - 2.0 ** -24, 1.0, 2.0, inf, nan):
        add(share=share)
        add(share=share, count=9)
    for floor in (0.0, -1.0, 1e-30, 0.999, 1.0, 2.0, inf, nan):
        add(floor=floor)
    masked = np.full(V, -inf)
    add(masked)
    one = masked.copy()
    one[V - 1] = -1e30
    add(one)
    add(one, count=5, share=0.1, floor=0.5)
    low = np.full(V, -3.4028234663852886e38)
    add(low)
    add(low, count=10)
    low = low.copy()
    low[5] = 3.4028234663852886e38
    add(low)
    for count in (0, 1, 3):
        many = row.copy()
        many[[3, 50, 999]] = inf
        many[::5] = nan
        many[3] = inf
        add(many, count=count)
        add(many, count=count, share=0.4)
    add(np.full(V, nan))
    lists = [np.array(a, dtype=np.float32) for a in (u, t, p, m)]
    x = np.stack(rows).astype(np.float32).astype(float)
    _check(x, lists[0], lists[1], np.array(k, dtype=np.int64).astype(np.int32), lists[2], lists[3])
    # u outside [0, 1)
    x = torch.from_numpy(np.tile(row, (4, 1))).float().cuda()
    z, _ = lda.sample_logits(x, torch.tensor([1.0, inf, nan, -3.0], device="cuda"),
                             top_k=torch.full((4,), 20, dtype=torch.int32, device="cuda"))
    stay = np.sort(np.argsort(-row.astype(np.float32), kind="stable")[:20])
    assert z.tolist() == [stay[-1], stay[-1], stay[0], stay[0]]
    # a temperature that is not a number
    z, prob = lda.sample_logits(x, torch.full((4,), 0.5, device="cuda"),
                                temperature=torch.full((4,), nan, device="cuda"))
    assert z.tolist() == [17] * 4 and prob.tolist() == [1.0] * 4


@pytest.mark.parametrize("dtype", TYPES)
def test_sample_rows_at_any_distance(dtype):
    import torch
    lda = _lda()
    g = np.random.default_rng(11)
    B, V = 12, 4321
    x = _rounded(g.normal(0, 3, (B, V)), dtype)
    u = _gpu(g.random(B).astype(np.float32))
    k = torch.full((B,), 40, dtype=torch.int32, device="cuda")
    p = torch.full((B,), 0.8, device="cuda")
    want = lda.sample_logits(_gpu(x, dtype), u, top_k=k, top_p=p)
    view, _ = _wide(x, dtype, 7, 3)
    out = torch.full((B,), -7, dtype=torch.int32, device="cuda"), torch.empty(B, device="cuda")
    got = lda.sample_logits(view, u, top_k=k, top_p=p, out=out)
    assert got[0] is out[0] and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one = _gpu(x[:1], dtype).expand(B, V)  # one row of logits, many numbers
    a, b = lda.sample_logits(one, u), lda.sample_logits(one.contiguous(), u)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_sample_shares():
    """Over evenly spread numbers each token is chosen as often as its share says, to one."""
    import torch
    lda = _lda()
    n = 20_000
    x = torch.randn(1, 50, device="cuda")
    u = (torch.arange(n, device="cuda") + 0.5) / n
    z, prob = lda.sample_logits(x.expand(n, 50), u.float())
    counts = torch.bincount(z.long(), minlength=50)
    want = torch.softmax(x[0].double(), 0) * n
    assert float((counts - want).abs().max()) <= 1.01
    assert bool((z[1:] >= z[:-1]).all())


# ---- together, on streams, in graphs


def _chain_of_calls(lda, x, res, w, table, scale, u, k, p):
    q, s, h = lda.add_norm_int8(x, w, residual=res)
    logits = lda.project_int8(q, s, table, scale)
    return (h, logits, *lda.sample_logits(logits, u, top_k=k, top_p=p))


def _chain_inputs(N=33, D=520, V=5003):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)

    def draw(*shape):
        return torch.randn(shape, device="cuda", generator=g)
    table = draw(V, D)
    import paper_1505_03851_amd as lda
    return (draw(N, D).bfloat16(), draw(N, D).bfloat16(), draw(D),
            *lda.quantise_rows(table), torch.rand(N, device="cuda", generator=g),
            torch.full((N,), 30, dtype=torch.int32, device="cuda"),
            torch.full((N,), 0.9, device="cuda")), table


def test_chain():
    """From activations to tokens, as an answering program calls it."""
    lda = _lda()
    args, table = _chain_inputs()
    x, res, w, qt, st, u, k, p = args
    h, logits, z, prob = _chain_of_calls(lda, *args)
    y, _ = ref.norm(_np(x), _np(w), 1e-6, _np(res))
    real, step = ref.quantise(y)
    q, s, _ = lda.add_norm_int8(x, w, residual=res)
    assert np.abs(_np(q) - real).max() <= 0.5 + 127 * (_chain(520) + 20) * EPS
    want, _ = ref.project(_np(q), _np(s), _np(qt), _np(st))
    _close(_np(logits), want, np.abs(want) * 4 * EPS, "bfloat16")
    _check(_np(logits), _np(u).astype(np.float32), None, _np(k), _np(p).astype(np.float32),
           view=logits)
    # the 8 bits cost what their steps say: half a step of each factor, at random
    off = _np(logits) - y @ _np(table).T
    d = table.shape[1]
    rms = np.sqrt(d * ((step[:, None] ** 2 / 12) * (_np(table) ** 2).mean()
                       + (_np(st) ** 2 / 12)[None, :] * (y ** 2).mean()))
    assert np.abs(off).max() < 8 * rms.max() + np.abs(want).max() * 2.0 ** -8


def test_chain_on_a_stream_and_in_a_graph():
    import torch
    lda = _lda()
    args, _ = _chain_inputs()
    want = [t.clone() for t in _chain_of_calls(lda, *args)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    x, res, w, table, scale, u, k, p = args
    q, s, h = lda.add_norm_int8(x, w, residual=res, stream=side)
    logits = lda.project_int8(q, s, table, scale, stream=side)
    z, prob = lda.sample_logits(logits, u, top_k=k, top_p=p, stream=side)
    side.synchronize()
    for a, b in zip((h, logits, z, prob), want):
        assert torch.equal(a, b)
    dy = torch.randn_like(x)
    grads = [t.clone() for t in lda.norm_grad(dy, h, w, residual_grad=res)]
    for _ in range(2):  # two graphs, each with its own memory
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = _chain_of_calls(lda, *args)
            back = lda.norm_grad(dy, got[0], w, residual_grad=res)
        for _ in range(4):
            for t in (*got, *back):
                t.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            _chain_of_calls(lda, *args)  # eager work between the replays
            for a, b in zip((*got, *back), (*want, *grads)):
                assert torch.equal(a, b)


def test_gradients_are_refused_and_writes_are_marked():
    import torch
    lda = _lda()
    x = torch.randn(4, 64, device="cuda", requires_grad=True)
    d, w = torch.randn(4, 64, device="cuda"), torch.randn(64, device="cuda")
    for call in (lambda: lda.add_norm(x, w), lambda: lda.add_norm_int8(x, w),
                 lambda: lda.add_norm(d, w, residual=x), lambda: lda.norm_grad(x, d, w),
                 lambda: lda.norm_grad(d, d, w, residual_grad=x), lambda: lda.quantise_rows(x),
                 lambda: lda.add_norm(d, w.clone().requires_grad_())):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    for out in (torch.empty_like(d),):
        saved = out._version
        lda.add_norm(d, w, out=out)
        assert out._version > saved
    total = torch.empty_like(w)
    saved = total._version
    lda.norm_grad(d, d, w, weight_out=total)
    assert total._version > saved
    lda.sample_logits(x, torch.rand(4, device="cuda"))  # (a token has no gradient)


def test_binding_refusals():
    import torch
    lda = _lda()
    dev = dict(device="cuda")
    x, w = torch.randn(4, 64, **dev), torch.randn(64, **dev)
    q, s = lda.quantise_rows(x)
    u = torch.rand(4, **dev)
    bad = [
        (ValueError, lambda: lda.add_norm(x, w[:63])),
        (TypeError, lambda: lda.add_norm(x, w.double())),
        (TypeError, lambda: lda.add_norm(x.double(), w)),
        (ValueError, lambda: lda.add_norm(x, w, residual=x[:3])),
        (TypeError, lambda: lda.add_norm(x, w, residual=x.bfloat16())),
        (ValueError, lambda: lda.add_norm(x.t(), torch.randn(4, **dev))),
        (ValueError, lambda: lda.add_norm(x, w, out=x[:1].expand(4, 64))),
        (ValueError, lambda: lda.add_norm(x.cpu(), w)),
        (ValueError, lambda: lda.add_norm(x, w.cpu())),
        (lda.LdaError, lambda: lda.add_norm(x, w, eps=0.0)),
        (TypeError, lambda: lda.add_norm_int8(x, w, out=(x, s))),
        (ValueError, lambda: lda.add_norm_int8(x, w, out=(q, s[:3]))),
        (ValueError, lambda: lda.norm_grad(x, x[:3], w)),
        (ValueError, lambda: lda.norm_grad(x, x, w, accumulate=True)),
        (TypeError, lambda: lda.norm_grad(x, x, w, weight_out=w.bfloat16())),
        (lda.LdaError, lambda: lda.norm_grad(x.repeat(20, 1), x.repeat(20, 1), w,
                                             workspace=torch.empty(8, dtype=torch.uint8, **dev))),
        (TypeError, lambda: lda.quantise_rows(q)),
        (TypeError, lambda: lda.project_int8(x, s, q, s)),
        (TypeError, lambda: lda.project_int8(q, s, x, s)),
        (ValueError, lambda: lda.project_int8(q, s, q[:, :60], s)),
        (ValueError, lambda: lda.project_int8(q, s[:3], q, s)),
        (ValueError, lambda: lda.project_int8(q, s, q, s[:3])),
        (ValueError, lambda: lda.project_int8(q, s, q, s, bias=s[:3])),
        (TypeError, lambda: lda.project_int8(q, s, q, s, dtype=torch.float64)),
        (TypeError, lambda: lda.project_int8(q, s, q, s, dtype=torch.float16, out=torch.empty(4, 4, **dev))),
        (ValueError, lambda: lda.project_int8(q, s, q, s, out=torch.empty(4, 5, **dev))),
        (ValueError, lambda: lda.project_int8(q, s, q.t(), torch.rand(64, **dev))),
        (TypeError, lambda: lda.sample_logits(x.double(), u)),
        (ValueError, lambda: lda.sample_logits(x, u[:3])),
        (TypeError, lambda: lda.sample_logits(x, u, top_k=u)),
        (TypeError, lambda: lda.sample_logits(x, u, top_p=u.half())),
        (ValueError, lambda: lda.sample_logits(x, u, min_p=u.cpu())),
    ]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            print("not refused:", i)
