"""The norm, the 8-bit rows and product and the sampling at the ends of their ranges: offsets past 32
bits, more rows than a launch takes, rows and settings that make the sampling narrow down several
times, two streams at once."""
import numpy as np
import pytest

from oracle import layers as ref
from test_layers_gpu import _check, _whole
from test_tokens_gpu import EPS, _close, _gpu, _lda, _np, _rounded

pytestmark = pytest.mark.gpu


# ---- offsets past 32 bits


def test_norm_rows_past_32_bits():
    """Rows 2^31 elements apart: the last starts at element 3 2^31."""
    import torch
    lda = _lda()
    N, D, apart = 4, 100, 2 ** 31
    buf = torch.zeros(3 * apart + D, dtype=torch.float16, device="cuda")
    rows = torch.as_strided(buf, (N, D), (apart, 1))
    x = torch.randn(N, D, device="cuda").half()
    rows.copy_(x)
    w = torch.randn(D, device="cuda")
    y, h = lda.add_norm(rows, w, residual=rows)
    want = lda.add_norm(x, w, residual=x)
    assert torch.equal(y, want[0]) and torch.equal(h, want[1])
    a, b = lda.quantise_rows(rows), lda.quantise_rows(x)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    a, b = lda.norm_grad(rows, rows, w, residual_grad=rows), lda.norm_grad(x, x, w, residual_grad=x)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    lda.norm_grad(x, x, w, residual_grad=x, out=rows)
    assert torch.equal(rows, b[0]) and int(buf.count_nonzero()) <= N * D
    lda.add_norm(x, w, out=rows)
    assert torch.equal(rows, lda.add_norm(x, w))


@pytest.mark.parametrize("M,N,K", [(3, 40, 100), (20, 4, 64), (70, 130, 192)])
def test_project_rows_past_32_bits(M, N, K):
    """Lines and output rows far apart."""
    import torch
    lda = _lda()
    g = np.random.default_rng(M)
    q, w = _gpu(_whole(g, (M, K))), _gpu(_whole(g, (N, K)))
    s, ws = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    want = lda.project_int8(q, s, w, ws)
    apart = 2 ** 32 // (M - 1) // 16 * 16 + 16  # the last line past 2^32 bytes
    buf = torch.zeros((M - 1) * apart + K, dtype=torch.int8, device="cuda")
    far = torch.as_strided(buf, (M, K), (apart, 1))
    far.copy_(q)
    assert torch.equal(lda.project_int8(far, s, w, ws), want)
    del buf, far
    apart = 2 ** 32 // (N - 1) // 16 * 16 + 16
    buf = torch.zeros((N - 1) * apart + K, dtype=torch.int8, device="cuda")
    far = torch.as_strided(buf, (N, K), (apart, 1))
    far.copy_(w)
    assert torch.equal(lda.project_int8(q, s, far, ws), want)
    del buf, far
    apart = 2 ** 32 // (M - 1) + 3
    buf = torch.zeros((M - 1) * apart + N, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(buf, (M, N), (apart, 1))
    lda.project_int8(q, s, w, ws, out=far)
    assert torch.equal(far, want) and int(buf.count_nonzero()) <= M * N


def test_project_output_past_32_bits():
    """More than 2^32 sums: the last rows against the same rows alone."""
    import torch
    lda = _lda()
    M, N, K = 70_000, 65_000, 64
    q = torch.randint(-128, 128, (M, K), dtype=torch.int8, device="cuda")
    w = torch.randint(-128, 128, (N, K), dtype=torch.int8, device="cuda")
    s, ws = torch.rand(M, device="cuda"), torch.rand(N, device="cuda")
    y = lda.project_int8(q, s, w, ws)
    for at in (0, 33_000, 66_000, M - 300):
        rows = lda.project_int8(q[at:at + 300], s[at:at + 300], w, ws)
        assert torch.equal(y[at:at + 300], rows)


def test_sample_rows_past_32_bits():
    import torch
    lda = _lda()
    B, V, apart = 3, 5000, 2 ** 32
    buf = torch.zeros(2 * apart + V, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(buf, (B, V), (apart, 1))
    x = torch.randn(B, V, device="cuda").bfloat16()
    rows.copy_(x)
    u, p = torch.rand(B, device="cuda"), torch.full((B,), 0.9, device="cuda")
    a, b = lda.sample_logits(rows, u, top_p=p), lda.sample_logits(x, u, top_p=p)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- many rows


def test_more_rows_than_a_launch():
    """Norms and 8-bit rows are launched 2^22 at a time, choices 2^20, and the direct product's
    workgroups stride from 2^20 tiles on."""
    import torch
    lda = _lda()
    N, D = 2 ** 22 + 5, 9
    x = torch.randn(N, D, device="cuda")
    r = torch.randn(N, D, device="cuda")
    w = torch.randn(D, device="cuda")
    tail = slice(N - 7, N)
    y, h = lda.add_norm(x, w, residual=r)
    want = lda.add_norm(x[tail], w, residual=r[tail])
    assert torch.equal(y[tail], want[0]) and torch.equal(h[tail], want[1])
    q, s, h = lda.add_norm_int8(x, w, residual=r)
    want = lda.add_norm_int8(x[tail], w, residual=r[tail])
    assert torch.equal(q[tail], want[0]) and torch.equal(s[tail], want[1]) and torch.equal(h[tail], want[2])
    q, s = lda.quantise_rows(x)
    want = lda.quantise_rows(x[tail])
    assert torch.equal(q[tail], want[0]) and torch.equal(s[tail], want[1])
    dx, dw = lda.norm_grad(r, x, w)
    assert torch.equal(dx[tail], lda.norm_grad(r[tail], x[tail], w)[0])
    unit = x.double() / (x.double().square().mean(1, keepdim=True) + 1e-6).sqrt()
    terms = r.double() * unit
    bound = terms.abs().sum(0) * (N // 256 + 80 + 40) * EPS
    assert bool(((dw.double() - terms.sum(0)).abs() <= bound).all())
    B = 2 ** 20 + 3
    u = torch.rand(B, device="cuda")
    z, prob = lda.sample_logits(x[:B], u, top_k=torch.full((B,), 4, dtype=torch.int32, device="cuda"))
    a = lda.sample_logits(x[B - 5:B], u[B - 5:], top_k=torch.full((5,), 4, dtype=torch.int32, device="cuda"))
    assert torch.equal(z[B - 5:], a[0]) and torch.equal(prob[B - 5:], a[1]) and int(z.min()) >= 0
    M, N, K = 70_000, 4000, 8  # lines shorter than a piece: 1.1M tiles of the direct product
    q = torch.randint(-128, 128, (M, K), dtype=torch.int8, device="cuda")
    w = torch.randint(-128, 128, (N, K), dtype=torch.int8, device="cuda")
    ones = torch.ones(M, device="cuda")
    y = lda.project_int8(q, ones, w, ones[:N], dtype=torch.float32)
    assert torch.equal(y, q.float() @ w.float().t())  # (whole numbers below 2^24)


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 63, 64, 65, 129, 255, 256, 257])
def test_project_every_tile(M):
    """Each tile's shape at its edges, with lines that are aligned and that are not."""
    import torch
    lda = _lda()
    g = torch.Generator(device="cuda").manual_seed(M)
    for N, K in ((1, 16), (31, 1024), (33, 1040), (64, 2000), (500, 528), (4097, 512), (4100, 1030),
                 (16_400, 1024), (30_000, 130), (65_600, 48)):
        q = torch.randint(-128, 128, (M, K), dtype=torch.int8, device="cuda", generator=g)
        w = torch.randint(-128, 128, (N, K), dtype=torch.int8, device="cuda", generator=g)
        s = torch.rand(M, device="cuda", generator=g)
        ws = torch.rand(N, device="cuda", generator=g)
        want = (q.double() @ w.double().t()) * s.double()[:, None] * ws.double()
        for a, b in ((q, w), (torch.cat([q, q], 1)[:, :K], torch.cat([w, w[:, :5]], 1)[:, :K])):
            got = lda.project_int8(a, s, b, ws, dtype=torch.float32)
            bound = want.abs() * 5 * EPS
            assert bool(((got.double() - want).abs() <= bound).all()), (M, N, K)


# ---- the sampling's ways


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("spread", [1e-6, 0.01, 0.3, 3.0, 300.0])
def test_sample_at_any_spread(dtype, spread):
    """Logits close together or far apart: bins that hold too many, lists of every length."""
    g = np.random.default_rng(int(spread * 1e6) % 1000)
    for V in (1025, 20_000, 90_000):
        B = 8
        x = _rounded(g.normal(0, spread, (B, V)) + g.choice([0.0, 5.0, -40.0], (B, 1)), dtype)
        u = g.random(B).astype(np.float32)
        t = g.choice([1.0, 0.5, 20.0], B).astype(np.float32)
        k = np.array([0, 1, 40, 300, 512, 513, 1000, V // 2], dtype=np.int32)
        p = g.choice([0.2, 0.9, 0.99, 1.0], B).astype(np.float32)
        m = g.choice([0.0, 0.01, 0.5], B).astype(np.float32)
        for args in ((t, k), (t, None, p), (t, k, p), (t, k, p, m), (t, None, None, m)):
            _check(x, u, *args, dtype=dtype, what=(dtype, spread, V))


def test_sample_of_the_largest_range():
    """Logits over all of float's range at a temperature to match, more than a list in each bin."""
    g = np.random.default_rng(8)
    B, V = 6, 6000
    x = (g.uniform(-1, 1, (B, V)) * 3.3e38).astype(np.float32).astype(float)
    u = g.random(B).astype(np.float32)
    t = np.array([1e37, 1e38, 3e38, 1e30, 3e38, 3e38], dtype=np.float32)
    p = np.array([0.9, 0.5, 0.99, 0.5, 1.0, 0.3], dtype=np.float32)
    k = np.array([0, 0, 0, 0, 3000, 3000], dtype=np.int32)
    _check(x, u, t, None, p)
    _check(x, u, t, k, p)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [3000, 20_000, 150_000])
def test_sample_where_two_cuts_meet(dtype, V):
    """min_p before the place where top_p ends, at it and after it, a little and by far, with
    few and many logits around it, and with a top_k that ends before both or after them."""
    g = np.random.default_rng(V)
    B = 42
    p = g.uniform(0.03, 0.99, B).astype(np.float32)
    # the weights of logits that are evenly spaced: what top_p leaves ends at a weight of 1 - p
    m = np.exp(np.log1p(-p) + np.resize([-3, -0.3, -0.02, 0.0, 0.02, 0.3, 3], B))
    m = np.minimum(m, 1.0).astype(np.float32)
    t, u = np.ones(B, dtype=np.float32), g.random(B).astype(np.float32)
    x = _rounded(g.uniform(-16, 0, (B, V)), dtype)
    x[:, g.integers(0, V, V // 5)] = -np.inf
    args = dict(dtype=dtype, what=(dtype, V))
    _check(x, u, t, None, p, m, **args)
    _check(x, g.random(B).astype(np.float32), t, (g.uniform(0.01, 0.3, B) * V).astype(np.int32),
           p, m, **args)
    # half of all logits at one place, most often where one of the two ends
    at = _rounded(np.log(np.where(g.random(B) < 0.5, m, 1 - p)), dtype)
    x = np.where(g.random((B, V)) < 0.5, at[:, None], x)
    _check(x, u, t, None, p, m, **args)


def test_sample_min_p_between_two_bins():
    """A min_p whose logit is, but for 1e-9 of it, the border between two of the bins that
    top_p sums the weights in, half way between two of the 1,024 evenly spaced logits from
    the largest to the lowest."""
    border = (np.arange(64, 1023) + 0.5) / 64
    t = (border / np.log(2)).astype(np.float32)  # exp(-border / t) = 0.5
    off = np.abs(t.astype(float) * np.log(2) / border - 1)
    t = t[off < 6e-10]
    B, V = len(t), 2500
    assert B >= 5
    g = np.random.default_rng(23)
    x = _rounded(-g.uniform(0, 1023 / 64, (B, V)), "float32")
    x[:, 7], x[:, 1900] = 0.0, -1023 / 64
    m = np.full(B, 0.5, dtype=np.float32)
    for p in (0.999, 0.9, 0.6, 0.3):
        _check(x, g.random(B).astype(np.float32), t, None, np.full(B, p, dtype=np.float32), m,
               what=p)


def test_sample_at_extreme_temperatures():
    """An infinite temperature makes all logits' weights one, the smallest leaves the largest."""
    g = np.random.default_rng(5)
    B, V = 24, 5000
    x = _rounded(g.normal(0, 3, (B, V)), "float32")
    t = np.resize(np.array([np.inf, 3e38, 1e-30, 1e-45], dtype=np.float32), B)
    u = g.random(B).astype(np.float32)
    p = np.resize(np.array([0.3, 0.77, 1.0], dtype=np.float32), B)
    m = np.repeat(np.array([0.0, 0.4, 1.0], dtype=np.float32), B // 3)
    k = np.repeat(np.array([0, 700, 3000, 0], dtype=np.int32), B // 4)
    for args in ((t, None, p), (t, None, p, m), (t, k, p, m), (t, k)):
        _check(x, u, *args, what=len(args))


@pytest.mark.parametrize("V", [1024, 1025, 8192, 8193, 32_768, 32_769, 65_536, 65_537, 131_072, 131_080])
def test_sample_row_lengths(V):
    """Around the lengths where rows fill lists, chunks and registers: every choice near the end."""
    import torch
    lda = _lda()
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.full((4, V), -9.0, dtype=dtype, device="cuda")
        x[:, -1] = 3.0
        x[1, -8:] = 3.0
        x[2, 0] = 3.0
        u = torch.tensor([0.999999, 0.9999, 0.999999, 0.0], device="cuda")
        z, _ = lda.sample_logits(x, u)
        assert z.tolist() == [V - 1, V - 1, V - 1, 0]
        z, _ = lda.sample_logits(x, u, top_p=torch.full((4,), 0.2, device="cuda"))
        assert z[0] == V - 1 and z[2] in (0, V - 1) and V - 8 <= int(z[1]) < V


def test_two_streams():
    """Calls on two streams at once, each with its own tensors."""
    import torch
    lda = _lda()
    g = torch.Generator(device="cuda").manual_seed(2)
    sets = []
    for i in range(2):
        x = torch.randn(300 + i, 1000, device="cuda", generator=g).bfloat16()
        w = torch.randn(1000, device="cuda", generator=g)
        table = lda.quantise_rows(torch.randn(5000, 1000, device="cuda", generator=g))
        u = torch.rand(300 + i, device="cuda", generator=g)
        p = torch.full((300 + i,), 0.8, device="cuda")
        sets.append((x, w, table, u, p))

    def run(x, w, table, u, p):
        q, s, h = lda.add_norm_int8(x, w, residual=x)
        logits = lda.project_int8(q, s, *table)
        return (*lda.sample_logits(logits, u, top_p=p), *lda.norm_grad(x, h, w, residual_grad=x))
    want = [run(*a) for a in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for st, a in zip(streams, sets):
            with torch.cuda.stream(st):
                got.append(run(*a))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(c, d) for c, d in zip(a, b))


def test_same_bits_every_time():
    import torch
    lda = _lda()
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(5000, 1500, device="cuda", generator=g)
    w = torch.randn(1500, device="cuda", generator=g)
    dy = torch.randn(5000, 1500, device="cuda", generator=g)
    first = lda.norm_grad(dy, x, w)
    logits = torch.randn(40, 60_000, device="cuda", generator=g).bfloat16()
    u = torch.rand(40, device="cuda", generator=g)
    k = torch.randint(0, 2000, (40,), dtype=torch.int32, device="cuda", generator=g)
    p = torch.rand(40, device="cuda", generator=g)
    drawn = lda.sample_logits(logits, u, top_k=k, top_p=p)
    for _ in range(5):
        again = lda.norm_grad(dy, x, w)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
        more = lda.sample_logits(logits, u, top_k=k, top_p=p)
        assert torch.equal(more[0], drawn[0]) and torch.equal(more[1], drawn[1])


def test_sums_that_are_large():
    """Rows whose squares come near float's range, and a residual that cancels."""
    import torch
    lda = _lda()
    D = 500
    x = torch.full((2, D), 2.0 ** 58, device="cuda")
    w = torch.ones(D, device="cuda")
    y = lda.add_norm(x, w)
    assert bool(((y - 1).abs() <= (38 / 2 + 8) * 2 * EPS).all())
    y, h = lda.add_norm(x, w, residual=-x)
    assert not y.any() and not h.any()
    want, _ = ref.norm(_np(x) * 2.0 ** -70, _np(w), 1e-6)
    got = lda.add_norm(x * 2.0 ** -70, w)
    _close(_np(got), want, np.abs(want) * (38 / 2 + 8) * EPS, "float32")
