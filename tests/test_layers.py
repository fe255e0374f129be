"""The norm, the 8-bit rows and product, and the sampling on the CPU: the C ABI's refusals
(before any HIP call), the binding's, and the oracle's own definitions."""
import numpy as np
import pytest

from oracle import layers as ref

A = 4096  # an aligned stand-in address, never read by a refused call
F32, BF16, F16, I8 = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    from paper_1505_03851_amd import _lib
    return _lib.load()


@pytest.fixture(scope="module")
def st():
    from paper_1505_03851_amd._lib import STATUS
    return {k[8:]: v for k, v in STATUS.items() if k != "LDA_OK"}


def norm(lib, x=A, ldx=16, r=A, ldr=16, w=A, out=A, ldo=16, total=2 * A, ldt=16, scale=A, N=10, D=16,
         dtype=F32, wt=F32, ot=F32, eps=1e-6):
    return lib.lda_add_norm(x, ldx, r, ldr, w, out, ldo, total, ldt, scale, N, D, dtype, wt, ot,
                            eps, None)


def grad(lib, g=A, ldg=16, h=A, ldh=16, r=A, ldr=16, w=A, dx=A, ldx=16, dw=A, N=10, D=16,
         dtype=F32, wt=F32, eps=1e-6, ws=A, size=1 << 30):
    return lib.lda_norm_grad(g, ldg, h, ldh, r, ldr, w, dx, ldx, dw, N, D, dtype, wt, eps, 0, ws,
                             size, None)


def quantise(lib, x=A, ldx=16, q=A, ldq=16, scale=A, N=10, D=16, dtype=F32):
    return lib.lda_quantise_rows(x, ldx, q, ldq, scale, N, D, dtype, None)


def project(lib, q=A, ldq=16, s=A, w=A, ldw=16, ws=A, b=A, out=A, ldo=8, M=10, N=8, K=16,
            dtype=F32):
    return lib.lda_project_int8(q, ldq, s, w, ldw, ws, b, out, ldo, M, N, K, dtype, None)


def sample(lib, x=A, ld=40, B=3, V=40, dtype=F32, u=A, t=A, k=A, p=A, m=A, z=A, prob=A):
    return lib.lda_sample_logits(x, ld, B, V, dtype, u, t, k, p, m, z, prob, None)


def test_norm_refusals(lib, st):
    for kw in (dict(N=-1), dict(D=0), dict(D=-3)):
        assert norm(lib, **kw) == st["SHAPE"], kw
    for kw in (dict(N=2 ** 33), dict(dtype=BF16, ot=F32), dict(dtype=BF16, wt=F16, ot=BF16),
               dict(dtype=F32, wt=BF16), dict(dtype=F32, ot=F16)):
        assert norm(lib, **kw) == st["UNSUPPORTED"], kw
    for kw in (dict(dtype=I8), dict(dtype=-1), dict(wt=I8), dict(ot=4), dict(ldx=-1), dict(ldr=-2),
               dict(ldo=15), dict(ldt=15), dict(ldo=15, ot=I8), dict(eps=0.0), dict(eps=-1e-6),
               dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e-60), dict(eps=1e60),
               dict(total=A)):
        assert norm(lib, **kw) == st["VALUE"], kw
    for key in ("x", "w", "out"):
        assert norm(lib, **{key: None}) == st["NULL"], key
    assert norm(lib, ot=I8, scale=None) == st["NULL"]
    for key in ("x", "r", "w", "out", "total"):
        assert norm(lib, **{key: A + 2}) == st["ALIGN"], key
        assert norm(lib, dtype=F16, wt=F16, ot=F16, **{key: A + 1}) == st["ALIGN"], key
    assert norm(lib, ot=I8, scale=A + 1) == st["ALIGN"]
    assert norm(lib, N=0, x=None, w=None, out=None) == 0


def test_norm_grad_refusals(lib, st):
    for kw in (dict(N=-1), dict(D=0)):
        assert grad(lib, **kw) == st["SHAPE"], kw
    for kw in (dict(N=2 ** 33), dict(dtype=BF16, wt=F16), dict(wt=F16)):
        assert grad(lib, **kw) == st["UNSUPPORTED"], kw
    for kw in (dict(dtype=I8), dict(wt=9), dict(ldg=-1), dict(ldh=-1), dict(ldr=-1), dict(ldx=15),
               dict(eps=0.0), dict(eps=float("nan"))):
        assert grad(lib, **kw) == st["VALUE"], kw
    for key in ("g", "h", "w", "dx", "dw"):
        assert grad(lib, **{key: None}) == st["NULL"], key
    assert grad(lib, N=100, ws=None) == st["NULL"]
    assert grad(lib, N=0, dw=None) == st["NULL"]  # dweight is cleared
    for key in ("g", "h", "r", "w", "dx", "dw"):
        assert grad(lib, **{key: A + 2}) == st["ALIGN"], key
    assert grad(lib, ws=A + 4) == st["ALIGN"]
    need = lib.lda_norm_grad_workspace_bytes(100, 16)
    assert need >= 64 and grad(lib, N=100, size=need - 1) == st["WORKSPACE"]
    assert lib.lda_norm_grad_workspace_bytes(10, 16) == 0  # a few rows need none
    for bad in ((0, 16), (-1, 16), (10, 0), (10, -1), (2 ** 33, 16)):
        assert lib.lda_norm_grad_workspace_bytes(*bad) == 0
    assert lib.lda_norm_grad_workspace_bytes(2 ** 32 - 65536, 2 ** 31 - 1) > 2 ** 40


def test_quantise_refusals(lib, st):
    for kw in (dict(N=-1), dict(D=0)):
        assert quantise(lib, **kw) == st["SHAPE"], kw
    assert quantise(lib, N=2 ** 33) == st["UNSUPPORTED"]
    for kw in (dict(dtype=I8), dict(ldx=-1), dict(ldq=15)):
        assert quantise(lib, **kw) == st["VALUE"], kw
    for key in ("x", "q", "scale"):
        assert quantise(lib, **{key: None}) == st["NULL"], key
    for kw in (dict(x=A + 2), dict(scale=A + 2), dict(x=A + 1, dtype=BF16)):
        assert quantise(lib, **kw) == st["ALIGN"], kw
    assert quantise(lib, N=0, x=None, q=None, scale=None) == 0


def test_project_refusals(lib, st):
    for kw in (dict(M=-1), dict(N=0), dict(K=0), dict(K=-5)):
        assert project(lib, **kw) == st["SHAPE"], kw
    for kw in (dict(M=2 ** 33), dict(K=131072, ldq=131072, ldw=131072)):
        assert project(lib, **kw) == st["UNSUPPORTED"], kw
    for kw in (dict(dtype=I8), dict(ldq=-1), dict(ldw=-1), dict(ldo=7)):
        assert project(lib, **kw) == st["VALUE"], kw
    for key in ("q", "s", "w", "ws", "out"):
        assert project(lib, **{key: None}) == st["NULL"], key
    for key in ("s", "ws", "b", "out"):
        assert project(lib, **{key: A + 2}) == st["ALIGN"], key
    assert project(lib, dtype=BF16, out=A + 1) == st["ALIGN"]
    assert project(lib, M=0, q=None, s=None, w=None, ws=None, out=None) == 0


def test_sample_refusals(lib, st):
    for kw in (dict(B=-1), dict(V=0)):
        assert sample(lib, **kw) == st["SHAPE"], kw
    assert sample(lib, B=2 ** 31) == st["UNSUPPORTED"]
    for kw in (dict(dtype=I8), dict(dtype=-1), dict(ld=-1)):
        assert sample(lib, **kw) == st["VALUE"], kw
    for key in ("x", "u", "z", "prob"):
        assert sample(lib, **{key: None}) == st["NULL"], key
    for key in ("x", "u", "t", "k", "p", "m", "z", "prob"):
        assert sample(lib, **{key: A + 2}) == st["ALIGN"], key
    assert sample(lib, B=0, x=None, u=None, z=None, prob=None) == 0


def test_binding_refuses_cpu_tensors():
    import torch

    import paper_1505_03851_amd as lda
    x, v = torch.zeros(2, 8), torch.zeros(8)
    q = torch.zeros(2, 8, dtype=torch.int8)
    for call in (lambda: lda.add_norm(x, v), lambda: lda.add_norm_int8(x, v),
                 lambda: lda.norm_grad(x, x, v), lambda: lda.quantise_rows(x),
                 lambda: lda.project_int8(q, v[:2], q, v[:2]), lambda: lda.sample_logits(x, v[:2])):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(TypeError):
        lda.add_norm([1.0], v)
    assert lda.norm_grad_workspace_bytes(5, 2 ** 31) == 0


# ---- the oracle


def test_oracle_gradient_against_differences():
    g = np.random.default_rng(1)
    N, D, eps = 3, 7, 1e-3
    x, r, w = g.normal(size=(N, D)), g.normal(size=(N, D)), g.normal(size=D)
    dy, dh = g.normal(size=(N, D)), g.normal(size=(N, D))

    def loss(x, w):
        y, h = ref.norm(x, w, eps, r)
        return (y * dy).sum() + (h * dh).sum()
    dx, dw, _, _ = ref.norm_grad(dy, x + r, w, eps, dh)
    step = 1e-6
    for i in np.ndindex(N, D):
        e = np.zeros((N, D))
        e[i] = step
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * step) - dx[i]) < 1e-7
    for i in range(D):
        e = np.zeros(D)
        e[i] = step
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * step) - dw[i]) < 1e-7


def test_oracle_sample_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert [ref.sample(x, u)[0] for u in (0.0, 0.05, 0.15, 0.45, 0.55, 0.65, 0.75, 0.99, 1.0)] == [
        0, 0, 1, 1, 2, 2, 3, 3, 3]
    # two stay: 1 and 3
    assert [ref.sample(x, u, top_k=2)[0] for u in (0.0, 0.5, 0.6, 0.99)] == [1, 1, 3, 3]
    assert ref.sample(x, 0.9, top_k=1)[:2] == (1, 1.0)
    # 0.65 is reached by two, 0.75 by three, 0.3 by one
    assert [ref.sample(x, 0.99, top_p=p)[0] for p in (0.3, 0.65, 0.75, 0.95)] == [1, 3, 3, 3]
    assert abs(ref.sample(x, 0.0, top_p=0.75)[1] - 4 / 9) < 1e-12
    # of the likeliest two, half of what they hold is one
    assert ref.sample(x, 0.99, top_k=2, top_p=0.5)[:2] == (1, 1.0)
    assert ref.sample(x, 0.0, min_p=0.6)[0] == 1 and ref.sample(x, 0.99, min_p=0.6)[0] == 3
    # equal logits: the lower numbers first
    assert [ref.sample(np.zeros(6), u, top_k=3)[0] for u in (0.0, 0.4, 0.99)] == [0, 1, 2]
    assert ref.sample(x, 0.99, temperature=0.0)[:2] == (1, 1.0)
    assert ref.sample(np.full(3, -np.inf), 0.5)[:2] == (-1, 0.0)
    y = np.array([0.0, np.inf, 1.0, np.inf, np.nan])
    assert [ref.sample(y, u)[0] for u in (0.0, 0.49, 0.5, 0.99)] == [1, 1, 3, 3]


def test_oracle_quantise_by_hand():
    q, s = ref.quantise(np.array([[1.0, -2.0, 0.5], [0, 0, 0], [np.nan, 1, 2], [1, np.inf, 0]]))
    assert np.array_equal(q[0], [63.5, -127, 31.75]) and s[0] == 2 / 127
    assert not q[1:].any() and s[1] == 0 and np.isnan(s[2:]).all()
