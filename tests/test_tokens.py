"""The token operators on the CPU: the C ABI's refusals (before any HIP call),
the binding's, and the oracle's own definitions."""
import ctypes

import numpy as np
import pytest

from oracle import tokens as ref

A = 4096  # an aligned stand-in address, never read by a refused call
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_1505_03851_amd import _lib
    return _lib.load()


@pytest.fixture(scope="module")
def st():
    from paper_1505_03851_amd._lib import STATUS
    return {k[8:]: v for k, v in STATUS.items() if k != "LDA_OK"}


def embed(lib, table=A, ldt=16, ids=A, out=A, ldo=16, N=10, V=5, D=16, dtype=F32, scale=1.0,
          p=0.0):
    return lib.lda_embed(table, ldt, ids, out, ldo, N, V, D, dtype, scale, p, 1, 0, None)


def grad(lib, g=A, ldg=16, ids=A, out=A, ldo=16, N=10, V=5, D=16, gt=F32, ot=F32, p=0.0,
         ws=A, size=1 << 30):
    return lib.lda_embed_grad(g, ldg, ids, out, ldo, N, V, D, gt, ot, 1.0, p, 1, 0, 0, ws, size,
                              None)


def drop(lib, x=A, ldx=16, out=A, ldo=16, rows=10, cols=16, dtype=F32, p=0.5):
    return lib.lda_dropout(x, ldx, out, ldo, rows, cols, dtype, p, 1, 0, None)


def test_embed_refusals(lib, st):
    for kw in (dict(N=-1), dict(V=0), dict(V=-3), dict(D=0)):
        assert embed(lib, **kw) == st["SHAPE"], kw
    assert embed(lib, N=2 ** 33) == st["UNSUPPORTED"]
    for kw in (dict(dtype=3), dict(dtype=-1), dict(p=1.0), dict(p=-0.1), dict(p=float("nan")),
               dict(ldt=-1), dict(ldo=15), dict(ldo=0)):
        assert embed(lib, **kw) == st["VALUE"], kw
    for key in ("table", "ids", "out"):
        assert embed(lib, **{key: None}) == st["NULL"], key
        assert embed(lib, **{key: A + 2}) == st["ALIGN"], key
    for dtype in (BF16, F16):
        assert embed(lib, table=A + 1, dtype=dtype) == st["ALIGN"]
    assert embed(lib, N=0, table=None, ids=None, out=None) == 0


def test_embed_grad_refusals(lib, st):
    for kw in (dict(N=-1), dict(V=0), dict(D=-2)):
        assert grad(lib, **kw) == st["SHAPE"], kw
    assert grad(lib, N=2 ** 31) == st["UNSUPPORTED"]
    assert grad(lib, gt=F32, ot=BF16) == st["UNSUPPORTED"]
    assert grad(lib, gt=F16, ot=BF16) == st["UNSUPPORTED"]
    for kw in (dict(gt=7), dict(ot=-1), dict(p=1.5), dict(ldg=-16), dict(ldo=8)):
        assert grad(lib, **kw) == st["VALUE"], kw
    for key in ("g", "ids", "out"):
        assert grad(lib, **{key: None}) == st["NULL"], key
    assert grad(lib, N=1000, ws=None) == st["NULL"]
    for key in ("g", "ids", "out"):
        assert grad(lib, **{key: A + 2}) == st["ALIGN"], key
    assert grad(lib, ws=A + 4) == st["ALIGN"]
    assert grad(lib, N=0, out=None) == st["NULL"]  # out is cleared
    need = lib.lda_embed_grad_workspace_bytes(1000, 5, 16)
    assert need > 0 and grad(lib, N=1000, size=need - 1) == st["WORKSPACE"]


def test_embed_grad_workspace(lib):
    f = lib.lda_embed_grad_workspace_bytes
    for bad in ((0, 5, 16), (-1, 5, 16), (10, 0, 16), (10, 5, 0), (2 ** 31, 5, 16)):
        assert f(*bad) == 0, bad
    for N in (1, 7, 128):  # a few tokens need none
        assert f(N, 50_000, 64) == 0
    last = 0
    for N in (129, 1000, 4096, 4097, 70_000, 1 << 20, 2 ** 31 - 1):
        assert f(N, 50_000, 64) >= max(last, 16 * N)
        last = f(N, 50_000, 64)
    assert f(1000, 2 ** 31 - 1, 8) > 0


def test_dropout_refusals(lib, st):
    for kw in (dict(rows=-1), dict(cols=0)):
        assert drop(lib, **kw) == st["SHAPE"], kw
    for kw in (dict(rows=2 ** 33), dict(cols=2 ** 35, ldx=2 ** 35, ldo=2 ** 35)):
        assert drop(lib, **kw) == st["UNSUPPORTED"], kw
    for kw in (dict(dtype=9), dict(p=1.0), dict(p=-1e-9), dict(ldx=-1), dict(ldo=15)):
        assert drop(lib, **kw) == st["VALUE"], kw
    for key in ("x", "out"):
        assert drop(lib, **{key: None}) == st["NULL"], key
        assert drop(lib, **{key: A + 1}) == st["ALIGN"], key
    assert drop(lib, rows=0, x=None, out=None) == 0


def _rules(**kw):
    from paper_1505_03851_amd._tokens import LogitRules
    r = LogitRules()
    for k, v in kw.items():
        setattr(r, k, v)
    return ctypes.byref(r)


def penalise(lib, x=A, ld=40, out=A, ldo=40, B=3, V=40, dtype=F32, rules=None):
    return lib.lda_penalise_logits(x, ld, out, ldo, B, V, dtype, rules, None)


def draw(lib, x=A, ld=40, B=3, V=40, dtype=F32, rules=None, t=A, m=A, seed=A, pos=A, z=A, prob=A,
         ws=A, size=1 << 20):
    return lib.lda_draw_logits(x, ld, B, V, dtype, rules, t, m, seed, pos, z, prob, ws, size, None)


@pytest.mark.parametrize("fn", [penalise, draw])
def test_logits_refusals(lib, st, fn):
    for kw in (dict(B=-1), dict(V=0)):
        assert fn(lib, **kw) == st["SHAPE"], kw
    assert fn(lib, B=2 ** 31) == st["UNSUPPORTED"]
    for kw in (dict(dtype=3), dict(ld=-1)):
        assert fn(lib, **kw) == st["VALUE"], kw
    assert fn(lib, x=None) == st["NULL"]
    assert fn(lib, x=A + 2) == st["ALIGN"]
    assert fn(lib, B=0, x=None) == 0
    for name in ("history", "bias", "mask"):
        assert fn(lib, rules=_rules(**{name: A + 2})) == st["ALIGN"], name
    assert fn(lib, rules=_rules(history=A, capacity=4, ld_history=4)) == st["NULL"]  # no lengths
    assert fn(lib, rules=_rules(history=A, lengths=A, capacity=-1)) == st["SHAPE"]
    assert fn(lib, rules=_rules(history=A, lengths=A, capacity=2 ** 30 + 1,
                                ld_history=2 ** 31)) == st["UNSUPPORTED"]
    for kw in (dict(history=A, lengths=A, capacity=5, ld_history=4), dict(bias=A, ld_bias=39),
               dict(mask=A, ld_mask=1), dict(bias=A, ld_bias=-40)):
        assert fn(lib, rules=_rules(**kw)) == st["VALUE"], kw


def test_logits_own_refusals(lib, st):
    assert penalise(lib, ldo=39) == st["VALUE"]
    assert penalise(lib, out=None) == st["NULL"]
    for key in ("seed", "pos", "z", "prob"):
        assert draw(lib, **{key: None}) == st["NULL"], key
    assert draw(lib, V=40_000, ld=40_000, ws=None) == st["NULL"]
    for key in ("t", "m", "pos", "z", "prob"):
        assert draw(lib, **{key: A + 2}) == st["ALIGN"], key
    for key in ("seed", "ws"):
        assert draw(lib, **{key: A + 4}) == st["ALIGN"], key
    need = lib.lda_draw_logits_workspace_bytes(3, 40_000)
    assert need == 960 and draw(lib, V=40_000, ld=40_000, size=need - 1) == st["WORKSPACE"]
    assert lib.lda_draw_logits_workspace_bytes(2, 32_769) == 528
    assert lib.lda_draw_logits_workspace_bytes(2, 32_768) == 0  # short rows need none
    for bad in ((0, 5), (3, 0), (2 ** 31, 5)):
        assert lib.lda_draw_logits_workspace_bytes(*bad) == 0


def test_binding_refuses_cpu_tensors():
    import torch
    import paper_1505_03851_amd as lda
    x, i = torch.zeros((3, 8)), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: lda.embed(x, i), lambda: lda.embed_grad(x, i, 5),
                 lambda: lda.dropout(x, 0.5, 1), lambda: lda.penalise_logits(x),
                 lambda: lda.draw_logits(x, i.long(), i)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        lda.dropout([1.0], 0.5, 1)


# ---- the oracle's definitions


def test_oracle_keep_factor():
    """The mask keeps the rounded share, row by row and column by column."""
    from oracle.philox import philox4
    f = ref.keep_factor(300, 1003, 0.3, (7 << 32) | 9, 5)
    q = round(65536 * 0.3)
    assert set(np.unique(f)) == {0.0, 65536.0 / (65536 - q)}
    assert abs((f > 0).mean() - (1 - q / 65536)) < 5 * np.sqrt(0.21 / f.size)
    for row, col in ((0, 0), (2, 13), (299, 1002)):
        w = philox4((col // 8, row, 5, 1), (9, 7))[col % 8 // 2]
        assert (f[row, col] > 0) == ((w >> 16 if col % 2 else w & 0xFFFF) >= q)
    assert (ref.keep_factor(2, 9, 0.999999999, 1, 0) > 0).sum() < 18  # q stays below 2^16


def test_oracle_draw_follows_the_weights():
    """Frequencies of many draws against the softmax (chi-square of 30 cells:
    above 70 with probability 5e-5)."""
    g = np.random.default_rng(5)
    x = g.normal(0, 1.5, 30)
    w = np.exp((x - x.max()) / 0.8)
    n = 4000
    got = np.bincount([ref.draw(x, 0.8, 0.0, 11, i)[0] for i in range(n)], minlength=30)
    want = n * w / w.sum()
    assert ((got - want) ** 2 / want).sum() < 70
    # two groups: the group's share is drawn first
    y = np.full(1500, -30.0)
    y[[3, 1200]] = [0.0, np.log(3.0)]
    second = np.mean([ref.draw(y, 1.0, 0.0, 3, i)[0] == 1200 for i in range(n)])
    assert abs(second - 0.75) < 5 * np.sqrt(0.75 * 0.25 / n)


def test_oracle_penalise_by_hand():
    x = np.array([[2.0, -2.0, 1.0, 4.0]])
    h = np.array([[0, 1, 1, 2, 9, -1]])
    y, _ = ref.penalise(x, h, [6], [2], [2.0], [0.5], [0.25],
                        np.array([0.0, 0.0, 1.0, 0.0]), np.array([True, True, True, False]))
    # 0: prompt only; 1: prompt and one use; 2: one use; 9 and -1: no tokens
    assert y.tolist() == [[1.0, -4.0 - 0.5 - 0.25, 0.5 - 0.5 - 0.25 + 1.0, -np.inf]]
