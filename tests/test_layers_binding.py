"""The binding of the operators between a layer's last activations and the next token, on the CPU:
what a call of the library is given, with the library's call put aside."""
import ctypes

import numpy as np
import pytest


@pytest.fixture
def calls(monkeypatch):
    """The binding on CPU tensors: [(name, arguments)] of what would be launched."""
    from paper_1505_03851_amd import _layers
    made = []
    monkeypatch.setattr(_layers, "_run", lambda name, dev, *args: made.append((name, args)))
    return made


def _floats(address, n):
    return np.ctypeslib.as_array(ctypes.cast(address, ctypes.POINTER(ctypes.c_float)), (n,))


@pytest.mark.parametrize("given", [False, True])
def test_project_scale_lives_until_the_launch(monkeypatch, given):
    """A scale of several dimensions that is not contiguous is copied: the copy's memory is not to
    be handed out again, for the output above all, before the kernel is launched."""
    import weakref

    import torch

    from paper_1505_03851_amd import _layers
    scale = torch.arange(6 * 500, dtype=torch.float32).view(6, 500).t()  # [500][6]
    q = torch.zeros(500, 6, 8, dtype=torch.int8)
    w, ws = torch.zeros(5, 8, dtype=torch.int8), torch.ones(5)
    seen, launched = {}, []
    vector = _layers._vector

    def watched(t, name, *args):
        seen[name] = weakref.ref(t), t.data_ptr()
        return vector(t, name, *args)

    def run(name, dev, *args):
        alive, address = seen["scale"]
        assert alive() is not None, "the scale is freed before the launch"
        assert args[2] == address
        assert np.array_equal(_floats(args[2], 3000), scale.reshape(-1).numpy())
        launched.append(name)
    monkeypatch.setattr(_layers, "_vector", watched)
    monkeypatch.setattr(_layers, "_run", run)
    out = torch.empty(500, 6, 5) if given else None
    y = _layers.project_int8.__wrapped__(q, scale, w, ws, dtype=torch.float32, out=out)
    assert launched == ["lda_project_int8"] and y.shape == (500, 6, 5)


def test_scales_to_overwrite_that_are_not_contiguous(calls):
    """Refused as other vectors are, in the binding's words, before anything is launched."""
    import torch

    from paper_1505_03851_amd import _layers
    x, w = torch.zeros(4, 6, 8), torch.ones(8)
    q, scale = torch.zeros(4, 6, 8, dtype=torch.int8), torch.zeros(6, 4).t()
    for call in (lambda: _layers.quantise_rows.__wrapped__(x, out=(q, scale)),
                 lambda: _layers.add_norm_int8.__wrapped__(x, w, out=(q, scale))):
        with pytest.raises(ValueError, match="contiguous"):
            call()
    assert not calls
    _layers.quantise_rows.__wrapped__(x, out=(q, torch.zeros(4, 6)))
    _layers.add_norm_int8.__wrapped__(x, w, out=(q, torch.zeros(4, 6)))
    assert [name for name, _ in calls] == ["lda_quantise_rows", "lda_add_norm"]


def test_draws_over_tensors_that_require_a_gradient(calls, monkeypatch):
    """Refused where gradients are recorded, as every other tensor to overwrite is."""
    import torch

    from paper_1505_03851_amd import _layers, _tokens
    monkeypatch.setattr(_tokens, "_run", lambda name, dev, *args: calls.append((name, args)))
    monkeypatch.setattr(_tokens, "draw_logits_workspace_bytes", lambda B, V: 0)
    x, u = torch.zeros(3, 50), torch.zeros(3)
    z, prob = torch.zeros(3, dtype=torch.int32), torch.zeros(3, requires_grad=True)
    seed = torch.zeros(3, dtype=torch.int64)
    for call in (lambda p: _layers.sample_logits.__wrapped__(x, u, out=(z, p)),
                 lambda p: _tokens.draw_logits.__wrapped__(x, seed, z, out=(z, p))):
        with pytest.raises(ValueError, match="gradient"):
            call(prob)
        assert not calls and prob._version == 0
        with torch.no_grad():
            call(prob)
        call(prob.detach().clone())
        assert len(calls) == 2
        calls.clear()
        prob = torch.zeros(3, requires_grad=True)


def test_forward_mode_tangents_are_refused(calls, monkeypatch):
    """A dual tensor does not require a gradient, and its tangent would be lost without a word."""
    import torch
    import torch.autograd.forward_ad as forward

    import paper_1505_03851_amd as lda
    from paper_1505_03851_amd import _layers, _tokens
    x, v, h = torch.zeros(2, 8), torch.ones(8), torch.zeros(2, 8)
    q, s, ids = torch.zeros(2, 8, dtype=torch.int8), torch.ones(2), torch.zeros(2, dtype=torch.int32)
    with forward.dual_level():
        def dual(t):
            return forward.make_dual(t, torch.ones_like(t))
        for call in (
                lambda: lda.add_norm(dual(x), v), lambda: lda.add_norm(x, dual(v)),
                lambda: lda.add_norm(x=dual(x), weight=v), lambda: lda.add_norm(x, v, residual=dual(h)),
                lambda: lda.add_norm(x, v, out=dual(h)), lambda: lda.add_norm_int8(dual(x), v),
                lambda: lda.add_norm_int8(x, v, out=(q, dual(s))),
                lambda: lda.norm_grad(x, dual(h), v), lambda: lda.quantise_rows(dual(x)),
                lambda: lda.project_int8(q, dual(s), q, s), lambda: lda.embed(dual(x), ids),
                lambda: lda.embed_grad(dual(x), ids, 5), lambda: lda.dropout(dual(x), 0.5, 1),
                lambda: lda.penalise_logits(dual(x)), lambda: lda.penalise_logits(x, bias=dual(v)),
                lambda: lda.sample_logits(x, s, out=(ids, dual(s)))):
            with pytest.raises(ValueError, match="tangent"):
                call()
        # what has none goes on to the next check, and so does what a token is drawn from
        for call in (lambda: lda.add_norm(x, v), lambda: lda.sample_logits(dual(x), s),
                     lambda: lda.draw_logits(dual(x), ids.long(), ids)):
            with pytest.raises(ValueError, match="on the GPU"):
                call()
