"""The layer's autograd functions on the CPU, the operators' calls replaced by their plain forms in 64 bits."""
import pytest
import torch

import seq_util as U
from paper_2305_16513_amd import delta_layer as D


def _conv(x, w, bias=None, act=0, unit=0, unit_channels=0, eps=1e-6, **_):
    return torch.stack([U.short_conv(s, w, bias, act, unit, unit_channels, eps)[0] for s in x])


def _rule(q, k, v, g, beta, scale=None, **_):
    return U.delta_rule(q, k, v, g, beta, q.shape[-1] ** -0.5 if scale is None else scale)[0]


def _grads(f, ins, gouts):
    with torch.enable_grad():
        live = [t if t is None else t.detach().clone().requires_grad_(True) for t in ins]
        outs = f(*live)
        outs = outs if isinstance(outs, tuple) else (outs,)
        pairs = [(o, g) for o, g in zip(outs, gouts) if g is not None]
        got = iter(torch.autograd.grad([p[0] for p in pairs], [t for t in live if t is not None], [p[1] for p in pairs]))
    return [t if t is None else next(got) for t in live]


@pytest.fixture
def plain(monkeypatch):
    def norm_add(r, w, x=None, gain=None, eps=1e-6):
        return U.norm_add(r, w, x, gain, eps)

    def norm_add_grad(r, w, gn, x=None, gain=None, gh=None, eps=1e-6):
        gr, gw, gx, ggain = _grads(lambda *t: U.norm_add(*t, eps=eps), (r, w, x, gain), (gh, gn))
        return gr, gx, gw, ggain

    def norm_gate_grad(x, z, w, gy, eps=1e-6):
        return tuple(_grads(lambda *t: U.norm_gate(*t, eps), (x, z, w), (gy,)))

    def conv_grad(x, w, gy, bias=None, **how):
        return tuple(_grads(lambda x, w, bias: _conv(x, w, bias, **how), (x, w, bias), (gy,)))

    def rule_grad(q, k, v, g, beta, go, scale=None, gq=None, gk=None, gv=None, **_):
        got = _grads(_rule, (q, k, v, g, beta), (go,))
        for to, x in zip((gq, gk, gv), got):
            to.copy_(x)
        return gq, gk, gv, got[3], got[4], None
    for name, f in (("norm_add", norm_add), ("norm_add_grad", norm_add_grad), ("norm_gate", U.norm_gate), ("norm_gate_grad", norm_gate_grad), ("short_conv", _conv),
                    ("short_conv_grad", conv_grad), ("delta_rule", _rule), ("delta_rule_grad", rule_grad)):
        monkeypatch.setattr(D.B, "sws_" + name, f)


def _operators(gen):
    """Each function with its inputs, all of which have gradients."""
    n = lambda *shape: U.normal(gen, *shape, dtype=torch.float64).requires_grad_(True)
    yield D._NormAdd, (n(3, 8), n(8), n(3, 8), n(8))
    yield D._NormAdd, (n(3, 8), n(8), None, None)
    yield D._ShortConv, (n(2, 5, 6), n(6, 3), n(6), 3, 3)
    block = D.DeltaBlock(8, 1, 2, 3, 2, device="cpu")
    yield D._DeltaRule, (n(1, 4, block.channels), n(1, 4, 2), n(1, 4, 2), block.parts)
    yield D._NormGate, (n(2, 2, 4), n(2, 2, 4), n(4))


def test_gradients_are_those_of_the_plain_forms(plain):
    for f, args in _operators(torch.Generator().manual_seed(1)):
        ins = [a for a in args if isinstance(a, torch.Tensor)]

        def call(*t):
            it = iter(t)
            return f.apply(*[next(it) if isinstance(a, torch.Tensor) else a for a in args])
        assert torch.autograd.gradcheck(call, ins)


def test_second_derivatives_are_refused(plain):
    """They are not there: a gradient that is itself differentiated has to say so."""
    for f, args in _operators(torch.Generator().manual_seed(2)):
        ins = [a for a in args if isinstance(a, torch.Tensor)]
        outs = f.apply(*args)
        outs = outs if isinstance(outs, tuple) else (outs,)
        grads = torch.autograd.grad(sum(o.square().sum() for o in outs), ins, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            sum(g.square().sum() for g in grads).backward()


def test_whatever_the_gradients_read_is_saved(plain):
    """An input that is changed in place between a call and its gradients is an error, and hooks on saved tensors see every one."""
    gen = torch.Generator().manual_seed(3)
    for which, (f, args) in enumerate(_operators(gen)):
        ins = [a for a in args if isinstance(a, torch.Tensor)]
        for i in range(len(ins)):
            seen = []
            with torch.autograd.graph.saved_tensors_hooks(lambda t: seen.append(t.data_ptr()) or t, lambda t: t):
                out = f.apply(*args)
            assert ins[i].data_ptr() in seen, (which, i)
            out = f.apply(*args)
            out = out if isinstance(out, tuple) else (out,)
            with torch.no_grad():
                ins[i].mul_(2)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                sum(o.sum() for o in out).backward()


def test_serving_has_no_gradients(plain):
    """Calls with caches write them in place: what they return does not pretend to have gradients, of which some paths would be missing."""
    torch.manual_seed(4)
    m = D.DeltaModel(5, 8, 2, 1, 2, 4, 3, dtype=torch.float32, device="cpu")
    tokens = torch.tensor([[1, 2, 3]])
    assert m(tokens).requires_grad
    assert not m(tokens, m.caches(1)).requires_grad
    h, x = m.blocks[0](m.table(tokens), cache=m.caches(1)[0])
    assert not x.requires_grad
    assert torch.is_grad_enabled()


def test_no_symbols_are_asked_for(plain):
    m = D.DeltaModel(5, 8, 1, 1, 2, 4, 3, dtype=torch.float32, device="cpu")
    assert m.answer([[1], [2, 3]], 0) == [[], []] and [len(a) for a in m.answer([[1], [2, 3]], 2)] == [2, 2]
