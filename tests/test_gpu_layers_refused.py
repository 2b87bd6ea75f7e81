"""Kinds of derivative that the layers refuse rather than lose."""
import pytest
import torch
import torch.autograd.forward_ad as fwad

from tests.test_gpu_layers import DEV, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers():
    from paper_2607_11985_amd import layers as m
    return m


def ops_on(layers):
    t = torch.tensor([0, 2], device=DEV)
    f = lambda *s: rand(s, sum(s), torch.float32)
    return {
        "layer_norm": (lambda x, w, b: layers.layer_norm(x, w, b), [f(2, 8), f(8), f(8)]),
        "linear": (lambda x, w, b, r: layers.linear(x, w, b, "tanh", r),
                   [f(2, 8), f(3, 8), f(3), f(2, 3)]),
        "log_probs": (lambda z: layers.log_probs(z, t, 1), [f(2, 8)]),
        "weights": (lambda z: layers.log_probs(z, t, 1, "weights"), [f(2, 8).abs()]),
    }


@pytest.mark.parametrize("op", ["layer_norm", "linear", "log_probs", "weights"])
def test_forward_mode_is_refused(layers, op):
    """A tangent must not vanish without a word, whichever input carries it, also beside inputs
    that want a gradient and without grad mode."""
    call, ins = ops_on(layers)[op]
    for k in range(len(ins)):
        for other in (False, True):
            with fwad.dual_level():
                v = [i.detach().requires_grad_(other and op != "weights") for i in ins]
                v[k] = fwad.make_dual(ins[k], torch.ones_like(ins[k]))
                with pytest.raises(ValueError, match="forward-mode"):
                    call(*v)
                with torch.no_grad(), pytest.raises(ValueError, match="forward-mode"):
                    call(*v)
                call(*[i.detach() for i in ins])
        with pytest.raises(Exception):
            torch.func.jvp(lambda i: call(*ins[:k], i, *ins[k + 1:]), (ins[k],),
                           (torch.ones_like(ins[k]),))


def test_gradients_of_constant_cotangents_cannot_be_differentiated(layers):
    """A penalty on a gradient has to raise also where the cotangent itself is a constant."""
    x, w, b, n, m = (rand(s, i, torch.float32) for i, s in
                     enumerate([(3, 8), (4, 8), (4,), (8,), (8,)]))
    t = torch.zeros(3, dtype=torch.int64, device=DEV)

    def raises(make, wanted, leaves):
        v = [i.detach().requires_grad_(k in leaves) for k, i in enumerate(make[1])]
        y = make[0](*v)
        g, = torch.autograd.grad(y.sum(), (v[wanted],), create_graph=True)
        other = torch.ones((), device=DEV, requires_grad=True)
        with pytest.raises(RuntimeError, match="cannot be differentiated again"):
            (other * 2 + g.square().sum()).backward()

    norm = (lambda x, w, b: layers.layer_norm(x, w, b), [x, n, m])
    for wanted, leaves in ((0, {0}), (0, {0, 1, 2}), (1, {0, 1}), (0, {0, 1})):
        raises(norm, wanted, leaves)
    for act in ("gelu", "silu", "tanh"):
        lin = (lambda x, w, b: layers.linear(x, w, b, act), [x, w, b])
        for wanted, leaves in ((0, {0}), (1, {1}), (2, {2}), (2, {0, 2}), (0, {0, 1, 2})):
            raises(lin, wanted, leaves)
    for act in ("none", "relu"):
        lin = (lambda x, w, b: layers.linear(x, w, b, act), [x, w, b])
        for wanted, leaves in ((0, {0, 1}), (1, {0, 1})):
            raises(lin, wanted, leaves)
    raises((lambda x: layers.log_probs(x, t).logp, [x]), 0, {0})
    raises((lambda x: layers.log_probs(x).entropy, [x]), 0, {0})


def test_gradients_that_are_constants_stay_usable(layers):
    """With create_graph, gradients that depend on nothing that wants one are plain constants, and
    first derivatives go on as ever."""
    x, w, b, n, m = (rand(s, i, torch.float32) for i, s in
                     enumerate([(3, 8), (4, 8), (4,), (8,), (8,)]))
    for act in ("none", "relu"):
        for k in range(3):
            v = [i.detach().requires_grad_(j == k) for j, i in enumerate((x, w, b))]
            g, = torch.autograd.grad(layers.linear(*v, act).sum(), (v[k],), create_graph=True)
            assert not g.requires_grad
    v = [i.detach().requires_grad_(True) for i in (x, n, m)]
    db, = torch.autograd.grad(layers.layer_norm(*v).sum(), (v[2],), create_graph=True)
    assert not db.requires_grad and (db == 3).all()
    v = [i.detach().requires_grad_(True) for i in (x, n, m)]
    layers.layer_norm(*v).sum().backward(create_graph=True)
    u = [i.detach().requires_grad_(True) for i in (x, n, m)]
    layers.layer_norm(*u).sum().backward()
    assert all(torch.equal(i.grad, j.grad) for i, j in zip(u, v))
