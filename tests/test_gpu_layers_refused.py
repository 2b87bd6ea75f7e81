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
