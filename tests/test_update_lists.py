"""Lists of weights some of which have no gradient, or one gradient together (no GPU needed: the lists are only made)."""
import pytest
import torch

from paper_2606_19004_amd import ditstep as d

BF = torch.bfloat16


def weights(n=4):
    p = [torch.zeros(3, i + 2) for i in range(n)]
    return dict(params=p, grads=[torch.zeros_like(t, dtype=BF) for t in p], m=[torch.zeros_like(t) for t in p],
                v=[torch.zeros_like(t) for t in p], copies=[torch.zeros_like(t, dtype=BF) for t in p])


def addresses(a):
    return [(t.param, t.grad, t.m, t.v, t.copy, t.count) for t in a.array[:a.count]]


def test_weights_without_a_gradient_are_left_out():
    """As grad_list leaves them out: p.grad of the same parameters goes to both."""
    w = weights()
    whole = addresses(d.adamw_list(**w))
    w["grads"][1] = None
    w["m"][1] = w["v"][1] = None       # (no state either, before the first gradient)
    some = d.adamw_list(**w)
    assert addresses(some) == whole[:1] + whole[2:] and some.count == d.grad_list(w["grads"]).count == 3
    for row in ("params", "m", "v"):   # a generator, as a program has them
        d.adamw_list(**{**w, row: (t for t in w[row])})
    w["grads"][0] = None
    assert addresses(d.adamw_list(**w)) == whole[2:]
    none = d.adamw_list(**{**w, "grads": [None] * 4})
    assert none.count == 0


def test_lengths_are_compared_before_weights_are_left_out():
    w = weights()
    with pytest.raises(ValueError):
        d.adamw_list(**{**w, "grads": [None, *w["grads"]]})


def test_the_other_tensors_of_a_weight_are_there():
    for row in ("params", "m", "v"):
        w = weights()
        w[row][2] = None
        with pytest.raises((ValueError, AttributeError)):
            d.adamw_list(**w)
