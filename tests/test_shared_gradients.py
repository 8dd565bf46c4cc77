"""Weights that share a gradient: it is read only, so it may stand in a list twice or overlap another one; nothing that is written may
(no GPU needed: the lists are only made)."""
import pytest
import torch

from paper_2606_19004_amd import ditstep as d


def weights(grads):
    return [[torch.zeros(g.shape) for g in grads] for _ in range(3)]


def lists(grads, change=None):
    p, m, v = weights(grads)
    if change:
        change(p, m, v)
    return d.adamw_list(p, grads, m, v)


def test_gradients_may_be_the_same():
    flat = torch.zeros(100)
    g = torch.zeros(6)
    for grads in ([g, g], [g, g, g], [flat[:10], flat[5:15], flat[50:]], [flat[:60], flat[10:20], flat[30:40]], [flat[40:], g, flat[:41], g]):
        a = lists(grads)
        assert [t.grad for t in a.array[:a.count]] == [t.data_ptr() for t in grads]


def test_what_is_written_may_not_overlap():
    flat = torch.zeros(100)

    def put(row, i, t):
        def change(p, m, v):
            (p, m, v)[row][i] = t
        return change
    for row in range(3):
        for t in (flat[0:10], flat[9:19], flat[14:24], flat[25:35]):
            with pytest.raises(ValueError, match="share memory"):
                lists([flat[:10], flat[5:15], flat[30:40]], put(row, 0, t))
        lists([flat[:10], flat[5:15], flat[30:40]], put(row, 0, flat[15:25]))
        lists([flat[:10], flat[5:15], flat[30:40]], put(row, 0, flat[40:50]))
    with pytest.raises(ValueError, match="share memory"):
        lists([torch.zeros(10), torch.zeros(10)], lambda p, m, v: p.__setitem__(1, p[0]))
