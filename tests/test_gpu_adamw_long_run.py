"""The means of the gradient and of its square after thousands of steps.

From zero, with one gradient g in every step, m is g (1 - beta1^t) and v is g^2 (1 - beta2^t). Each step rounds the decayed mean and the new one,
2^-24 of the mean each at most, so the mean of one weight is off by at most A = 2 t 2^-24 of itself, as often up as down. The mean of that over n weights
of unlike gradients lies within 8 A / sqrt(n), except with a probability of 2 exp(-8^2 / 2) (Hoeffding). What is rounded away of a decay is spread over the
units that the decay passes through, 800 of them at 1 - beta = 1e-4 (2^23 1e-4), so its mean is below 1/800 of half a unit: A / 800. 1 - beta and the
product with g are off by 2^-25 and 2^-24. A beta that is itself rounded to fp32 is off by 1.7e-4 of 1 - beta, which shows as 2.3e-5 after 3000 steps."""
import numpy as np
import pytest
import torch

from tests.gpu_util import host64

pytestmark = pytest.mark.gpu


def test_means_after_many_steps():
    from paper_2606_19004_amd import ditstep as d
    n, t, beta = 1 << 20, 3000, 0.9999
    gen = torch.Generator(device="cuda").manual_seed(6)
    g = torch.randn(n, generator=gen, device="cuda")
    g += 0.1 * torch.sign(g)
    p, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
    w = d.adamw_list([p], [g], [m], [v])
    for _ in range(t):
        d.adamw_step(w, lr=0.0, beta1=beta, beta2=beta, step=1)
    share, a = -np.expm1(t * np.log(beta)), 2 * t * 2.0 ** -24
    bound = 8 * a / np.sqrt(n) + a / 800 + 2.0 ** -23
    for mean, want in ((m, host64(g)), (v, host64(g) ** 2)):
        off = host64(mean) / (want * share) - 1
        assert np.abs(off).max() <= a + 2.0 ** -23
        assert abs(off.mean()) <= bound, (off.mean(), bound)
