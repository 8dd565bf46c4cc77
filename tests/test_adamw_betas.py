"""Betas that fp32 does not tell from 1: a mean held in fp32 would never decay (no GPU needed: lists without elements)."""
import ctypes as C

import pytest

from paper_2606_19004_amd import ditstep as d

OK, DOMAIN = 0, 3


def status(beta1, beta2):
    cfg = d.AdamwConfig(1e-3, beta1, beta2, 1e-8, 0.0, 1)
    return d.lib().adamw_step(C.byref(cfg), None, 0, None, None, None)


@pytest.mark.parametrize("beta", [1 - 2.0 ** -25, 1 - 2.0 ** -26, 1 - 1e-9, 1 - 2.0 ** -53])
def test_betas_that_round_to_1(beta):
    assert status(beta, 0.999) == DOMAIN and status(0.9, beta) == DOMAIN


@pytest.mark.parametrize("beta", [0.0, 1e-300, 0.5, 0.999999, 1 - 2.0 ** -24])
def test_betas_below_1(beta):
    assert status(beta, 0.999) == OK and status(0.9, beta) == OK
