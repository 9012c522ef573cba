"""Gradients of layer norm's parameters over very many rows whose terms have one sign.

A term is g = 1 + 2^-13 - 2^-23: added one after the other, every one loses 2^-13 where the sum is between 2^11 and 2^12.  The sums are exact multiples of the term.  Tolerance: U = 2^-24; at most
512 rows of a thread, 32 side by side in a block, then 64, as many as there are of these (16 at these sizes), and 5 additions across a warp: 629 additions, each off by U of the sum at most.
"""
import numpy as np
import pytest

from tests.rows_util import U, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d", [(60_000_000, 4), (6_250_000, 516), (7_000_000, 8)])
def test_sums_over_many_rows(rows, d):
    import torch
    import paper_2308_13466_b200.binding as B
    ctx = B.sat_create(0, 0)
    try:
        term = 1 + 2.0 ** -13 - 2.0 ** -23
        x = torch.full((rows, d), term, device="cuda")
        g_gamma, g_beta = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        B.sat_layernorm_bwd(ctx, x, x, None, torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda"), None, g_gamma, g_beta)
        B.sat_sync_status(ctx)
        assert np.all(np.abs(host(g_beta) - rows * term) <= 629 * U * rows * term)
        assert np.all(np.abs(host(g_gamma) - rows * term ** 2) <= 631 * U * rows * term ** 2)   # (x - mean) rstd is the term again, its square is added without a rounding of its own
    finally:
        B.sat_destroy(ctx)
