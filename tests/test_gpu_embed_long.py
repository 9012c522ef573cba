"""Gradients of tokens that make up a batch of very many positions.

Every term is 1 + 2^-13 - 2^-23: added one after the other, each loses 2^-13 where the sum is between 2^11 and 2^12.  Tolerance: U = 2^-24; at most 256 positions of a run (512 of a token that crosses one border), the
runs of a long token 64 at a time by up to 1,024 threads, as many as there are of these (15 at these sizes), and those side by side in 10 steps; scaled by 1: 345 additions each off by U of the sum at most, 512 of a short token.
"""
import numpy as np
import pytest

from tests.rows_util import U, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d", [(240_000_000, 4), (20_000_000, 128), (1_000_000, 4)])
def test_one_token_of_many_positions(n, d):
    import torch
    import paper_2308_13466_b200.binding as B
    ctx = B.sat_create(0, 0)
    try:
        term = 1 + 2.0 ** -13 - 2.0 ** -23
        g = torch.full((n, d), term, device="cuda")
        order = B.new_token_order(n, 3)
        tokens, index = order._keep
        short = 300                                                             # a first token that crosses a border of the longest runs, then the long one
        tokens.fill_(1)
        tokens[:short] = 0
        torch.arange(n, out=index)
        table = torch.full((3, d), np.nan, device="cuda")
        B.sat_embed_bwd(ctx, order, g, 1.0, table)
        B.sat_sync_status(ctx)
        got = host(table)
        assert np.all(np.abs(got[0] - short * term) <= 512 * U * short * term) and np.all(got[2] == 0)
        assert np.all(np.abs(got[1] - (n - short) * term) <= 345 * U * (n - short) * term)
    finally:
        B.sat_destroy(ctx)


@pytest.mark.parametrize("n,vocabulary,d", [(6_000_000, 5000, 132), (40_000_000, 700, 8)])
def test_runs_of_their_longest(n, vocabulary, d):
    """Whole numbers, whose sums fp32 holds: every position is added once, wherever tokens and runs begin and end."""
    import torch
    import paper_2308_13466_b200.binding as B
    ctx = B.sat_create(0, 0)
    try:
        gen = torch.Generator(device="cuda").manual_seed(4)
        tokens = (vocabulary * torch.rand(n, device="cuda", generator=gen) ** 3).int().clamp(max=vocabulary - 1)
        order = B.new_token_order(n, vocabulary)
        B.sat_token_sort(ctx, tokens, 2, order)
        g = torch.randint(-3, 4, (n, d), device="cuda", generator=gen).float()
        table = torch.full((vocabulary, d), np.nan, device="cuda")
        B.sat_embed_bwd(ctx, order, g, 1.0, table)
        B.sat_sync_status(ctx)
        want = torch.zeros((vocabulary, d), dtype=torch.float64, device="cuda").index_add_(0, tokens.long(), g.double())
        want[2] = 0
        assert torch.equal(table.double(), want)
    finally:
        B.sat_destroy(ctx)
