"""Statistics that layer norm leaves of rows that are no numbers, and of constant ones."""
import numpy as np
import pytest

from tests.rows_util import host, matrix, room

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("d", [1, 30, 512, 1500, 9000])
def test_statistics(d, t):
    import torch
    import paper_2308_13466_b200.binding as B
    rng = np.random.default_rng(d)
    x = rng.normal(size=(7, d))
    x[1, d // 2], x[3, d - 1], x[4, 0] = np.nan, np.inf, -np.inf
    x[5] = 3.25
    ctx = B.sat_create(0, 0)
    try:
        xt, y = matrix(x, t)[0], room(7, d, t)[0]
        mean, rstd = (torch.zeros(7, device="cuda") for _ in range(2))
        B.sat_layernorm_fwd(ctx, xt, None, None, 0.25, y, mean, rstd)
        B.sat_sync_status(ctx)
        bad = np.isin(np.arange(7), [1, 3, 4])
        assert np.isnan(host(mean)[bad]).all() and np.isnan(host(rstd)[bad]).all() and np.isnan(host(y)[bad]).all()
        assert np.isfinite(host(mean)[~bad]).all() and np.isfinite(host(rstd)[~bad]).all() and np.isfinite(host(y)[~bad]).all()
        assert host(mean)[5] == 3.25 and host(rstd)[5] == 2.0 and bool((y[5] == 0).all())
    finally:
        B.sat_destroy(ctx)
