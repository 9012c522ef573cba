"""One SatEpoch with tables of different sizes one after the other, and learned inputs that are shared."""
import numpy as np
import pytest

from sat_synth import make_workload
from tests.gpu_util import dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2308_13466_b200.binding as binding
    return binding


def _epoch(B, wl):
    from paper_2308_13466_b200.epoch import SatEpoch
    ep = SatEpoch(wl.rowptr, wl.col, wl.M, wl.dims, wl.tau, wl.loss, part_given=wl.part_given)
    perm = np.concatenate([B.sat_part_lists(ep.ctx, m)["inner_gid"] for m in range(wl.M)])
    ep.set_inputs(None, dev(wl.labels[perm]))
    return ep


def _params(rng, wl, words):
    f = lambda *s: dev(rng.normal(size=s).astype(np.float32))
    d = wl.dims
    return dict(table=f(words, d[0]), W=[dev(w) for w in wl.W], b=[0.1 * f(x) for x in d[1:]], gamma=[1 + 0.2 * f(x) for x in d[1:-1]], beta=[0.2 * f(x) for x in d[1:-1]])


def _flat(g):
    return [g["table"]] + [t for k in ("W", "b", "gamma", "beta") for t in g[k]]


def test_tables_of_two_sizes(B):
    import torch
    from paper_2308_13466_b200.epoch import TokenInputs
    wl, rng = make_workload("tiny"), np.random.default_rng(1)
    sets = [(_params(rng, wl, words), dev(rng.integers(0, words, wl.n).astype(np.int32)), words) for words in (40, 90)]
    got = []
    for fresh in (False, True):                                                 # gradients of the second table in the object's own tensors, and in new ones
        ep = _epoch(B, wl)
        try:
            for p, tokens, words in sets:
                if fresh and hasattr(ep, "token_grads"):
                    del ep.token_grads
                    ep._token_layout = None
                ep.step_tokens(TokenInputs(ep, tokens, words), p, None, lr=0.0)
            B.sat_sync_status(ep.ctx)
            assert ep.token_grads["table"].shape == (90, wl.dims[0])
            got.append([t.clone() for t in _flat(ep.token_grads)])
        finally:
            ep.close()
    for a, b in zip(*got):
        assert torch.equal(a, b) and bool((a != 0).any())


def test_inputs_of_another_epoch_object(B):
    """The same graph and partitions: the same inputs serve.  Another partitioning: refused, and the epoch can be run all the same afterwards."""
    import torch
    from paper_2308_13466_b200.epoch import SatEpoch, TokenInputs
    wl, rng = make_workload("tiny"), np.random.default_rng(2)
    p, tokens = _params(rng, wl, 40), dev(rng.integers(0, 40, wl.n).astype(np.int32))
    a, b = _epoch(B, wl), _epoch(B, wl)
    c = SatEpoch(wl.rowptr, wl.col, wl.M + 1, wl.dims, wl.tau, wl.loss)
    try:
        inputs = TokenInputs(a, tokens, 40)
        for ep in (a, b):
            ep.step_tokens(inputs, p, None)
        B.sat_sync_status(b.ctx)
        for x, y in zip(_flat(a.token_grads), _flat(b.token_grads)):
            assert torch.equal(x, y)
        c.set_inputs(None, dev(wl.labels))
        with pytest.raises(AssertionError):
            c.step_tokens(inputs, p, None)
        assert B.sat_cache_state(c.ctx)[1] == 0                                 # nothing was pushed and committed
        c.step_tokens(TokenInputs(c, tokens, 40), p, None)
        B.sat_sync_status(c.ctx)
    finally:
        for ep in (a, b, c):
            ep.close()


def test_called_on_another_stream(B):
    """The library's stream is the one that was current when the SatEpoch was made; what the calls make by themselves goes there, also from another one that is busy."""
    import torch
    from paper_2308_13466_b200.epoch import TokenInputs
    wl, rng = make_workload("tiny"), np.random.default_rng(3)
    p, ids = _params(rng, wl, 40), rng.integers(0, 40, wl.n).astype(np.int32)
    tokens, a, b = dev(ids), _epoch(B, wl), _epoch(B, wl)
    try:
        one = TokenInputs(a, tokens, 40)
        for _ in range(2):
            a.step_tokens(one, p, None)
        side, busy = torch.cuda.Stream(), torch.zeros((4096, 4096), device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(30):
                busy = busy @ busy
            late = dev(ids)[:] + 0                                              # tokens that are there only when `side` has got that far
            two = TokenInputs(b, late, 40)
            for _ in range(2):
                for _ in range(30):
                    busy = busy @ busy
                b.step_tokens(two, p, None)
        torch.cuda.synchronize()
        for x, y in zip((*one.order._keep, a.loss_sum, *_flat(a.token_grads)), (*two.order._keep, b.loss_sum, *_flat(b.token_grads))):
            assert torch.equal(x, y)
        B.sat_sync_status(b.ctx)
    finally:
        a.close()
        b.close()
