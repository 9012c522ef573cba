"""Layers that keep their aggregated inputs in 8 bits (SAT_FWD_KEEP8, SAT_EPOCH_KEEP8).

Nothing but the weight gradient may change: outputs, losses, gradients handed down and the ring are compared bit by bit with those of the same
calls without the flag.  The weight gradient is the formula's on the rounded rows: exactly so on a graph without edges, where the propagation
matrix is the identity and the aggregated rows are the inputs; elsewhere it is held against the unrounded one.  There an element of AGG is off by
at most 2^-4 of itself (half a unit of three fraction bits) or 2^-10 2^e <= 2^-10 max / 224 of its group, so |g_W8 - g_W| <= sum (2^-4 |AGG| + 2^-17 max) |D|,
and since roundings are independent and unbiased far less: the 2-norm of the difference is at most 2^-4 / sqrt(3) of sqrt(sum AGG^2 D^2), taken twice as much here.
"""
import numpy as np
import pytest

from oracle import mx_ref as mx
from oracle import sat_ref as orc
from sat_synth import make_workload
from tests.gpu_util import dev, dev2d, empty2d, pred_to_device

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2308_13466_b200.binding as binding
    return binding


def _no_edges(B, n, M):
    ctx = B.sat_create(0, 0)
    B.sat_graph_load(ctx, np.zeros(n + 1, dtype=np.int64), np.zeros(0, dtype=np.int32))
    B.sat_partition(ctx, M, B.SAT_PART_CONTIG_BLOCKS)
    return ctx


@pytest.mark.parametrize("n,d_in,d_out,relu,parts", [(1, 5, 3, True, 1), (40, 33, 7, False, 2), (300, 100, 47, True, 3), (3000, 256, 128, True, 4), (3001, 130, 300, False, 1)])
def test_weight_gradient_of_the_rounded_rows(B, n, d_in, d_out, relu, parts):
    import torch
    rng = np.random.default_rng(n + d_in)
    x = (rng.normal(size=(n, d_in)) * np.exp(rng.normal(size=(n, 1)))).astype(np.float32)
    w, b, g = rng.normal(size=(d_in, d_out)).astype(np.float32), rng.normal(size=d_out).astype(np.float32), rng.normal(size=(n, d_out)).astype(np.float32)
    xq = mx.dequantise(*mx.quantise(x, 8), d_in, 8)
    ctx = _no_edges(B, n, parts)
    try:
        xd, wd, bd, gd = dev2d(x), dev(w), dev(b), dev2d(g)
        h, gx = empty2d(n, d_out), empty2d(n, d_in)
        gw, gb = torch.full((d_in, d_out), 5.0, device="cuda"), torch.full((d_out,), 5.0, device="cuda")
        act = B.SAT_ACT_RELU if relu else B.SAT_ACT_NONE
        B.sat_layer_fwd(ctx, B.SAT_ALL_PARTS, 1, xd, None, wd, bd, act | B.SAT_FWD_KEEP8, h)
        B.sat_layer_bwd(ctx, B.SAT_ALL_PARTS, 1, gd, wd, gw, gb, 0, gx)
        B.sat_sync_status(ctx)
        D = np.where(h.cpu().numpy() > 0, g, 0).astype(np.float64) if relu else g.astype(np.float64)
        # sums of n terms in fp32: additions times a unit of sum |x| |D| (three bf16 terms, 16 products an addition, or one product an addition)
        bound = (n / 2 + 6 * (n / 16 + 1) + 8) * 2.0 ** -23 * (np.abs(xq).T @ np.abs(D)) + 1e-40
        got = gw.cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - xq.T @ D) <= bound)
        assert np.all(np.abs(gb.cpu().numpy() - D.sum(0)) <= (n + 8) * 2.0 ** -23 * np.abs(D).sum(0) + 1e-40)
        if n >= 100:
            spread = np.sqrt((x.astype(np.float64) ** 2).T @ D ** 2)
            assert np.linalg.norm(got - x.astype(np.float64).T @ D) <= 2 * 2.0 ** -4 / np.sqrt(3) * np.linalg.norm(spread)
            assert not np.allclose(got, x.astype(np.float64).T @ D, rtol=1e-6, atol=0)     # the image was used
        # partition by partition, adding up, gives the sum; and everything else is what the call without the flag gives
        off = np.concatenate([[0], np.cumsum([B.sat_part_sizes(ctx, m)[0] for m in range(parts)])])
        gw2, gb2 = torch.zeros_like(gw), torch.zeros_like(gb)
        h2, gx2 = empty2d(n, d_out), empty2d(n, d_in)
        for m in range(parts):
            s = slice(off[m], off[m + 1])
            B.sat_layer_fwd(ctx, m, 1, xd[s], None, wd, bd, act | B.SAT_FWD_KEEP8, h2[s])
            B.sat_layer_bwd(ctx, m, 1, gd[s], wd, gw2, gb2, 1 if m else 0, gx2[s])
        B.sat_sync_status(ctx)
        assert bool(torch.equal(h, h2)) and bool(torch.equal(gx, gx2))
        assert np.all(np.abs(gw2.cpu().numpy() - xq.T @ D) <= 2 * bound)
        h3, gx3, gw3, gb3 = empty2d(n, d_out), empty2d(n, d_in), torch.zeros_like(gw), torch.zeros_like(gb)
        B.sat_layer_fwd(ctx, B.SAT_ALL_PARTS, 1, xd, None, wd, bd, act, h3)
        B.sat_layer_bwd(ctx, B.SAT_ALL_PARTS, 1, gd, wd, gw3, gb3, 0, gx3)
        assert bool(torch.equal(h, h3)) and bool(torch.equal(gx, gx3))
        # a change of the form drops what the other partitions had
        B.sat_layer_fwd(ctx, 0, 1, xd[:off[1]], None, wd, bd, act | B.SAT_FWD_KEEP8, h3[:off[1]])
        if parts > 1:
            with pytest.raises(B.SatError) as e:
                B.sat_layer_bwd(ctx, 1, 1, gd[off[1]:off[2]], wd, gw3, gb3, 0, gx3[off[1]:off[2]])
            assert e.value.status == B.SAT_ESTATE
    finally:
        B.sat_destroy(ctx)


@pytest.mark.parametrize("kind,shrink,by_part,history", [("tiny", 1, False, False), ("odd", 1, False, True), ("odd", 1, True, False), ("medium", 8, False, True), ("medium", 16, True, True)])
def test_epochs_change_in_their_weight_gradients_only(B, kind, shrink, by_part, history):
    import torch
    from paper_2308_13466_b200.epoch import SatEpoch
    wl = make_workload(kind, shrink=shrink)
    part = wl.part_given if wl.part_given is not None else orc.contig_blocks(wl.n, wl.M)
    P = orc.build_partition(wl.rowptr, wl.col, part, wl.M)
    perm = np.concatenate(P.inner_gid)
    runs = []
    for keep8 in (False, True):
        ep = SatEpoch(wl.rowptr, wl.col, wl.M, wl.dims, wl.tau, wl.loss, part_given=wl.part_given)
        ep.set_inputs(dev2d(wl.X), dev(wl.labels[perm]))
        W, b, preds = [dev(w) for w in wl.W], [dev(x) for x in wl.b], pred_to_device(wl.pred, B)
        for _ in range(3):                                       # no parameter step: every epoch's numbers can be compared
            if by_part:
                ep.step_per_partition(W, b, preds, grad_history=history, keep8=keep8)
            else:
                ep.step(W, b, preds, grad_history=history, keep8=keep8)
        B.sat_sync_status(ep.ctx)
        runs.append(dict(H=[t.clone() for t in ep.H[1:]], G=[t.clone() for t in ep.G[1:]], loss=ep.loss_sum.clone(), gW=[t.double().cpu().numpy() for t in ep.gW],
                         gb=[t.double().cpu().numpy() for t in ep.gb], ring=[B.sat_cache_read(ep.ctx, l, 0, P.n_slots, wl.dims[l]) for l in range(1, wl.L)]))
        ep.close()
    a, c = runs
    for x, y in zip(a["H"] + a["G"] + [a["loss"]], c["H"] + c["G"] + [c["loss"]]):
        assert bool(torch.equal(x, y))
    for x, y in zip(a["ring"], c["ring"]):
        assert np.array_equal(x, y)
    for l, (x, y) in enumerate(zip(a["gb"], c["gb"])):
        assert np.linalg.norm(x - y) <= 1e-5 * max(np.linalg.norm(x), 1e-12), l      # the same sums in another order
    for l, (x, y) in enumerate(zip(a["gW"], c["gW"])):
        rel = np.linalg.norm(x - y) / np.linalg.norm(x)
        assert 1e-7 < rel < 0.2, (l, rel)


def test_training_goes_on_from_kept_inputs(B):
    from paper_2308_13466_b200.epoch import SatEpoch
    wl = make_workload("tiny")
    ep = SatEpoch(wl.rowptr, wl.col, wl.M, wl.dims, wl.tau, wl.loss, part_given=wl.part_given)
    P = orc.build_partition(wl.rowptr, wl.col, wl.part_given, wl.M)
    ep.set_inputs(dev2d(wl.X), dev(wl.labels[np.concatenate(P.inner_gid)]))
    W, b, preds = [dev(w) for w in wl.W], [dev(x) for x in wl.b], pred_to_device(wl.pred, B)
    for i in range(4):
        ep.step(W, b, preds, lr=0.01, keep8=bool(i % 2))       # the form may change from epoch to epoch
        assert np.isfinite(float(ep.loss_sum))
    ep.step(W, b, preds, lr=0.01, pred_lr=1e-3, keep8=True)
    B.sat_sync_status(ep.ctx)
    with pytest.raises(B.SatError):
        B.sat_epoch(ep.ctx, ep._described(W, b, preds), None, 32)
    ep.close()
