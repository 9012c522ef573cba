"""Learned inputs, layer norm and distillation together, as an epoch runs them: against the same network in 64 bits with automatic differentiation."""
import numpy as np
import pytest

from sat_synth import make_workload
from tests.gpu_util import assert_close, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_2308_13466_b200.binding as binding
    return binding


def _propagation(wl, part):
    """(P_in, P_out) dense in 64 bits, global id order"""
    import torch
    n = wl.n
    deg = np.diff(wl.rowptr) + 1
    rows = np.repeat(np.arange(n), np.diff(wl.rowptr))
    P = np.zeros((n, n))
    P[rows, wl.col] = 1.0
    P[np.arange(n), np.arange(n)] = 1.0
    P *= 1 / np.sqrt(deg)[:, None] / np.sqrt(deg)[None, :]
    same = part[:, None] == part[None, :]
    return torch.from_numpy(P * same).cuda(), torch.from_numpy(P * ~same).cuda()


def _network(p, tokens, padding, scale, P_in, P_out, pulled, eps):
    """Outputs and the hidden layers' rows, global id order"""
    import torch
    x = torch.where((tokens != padding)[:, None], p["table"][tokens.long()] * scale, 0.0)
    halo, hidden = x, []
    for l, (W, b) in enumerate(zip(p["W"], p["b"])):
        z = (P_in @ x + P_out @ halo) @ W + b
        if l == len(p["W"]) - 1:
            return z, hidden
        h = torch.relu(z)
        var, mean = torch.var_mean(h, 1, unbiased=False, keepdim=True)
        x = (h - mean) / torch.sqrt(var + eps) * p["gamma"][l] + p["beta"][l]
        hidden.append(x.detach())
        halo = pulled[l]


def _flat(p):
    return [("table", p["table"])] + [(f"{k}[{i}]", t) for k in ("W", "b", "gamma", "beta") for i, t in enumerate(p[k])]


@pytest.mark.parametrize("objective", ["labels", "teacher", "both"])
@pytest.mark.parametrize("name,vocabulary,padding", [("tiny", 40, -1), ("odd", 6000, 3)])
def test_epochs(B, name, vocabulary, padding, objective):
    import torch
    from paper_2308_13466_b200.epoch import SatEpoch, TokenInputs
    wl = make_workload(name, dims=[52, 72, 40, 7]) if name == "odd" else make_workload(name)
    part = wl.part_given if wl.part_given is not None else (np.arange(wl.n, dtype=np.int64) * wl.M // wl.n)
    rng = np.random.default_rng(11)
    ep = SatEpoch(wl.rowptr, wl.col, wl.M, wl.dims, wl.tau, wl.loss, part_given=wl.part_given)
    try:
        perm = np.concatenate([B.sat_part_lists(ep.ctx, m)["inner_gid"] for m in range(wl.M)])
        tokens = dev(rng.integers(0, vocabulary, wl.n).astype(np.int32)) if vocabulary < wl.n else dev(rng.permutation(wl.n).astype(np.int32))
        d, classes, k = wl.dims, wl.dims[-1], 3
        f = lambda *s: dev(rng.normal(size=s).astype(np.float32))
        params = dict(table=f(vocabulary, d[0]), W=[dev(w) for w in wl.W], b=[0.1 * f(x) for x in d[1:]], gamma=[1 + 0.2 * f(x) for x in d[1:-1]],
                      beta=[0.2 * f(x) for x in d[1:-1]])
        ids = np.stack([rng.permutation(classes)[:k] for _ in range(wl.n)]).astype(np.int32)
        ids[::7, 1:] = -1
        logits = rng.normal(size=(wl.n, k)).astype(np.float32)
        hard = {"labels": 1.0, "teacher": 0.0, "both": 0.4}[objective]
        teacher = None if objective == "labels" else dict(ids=dev(ids[perm]), logits=dev(logits[perm]), temperature=2.0, hard=hard)
        ep.set_inputs(None, dev(wl.labels[perm]))
        inputs = TokenInputs(ep, tokens, vocabulary, padding, scale=1.5)
        P_in, P_out = _propagation(wl, part)
        ref = {key: v.double() if key == "table" else [t.double() for t in v] for key, v in params.items()}
        leaves = [t.requires_grad_() for _, t in _flat(ref)]
        pulled = [torch.zeros((wl.n, x), dtype=torch.float64, device="cuda") for x in d[1:-1]]
        y, t_ids, t_log = torch.from_numpy(wl.labels).cuda().long(), torch.from_numpy(ids).cuda().long(), torch.from_numpy(logits).cuda().double()
        for epoch in range(3):
            z, hidden = _network(ref, tokens, padding, 1.5, P_in, P_out, pulled, ep.NORM_EPS)
            loss = hard * -torch.log_softmax(z, 1).gather(1, y[:, None]).sum() / wl.n
            if hard < 1:
                lp = torch.where(t_ids >= 0, t_log / 2, -1e9).log_softmax(1)
                lq = (z / 2).log_softmax(1).gather(1, t_ids.clamp(min=0))
                loss = loss + (1 - hard) * 4 * torch.where(t_ids >= 0, lp.exp() * (lp - lq), 0.0).sum() / wl.n
            grads = torch.autograd.grad(loss, leaves)
            ep.step_tokens(inputs, params, None, teacher=teacher)
            B.sat_sync_status(ep.ctx)
            assert_close(ep.H[ep.L].cpu().numpy(), z.detach()[torch.from_numpy(perm.astype(np.int64)).cuda()].cpu().numpy(), f"outputs, epoch {epoch}")
            assert_close(ep.loss_sum.cpu().numpy(), loss.detach().reshape(1).cpu().numpy(), f"loss, epoch {epoch}")
            for (what, got), want in zip(_flat(ep.token_grads), grads):
                assert_close(got.cpu().numpy(), want.cpu().numpy(), f"gradient of {what}, epoch {epoch}")
            pulled = hidden
        before = [t.clone() for _, t in _flat(params)]                          # the parameter step
        ep.step_tokens(inputs, params, None, lr=0.5, teacher=teacher)
        for (what, t), old, (_, g) in zip(_flat(params), before, _flat(ep.token_grads)):
            assert_close(t.cpu().numpy(), (old.double() - 0.5 * g.double()).cpu().numpy(), f"step of {what}", 1e-6)
        B.sat_sync_status(ep.ctx)
    finally:
        ep.close()
