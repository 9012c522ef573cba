"""What an epoch with learned inputs is refused for, before any of it has run (no GPU: nothing of the library is called)."""
import weakref

import numpy as np
import pytest
import torch

DIMS, N, HALO, WORDS = [8, 6, 5, 3], 12, 4, 20


@pytest.fixture(scope="module", autouse=True)
def built():
    import __graft_entry__
    __graft_entry__.build()


def _epoch(n=N, nb=HALO, dims=DIMS):
    from paper_2308_13466_b200.epoch import SatEpoch
    ep = SatEpoch.__new__(SatEpoch)
    ep.ctx, ep.device, ep.n, ep.nb, ep.M, ep.dims, ep.L = None, torch.device("cpu"), n, nb, 1, list(dims), len(dims) - 1
    ep.labels, ep.loss = torch.zeros(n, dtype=torch.int32), "ce"
    return ep


def _inputs(ep, gids=None):
    from paper_2308_13466_b200.epoch import TokenInputs
    it = TokenInputs.__new__(TokenInputs)
    it.gids = np.arange(ep.n + ep.nb, dtype=np.int32) % ep.n if gids is None else gids
    it.tokens, it.vocabulary, it.padding, it.scale, it.d, it._for = torch.zeros(ep.n, dtype=torch.int32), WORDS, -1, 1.0, ep.dims[0], weakref.WeakSet()
    return it


def _params(dims=DIMS, words=WORDS):
    return dict(table=torch.zeros(words, dims[0]), W=[torch.zeros(a, b) for a, b in zip(dims, dims[1:])], b=[torch.zeros(x) for x in dims[1:]], gamma=[torch.ones(x) for x in dims[1:-1]],
                beta=[torch.zeros(x) for x in dims[1:-1]])


def _teacher(n=N, k=3, **kw):
    return dict(dict(ids=torch.zeros((n, k), dtype=torch.int32), logits=torch.zeros(n, k), temperature=2.0, hard=0.5), **kw)


class Ran(Exception):
    pass


@pytest.fixture
def library(monkeypatch):
    """Calls of the library raise Ran; the lists of a partition are those of _inputs."""
    import paper_2308_13466_b200.binding as B
    for name in B.EXPORTS:
        def call(*a, **kw):
            raise Ran(name)
        monkeypatch.setattr(B, name, call)
    monkeypatch.setattr(B, "sat_part_lists", lambda ctx, m: dict(inner_gid=np.arange(N, dtype=np.int32), halo_gid=np.arange(HALO, dtype=np.int32)))


def test_what_an_epoch_is_refused_for(library):
    ep = _epoch()
    ep._token_check(_inputs(ep), _params(), None, None)
    ep._token_check(_inputs(ep), _params(), [None, None], _teacher())
    other = _epoch(n=N - 2)
    wrong = dict(
        graph=dict(inputs=_inputs(other)), partitions=dict(inputs=_inputs(ep, np.arange(N + HALO, dtype=np.int32)[::-1] % N)), width=dict(inputs=_inputs(_epoch(dims=[4, 6, 5, 3]))),
        table=dict(params=_params(words=WORDS + 1)), weights=dict(params=_params([8, 7, 5, 3])), narrow=dict(params=_params([8, 6, 5, 2])), layers=dict(params=_params([8, 6, 3])),
        gamma=dict(params=dict(_params(), gamma=[])), half=dict(params=dict(_params(), table=torch.zeros(WORDS, 8).half())),
        strided=dict(params=dict(_params(), W=[torch.zeros(6, 8).t(), *_params()["W"][1:]])), pred=dict(pred=[None]), rows=dict(teacher=_teacher(N - 1)), k=dict(teacher=_teacher(k=257)),
        ids=dict(teacher=_teacher(ids=torch.zeros((N, 3)))), logits=dict(teacher=_teacher(logits=torch.zeros(N, 2))), temperature=dict(teacher=_teacher(temperature=0.0)), hard=dict(teacher=_teacher(hard=1.5)))
    for what, kw in wrong.items():
        args = dict(dict(inputs=_inputs(ep), params=_params(), pred=None, teacher=None), **kw)
        with pytest.raises(AssertionError):
            ep.step_tokens(**args)
            pytest.fail(what)
    ep.labels = None
    for teacher in (None, _teacher()):
        with pytest.raises(AssertionError):
            ep.step_tokens(_inputs(ep), _params(), None, teacher=teacher)
    ep._token_check(_inputs(ep), _params(), None, _teacher(hard=0.0))
    ep.labels = torch.zeros((N, 3), dtype=torch.uint8)
    with pytest.raises(AssertionError):
        ep.step_tokens(_inputs(ep), _params(), None, teacher=_teacher())


def test_inputs_fit_every_epoch_over_the_same_rows(library):
    a, b = _epoch(), _epoch()
    it = _inputs(a)
    assert it.fits(a) and it.fits(b) and a in it._for and b in it._for and not it.fits(_epoch(nb=HALO - 1))


def test_gradients_follow_the_parameters():
    ep = _epoch()
    p = _params()
    ep._token_room(p)
    first, rows = ep.token_grads, ep.normed
    ep._token_room(_params())
    assert ep.token_grads is first                                              # the same shapes: the same tensors
    ep._token_room(_params(words=WORDS + 5))
    assert ep.token_grads["table"].shape == (WORDS + 5, 8) and ep.normed is rows
    q = _params()
    q["W"].append(torch.zeros(2, 2))                                            # one more than there are layers
    ep._token_room(q)
    assert [t.shape for t in ep.token_grads["W"]] == [t.shape for t in q["W"]] and ep.token_grads["table"].shape == (WORDS, 8)
