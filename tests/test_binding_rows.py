"""Marshalling of the row operators, without a GPU: the binding needs no torch of its own, and numbers that 32 bits do not hold are not cut to them."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def B():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2308_13466_b200.binding as binding
    return binding


def test_binding_without_torch(B):
    code = "import sys; sys.modules['torch'] = None\nimport paper_2308_13466_b200.binding as B\nassert B.sat_last_error is not None and len(B.EXPORTS) > 30"
    subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True)


class Rows:
    """What a CUDA matrix says of itself."""

    def __init__(self, shape, stride=None, dtype=None):
        import torch
        self.shape, self.dtype = tuple(shape), torch.float32 if dtype is None else dtype
        self._stride = tuple(stride) if stride else (shape[1], 1) if len(shape) == 2 else (1,)

    def stride(self):
        return self._stride

    def get_device(self):
        return 0

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def is_contiguous(self):
        return True


@pytest.fixture
def calls(B, monkeypatch):
    """The row operators' entry points take note of a call and do nothing."""
    seen = []
    for name in ("sat_layernorm_fwd", "sat_layernorm_bwd", "sat_embed_fwd", "sat_token_sort", "sat_embed_bwd", "sat_distill_grad"):
        class Fake:
            def __call__(self, *a, name=name):
                seen.append(name)
                return 0
        monkeypatch.setattr(B._lib, name, Fake(), raising=False)
    return seen


def _calls(B, ctx):
    import torch
    ints = lambda *s: Rows(s, dtype=torch.int32)
    B.new_token_order(0, 1, "cpu")
    order = B.sat_token_order(1 << 20, 1 << 20, 4, 9)
    order._keep = (ints(4), ints(4))
    return [lambda: B.sat_layernorm_fwd(ctx, Rows((4, 8)), None, None, 1e-5, Rows((4, 8))), lambda: B.sat_layernorm_bwd(ctx, Rows((4, 8)), Rows((4, 8)), None, Rows((4,)), Rows((4,)), Rows((4, 8))),
            lambda: B.sat_embed_fwd(ctx, ints(4), Rows((9, 8)), 1.0, -1, Rows((4, 8))), lambda: B.sat_token_sort(ctx, ints(4), 2 ** 31 - 1, order),
            lambda: B.sat_embed_bwd(ctx, order, Rows((4, 8)), 1.0, Rows((9, 8))),
            lambda: B.sat_distill_grad(ctx, Rows((4, 8)), ints(4, 2), Rows((4, 2)), 1.0, 0.0, None, None, 1.0, None, Rows((4, 8)))]


def test_tensors_of_another_device(B, calls):
    """The context's device is the one that kernels run on: memory of another is not theirs."""
    import ctypes
    ctx = ctypes.c_void_p(1 << 20)
    ctx.device = 0
    here = _calls(B, ctx)
    for call in here:
        call()
    assert len(calls) == len(here)
    ctx.device = 1
    for call in here:
        with pytest.raises(AssertionError):
            call()
    assert len(calls) == len(here)


def test_numbers_beyond_32_bits(B, calls):
    import torch
    i32, big = torch.int32, 2 ** 32
    ints = lambda *s: Rows(s, dtype=i32)
    order = B.sat_token_order(1 << 20, 1 << 20, 4, 9)
    order._keep = (ints(4), ints(4))
    ok = _calls(B, None)
    for call in ok:
        call()
    assert len(calls) == len(ok)
    wide, far = Rows((1, big + 8)), Rows((4, 8), (big + 8, 1))
    bad = [lambda: B.sat_layernorm_fwd(None, wide, None, None, 1e-5, wide), lambda: B.sat_layernorm_fwd(None, far, None, None, 1e-5, Rows((4, 8))),
           lambda: B.sat_layernorm_fwd(None, Rows((4, 8)), None, None, 1e-5, far), lambda: B.sat_layernorm_bwd(None, Rows((4, 8)), far, None, Rows((4,)), Rows((4,)), Rows((4, 8))),
           lambda: B.sat_embed_fwd(None, ints(4), Rows((big + 9, 8)), 1.0, -1, Rows((4, 8))), lambda: B.sat_embed_fwd(None, ints(4), Rows((9, 8)), 1.0, big, Rows((4, 8))),
           lambda: B.sat_embed_fwd(None, ints(4), Rows((9, 8)), 1.0, -1, far), lambda: B.sat_token_sort(None, ints(4), big, order), lambda: B.sat_embed_bwd(None, order, far, 1.0, Rows((9, 8))),
           lambda: B.sat_embed_bwd(None, order, Rows((4, 8)), 1.0, Rows((9, 8), (big + 8, 1))), lambda: B.new_token_order(4, big + 5, "cpu"),
           lambda: B.sat_distill_grad(None, wide, ints(1, 2), Rows((1, 2)), 1.0, 0.0, None, None, 1.0, None, wide),
           lambda: B.sat_distill_grad(None, Rows((1, 8)), ints(1, big + 1), Rows((1, big + 1)), 1.0, 0.0, None, None, 1.0, None, Rows((1, 8)))]
    for call in bad:
        with pytest.raises(AssertionError):
            call()
    assert len(calls) == len(ok)
