"""Whose memory a token operator's call may still read."""
import gc
import weakref

import pytest
import torch

from paper_1912_03203_amd import dynconv as dc
from tests.test_gpu_tokens import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dc.load()


def new(*shape, dtype=torch.float16):
    return torch.zeros(shape, dtype=dtype, device=DEV)


def test_prepared_calls_hold_their_tensors():
    """A prepared call has the addresses of the tensors that it was made with, so it
    holds those, also when the objects that carried them are given others."""
    x = new(6, 16)
    weights = dc.ExpertWeights(new(4, 8, 16), new(4, 16, 8), w_gate=new(4, 8, 16), b_project=new(4, 16, dtype=torch.float32))
    routes = dc.Routes.alloc(6, 4, 2, DEV)
    adapters = dc.Adapters(new(2, 8, 16), new(2, 24, 8), scales=new(2, dtype=torch.float32))
    calls = [dc.Router(new(6, 4), 2, routes=routes), dc.Experts(x, new(6, 16), weights, routes),
             dc.AdapterLinear(x, new(6, 24), new(24, 16), None, adapters, new(6, dtype=torch.int32))]
    held = []
    for carrier in (weights, routes, adapters):
        for name, t in list(vars(carrier).items()):
            if isinstance(t, torch.Tensor):
                held.append((name, weakref.ref(t)))
                setattr(carrier, name, torch.zeros_like(t))
    del t
    gc.collect()
    assert [name for name, r in held if r() is None] == []
    del calls
    gc.collect()
    assert [name for name, r in held if r() is not None] == []
