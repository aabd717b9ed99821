"""Arguments of the token operators that must not pass as others, on the CPU."""
import ctypes

import pytest
import torch

from paper_1912_03203_amd import dynconv as dc
from tests.test_boundary_tokens import ERR_ARG, ERR_WORKSPACE, FAKE, lib  # noqa: F401


def test_route_flags(lib):  # noqa: F811
    def call(flags):
        r = dc.RoutesStruct(FAKE, FAKE, FAKE, FAKE, 800)
        return lib.dynconv_route(FAKE, 100, 0, 64, 8, FAKE, None, flags, 1.0, ctypes.byref(r), None, 0, None)

    every = dc.ROUTE_SIGMOID | dc.ROUTE_RENORMALIZE | dc.ROUTE_SCORE_BIAS
    assert call(every) == ERR_WORKSPACE  # the flags are fine
    for flags in (4, 16, -1, every | 4):
        assert call(flags) == ERR_ARG


@pytest.mark.parametrize("value", [2**32, 2**31, -2**31 - 1, 1.5, float("inf"), "1", None])
def test_numbers_are_not_cut_to_32_bits(value):
    """A number past 32 bits would arrive as another one, a fraction as its whole part."""
    def bad(name, f):
        with pytest.raises(dc.DynconvError, match=name + ":"):
            f()

    x, w = torch.zeros(6, 16, dtype=torch.float16), torch.zeros(3, 8, 16, dtype=torch.float16)
    y, starts = torch.zeros(6, 8, dtype=torch.float16), torch.zeros(4, dtype=torch.int32)
    bad("top_k", lambda: dc.Router(torch.zeros(4, 8), value))
    bad("flags", lambda: dc.Router(torch.zeros(4, 8), 2, flags=value))
    bad("act", lambda: dc.GroupedLinear(x, y, w, None, starts, act=value))
    bad("src_div", lambda: dc.GroupedLinear(x, y, w, None, starts, src=starts, src_div=value))
    weights = dc.ExpertWeights(w, torch.zeros(3, 16, 8, dtype=torch.float16))
    routes = dc.Routes.alloc(6, 3, 2, "cpu")
    bad("flags", lambda: dc.Experts(x, torch.zeros_like(x), weights, routes, flags=value))
    weights.act = value
    bad("act", lambda: dc.Experts(x, torch.zeros_like(x), weights, routes))
    adapters = dc.Adapters(torch.zeros(2, 8, 16, dtype=torch.float16), torch.zeros(2, 8, 8, dtype=torch.float16))
    ids = torch.zeros(6, dtype=torch.int32)
    bad("act", lambda: dc.AdapterLinear(x, y, w[0].contiguous(), None, adapters, ids, act=value))
