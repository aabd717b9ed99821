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
