"""Every form of the router: experts on 16 or 64 lanes with 1 to 16 of them a lane,
one launch (up to 128 rows) or three, with fewer or more rows a workgroup than its
groups of lanes (8192 rows and more: more).  Choices against a stable sort, weights
against 64 bits."""
import math

import pytest
import torch

from oracle import tokens as plain
from paper_1912_03203_amd import dynconv as dc
from tests.test_gpu_tokens import TYPES, dev, gen_for, normal, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dc.load()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens", [101, 1500, 9001])
@pytest.mark.parametrize("experts", [10, 31, 64, 119, 200, 511, 700])
def test_route_forms(experts, tokens, dtype):
    gen = gen_for("router forms", experts, tokens)
    top_k, flags = min(4, experts), (experts + tokens) % 4
    logits = normal(gen, (tokens, experts), dtype, 2.0)
    logits[::17, experts // 3] = math.nan
    logits[::19, experts // 2:] = -math.inf
    bias = 0.5 * torch.randn(experts, generator=gen)
    mask = (torch.rand(tokens, generator=gen) > 0.1).to(torch.uint8)
    key = logits.float() + bias
    key = key.masked_fill(~(key > -math.inf) | (mask[:, None] == 0), -math.inf)
    best, order = torch.sort(key, dim=1, descending=True, stable=True)  # ties: the lowest expert
    want = torch.where(best[:, :top_k] == -math.inf, -1, order[:, :top_k]).to(torch.int32)
    r = dc.route(dev(logits), top_k, bias=dev(bias), mask=dev(mask), flags=flags, scale=1.5)
    assert torch.equal(r.expert.cpu(), want)
    weight, rows, starts = plain.route_of(logits, want, mask, bool(flags & 1), bool(flags & 2), 1.5)
    assert torch.equal(r.rows.cpu(), rows) and torch.equal(r.starts.cpu(), starts)
    within(r.weight, weight, (2.0 ** -20 + (experts + 100) * plain.EPS32) * weight + 1e-37, "weight")
