"""The router's weights where scores underflow, and biases that are added to the
scores.  The examples are worked out here, apart from oracle/tokens.py."""
import math

import pytest
import torch

from oracle import tokens as plain
from paper_1912_03203_amd import dynconv as dc
from tests.test_gpu_tokens import TYPES, dev, gen_for, normal, within

pytestmark = pytest.mark.gpu
SIGMOID_SHARES = dc.ROUTE_SIGMOID | dc.ROUTE_RENORMALIZE


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dc.load()


def shares(logits, scale=1.0):
    """Renormalised sigmoid weights from the logits' logarithms, which do not underflow."""
    logs = [v - (math.log1p(math.exp(v)) if v < 0 else v + math.log1p(math.exp(-v))) for v in logits]
    top = max(logs)
    total = sum(math.exp(v - top) for v in logs)
    return [scale * math.exp(v - top) / total for v in logs]


@pytest.mark.parametrize("top_k", [1, 2, 4])
def test_sigmoid_shares_of_far_logits(top_k):
    """Rows whose scores are subnormal in fp32, or 0, share like any other."""
    rows = [[-90.0, -91.0, -92.5, -300.0], [-100.0] * 4, [-88.5, -88.75, -89.0, -87.0], [-3.4e38] * 4,
            [-104.0, -103.0, -103.5, -110.0], [5.0, -200.0, -90.0, 3.0], [80.0, 90.0, 100.0, 300.0],
            [0.0, -1e-3, 1e-3, -50.0], [-1000.0, -1001.0, -999.0, -3e38]]
    r = dc.route(torch.tensor(rows, device="cuda"), top_k, flags=SIGMOID_SHARES, scale=2.5)
    for row, experts, weights in zip(rows, r.expert.tolist(), r.weight.tolist()):
        chosen = sorted(range(4), key=lambda e: (-row[e], e))[:top_k]
        assert experts == chosen
        for got, want in zip(weights, shares([row[e] for e in chosen], 2.5)):
            # exponentials off by 2^-22, their argument by 2^-24 of up to 100
            assert abs(got - want) <= (2.0 ** -20 + 100 * 2.0 ** -24) * want + 1e-37
        assert abs(sum(weights) - 2.5) < 1e-5


@pytest.mark.parametrize("dtype", TYPES)
def test_sigmoid_shares_of_many_rows(dtype):
    gen = gen_for("far")
    for tokens, experts, top_k in ((40, 9, 3), (700, 40, 6), (300, 300, 16)):
        logits = (normal(gen, (tokens, experts), torch.float32, 4.0) - 120 * torch.rand((tokens, 1), generator=gen)).to(dtype)
        r = dc.route(dev(logits), top_k, flags=SIGMOID_SHARES)
        want = plain.route(logits, top_k, None, None, True, True)
        assert torch.equal(r.expert.cpu(), want[0]) and torch.equal(r.rows.cpu(), want[2])
        within(r.weight, want[1], (2.0 ** -20 + 200 * plain.EPS32) * want[1] + 1e-37, "weight")
