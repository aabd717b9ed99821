"""Every form of the products that a call may be given, by its size: few rows a
group at 16 to 64 rows a workgroup, tiles of 64, 128 and 256 rows, each plain,
gated and with fp32 results; against the 64-bit forms of oracle/tokens.py.

A call takes few rows up to a mean of 16 rows a group, and up to 64 where its
64-row tiles are fewer than 192; then the largest tile of which it has 192 (256
rows: 16-bit types and a mean of 256)."""
import math

import pytest
import torch

from oracle import tokens as plain
from paper_1912_03203_amd import dynconv as dc
from tests import util
from tests.test_gpu_tokens import DEV, TYPES, dev, device_weights, expert_case, gen_for, normal, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dc.load()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,groups,c_in,c_out", [
    (120, 3, 136, 104), (168, 3, 72, 72), (118, 3, 8, 24),        # means of 40 and 56: 48 and 64 rows a workgroup
    (5200, 130, 40, 24), (7280, 130, 40, 24),                     # the same with more groups than a wave's lanes
    (9100, 130, 40, 200), (34000, 130, 40, 264), (1100, 5, 264, 1352)])  # 128-, 256- and 128-row tiles
def test_grouped_forms(dtype, rows, groups, c_in, c_out):
    gen = gen_for("forms", rows, groups)
    share = torch.rand(groups, generator=gen) + 0.5
    share[groups // 3] = 0
    cuts = (share.cumsum(0) / share.sum() * rows).round().to(torch.int32)
    cuts[-1] = rows
    starts = torch.cat([torch.zeros(1, dtype=torch.int32), cuts])
    x, w = normal(gen, (rows, c_in), dtype), normal(gen, (groups, c_out, c_in), dtype, c_in ** -0.5)
    b = 0.3 * torch.randn((groups, c_out), generator=gen)
    src, dst = torch.randperm(rows, generator=gen), torch.randperm(rows, generator=gen)
    y = util.Guarded(rows * c_out, dtype, math.nan)
    dc.grouped_linear(dev(x), y.t.view(rows, c_out), dev(w), dev(b), dev(starts), src=dev(src.int()), dst=dev(dst.int()),
                      act=dc.ACT_SILU)
    torch.cuda.synchronize()
    assert y.intact()
    got = y.t.view(rows, c_out).cpu()
    for g in range(groups):
        lo, hi = int(starts[g]), int(starts[g + 1])
        want, err = plain.linear(x[src[lo:hi]], w[g], b[g], plain.SILU)
        within(got[dst[lo:hi]], want, plain.stored(want, err, dtype), "group %d" % g)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,hidden,c_out", [
    (60, 3, 104, 72), (84, 3, 72, 104), (27, 2, 40, 40),    # 48, 64 and 32 rows a workgroup, gated, then with fp32 results
    (200, 2, 72, 104),                                      # 64-row tiles
    (900, 2, 1800, 40), (900, 2, 40, 1800),                 # 128-row tiles: the first product, the second
    (3301, 2, 1096, 40), (3301, 2, 40, 2056)])              # 256-row tiles likewise
@pytest.mark.parametrize("gated", [True, False])
def test_experts_forms(dtype, tokens, experts, hidden, c_out, gated):
    top_k = 2
    x, weights, logits, mask = expert_case(("forms", tokens, hidden), tokens, experts, top_k, 72, hidden, c_out, dtype, gated,
                                           True, dc.ACT_SILU if gated else dc.ACT_RELU, 0.05)
    r = dc.route(dev(logits), top_k, mask=dev(mask))
    some = torch.arange(tokens) if tokens <= 200 else torch.cat([torch.arange(0, tokens, 211), torch.arange(tokens - 5, tokens)])
    want, bound = plain.experts(x[some], weights, r.expert.cpu()[some], r.weight.cpu()[some])
    y = util.Guarded(tokens * c_out, dtype, math.nan)
    call = dc.Experts(dev(x), y.t.view(tokens, c_out), device_weights(weights), r)
    call.ws.fill_(0xFF)
    got = call()
    torch.cuda.synchronize()
    assert y.intact()
    within(got.cpu()[some], want, bound, "experts")
    assert bool(torch.isfinite(got).all())
