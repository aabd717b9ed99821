"""The token operators on the GPU against plain 64-bit forms (oracle/tokens.py).
Choices and lists are exact; every output value lies within the elementwise
bound that the oracle derives from the roundings."""
import math
import zlib

import pytest
import torch

from oracle import tokens as plain
from paper_1912_03203_amd import dynconv as dc
from tests import util

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dc.load()


def gen_for(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


def dev(t):
    return None if t is None else t.to(DEV)


def within(got, want, bound, what):
    got = got.cpu().double()
    both_nan = torch.isnan(got) & torch.isnan(want)
    off = torch.where(both_nan | (got == want), torch.zeros_like(want), (got - want).abs())
    bad = ~(off <= bound)
    assert not bool(bad.any()), "%s: %d values outside their bound, worst %.3g of it" % (
        what, int(bad.sum()), float((off / bound.clamp(min=1e-300)).max()))


# -------------------------------------------------------------------- router
def check_route(logits, top_k, bias=None, mask=None, flags=0, scale=1.0):
    want = plain.route(logits, top_k, bias, mask, bool(flags & dc.ROUTE_SIGMOID), bool(flags & dc.ROUTE_RENORMALIZE), scale)
    r = dc.route(dev(logits), top_k, bias=dev(bias), mask=dev(mask), flags=flags, scale=scale)
    torch.cuda.synchronize()
    assert torch.equal(r.expert.cpu(), want[0])
    assert torch.equal(r.starts.cpu(), want[3])
    assert torch.equal(r.rows.cpu(), want[2])
    # exponentials off by 2^-22, their argument by 2^-24 of up to 100, sums of up to 1024 terms
    bound = (2.0 ** -20 + logits.shape[1] * plain.EPS32 + 100 * plain.EPS32) * want[1].abs() + 1e-37
    within(r.weight, want[1], bound, "weight")
    return r


@pytest.mark.parametrize("tokens,experts,top_k", [
    (1, 1, 1), (1, 64, 8), (3, 5, 5), (7, 16, 4), (33, 17, 2), (255, 32, 8), (256, 64, 8), (257, 64, 8), (100, 128, 16),
    (129, 129, 16), (300, 256, 3), (500, 257, 1), (1000, 512, 7), (70, 1024, 16), (1500, 1000, 2), (4097, 8, 2)])
def test_route_sizes(tokens, experts, top_k):
    gen = gen_for("route", tokens, experts)
    dtype = TYPES[(tokens + experts) % 3]
    flags = (tokens % 2) * dc.ROUTE_SIGMOID + (experts % 2) * dc.ROUTE_RENORMALIZE
    mask = (torch.rand(tokens, generator=gen) > 0.2).to(torch.uint8) * 3 if tokens % 3 else None
    bias = 0.5 * torch.randn(experts, generator=gen) if top_k % 2 else None
    check_route(normal(gen, (tokens, experts), dtype), top_k, bias, mask, flags, 1.5)


@pytest.mark.parametrize("flags", range(4))
@pytest.mark.parametrize("dtype", TYPES)
def test_route_weights(flags, dtype):
    gen = gen_for("weights", flags)
    check_route(normal(gen, (37, 40), dtype, 4.0), 6, None, None, flags, 2.0)
    check_route(normal(gen, (37, 40), dtype, 4.0), 6, torch.randn(40, generator=gen), None, flags)


@pytest.mark.parametrize("flags", range(4))
def test_route_ties_and_special_values(flags):
    inf, nan = math.inf, math.nan
    rows = [[0.0] * 8, [-0.0, 0.0] * 4, [nan] * 8, [-inf] * 8, [nan, -inf, 1, -inf, nan, 1, -inf, -inf],
            [inf, 0, inf, -inf, 1, 2, 3, nan], [3.4e38, -3.4e38, 3.4e38, 0, 0, 0, 0, 0], [1, 2, 2, 3, 3, 3, -inf, 2],
            [-100.0] * 8, [-3.4e38] * 8, [88, -88, 0, 1e-40, -1e-40, 0, 5, 5], [-inf] * 7 + [-5.0]]
    for top_k in (1, 3, 8):
        logits = torch.tensor(rows)
        want = plain.route(logits, top_k, None, None, bool(flags & 1), bool(flags & 2))
        r = dc.route(dev(logits), top_k, flags=flags)
        assert torch.equal(r.expert.cpu(), want[0]) and torch.equal(r.rows.cpu(), want[2])
        # the sigmoids of -100 and below are subnormal in fp32, or 0: what they share is not held to a bound
        fine = [i for i in range(len(rows)) if not (flags & 1 and i in (6, 8, 9, 10))]
        within(r.weight[fine], want[1][fine], 2.0 ** -19 * want[1][fine].abs() + 1e-37, "weight")
        assert bool(torch.isfinite(r.weight).all())


def test_route_masks():
    gen = gen_for("mask")
    logits = normal(gen, (700, 24), torch.float32)
    for mask in (torch.zeros(700), torch.ones(700), (torch.arange(700) % 7 == 0), (torch.arange(700) > 690)):
        check_route(logits, 4, None, mask.to(torch.uint8))
    logits[:, 3:] = -math.inf  # one expert takes every row, slots stay empty
    logits[:, :2] = math.nan
    check_route(logits, 4)


def test_route_unaligned_rows_and_no_rows():
    gen = gen_for("odd")
    base = normal(gen, (1 + 41 * 23,), torch.float16).to(DEV)
    view = base[1:].view(41, 23)  # 2-byte aligned
    got = dc.route(view, 3)
    want = plain.route(view.cpu(), 3)
    assert torch.equal(got.expert.cpu(), want[0]) and torch.equal(got.rows.cpu(), want[2])
    empty = dc.route(torch.empty((0, 23), dtype=torch.float16, device=DEV), 3)
    assert empty.starts.cpu().tolist() == [0] * 24


def test_route_stays_in_its_buffers():
    gen = gen_for("guard")
    for tokens, experts, top_k in ((5, 9, 4), (900, 33, 5)):
        n = tokens * top_k
        bufs = [util.Guarded(n, torch.int32), util.Guarded(n, torch.float32), util.Guarded(n, torch.int32),
                util.Guarded(experts + 1, torch.int32)]
        ws = util.Guarded(dc.load().dynconv_route_workspace_bytes(tokens, experts, top_k), torch.uint8)
        routes = dc.Routes(bufs[0].t.view(tokens, top_k), bufs[1].t.view(tokens, top_k), bufs[2].t, bufs[3].t)
        dc.Router(normal(gen, (tokens, experts), torch.float32).to(DEV), top_k, routes=routes, ws=ws.t)()
        torch.cuda.synchronize()
        assert all(b.intact() for b in bufs) and ws.intact()


# ------------------------------------------------------------------ products
def split(gen, rows, groups, empty):
    """starts of `groups` ragged groups of `rows` rows, some of them empty."""
    share = torch.rand(groups, generator=gen) ** 2
    share[torch.rand(groups, generator=gen) < empty] = 0
    if float(share.sum()) == 0:
        share[groups // 2] = 1
    cuts = (share.cumsum(0) / share.sum() * rows).round().to(torch.int32)
    cuts[-1] = rows
    return torch.cat([torch.zeros(1, dtype=torch.int32), cuts])


def check_grouped(key, rows, groups, c_in, c_out, dtype, lists="none", kind=dc.ACT_NONE, bias=True, empty=0.2, div=1):
    gen = gen_for("grouped", key)
    starts = split(gen, rows, groups, empty)
    w = normal(gen, (groups, c_out, c_in), dtype, c_in ** -0.5)
    b = 0.3 * torch.randn((groups, c_out), generator=gen) if bias else None
    x = normal(gen, (rows if lists in ("none", "scatter") else max(1, rows // div + 3), c_in), dtype)
    src = torch.randint(0, x.shape[0] * div, (rows,), generator=gen, dtype=torch.int32) if lists in ("gather", "both") else None
    y_rows = rows + (5 if lists in ("scatter", "both") else 0)
    dst = torch.randperm(y_rows, generator=gen)[:rows].to(torch.int32) if lists in ("scatter", "both") else None
    y = torch.full((y_rows, c_out), 7.0, dtype=dtype)
    want, bound = plain.grouped(x, y, w, b, starts, src, div, dst, kind)
    out = util.Guarded(y.numel(), dtype, 7.0)
    got = dc.grouped_linear(dev(x), out.t.view(y.shape), dev(w), dev(b), dev(starts), dev(src), div, dev(dst), kind)
    torch.cuda.synchronize()
    assert out.intact()
    within(got, want, bound, "grouped")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,groups,c_in,c_out", [
    (1, 1, 8, 8), (1, 4, 64, 24), (15, 3, 72, 40), (40, 16, 136, 16), (90, 3, 200, 104), (17, 1, 512, 8), (64, 1, 40, 72),
    (150, 3, 264, 48), (300, 2, 64, 136), (131, 1, 8, 264), (400, 3, 328, 264), (257, 1, 128, 128)])
def test_grouped_sizes(dtype, rows, groups, c_in, c_out):
    check_grouped((rows, groups, c_in), rows, groups, c_in, c_out, dtype)


@pytest.mark.parametrize("lists", ["gather", "scatter", "both"])
@pytest.mark.parametrize("rows,groups", [(30, 7), (200, 4), (500, 2)])
def test_grouped_lists(lists, rows, groups):
    check_grouped((lists, rows), rows, groups, 96, 56, TYPES[rows % 3], lists, dc.ACT_RELU, empty=0.4, div=3 if rows != 200 and lists != "scatter" else 1)


@pytest.mark.parametrize("kind", range(5))
@pytest.mark.parametrize("rows", [20, 300])
def test_grouped_activations(kind, rows):
    check_grouped((kind, rows), rows, 2, 48, 40, TYPES[kind % 3], kind=kind)
    check_grouped((kind, rows, 1), rows, 2, 48, 40, TYPES[(kind + 1) % 3], kind=kind, bias=False)


@pytest.mark.parametrize("rows,c_out,dtype", [(1700, 2000, t) for t in TYPES] + [(5000, 4104, t) for t in TYPES[1:]])
def test_grouped_large_tiles(rows, c_out, dtype):
    """Sizes that take 128- and 256-row tiles, odd edges on every side."""
    gen = gen_for("large", rows)
    groups, c_in = 3, 200
    cut = rows // 3 - 17
    starts = torch.tensor([0, cut, cut, rows], dtype=torch.int32)
    w = normal(gen, (groups, c_out, c_in), dtype, c_in ** -0.5)
    x = normal(gen, (rows, c_in), dtype)
    b = torch.randn((groups, c_out), generator=gen)
    src, dst = torch.randperm(rows, generator=gen), torch.randperm(rows, generator=gen)
    y = dc.grouped_linear(dev(x), torch.empty((rows, c_out), dtype=dtype, device=DEV), dev(w), dev(b), dev(starts),
                          src=dev(src.int()), dst=dev(dst.int()), act=dc.ACT_GELU).cpu()
    for lo, hi, g in ((0, cut, 0), (cut, rows, 2)):
        want, err = plain.linear(x[src[lo:hi]], w[g], b[g], plain.GELU)
        within(y[dst[lo:hi]], want, plain.stored(want, err, dtype), "large")


def test_grouped_skips_what_lists_do_not_name():
    """Entries outside their range, starts past the list, rows behind the last
    group: nothing is computed or written for them."""
    gen = gen_for("skip")
    for rows in (24, 700):
        x, w = normal(gen, (rows, 64), torch.float16), normal(gen, (2, 32, 64), torch.float16, 0.125)
        src = torch.arange(rows, dtype=torch.int32)
        dst = torch.arange(rows, dtype=torch.int32)
        src[3], src[7], dst[5], dst[9] = -1, rows, -5, rows + 2
        y = torch.full((rows, 32), 3.0, dtype=torch.float16)
        for starts in ([0, rows // 2, rows - 4], [-3, rows // 3, rows + 100], [0, 0, 0], [rows, rows, rows]):
            st = torch.tensor(starts, dtype=torch.int32)
            want, bound = plain.grouped(x, y, w, None, st, src, 1, dst)
            got = dc.grouped_linear(dev(x), dev(y), dev(w), None, dev(st), src=dev(src), dst=dev(dst))
            within(got, want, bound, "skip")


@pytest.mark.parametrize("rows", [20, 900])
def test_grouped_refuses_starts_that_do_not_ascend(rows):
    """Nothing is computed or written, whatever the groups around the fault."""
    gen = gen_for("descend", rows)
    x, w = normal(gen, (rows, 64), torch.float16), normal(gen, (70, 32, 64), torch.float16, 0.125)
    for at in (1, 40, 66):
        starts = torch.arange(71, dtype=torch.int32) * rows // 70
        starts[at] = rows + 7 if at < 60 else -2
        y = torch.full((rows, 32), 3.0, dtype=torch.float16, device=DEV)
        dc.grouped_linear(dev(x), y, dev(w), None, dev(starts))
        assert bool((y == 3.0).all())


def test_grouped_many_groups():
    """More groups than a wave looks at in one step, in every form of the products."""
    for rows, groups in ((300, 130), (2600, 130), (9000, 70)):
        check_grouped(("many", rows), rows, groups, 40, 24, TYPES[rows % 3], kind=dc.ACT_RELU)
        check_grouped(("many", rows, 1), rows, groups, 40, 24, TYPES[(rows + 1) % 3], "both", div=2)


def test_grouped_keeps_nan_in_its_rows():
    gen = gen_for("nan")
    for rows in (30, 400):
        x, w = normal(gen, (rows, 72), torch.bfloat16), normal(gen, (2, 40, 72), torch.bfloat16, 0.1)
        x[4], x[11] = math.nan, math.inf
        starts = torch.tensor([0, 8, rows - 3], dtype=torch.int32)
        x[rows - 2] = math.nan  # behind the last group
        y = torch.zeros((rows, 40), dtype=torch.bfloat16)
        for kind in range(1, 5):
            acted = dc.grouped_linear(dev(x), dev(y), dev(w), None, dev(starts), act=kind).cpu()
            assert bool(torch.isnan(acted[4]).all()) and not bool(torch.isnan(acted[5:11]).any())
        want, bound = plain.grouped(x, y, w, None, starts)
        got = dc.grouped_linear(dev(x), dev(y), dev(w), None, dev(starts)).cpu().double()
        fine = torch.tensor([i for i in range(rows) if i not in (4, 11)])
        within(got[fine], want[fine], bound[fine], "beside NaN")
        assert bool(torch.isnan(got[4]).all()) and not bool(torch.isfinite(got[11]).any())


# ------------------------------------------------------------------- experts
def expert_case(key, tokens, experts, top_k, c_in, hidden, c_out, dtype, gated, biases, kind, masked=0.0):
    gen = gen_for("experts", key)
    weights = {"w_expand": normal(gen, (experts, hidden, c_in), dtype, c_in ** -0.5),
               "w_gate": normal(gen, (experts, hidden, c_in), dtype, c_in ** -0.5) if gated else None,
               "w_project": normal(gen, (experts, c_out, hidden), dtype, hidden ** -0.5), "act": kind}
    for name, width in (("b_expand", hidden), ("b_gate", hidden if gated else 0), ("b_project", c_out)):
        weights[name] = 0.2 * torch.randn((experts, width), generator=gen) if biases and width else None
    x = normal(gen, (tokens, c_in), dtype)
    logits = normal(gen, (tokens, experts), torch.float32) + torch.randn(experts, generator=gen)
    mask = (torch.rand(tokens, generator=gen) >= masked).to(torch.uint8) if masked else None
    return x, weights, logits, mask


def device_weights(weights):
    return dc.ExpertWeights(**{k: v if k == "act" else dev(v) for k, v in weights.items()})


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,top_k,c_in,hidden,c_out,gated,biases,residual", [
    (1, 8, 2, 64, 48, 64, True, False, True), (5, 4, 4, 40, 24, 72, False, True, False),
    (33, 6, 2, 136, 72, 136, True, True, True), (120, 3, 2, 96, 104, 96, True, False, False),
    (200, 2, 1, 48, 136, 48, False, False, True), (260, 3, 3, 72, 264, 200, True, True, False),
    # few tokens, whose experts seldom meet: more slots than waves, masked tokens, one expert
    (1, 40, 16, 200, 88, 72, False, True, False), (10, 96, 4, 72, 264, 72, True, True, True),
    (3, 64, 10, 136, 40, 136, True, False, True), (1, 1, 1, 8, 8, 8, True, True, True)])
def test_experts(dtype, tokens, experts, top_k, c_in, hidden, c_out, gated, biases, residual):
    kind = dc.ACT_SILU if gated else dc.ACT_GELU
    x, weights, logits, mask = expert_case((tokens, experts), tokens, experts, top_k, c_in, hidden, c_out, dtype, gated,
                                           biases, kind, 0.3 if tokens % 5 == 0 else 0.0)
    r = dc.route(dev(logits), top_k, mask=dev(mask), flags=dc.ROUTE_RENORMALIZE)
    want, bound = plain.experts(x, weights, r.expert.cpu(), r.weight.cpu(), residual)
    y = util.Guarded(tokens * c_out, dtype, math.nan)
    call = dc.Experts(dev(x), y.t.view(tokens, c_out), device_weights(weights), r,
                      flags=dc.EXPERTS_RESIDUAL if residual else 0)
    call.ws.fill_(0xFF)  # NaN everywhere: what is not written must not count
    got = call()
    torch.cuda.synchronize()
    assert y.intact()
    within(got, want, bound, "experts")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,experts,top_k,c_in,hidden,c_out,gated", [
    (1, 8, 8, 72, 1096, 168, True), (1, 1, 1, 136, 40, 72, False), (2, 22, 4, 168, 1568, 168, True),
    (3, 64, 10, 136, 264, 136, False), (8, 1024, 16, 64, 72, 64, True)])
def test_experts_of_few_tokens_keep_the_hidden_rows(dtype, tokens, experts, top_k, c_in, hidden, c_out, gated):
    """The bound without the hidden rows' rounding, which small results would go past:
    it leaves the result's own."""
    kind = dc.ACT_SILU if gated else dc.ACT_GELU
    x, weights, logits, _ = expert_case(("few", tokens, experts), tokens, experts, top_k, c_in, hidden, c_out, dtype,
                                        gated, True, kind)
    r = dc.route(dev(logits), top_k)
    want, bound = plain.experts(x, weights, r.expert.cpu(), r.weight.cpu(), few=True)
    y = util.Guarded(tokens * c_out, dtype, math.nan)
    call = dc.Experts(dev(x), y.t.view(tokens, c_out), device_weights(weights), r)
    guard = util.Guarded(call.ws.numel(), torch.uint8)
    call = dc.Experts(dev(x), y.t.view(tokens, c_out), device_weights(weights), r, ws=guard.t)
    guard.t.fill_(0xFF)
    got = call()
    torch.cuda.synchronize()
    assert y.intact() and guard.intact()
    within(got, want, bound, "few tokens")


def test_experts_of_few_tokens_beside_infinities():
    """An infinite weight meets the second half of a hidden entry, which may be zero or of
    the other sign: the result is still the formula's infinity; a hidden entry past fp16's
    largest value is infinite alone."""
    for dtype in TYPES[1:]:
        x, weights, logits, _ = expert_case("inf", 1, 4, 1, 64, 64, 64, dtype, False, False, dc.ACT_RELU)
        r = dc.route(dev(logits), 1)
        e = int(r.expert[0, 0])
        h = torch.relu(weights["w_expand"][e].double() @ x[0].double())
        k = int(h.argmax())
        weights["w_project"][e, 5, k] = math.inf
        weights["w_project"][e, 6, k] = -math.inf
        y = torch.zeros((1, 64), dtype=dtype, device=DEV)
        got = dc.experts_forward(dev(x), y, device_weights(weights), r).cpu()[0]
        assert got[5] == math.inf and got[6] == -math.inf and int(torch.isfinite(got).sum()) == 62
        weights["w_project"][e, 5:7, k] = 1.0
        weights["b_expand"] = torch.zeros((4, 64))
        weights["b_expand"][e, k] = math.inf
        weights["w_project"][e, :, k] = 0.5
        got = dc.experts_forward(dev(x), y, device_weights(weights), r).cpu()[0]
        assert bool((got == math.inf).all())


@pytest.mark.parametrize("tokens,dtype", [(900, t) for t in TYPES] + [(3301, t) for t in TYPES[1:]])
def test_experts_large_tiles(tokens, dtype):
    """Rows and widths for the 128- and 256-row tiles, gated, with edges on every side."""
    top_k = 2
    x, weights, logits, mask = expert_case("large", tokens, 2, top_k, 72, 1096, 72, dtype, True, True, dc.ACT_SILU, 0.05)
    r = dc.route(dev(logits), top_k, mask=dev(mask))
    some = torch.cat([torch.arange(0, tokens, 97), torch.arange(tokens - 9, tokens)])
    want, bound = plain.experts(x[some], weights, r.expert.cpu()[some], r.weight.cpu()[some], True)
    got = dc.experts_forward(dev(x), torch.full((tokens, 72), math.nan, dtype=dtype, device=DEV), device_weights(weights), r,
                             flags=dc.EXPERTS_RESIDUAL)
    within(got.cpu()[some], want, bound, "large experts")
    assert bool(torch.isfinite(got).all())


def test_experts_in_place_and_all_rows_masked():
    x, weights, logits, _ = expert_case("place", 50, 4, 2, 64, 40, 64, torch.bfloat16, True, False, dc.ACT_SILU)
    for mask in (None, torch.zeros(50, dtype=torch.uint8)):
        r = dc.route(dev(logits), 2, mask=dev(mask))
        want, bound = plain.experts(x, weights, r.expert.cpu(), r.weight.cpu(), True)
        xd = dev(x)
        got = dc.experts_forward(xd, xd, device_weights(weights), r, flags=dc.EXPERTS_RESIDUAL)
        within(got, want, bound, "in place")
        y = dc.experts_forward(dev(x), torch.full_like(xd, math.nan), device_weights(weights), r)
        if mask is not None:
            assert torch.equal(got.cpu(), x) and int(torch.count_nonzero(y)) == 0


# ------------------------------------------------------------------ adapters
def check_adapters(key, rows, adapters, max_rank, c_in, c_out, dtype, ranks=True, scales=True, kind=dc.ACT_NONE,
                   order="runs"):
    gen = gen_for("adapters", key)
    x, w = normal(gen, (rows, c_in), dtype), normal(gen, (c_out, c_in), dtype, c_in ** -0.5)
    b = 0.2 * torch.randn(c_out, generator=gen)
    down = normal(gen, (adapters, max_rank, c_in), dtype, c_in ** -0.5)
    up = normal(gen, (adapters, c_out, max_rank), dtype, max_rank ** -0.5)
    ids = torch.randint(-1, adapters, (rows,), generator=gen, dtype=torch.int32)
    if order == "runs":
        ids = ids.sort().values
        ids = ids.roll(rows // 3)
    if order == "none":
        ids[:] = -1
    if rows > 4:
        ids[2] = adapters + 3  # no such adapter
    rk = torch.randint(0, max_rank + 1, (adapters,), generator=gen, dtype=torch.int32) if ranks else None
    if ranks:
        rk[0] = max_rank + 9  # counts as max_rank
        for i in range(adapters):
            down[i, min(int(rk[i]), max_rank):] = math.nan  # not read
    sc = torch.rand(adapters, generator=gen) + 0.5 if scales else None
    want, bound = plain.adapted(x, w, b, down, up, ids, sc, rk, kind)
    y = util.Guarded(rows * c_out, dtype, math.nan)
    call = dc.AdapterLinear(dev(x), y.t.view(rows, c_out), dev(w), dev(b), dc.Adapters(dev(down), dev(up), dev(sc), dev(rk)),
                            dev(ids), act=kind)
    call.ws.fill_(0xFF)
    got = call()
    torch.cuda.synchronize()
    assert y.intact()
    within(got, want, bound, "adapters")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,adapters,max_rank,c_in,c_out", [
    (1, 1, 8, 8, 8), (1, 5, 16, 136, 40), (7, 20, 24, 72, 24), (33, 3, 64, 200, 72), (64, 64, 16, 64, 136),
    (100, 4, 40, 96, 72), (260, 7, 128, 72, 136), (300, 2, 256, 328, 40)])
def test_adapters(dtype, rows, adapters, max_rank, c_in, c_out):
    check_adapters((rows, adapters, max_rank), rows, adapters, max_rank, c_in, c_out, dtype)


@pytest.mark.parametrize("order", ["mixed", "none"])
@pytest.mark.parametrize("rows", [20, 60, 200])
def test_adapters_in_any_order(order, rows):
    check_adapters((order, rows), rows, 9, 16, 72, 56, TYPES[rows % 3], rows != 60, rows != 20, dc.ACT_SILU, order)


@pytest.mark.parametrize("rank,c_out,dtype", [(16, 72, torch.float16), (24, 4104, torch.bfloat16), (128, 136, torch.bfloat16),
                                              (64, 72, torch.float32), (40, 1000, torch.bfloat16), (8, 1000, torch.float32)])
def test_adapters_large_tiles(rank, c_out, dtype):
    gen = gen_for("adapters large", rank)
    rows, c_in, n = 4200, 136, 5
    x, w = normal(gen, (rows, c_in), dtype), normal(gen, (c_out, c_in), dtype, c_in ** -0.5)
    down, up = normal(gen, (n, rank, c_in), dtype, c_in ** -0.5), normal(gen, (n, c_out, rank), dtype, rank ** -0.5)
    ids = (torch.arange(rows) // 700 - 1).to(torch.int32)
    y = dc.adapter_linear(dev(x), torch.empty((rows, c_out), dtype=dtype, device=DEV), dev(w), None,
                          dc.Adapters(dev(down), dev(up)), dev(ids))
    for i in range(-1, n):
        at = torch.nonzero(ids == i).flatten()
        want, err = plain.linear(x[at], w, None)
        if i >= 0:
            v, ev = plain.linear(x[at], down[i], None)
            more, em = plain.linear((v, plain.stored(v, ev, dtype)), up[i], None)
            want, err = want + more, err + em + plain.MORE * plain.EPS32 * (want.abs() + more.abs())
        within(y[at.to(DEV)], want, plain.stored(want, err, dtype), "adapter %d" % i)


# ------------------------------------------------------------------ together
def layer(gen, dtype, tokens, c, hidden, experts, top_k):
    """Everything of one layer: a mask unit decides which rows run, a projection
    with adapters makes the router's logits, the router and the experts do the rest."""
    s = {"x": dev(normal(gen, (tokens, c), dtype)), "w_mask": dev(torch.randn(c, generator=gen)),
         "w": dev(normal(gen, (experts, c), dtype, c ** -0.5)),
         "adapters": dc.Adapters(dev(normal(gen, (3, 8, c), dtype, c ** -0.5)), dev(normal(gen, (3, experts, 8), dtype, 0.3))),
         "ids": dev(torch.randint(-1, 3, (tokens,), generator=gen, dtype=torch.int32)),
         "weights": dc.ExpertWeights(dev(normal(gen, (experts, hidden, c), dtype, c ** -0.5)),
                                     dev(normal(gen, (experts, c, hidden), dtype, hidden ** -0.5)),
                                     w_gate=dev(normal(gen, (experts, hidden, c), dtype, c ** -0.5)))}
    s["mask"] = torch.empty(tokens, dtype=torch.uint8, device=DEV)
    s["logits"] = torch.empty((tokens, experts), dtype=dtype, device=DEV)
    s["y"] = torch.empty_like(s["x"])
    s["project"] = dc.AdapterLinear(s["x"], s["logits"], s["w"], None, s["adapters"], s["ids"])
    s["router"] = dc.Router(s["logits"], top_k, mask=s["mask"], flags=dc.ROUTE_RENORMALIZE)
    s["experts"] = dc.Experts(s["x"], s["y"], s["weights"], s["router"].routes, flags=dc.EXPERTS_RESIDUAL)
    return s


def run_layer(s, stream=None):
    x = s["x"]
    dc.mask(x.view(x.shape[0], 1, 1, -1), s["w_mask"], 0.1, out=s["mask"], stream=stream)
    s["project"](stream)
    s["router"](stream)
    return s["experts"](stream)


@pytest.mark.parametrize("tokens", [1, 90, 700])
def test_a_layer_of_them(tokens):
    """Mask unit, projection with adapters, router and experts as one layer, then
    the same layer on another stream and as a graph replayed on new inputs."""
    gen = gen_for("layer", tokens)
    dtype = torch.bfloat16
    s = layer(gen, dtype, tokens, 64, 48, 8, 2)
    run_layer(s)
    torch.cuda.synchronize()
    on = s["mask"].cpu()
    logits, lb = plain.adapted(s["x"].cpu(), s["w"].cpu(), None, s["adapters"].down.cpu(), s["adapters"].up.cpu(), s["ids"].cpu())
    within(s["logits"], logits, lb, "logits")
    r = plain.route(s["logits"].cpu(), 2, None, on, False, True)
    assert torch.equal(s["router"].routes.expert.cpu(), r[0]) and torch.equal(s["router"].routes.rows.cpu(), r[2])
    weights = {k: None if getattr(s["weights"], k) is None else getattr(s["weights"], k).cpu()
               for k in ("w_expand", "w_gate", "w_project", "b_expand", "b_gate", "b_project")}
    weights["act"] = dc.ACT_SILU
    want, bound = plain.experts(s["x"].cpu(), weights, r[0], s["router"].routes.weight.cpu(), True)
    within(s["y"], want, bound, "layer")
    assert torch.equal(s["y"].cpu()[on == 0], s["x"].cpu()[on == 0])

    first = s["y"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s["y"].fill_(math.nan)
    torch.cuda.synchronize()
    run_layer(s, side)
    side.synchronize()
    assert torch.equal(s["y"], first)

    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run_layer(s, side)
    torch.cuda.synchronize()
    for i in range(4):
        fresh = normal(gen, (tokens, 64), dtype).to(DEV)
        s["x"].copy_(fresh)
        s["y"].fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        replayed = s["y"].clone()
        run_layer(s)
        torch.cuda.synchronize()
        assert torch.equal(replayed, s["y"]) and bool(torch.isfinite(replayed).all())


def test_two_layers_at_once():
    """Two streams with buffers of their own do not disturb each other."""
    gen = gen_for("two")
    layers = [layer(gen, torch.float16, n, 128, 64, 16, 4) for n in (300, 37)]
    alone = []
    for s in layers:
        alone.append(run_layer(s).clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for s, st in zip(layers, streams):
            run_layer(s, st)
    torch.cuda.synchronize()
    assert all(torch.equal(s["y"], a) for s, a in zip(layers, alone))


def test_runs_repeat_bit_for_bit():
    gen = gen_for("repeat")
    s = layer(gen, torch.bfloat16, 1000, 256, 128, 32, 4)
    first = run_layer(s).clone()
    routes = [t.clone() for t in (s["router"].routes.rows, s["router"].routes.weight)]
    for _ in range(3):
        assert torch.equal(run_layer(s), first)
        assert torch.equal(s["router"].routes.rows, routes[0]) and torch.equal(s["router"].routes.weight, routes[1])
