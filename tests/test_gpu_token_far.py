"""The token operators past 2^31 entries and bytes, and at the largest widths."""
import pytest
import torch

from oracle import tokens as plain
from paper_1912_03203_amd import dynconv as dc
from tests.test_gpu_tokens import DEV, dev, gen_for, normal, within

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    dc.load()


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def test_route_past_2_to_31_logits():
    tokens, experts, top_k = 8_500_003, 256, 2  # 2.18e9 logits
    logits = torch.zeros((tokens, experts), dtype=BF16, device=DEV)
    gen = gen_for("far route")
    some = torch.cat([torch.arange(40), torch.randint(0, tokens, (200,), generator=gen), torch.arange(tokens - 40, tokens)])
    some = some.unique()
    logits[some.to(DEV)] = dev(normal(gen, (len(some), experts), BF16))
    r = dc.route(logits, top_k, flags=dc.ROUTE_RENORMALIZE)
    want = plain.route(logits[some.to(DEV)].cpu(), top_k, renormalize=True)
    assert torch.equal(r.expert[some.to(DEV)].cpu(), want[0])
    within(r.weight[some.to(DEV)], want[1], 2.0 ** -19 * want[1], "weight")
    # the lists against a stable sort of all assignments
    flat = r.expert.reshape(-1)
    rows = torch.sort(flat, stable=True).indices.to(torch.int32)
    assert torch.equal(r.rows, rows)
    counts = torch.bincount(flat, minlength=experts).cumsum(0)
    assert torch.equal(r.starts[1:].long(), counts) and int(r.starts[0]) == 0


@pytest.mark.parametrize("rows", [40, 9800])
def test_grouped_of_far_rows_and_weights(rows):
    """Rows and weights on both sides of 2^31 entries; in the few-rows form and in tiles."""
    gen = gen_for("far rows", rows)
    c, groups, far = 4096, 140, 600_000  # 2.46e9 entries of x and y, 2.35e9 of w
    x = torch.zeros((far, c), dtype=BF16, device=DEV)
    w = torch.zeros((groups, c, c), dtype=BF16, device=DEV)
    y = torch.full((far, c), 5.0, dtype=BF16, device=DEV)
    starts = torch.zeros(groups + 1, dtype=torch.int32)
    starts[1:] = rows // 2
    starts[groups - 1:] = rows // 2 + 3
    starts[groups:] = rows
    for g in (0, groups - 2, groups - 1):
        w[g, :64] = dev(normal(gen, (64, c), BF16, c ** -0.5))
        w[g, -64:] = dev(normal(gen, (64, c), BF16, c ** -0.5))
    src = torch.cat([torch.arange(rows // 2), torch.arange(far - (rows - rows // 2), far)]).to(torch.int32)
    dst = src.flip(0).contiguous()
    x[dev(src.long())] = dev(normal(gen, (rows, c), BF16))
    dc.grouped_linear(x, y, w, None, dev(starts), src=dev(src), dst=dev(dst))
    got, taken = y[dev(dst.long())].cpu(), x[dev(src.long())].cpu()
    for lo, hi, g in ((0, rows // 2, 0), (rows // 2, rows // 2 + 3, groups - 2), (rows // 2 + 3, rows, groups - 1)):
        at = torch.arange(lo, hi, max(1, (hi - lo) // 100))
        want, err = plain.linear(taken[at], w[g].cpu(), None)
        within(got[at], want, plain.stored(want, err, BF16), "group %d" % g)
    y[dev(dst.long())] = 5.0
    assert bool((y == 5.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_grouped_at_the_largest_widths(dtype):
    gen = gen_for("wide")
    for rows, c_in, c_out in ((3, 65536, 8), (70, 65536, 40), (3, 8, 65536), (300, 16, 65536)):
        x, w = normal(gen, (rows, c_in), dtype), normal(gen, (1, c_out, c_in), dtype, c_in ** -0.5)
        y = torch.empty((rows, c_out), dtype=dtype, device=DEV)
        starts = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
        got = dc.grouped_linear(dev(x), y, dev(w), None, starts)
        want, err = plain.linear(x, w[0], None)
        within(got, want, plain.stored(want, err, dtype), "wide")


def test_adapters_of_far_rows():
    """2.2 GB of first halves' results, adapters past 2^31 bytes."""
    gen = gen_for("far adapters")
    rows, c_in, c_out, rank, adapters = 2_200_000, 8, 8, 256, 600_000
    x, w = normal(gen, (rows, c_in), BF16), normal(gen, (c_out, c_in), BF16)
    down = torch.zeros((adapters, rank, c_in), dtype=BF16, device=DEV)
    up = torch.zeros((adapters, c_out, rank), dtype=BF16, device=DEV)
    used = torch.tensor([0, 1, adapters // 2, adapters - 2, adapters - 1])
    down[dev(used)] = dev(normal(gen, (5, rank, c_in), BF16, 0.3))
    up[dev(used)] = dev(normal(gen, (5, c_out, rank), BF16, 0.1))
    ids = used[torch.arange(rows) * 5 // rows].to(torch.int32)
    y = torch.empty((rows, c_out), dtype=BF16, device=DEV)
    got = dc.adapter_linear(dev(x), y, dev(w), None, dc.Adapters(down, up), dev(ids))
    some = torch.cat([torch.arange(300), torch.randint(0, rows, (500,), generator=gen), torch.arange(rows - 300, rows)])
    small = torch.searchsorted(used, ids[some].long()).to(torch.int32)
    want, bound = plain.adapted(x[some], w, None, down[dev(used)].cpu(), up[dev(used)].cpu(), small, halves=True)
    within(got[dev(some)], want, bound, "far adapters")
