"""Norms of queries and keys with the rotation: calls at the edges of what the entry points take."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("empty", [0, 1], ids=["queries", "keys"])
@pytest.mark.parametrize("B,T", [(2, 40), (700, 4)], ids=["chunks", "few"])
@pytest.mark.parametrize("D", [64, 72, 33])
def test_a_descriptor_without_heads_needs_no_addresses(empty, B, T, D):
    """Its rows are zeros, the other one's results those of a call by itself."""
    x, dy = (torch.randn(B, T, 3, D, device="cuda") for _ in range(2))
    none = torch.empty(B, T, 0, D, device="cuda")
    gain = 1 + 0.1 * torch.randn(D, device="cuda")
    freqs = dp.rotary_freqs(32)
    sq1, rows1, dx1 = dp.headnorm_sqnorm([(x, gain)], [dy], freqs=freqs)
    y1, = dp.headnorm([(x, gain)], freqs=freqs)
    order = (lambda a, b: [b, a]) if empty == 0 else (lambda a, b: [a, b])
    out, dx, rows = torch.empty_like(x), torch.empty_like(x), [torch.full((B, D), 7.0, device="cuda") for _ in range(2)]
    fwd = dp.head_descs(order((x, gain), (none, gain)), order(out, none))
    bwd = dp.head_descs(order((x, gain), (none, gain)), order(dx, none), order(dy, none), rows)
    for d in (fwd, bwd):
        d.arr[empty].x = d.arr[empty].gain = d.arr[empty].out = d.arr[empty].dy = None
    dp.headnorm(None, freqs=freqs, descs=fwd)
    sq, _, _ = dp.headnorm_sqnorm(None, None, freqs=freqs, descs=bwd)
    assert torch.equal(out, y1) and bool((rows[empty] == 0).all())
    assert torch.equal(dx, dx1[0])
    # the chunks may be others, so that sums of the same terms are taken in another order: 88 half steps of float32 of the sum of
    # magnitudes on each side, a term's at most |x r| and twice the largest number of dy's row
    xh = x.double() * (x.double().square().mean(-1, keepdim=True) + 1e-6).rsqrt()
    off = 2 * 88 * 2.0 ** -24 * (2 * dy.double().abs().amax(-1, keepdim=True) * xh.abs()).sum((1, 2))
    g = rows1[0].double()
    assert bool(((rows[1 - empty].double() - g).abs() <= off).all())
    assert bool(((sq.double() - sq1.double()).abs() <= (2 * g.abs() * off + off.square()).sum(1) + 2.0 ** -22 * sq1).all())


# one token of many heads (a chain of 2500 steps for each lane, were it not cut), and a batch that leaves one chunk to an example (600)
@pytest.mark.parametrize("B,T,H", [(1, 1, 20000), (2400, 1200, 4)], ids=["heads", "tokens"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_long_sums_of_a_gain(B, T, H, dtype):
    """Equal rows: every addition of a column's chain is rounded the same way between two powers of two, so that errors add up instead of
    cancelling.  A term u x r is off by 24 half steps of float32 (here: r, two products); with at most 64 additions one after the
    other in float32, 6 between lanes, and a rounding of the chunk's sum and of the row: 24 + 64 + 6 + 2 = 96 of the sum."""
    D = 512
    x, gain = (1.0 + torch.arange(D, device="cuda") / D).to(dtype), torch.ones(D, device="cuda")
    dy = (1.0 + torch.arange(D, device="cuda") / 397).to(dtype)
    shape = (B, T, H, D)
    dx = torch.empty(shape, device="cuda", dtype=dtype)
    sq, (rows,), _ = dp.headnorm_sqnorm([(x.expand(shape), gain)], [dy.expand(shape)], outs=[dx], eps=1e-6)
    want = dy.double() * x.double() / (x.double().square().mean() + 1e-6) ** 0.5 * (T * H)
    off = (rows.double() - want).abs() / want * 2.0 ** 24
    assert float(off.max()) <= 96, float(off.max())
    assert torch.equal(rows, rows[:1].expand_as(rows))
    s = want.square().sum()
    assert float((sq.double() - s).abs().max()) <= 2 * 97 * 2.0 ** -24 * float(s)


def only(x, column):
    """Whether of the last dimension's columns just this one is not finite."""
    bad = (~x.isfinite()).flatten(0, -2).any(0)
    return bad.nonzero().flatten().tolist() == [column]


@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("D,rot,column", [(64, 32, 40), (64, 32, 57), (64, 0, 9), (80, 32, 79), (72, 24, 30), (33, 10, 11), (110, 54, 54), (128, 8, 9), (50, 20, 49)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_what_does_not_turn_keeps_to_its_column(pairs, D, rot, column, dtype):
    """An infinite gradient, or gain, of a number behind the ones that turn is no other column's."""
    gen = torch.Generator(device="cuda").manual_seed(D)
    x, dy = (torch.randn(2, 7, 3, D, device="cuda", generator=gen).to(dtype) for _ in range(2))
    gain = 1 + 0.1 * torch.randn(D, device="cuda", generator=gen)
    freqs = dp.rotary_freqs(rot) if rot else None
    _, (want,), _ = dp.headnorm_sqnorm([(x, gain)], [dy], freqs=freqs, pairs=pairs)
    before, = dp.headnorm([(x, gain)], freqs=freqs, pairs=pairs)
    dy[1, 3, 2, column] = float("inf")
    sq, (rows,), _ = dp.headnorm_sqnorm([(x, gain)], [dy], freqs=freqs, pairs=pairs)
    assert torch.equal(rows[0], want[0]) and sq[0].isfinite() and sq[1].isinf()
    assert only(rows[1:], column) and rows[1, column].isinf()
    others = [j for j in range(D) if j != column]
    assert torch.equal(rows[:, others], want[:, others])
    gain[column] = float("inf")
    y, = dp.headnorm([(x, gain)], freqs=freqs, pairs=pairs)
    assert only(y, column) and bool(y[..., column].isinf().all()) and torch.equal(y[..., others], before[..., others])


@pytest.mark.parametrize("D,rot", [(64, 64), (80, 80), (80, 48), (72, 72), (100, 48), (36, 0), (33, 32), (176, 96)])
@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("B", [2, 500], ids=["chunks", "few"])
@pytest.mark.parametrize("last", [False, True])
def test_an_infinite_gain_meets_its_row_only(D, rot, pairs, B, last):
    """dx = r (u w - x r mean(u w x r)): the mean is infinite, and so is every column but the gain's own, where infinities may cancel."""
    gen = torch.Generator(device="cuda").manual_seed(D)
    x, dy = (torch.randn(B, 3, 3, D, device="cuda", generator=gen) for _ in range(2))
    gain = torch.ones(D, device="cuda")
    column = D - 1 if last else 0
    gain[column] = float("inf")
    _, _, (dx,) = dp.headnorm_sqnorm([(x, gain)], [dy], freqs=dp.rotary_freqs(rot) if rot else None, pairs=pairs)
    others = torch.cat((dx[..., :column], dx[..., column + 1:]), -1)
    assert bool(others.isinf().all()), int(others.isnan().sum())


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,rot", [(64, 64), (72, 72), (100, 48), (110, 54), (33, 0), (16, 16)])
@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "pairs"])
def test_sums_of_many_heads(dtype, D, rot, pairs):
    """More rows for each lane than a chain of float32 has, of two descriptors with different numbers of them."""
    from test_gpu_headnorm import check, full, make
    lengths = torch.tensor([2, 1], dtype=torch.int32, device="cuda")
    heads, dys = make(2, 2, (30000, 20), D, dtype, seed=D, lengths=lengths)
    check(heads, dys, full(heads), full(heads), dp.rotary_freqs(rot) if rot else None, lengths=lengths, pairs=pairs)
