"""Relative position bias against 64-bit arithmetic.

Tolerances.  Adding: one float32 sum (half a step, 2^-24) and one rounding to the type (half a step).  Gradients: the sums are taken
in 64 bits (or, over a few elements of neighbouring rows, in float32: at most 8 additions) and rounded to float32 once: 9 half
steps, 9 * 2^-24, of the sum of the magnitudes.  The norm adds up rows of n float32 squares in float32, in at most n / 64 + 6
additions one after the other: (n / 64 + 8) * 2^-24 of it, and twice the rows' own errors."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def windows(B, Tq, Tk, q_start, q_lens, k_lens, causal):
    q = torch.arange(Tq, device="cuda").view(1, -1, 1)
    k = torch.arange(Tk, device="cuda").view(1, 1, -1)
    start = 0 if q_start is None else q_start.view(-1, 1, 1)
    dist = (k - q - start).expand(B, Tq, Tk)
    live = torch.ones_like(dist, dtype=torch.bool)
    if q_lens is not None:
        live &= q < q_lens.view(-1, 1, 1)
    if k_lens is not None:
        live &= k < k_lens.view(-1, 1, 1)
    if causal:
        live &= dist <= 0
    return dist, live


def check(x, table, buckets, **how):
    """Both directions of one problem; x: scores or their gradients, with NaN wherever nothing is live."""
    B, H, Tq, Tk = x.shape
    nb, reach = table.shape[0], buckets.numel() // 2
    dist, live = windows(B, Tq, Tk, how.get("q_start"), how.get("q_lens"), how.get("k_lens"), how.get("causal", False))
    j = buckets[dist.clamp(-reach, reach) + reach].long()
    known = (j >= 0) & (j < nb)
    x.masked_fill_(~live.unsqueeze(1), float("nan"))
    # adding
    bias = torch.where(known.unsqueeze(-1), table.double()[j.clamp(0, nb - 1)], 0.0).permute(0, 3, 1, 2)
    want = x.double() + bias
    out = torch.full((B, H, Tq, Tk + 3), 77.0, device="cuda", dtype=x.dtype)[..., 1:Tk + 1]
    got = dp.posbias_add(x, table, buckets, out, **how)
    assert got is out
    l4 = live.unsqueeze(1).expand_as(x)
    assert bool((out[~l4] == 77.0).all())
    bound = 2.0 ** -24 * want.abs() + (torch.finfo(x.dtype).eps / 2 * want.abs() * (1 + 2.0 ** -20) if x.dtype != F32 else 0.0) + 2.0 ** -24 * (x.dtype == F16)
    assert bool(((out.double() - want).abs()[l4] <= bound[l4]).all())
    y = x.clone()
    assert dp.posbias_add(y, table, buckets, **how) is y                       # in place
    assert torch.equal(y[l4], out[l4])
    # the gradient
    xd = torch.where(l4, x.double(), 0.0)
    member = torch.where(known & live, j, nb)                                  # nb: no bucket
    rows, mags = torch.zeros(B, nb + 1, H, device="cuda", dtype=torch.float64), torch.zeros(B, nb + 1, H, device="cuda", dtype=torch.float64)
    index = member.view(B, -1, 1).expand(-1, -1, H)
    rows.scatter_add_(1, index, xd.flatten(2).transpose(1, 2))
    mags.scatter_add_(1, index, xd.abs().flatten(2).transpose(1, 2))
    rows, mags = rows[:, :nb], mags[:, :nb]
    sq = torch.full((B,), 3.0, device="cuda")
    sq, r = dp.posbias_sqnorm(x, buckets, nb, sq, accumulate=True, **how)
    off = 9 * 2.0 ** -24 * mags
    assert bool(((r.double() - rows).abs() <= off + 1e-40).all()), float(((r.double() - rows).abs() - off).max())
    n = nb * H
    s = rows.square().sum((1, 2))
    slack = (n / 64 + 8) * 2.0 ** -24 * (s + 3) + 2 * (rows.abs() * off).sum((1, 2)) + off.square().sum((1, 2))
    assert bool(((sq.double() - s - 3.0).abs() <= slack).all())
    sq2, r2 = dp.posbias_sqnorm(x, buckets, nb, **how)
    assert torch.equal(r2, r) and bool(((sq2.double() - s).abs() <= slack).all())
    return r


def make(B, H, Tq, Tk, dtype, seed=0, nb=32, reach=128, both=True):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(B, H, Tq, Tk, device="cuda", generator=gen).to(dtype)
    table = torch.randn(nb, H, device="cuda", generator=gen)
    return x, table, dp.relative_buckets(nb, reach, both)


SHAPES = [(1, 1, 1, 1), (2, 3, 1, 7), (2, 3, 7, 1), (3, 2, 8, 8), (1, 4, 9, 17), (2, 2, 63, 65), (1, 3, 64, 64), (2, 1, 200, 197),
          (2, 2, 512, 513), (1, 2, 530, 1100), (1, 1, 1300, 70), (40, 17, 5, 6), (1, 1, 2000, 2011), (1, 2, 1, 5000)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("causal", [False, True], ids=["both", "causal"])
def test_shapes(dtype, shape, causal):
    x, table, buckets = make(*shape, dtype, seed=sum(shape), both=not causal)
    check(x, table, buckets, causal=causal)


@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("causal", [False, True], ids=["both", "causal"])
def test_scores_that_fit_the_cache_without_the_output(dtype, causal):
    """162 MB and as much again, of 256 MB: the outputs take another way than those in place, which is checked elsewhere."""
    x, table, buckets = make(3, 16, 1300, 1301, dtype, seed=12, both=not causal)
    k_lens = torch.tensor([1301, 1000, 37], dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 77.0)
    dp.posbias_add(x, table, buckets, out, causal=causal, k_lens=k_lens)
    y = x.clone()
    dp.posbias_add(y, table, buckets, causal=causal, k_lens=k_lens)
    live = windows(3, 1300, 1301, None, None, k_lens, causal)[1].unsqueeze(1)
    assert torch.equal(out, torch.where(live, y, 77.0)) and torch.equal(torch.where(live, 0.0, y), torch.where(live, 0.0, x))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("Tq,Tk", [(1, 300), (77, 300), (300, 300), (520, 90)])
@pytest.mark.parametrize("causal", [False, True], ids=["both", "causal"])
def test_windows(dtype, Tq, Tk, causal):
    """Padded batches, chunks and steps: rows without a key, examples without a query, lengths out of range."""
    B = 6
    x, table, buckets = make(B, 3, Tq, Tk, dtype, seed=Tq, both=not causal)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    check(x.clone(), table, buckets, causal=causal, q_lens=i32(Tq, 0, 1, Tq // 2, Tq, Tq), k_lens=i32(Tk, Tk, Tk // 3, 1, 0, Tk - 1))
    check(x.clone(), table, buckets, causal=causal, q_start=i32(0, Tk - 1, -5, Tk // 2, 100000, -100000))
    check(x.clone(), table, buckets, causal=causal, q_start=i32(2 ** 31 - 1, -2 ** 31, 3, 4, 5, 6), k_lens=i32(5, 6, 7, 8, 9, 10))
    # lengths out of range are taken as the nearest that is in it
    lo = check(x.clone(), table, buckets, causal=causal, q_lens=i32(0, Tq, 0, Tq, 1, 0), k_lens=i32(Tk, 0, Tk, Tk, 1, 0))
    dS = x.clone()
    _, r = dp.posbias_sqnorm(dS, buckets, 32, causal=causal, q_lens=i32(-3, Tq + 9, -1, 2 ** 31 - 1, 1, 0), k_lens=i32(Tk + 1, -7, Tk, Tk, 1, -2 ** 31))
    assert torch.equal(r, lo)


def test_buckets_of_any_order():
    """Tables with buckets in no order, unused and unknown ones, a single one, and as many as there may be."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    for nb, reach, low, high in ((1, 0, 0, 1), (7, 50, -2, 9), (1024, 700, 0, 1024), (5, 3, 9, 10), (32, 1000, 3, 4)):
        x, table = make(2, 3, 130, 141, BF16, seed=nb)[0], torch.randn(nb, 3, device="cuda", generator=gen)
        buckets = torch.randint(low, high, (2 * reach + 1,), device="cuda", generator=gen, dtype=torch.int32)
        check(x, table, buckets)


def test_strides():
    gen = torch.Generator(device="cuda").manual_seed(6)
    _, table, buckets = make(1, 1, 1, 1, F32, nb=32)
    table = torch.randn(32, 4, device="cuda")
    base = torch.randn(3, 50, 4, 70, device="cuda", generator=gen).to(BF16)
    check(base.permute(0, 2, 1, 3)[..., 3:64], table, buckets)                         # heads inside the rows, a piece of the keys
    check(torch.randn(3, 4, 50, 64, device="cuda", generator=gen).to(F16)[:, :, 1::2, 5:], table, buckets, causal=True)
    one = torch.randn(1, 1, 1, 90, device="cuda", generator=gen)
    dS = one.expand(3, 4, 60, 90)                                                      # a broadcast gradient
    _, r = dp.posbias_sqnorm(dS, buckets, 32)
    _, r2 = dp.posbias_sqnorm(dS.contiguous(), buckets, 32)
    assert torch.equal(r, r2)
    with pytest.raises(dp.DpclipError):
        dp.posbias_add(dS, table, buckets)                                             # in place onto shared elements
    with pytest.raises(ValueError):
        dp.posbias_add(base, table, buckets)
    with pytest.raises(TypeError):
        dp.posbias_sqnorm(dS, buckets.long(), 32)


def test_nan_and_infinity_that_are_live_show():
    x, table, buckets = make(2, 2, 40, 40, BF16)
    x[1, 0, 3, 3] = float("inf")
    _, r = dp.posbias_sqnorm(x, buckets, 32)
    assert bool(r[1, 0, 0].isinf()) and int((~r.isfinite()).sum()) == 1


def test_more_than_two_to_the_32_elements():
    B, H, T = 5, 52, 4096
    x = torch.zeros((B, H, T, T), device="cuda", dtype=BF16)
    x[-1, -1, -1, -1], x[-1, -1, -1, 0], x[0, 0, 0, 5] = 2.0, 3.0, 4.0
    buckets = dp.relative_buckets(32, 128)
    _, r = dp.posbias_sqnorm(x, buckets, 32)
    want = torch.zeros_like(r)
    want[-1, 0, -1], want[-1, 15, -1], want[0, 16 + 5, 0] = 2.0, 3.0, 4.0
    assert torch.equal(r, want)
    table = torch.ones(32, H, device="cuda")
    dp.posbias_add(x, table, buckets)
    assert float(x[-1, -1, -1, -1]) == 3.0 and float(x[-1, -1, -1, 0]) == 4.0 and float(x[2, 7, 100, 9]) == 1.0


def test_gradient_of_adding():
    """The gradient against central differences of a function of the table: sum(w * (s + bias)), linear in it."""
    x, table, buckets = make(2, 3, 33, 41, F32, nb=8, reach=16)
    w = torch.randn(2, 3, 33, 41, device="cuda")
    _, rows = dp.posbias_sqnorm(w, buckets, 8)
    for j, h in ((0, 0), (3, 1), (7, 2)):
        up, down = table.clone(), table.clone()
        up[j, h] += 1.0
        down[j, h] -= 1.0
        d = (w.double() * (dp.posbias_add(x, up, buckets, torch.empty_like(x)).double() - dp.posbias_add(x, down, buckets, torch.empty_like(x)).double())).sum((1, 2, 3)) / 2
        # each sum of adding is off by at most 2^-24 of its size (below 16)
        slack = 2.0 ** -20 * w.double().abs()[:, h].sum((1, 2))
        assert bool(((d - rows[:, j, h].double()).abs() <= slack).all())


def test_graph_replays_and_streams():
    x, table, buckets = make(3, 4, 100, 120, BF16)
    out, sq, rows = torch.zeros_like(x), torch.empty(3, device="cuda"), torch.empty(3, 32, 4, device="cuda")
    ws = torch.empty(dp.posbias_workspace_bytes(x), dtype=torch.uint8, device="cuda")
    def step(**how):
        dp.posbias_add(x, table, buckets, out, **how)
        dp.posbias_sqnorm(x, buckets, 32, sq, rows, workspace=ws, **how)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for k in range(4):
        x.copy_(torch.randn(x.shape, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, sq, rows)]
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, sq, rows)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sq2, rows2 = dp.posbias_sqnorm(x, buckets, 32, stream=side)
    side.synchronize()
    assert torch.equal(sq2, sq) and torch.equal(rows2, rows)
