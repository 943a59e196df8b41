"""Norms of queries and keys with the rotation, forward and backward, against 64-bit arithmetic.

Tolerances, in half steps of float32 (2^-24), from the chains of float32 operations:
  r: a sum of squares in chains of at most 16 additions and 6 between lanes, one rounding per square: 23 of the sum, half of that for
     its root; the mean, eps, root and quotient: at most 4 more: 16.
  y: r, two products (18), sine and cosine to 4 (the series' argument and terms), a product and a sum (2): 24 of |a| + |b|, the
     magnitudes of the pair before the turn; one rounding to the type behind it.
  u: 4 + 2 of |dy_a| + |dy_b| =: U.   x r: 17.   mean(u w x r): 6 + 1 + 17 + 1 of each term and 23 for the sum: 48 of the mean of
     magnitudes M.   dx = r (u w - x r mean): r (25 U |w| + 84 |x r| M).
  gain_rows: 24 of each term U |x r|, and at most 64 additions one after the other before the chunks are added in 64 bits (a wave's
     steps over its tokens and heads: 18 in the longest of these cases): 88 of the sum of magnitudes.
  The angle itself is a product of the position with a frequency in turns, taken twice here: three roundings of 2^-53 of it come on
     top of the 24, 25, 84 and 88, which counts for positions beyond some ten millions."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS = 1e-6
H24 = 2.0 ** -24


def turn(x, cos, sin, rot, pairs):
    y = x.clone()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    ya, yb = a * cos - b * sin, a * sin + b * cos
    if pairs:
        y[..., 0:rot:2], y[..., 1:rot:2] = ya, yb
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = ya, yb
    return y


def pair_size(x, rot, pairs):
    """|a| + |b| of each number's pair; the number's own magnitude where nothing turns."""
    y = x.abs()
    one = torch.ones((), device=x.device, dtype=x.dtype)
    s = turn(y, one, -one, rot, pairs) if rot else y          # (a + b, b - a)
    t = turn(y, one, one, rot, pairs) if rot else y           # (a - b, a + b)
    return torch.maximum(s, t)


def rounding(y):
    return torch.finfo(y.dtype).eps / 2 * (1 + 2.0 ** -10) if y.dtype != F32 else 0.0


def check(heads, dys, outs, back_outs, freqs, positions=None, lengths=None, pairs=False):
    """heads, dys: with NaN in the tokens that lengths leave out; outs, back_outs: filled with 77."""
    B, T, _, D = heads[0][0].shape
    rot = 0 if freqs is None else 2 * freqs.numel()
    pos = torch.arange(T, device="cuda").expand(B, T) if positions is None else positions.expand(B, T)
    live = torch.ones((B, T), dtype=torch.bool, device="cuda")
    if lengths is not None:
        live = torch.arange(T, device="cuda").view(1, -1) < lengths.view(-1, 1)
    l4 = live.view(B, T, 1, 1)
    angle = pos.double().view(B, T, 1, 1) * (freqs if rot else torch.zeros(0, device="cuda", dtype=torch.float64))
    cos, sin = angle.cos(), angle.sin()
    far = 3 * 2.0 ** -53 / H24 * angle.abs().amax(-1, keepdim=True) if rot else torch.zeros((B, T, 1, 1), device="cuda", dtype=torch.float64)
    how = dict(freqs=freqs, positions=positions, lengths=lengths, pairs=pairs, eps=EPS)
    got = dp.headnorm(heads, outs, **how)
    sq, rows, dxs = dp.headnorm_sqnorm(heads, dys, torch.full((B,), 2.0, device="cuda"), back_outs, accumulate=True, **how)
    want_sq, slack = torch.full((B,), 2.0, device="cuda", dtype=torch.float64), torch.zeros(B, device="cuda", dtype=torch.float64)
    for i, ((x, w), dy, o, dx) in enumerate(zip(heads, dys, got, dxs)):
        x64, dy64, w64 = torch.where(l4, x.double(), 0.0), torch.where(l4, dy.double(), 0.0), w.double()
        r = 1.0 / (x64.square().mean(-1, keepdim=True) + EPS).sqrt()
        xh = x64 * r
        # forward
        y = turn(xh * w64, cos, sin, rot, pairs)
        bound = (24 + far) * H24 * pair_size(xh * w64, rot, pairs) + rounding(o) * y.abs() + (2.0 ** -24 if o.dtype == F16 else 1e-38)
        err = torch.where(l4, (o.double() - y).abs(), 0.0)
        assert bool((err <= bound).all()), ("y", i, float((err / bound).max()))
        assert bool(torch.where(l4, True, o == 77.0).all())
        # backward
        u = turn(dy64, cos, -sin, rot, pairs)
        U = pair_size(dy64, rot, pairs)
        uw = u * w64
        m, M = (uw * xh).mean(-1, keepdim=True), (U * w64.abs() * xh.abs()).mean(-1, keepdim=True)
        want = r * (uw - xh * m)
        bound = r * ((25 + far) * U * w64.abs() + (84 + far) * xh.abs() * M) * H24 + rounding(dx) * want.abs() + (2.0 ** -24 if o.dtype == F16 else 1e-38)
        err = torch.where(l4, (dx.double() - want).abs(), 0.0)
        assert bool((err <= bound).all()), ("dx", i, float((err / bound).max()))
        assert bool(torch.where(l4, True, dx == 77.0).all())
        g = (u * xh).sum((1, 2))
        off = H24 * ((88 + far) * U * xh.abs()).sum((1, 2)) + 1e-38
        err = (rows[i].double() - g).abs()
        assert bool((err <= off).all()), ("rows", i, float((err / off).max()))
        want_sq += g.square().sum(1)
        slack += (2 * g.abs() * off + off.square()).sum(1)
    assert bool(((sq.double() - want_sq).abs() <= slack + 2 * H24 * want_sq).all())
    # without accumulating, and the same bits again
    sq2, rows2, dxs2 = dp.headnorm_sqnorm(heads, dys, **how)
    assert bool(((sq2.double() + 2.0 - want_sq).abs() <= slack + 4 * H24 * want_sq).all())
    for a, b, c, d in zip(rows, rows2, dxs, dxs2):
        assert torch.equal(a, b) and torch.equal(torch.where(l4, c, 0), torch.where(l4, d, 0))
    return got, rows, dxs


def make(B, T, Hs, D, dtype, seed=0, lengths=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    def t(*shape):
        return torch.randn(shape, device="cuda", generator=gen)
    def strip(x):
        if lengths is not None:
            x.masked_fill_((torch.arange(T, device="cuda").view(1, -1) >= lengths.view(-1, 1)).view(B, T, 1, 1), float("nan"))
        return x
    heads = [(strip(t(B, T, H, D).to(dtype)), 1 + 0.2 * t(D)) for H in Hs]
    dys = [strip(t(B, T, H, D).to(dtype)) for H in Hs]
    return heads, dys


def full(heads):
    return [torch.full_like(x, 77.0) for x, _ in heads]


CASES = [  # B, T, heads, D, rot
    (1, 1, (1,), 1, 0), (1, 1, (1, 1), 2, 2), (2, 3, (4, 2), 7, 4), (1, 9, (3, 1), 8, 8), (3, 5, (5,), 16, 16), (2, 17, (6, 2), 20, 10),
    (1, 33, (2, 2), 33, 32), (2, 40, (12, 12), 64, 64), (1, 21, (8, 8), 80, 80), (2, 19, (3, 1), 96, 48), (5, 1, (32, 8), 128, 128),
    (1, 300, (4, 4), 128, 64), (2, 13, (7, 1), 130, 66), (1, 37, (16, 2), 256, 256), (1, 5, (3,), 200, 200), (1, 7, (2, 1), 511, 510),
    (1, 4, (2, 3), 512, 512), (1, 3, (1, 2), 509, 6), (2, 9, (4, 1), 110, 110), (1, 33, (2, 5), 118, 38), (300, 2, (1, 1), 32, 32), (1, 2000, (1,), 64, 32), (3000, 1, (2, 1), 16, 16),
    (2, 31, (0, 3), 48, 16), (2, 11, (3, 0), 48, 32), (1, 4, (16, 16), 112, 112), (2, 70, (5, 3), 176, 96),
    (2, 31, (5, 2), 72, 72), (1, 9, (4, 1), 4, 0), (3, 8, (2, 2), 12, 8), (1, 6, (2,), 508, 504), (2, 21, (3, 1), 100, 48),
    (400, 3, (4, 1), 72, 72), (500, 5, (3, 2), 64, 32), (450, 2, (1, 2), 110, 110), (700, 4, (0, 2), 33, 32), (390, 9, (5,), 128, 128),
]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(v) for v in c).replace(" ", ""))
@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "pairs"])
def test_sizes(dtype, case, pairs):
    B, T, Hs, D, rot = case
    heads, dys = make(B, T, Hs, D, dtype, seed=D)
    check(heads, dys, full(heads), full(heads), dp.rotary_freqs(rot) if rot else None, pairs=pairs)


@pytest.mark.parametrize("D", [64, 72, 30])
def test_many_padded_examples(D):
    B, T = 600, 6
    lengths = torch.randint(-2, T + 3, (B,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(D))
    heads, dys = make(B, T, (4, 1), D, BF16, seed=4, lengths=lengths)
    check(heads, dys, full(heads), full(heads), dp.rotary_freqs(D // 4 * 2), lengths=lengths)


LONG = [(3, 9000, (8, 2), 64, 64), (7, 3001, (5, 1), 80, 40), (200, 70, (2, 2), 256, 256), (2, 20000, (9, 2), 128, 128), (9, 2600, (6, 2), 110, 110),
        (1, 25000, (16, 8), 128, 64)]       # 153 MB and as much of outputs: more than the last-level cache together


@pytest.mark.parametrize("padded", [False, True], ids=["full", "padded"])
@pytest.mark.parametrize("case", LONG, ids=lambda c: "x".join(str(v) for v in c).replace(" ", ""))
def test_several_tokens_of_each_wave(case, padded):
    B, T, Hs, D, rot = case
    lengths = torch.tensor([T - i * T // B for i in range(B - 1)] + [0], dtype=torch.int32, device="cuda") if padded else None
    heads, dys = make(B, T, Hs, D, BF16, seed=D + 1, lengths=lengths)
    check(heads, dys, full(heads), full(heads), dp.rotary_freqs(rot), lengths=lengths)


@pytest.mark.parametrize("D,rot", [(64, 64), (64, 32), (24, 10)])
@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "pairs"])
def test_positions(D, rot, pairs):
    heads, dys = make(3, 50, (4, 2), D, F32, seed=1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    for low, high in ((0, 50), (-100, 100), (1_000_000, 1_001_000), (-2 ** 31, 2 ** 31 - 1)):
        check(heads, dys, full(heads), full(heads), dp.rotary_freqs(rot), pairs=pairs,
              positions=torch.randint(low, high, (3, 50), device="cuda", generator=gen, dtype=torch.int32))
    check(heads, dys, full(heads), full(heads), dp.rotary_freqs(rot, 500000.0), pairs=pairs, positions=torch.arange(7, 57, device="cuda", dtype=torch.int32))
    # angles beyond a turn per position, negative and zero
    freqs = torch.linspace(-20.0, 20.0, rot // 2, device="cuda", dtype=torch.float64)
    check(heads, dys, full(heads), full(heads), freqs, pairs=pairs)


@pytest.mark.parametrize("D", [64, 30])
def test_padded_batches(D):
    lengths = torch.tensor([40, 0, 1, 39, 17, 40], device="cuda", dtype=torch.int32)
    heads, dys = make(6, 40, (4, 2), D, BF16, seed=3, lengths=lengths)
    check(heads, dys, full(heads), full(heads), dp.rotary_freqs(D), lengths=lengths)
    # out of range: the nearest that is in it
    heads, dys = make(6, 40, (4, 2), D, BF16, seed=3, lengths=lengths)
    how = dict(freqs=dp.rotary_freqs(D))
    a = dp.headnorm_sqnorm(heads, dys, lengths=lengths, **how)
    b = dp.headnorm_sqnorm(heads, dys, lengths=torch.tensor([2 ** 31 - 1, -2 ** 31, 1, 39, 17, 41], device="cuda", dtype=torch.int32), **how)
    assert torch.equal(a[0], b[0]) and all(torch.equal(x, y) for x, y in zip(a[1] + a[2], b[1] + b[2]))


@pytest.mark.parametrize("D,rot", [(64, 64), (128, 32), (36, 36)])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_strides(D, rot, dtype):
    """Packed projections, heads outside of tokens, tensors that begin at any element, broadcast inputs, and in place."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    B, T, freqs = 2, 23, dp.rotary_freqs(rot)
    def packed(shift):
        return torch.randn(B * T * 11 * D + 8, device="cuda", generator=gen).to(dtype)[shift:shift + B * T * 11 * D].view(B, T, 11, D)
    gains = [1 + 0.1 * torch.randn(D, device="cuda", generator=gen) for _ in range(2)]
    def split(p):
        return [p[:, :, :6], p[:, :, 6:9]]
    x, dy, o, d = packed(0), packed(1), packed(3).fill_(77.0), packed(5).fill_(77.0)
    heads = list(zip(split(x), gains))
    outs, rows, dxs = check(heads, split(dy), split(o), split(d), freqs)
    assert bool((o[:, :, 9:] == 77.0).all()) and bool((d[:, :, 9:] == 77.0).all())
    # in place: of x forward, of dy backward
    y = x.clone()
    dp.headnorm(list(zip(split(y), gains)), split(y), freqs=freqs)
    assert torch.equal(y[:, :, :9], o[:, :, :9]) and torch.equal(y[:, :, 9:], x[:, :, 9:])
    y = dy.clone()
    dp.headnorm_sqnorm(heads, split(y), outs=split(y), freqs=freqs)
    assert torch.equal(y[:, :, :9], d[:, :, :9]) and torch.equal(y[:, :, 9:], dy[:, :, 9:])
    # heads outside of tokens
    t = x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    again = dp.headnorm(list(zip(split(t), gains)), freqs=freqs)
    assert all(torch.equal(a, b) for a, b in zip(again, outs))
    # one token's row for all
    row = x[:1, :1, :1].expand(B, T, 4, D)
    check([(row, gains[0])], [dy[:, :, :4]], [o[:, :, :4].fill_(77.0)], [d[:, :, :4].fill_(77.0)], freqs)
    with pytest.raises(dp.DpclipError):
        dp.headnorm([(row, gains[0])], [row], freqs=freqs)
    with pytest.raises(ValueError):
        dp.headnorm([(x.transpose(2, 3), gains[0])], freqs=freqs)
    with pytest.raises(TypeError):
        dp.headnorm([(x, gains[0])], freqs=freqs.float())
    with pytest.raises(TypeError):
        dp.headnorm([(x, gains[0])], freqs=freqs, positions=torch.arange(T, device="cuda"))


def test_rows_of_zeros_and_large_values():
    heads, dys = make(1, 6, (2, 1), 64, F32, seed=5)
    heads[0][0][0, 2] = 0.0
    heads[0][0][0, 3] *= 1e15
    heads[1][0][0, 4] *= 1e-15
    check(heads, dys, full(heads), full(heads), dp.rotary_freqs(64))


@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "pairs"])
def test_gradients_against_differences(pairs):
    """sum(dy * y) along single inputs and gains.  Outputs that do not depend on the changed number keep their bits, so the
    difference is the row's (or the example's) alone; y is off by 24 half steps of its pair, twice, over a distance of 2 h.  The
    function of x is sum(dy r x): its third derivative is below 15 |dy| r / |x|^2, the error of central differences h^2 / 6 of it."""
    B, T, H, D = 2, 5, 2, 32
    heads, dys = make(B, T, (H,), D, F32, seed=6)
    (x, w), dy, freqs = heads[0], dys[0], dp.rotary_freqs(32)
    how = dict(freqs=freqs, pairs=pairs)
    _, rows, dx = dp.headnorm_sqnorm(heads, dys, **how)
    y0 = dp.headnorm(heads, **how)[0].double()
    def f(x, w):
        return (dp.headnorm([(x, w)], **how)[0].double() * dy.double())
    h = 2.0 ** -6
    for b, t, k, j in ((0, 0, 0, 0), (1, 4, 1, 17), (0, 2, 1, 31)):
        up, down = x.clone(), x.clone()
        up[b, t, k, j] += h
        down[b, t, k, j] -= h
        step = float(up[b, t, k, j].double() - down[b, t, k, j].double())
        diff = float((f(up, w) - f(down, w)).sum()) / step
        row = pair_size(y0, 32, pairs)[b, t, k]
        n2 = float(x[b, t, k].double().square().sum())
        slack = 2 * 24 * H24 * 2 * float((dy[b, t, k].double().abs() * row).sum()) / step
        slack += h * h / 6 * 15 * float(dy[b, t, k].double().norm() * w.double().abs().max()) * (D / n2) ** 0.5 / n2
        assert abs(diff - float(dx[0][b, t, k, j])) <= slack + 1e-6, (diff, float(dx[0][b, t, k, j]), slack)
    for j in (0, 13, 31):
        up, down = w.clone(), w.clone()
        up[j] += 0.5
        down[j] -= 0.5
        diff = (f(x, up) - f(x, down)).sum((1, 2, 3)) / (up[j].double() - down[j].double())
        mags = (pair_size(dy.double(), 32, pairs) * 2 * pair_size(y0, 32, pairs)).sum((1, 2, 3))
        assert bool(((diff - rows[0][:, j].double()).abs() <= 4 * 88 * H24 * mags).all())


def test_more_than_two_to_the_32_bytes():
    B, T, H, D = 2, 34000, 260, 128
    x = torch.zeros((B, T, H, D), device="cuda", dtype=BF16)
    x[-1, -1, -1, :] = 3.0
    w = torch.ones(D, device="cuda")
    out = torch.full_like(x, 5.0)
    dp.headnorm([(x, w)], [out])
    assert bool((out[-1, -1, -1] == 1.0).all()) and bool((out[-1, -1, :-1] == 0).all()) and bool((out[0] == 0).all())
    x[0, -1, 3, 7] = 2.0
    _, rows, _ = dp.headnorm_sqnorm([(x, w)], [x], outs=[out])
    # u = dy = x: the sum of x^2 r
    assert torch.allclose(rows[0][1], torch.full((D,), 3.0, device="cuda"), rtol=1e-6)
    one = torch.zeros(D, device="cuda")
    one[7] = 4.0 / (4.0 / 128 + 1e-6) ** 0.5
    assert torch.allclose(rows[0][0], one, rtol=1e-5)


def test_graph_replays_and_streams():
    heads, dys = make(3, 60, (4, 2), 64, BF16, seed=7)
    outs, dxs = full(heads), full(heads)
    rows, sq = [torch.empty(3, 64, device="cuda") for _ in range(2)], torch.empty(3, device="cuda")
    fwd, bwd = dp.head_descs(heads, outs), dp.head_descs(heads, dxs, dys, rows)
    ws = torch.empty(dp.headnorm_workspace_bytes(bwd), dtype=torch.uint8, device="cuda")
    freqs = dp.rotary_freqs(64)
    def step():
        dp.headnorm(None, freqs=freqs, descs=fwd)
        dp.headnorm_sqnorm(None, None, sq, freqs=freqs, descs=bwd, workspace=ws)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for k in range(4):
        for x, _ in heads:
            x.copy_(torch.randn(x.shape, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*outs, *dxs, *rows, sq)]
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, (*outs, *dxs, *rows, sq)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sq2, rows2, _ = dp.headnorm_sqnorm(heads, dys, freqs=freqs, stream=side)
    side.synchronize()
    assert torch.equal(sq2, sq) and all(torch.equal(a, b) for a, b in zip(rows, rows2))
    with pytest.raises(ValueError):
        dp.headnorm_sqnorm(None, None, sq, freqs=freqs, descs=fwd)


def test_shapes_of_positions():
    heads, _ = make(3, 5, (2,), 8, F32)
    for shape in ((3, 5), (5,)):
        dp.headnorm(heads, freqs=dp.rotary_freqs(8), positions=torch.zeros(shape, dtype=torch.int32, device="cuda"))
    for shape in ((5, 3), (15,), (3,), (1, 5), (3, 5, 1)):
        with pytest.raises(ValueError):
            dp.headnorm(heads, freqs=dp.rotary_freqs(8), positions=torch.zeros(shape, dtype=torch.int32, device="cuda"))
