"""Norm and clipping of many tensors against 64-bit arithmetic.

Tolerances: the norm is taken in 64 bits and rounded to float32 once, then the factor is a float32 quotient of it: the norm is
within half a step, 2^-24, of the exact one (and of the 64-bit sum's own error, far below); the factor within 3 half steps (the
norm's rounding, norm / C and the reciprocal); an output within one more of its own type.  A factor that differs by 3 float32 half
steps may move a 16-bit output to the neighbour of the nearest value where the product lies between two: a whole step."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def make(sizes, types, std=1.0, seed=0, shift=0):
    """Tensors of these sizes inside flat buffers, each `shift` elements behind a 16-byte boundary."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for n, t in zip(sizes, types):
        flat = torch.zeros(n + 16, device="cuda", dtype=t)
        x = flat[shift:shift + n]
        x.copy_(torch.randn(n, device="cuda", generator=gen) * std)
        out.append(x)
    return out


def exact(xs, C, old=0.0):
    squares = [x.double().square().sum() for x in xs]
    norm = (sum(squares) + old ** 2).sqrt()
    return norm, torch.stack(squares).sqrt(), 1.0 / torch.clamp(norm / C, min=1.0)


def check(xs, outs, norm, C, before=None, norms=None):
    want, each, c = exact(xs, C)
    assert abs(norm.item() - want.item()) <= 2.0 ** -23 * want.item()
    if norms is not None:
        assert bool(((norms.double() - each).abs() <= 2.0 ** -23 * each).all())
    for i, (x, o) in enumerate(zip(xs, outs)):
        y = x.double() * c
        if before is not None:
            y = y + before[i].double()
            # the product's and the sum's roundings
            bound = 4 * 2.0 ** -24 * (x.double() * c).abs() + 2.0 ** -24 * y.abs()
        else:
            bound = (4 * 2.0 ** -24 if o.dtype == F32 else torch.finfo(o.dtype).eps) * y.abs()
        if o.dtype == F16:
            bound = bound + 2.0 ** -24            # a step of the subnormal numbers
        assert bool(((o.double() - y).abs() <= bound + 1e-45).all()), (i, x.shape, x.dtype, o.dtype)


SIZES = [
    [1], [7], [8], [2049], [4096], [4097], [100000],
    [1, 2, 3, 5, 8, 13, 1000, 4095, 4096, 4097, 12289],
    [3] * 111 + [5000], [17] * 113, [1 + i % 40 for i in range(700)] + [300000],
    [9_000_011, 5, 1_000_000, 3_000_001], [40_000_003, 5, 1, 30_000_001, 9_000_000],
]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("types", [(F32,), (BF16,), (F16,), (F32, BF16, F16)], ids=["f32", "bf16", "f16", "mixed"])
def test_norm_and_clip(sizes, types):
    ts = [types[i % len(types)] for i in range(len(sizes))]
    for shift, C in ((0, 1.0), (3, 0.25), (1, 1e9)):
        xs = make(sizes, ts, seed=len(sizes) + shift, shift=shift)
        outs = make(sizes, ts, seed=99, shift=(shift * 2) % 5)
        norms = torch.full((len(xs),), float("nan"), device="cuda")
        norm = dp.tensors_norm_clip(xs, C, outs, tensor_norms=norms)
        check(xs, outs, norm, C, norms=norms)
        # the two calls by themselves: the same bits
        outs2 = make(sizes, [F32] * len(sizes), seed=98)
        n2, norms2 = torch.empty(1, device="cuda"), torch.empty(len(xs), device="cuda")
        dp.tensors_norm(xs, n2, tensor_norms=norms2)
        assert torch.equal(n2, norm) and torch.equal(norms2, norms)
        dp.tensors_clip(xs, n2, C, outs2)
        check(xs, outs2, n2, C)
        for o, p in zip(outs, outs2):
            assert torch.equal(o, p.to(o.dtype))
        # added to float32 sums
        before = [o.clone() for o in outs2]
        dp.tensors_norm_clip(xs, C, outs2, accumulate=True)
        check(xs, outs2, norm, C, before=before)
        # in place
        kept = [x.clone() for x in xs]
        dp.tensors_norm_clip(xs, C)
        for x, o, k in zip(xs, outs, kept):
            assert torch.equal(x, o if C < 1e9 else k)


def test_neighbours_are_left_alone():
    flat = torch.ones(10000, device="cuda", dtype=BF16)
    out = torch.full((10000,), 7.0, device="cuda", dtype=BF16)
    dp.tensors_norm_clip([flat[5:4103], flat[4103:9001]], 1.0, [out[11:4109], out[5000:9898]])
    assert bool((out[:11] == 7).all()) and bool((out[4109:5000] == 7).all()) and bool((out[9898:] == 7).all())
    assert bool((out[11:4109] < 1).all()) and bool((out[5000:9898] < 1).all())


def test_values_whose_squares_leave_float32():
    x = torch.full((1000,), 3e30, device="cuda")
    y = torch.full((7,), 1e-30, device="cuda")
    n = dp.tensors_norm([y])
    assert abs(n.item() / (7 ** 0.5 * 1e-30) - 1) < 1e-6
    n = dp.tensors_norm_clip([x], 2.0)
    assert abs(n.item() / (1000 ** 0.5 * 3e30) - 1) < 1e-6
    assert torch.allclose(x, torch.full_like(x, 2.0 / 1000 ** 0.5), rtol=1e-6)


def test_nan_infinity_and_zeros():
    z = torch.zeros(100, device="cuda")
    assert dp.tensors_norm_clip([z], 1.0).item() == 0 and bool((z == 0).all())
    for bad in (float("nan"), float("inf")):
        x = torch.ones(5000, device="cuda", dtype=F16)
        x[4321] = bad
        y = torch.ones(10, device="cuda")
        n = dp.tensors_norm_clip([x, y], 1.0)
        if bad != bad:
            assert bool(n.isnan()) and bool(x.isnan().all()) and bool(y.isnan().all())
        else:                                     # a factor of 0: what was infinite is NaN, the rest 0
            assert bool(n.isinf()) and bool((y == 0).all()) and bool(x[4321].isnan()) and int(x.isnan().sum()) == 1


def test_norm_accumulates_and_empty_tensors():
    a, b = torch.full((3,), 2.0, device="cuda"), torch.full((0,), 1.0, device="cuda")
    norms = torch.full((3,), 5.0, device="cuda")
    n = dp.tensors_norm([b, a, b], tensor_norms=norms)
    assert torch.allclose(n, torch.tensor([12.0 ** 0.5], device="cuda")) and norms.tolist()[0::2] == [0.0, 0.0]
    dp.tensors_norm([torch.full((4,), 1.0, device="cuda")], n, accumulate=True)
    assert torch.allclose(n, torch.tensor([4.0], device="cuda"))
    assert dp.tensors_norm_clip([b], 1.0).item() == 0


def test_a_tensor_of_more_than_four_gigabytes():
    n = (1 << 32) + 4099
    x = torch.zeros(n, device="cuda", dtype=BF16)
    x[-3:] = 3.0
    x[5] = 4.0
    out = torch.full((n,), 9.0, device="cuda", dtype=BF16)
    norm = dp.tensors_norm_clip([x], 1.0, [out])
    assert abs(norm.item() - 43.0 ** 0.5) < 1e-5
    assert int((out != 0).sum()) == 4 and abs(out[-1].item() - 3 / 43.0 ** 0.5) < 2e-3 and abs(out[5].item() - 4 / 43.0 ** 0.5) < 3e-3


def test_graph_replays_and_streams():
    xs = make([5000, 33, 70000], [F32, BF16, F16], seed=4)
    outs = [torch.empty_like(x) for x in xs]
    descs = dp.tensor_descs(xs, outs)
    ws = torch.empty(dp.tensors_workspace_bytes(descs), dtype=torch.uint8, device="cuda")
    norm = torch.empty(1, device="cuda")
    dp.tensors_norm_clip(None, 1.0, norm=norm, descs=descs, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dp.tensors_norm_clip(None, 1.0, norm=norm, descs=descs, workspace=ws)
    for k in range(4):
        for x in xs:
            x.mul_(1.5 if k % 2 else 0.3)
        for o in outs:
            o.fill_(-1.0)
        g.replay()
        torch.cuda.synchronize()
        check(xs, outs, norm, 1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = dp.tensors_norm_clip(xs, 1.0, outs, stream=side)
    side.synchronize()
    assert torch.equal(got, norm)


def test_long_lists_in_graphs_and_calls_at_once():
    """More tensors than a launch's arguments hold, captured; two lists on two streams at the same time."""
    lists = [make([100 + 7 * i for i in range(150)], [F32, BF16, F16] * 50, seed=s) for s in (1, 2)]
    outs = [[torch.empty_like(x) for x in xs] for xs in lists]
    descs = [dp.tensor_descs(xs, os) for xs, os in zip(lists, outs)]
    norms = [torch.empty(1, device="cuda") for _ in lists]
    ws = [torch.empty(dp.tensors_workspace_bytes(d), dtype=torch.uint8, device="cuda") for d in descs]
    streams = [torch.cuda.Stream() for _ in lists]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, st in enumerate(streams):
            dp.tensors_norm_clip(None, 1.0, norm=norms[i], descs=descs[i], workspace=ws[i], stream=st)
    torch.cuda.synchronize()
    for i in range(2):
        check(lists[i], outs[i], norms[i], 1.0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dp.tensors_norm_clip(None, 1.0, norm=norms[0], descs=descs[0], workspace=ws[0])
    for k in range(3):
        for x in lists[0]:
            x.mul_(0.5)
        g.replay()
        torch.cuda.synchronize()
        check(lists[0], outs[0], norms[0], 1.0)


def test_results_repeat():
    xs = make([1_000_003, 12345, 8], [F32, BF16, F16], seed=6)
    first = [t.clone() for t in (dp.tensors_norm_clip(xs, 1.0, [torch.empty_like(x) for x in xs]),)]
    for _ in range(3):
        assert torch.equal(dp.tensors_norm(xs), first[0])
