"""Norm and clipping of many tensors where a norm, or norm / C, leaves float32.

Tolerances: the factor 1 / max(1, norm / C) is within 3 half steps of float32 of the exact one (a norm's rounding, a quotient, its own
rounding), a product within one more; below the normal numbers x is scaled first and the factor may be there too, each within
half a step, 2^-150, times at most 4 and 1, and the result's own rounding is another: 3 * 2^-149 together cover them."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16

# tensors, C: norms beyond float32, and quotients beyond it; sets of one launch, of a workgroup's own sums and of a launch for the sums
SETS = {"one launch": [4], "own sums": [100_000, 3], "long list": [300] * 4200, "large": [68_000_000]}


def build(sizes, value, dtype):
    gen = torch.Generator(device="cuda").manual_seed(len(sizes))
    flat = (torch.rand(sum(sizes), device="cuda", generator=gen) * 0.5 + 0.5) * value
    flat = flat.to(dtype)
    return flat, list(flat.split(sizes))


def expect(flat, C):
    norm = flat.double().square().sum().sqrt()
    return norm, torch.clamp(C / norm, max=1.0) * flat.double()


def close(got, want):
    # a 16-bit output: one step, where float32's errors move it across a border
    rel = 4 * 2.0 ** -24 if got.dtype == F32 else torch.finfo(got.dtype).eps
    return bool(((got.double() - want).abs() <= rel * want.abs() + 3 * 2.0 ** -149 + (2.0 ** -133 if got.dtype == BF16 else 0.0)).all())


@pytest.mark.parametrize("sizes", SETS.values(), ids=SETS.keys())
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("value,C", [(3e38, 1.0), (3e38, 1e38), (3e38, 3e-44), (1e30, 1e-10), (1e30, 2.0 ** -130), (1e-3, 2e-45), (2.0 ** 100, 2.0 ** -27)],
                         ids=str)
def test_norms_and_quotients_beyond_float32(sizes, dtype, value, C):
    flat, xs = build(sizes, value, dtype)
    C = float(torch.tensor(C))                         # as the call takes it
    norm, want = expect(flat, C)
    beyond = float(norm) > torch.finfo(F32).max
    out = torch.empty_like(flat)
    n = dp.tensors_norm_clip(xs, C, list(out.split(sizes)))
    assert n.isinf().item() if beyond else abs(n.item() / norm.item() - 1) <= 2.0 ** -23
    assert close(out, want)
    before = torch.full((flat.numel(),), 2.0 ** -60, device="cuda")
    sums = before.clone()
    dp.tensors_norm_clip(xs, C, list(sums.split(sizes)), accumulate=True)
    y = want + before.double()
    assert bool(((sums.double() - y).abs() <= 4 * 2.0 ** -24 * want.abs() + 2.0 ** -24 * y.abs() + 3 * 2.0 ** -149).all())
    # the two calls by themselves: the same bits, or an infinite norm and its factor 0
    other = torch.empty_like(flat)
    dp.tensors_clip(xs, dp.tensors_norm(xs), C, list(other.split(sizes)))
    assert bool((other == 0).all()) if beyond else torch.equal(other, out)
    # in place
    dp.tensors_norm_clip(xs, C)
    assert torch.equal(flat, out)


def test_an_unbounded_threshold():
    flat, xs = build([1000], 3e38, F32)
    kept = flat.clone()
    assert dp.tensors_norm_clip(xs, float("inf")).isinf().item() and torch.equal(flat, kept)


@pytest.mark.parametrize("n", [5, 50_000])
def test_infinite_elements_give_the_factor_zero(n):
    x = torch.ones(n, device="cuda")
    x[3] = float("inf")
    assert dp.tensors_norm_clip([x], 1.0).isinf().item()
    assert bool(x[3].isnan()) and int((x != 0).sum()) == 1
