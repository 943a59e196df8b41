"""The forward calls inside a program that uses autograd: gradients end nowhere in silence, and what a graph has saved is not
overwritten without its notice."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

pytestmark = pytest.mark.gpu


def problem():
    x, gain = torch.randn(2, 5, 3, 32, device="cuda"), torch.ones(32, device="cuda")
    s, table = torch.randn(2, 3, 7, 9, device="cuda"), torch.randn(8, 3, device="cuda")
    return x, gain, s, table, dp.relative_buckets(8, 6)


def test_leaves_are_refused_unless_gradients_are_off():
    x, gain, s, table, buckets = problem()
    y, = dp.headnorm([(x, gain)])
    z = dp.posbias_add(s, table, buckets, torch.empty_like(s))
    gain.requires_grad_()
    table.requires_grad_()
    descs = dp.head_descs([(x, gain)], [torch.empty_like(x)])
    for call in (lambda: dp.headnorm([(x, gain)]), lambda: dp.headnorm(None, descs=descs), lambda: dp.posbias_add(s, table, buckets, torch.empty_like(s))):
        with pytest.raises(RuntimeError, match="records no gradients"):
            call()
        with torch.no_grad():
            call()
    with torch.no_grad():
        assert torch.equal(dp.headnorm(None, descs=descs)[0], y)
        assert torch.equal(dp.posbias_add(s, table, buckets, torch.empty_like(s)), z)
    with torch.inference_mode():
        assert torch.equal(dp.headnorm([(x, gain)])[0], y) and torch.equal(dp.posbias_add(s.clone(), table, buckets), z)


def test_the_backward_calls_take_leaves():
    x, gain, s, table, buckets = problem()
    sq, rows, _ = dp.headnorm_sqnorm([(x, gain)], [x])
    sq2, rows2, _ = dp.headnorm_sqnorm([(x.requires_grad_(), gain.requires_grad_())], [x])
    assert torch.equal(sq, sq2) and torch.equal(rows[0], rows2[0])
    assert torch.equal(dp.posbias_sqnorm(s, buckets, 8)[0], dp.posbias_sqnorm(s.requires_grad_(), buckets, 8)[0])


@pytest.mark.parametrize("which", ["posbias", "heads"])
def test_a_saved_tensor_that_is_written_is_noticed(which):
    x, gain, s, table, buckets = problem()
    t = s if which == "posbias" else x
    w = torch.ones_like(t).requires_grad_()
    loss = (w * t).sum()                                     # saves t
    if which == "posbias":
        dp.posbias_add(s, table, buckets)
    else:
        dp.headnorm([(x, gain)], [x])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_inside_a_function_of_ones_own():
    """The calls as a differentiable step: forward without a graph, backward by the backward calls."""
    x, gain, *_ = problem()
    freqs = dp.rotary_freqs(32)

    class Heads(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, gain):
            ctx.save_for_backward(x, gain)
            return dp.headnorm([(x, gain)], freqs=freqs)[0]

        @staticmethod
        def backward(ctx, dy):
            x, gain = ctx.saved_tensors
            _, (rows,), (dx,) = dp.headnorm_sqnorm([(x, gain)], [dy.contiguous()], freqs=freqs)
            return dx, rows.sum(0)

    leaves = [t.double().requires_grad_() for t in (x, gain)]
    y = leaves[0] * (leaves[0].square().mean(-1, keepdim=True) + 1e-6).rsqrt() * leaves[1]
    angle = torch.arange(5, device="cuda").double().view(1, 5, 1, 1) * freqs
    a, b = y[..., :16], y[..., 16:]
    y = torch.cat((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()), -1)
    cot = torch.randn_like(x)
    want = torch.autograd.grad((y * cot.double()).sum(), leaves)
    ours = [t.clone().requires_grad_() for t in (x, gain)]
    got = torch.autograd.grad((Heads.apply(*ours) * cot).sum(), ours)
    # rows of 32 numbers, 30 terms of a gain: 130 half steps of sums of magnitudes (r, products, turn: 84; sums: 40), below 40 here
    for g, w in zip(got, want):
        assert float((g.double() - w).abs().max()) <= 130 * 2.0 ** -24 * 40
