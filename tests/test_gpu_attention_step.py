"""A private step of one attention block, its parameters' calls together: the linear projection, the gains of the norms of queries and
keys and the table of the relative position bias add up in one norm per example; the clipped sums are clipped once more as a whole.
Against per-example gradients by 64-bit differentiation.

The block's own products and its softmax are taken in 64 bits on both sides, so what is compared are the calls.  A score is a sum of 16
products of normalised numbers, each off by at most 2 x 24 half steps of float32 (the two sides' norms and turns), and one float32 sum
with the bias: at most 50 * 2^-24 * sum |q k| / 4 < 50 * 6e-8 * 30 = 9e-5, which the softmax passes on as a relative error of its
weights and gradients.  The calls' own errors (at most 88 half steps, 5e-6) are behind that: 2e-4 of a result's 2-norm."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

pytestmark = pytest.mark.gpu

TOL = 2e-4
B, T, d, Hq, Hk, D, NB, REACH, C = 6, 29, 24, 4, 2, 16, 16, 12, 3.0


def off(x, y):
    return float((x.double() - y).norm() / y.norm())


def attend(q, k, v, bias, live):
    """Scores (without bias), weights and outputs; key heads are shared by Hq / Hk query heads."""
    k, v = (t.repeat_interleave(Hq // Hk, 2) for t in (k, v))
    s = torch.matmul(q.transpose(1, 2), k.permute(0, 2, 3, 1).contiguous()) / D ** 0.5
    p = torch.where(live, s + bias, -torch.inf).softmax(-1)
    return s, p, torch.matmul(p, v.transpose(1, 2).contiguous())


@pytest.mark.parametrize("ragged", [False, True], ids=["full", "ragged"])
def test_step(ragged):
    gen = torch.Generator(device="cuda").manual_seed(11)
    def t(*shape, std=1.0):
        return torch.randn(shape, device="cuda", generator=gen) * std
    x, W = t(B, T, d), t(d, (Hq + 2 * Hk) * D, std=0.3)
    gq, gk, table = 1 + t(D, std=0.2), 1 + t(D, std=0.2), t(NB, Hq, std=0.5)
    cot = t(B, Hq, T, D) * torch.logspace(-2, 0.5, B, device="cuda").view(B, 1, 1, 1)
    lens = torch.tensor([T, 17, 1, T, 8, 20] if ragged else [T] * B, device="cuda", dtype=torch.int32)
    here = (torch.arange(T, device="cuda").view(1, -1) < lens.view(-1, 1))
    cot = cot * here.view(B, 1, T, 1)
    x = x * here.unsqueeze(-1)
    freqs, buckets = dp.rotary_freqs(D), dp.relative_buckets(NB, REACH, both=False)
    pos = torch.arange(T, device="cuda")
    # (queries behind a sequence's end keep a live key, their outputs have no gradient)
    live = (pos.view(1, -1) <= pos.view(-1, 1)).view(1, 1, T, T)
    dist = (pos.view(1, -1) - pos.view(-1, 1)).clamp(-REACH, REACH) + REACH

    # per-example gradients in 64 bits: every example with copies of the parameters
    copies = [p.double().unsqueeze(0).repeat(B, *([1] * p.dim())).requires_grad_() for p in (W, gq, gk, table)]
    Wc, gqc, gkc, tc = copies
    qkv = torch.matmul(x.double(), Wc).view(B, T, Hq + 2 * Hk, D)
    angle = pos.double().view(-1, 1) * freqs
    cos, sin = angle.cos().view(1, T, 1, -1), angle.sin().view(1, T, 1, -1)
    def norm_turn(z, g):
        y = z * (z.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * g.view(B, 1, 1, D)
        a, b = y[..., :D // 2], y[..., D // 2:]
        return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    bias = tc[:, buckets.long()[dist]].permute(0, 3, 1, 2)
    _, _, out = attend(norm_turn(qkv[:, :, :Hq], gqc), norm_turn(qkv[:, :, Hq:Hq + Hk], gkc), qkv[:, :, Hq + Hk:], bias, live)
    per_example = torch.autograd.grad((out * cot.double()).sum(), copies)
    sq_ref = sum(g.flatten(1).square().sum(1) for g in per_example)
    clip_ref = 1.0 / torch.clamp(sq_ref.sqrt() / C, min=1.0)
    sums_ref = [torch.tensordot(clip_ref, g, dims=1) for g in per_example]
    assert 0 < int((clip_ref < 1).sum()) < B                              # some examples are clipped, some are not

    # the calls
    qkv = torch.matmul(x.double(), W.double()).float().view(B, T, Hq + 2 * Hk, D)
    heads = [(qkv[:, :, :Hq], gq), (qkv[:, :, Hq:Hq + Hk], gk)]
    window = dict(q_lens=lens, k_lens=lens, causal=True) if ragged else dict(causal=True)
    turned = [torch.zeros(B, T, h, D, device="cuda") for h in (Hq, Hk)]
    dp.headnorm(heads, turned, freqs=freqs, lengths=lens if ragged else None)
    q, k = (z.double() for z in turned)
    v = qkv[:, :, Hq + Hk:].double()
    s, _, _ = attend(q, k, v, torch.zeros((), device="cuda"), live)
    s = dp.posbias_add(s.float(), table, buckets, **window).double()
    p = torch.where(live, s, -torch.inf).softmax(-1)
    vr, kr = v.repeat_interleave(Hq // Hk, 2).transpose(1, 2), k.repeat_interleave(Hq // Hk, 2).transpose(1, 2).contiguous()
    dp_ = torch.matmul(cot.double(), vr.transpose(2, 3).contiguous())
    ds = p * (dp_ - (dp_ * p).sum(-1, keepdim=True))
    dv = torch.matmul(p.transpose(2, 3).contiguous(), cot.double()).view(B, Hk, Hq // Hk, T, D).sum(2).transpose(1, 2)
    dq = torch.matmul(ds, kr).transpose(1, 2) / D ** 0.5
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q.transpose(1, 2).contiguous()).view(B, Hk, Hq // Hk, T, D).sum(2).transpose(1, 2) / D ** 0.5
    G = torch.zeros_like(qkv)                                             # the projection's gradient, packed like its output
    G[:, :, Hq + Hk:] = dv.float()
    sq = torch.full((B,), float("nan"), device="cuda")
    rows = [torch.empty(B, D, device="cuda") for _ in range(2)]
    dp.headnorm_sqnorm(heads, [dq.float().contiguous(), dk.float().contiguous()], sq, [G[:, :, :Hq], G[:, :, Hq:Hq + Hk]], rows,
                       freqs=freqs, lengths=lens if ragged else None)
    _, table_rows = dp.posbias_sqnorm(ds.float(), buckets, NB, sq, accumulate=True, **window)
    layers = [(x, G.view(B, T, -1))]
    dp.layers_sqnorm(layers, sq, accumulate=True)
    clip = dp.clip_factors(sq, C)
    sums = dp.layers_clipped_grad(layers, clip) + [dp.clipped_bias_grad(r, clip) for r in rows] + \
        [dp.clipped_bias_grad(table_rows.view(B, -1), clip).view(NB, Hq)]
    assert off(sq, sq_ref) <= 2 * TOL and bool(((sq.double() - sq_ref).abs() <= 2 * TOL * sq_ref).all())
    for got, want in zip(sums, sums_ref):
        assert off(got, want) <= TOL, (got.shape, off(got, want))

    # the sum of the clipped gradients, clipped as a whole and added to an earlier one (a user's, a micro-batch's)
    total = [torch.ones_like(g) for g in sums]
    whole = sum(g.square().sum() for g in sums_ref).sqrt()
    norm = dp.tensors_norm_clip(sums, float(whole) / 3, total, accumulate=True)
    assert off(norm, whole.view(1)) <= TOL
    for got, want in zip(total, sums_ref):
        assert off(got - 1, want / 3) <= 2 * TOL + 2.0 ** -23 * want.numel() ** 0.5 / float((want / 3).norm())
