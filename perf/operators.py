"""The operators around a private training step of an attention model, as measurable cases.

Beside its linear layers an attention block has two kinds of parameters whose per-example gradients enter the same norm:
the gains of the norms of queries and keys, and the table of a relative position bias.  And a finished gradient of many
tensors (a model's, a micro-batch's, a user's) is clipped as a whole.

  "clip"        the norm over many tensors and all of them scaled by min(1, C / norm)
  "bias"        scores + table[bucket of the distance between key and query, head]
  "bias_grad"   the gradient of that table for each example, and its squared norm
  "heads"       queries and keys normalised head by head, times a gain, rotated by their positions
  "heads_grad"  the gradients of that: the inputs', each example's gains', and the squared norm of the latter

A case is a dict of plain values.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def listed():
    return [
        # the smallest model gradient: one dense layer of 64 x 32 with its bias, where launches and the call itself count
        {"name": "clip_dense_f32", "kind": "clip", "tensors": "f32:64x32 f32:32", "packed": False, "each": False, "C": 1.0, "std": 0.1},
        # a twelve-block transformer's float32 gradient in one flat buffer: linears, biases and norms, with the norm of each
        # tensor for the log
        {"name": "clip_transformer_f32", "kind": "clip", "packed": False, "each": True, "C": 1.0, "std": 1e-3,
         "tensors": "f32:768x2304*12 f32:2304*12 f32:768x768*12 f32:768*72 f32:768x3072*12 f32:3072*12 f32:3072x768*12"},
        # a large model's 16-bit gradients packed back to back at odd sizes, its small parameters in float32: the largest
        {"name": "clip_large_bf16", "kind": "clip", "packed": True, "each": False, "C": 1.0, "std": 1e-3,
         "tensors": "bf16:2048x6144*20 bf16:2048x2048*20 bf16:2048x8191*20 bf16:8191x2048*20 f32:2049*160 f32:50257 f16:2047x1023*4"},
        # attention scores of a padded batch of sentences, both directions
        {"name": "bias_bf16", "kind": "bias", "dtype": "bf16", "B": 32, "H": 12, "Tq": 512, "Tk": 512, "buckets": 32,
         "reach": 128, "causal": False, "way": "ragged", "padded": False},
        # one new token for each of 64 sequences against their caches
        {"name": "bias_step_f16", "kind": "bias", "dtype": "f16", "B": 64, "H": 16, "Tq": 1, "Tk": 2048, "buckets": 32,
         "reach": 128, "causal": True, "way": "step", "padded": False},
        # a small batch of odd lengths in float32
        {"name": "bias_grad_odd_f32", "kind": "bias_grad", "dtype": "f32", "B": 3, "H": 5, "Tq": 197, "Tk": 197, "buckets": 32,
         "reach": 128, "causal": False, "way": "full", "padded": False},
        # the transformer's batch: 64 examples of 512 positions and 12 heads
        {"name": "bias_grad_bf16", "kind": "bias_grad", "dtype": "bf16", "B": 64, "H": 12, "Tq": 512, "Tk": 512, "buckets": 32,
         "reach": 128, "causal": False, "way": "full", "padded": False},
        # long causal sequences, a table of finer buckets
        {"name": "bias_grad_long_bf16", "kind": "bias_grad", "dtype": "bf16", "B": 4, "H": 16, "Tq": 4096, "Tk": 4096,
         "buckets": 64, "reach": 1024, "causal": True, "way": "ragged", "padded": False},
        # one new token for each of 32 sequences, at far positions
        {"name": "heads_step_bf16", "kind": "heads", "dtype": "bf16", "B": 32, "T": 1, "Hq": 32, "Hk": 8, "D": 128, "rot": 128,
         "pairs": False, "start": 100000, "ragged": False},
        # long sequences with shared key heads, queries and keys inside the packed projection
        {"name": "heads_long_bf16", "kind": "heads", "dtype": "bf16", "B": 4, "T": 8192, "Hq": 32, "Hk": 8, "D": 128, "rot": 128,
         "pairs": False, "start": 0, "ragged": False},
        # the transformer's batch, backward
        {"name": "heads_grad_bf16", "kind": "heads_grad", "dtype": "bf16", "B": 64, "T": 512, "Hq": 12, "Hk": 12, "D": 64,
         "rot": 64, "pairs": False, "start": 0, "ragged": False},
        # a padded float32 batch of odd lengths, a part of each head rotated, neighbours in pairs
        {"name": "heads_grad_odd_f32", "kind": "heads_grad", "dtype": "f32", "B": 5, "T": 199, "Hq": 6, "Hk": 2, "D": 80,
         "rot": 40, "pairs": True, "start": 1000, "ragged": True},
    ]


def _log_int(rng, lo, hi):
    """Whole number between lo and hi, evenly spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("clip", "bias", "bias_grad", "heads", "heads_grad"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    if kind == "clip":                       # from a handful of tensors to hundreds, from one element to tens of millions
        most = _log_int(rng, 1000, 30_000_000)
        tensors = " ".join(f"{rng.choice((dtype, dtype, 'f32'))}:{_log_int(rng, 1, most)}" for _ in range(_log_int(rng, 1, 400)))
        case = {"kind": kind, "tensors": tensors, "packed": rng.random() < 0.5, "each": rng.random() < 0.5,
                "C": rng.choice((1.0, 1.0, 1e9)), "std": rng.choice((1e-3, 1.0))}
    elif kind in ("bias", "bias_grad"):      # one query to thousands, any length, whole and padded batches, chunks and steps
        way = rng.choice(("full", "ragged", "chunk") + (("step",) if kind == "bias" else ()))
        Tk = _log_int(rng, 16, 4096)
        Tq = {"step": 1, "chunk": max(1, Tk // rng.randint(2, 5))}.get(way, rng.choice((Tk, Tk, Tk, _log_int(rng, 16, 2048))))
        if rng.random() < 0.4:
            Tk = max(1, Tk // 64 * 64) if Tk >= 64 else Tk
            Tq = Tk if way in ("full", "ragged") else Tq
        reach = rng.choice((32, 128, 128, 1000))
        case = {"kind": kind, "dtype": dtype, "B": _log_int(rng, 1, 64), "H": rng.randint(1, 32), "Tq": Tq, "Tk": Tk,
                "buckets": rng.choice((16, 32, 32, 64)), "reach": reach, "causal": rng.random() < 0.5, "way": way,
                "padded": rng.random() < 0.3}
    else:                                    # one token to thousands, shared key heads, whole and partial rotations
        D = rng.choice((64, 128, 128, 256, 96, 80, 2 * rng.randint(4, 100)))
        Hk = rng.choice((1, 2, 4, 8))
        case = {"kind": kind, "dtype": dtype, "B": _log_int(rng, 1, 64), "T": 1 if kind == "heads" and rng.random() < 0.3 else _log_int(rng, 1, 8192),
                "Hq": Hk * rng.randint(1, 6), "Hk": Hk, "D": D, "rot": rng.choice((D, D, D // 4 * 2)), "pairs": rng.random() < 0.3,
                "start": rng.choice((0, 0, 1000, 1000000)), "ragged": rng.random() < 0.4}
    cap = max(work(c)["bytes"] for c in listed() if c["kind"] == kind)
    while work(case)["bytes"] > cap:
        if kind == "clip":
            items = case["tensors"].split()
            case["tensors"] = " ".join(items[: max(1, len(items) * 2 // 3)])
        elif case["B"] > 1:
            case["B"] = max(1, case["B"] * 2 // 3)
        else:
            case["H" if "H" in case else "T"] = max(1, case["H" if "H" in case else "T"] // 2)
    return case


def _shapes(case):
    """[(dtype, elements), ...] of a "clip" case."""
    out = []
    for item in case["tensors"].split():
        body, _, times = item.partition("*")
        dt, sizes = body.split(":")
        out += [(dt, math.prod(int(v) for v in sizes.split("x")))] * (int(times) if times else 1)
    return out


def _lengths(T, B, ragged):
    """The examples' lengths: all T, or spread evenly from T down to a quarter of it; the last of three or more is empty."""
    if not ragged:
        return [T] * B
    lens = [T - (T * 3 // 4) * i // max(1, B - 1) for i in range(B)]
    if B >= 3:
        lens[-1] = 0
    return lens


def _windows(case):
    """Per example of a "bias" case: position of its first query, number of queries, number of keys."""
    B, Tq, Tk = case["B"], case["Tq"], case["Tk"]
    if case["way"] == "step":                # the query is the last of the keys; caches of different lengths
        lens = [max(1, n) for n in _lengths(Tk, B, True)]
        return [n - 1 for n in lens], [1] * B, lens
    if case["way"] == "chunk":               # the last queries of a longer context
        return [Tk - Tq] * B, [Tq] * B, [Tk] * B
    ragged = case["way"] == "ragged"
    return [0] * B, _lengths(Tq, B, ragged), _lengths(Tk, B, ragged)


def work(case):
    """Bytes (each input read once, each output written once) and operations of one pass."""
    if case["kind"] == "clip":
        sizes = _shapes(case)
        size = {"f32": 4, "bf16": 2, "f16": 2}
        return {"bytes": sum(2 * n * size[dt] for dt, n in sizes) + 4, "flops": 3 * sum(n for _, n in sizes)}
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("bias", "bias_grad"):
        live = 0
        for start, nq, nk in zip(*_windows(case)):
            if not case["causal"]:
                live += nq * nk
            else:                            # query q sees min(nk, q + start + 1) keys
                short = min(nq, max(0, nk - start))
                live += short * (short + 1) // 2 + short * start + (nq - short) * nk
        live *= case["H"]
        if case["kind"] == "bias":
            return {"bytes": 2 * es * live + 4 * case["buckets"] * case["H"], "flops": live}
        return {"bytes": es * live + 4 * case["B"] * (case["buckets"] * case["H"] + 1), "flops": live}
    rows = sum(_lengths(case["T"], case["B"], case["ragged"])) * (case["Hq"] + case["Hk"])
    n = rows * case["D"]
    if case["kind"] == "heads":
        return {"bytes": 2 * es * n + 8 * case["D"] + 4 * case["B"] * case["T"], "flops": 7 * n}
    return {"bytes": 3 * es * n + 8 * case["D"] + 4 * case["B"] * (case["T"] + 2 * case["D"] + 1), "flops": 15 * n}


def _buckets(n, reach, both):
    """Bucket of each distance from -reach to reach (key minus query): half of the buckets for single distances, the others
    ever wider up to `reach`; with `both` the upper half of them is for the keys behind the query."""
    half = n // 2 if both else n
    single = half // 2
    wide = half - single

    def bucket(d):                           # compared in whole numbers: d^wide * single^j against reach^j * single^wide
        if d < single:
            return d
        j = 0
        while j + 1 < wide and d ** wide * single ** (j + 1) >= reach ** (j + 1) * single ** wide:
            j += 1
        return single + j

    back = [bucket(d) for d in range(reach + 1)]
    ahead = [half + b if both else 0 for b in back]
    return [back[-d] if d <= 0 else ahead[d] for d in range(-reach, reach + 1)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def values(shape, dtype, std=1.0):
        x = torch.empty(shape, device="cuda", dtype=dtype)
        return x.normal_(0.0, std, generator=gen)

    def zeros(shape, dtype=torch.float32):
        return torch.zeros(shape, device="cuda", dtype=dtype)

    def ints(v):
        return torch.tensor(v, device="cuda", dtype=torch.int32)

    st = {"case": case}
    if case["kind"] == "clip":
        sizes = _shapes(case)
        # the tensors of a type lie one after the other in a flat buffer: packed, or each on a 16-byte boundary
        at, places = {}, []
        for dt, n in sizes:
            places.append(at.get(dt, 0))
            at[dt] = places[-1] + (n if case["packed"] else (n + 7) // 8 * 8)
        flat = {dt: zeros(total, TYPES[dt]) for dt, total in at.items()}
        outs = {dt: zeros(total, TYPES[dt]) for dt, total in at.items()}
        xs = [flat[dt][p:p + n] for (dt, n), p in zip(sizes, places)]
        if case["packed"]:
            for x in flat.values():
                x.normal_(0.0, case["std"], generator=gen)
        else:
            for x in xs:
                x.normal_(0.0, case["std"], generator=gen)
        st.update(flat=flat, outs=outs, xs=xs, norm=zeros(1), norms=zeros(len(sizes)) if case["each"] else None)
        if own:
            from paper_2009_03106_amd import dpclip as dp
            st["descs"] = dp.tensor_descs(xs, [outs[dt][p:p + n] for (dt, n), p in zip(sizes, places)])
            st["workspace"] = torch.empty(dp.tensors_workspace_bytes(st["descs"]), device="cuda", dtype=torch.uint8)
        return st
    dtype = TYPES[case["dtype"]]
    if case["kind"] in ("bias", "bias_grad"):
        B, H, Tq, Tk = (case[k] for k in ("B", "H", "Tq", "Tk"))
        start, nq, nk = _windows(case)
        width = Tk if not case["padded"] else (Tk + 15) // 16 * 16       # rows on 16-element boundaries
        grad = case["kind"] == "bias_grad"
        # scores of unit size; gradients of scores go with the attention weights, about one over the length
        st.update(x=values((B, H, Tq, width), dtype, 1.0 / Tk if grad else 1.0)[..., :Tk],
                  buckets=ints(_buckets(case["buckets"], case["reach"], not case["causal"])),
                  q_start=ints(start) if any(start) else None,
                  q_lens=ints(nq) if min(nq) < Tq else None, k_lens=ints(nk) if min(nk) < Tk else None)
        if grad:
            st.update(sqnorm=zeros(B), rows=zeros((B, case["buckets"], H)))
            if own:
                from paper_2009_03106_amd import dpclip as dp
                st["workspace"] = torch.empty(dp.posbias_workspace_bytes(st["x"]), device="cuda", dtype=torch.uint8)
        else:
            st.update(table=values((case["buckets"], H), torch.float32), out=zeros((B, H, Tq, width), dtype)[..., :Tk])
        return st
    B, T, Hq, Hk, D = (case[k] for k in ("B", "T", "Hq", "Hk", "D"))
    packed = values((B, T, Hq + 2 * Hk, D), dtype)                       # queries, keys and values of one projection
    # float64 angles per position, base 10000
    freqs = torch.tensor([10000.0 ** (-2.0 * j / case["rot"]) for j in range(case["rot"] // 2)], device="cuda", dtype=torch.float64)
    lens = _lengths(T, B, case["ragged"])
    st.update(heads=[(packed[:, :, :Hq], 1.0 + values((D,), torch.float32, 0.1)),
                     (packed[:, :, Hq:Hq + Hk], 1.0 + values((D,), torch.float32, 0.1))],
              freqs=freqs, lengths=ints(lens) if case["ragged"] else None,
              positions=ints([[case["start"] + 17 * b + t for t in range(T)] for b in range(B)]))
    if case["kind"] == "heads":
        st["outs"] = [zeros((B, T, Hq, D), dtype), zeros((B, T, Hk, D), dtype)]
        if own:
            from paper_2009_03106_amd import dpclip as dp
            st["descs"] = dp.head_descs(st["heads"], st["outs"])
        return st
    dpacked = zeros((B, T, Hq + 2 * Hk, D), dtype)                       # its gradient; the values' part is another's
    st.update(dpacked=dpacked, outs=[dpacked[:, :, :Hq], dpacked[:, :, Hq:Hq + Hk]], sqnorm=zeros(B),
              gain_rows=[zeros((B, D)), zeros((B, D))],
              grads=[values((B, T, Hq, D), dtype, 1e-2), values((B, T, Hk, D), dtype, 1e-2)])
    if own:
        from paper_2009_03106_amd import dpclip as dp
        st["descs"] = dp.head_descs(st["heads"], st["outs"], st["grads"], st["gain_rows"])
        st["workspace"] = torch.empty(dp.headnorm_workspace_bytes(st["descs"]), device="cuda", dtype=torch.uint8)
    return st


def run(state):
    case = state["case"]
    return _run_own(state, case) if own else _run_plain(state, case)


def _run_own(st, case):
    from paper_2009_03106_amd import dpclip as dp
    kind = case["kind"]
    if kind == "clip":
        dp.tensors_norm_clip(None, case["C"], norm=st["norm"], tensor_norms=st["norms"], descs=st["descs"], workspace=st["workspace"])
        return {"norm": st["norm"], "norms": st["norms"], "outs": st["outs"]} if case["each"] else {"norm": st["norm"], "outs": st["outs"]}
    if kind in ("bias", "bias_grad"):
        window = {"q_start": st["q_start"], "q_lens": st["q_lens"], "k_lens": st["k_lens"], "causal": case["causal"]}
        if kind == "bias":
            return dp.posbias_add(st["x"], st["table"], st["buckets"], st["out"], **window)
        dp.posbias_sqnorm(st["x"], st["buckets"], case["buckets"], st["sqnorm"], st["rows"], workspace=st["workspace"], **window)
        return {"sqnorm": st["sqnorm"], "rows": st["rows"]}
    how = {"freqs": st["freqs"], "positions": st["positions"], "lengths": st["lengths"], "pairs": case["pairs"], "eps": EPS}
    if kind == "heads":
        dp.headnorm(None, descs=st["descs"], **how)
        return st["outs"]
    dp.headnorm_sqnorm(None, None, st["sqnorm"], descs=st["descs"], workspace=st["workspace"], **how)
    return {"sqnorm": st["sqnorm"], "gain_rows": st["gain_rows"], "dx": st["dpacked"]}


def _live(st, case):
    """Which (query, key) of a "bias" case take part, [B or 1, 1, Tq, Tk], and the distances key minus query, [B or 1, Tq, Tk]."""
    q = torch.arange(case["Tq"], device="cuda").view(1, -1, 1)
    k = torch.arange(case["Tk"], device="cuda").view(1, 1, -1)
    dist = k - q
    if st["q_start"] is not None:
        dist = dist - st["q_start"].view(-1, 1, 1)
    live = torch.ones_like(dist, dtype=torch.bool)
    if case["causal"]:
        live = live & (dist <= 0)
    if st["q_lens"] is not None:
        live = live & (q < st["q_lens"].view(-1, 1, 1))
    if st["k_lens"] is not None:
        live = live & (k < st["k_lens"].view(-1, 1, 1))
    return live.unsqueeze(1), dist


def _turn(st, case, sign):
    """cos and sin (times sign) of the rotation of each token, [B, T, 1, rot / 2], float32 from 64-bit angles."""
    angle = st["positions"].double().unsqueeze(-1) * st["freqs"]
    return angle.cos().float().unsqueeze(2), (sign * angle.sin()).float().unsqueeze(2)


def _rotate(x, cos, sin, rot, pairs):
    y = x.clone()
    if pairs:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, a * sin + b * cos
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, a * sin + b * cos
    return y


def _run_plain(st, case):
    kind = case["kind"]
    if kind == "clip":
        # long sums: in 64 bits
        norms = torch.stack([x.double().square().sum() for x in st["xs"]]).sqrt()
        norm = norms.square().sum().sqrt()
        factor = (case["C"] / norm).clamp(max=1.0).float()
        outs = {dt: (x.float() * factor).to(x.dtype) for dt, x in st["flat"].items()}
        return {"norm": norm.float().view(1), "norms": norms.float(), "outs": outs} if case["each"] else {"norm": norm.float().view(1), "outs": outs}
    if kind in ("bias", "bias_grad"):
        live, dist = _live(st, case)
        x, reach = st["x"], case["reach"]
        if kind == "bias":
            bias = st["table"][st["buckets"][dist.clamp(-reach, reach) + reach].long()].permute(0, 3, 1, 2)
            return torch.where(live, x.float() + bias, 0.0).to(x.dtype)
        B, H, Tq, Tk = x.shape
        # the diagonals as columns: rows from the last to the first, each one place further to the right; then the sums
        # of the diagonals (in 64 bits) by their distances' buckets
        flipped = torch.where(live, x.float(), 0.0).flip(2)
        skewed = torch.nn.functional.pad(flipped, (0, Tq)).view(B, H, -1)[..., :Tq * (Tk + Tq - 1)].view(B, H, Tq, Tk + Tq - 1)
        sums = skewed.sum(2, dtype=torch.float64)
        d = torch.arange(1 - Tq, Tk, device="cuda").view(1, -1)
        if st["q_start"] is not None:
            d = d - st["q_start"].view(-1, 1)
        member = st["buckets"][d.clamp(-reach, reach) + reach].unsqueeze(-1) == torch.arange(case["buckets"], device="cuda")
        rows = torch.matmul(sums, member.double()).transpose(1, 2).contiguous()
        return {"sqnorm": rows.square().sum((1, 2)).float(), "rows": rows.float()}
    rot, pairs, lens = case["rot"], case["pairs"], st["lengths"]
    kept = None if lens is None else (torch.arange(case["T"], device="cuda").view(1, -1) < lens.view(-1, 1)).view(case["B"], case["T"], 1, 1)
    if kind == "heads":
        cos, sin = _turn(st, case, 1.0)
        outs = []
        for x, gain in st["heads"]:
            x32 = x.float()
            y = _rotate(x32 * (x32.square().mean(-1, keepdim=True) + EPS).rsqrt() * gain, cos, sin, rot, pairs)
            outs.append((y if kept is None else torch.where(kept, y, 0.0)).to(x.dtype))
        return outs
    cos, sin = _turn(st, case, -1.0)
    dx, rows = torch.zeros_like(st["dpacked"]), []
    at = 0
    for (x, gain), dy in zip(st["heads"], st["grads"]):
        x32 = x.float()
        r = (x32.square().mean(-1, keepdim=True) + EPS).rsqrt()
        xhat, n = x32 * r, _rotate(dy.float(), cos, sin, rot, pairs)
        if kept is not None:
            n = torch.where(kept, n, 0.0)
        rows.append((n * xhat).sum((1, 2)))
        u = n * gain
        dx[:, :, at:at + x.shape[2]] = (r * (u - xhat * (u * xhat).mean(-1, keepdim=True))).to(dx.dtype)
        at += x.shape[2]
    return {"sqnorm": rows[0].square().sum(1) + rows[1].square().sum(1), "gain_rows": rows, "dx": dx}


def exact(case, seed):
    """The operators by their definitions in 64 bits."""
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "clip":
        squares = [torch.dot(x.double(), x.double()) for x in st["xs"]]
        norm = torch.sqrt(sum(squares))
        c = 1.0 / torch.maximum(norm / case["C"], torch.ones_like(norm))
        out = {"norm": norm.view(1), "outs": {dt: x.double() * c for dt, x in st["flat"].items()}}
        return {"norm": out["norm"], "norms": torch.sqrt(torch.stack(squares)), "outs": out["outs"]} if case["each"] else out
    if kind in ("bias", "bias_grad"):
        B, H, Tq, Tk = (case[k] for k in ("B", "H", "Tq", "Tk"))
        buckets, reach = st["buckets"].tolist(), case["reach"]
        start, nq, nk = _windows(case)
        x = st["x"]
        if kind == "bias":                   # query by query: the row of the table for each key
            out = torch.zeros((B, H, Tq, Tk), device="cuda", dtype=torch.float64)
            by_distance = st["table"].double()[torch.tensor(buckets, device="cuda")]
            for b in range(B):
                if nq[b] * nk[b] == 0:
                    continue
                place = torch.arange(nq[b], device="cuda")[:, None] + start[b]
                delta = torch.arange(nk[b], device="cuda")[None, :] - place
                part = x[b, :, :nq[b], :nk[b]].double() + by_distance[delta.clamp(-reach, reach) + reach].movedim(-1, 0)
                if case["causal"]:
                    part = part.tril(start[b])
                out[b, :, :nq[b], :nk[b]] = part
            return out
        rows = torch.zeros((B, case["buckets"], H), device="cuda", dtype=torch.float64)
        if B * (Tq + Tk) > 200_000:
            return None                      # a diagonal at a time would take too long
        for b in range(B):                   # diagonal by diagonal
            part = x[b, :, :nq[b], :nk[b]]
            for d in range(1 - nq[b], nk[b]) if nq[b] * nk[b] else ():
                delta = d - start[b]
                if case["causal"] and delta > 0:
                    break
                rows[b, buckets[max(-reach, min(reach, delta)) + reach]] += part.diagonal(d, 1, 2).sum(-1, dtype=torch.float64)
        return {"sqnorm": rows.pow(2).sum((1, 2)), "rows": rows}
    # the rotation as a product of complex numbers, the gradients by differentiation
    rot, B, T = case["rot"], case["B"], case["T"]
    angle = st["positions"].to(torch.float64)[:, :, None, None] * st["freqs"]
    turn = torch.polar(torch.ones_like(angle), angle)

    def forward(x, gain):                    # gain: [B, 1, 1, D], a copy for each example
        y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["D"] + EPS) * gain
        z = y[..., :rot].unflatten(-1, (rot // 2, 2) if case["pairs"] else (2, rot // 2))
        z = torch.complex(*(z.unbind(-1) if case["pairs"] else z.unbind(-2))) * turn
        z = torch.stack((z.real, z.imag), -1 if case["pairs"] else -2).flatten(-2)
        return torch.cat((z, y[..., rot:]), -1)

    lens = _lengths(T, B, case["ragged"])
    keep = (torch.arange(T)[None, :] < torch.tensor(lens)[:, None]).to("cuda", torch.float64)[:, :, None, None]
    if kind == "heads":
        return [forward(x.double(), gain.double()) * keep for x, gain in st["heads"]]
    dx, rows, at = torch.zeros(st["dpacked"].shape, device="cuda", dtype=torch.float64), [], 0
    for (x, gain), dy in zip(st["heads"], st["grads"]):
        leaf = x.double().requires_grad_()
        copies = gain.double().view(1, 1, 1, -1).repeat(B, 1, 1, 1).requires_grad_()
        gx, gg = torch.autograd.grad((forward(leaf, copies) * keep * dy.double()).sum(), (leaf, copies))
        dx[:, :, at:at + x.shape[2]] = gx
        rows.append(gg.view(B, -1))
        at += x.shape[2]
    return {"sqnorm": rows[0].pow(2).sum(1) + rows[1].pow(2).sum(1), "gain_rows": rows, "dx": dx}
