"""Relative position bias: the buckets, and what the entry points refuse before anything is launched.  The addresses are made
up and never touched; a gradient call that passes every check stops at the missing workspace."""
import math

import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

A = 0x10000000


@pytest.fixture(scope="module")
def lib():
    return dp.load_library()


def desc(**over):
    d = dict(B=2, H=3, Tq=5, Tk=7, s_b=105, s_h=35, s_q=7, o_b=105, o_h=35, o_q=7, buckets=A, reach=4, n_buckets=8,
             q_start=None, q_lens=None, k_lens=None, causal=0)
    return dp.PosbiasDesc(**{**d, **over})


def grad(lib, dS=A, dtype=dp.DP_BF16, sqnorm=A, rows=A, ws=None, ws_bytes=0, **over):
    return lib.dp_posbias_sqnorm(desc(**over), dS, dtype, 0, sqnorm, rows, ws, ws_bytes, None)


def test_gradient_refusals(lib):
    assert grad(lib) == dp.DP_ERR_WORKSPACE
    for name in ("B", "H", "Tq", "Tk", "s_b", "s_h", "s_q", "reach"):
        assert grad(lib, **{name: -1}) == dp.DP_ERR_INVALID_ARG, name
    assert grad(lib, n_buckets=0) == dp.DP_ERR_INVALID_ARG
    assert grad(lib, n_buckets=1024) == dp.DP_ERR_WORKSPACE and grad(lib, n_buckets=1025) == dp.DP_ERR_UNSUPPORTED
    assert grad(lib, reach=1 << 20) == dp.DP_ERR_WORKSPACE and grad(lib, reach=(1 << 20) + 1) == dp.DP_ERR_UNSUPPORTED
    assert grad(lib, dtype=dp.DP_F8_E4M3) == dp.DP_ERR_UNSUPPORTED and grad(lib, dtype=9) == dp.DP_ERR_INVALID_ARG
    assert grad(lib, dS=None) == dp.DP_ERR_INVALID_ARG and grad(lib, dS=A + 1) == dp.DP_ERR_INVALID_ARG
    assert grad(lib, dS=A + 2) == dp.DP_ERR_WORKSPACE and grad(lib, dS=A + 2, dtype=dp.DP_F32) == dp.DP_ERR_INVALID_ARG
    assert grad(lib, sqnorm=None) == dp.DP_ERR_INVALID_ARG and grad(lib, rows=None) == dp.DP_ERR_INVALID_ARG
    assert grad(lib, buckets=None) == dp.DP_ERR_INVALID_ARG
    assert grad(lib, s_b=0, s_h=0, s_q=0) == dp.DP_ERR_WORKSPACE                 # broadcast gradients
    assert grad(lib, s_b=1 << 49) == dp.DP_ERR_UNSUPPORTED
    assert grad(lib, B=1 << 31) == dp.DP_ERR_UNSUPPORTED
    for name in ("Tq", "Tk"):
        assert grad(lib, **{name: 1 << 20}) == dp.DP_ERR_WORKSPACE and grad(lib, **{name: (1 << 20) + 1}) == dp.DP_ERR_UNSUPPORTED
    assert grad(lib, B=1 << 20, H=1 << 20) == dp.DP_ERR_UNSUPPORTED
    assert lib.dp_posbias_sqnorm(None, A, dp.DP_F32, 0, A, A, None, 0, None) == dp.DP_ERR_INVALID_ARG
    need = lib.dp_posbias_workspace_bytes(2, 3, 5, 7)
    assert need > 0 and grad(lib, ws=A, ws_bytes=need - 1) == dp.DP_ERR_WORKSPACE and grad(lib, ws=A + 8, ws_bytes=need) == dp.DP_ERR_WORKSPACE
    assert grad(lib, B=0) == dp.DP_OK


def test_add_refusals(lib):
    def add(scores=A, table=A, out=A, dtype=dp.DP_F32, **over):
        return lib.dp_posbias_add(desc(**over), scores, table, dtype, out, None)
    bad = dp.DP_ERR_INVALID_ARG
    assert add(B=0) == add(H=0) == add(Tq=0) == add(Tk=0) == dp.DP_OK            # nothing to do
    assert add(scores=None) == add(table=None) == add(out=None) == add(buckets=None) == bad
    assert add(scores=A + 2, out=A + 2) == bad
    for name in ("o_b", "o_h", "o_q"):
        assert add(**{name: -1}) == bad
    assert add(dtype=dp.DP_F8_E5M2) == dp.DP_ERR_UNSUPPORTED
    # outputs that share elements with the scores, or with each other
    assert add(out=A + 4) == bad and add(out=A + 4 * 209) == bad
    assert add(o_h=36, o_b=108) == bad                                           # in place with other strides
    far = A + 4 * 1000
    assert add(out=far, o_b=0) == bad and add(out=far, o_h=0) == bad and add(out=far, o_q=6) == bad
    assert add(out=far, o_q=7, o_h=34, o_b=105) == bad


def test_size_of_the_table(lib):
    # offsets of its elements are 32-bit numbers
    H = 1 << 20
    wide = dict(B=1, H=H, Tq=1, Tk=1, s_b=H, s_h=1, s_q=1, o_b=H, o_h=1, o_q=1)
    assert grad(lib, n_buckets=1024, **wide) == dp.DP_ERR_WORKSPACE
    wide["H"] += 1
    assert grad(lib, n_buckets=1024, **wide) == dp.DP_ERR_UNSUPPORTED
    assert lib.dp_posbias_add(desc(n_buckets=1024, **wide), A, A, dp.DP_F32, A, None) == dp.DP_ERR_UNSUPPORTED


def test_workspace_sizes(lib):
    f = lib.dp_posbias_workspace_bytes
    assert f(0, 3, 5, 7) == f(2, 3, 0, 7) == f(-1, 3, 5, 7) == f(1 << 31, 1, 1, 1) == 0
    for s in ((1, 1, 1, 1), (64, 12, 512, 512), (3, 5, 197, 64), (1, 1, 1, 100000)):
        assert f(*s) > 0


@pytest.mark.parametrize("n,reach,both", [(32, 128, True), (32, 128, False), (64, 1024, True), (2, 5, False), (8, 9, True), (16, 1000, False)])
def test_buckets(n, reach, both):
    got = dp.relative_buckets(n, reach, both, device="cpu").tolist()
    assert len(got) == 2 * reach + 1 and min(got) >= 0 and max(got) == n - 1
    half = n // 2 if both else n
    single = half // 2
    for d in range(-reach, reach + 1):
        b = got[d + reach]
        if d > 0:
            assert b == (half + got[reach - d] if both else 0)
        elif -d < single:
            assert b == -d
        else:                                            # away from the borders the logarithm says the same
            exact = math.log(-d / single) / math.log(reach / single) * (half - single)
            if abs(exact - round(exact)) > 1e-9:
                assert b == min(half - 1, single + math.floor(exact)), d
            else:
                assert b == min(half - 1, single + round(exact)), d
    back = got[:reach + 1][::-1]
    assert all(a <= b for a, b in zip(back, back[1:]))


def test_binding_refusals():
    for args in ((1, 5), (3, 100), (32, 8), (0, 5), (32, -1)):
        with pytest.raises(ValueError):
            dp.relative_buckets(*args, device="cpu")
    x, t, b = torch.zeros(1, 2, 3, 4), torch.zeros(8, 2), torch.zeros(9, dtype=torch.int32)
    with pytest.raises(ValueError):
        dp.posbias_add(x, t, b)
    with pytest.raises(ValueError):
        dp.posbias_sqnorm(x, b, 8)
