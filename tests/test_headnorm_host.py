"""Norms of queries and keys with the rotation: what the entry points refuse before anything is launched.  The addresses are made up
and never touched; a backward call that passes every check stops at the missing workspace."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

A, FAR, FAR2 = 0x10000000, 0x20000000, 0x30000000
B, T, D = 2, 5, 8


@pytest.fixture(scope="module")
def lib():
    return dp.load_library()


def desc(**over):
    d = dict(B=B, T=T, D=D, rot=8, rotation=0, eps=1e-6, positions=None, positions_b=0, freqs=A, lengths=None)
    return dp.HeadnormDesc(**{**d, **over})


def heads(*each):
    """Descriptors of contiguous [B, T, 4, D] tensors, with changes."""
    each = each or ({},)
    arr = (dp.HeadsDesc * len(each))()
    for i, over in enumerate(each):
        s = (T * 4 * D, 4 * D, D)
        d = dict(x=A + 0x100000 * i, x_b=s[0], x_t=s[1], x_h=s[2], H=4, gain=A, out=FAR + 0x100000 * i, o_b=s[0], o_t=s[1], o_h=s[2],
                 dy=FAR2 + 0x100000 * i, dy_b=s[0], dy_t=s[1], dy_h=s[2], gain_rows=A + 0x1000 * i)
        arr[i] = dp.HeadsDesc(**{**d, **over})
    return arr


def back(lib, d=None, h=None, n=None, dtype=dp.DP_BF16, sqnorm=A, ws=None, ws_bytes=0):
    h = heads() if h is None else h
    return lib.dp_headnorm_sqnorm(desc() if d is None else d, h, len(h) if n is None else n, dtype, 0, sqnorm, ws, ws_bytes, None)


OK, BAD, NO = dp.DP_ERR_WORKSPACE, dp.DP_ERR_INVALID_ARG, dp.DP_ERR_UNSUPPORTED


def test_sizes_and_types(lib):
    assert back(lib) == OK and back(lib, h=heads({}, {})) == OK
    for over in ({"B": -1}, {"T": -1}, {"D": 0}, {"rot": -2}, {"rot": 3}, {"rot": 10}, {"eps": 0.0}, {"eps": -1.0}, {"eps": float("nan")},
                 {"rotation": 2}, {"rotation": -1}, {"positions_b": -1}, {"freqs": None}):
        assert back(lib, desc(**over)) == BAD, over
    assert back(lib, desc(rot=0, freqs=None)) == OK and back(lib, desc(rot=2, rotation=1)) == OK
    assert back(lib, n=0) == BAD and back(lib, n=3) == BAD
    assert lib.dp_headnorm_sqnorm(None, heads(), 1, dp.DP_F32, 0, A, None, 0, None) == BAD
    assert lib.dp_headnorm_sqnorm(desc(), None, 1, dp.DP_F32, 0, A, None, 0, None) == BAD
    assert lib.dp_headnorm(desc(), None, 1, dp.DP_F32, None) == BAD and lib.dp_headnorm(None, heads(), 1, dp.DP_F32, None) == BAD
    assert back(lib, dtype=dp.DP_F8_E4M3) == NO and back(lib, dtype=11) == BAD
    assert back(lib, desc(D=513, rot=0)) == NO and back(lib, desc(B=1 << 22)) == NO and back(lib, desc(B=1 << 20, T=1 << 20)) == NO
    assert back(lib, sqnorm=None) == BAD
    assert back(lib, desc(B=0), sqnorm=None) == dp.DP_OK
    assert lib.dp_headnorm(desc(T=0), heads(), 1, dp.DP_F32, None) == dp.DP_OK
    assert lib.dp_headnorm(desc(), heads({"H": 0}), 1, dp.DP_F32, None) == dp.DP_OK
    need = lib.dp_headnorm_workspace_bytes(1, B, T, D)
    assert need > 0 and back(lib, ws=A, ws_bytes=need - 1) == OK and back(lib, ws=A + 8, ws_bytes=need) == OK


def test_addresses_and_strides(lib):
    for name in ("x", "gain", "out", "dy", "gain_rows"):
        assert back(lib, h=heads({name: None})) == BAD, name
    for name in ("x", "out", "dy"):
        assert back(lib, h=heads({name: FAR + 0x900001})) == BAD and back(lib, h=heads({name: FAR + 0x900002})) == OK, name
        assert back(lib, h=heads({name: FAR + 0x900002}), dtype=dp.DP_F32) == BAD
    for name in ("x_b", "x_t", "x_h", "o_b", "o_t", "o_h", "dy_b", "dy_t", "dy_h", "H"):
        assert back(lib, h=heads({name: -1})) == BAD, name
    for name in ("x_b", "o_t", "dy_h"):
        assert back(lib, h=heads({name: 1 << 50})) == NO, name
    assert back(lib, h=heads({"x_b": 0, "x_t": 0, "x_h": 0})) == OK                 # a broadcast input
    assert back(lib, h=heads({"o_t": 0})) == BAD and back(lib, h=heads({"o_h": 7})) == BAD


def test_each_descriptor_has_rows_of_its_own(lib):
    size = 4 * B * D
    assert back(lib, h=heads({}, {"gain_rows": A})) == BAD and back(lib, h=heads({}, {"gain_rows": A + size - 4})) == BAD
    assert back(lib, h=heads({}, {"gain_rows": A + size})) == OK


def test_number_of_heads(lib):
    def wide(H):
        t, b = H * D, T * H * D
        return dict(H=H, x_t=t, x_b=b, o_t=t, o_b=b, dy_t=t, dy_b=b, out=A, dy=1 << 40)
    big = 1 << 20
    assert back(lib, h=heads(wide(big))) == OK and back(lib, h=heads(wide(big + 1))) == NO
    assert back(lib, h=heads({"H": 0}, wide(big + 1))) == NO


def test_outputs_share_nothing(lib):
    es = 2
    # in place of x, or of dy, but not shifted, nor with other strides
    assert back(lib, h=heads({"out": A})) == OK and back(lib, h=heads({"out": FAR2})) == OK
    assert back(lib, h=heads({"out": A + es})) == BAD and back(lib, h=heads({"out": FAR2 + es})) == BAD
    assert back(lib, h=heads({"out": A, "o_t": 5 * D, "o_b": 5 * T * D * 4})) == BAD
    # one descriptor's output in place of the other's input
    assert back(lib, h=heads({"out": A + 0x100000}, {})) == BAD
    assert back(lib, h=heads({}, {"out": FAR})) == BAD
    # queries, keys and values side by side, [B, T, 4 + 4 + 4, D]: outputs in place, or in a packed buffer of their own
    side = dict(x_b=T * 12 * D, x_t=12 * D, o_b=T * 12 * D, o_t=12 * D)
    q, k = dict(side, x=A, out=A), dict(side, x=A + 4 * D * es, out=A + 4 * D * es)
    assert back(lib, h=heads(q, k)) == OK
    assert back(lib, h=heads(dict(q, out=FAR), dict(k, out=FAR + 4 * D * es))) == OK
    assert back(lib, h=heads(q, dict(k, out=A + 8 * D * es))) == OK                 # the keys' where the values were
    assert back(lib, h=heads(q, dict(k, out=A + 7 * D * es))) == BAD                # a head too early: the last key is still read
    assert back(lib, h=heads(q, dict(k, out=A + 9 * D * es))) == BAD                # the last one in the next token's queries
    # heads outside of tokens, [B, 12, T, D]
    out = dict(x_b=T * 12 * D, x_h=T * D, x_t=D, o_b=T * 12 * D, o_h=T * D, o_t=D)
    q, k = dict(out, x=A, out=A), dict(out, x=A + 4 * T * D * es, out=A + 4 * T * D * es)
    assert back(lib, h=heads(q, k)) == OK
    assert back(lib, h=heads(q, dict(k, out=A + (4 * T - 1) * D * es))) == BAD
    # the forward pass looks at no dy
    assert lib.dp_headnorm(desc(), heads({"out": A + es}), 1, dp.DP_BF16, None) == BAD


def test_workspace_sizes(lib):
    f = lib.dp_headnorm_workspace_bytes
    assert f(0, 1, 1, 1) == f(3, 1, 1, 1) == f(1, 0, 1, 1) == f(1, 1, 0, 1) == f(1, 1, 1, 0) == f(1, 1, 1, 513) == f(1, 1 << 22, 1, 8) == 0
    for s in ((1, 1, 1, 1), (2, 64, 512, 64), (2, 1, 100000, 128), (1, (1 << 22) - 1, 1, 512)):
        assert f(*s) >= 4 * s[0] * s[1] * s[3]


def test_binding_refusals():
    x, g = torch.zeros(1, 2, 3, 4), torch.zeros(4)
    with pytest.raises(ValueError):
        dp.headnorm([(x, g)])
    with pytest.raises(ValueError):
        dp.head_descs([], [])
    with pytest.raises(ValueError):
        dp.head_descs([(x, g)], [])
    with pytest.raises(ValueError):
        dp.head_descs([(x, g)], [x], [x])
    with pytest.raises(ValueError):
        dp.headnorm_sqnorm([(x, g)], [x], accumulate=True)
    assert torch.allclose(dp.rotary_freqs(8, device="cpu"), torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-15, atol=0)
