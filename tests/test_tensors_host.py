"""Norm and clipping of many tensors: what the entry points refuse, before anything is launched.  The addresses are made up and
never touched; a call that passes every check stops at the missing workspace."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp

F32, BF16, F16 = dp.DP_F32, dp.DP_BF16, dp.DP_F16
A = 0x10000000


@pytest.fixture(scope="module")
def lib():
    return dp.load_library()


def descs(*items):
    arr = (dp.TensorDesc * max(1, len(items)))()
    for i, it in enumerate(items):
        arr[i] = dp.TensorDesc(*it)
    return arr, len(items)


def norm(lib, *items, out=A, ws=None, ws_bytes=0):
    arr, n = descs(*items)
    return lib.dp_tensors_norm(arr, n, 0, out, None, ws, ws_bytes, None)


def clip(lib, *items, C=1.0, accumulate=0, out=0x800):
    arr, n = descs(*items)
    both = lib.dp_tensors_norm_clip(arr, n, C, accumulate, out, None, None, 0, None)
    assert lib.dp_tensors_clip(arr, n, out, C, accumulate, None, 0, None) == both
    return both


def test_norm_refusals(lib):
    ok = (A, None, 100, F32, F32)
    assert norm(lib, ok) == dp.DP_ERR_WORKSPACE
    assert norm(lib, ok, out=None) == dp.DP_ERR_INVALID_ARG
    assert norm(lib, (None, None, 100, F32, F32)) == dp.DP_ERR_INVALID_ARG
    assert norm(lib, (None, None, 0, F32, F32)) == dp.DP_ERR_WORKSPACE            # an empty tensor needs no address
    assert norm(lib, (A, None, -1, F32, F32)) == dp.DP_ERR_INVALID_ARG
    assert norm(lib, (A + 2, None, 100, F32, F32)) == dp.DP_ERR_INVALID_ARG       # not on an element
    assert norm(lib, (A + 2, None, 100, BF16, F32)) == dp.DP_ERR_WORKSPACE
    assert norm(lib, (A + 1, None, 100, F16, F32)) == dp.DP_ERR_INVALID_ARG
    assert norm(lib, (A, None, 100, dp.DP_F8_E5M2, F32)) == dp.DP_ERR_UNSUPPORTED
    assert norm(lib, (A, None, 100, 17, F32)) == dp.DP_ERR_INVALID_ARG
    assert norm(lib, (A, None, (1 << 48) + 1, F32, F32)) == dp.DP_ERR_UNSUPPORTED
    assert norm(lib, (A, None, 1 << 48, F32, F32), (A, None, 1, F32, F32)) == dp.DP_ERR_UNSUPPORTED
    need = lib.dp_tensors_workspace_bytes(1)
    assert norm(lib, ok, ws=A, ws_bytes=need - 1) == dp.DP_ERR_WORKSPACE
    assert norm(lib, ok, ws=A + 8, ws_bytes=need) == dp.DP_ERR_WORKSPACE
    arr, _ = descs(ok)
    assert lib.dp_tensors_norm(arr, -1, 0, A, None, None, 0, None) == dp.DP_ERR_INVALID_ARG
    assert lib.dp_tensors_norm(None, 1, 0, A, None, None, 0, None) == dp.DP_ERR_INVALID_ARG
    assert lib.dp_tensors_norm(arr, (1 << 20) + 1, 0, A, None, None, 0, None) == dp.DP_ERR_UNSUPPORTED


def test_clip_refusals(lib):
    assert clip(lib, (A, A, 100, F32, F32)) == dp.DP_ERR_WORKSPACE                # in place
    assert clip(lib, (A, A + 400, 100, F32, F32)) == dp.DP_ERR_WORKSPACE          # right behind
    assert clip(lib, (A, A + 396, 100, F32, F32)) == dp.DP_ERR_INVALID_ARG        # one element shared
    assert clip(lib, (A + 396, A, 100, F32, F32)) == dp.DP_ERR_INVALID_ARG
    assert clip(lib, (A, A, 100, BF16, F32)) == dp.DP_ERR_INVALID_ARG             # a wider type in place
    assert clip(lib, (A, A + 200, 100, BF16, F32)) == dp.DP_ERR_WORKSPACE
    assert clip(lib, (A, A + 4, 100, BF16, F16)) == dp.DP_ERR_INVALID_ARG         # other types
    assert clip(lib, (A, A + 4000, 100, F32, BF16)) == dp.DP_ERR_INVALID_ARG
    assert clip(lib, (A, None, 100, F32, F32)) == dp.DP_ERR_INVALID_ARG
    assert clip(lib, (A, None, 0, F32, F32)) == dp.DP_ERR_WORKSPACE
    assert clip(lib, (A, A + 401, 100, F32, F32)) == dp.DP_ERR_INVALID_ARG
    assert clip(lib, (A, A, 100, F32, dp.DP_F8_E4M3)) == dp.DP_ERR_UNSUPPORTED
    for C in (0.0, -1.0, float("nan")):
        assert clip(lib, (A, A, 100, F32, F32), C=C) == dp.DP_ERR_INVALID_ARG
    assert clip(lib, (A, A, 100, F32, F32), out=None) == dp.DP_ERR_INVALID_ARG
    # sums go into float32
    assert clip(lib, (A, A + 200, 100, BF16, BF16), accumulate=1) == dp.DP_ERR_INVALID_ARG
    assert clip(lib, (A, A + 200, 100, BF16, F32), accumulate=1) == dp.DP_ERR_WORKSPACE


def test_outputs_of_several_tensors_are_apart(lib):
    def t(x, o, n=100):
        return (A + x, A + o, n, F32, F32)
    assert clip(lib, t(0, 0), t(400, 400)) == dp.DP_ERR_WORKSPACE
    assert clip(lib, t(400, 400), t(0, 0)) == dp.DP_ERR_WORKSPACE                 # in any order
    assert clip(lib, t(0, 0), t(0, 0)) == dp.DP_ERR_INVALID_ARG                   # the same tensor twice, in place
    assert clip(lib, t(0, 4000), t(0, 8000)) == dp.DP_ERR_WORKSPACE               # twice, apart
    assert clip(lib, t(0, 4000), t(400, 4000)) == dp.DP_ERR_INVALID_ARG
    assert clip(lib, t(0, 4000), t(400, 4396)) == dp.DP_ERR_INVALID_ARG
    assert clip(lib, t(0, 400), t(400, 0)) == dp.DP_ERR_INVALID_ARG               # each other's inputs
    assert clip(lib, t(0, 0), t(400, 800), t(800, 400)) == dp.DP_ERR_INVALID_ARG
    assert clip(lib, t(0, 0), t(2000, 1000), t(400, 400)) == dp.DP_ERR_WORKSPACE
    assert clip(lib, t(0, 0, 1000), t(400, 8000)) == dp.DP_ERR_INVALID_ARG        # an input inside another's output
    many = [t(800 * i, 800 * i + 400) for i in range(300)]
    assert clip(lib, *many) == dp.DP_ERR_WORKSPACE
    assert clip(lib, *many, t(800 * 7 + 396, 1 << 20, 1)) == dp.DP_ERR_WORKSPACE  # an input inside another input
    assert clip(lib, *many, t(1 << 20, 800 * 7 + 796, 1)) == dp.DP_ERR_INVALID_ARG


def test_workspace_sizes(lib):
    f = lib.dp_tensors_workspace_bytes
    assert f(-1) == 0 and f((1 << 20) + 1) == 0
    assert all(f(n) >= 8 * (2048 + n) for n in (0, 1, 112, 113, 5000, 1 << 20))
    assert all(f(n + 1) >= f(n) for n in (0, 1, 111, 112, 113, 4000))


def test_binding_refuses_host_tensors_and_wrong_outputs():
    x = torch.zeros(4)
    with pytest.raises(ValueError):
        dp.tensor_descs([x])
    with pytest.raises(ValueError):
        dp.tensor_descs([])
    with pytest.raises(ValueError):
        dp.tensor_descs([x], [x, x])
    with pytest.raises(ValueError):
        dp.tensor_descs([x], [x], in_place=True)
    with pytest.raises(ValueError):
        dp.tensors_norm_clip([x], 1.0, accumulate=True)
    with pytest.raises(ValueError):
        dp.tensors_clip([x], x, 1.0, accumulate=True)
    with pytest.raises(ValueError):
        dp.tensors_norm([x], accumulate=True)
