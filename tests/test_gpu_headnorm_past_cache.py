"""Norms of queries and keys whose inputs fit the last-level cache of 256 MB without the outputs, which then take another way to
memory: every type and pairing, against 64-bit arithmetic with the tolerances of the other sizes."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp
from test_gpu_headnorm import check, full, make

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
# heads' bytes between 128 and 256 MB (forward), between 85 and 128 MB (backward, of two inputs)
FORWARD, BACKWARD = 146_000_000, 105_000_000


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "pairs"])
@pytest.mark.parametrize("size", [FORWARD, BACKWARD], ids=["forward", "backward"])
@pytest.mark.parametrize("D,rot,padded", [(64, 64, False), (96, 32, True)])
def test_outputs_past_the_cache(dtype, pairs, size, D, rot, padded):
    B, Hs = 2, (6, 3)
    T = size // (B * sum(Hs) * D * (4 if dtype == F32 else 2))
    lengths = torch.tensor([T, T - 700], dtype=torch.int32, device="cuda") if padded else None
    heads, dys = make(B, T, Hs, D, dtype, seed=D, lengths=lengths)
    check(heads, dys, full(heads), full(heads), dp.rotary_freqs(rot), lengths=lengths, pairs=pairs)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("pairs", [False, True], ids=["halves", "pairs"])
def test_many_heads_of_one_token(dtype, pairs):
    """Sums of more rows than a chain of float32 has, and outputs past the cache."""
    D = 512
    heads, dys = make(1, 1, (BACKWARD // (D * (4 if dtype == F32 else 2)),), D, dtype, seed=3)
    check(heads, dys, full(heads), full(heads), dp.rotary_freqs(64), pairs=pairs)
