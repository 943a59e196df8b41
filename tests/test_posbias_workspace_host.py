"""Scratch of the relative position bias's gradient: in proportion to the table, and what the call asks for."""
import pytest

from paper_2009_03106_amd import dpclip as dp

A = 0x10000000


@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (64, 12, 512, 512), (3, 5, 197, 64), (1, 1, 1, 100000), (4, 16, 4096, 4096)])
def test_sizes(shape):
    lib = dp.load_library()
    f = lambda nb: lib.dp_posbias_table_workspace_bytes(*shape, nb)
    assert f(1024) == lib.dp_posbias_workspace_bytes(*shape) > 0
    assert f(0) == f(-1) == f(1025) == 0
    for nb in (1, 7, 32, 100):
        assert f(nb) % 16 == 0 and f(nb) <= max(16, -(-f(1024) * nb // 1024) + 15)
        B, H, Tq, Tk = shape
        d = dp.PosbiasDesc(B=B, H=H, Tq=Tq, Tk=Tk, s_b=H * Tq * Tk, s_h=Tq * Tk, s_q=Tk, o_b=0, o_h=0, o_q=0, buckets=A, reach=4, n_buckets=nb)
        assert lib.dp_posbias_sqnorm(d, A, dp.DP_F32, 0, A, A, A, f(nb) - 1, None) == dp.DP_ERR_WORKSPACE


def test_refused_sizes():
    f = dp.load_library().dp_posbias_table_workspace_bytes
    assert f(0, 3, 5, 7, 8) == f(2, 3, 0, 7, 8) == f(-1, 3, 5, 7, 8) == f(1 << 31, 1, 1, 1, 8) == 0


def test_a_batch_of_512_positions():
    # 768 heads of up to nine workgroups each, 32 numbers of 64 bits
    assert dp.load_library().dp_posbias_table_workspace_bytes(64, 12, 512, 512, 32) <= 2 << 20
