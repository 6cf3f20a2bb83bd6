"""Linear attention and group norm at the edges of what their entry points take, on the CPU:
sizes, workspaces and refusals."""

import torch

import paper_2606_06034_amd as G


def test_no_sequences_take_no_workspace():
    """Packed tokens of which no sequence has any: no segments, no states, no sums of tokens
    (cu_seqlens holds one offset; a segment would read the next one)."""
    for T in (64, 512, 100_000):
        for dims in ((1, 2, 64, 64), (4, 4, 128, 128), (2, 6, 128, 64)):
            assert G.gdn_linear_forward_workspace(0, T, *dims, packed=True) == 0
            assert G.gdn_linear_backward_workspace(0, T, *dims, packed=True) == 0


def test_rows_of_a_short_chunk_in_reversed_time():
    """dK and dV place a chunk's rows from the end of a block of 16, at 32-bit byte offsets of fp32
    rows: 16 rows of all heads, however few tokens there are, hold 2^30 values at most."""
    ptr = [k << 44 for k in range(1, 14)]  # (a tensor of these sizes is under 2^44 bytes)

    def call(T, H, dtype, dk=128, dv=128, Q=ptr[0]):
        return G.lib.gdn_linear_backward(
            Q, ptr[1], ptr[2], ptr[3], 0, ptr[4], None, None, ptr[5], ptr[6], ptr[7], ptr[8], None,
            ptr[9], 1 << 43, None, 1, T, H, H, dk, dv, 1.0, dtype, None)

    SHAPE, NULL = -2, -1
    most = (1 << 30) // 16 // 128  # heads
    for dtype in (0, 1):
        for T in (1, 7, 15, 16):
            assert call(T, 600_000, dtype) == SHAPE
            assert call(T, most + 1, dtype) == SHAPE
            assert call(T, most, dtype, Q=None) == NULL  # past the sizes
            assert call(T, 2 * most + 2, dtype, 64, 64) == SHAPE
        assert call(17, most, dtype) == SHAPE


def test_group_norm_gradients_of_many_rows_take_few_sums():
    """Past some thousand n's, one more takes two sums of each group and part of it (in 256 pieces),
    and no row of dw and db of its own."""
    for dtype, dt, V in ((torch.bfloat16, 1, 8), (torch.float32, 0, 4)):
        for S, C, groups in ((1, 16384, 1), (4, 64, 8), (2, 64, 8), (49, 40, 5), (7, 8192, 2)):
            parts = max(1, -(-(C // groups // V) // 256))
            f = lambda N: G.gdn_group_norm_backward_workspace(N, S, C, groups, dtype)  # noqa: E731
            assert f(20_000) - f(10_000) == 10_000 * groups * parts * 2 * 4
            x = 20_000 * S * C * (2 if dt else 4)
            # rows of dw and db: as many as the workgroups that run at a time have channels
            assert f(20_000) <= x // 3 + 2 * 2048 * 256 * V * 4


def test_sequences_and_heads_of_the_recurrent_form():
    """A wave takes 32 value columns of a head, a workgroup of 256 work items four waves: 2^26 waves
    are past HIP's 2^32 work items, a workgroup less is not."""
    ptr = [k << 50 for k in range(1, 8)]

    def call(nseq, Hv, dv, Q=None):
        return G.lib.gdn_linear_recurrent(Q, ptr[1], ptr[2], ptr[3], 0, None, ptr[4], None, None, 0,
                                          None, nseq, 1, 1, Hv, 64, dv, 1.0, 1, None)

    SHAPE, NULL = -2, -1
    for dv in (64, 128):
        waves = 1 << 26
        heads = waves // (dv // 32)
        assert call(heads // 4, 4, dv) == SHAPE
        assert call(heads // 4 - 1, 4, dv) == NULL  # past the sizes
        assert call(heads // 4 // 4, 4, dv) == NULL
        assert call(1 << 30, 1 << 30, dv) == SHAPE
        assert call((1 << 31) - 1, (1 << 31) - 1, dv) == SHAPE


def test_group_norm_gradients_without_sums_of_rows():
    """Rows in registers use the workspace for dw and db alone: without these it may be NULL."""
    ptr = [k << 40 for k in range(1, 10)]

    def call(S, dw, db, ws, wsb=0, dx=ptr[5] + 4, C=96, N=8):
        return G.lib.gdn_group_norm_backward(ptr[0], ptr[1], ptr[2], None, None, ptr[3], ptr[4], dx,
                                             dw, db, None, ws, wsb, N, S, C, 8, 0, 1, 0, None)

    NULL, ALIGN, WS = -1, -5, -9
    assert call(1, None, None, None) == ALIGN  # past the workspace: dx is refused
    assert call(1, ptr[6], None, None) == NULL
    assert call(1, None, ptr[6], None) == NULL
    assert call(1, ptr[6], None, ptr[7], 4) == WS
    assert call(5, None, None, None) == NULL  # read twice: the groups' sums
    assert call(1, None, None, None, C=65536) == ALIGN
