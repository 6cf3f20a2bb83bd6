"""Linear attention and group norm at the edges of what their entry points take, on the CPU:
sizes, workspaces and refusals."""

import paper_2606_06034_amd as G


def test_no_sequences_take_no_workspace():
    """Packed tokens of which no sequence has any: no segments, no states, no sums of tokens
    (cu_seqlens holds one offset; a segment would read the next one)."""
    for T in (64, 512, 100_000):
        for dims in ((1, 2, 64, 64), (4, 4, 128, 128), (2, 6, 128, 64)):
            assert G.gdn_linear_forward_workspace(0, T, *dims, packed=True) == 0
            assert G.gdn_linear_backward_workspace(0, T, *dims, packed=True) == 0
