"""Sizes of the adapters' workspaces: what they take beside the operands is bounded, whatever the tokens."""
import pytest

import paper_2604_06916_amd as sol

MB = 1 << 20


def sums_bytes(adapters, N, K, rank):
    """da and db of the adapters and of two more, at the next rank of 32, 64 and 128 and rows of up to 128
    columns more; and the slices', 16 KB a wave of eight a CU, twice."""
    rank = 32 if rank <= 32 else 64 if rank <= 64 else 128
    return 4 * rank * (adapters + 2) * (N + K + 256) + 2 * 8 * 256 * (16 << 10)


@pytest.mark.parametrize("tokens", [1, 777, 26574, 1 << 20, (1 << 27) - 1])
@pytest.mark.parametrize("N,K", [(16, 16), (7296, 2432), (9728, 9728), (40, 65536)])
@pytest.mark.parametrize("rank", [1, 32, 64, 128])
@pytest.mark.parametrize("adapters", [1, 48])
def test_gradients(tokens, N, K, rank, adapters):
    for planned in {adapters > 1, True}:
        need = sol.adapters_backward_workspace_bytes(tokens, adapters, planned, N, K, rank)
        assert 0 < need <= 256 * MB + sums_bytes(adapters, N, K, rank)


def test_gradients_of_the_widest_rows():
    # a tile's shares of g alone pass the bound: one tile at a time
    need = sol.adapters_backward_workspace_bytes(1000, 1, False, (1 << 22) - 1, 64, 128)
    assert need <= 32 * 128 * 4 * (1 << 14) + 64 * 1024 + sums_bytes(1, 1 << 22, 64, 128)


def test_figures():
    size = sol.adapters_backward_workspace_bytes
    assert size(26574, 2, True, 7296, 2432, 128) < 340 * MB and size(1 << 20, 2, True, 9728, 9728, 128) < 360 * MB
    # one run
    assert size(26574, 2, True, 7296, 2432, 32) < 128 * MB
