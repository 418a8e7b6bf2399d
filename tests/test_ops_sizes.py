"""What the linear and differential attention's workspace queries answer for sizes
that the calls refuse, without a GPU."""
import pytest

from paper_2609_35110_amd import sol
from test_ops_abi import L  # noqa: F401 (the library is built)

K = 1 << 10


@pytest.mark.parametrize("query", [sol.sol_diff_attn_fwd_workspace_bytes, sol.sol_diff_attn_bwd_workspace_bytes])
@pytest.mark.parametrize("shape", [
    (4 * K, 4 * K, 1, 1, 1, 128),                              # B H = 2^24
    (2 * K, 2, 2, 1, K * K, 128),                              # B Hv M = 2^32
    (2 * K, 1, 1, K * K, 1, 128),                              # B H N = 2^31
    (2 ** 31 - 1, 2 ** 31 - 1, 1, 8 * K * K, 1, 128),          # the product passes 64 bits
])
def test_differential_queries_of_sizes_that_calls_refuse(query, shape):
    assert query(*shape) == 0


def test_linear_queries_of_sizes_that_calls_refuse():
    assert sol.sol_lin_attn_bwd_workspace_bytes(1, 64, 32, 4 * K * K, 128) == 0     # B Hk N = 2^27
    assert sol.sol_lin_attn_bwd_workspace_bytes(1, 64, 32, 2 * K * K, 128) > 0
    assert sol.sol_lin_attn_bwd_workspace_bytes(1, 8, 8, 8 * K * K, 128) > 0        # (heads of their own: no such sum)
    assert sol.sol_lin_attn_bwd_workspace_bytes(2 ** 31 - 1, 2 ** 31 - 1, 1, 8 * K * K, 128) == 0
    assert sol.sol_lin_attn_fwd_workspace_bytes(2 ** 31 - 1, 2 ** 31 - 1, 8 * K * K, 128) == 0
