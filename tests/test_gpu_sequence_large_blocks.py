"""The gradient over lists of large blocks: one block is many key tiles, and parts of its rows are joined."""
import pytest

from test_gpu_sequence_attention import run_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,dtype,d", [
    # B, Hq, Hkv, N, M, q_group, block, top, k_len, q_pos, causal
    ((1, 4, 1, 700, 2500, 64, 1024, 2, None, None, True), "bf16", 128),        # 256 rows a list, a last block of 452 keys
    ((2, 4, 2, 333, 3000, 32, 1024, 3, [3000, 1100], None, True), "f16", 64),
    ((1, 2, 1, 900, 5000, 16, 4096, 2, [4999], None, False), "bf16", 64),
    ((1, 4, 2, 150, 4200, 1, 4096, 1, None, None, True), "f16", 128),           # lists of single queries
    ((1, 2, 2, 1300, 1300, 32, 256, 4, None, None, True), "bf16", 128),
])
def test_gradient(shape, dtype, d):
    run_case(shape, dtype, d, where="tokens", backward=True, seed=121)
