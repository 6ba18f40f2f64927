"""More units (an entry and a key head) than a die goes through at a time: each has its results, the last group's among them."""
import pytest

from test_gpu_attention import BF16, F32, both, inputs

pytestmark = pytest.mark.gpu


# three tiles of 128 rows and of 128 keys, of 40 and 36 units a die, 22 at a time: the last group has 18 and 14; 41 x 7 leaves one place of
# 8 x 36 without a unit
@pytest.mark.parametrize("B,H", [(40, 8), (41, 7)])
@pytest.mark.parametrize("dtype,causal", [(BF16, True), (F32, False)])
def test_units_of_a_die_in_groups(B, H, dtype, causal):
    T = 260
    lens = [T - 3 * b for b in range(B)]
    both(*inputs(B, T, T, H, H, 24, dtype), causal=causal, q_lens=lens, k_lens=lens)
