"""Selection for one and two queries of many sequences: either side of the choice between the two kernels."""
import pytest

pytestmark = pytest.mark.gpu
from test_gpu_block_select import test_selection as check  # noqa: E402


@pytest.mark.parametrize("T", [1, 2, 3])
@pytest.mark.parametrize("B,S,H,G,D,block,n_select,dtype", [(130, 515, 16, 8, 64, 32, 8, "bf16"), (256, 300, 4, 4, 40, 32, 4, "f32"), (90, 2100, 12, 12, 24, 64, 20, "bf16")])
def test_single_tokens_of_many_sequences(T, B, S, H, G, D, block, n_select, dtype):
    assert B * G >= 1024
    lengths = [max(0, S - 7 * b) for b in range(B)]                 # some empty or shorter than the queries
    check(B, T, S, H, G, D, block, n_select, dtype, lengths)
