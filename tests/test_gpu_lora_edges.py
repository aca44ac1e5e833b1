"""heal_lora_add where loads of four elements reach the end of the bank."""
import pytest

from gpu_util import needs_gpu
from test_gpu_lora import TYPES, check, make

pytestmark = [pytest.mark.gpu, needs_gpu]


@pytest.mark.parametrize("type_", list(TYPES))
@pytest.mark.parametrize("N", [1, 2, 31, 32, 33, 34, 35, 36, 65, 66, 129, 1057, 4098])
@pytest.mark.parametrize("rank", [1, 2, 3, 5])
def test_the_last_columns_of_the_last_adapter(rank, N, type_):
    """Few and many tokens with the bank's last adapter, widths at which its last rows of B are a
    group's last ones."""
    bank = make(2, rank, 68, N, TYPES[type_], ranks=False, seed=N)
    check(bank, [1], [1], ragged=False)
    check(bank, [1, 0, 1], [1, 2, 40])
    check(bank, [0, 1], [30, 70], place="y")
