"""Adapters of batches with more sequences than the sorting keeps in registers."""
import pytest

from tests.test_gpu_adapters import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", [0, 1])
@pytest.mark.parametrize("shape", [(1, 4097, 24, 16, 4, 3), (1, 5000, 24, 16, 4, 2500), (2, 9000, 16, 8, 2, 4096), (3, 7000, 8, 12, 3, 1)], ids=str)
def test_more_sequences_than_the_sorting_keeps(shape, mode):
    check(sum(shape), (*shape, mode))
