"""Eviction from caches that hold nothing, or next to nothing."""
import pytest

from test_gpu_cache import Caches, check_evict

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 96)])
@pytest.mark.parametrize("lens,cap,budget,recent", [([0, 0, 0], 50, 20, 4), ([0], 1, 1, 1), ([0, 1, 0], 1, 1, 0), ([0, 2, 0, 1], 2, 1, 1),
                                                    ([0, 900, 0], 900, 899, 0)])
def test_eviction_from_empty_caches(dtype, D, lens, cap, budget, recent):
    check_evict(Caches(dtype, 2, len(lens), 2, D, cap, lens, seed=cap), budget, recent)
