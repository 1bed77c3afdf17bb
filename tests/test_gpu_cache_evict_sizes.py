"""Eviction on both sides of every capacity at which another kernel chooses, against the oracle, bit for bit."""

import pytest

from test_gpu_cache_evict import build, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("weights", ["spread", "ties", "special"])
@pytest.mark.parametrize("cap", [1024, 1025, 4096, 4097, 12288, 12289, 16500, 20480, 20481, 32768, 32769])
def test_capacities(cap, weights):
    # caches that are full and not quite (behind a budget of all slots but one: not over it); budgets inside the first run of 64 slots and past it
    for budget in (cap // 3, cap - 1, 40):
        check(*build(2, 2, 64, cap, [cap, cap - 1 if budget < cap - 1 else cap // 2], "bf16", cap + budget, weights), budget, sinks=3, keep_from=[cap - 7, cap])


@pytest.mark.parametrize("cap", [20480, 32768, 40000])
def test_all_weights_equal(cap):
    check(*build(2, 1, 128, cap, [cap, cap - 100], "fp16", cap, "equal"), cap // 2)
