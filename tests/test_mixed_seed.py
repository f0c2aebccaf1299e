"""Masks of the dropout under seeds made by mixed_seed, from the generator's definition (no GPU needed)."""
import math

import numpy as np

from paper_2101_03961_amd.layer import mixed_seed
from test_operators_gpu import keep_factor

RATE, RUN = 0.25, 2048


def dropped(seed, n):
    return keep_factor(n, RATE, seed).numpy() == 0


def test_seeds_are_64_bits_and_all_differ():
    seeds = [mixed_seed(step, part) for step in range(64) for part in range(64)]
    assert all(0 <= s < 1 << 64 for s in seeds)
    for half in ({s & 0xFFFFFFFF for s in seeds}, {s >> 32 for s in seeds}):
        assert len(half) > 4096 - 8   # 4096^2 / 2^33 = 0.002 equal pairs by chance
    assert mixed_seed(1, 2) != mixed_seed(2, 1) and mixed_seed(0) != mixed_seed(0, 0) and mixed_seed(-1) >= 0


def test_counted_seeds_permute_a_mask_and_mixed_ones_do_not():
    """Dropped elements of aligned runs: a binomial number under mixed seeds, the same under all that share their upper half."""
    n, seeds = 8 * RUN, 256
    counted = np.stack([dropped(s, n).reshape(-1, RUN).sum(1) for s in range(seeds)])
    assert (counted == counted[0]).all()
    for make in (mixed_seed, lambda s: mixed_seed(7, s), lambda s: mixed_seed(s, 7)):
        mixed = np.stack([dropped(make(s), n).reshape(-1, RUN).sum(1) for s in range(seeds)])
        samples, variance = mixed.size, RUN * RATE * (1 - RATE)
        assert abs(mixed.mean() - RUN * RATE) < 6 * math.sqrt(variance / samples)
        assert abs(mixed.var() / variance - 1) < 6 * math.sqrt(2 / samples)


def test_masks_of_neighbouring_counters_agree_by_chance():
    n = 1 << 16
    masks = [dropped(mixed_seed(s), n).reshape(-1, 2) for s in range(12)]
    pairs = np.arange(n // 2)
    both = RATE * RATE
    for a in range(11):
        for other in (0, 1, 2, 3, 8, 64):   # the same pair of elements and its neighbours
            share = float((masks[a] & masks[a + 1][pairs ^ other]).mean())
            assert abs(share - both) < 6 * math.sqrt(both * (1 - both) / n), (a, other)
