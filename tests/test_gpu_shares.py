"""Schedules of latent attention that mix long and short requests, whole tiles and halves, units that are cut and units that are not."""
import numpy as np
import pytest

import latent_reference as ref
from test_gpu_expanded import _check as check_expanded
from test_gpu_latent import _check as check_latent

pytestmark = pytest.mark.gpu


# 64 rows or fewer in a pair's last tile: all of them cut; some of them as short as a share; more than one tile before the half
HALVES = {
    "cut": (32, [4, 2, 1], [3000, 2900, 3100], 64), "one_past_a_tile": (32, [5, 4, 2], [2000, 1777, 1999], 16), "short_ones": (32, [4, 4, 1, 2, 4], [2500, 40, 33, 100, 1500], 16),
    "odd_steps": (32, [4, 1, 2, 4], [1025, 1089, 1151, 1200], 48), "tables_end": (32, [4, 2, 2], [2000, 1000, 1500], 16), "many": (32, [4, 1, 2, 3] * 20, [700 + 37 * i for i in range(80)], 64),
    "nothing_cached": (32, [4, 2, 4, 2], [2000, 1, 3000, 0], 16),
}


@pytest.mark.parametrize("latent", [512, 256])
@pytest.mark.parametrize("kind", list(HALVES))
def test_halves_of_the_absorbed_form(kind, latent):
    heads, new, total, page = HALVES[kind]
    check_latent(ref.latent_inputs(heads, latent, page, new, total, seed=len(kind), gap=2, width=70 if kind == "tables_end" else None))


@pytest.mark.parametrize("seed", range(6))
def test_lengths_of_all_sizes_absorbed(seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(2, 40))
    new = [int(x) for x in rng.integers(0, 6, n)]
    total = [int(x) for x in np.exp(rng.uniform(0, np.log(4000 if n < 12 else 900), n))]
    check_latent(ref.latent_inputs(int(rng.choice([16, 20, 40])), int(rng.choice([256, 512])), int(rng.choice([16, 48, 64])), new, total, seed=seed, gap=1))


@pytest.mark.parametrize("seed", range(6))
def test_lengths_of_all_sizes_expanded(seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(1, 9))
    new = [int(x) for x in rng.integers(0, 600, n)]
    total = [int(x) for x in np.exp(rng.uniform(0, np.log(4000), n))]
    check_expanded(ref.expanded_inputs(int(rng.choice([1, 3, 8])), new, total, seed=seed, gap=1))


@pytest.mark.parametrize("heads", [1, 40])
def test_more_requests_than_threads_absorbed(heads):
    """Runs of several requests per thread of the schedule; one long request among short and empty ones."""
    rng = np.random.default_rng(heads)
    new = [int(x) for x in rng.integers(0, 4, 1500)]
    total = [int(x) for x in rng.integers(0, 90, 1500)]
    total[777], new[777] = 6000, 3
    check_latent(ref.latent_inputs(heads, 256, 16, new, total, seed=1))


def test_more_requests_than_threads_expanded():
    rng = np.random.default_rng(2)
    new = [int(x) for x in rng.integers(0, 3, 1500)]
    total = [int(x) for x in rng.integers(0, 60, 1500)]
    total[1201], new[1201] = 5000, 300
    check_expanded(ref.expanded_inputs(2, new, total, seed=1))


def test_the_most_requests():
    """4096 of one token each: the limit of a call."""
    check_latent(ref.latent_inputs(2, 256, 16, [1] * 4096, [1 + 7 * i % 40 for i in range(4096)], seed=1))
