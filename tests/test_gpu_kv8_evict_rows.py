"""Evictions of rows that the selection treats differently, in one batch: rows longer than the ranks that are held in LDS, rows most of whose
wavefronts have no slots, many rows of four wavefronts.  All exactly as the oracle's, which sorts."""
import pytest
import torch

from kv8_util import Twin
from test_gpu_kv8 import evict_and_check

pytestmark = pytest.mark.gpu


def weights_and_positions(t):
    w, _, pos = t.weight_arrays()
    w[t.rng.random(w.shape) < 0.4] = 0.5
    w[t.rng.random(w.shape) < 0.1] = 0.0
    for s, n in enumerate(t.len):
        pos[s, :, :n] = torch.arange(n, device="cuda", dtype=torch.int32)
    return w, pos


@pytest.mark.parametrize("in_place", [False, True])
def test_rows_longer_than_the_ranks_that_are_held(in_place):
    """16 wavefronts hold 2048 ranks each"""
    with Twin(1024, 32, 1, 1, max_seqs=4, max_tokens=40100) as t:
        t.step([0, 1, 2, 3], [40000, 32769, 70, 33000])
        w, pos = weights_and_positions(t)
        w[3] = 0.5  # equal ones only: the lower slots stay
        evict_and_check(t, [0, 1, 2, 3], [39500, 32500, 20, 32800], 100, w, pos, in_place)


@pytest.mark.parametrize("recent", [0, 37])
def test_rows_most_of_whose_wavefronts_have_no_slots(recent):
    with Twin(2048, 64, 4, 1, max_seqs=6, max_tokens=4200) as t:
        t.step([0, 1, 2, 3, 4, 5], [4097, 64, 1, 130, 2000, 65])
        w, pos = weights_and_positions(t)
        evict_and_check(t, [0, 1, 2, 3, 4, 5], [3900, 60, 1, 1, 1990, 64], recent, w, pos)


def test_more_rows_than_compute_units():
    """four wavefronts a row, up to 2048 slots each"""
    with Twin(2048, 32, 32, 1, max_seqs=9, max_tokens=8192) as t:
        size = [8190, 5000, 3, 64, 65, 100, 256, 300, 40]
        t.step(list(range(9)), size)
        w, pos = weights_and_positions(t)
        evict_and_check(t, list(range(9)), [8040, 4900, 1, 64, 60, 5, 200, 0, 33], 20, w, pos)
