"""The lists in which the log probabilities' kernels gather candidates for the top alternatives hold those of ordinary rows."""
import os
import re

import numpy as np
import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1910_05124_b200", "csrc", "pm_logprob.cu")


def constant(name):
    return int(re.search(rf"constexpr int [^;]*\b{name} = (\d+)", open(SOURCE).read()).group(1))


def entries(kind, k):
    return constant("kLpShortList") if kind == "warp" and k <= constant("kLpShortK") else constant("kLpList")


@pytest.mark.parametrize("kind", ["warp", "block"])
@pytest.mark.parametrize("vocab,per_vector", [(500, 8), (1000, 4), (4000, 4)])
@pytest.mark.parametrize("k", [1, 8, 20, 28, 29, 31, 32])
def test_overflow_is_rare(kind, vocab, per_vector, k):
    """Independent logits, by rank: vectors go round 32 lanes, the threshold is the k-th largest of the lanes' maxima, and a list that
    overflows costs k more passes over the row.  Few enough elements reach the threshold in all but one row of a thousand."""
    size, rng, rows = entries(kind, k), np.random.default_rng(k), 4000
    order = rng.permuted(np.tile(np.arange(vocab, dtype=np.int16), (rows, 1)), axis=1)
    lane = np.arange(vocab) // per_vector % 32
    best = np.stack([order[:, lane == i].max(1) for i in range(32)], 1)
    threshold = np.sort(best, 1)[:, 32 - k]
    candidates = (order >= threshold[:, None]).sum(1)
    assert (candidates > size).mean() <= 1 / 1000, (candidates.mean(), candidates.std(), (candidates > size).mean())
