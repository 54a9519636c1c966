"""Draws with top-p whose cut lies where a running sum is within its rounding of what is wanted: one word may stay or go for it, and no more."""
import random

import pytest
import torch

import paper_2508_06041_amd as dp

pytestmark = pytest.mark.gpu

# Logits are whole multiples -j of 2^-22, and j + HALF is half as likely as j to 2e-14: HALF / 4410929 is next to ln 2.
HALF, TEMPERATURE = 3057423, 4410929 * 2.0 ** -22
WORDS = 16384


def row(rng):
    """A row in which the words in front of a cut within a step of the histogram make half of the whole, as every word behind them goes with one in front: two that are half as likely, or one in front
    that is twice as likely as each of two.  Returns the logits and how many are in front."""
    low, high = HALF + 1, HALF + HALF // 8
    middle = rng.randint(low + (high - low) // 10, high - (high - low) // 10)
    n = rng.randint(400, 3000)
    values = [rng.randint(low, middle) for _ in range(rng.choice([1, 2, 3, 5, 9, 40, n]))]
    above = [rng.choice(values) for _ in range(n)]
    gap = rng.choice([1, (high - low) // 200, (high - low) // 20])
    values = [rng.randint(min(middle + gap, high), high) for _ in range(rng.choice([1, 2, 5, 40]))]
    below = [rng.choice(values) for _ in range(rng.randint(200, 1500))]
    front = [0] + [j - HALF for j in below] + above
    behind = 2 * below + [j + HALF for j in 2 * above] + 16 * [4 * HALF]
    x = front + behind
    rng.shuffle(x)
    return [-j * 2.0 ** -22 for j in x] + [float("-inf")] * (WORDS - len(x)), len(front)


@pytest.mark.parametrize("seed", [0, 1, 5, 6, 11, 13, 21, 34, 45, 46])
def test_a_cut_within_rounding(seed):
    rng = random.Random(seed)
    made = [row(rng) for _ in range(64)]
    x = torch.tensor([r for r, _ in made], dtype=torch.float32, device="cuda")

    def all_of(v):
        return torch.full((64,), v, device="cuda")
    kept = torch.zeros(64, dtype=torch.int32, device="cuda")
    words = dp.dpllm_sample(x, all_of(0.999), all_of(TEMPERATURE), top_p=all_of(0.5), kept=kept)
    over = [k - n for k, (_, n) in zip(kept.tolist(), made)]
    assert all(d in (0, 1) for d in over), over
    least = torch.sort(x, dim=1, descending=True).values.gather(1, kept.long()[:, None] - 1)
    assert (x.gather(1, words.long()[:, None]) >= least).all()
