"""Dropout and the serendipity noise draw apart under one seed and draw.  Both number Philox blocks from 0; what a block's
words decide is compared with what the same block decides for the other operator.  That words in common would show is
tested on the CPU, with the oracle's key, and on the device, with a seed that takes back what dropout does to the key."""
import numpy as np
import pytest
import torch

import block_oracle as bo
import oracle
import paper_2502_11490_amd as ann

BLOCKS, SEED, DRAW = 8192, (3 << 35) + 11, 4


def _agreement(noise, kept):
    """How far the signs and the magnitudes of the noise of a block agree with what is kept by the same block's words, beyond
    chance: noise element 4 b + k is drawn from words k and k ^ 1 of block b, kept element 8 b + 2 k + i from half i of word k."""
    z, kept = torch.as_tensor(noise).reshape(BLOCKS, 4), torch.as_tensor(kept).reshape(BLOCKS, 8)
    return max(abs(float((a == kept[:, j]).float().mean()) - 0.5)
               for k in range(4) for a in (z[:, k] > 0, z[:, k].abs() > 0.6745) for j in range(8))


CHANCE = 6 * 0.5 / BLOCKS ** 0.5  # six standard deviations of the mean of BLOCKS fair coins


def test_agreement_sees_the_same_words():
    noise = oracle.users_add_noise(np.zeros((1, 4 * BLOCKS), np.float32), 1.0, SEED, DRAW)
    elements = np.arange(8 * BLOCKS)
    assert _agreement(noise, bo.kept(elements, 0.5, SEED, DRAW)[0]) < CHANCE
    same_key = SEED ^ (0x64726F70 << 32)  # takes back what dropout does to the key
    assert _agreement(noise, bo.kept(elements, 0.5, same_key, DRAW)[0]) > 10 * CHANCE


@pytest.mark.gpu
def test_dropout_draws_other_words_than_the_noise():
    noise = ann.ann_users_add_noise(torch.zeros(1, 4 * BLOCKS, device="cuda"), 1.0, SEED, DRAW)
    kept = ann.ann_dropout(torch.ones(8 * BLOCKS, device="cuda"), 0.5, SEED, DRAW) != 0
    assert _agreement(noise.cpu(), kept.cpu()) < CHANCE
    same = ann.ann_dropout(torch.ones(8 * BLOCKS, device="cuda"), 0.5, SEED ^ (0x64726F70 << 32), DRAW) != 0
    assert _agreement(noise.cpu(), same.cpu()) > 10 * CHANCE
