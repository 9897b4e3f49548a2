"""How far the 8-bit form of activations lies from the values, as include/cbm.h states it: half a step but for the smallest values and the topmost 1/128 of a binade, a step at most."""
import os
import re

import numpy as np

from oracle import train_oracle as orc

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "cbm.h")


def _top_of_a_binade():
    """Blocks whose largest value lies in [64, 128) steps, every 1/16 of a step of it."""
    x = np.zeros((64 * 16, 32))
    x[:, 0] = 64 + np.arange(64 * 16) / 16
    q, e = orc.keep(x)
    assert not e.any()
    return x[:, 0], np.abs(orc.kept_values(q, e)[:, 0] - x[:, 0])


def test_half_a_step_below_the_topmost_128th_of_a_binade():
    with open(HEADER) as f:
        share = int(re.search(r"topmost 1 / (\d+) of a binade", f.read()).group(1))
    x, off = _top_of_a_binade()
    top = x > 128 - 64 / share
    assert np.all(off[~top] <= 0.5) and np.all((off[top] > 0.5) & (off[top] < 1))


def test_a_step_at_most_for_the_smallest_values():
    x = np.zeros((200, 32))
    x[:, 0], x[:, 1] = 64.0, np.arange(200) / 400  # below half a step: they keep one
    q, e = orc.keep(x)
    off = np.abs(orc.kept_values(q, e)[:, 1] - x[:, 1])
    assert off[0] == 0 and np.all((off[1:] > 0.5) & (off[1:] < 1))
