"""Attention over 4-bit pools in batches whose sequences differ most: many single tokens beside one long turn (whose row blocks a few
workgroups then walk one after the other) and one long history beside many short ones."""
import math

import numpy as np
import pytest

from paper_2601_11589_amd import inputs
from test_gpu_kv4 import Batch, plan

pytestmark = pytest.mark.gpu

# new tokens, longest prefixes, query rows a workgroup, spare pages of the table, keys in parts
BATCHES = {
    "one_tile": (inputs.qwen14b_cfg, [1] * 127 + [64], 300, 16, 2, False),
    "two_tiles": (inputs.qwen14b_cfg, [1] * 95 + [350], 200, 32, 2, False),
    "two_tiles_in_parts": (inputs.qwen7b_cfg, [1] * 20 + [100], 3000, 32, 40, True),
    "long_turn_first": (inputs.qwen7b_cfg, [200] + [1] * 60, 500, 32, 300, True),
    "small_heads": (inputs.tiny_cfg, [1] * 200 + [300, 0], 700, 16, 2, False),
}


@pytest.mark.parametrize("name", sorted(BATCHES))
def test_single_tokens_beside_a_long_turn(name):
    cfgf, new, longest, rows, spare, parts = BATCHES[name]
    g = np.random.default_rng(len(new))
    b = Batch(cfgf(1), new, g.integers(0, longest, len(new)), spare=spare).write()
    p, group = plan(b), b.cfg.n_q_heads // b.cfg.n_kv_heads
    assert p[0] == rows and max(new) * group > 2 * p[0] * p[1], p       # the long turn's blocks are walked in turns
    assert (p[2] > 1) == parts, p
    b.check(b.attend())
    b.ctx.close()


def test_a_nan_that_only_later_blocks_of_a_walk_see():
    cfgf, new, _, _, spare, _ = BATCHES["one_tile"]
    for which in ("v", "k"):
        b = Batch(cfgf(1), new, [7] * 127 + [100], spare=spare)
        at = int(b.first[127]) + 100 + 40                               # the long turn's 41st new token
        (b.v if which == "v" else b.k)[at, 1, 37] = math.nan
        b.write()
        want = b.oracle()
        row = np.isnan(want[0]).any((1, 2))
        assert row[int(b.cu[127]) + 40:].all() and not row[:int(b.cu[127]) + 40].any()
        b.check(b.attend(), want)
        b.ctx.close()


@pytest.mark.parametrize("cfgf", [inputs.tiny_cfg, inputs.qwen7b_cfg])
def test_one_long_history_beside_short_ones(cfgf):
    b = Batch(cfgf(1), [1] * 40, [9000] + [37 * i % 200 for i in range(39)], spare=1).write()
    b.check(b.attend())
    b.ctx.close()
