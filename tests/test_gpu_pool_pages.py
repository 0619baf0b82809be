"""How many pages the pools hold (laps_ctx_set_pool_pages) is a property of each call's own pools: a captured graph keeps that of its
capture, whatever pools of another size the same context is given afterwards."""
import ctypes as C

import numpy as np
import pytest
import torch

from gpu_harness import Case
from paper_2601_11589_amd import api, inputs

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def write_4bit_pools(ctx, n_pages):
    """One token into the last of n_pages 4-bit pages."""
    cfg = ctx.cfg
    x = torch.ones((1, cfg.n_kv_heads, cfg.head_dim), dtype=torch.bfloat16, device="cuda")
    k4, v4 = ctx.new_kv4_pools(n_pages, 1, zero=True)
    ctx.laps_kv4_scatter(dev([0, 1]), dev([0]), dev([[n_pages - 1]]), x, x, k4[0], v4[0])
    assert bool(k4[0][n_pages - 1].any())


@pytest.mark.parametrize("between", ["fewer 4-bit pages", "more 4-bit pages", "another count set"])
def test_a_graph_keeps_the_page_count_of_its_capture(between):
    """Two sequences whose new tokens lie on the last pages, one of them listing a page past the pools.  The pools are the first
    part of larger tensors, so that such a page is memory of this test whatever the count says."""
    cfg = inputs.tiny_cfg(2)
    ctx = api.LapsCtx(cfg, 256)
    case = Case(cfg, [5, 9], [36, 20], 11)
    n = case.n_pages
    case.to_device(ctx)
    large = [torch.full((2 * n + 4,) + tuple(p.shape[1:]), 776.0, dtype=p.dtype, device="cuda") for p in case.k_pools + case.v_pools]
    for big, pool in zip(large, case.k_pools + case.v_pools):
        big[:n] = pool
    pools = [big[:n] for big in large]
    k_pools, v_pools = pools[:cfg.n_layers], pools[cfg.n_layers:]
    start = [big.clone() for big in large]
    table = case.page_table.copy()
    assert table[0, 2] >= 0 and table[1, 1] >= 0
    table[1, 1] = n + 2                                  # of both the cached and the new tokens, past the pools
    stream = torch.cuda.Stream()
    graph = ctx.laps_graph_capture(case.dev_layers, 16, 2, table.shape[1], k_pools, v_pools, stream)
    stream.synchronize()

    def replay():
        for big, was in zip(large, start):
            big.copy_(was)
        out = torch.zeros((case.T, cfg.hidden), device="cuda")
        lens, pre, t = dev(case.new_len), dev(case.prefix_len), dev(table)
        torch.cuda.synchronize()
        graph.laps_graph_stage(2, lens, pre, t, case.d_x, stream)
        graph.laps_graph_replay(stream)
        graph.laps_graph_read_output(case.T, out, stream)
        torch.cuda.synchronize()
        return out, [big.clone() for big in large]

    out, after = replay()
    new = table[0, 2]                                    # positions 36..40 of sequence 0: offsets 4..8 of its third page
    assert bool(torch.isfinite(out[:5]).all())
    for got, was in zip(after, start):
        assert torch.equal(got[n:], was[n:])             # nothing past the pools
    for got in after[:cfg.n_layers]:
        assert bool(torch.isfinite(got[new, :, 4:9].float()).all())
    if between == "another count set":
        assert api.lib().laps_ctx_set_pool_pages(ctx._h, C.c_int32(1)) == 0
    else:
        write_4bit_pools(ctx, 1 if between.startswith("fewer") else 2 * n + 4)
    for _ in range(2):
        again, pools_again = replay()
        assert torch.equal(out[:5], again[:5])
        for got, want in zip(pools_again, after):
            assert torch.equal(got.view(torch.int16), want.view(torch.int16))
    graph.close()
    ctx.close()
