"""How many pages the pools hold (laps_ctx_set_pool_pages and its 4-bit counterpart) is a property of each call's own pools: a
captured graph keeps that of its capture, and pools of another size in the same context change nothing for it."""
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


def raw_gather(ctx, table, kp, vp, n):
    """laps_kv_gather of n tokens without the binding, which would say how many pages there are."""
    cfg = ctx.cfg
    k, v = (torch.full((n, cfg.n_kv_heads, cfg.head_dim), 3.25, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    p = lambda t: C.c_void_p(t.data_ptr())
    cu, start, table = dev([0, n]), dev([0]), dev(table)
    assert api.lib().laps_kv_gather(ctx._h, C.c_int32(1), C.c_int32(n), p(cu), p(start), p(table), C.c_int32(table.shape[1]), p(kp), p(vp),
                                    p(k), p(v), None) == 0
    torch.cuda.synchronize()
    return k, v


def test_4bit_calls_leave_the_bf16_count_alone():
    cfg = inputs.tiny_cfg(1)
    ctx = api.LapsCtx(cfg, 64)
    kp, vp = ctx.new_pools(8, 1, zero=True)
    table = [[6, 3, 7]]
    assert api.lib().laps_ctx_set_pool_pages(ctx._h, C.c_int32(7)) == 0
    write_4bit_pools(ctx, 2)
    for got in raw_gather(ctx, table, kp[0], vp[0], 48):
        assert bool((got[:32] == 0).all()) and bool((got[32:] == 3.25).all())      # pages 6 and 3 are inside 7 pages, 7 is not
    write_4bit_pools(ctx, 90)
    for got in raw_gather(ctx, table, kp[0], vp[0], 48):
        assert bool((got[:32] == 0).all()) and bool((got[32:] == 3.25).all())
    ctx.close()


def test_the_4bit_count_guards_4bit_calls_and_falls_back_to_the_other():
    """Without the binding: a token on page 5 of 8 is written where the count in force says that there is such a page."""
    cfg = inputs.tiny_cfg(1)
    ctx = api.LapsCtx(cfg, 64)
    L, p = api.lib(), lambda t: t.data_ptr()
    x = torch.ones((1, cfg.n_kv_heads, cfg.head_dim), dtype=torch.bfloat16, device="cuda")
    cu, start, table = dev([0, 1]), dev([0]), dev([[5]])
    for bf16_pages, kv4_pages, written in ((0, 0, True), (5, 0, False), (6, 0, True), (5, 6, True), (8, 5, False), (5, 8, True), (0, 5, False)):
        assert L.laps_ctx_set_pool_pages(ctx._h, C.c_int32(bf16_pages)) == 0 and L.laps_ctx_set_kv4_pool_pages(ctx._h, kv4_pages) == 0
        k4, v4 = ctx.new_kv4_pools(8, 1, zero=True)
        assert L.laps_kv4_scatter(ctx._h, 1, 1, p(cu), p(start), p(table), 1, p(x), p(x), p(k4[0]), p(v4[0]), None) == 0
        torch.cuda.synchronize()
        for pool in (k4[0], v4[0]):
            assert bool(pool[5].any()) == written and not bool(pool[:5].any()) and not bool(pool[6:].any()), (bf16_pages, kv4_pages)
    assert L.laps_ctx_set_kv4_pool_pages(ctx._h, -1) == -1 and b"kv4_pool_pages" in L.laps_last_error()
    ctx.close()
