"""4-bit calls on a stream of their own with arguments that the caller drops at once: their memory is nobody else's before the
stream has done the work."""
import types

import numpy as np
import pytest
import torch

from paper_2601_11589_amd import api, inputs

pytestmark = pytest.mark.gpu
CFG = inputs.tiny_cfg(1)
NEW, PRE = [3, 1, 6], [40, 0, 200]


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def arguments(ctx):
    need = [-(-(n + p) // 16) for n, p in zip(NEW, PRE)]
    table, at = np.full((3, max(need)), -1), 0
    for i, m in enumerate(need):
        table[i, :m] = np.arange(at, at + m)[::-1]
        at += m
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    k4, v4 = ctx.new_kv4_pools(at, 1, zero=True)
    total = sum(NEW)
    return types.SimpleNamespace(cu=dev([0, 3, 4, 10]), pre=dev(PRE), lens=dev(NEW), table=dev(table), k4=k4[0], v4=v4[0], total=total,
                                 k=rows(total, CFG.n_kv_heads, CFG.head_dim), v=rows(total, CFG.n_kv_heads, CFG.head_dim),
                                 q=rows(total, CFG.n_q_heads * CFG.head_dim), out=rows(total, CFG.n_q_heads * CFG.head_dim))


CALLS = {
    "scatter": (("cu", "pre", "table", "k", "v", "k4", "v4"),
                lambda ctx, a, s: ctx.laps_kv4_scatter(a.cu, a.pre, a.table, a.k, a.v, a.k4, a.v4, stream=s)),
    "gather": (("cu", "pre", "table", "k4", "v4", "k", "v"),
               lambda ctx, a, s: ctx.laps_kv4_gather(a.cu, a.pre, a.table, a.k4, a.v4, a.total, a.k, a.v, stream=s)),
    "attention": (("cu", "lens", "pre", "table", "k4", "v4", "q", "out"),
                  lambda ctx, a, s: ctx.laps_attention_kv4(a.cu, a.lens, a.pre, a.table, a.k4, a.v4, a.q, a.out, stream=s)),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_dropped_arguments_are_not_handed_out_again(name):
    ctx, side = api.LapsCtx(CFG, 64), torch.cuda.Stream()
    big = torch.zeros((8192, 8192), dtype=torch.bfloat16, device="cuda")
    torch.mm(big, big)
    torch.cuda.synchronize()
    names, call = CALLS[name]
    a = arguments(ctx)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(60):                               # some 50 ms of work ahead of the call
            busy = torch.mm(big, big)
    call(ctx, a, side)
    sizes = [(n, getattr(a, n).untyped_storage().nbytes(), getattr(a, n).data_ptr()) for n in names]
    del a
    fresh = [torch.empty(size, dtype=torch.uint8, device="cuda") for _, size, _ in sizes for _ in range(4)]
    assert not side.query(), "the stream was to be busy"
    taken = {t.data_ptr() for t in fresh}
    assert not [n for n, _, at in sizes if at in taken]
    side.synchronize()
    del busy
    ctx.close()


def test_a_captured_step_on_a_forked_stream_with_dropped_arguments():
    """Inside one capture: copies of the inputs, the calls on a second stream, the copies dropped, and memory of the same sizes filled on
    the first one before the two join."""
    ctx, side = api.LapsCtx(CFG, 64), torch.cuda.Stream()
    a = arguments(ctx)
    ctx.laps_kv4_scatter(a.cu, a.pre, a.table, a.k, a.v, a.k4, a.v4)
    ctx.laps_attention_kv4(a.cu, a.lens, a.pre, a.table, a.k4, a.v4, a.q)
    names = ("cu", "lens", "pre", "table", "k", "v", "q")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = types.SimpleNamespace(**{n: getattr(a, n).clone() for n in names})
        ctx.laps_kv4_scatter(c.cu, c.pre, c.table, c.k, c.v, a.k4, a.v4, stream=side)
        out = ctx.laps_attention_kv4(c.cu, c.lens, c.pre, c.table, a.k4, a.v4, c.q, stream=side)
        del c
        over = [torch.full_like(getattr(a, n), 3) for n in names for _ in range(2)]
        torch.cuda.current_stream().wait_stream(side)
    g = torch.Generator(device="cuda").manual_seed(3)
    for _ in range(5):
        for t in (a.k, a.v, a.q):
            t.normal_(0, 1, generator=g)
        graph.replay()
        torch.cuda.synchronize()
        pools = a.k4.clone(), a.v4.clone()
        ctx.laps_kv4_scatter(a.cu, a.pre, a.table, a.k, a.v, a.k4, a.v4)
        want = ctx.laps_attention_kv4(a.cu, a.lens, a.pre, a.table, a.k4, a.v4, a.q)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(pools[0], a.k4) and torch.equal(pools[1], a.v4)
        assert all(bool((t == 3).all()) for t in over) and bool(want.any())
    ctx.close()
