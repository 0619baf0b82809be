"""Moves of more rows than the L2 caches hold take other loads and stores than small ones: the same bits as the same tokens moved a
sequence at a time."""
import numpy as np
import pytest
import torch

from paper_2601_11589_amd import api, inputs

pytestmark = pytest.mark.gpu
STREAMED = 32 << 20      # bytes of K and V rows above which a call streams


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


@pytest.mark.parametrize("cfgf", [inputs.tiny_cfg, inputs.qwen7b_cfg])
def test_a_streamed_move_has_the_bits_of_small_ones(cfgf):
    cfg = cfgf(1)
    ctx, g = api.LapsCtx(cfg, 64), np.random.default_rng(9)
    row = cfg.n_kv_heads * cfg.head_dim * 2 * 2
    n = STREAMED // row + 1
    cuts = np.sort(g.choice(np.arange(1, n), 6, replace=False))
    lens = np.diff(np.concatenate([[0], cuts, [n]]))
    lens = np.concatenate([lens[:3], [0], lens[3:]])                       # one sequence without a token among them
    start = g.integers(0, 50, len(lens))
    assert lens.sum() * row > STREAMED and (lens * row <= STREAMED).all() and (start % 16 != 0).any()
    cu = np.concatenate([[0], np.cumsum(lens)])
    table, n_pages = inputs.make_page_table(3, lens + 1, start)
    gone = [(0, (start[0] + lens[0] // 2) // 16), (5, (start[5] + lens[5] - 1) // 16)]
    for s, p in gone:
        table[s, p] = -1
    gen = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.empty((n, cfg.n_kv_heads, cfg.head_dim), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=gen) for _ in range(2))
    k[::977, :, 3] = float("inf")
    stale = [torch.empty((n_pages,) + ctx.new_kv4_pools(1, 1)[0][0].shape[1:], dtype=torch.uint8, device="cuda").random_(0, 256, generator=gen)
             for _ in range(2)]
    d_cu, d_start, d_table = dev(cu), dev(start), dev(table)

    large = [p.clone() for p in stale]
    ctx.laps_kv4_scatter(d_cu, d_start, d_table, k, v, *large)
    small = [p.clone() for p in stale]
    for i in range(len(lens)):
        r = slice(int(cu[i]), int(cu[i + 1]))
        ctx.laps_kv4_scatter(dev([0, lens[i]]), dev(start[i:i + 1]), dev(table[i:i + 1]), k[r].contiguous(), v[r].contiguous(), *small)
    torch.cuda.synchronize()
    for a, b, was in zip(large, small, stale):
        assert torch.equal(a, b) and not torch.equal(a, was)

    def filled(rows):
        return [torch.full((rows, cfg.n_kv_heads, cfg.head_dim), 776.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    back = ctx.laps_kv4_gather(d_cu, d_start, d_table, *large, n + 40, *filled(n + 40))     # 40 rows behind the last sequence
    for i in range(len(lens)):
        r = slice(int(cu[i]), int(cu[i + 1]))
        one = ctx.laps_kv4_gather(dev([0, lens[i]]), dev(start[i:i + 1]), dev(table[i:i + 1]), *large, int(lens[i]), *filled(int(lens[i])))
        for a, b in zip(back, one):
            assert torch.equal(a[r].view(torch.int16), b.view(torch.int16))
    pos = np.concatenate([np.arange(s, s + m) for s, m in zip(start, lens)])
    seq = np.repeat(np.arange(len(lens)), lens)
    unset = torch.from_numpy(table[seq, pos // 16] < 0).cuda()
    assert bool(unset.any()) and not bool(unset.all())
    for a in back:
        kept = (a == 776.0).all(-1).all(-1)
        assert bool(kept[n:].all()) and torch.equal(kept[:n], unset)
    ctx.close()
