"""laps_kv8_scatter / laps_kv8_gather bit for bit against the definition, laps_attention_kv8 element by element against it in 64 bits,
and the three together as a server would call them."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import fp8_oracle as O
from oracle.kv4_oracle import attend
from paper_2601_11589_amd import api, inputs

pytestmark = pytest.mark.gpu
ULP = 2.0 ** -8      # half a step of bf16, relative


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def bf16(g, shape):
    return torch.from_numpy(g.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)


def wide(t):
    return t.double().cpu().numpy()


class Batch:
    """New tokens and cached ones of a few sequences over random pages, on the host and in 8-bit pools full of stale bytes.  pk, pv: what
    the pools hold by the definition."""

    def __init__(self, cfg, new, pre, seed=1, spare=2, pad=None, ctx=None):
        self.cfg, self.new, self.pre = cfg, np.asarray(new), np.asarray(pre)
        self.g = g = np.random.default_rng(seed)
        self.rows = self.new + (0 if pad is None else np.asarray(pad))
        self.cu = np.concatenate([[0], np.cumsum(self.rows)]).astype(np.int32)
        need = -(-(self.new + self.pre) // 16)
        n_pages = int(need.sum()) + 3
        order = g.permutation(n_pages)
        self.table = np.full((len(self.new), int(need.max()) + spare), -1, np.int32)
        at = 0
        for i, m in enumerate(need):
            self.table[i, :m] = order[at:at + m]
            at += m
        self.ctx = ctx or api.LapsCtx(cfg, 64)
        shape = (n_pages, O.page_bytes(cfg.n_kv_heads, cfg.head_dim))
        self.pk, self.pv = (g.integers(0, 256, shape).astype(np.uint8) for _ in range(2))
        self.k8, self.v8 = (torch.from_numpy(p.copy()).cuda() for p in (self.pk, self.pv))
        total = int((self.new + self.pre).sum())
        self.k, self.v = (bf16(g, (total, cfg.n_kv_heads, cfg.head_dim)) for _ in range(2))
        self.first = np.concatenate([[0], np.cumsum(self.new + self.pre)])
        self.q = bf16(g, (int(self.rows.sum()), cfg.n_q_heads * cfg.head_dim))

    def write(self, which="all"):
        """All tokens, the cached ones or the new ones into the pools, through the library and by the definition."""
        lo = self.pre if which == "new" else np.zeros_like(self.pre)
        n = {"all": self.new + self.pre, "new": self.new, "cached": self.pre}[which]
        at = np.concatenate([np.arange(f + a, f + a + m) for f, a, m in zip(self.first, lo, n)]).astype(np.int64)
        self.ctx.laps_kv8_scatter(dev(np.concatenate([[0], np.cumsum(n)])), dev(lo), dev(self.table), self.k[at].cuda(), self.v[at].cuda(),
                                  self.k8, self.v8)
        for i, (a, m) in enumerate(zip(lo, n)):
            span = slice(self.first[i] + a, self.first[i] + a + m)
            O.write_run(self.pk, self.table[i], int(a), wide(self.k[span]), False)
            O.write_run(self.pv, self.table[i], int(a), wide(self.v[span]), True)
        return self

    def attend(self, out=None, stream=None):
        seq_len = dev(self.new) if (self.rows != self.new).any() else None
        return self.ctx.laps_attention_kv8(dev(self.cu), seq_len, dev(self.pre), dev(self.table), self.k8, self.v8, self.q.cuda(), out, stream)

    def oracle(self):
        n_q, n_kv, hd = self.cfg.n_q_heads, self.cfg.n_kv_heads, self.cfg.head_dim
        out, spread = (np.zeros((len(self.q), n_q, hd)) for _ in range(2))
        bound = np.zeros((len(self.q), 1, 1))
        for i, (n, h) in enumerate(zip(self.new, self.pre)):
            if n == 0:
                continue
            k, v = (O.read_run(p, self.table[i], 0, int(n + h), n_kv, hd, t) for p, t in ((self.pk, False), (self.pv, True)))
            r = slice(self.cu[i], self.cu[i] + n)
            q = wide(self.q[r]).reshape(n, n_q, -1)
            out[r], spread[r] = attend(q, k, v, int(h))
            # largest sum |q k| of a score: what its float32 sum is off by, in units of 2^-24 a term
            bound[r] = np.abs(q).max() * np.nanmax(np.abs(k).sum(-1)) * math.sqrt(hd)
        return out, spread, bound

    def check(self, got, oracle=None):
        """|got - out| <= ULP (sum p|v| + 2 |out|): the weights p, their sum (it may be that of the rounded ones) and the output are
        rounded to bf16; and a float32 term: a score
        is off by hd terms of 2^-24, an exponential and the sums by less than 2^-20, which moves the weights by as much."""
        out, spread, bound = self.oracle() if oracle is None else oracle
        got = wide(got).reshape(out.shape)
        live = np.concatenate([np.arange(c, c + n) for c, n in zip(self.cu, self.new)]).astype(int)
        slack = ULP * (spread + 2 * np.abs(out)) * (1 + 4 * ULP) + 4 * spread * (bound * 2.0 ** -24 + 2.0 ** -20)
        with np.errstate(invalid="ignore"):
            bad = ~(np.abs(got - out) <= slack) & ~(np.isnan(got) & np.isnan(out))
        assert not bad[live].any(), (np.argwhere(bad[live])[:4], got[live][bad[live]][:4], out[live][bad[live]][:4])
        return live


# ------------------------------------------------------------------------------------------------ scatter, gather
def odd_values(g, shape):
    """Tokens of every size of exponent, with zeros, subnormals, the largest values, infinities and NaN among them."""
    bits = g.integers(0, 1 << 16, shape).astype(np.uint16)
    spread = inputs.f32_to_bf16_bits((g.standard_normal(shape) * np.exp2(g.integers(-20, 20, shape[:-1] + (1,)))).astype(np.float32))
    kind = np.repeat(g.integers(0, 5, shape[:-1] + (1,)), shape[-1], -1)
    bits = np.where(kind == 0, bits, np.where(kind == 1, spread, np.where(kind == 2, bits & 0x80ff, np.where(kind == 3, (bits & 0x807f) | 0x7f00, bits & 0xbfff))))
    return torch.from_numpy(bits.astype(np.uint16).view(np.int16)).view(torch.bfloat16)


def same_page(got, want, n_kv, hd):
    """Pages byte for byte; a NaN's sign and the padding behind the scales apart."""
    end = n_kv * 16 * hd
    nan = (want[:, :end] & 127) == 127
    assert np.array_equal((got[:, :end] & 127) == 127, nan)
    assert np.array_equal(np.where(nan, 0, got[:, :end]), np.where(nan, 0, want[:, :end]))
    assert np.array_equal(got[:, end:], want[:, end:])


@pytest.mark.parametrize("cfgf", [inputs.tiny_cfg, inputs.qwen7b_cfg])
@pytest.mark.parametrize("lens,start", [([1], [15]), ([1], [0]), ([16, 16], [0, 32]), ([17, 0, 3, 40, 1], [5, 9, 14, 31, 0]),
                                        ([0, 33, 100, 7], [3, 1, 16, 2000]), ([0], [0])])
def test_pools_hold_the_definition_and_read_back(lens, start, cfgf):
    cfg = cfgf(1)
    ctx = api.LapsCtx(cfg, 64)
    n, rows, g = len(lens), sum(lens), np.random.default_rng(sum(lens) * 7 + 1)
    n_kv, hd = cfg.n_kv_heads, cfg.head_dim
    table, n_pages = inputs.make_page_table(3, np.asarray(lens) + 1, np.asarray(start))
    if n > 1:
        table[n - 1, start[n - 1] // 16] = -1                              # unset entry: these tokens are not moved
    cu = np.concatenate([[0], np.cumsum(lens)])
    pk, pv = (g.integers(0, 256, (n_pages, O.page_bytes(n_kv, hd))).astype(np.uint8) for _ in range(2))
    k8, v8 = (torch.from_numpy(p.copy()).cuda() for p in (pk, pv))
    for turn in range(3):                                                  # the same places three times: what is kept is rounded again and again
        k, v = (odd_values(g, (rows, n_kv, hd)) for _ in range(2))
        if turn == 1:
            k, v = ((t.float() * 2.0 ** -9).to(torch.bfloat16) for t in (k, v))     # scales that stay
        for i in range(n):
            O.write_run(pk, table[i], start[i], wide(k)[cu[i]:cu[i + 1]], False)
            O.write_run(pv, table[i], start[i], wide(v)[cu[i]:cu[i + 1]], True)
        ctx.laps_kv8_scatter(dev(cu), dev(start), dev(table), k.cuda(), v.cuda(), k8, v8)
        same_page(k8.cpu().numpy(), pk, n_kv, hd)
        same_page(v8.cpu().numpy(), pv, n_kv, hd)
    outs = [torch.full((rows, n_kv, hd), 3.25, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    back = ctx.laps_kv8_gather(dev(cu), dev(start), dev(table), k8, v8, rows, *outs)
    for i, (got, p) in enumerate(zip(back, (pk, pv))):
        assert got is outs[i]
        for s in range(n):
            for t in range(lens[s]):
                page = table[s, (start[s] + t) // 16]
                want = O.read(p, page, n_kv, hd, i == 1)[(start[s] + t) % 16] if page >= 0 else np.full((n_kv, hd), 3.25)
                assert np.array_equal(wide(got[cu[s] + t]), want, equal_nan=True)
    ctx.close()


def test_every_bf16_value_as_a_page_of_its_own():
    cfg = inputs.tiny_cfg(1)
    ctx, hd = api.LapsCtx(cfg, 64), cfg.head_dim
    bits = np.arange(1 << 15).astype(np.uint16)
    x = np.zeros((1 << 15, cfg.n_kv_heads, hd), np.uint16)                 # a token a page, one value sets the scale
    x[:, 0, 5] = bits
    x[:, 1, 63] = bits | 0x8000
    x[:, :, 6:60] = np.clip(bits[:, None, None].astype(int) - np.arange(54) * 23, 0, 0x7fff)      # smaller ones beside it
    x = torch.from_numpy(x.view(np.int16)).view(torch.bfloat16)
    n = x.shape[0]
    table = dev(np.arange(n)[:, None])
    k8, v8 = ctx.new_kv8_pools(n, 1)
    one = dev(np.arange(n + 1)), dev(np.zeros(n))
    ctx.laps_kv8_scatter(*one, table, x.cuda(), x.flip(0).contiguous().cuda(), k8[0], v8[0])
    k, v = ctx.laps_kv8_gather(*one, table, k8[0], v8[0], n)
    w = wide(x)
    w[~np.isfinite(w).all(-1)] = np.nan
    top = np.nan_to_num(np.abs(w).max(-1))
    e = np.clip(np.ceil(np.log2(np.maximum(top, 1e-300) / 448)), O.LOWEST, O.HIGHEST)
    e = np.where(top > 448 * np.exp2(e), np.minimum(e + 1, O.HIGHEST), e)
    want = O.decode(O.encode(w * np.exp2(-e)[..., None], 0), 0) * np.exp2(e)[..., None]
    assert np.array_equal(wide(k), want, equal_nan=True) and np.array_equal(wide(v.flip(0)), want, equal_nan=True)
    ctx.close()


def test_large_moves_are_the_bits_of_small_ones():
    """Above 32 MiB rows stream past the caches."""
    cfg = inputs.qwen14b_cfg(1)
    ctx, n = api.LapsCtx(cfg, 64), 9003
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.empty((n, cfg.n_kv_heads, cfg.head_dim), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g) for _ in range(2))
    table = dev(np.random.default_rng(1).permutation(-(-n // 16))[None])
    whole, parts = (ctx.new_kv8_pools(table.shape[1], 1, zero=True) for _ in range(2))
    ctx.laps_kv8_scatter(dev([0, n]), dev([0]), table, k, v, whole[0][0], whole[1][0])
    for lo in range(0, n, 3200):
        hi = min(n, lo + 3200)
        ctx.laps_kv8_scatter(dev([0, hi - lo]), dev([lo]), table, k[lo:hi], v[lo:hi], parts[0][0], parts[1][0])
    assert torch.equal(whole[0][0], parts[0][0]) and torch.equal(whole[1][0], parts[1][0])
    rk, rv = ctx.laps_kv8_gather(dev([0, n]), dev([0]), table, whole[0][0], whole[1][0], n)
    for lo in range(0, n, 3200):
        hi = min(n, lo + 3200)
        pk, pv = ctx.laps_kv8_gather(dev([0, hi - lo]), dev([lo]), table, whole[0][0], whole[1][0], hi - lo)
        assert torch.equal(pk, rk[lo:hi]) and torch.equal(pv, rv[lo:hi])
    assert ((rk.float() - k.float()).abs() <= k.float().abs() * 2.0 ** -4 + 2.0 ** -14).all()
    ctx.close()


# ------------------------------------------------------------------------------------------------ attention
SHAPES = [
    ([1], [0]), ([1], [1]), ([1], [31]), ([1], [127]), ([1], [4001]),                 # a token with more and more behind it
    ([1] * 9, [0, 15, 16, 17, 300, 1000, 64, 2047, 5]),                               # a decode batch
    ([3, 0, 1, 5, 2], [0, 7, 500, 33, 1111]),                                         # drafted tokens, one sequence without any
    ([2], [40]), ([17], [0]), ([16], [1000]), ([33, 1, 64], [100, 3000, 0]),          # short turns
    ([130], [0]), ([257, 40], [70, 900]), ([0, 0, 1], [5, 0, 9]),
]


@pytest.mark.parametrize("cfgf", [inputs.tiny_cfg, inputs.qwen7b_cfg, inputs.qwen14b_cfg])
@pytest.mark.parametrize("new,pre", SHAPES)
def test_attention_matches_the_definition(new, pre, cfgf):
    b = Batch(cfgf(1), new, pre, seed=sum(new) + sum(pre)).write("cached").write("new")
    b.check(b.attend())
    b.ctx.close()


@pytest.mark.parametrize("spare", [0, 1, 60, 700])
def test_width_of_the_page_table(spare):
    b = Batch(inputs.qwen7b_cfg(1), [1, 1, 4], [900, 3, 2500], spare=spare).write()
    b.check(b.attend())
    b.ctx.close()


@pytest.mark.parametrize("heads", [(8, 8, 64), (1, 1, 128), (16, 1, 128), (34, 2, 64), (6, 2, 128), (10, 5, 64), (132, 132, 64)])
def test_head_layouts(heads):
    n_q, n_kv, hd = heads
    cfg = inputs.ModelCfg(256, n_q, n_kv, hd, 512, 1)
    b = Batch(cfg, [1, 2, 19], [700 if n_kv < 100 else 60, 33, 150], seed=n_q).write()
    b.check(b.attend())
    b.ctx.close()


# Blocks of 32 rows that share keys, dealt to the XCDs in groups where (sequence, part, kv head) are few: 1 unit, 2, 3, 8 and many, blocks that
# fill their groups and that do not
@pytest.mark.parametrize("heads,new,pre", [((16, 1, 128), [100], [300]), ((16, 1, 128), [33, 70, 2], [5, 900, 64]), ((4, 2, 64), [200], [100]),
                                           ((40, 8, 128), [90], [2500]), ((28, 4, 128), [5] * 9, [100, 0, 700, 64, 65, 31, 32, 33, 1]),
                                           ((40, 8, 128), [13, 1, 40, 0, 7, 22, 9], [70, 300, 0, 5, 1900, 16, 15]),
                                           ((28, 4, 128), [1] * 20 + [90], list(range(0, 420, 20)))])      # one turn of many times the mean
def test_row_blocks_of_the_same_keys(heads, new, pre):
    n_q, n_kv, hd = heads
    b = Batch(inputs.ModelCfg(256, n_q, n_kv, hd, 512, 1), new, pre, spare=3, seed=n_q + len(new)).write()
    p = plan(b)
    assert p[0] == 32 and p[1] > 1, p
    b.check(b.attend())
    b.ctx.close()


# Batches large enough for the kernels of 128 and 256 rows, 64 query heads over 8: (new, prefix, spare pages, rows a workgroup, shares)
BLOCKS = {
    "shares": ([300, 40, 260], [1500, 200, 0], 2, 256, True),
    "shares_wide_table": ([520, 1, 0, 77], [0, 3000, 5, 1100], 300, 256, True),
    "grid_of_256": ([400, 300], [100, 0], 0, 256, False),
    "one_prompt": ([600], [0], 2, 256, False),
    "halves": ([48] * 11 + [47], [70, 0, 150, 3, 64, 16, 15, 17, 100, 31, 1, 128], 0, 128, False),
    "one_tile": ([9] * 70 + [1, 0], [7] * 72, 0, 128, False),
    "plain": ([16] * 39 + [3], [30, 0, 200, 64] * 10, 0, 128, False),
}


def big_cfg(hd):
    return inputs.ModelCfg(256, 64, 8, hd, 512, 1)


def plan(b):
    out = (C.c_int64 * 6)()
    assert api.lib().laps_attention_kv8_plan_info(C.c_int32(len(b.new)), C.c_int32(len(b.q)), C.c_int32(b.cfg.n_q_heads),
                                                  C.c_int32(b.cfg.n_kv_heads), C.c_int32(b.cfg.head_dim), C.c_int32(b.table.shape[1]), out) == 0
    return list(out)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name", sorted(BLOCKS))
def test_blocks_match_the_definition(name, hd):
    new, pre, spare, rows, shares = BLOCKS[name]
    b = Batch(big_cfg(hd), new, pre, spare=spare, seed=hd).write()
    p = plan(b)
    assert p[0] == rows and (p[4] > 0) == shares, p
    b.check(b.attend())
    b.ctx.close()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("name,at", [("shares", 1700), ("shares", 1499), ("shares", 3), ("grid_of_256", 330), ("halves", 70), ("plain", 33)])
def test_a_nan_in_blocks_reaches_the_rows_that_see_it(name, at, hd):
    new, pre, spare, rows, _ = BLOCKS[name]
    for which in ("v", "k"):
        b = Batch(big_cfg(hd), new, pre, spare=spare, seed=at)
        (b.v if which == "v" else b.k)[at, 1, 37] = math.nan
        b.write()
        assert plan(b)[0] == rows
        want = b.oracle()
        assert np.isnan(want[0]).any() and not np.isnan(want[0]).all()
        b.check(b.attend(), want)
        b.ctx.close()


@pytest.mark.parametrize("name,rows", [("shares", 256), ("halves", 256), ("plain", 128)])     # by all rows, padding among them
def test_rows_without_a_token_stay_in_blocks(name, rows):
    new, pre, spare, _, _ = BLOCKS[name]
    b = Batch(big_cfg(128), new, pre, spare=spare, pad=[(3 * i) % 5 for i in range(len(new))]).write()
    assert plan(b)[0] == rows
    out = torch.full(b.q.shape, 7.5, dtype=torch.bfloat16, device="cuda")
    live = b.check(b.attend(out))
    rest = np.setdiff1d(np.arange(len(b.q)), live)
    assert len(rest) > 0 and (out[torch.from_numpy(rest).cuda()] == 7.5).all()
    b.ctx.close()


# Decode batches with one turn that a workgroup walks block after block: (heads, tokens of each sequence, rows of a block)
@pytest.mark.parametrize("heads,new,rows", [((4, 2, 64), [1] * 70 + [450], 16), ((28, 4, 128), [1] * 40 + [150] + [1] * 79, 16),
                                            ((40, 8, 128), [350] + [1] * 95, 32), ((28, 4, 128), [1] * 30 + [300, 0] + [1] * 29, 32)])
def test_single_tokens_and_one_long_turn(heads, new, rows):
    n_q, n_kv, hd = heads
    g = np.random.default_rng(len(new))
    pre = np.where(np.asarray(new) > 1, 333, g.integers(0, 120, len(new)))
    b = Batch(inputs.ModelCfg(256, n_q, n_kv, hd, 512, 1), new, pre, spare=3, seed=len(new)).write()
    p = plan(b)
    assert p[0] == rows and p[1] * rows < max(new) * n_q // n_kv, p
    b.check(b.attend())
    b.ctx.close()


def test_many_sequences():
    g = np.random.default_rng(8)
    b = Batch(inputs.tiny_cfg(1), g.integers(0, 3, 700), g.integers(0, 90, 700)).write()
    b.check(b.attend())
    b.ctx.close()


@pytest.mark.parametrize("cfgf", [inputs.tiny_cfg, inputs.qwen14b_cfg])
@pytest.mark.parametrize("new,pre,pad", [([3, 0, 1, 20], [50, 9, 400, 0], [2, 3, 0, 1]), ([1, 1], [5, 2000], [7, 1]), ([0, 0], [4, 0], [1, 3])])
def test_rows_without_a_token_stay(new, pre, pad, cfgf):
    b = Batch(cfgf(1), new, pre, pad=pad).write()
    out = torch.full((len(b.q) + 5, b.q.shape[1]), 7.5, dtype=torch.bfloat16, device="cuda")
    b.q = torch.cat([b.q, b.q[:1].expand(5, -1)])       # and rows behind the last sequence
    live = b.check(b.attend(out))
    rest = np.setdiff1d(np.arange(len(b.q)), live)
    assert (out[torch.from_numpy(rest).cuda()] == 7.5).all()
    b.ctx.close()


@pytest.mark.parametrize("cfgf", [inputs.tiny_cfg, inputs.qwen7b_cfg])
@pytest.mark.parametrize("new,pre,at", [([1, 1], [40, 900], 17), ([1, 1], [900, 700], 899), ([6, 3], [70, 40], 72), ([40, 20], [100, 9], 103),
                                        ([200, 150], [30, 0], 110), ([6, 3], [70, 40], 0)])
def test_a_nan_reaches_the_rows_that_see_it(new, pre, at, cfgf):
    """V, then K of key `at` of the first sequence not finite in one head: a page whose other tokens are as they would be without it."""
    for which in ("v", "k"):
        b = Batch(cfgf(1), new, pre, seed=at)
        (b.v if which == "v" else b.k)[at, 1, 37] = math.inf
        b.write()
        want = b.oracle()
        assert np.isnan(want[0]).any() and not np.isnan(want[0]).all()
        b.check(b.attend(), want)
        b.ctx.close()


def test_scores_far_apart_and_all_equal():
    cfg = inputs.qwen7b_cfg(1)
    for scale in (0.0, 30.0, 1e-30):
        b = Batch(cfg, [1, 2, 70], [1500, 33, 200])
        b.q = (b.q.float() * scale).to(torch.bfloat16)
        b.write()
        b.check(b.attend())
        b.ctx.close()


@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** 60])
def test_caches_of_tiny_and_huge_values(size):
    b = Batch(inputs.qwen7b_cfg(1), [1, 40], [700, 90])
    b.v = (b.v.float() * size).to(torch.bfloat16)
    b.k = (b.k.float() * 2.0 ** 30).to(torch.bfloat16)
    b.q = (b.q.float() * 2.0 ** -30).to(torch.bfloat16)
    b.write()
    b.check(b.attend())
    b.ctx.close()


def test_a_value_follows_its_own_key():
    """Keys that only one row's query matches: the output is that key's value to the last bit (all else has weight 2^-100)."""
    cfg = inputs.tiny_cfg(1)
    b = Batch(cfg, [5], [300])
    b.k[:] = 0
    b.q[:] = 0
    for t in range(5):
        b.k[60 * t + 7, :, t] = 4.0
        b.q.view(5, cfg.n_q_heads, cfg.head_dim)[t, :, t] = 400.0
    got = wide(b.write().attend()).reshape(5, cfg.n_q_heads, cfg.head_dim)
    want = O.read_run(b.pv, b.table[0], 0, 305, cfg.n_kv_heads, cfg.head_dim, True)
    for t in range(5):
        for h in range(cfg.n_q_heads):
            assert np.array_equal(got[t, h], want[60 * t + 7, h // 2])
    b.ctx.close()


def test_unset_pages_read_page_zero_and_lengths_are_cut():
    """What stale arrays can reach: unset and out-of-range ids fall back to page 0, a length to the rows a sequence owns, a
    prefix to the table's width.  Nothing outside the arrays is touched; rows of whole sequences stay right."""
    b = Batch(inputs.qwen7b_cfg(1), [2, 3, 1], [100, 50, 60], spare=0).write()
    want = b.oracle()
    table = b.table.copy()
    table[0, 1], table[0, 2], table[0, 3] = -1, 1 << 30, -(1 << 31)
    out = b.ctx.laps_attention_kv8(dev(b.cu), dev([9, 3, 1]), dev([100, 50, 1 << 30]), dev(table), b.k8, b.v8, b.q.cuda())
    b.new = np.array([0, 3, 0])
    b.check(out, want)
    b.ctx.close()


def test_long_offsets():
    """Pages at the end of pools of more than 4 GiB, more than 2^16 keys."""
    cfg = inputs.qwen7b_cfg(1)
    ctx = api.LapsCtx(cfg, 64)
    n, pages = 70001, 1 << 19
    k8, v8 = ctx.new_kv8_pools(pages, 1, zero=True)
    assert k8[0].numel() > 1 << 32
    table = dev((pages - 1 - np.arange(-(-n // 16)))[None])
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.empty((n, cfg.n_kv_heads, cfg.head_dim), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g) for _ in range(2))
    q = torch.empty((1, cfg.n_q_heads * cfg.head_dim), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    ctx.laps_kv8_scatter(dev([0, n]), dev([0]), table, k, v, k8[0], v8[0])
    rk, rv = ctx.laps_kv8_gather(dev([0, n]), dev([0]), table, k8[0], v8[0], n)
    for got, x in ((rk, k), (rv, v)):
        assert ((got.float() - x.float()).abs() <= x.float().abs() * 2.0 ** -4 + 2.0 ** -14).all()
    out = ctx.laps_attention_kv8(dev([0, 1]), None, dev([n - 1]), table, k8[0], v8[0], q)
    want, spread = attend(wide(q).reshape(1, cfg.n_q_heads, -1), wide(rk), wide(rv), n - 1)
    err = np.abs(wide(out).reshape(want.shape) - want)
    assert (err <= ULP * (spread + 2 * np.abs(want)) * (1 + 4 * ULP) + spread * 2.0 ** -14).all()
    ctx.close()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("cfgf", [inputs.tiny_cfg, inputs.qwen7b_cfg])
def test_decode_steps_and_a_chunk(cfgf):
    """A prompt written and attended to as one chunk, then the same tokens one at a time, each written before it is attended to: what a
    server does.  Both against the definition of their own history of writes, the pools to the last byte."""
    cfg = cfgf(1)
    b = Batch(cfg, [37, 20], [13, 160])
    b.write("cached")
    start = b.k8.clone(), b.v8.clone(), b.pk.copy(), b.pv.copy()
    b.write("new")
    b.check(b.attend())
    b.k8.copy_(start[0]), b.v8.copy_(start[1])
    b.pk[:], b.pv[:] = start[2], start[3]
    new, pre = b.new.copy(), b.pre.copy()
    for t in range(37):
        on = [i for i in range(2) if t < new[i]]
        src = torch.tensor([b.first[i] + pre[i] + t for i in on])
        table, pos, cu = dev(b.table[on]), dev([pre[i] + t for i in on]), dev(np.arange(len(on) + 1))
        b.ctx.laps_kv8_scatter(cu, pos, table, b.k[src].cuda(), b.v[src].cuda(), b.k8, b.v8)
        out = b.ctx.laps_attention_kv8(cu, None, pos, table, b.k8, b.v8, b.q[[b.cu[i] + t for i in on]].cuda())
        for j, i in enumerate(on):
            O.write_run(b.pk, b.table[i], int(pre[i]) + t, wide(b.k[src[j:j + 1]]), False)
            O.write_run(b.pv, b.table[i], int(pre[i]) + t, wide(b.v[src[j:j + 1]]), True)
        if t in (0, 2, 3, 18, 19, 36):
            step = one_token_each(b, on, t, pre)
            step.check(out)
    same_page(b.k8.cpu().numpy(), b.pk, cfg.n_kv_heads, cfg.head_dim)
    same_page(b.v8.cpu().numpy(), b.pv, cfg.n_kv_heads, cfg.head_dim)
    b.ctx.close()


def one_token_each(b, on, t, pre):
    """The single tokens t of the sequences `on` as a batch over the same pools."""
    s = object.__new__(Batch)
    s.cfg, s.new, s.pre, s.cu, s.table = b.cfg, np.ones(len(on), int), np.array([pre[i] + t for i in on]), np.arange(len(on) + 1), b.table[on]
    s.pk, s.pv, s.q = b.pk, b.pv, b.q[[b.cu[i] + t for i in on]]
    return s


def test_prefill_cache_goes_on_in_eight_bits():
    """K/V of a bf16 pool (the prefill path's) through laps_kv_gather into 8-bit pools, attention of the next token over them,
    against attention over bf16 pools that hold the rounded values."""
    cfg = inputs.qwen7b_cfg(1)
    b = Batch(cfg, [1, 1], [75, 300])
    cu, zero = dev(b.first), dev([0, 0])
    kp, vp = b.ctx.new_pools(b.k8.shape[0], 1)
    b.ctx.laps_kv_scatter(cu, zero, dev(b.table), b.k.cuda(), b.v.cuda(), kp[0], vp[0])
    k, v = b.ctx.laps_kv_gather(cu, zero, dev(b.table), kp[0], vp[0], len(b.k))
    b.write()
    b.ctx.laps_kv8_scatter(cu, zero, dev(b.table), k, v, b.k8, b.v8)
    k, v = b.ctx.laps_kv8_gather(cu, zero, dev(b.table), b.k8, b.v8, len(b.k))
    b.ctx.laps_kv_scatter(cu, zero, dev(b.table), k, v, kp[0], vp[0])
    want = b.oracle()
    b.check(b.attend(), want)
    b.check(b.ctx.laps_attention(dev(b.cu), None, dev(b.pre), dev(b.table), kp[0], vp[0], b.q.cuda()), want)
    b.ctx.close()


# ------------------------------------------------------------------------------------------------ streams, graphs, refusals
@pytest.mark.parametrize("new,pre", [([1, 1, 1], [700, 20, 3000]), ([40, 30], [500, 900]), ([1300], [100])])
def test_captured_steps_replay_with_new_contents(new, pre):
    """Two graphs of one step each (write, attend), replayed in turns with other tokens, lengths and queries in between eager calls."""
    b = Batch(inputs.qwen7b_cfg(1), new, pre).write("cached")
    cu, table, n = dev(b.cu), dev(b.table), int(b.new.sum())
    prefix, q = dev(b.pre), b.q.cuda()
    at = np.concatenate([np.arange(f + p, f + p + m) for f, p, m in zip(b.first, b.pre, b.new)])
    k, v = b.k[at].cuda(), b.v[at].cuda()

    def step():
        b.ctx.laps_kv8_scatter(cu, prefix, table, k, v, b.k8, b.v8)
        return b.ctx.laps_attention_kv8(cu, None, prefix, table, b.k8, b.v8, q)

    step()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    g = torch.Generator(device="cuda").manual_seed(4)
    for turn in range(6):
        for t in (k, v, q):
            t.normal_(0, 1, generator=g)
        if turn == 3:
            prefix.sub_(9)
        graph, out = graphs[turn % 2]
        graph.replay()
        pools = b.k8.clone(), b.v8.clone()
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.isfinite(want.float()).all()
        assert torch.equal(pools[0], b.k8) and torch.equal(pools[1], b.v8)     # the same tokens once more change nothing
    b.ctx.close()


def test_two_streams_at_once():
    cfg = inputs.qwen7b_cfg(1)
    ctx = api.LapsCtx(cfg, 64)
    batches = [Batch(cfg, [1] * 6, [900, 40, 2000, 7, 100, 1500], seed=s, ctx=ctx).write() for s in (1, 2)]
    want = [b.attend() for b in batches]
    streams = [torch.cuda.Stream() for _ in batches]
    got = [[b.attend(stream=s) for b, s in zip(batches, streams)] for _ in range(8)]
    torch.cuda.synchronize()
    for round_ in got:
        assert all(torch.equal(a, b) for a, b in zip(round_, want))
    for b, w in zip(batches, want):
        b.check(w)
    ctx.close()


@pytest.mark.parametrize("n_new", [1, 3, 400])
def test_pages_that_sequences_share(n_new):
    """Two sequences over one prefix's pages, one of them with a page of it twice; written and read back on another stream."""
    cfg = inputs.qwen7b_cfg(1)
    b = Batch(cfg, [n_new, n_new], [320, 320])
    b.table[1, :20] = b.table[0, :20]
    b.table[1, 7] = b.table[1, 3]
    side = torch.cuda.Stream()
    at = np.concatenate([np.arange(320 + n_new), b.first[1] + np.arange(320, 320 + n_new)])   # the prefix once
    cu, start, table = dev([0, 320 + n_new, 320 + 2 * n_new]), dev([0, 320]), dev(b.table)
    b.ctx.laps_kv8_scatter(cu, start, table, b.k[at].cuda(), b.v[at].cuda(), b.k8, b.v8, stream=side)
    for i in range(2):
        span = slice(0, 320 + n_new) if i == 0 else slice(b.first[1] + 320, b.first[1] + 320 + n_new)
        O.write_run(b.pk, b.table[i], (0, 320)[i], wide(b.k[span]), False)
        O.write_run(b.pv, b.table[i], (0, 320)[i], wide(b.v[span]), True)
    rk, rv = b.ctx.laps_kv8_gather(dev([0, 320 + n_new, 640 + 2 * n_new]), dev([0, 0]), table, b.k8, b.v8, 640 + 2 * n_new, stream=side)
    got = b.attend(stream=side)
    side.synchronize()
    for p, r, v in ((b.pk, rk, False), (b.pv, rv, True)):
        want = np.concatenate([O.read_run(p, b.table[i], 0, 320 + n_new, cfg.n_kv_heads, cfg.head_dim, v) for i in range(2)])
        assert np.array_equal(wide(r), want)
    b.check(got)
    b.ctx.close()


def test_results_repeat_and_do_not_depend_on_the_batch():
    b = Batch(inputs.qwen14b_cfg(1), [1] * 5, [3000, 10, 700, 64, 1999]).write()
    out = b.attend()
    assert torch.equal(out, b.attend())
    moved = b.pre.copy()
    moved[[0, 3]] = [5, 2]                 # other sequences get shorter
    other = b.ctx.laps_attention_kv8(dev(b.cu), None, dev(moved), dev(b.table), b.k8, b.v8, b.q.cuda())
    assert torch.equal(out[[1, 2, 4]], other[[1, 2, 4]])
    b.ctx.close()


def test_refusals():
    cfg = inputs.qwen7b_cfg(1)
    b = Batch(cfg, [1, 2], [40, 9]).write()
    cu, pre, table, q = dev(b.cu), dev(b.pre), dev(b.table), b.q.cuda()
    x = torch.zeros((3, cfg.n_kv_heads, cfg.head_dim), dtype=torch.bfloat16, device="cuda")
    before = b.k8.clone(), b.v8.clone()

    def refused(f, *args, match, **kw):
        with pytest.raises(api.LapsError, match=match):
            f(*args, **kw)

    at, sc, ga = b.ctx.laps_attention_kv8, b.ctx.laps_kv8_scatter, b.ctx.laps_kv8_gather
    refused(at, cu, None, pre, table, b.k8, b.v8, q[:0], match="bad size")
    refused(at, cu.cpu(), None, pre, table, b.k8, b.v8, q, match="cu")
    refused(at, cu, None, pre, table, b.k8[:0], b.v8[:0], q, match="0 pages|NULL")
    odd = torch.zeros(x.numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view(x.shape)
    refused(sc, cu, pre, table, odd, x, b.k8, b.v8, match="aligned")
    refused(ga, cu, pre, table, b.k8, b.v8, 3, x, odd, match="aligned")
    odd_q = torch.zeros(q.numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view(q.shape)
    refused(at, cu, None, pre, table, b.k8, b.v8, odd_q, match="aligned")
    need = b.ctx.laps_attention_kv8_workspace_bytes(2, 3, table.shape[1])
    p = lambda t: t.data_ptr()
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    call = lambda w, n, pages, held: api.lib().laps_attention_kv8(b.ctx._h, 2, 3, p(cu), None, p(pre), p(table), pages, held, p(b.k8), p(b.v8), p(q), p(q), w, n, None)
    assert call(ws.data_ptr(), need - 1, table.shape[1], 4) == -2
    assert call(ws.data_ptr() + 16, need, table.shape[1], 4) == -1
    assert call(ws.data_ptr(), need, (1 << 26) + 1, 4) == -1
    assert call(ws.data_ptr(), need, table.shape[1], 0) == -1
    assert b.ctx.laps_attention_kv8_workspace_bytes(1 << 20, 1 << 20, 4) == 0
    torch.cuda.synchronize()
    assert torch.equal(before[0], b.k8) and torch.equal(before[1], b.v8)
    b.ctx.close()
