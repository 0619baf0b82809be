"""8-bit matrices on the GPU: quantised and read back bit for bit, products exactly where float32 sums are exact and within their roundings
elsewhere, and a run of projections, cache and attention as a server would call them."""
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


@pytest.fixture(scope="module")
def ctx():
    c = api.LapsCtx(inputs.tiny_cfg(1), 64)
    yield c
    c.close()


def wide(t):
    return t.double().cpu().numpy()


def bits_of(g, shape):
    return torch.from_numpy(g.integers(0, 1 << 16, shape).astype(np.uint16).view(np.int16)).view(torch.bfloat16)


def same_codes(got, want):
    nan = (want & 127) == 127
    assert np.array_equal((got & 127) == 127, nan) and np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want))


# ------------------------------------------------------------------------------------------------ quant, dequant
@pytest.mark.parametrize("m,k", [(1, 1), (1, 128), (3, 127), (17, 129), (16, 256), (5, 640), (33, 1000), (2, 72), (40, 8), (1, 5000), (300, 136)])
@pytest.mark.parametrize("kind", ["normal", "any bits", "tiny", "huge"])
def test_matrices_hold_the_definition_and_read_back(ctx, m, k, kind):
    g = np.random.default_rng(m * 10007 + k)
    x = bits_of(g, (m, k)) if kind == "any bits" else torch.from_numpy(g.standard_normal((m, k)).astype(np.float32))
    x = (x * {"tiny": 2.0 ** -124, "huge": 2.0 ** 125}.get(kind, 1.0)).to(torch.bfloat16)
    codes, scales = ctx.laps_fp8_quant(x.cuda())
    want_codes, want_scales = O.quantise(wide(x))
    same_codes(codes.cpu().numpy(), want_codes)
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    back = ctx.laps_fp8_dequant(codes, scales, k)
    assert back.shape == (m, k) and np.array_equal(wide(back), O.value(want_codes, want_scales, k), equal_nan=True)


def test_every_bf16_value_in_a_block_of_its_own(ctx):
    x = torch.zeros((1 << 16, 128), dtype=torch.int16)
    bits = torch.arange(1 << 16).to(torch.int32)
    x[:, 77] = bits.to(torch.int16)
    x[:, :70] = ((bits & 0x7fff)[:, None] - torch.arange(70)[None] * 17).clamp(0, 0x7fff).to(torch.int16)
    x = x.view(torch.bfloat16)
    codes, scales = ctx.laps_fp8_quant(x.cuda())
    w = wide(x)
    top = np.where(np.isfinite(w), np.abs(w), 0).max(-1)
    e = np.array([O.exponent(t) for t in top])
    assert np.array_equal(scales.cpu().numpy()[0], e + 127)
    want = O.encode(w * np.exp2(-e.astype(float))[:, None], 0)
    same_codes(codes.cpu().numpy(), want)
    assert np.array_equal(wide(ctx.laps_fp8_dequant(codes, scales, 128)), O.decode(want, e[:, None]), equal_nan=True)


def test_rows_of_any_alignment_and_given_outputs(ctx):
    g = np.random.default_rng(5)
    flat = torch.from_numpy(g.standard_normal(40 * 256 + 3).astype(np.float32)).to(torch.bfloat16).cuda()
    x = flat[3:].view(40, 256)                        # two bytes on
    want = ctx.laps_fp8_quant(x.clone())
    codes, scales = torch.full((42, 256), 9, dtype=torch.uint8, device="cuda"), torch.full((3, 48), 9, dtype=torch.uint8, device="cuda")
    got = ctx.laps_fp8_quant(x, codes[:40], scales[:2])
    assert got[0].data_ptr() == codes.data_ptr() and all(torch.equal(a, b) for a, b in zip(got, want))
    assert (codes[40:] == 9).all() and (scales[2] == 9).all()
    out = torch.full((40 * 256 + 8,), 7.0, dtype=torch.bfloat16, device="cuda")
    ctx.laps_fp8_dequant(*want, 256, out=out[1:-7].view(40, 256))
    assert torch.equal(out[1:-7].view(40, 256), ctx.laps_fp8_dequant(*want, 256)) and out[0] == 7 and (out[-7:] == 7).all()


# ------------------------------------------------------------------------------------------------ products
def whole_numbers(g, rows, k, small):
    """Codes of whole numbers up to 3 under scales 2^0 to 2^small: every product and every sum is exact in float32."""
    codes = O.encode(g.integers(-3, 4, (rows, k)), 0)
    columns = -(-k // 128) * 128
    padded = np.zeros((rows, columns), np.uint8)
    padded[:, :k] = codes
    scales = g.integers(127, 128 + small, (columns // 128, -(-rows // 16) * 16)).astype(np.uint8)
    return padded, scales


def product(ctx, a, w, out=None, stream=None):
    t = [torch.from_numpy(x).cuda() for x in (*a, *w)]
    return ctx.laps_gemm_fp8(*t, out=out, stream=stream)


def exact(a, w):
    return O.value(*a) @ O.value(*w).T


def plan(m, n, k):
    out = (C.c_int32 * 5)()
    assert api.lib().laps_gemm_fp8_plan_info(m, n, k, out) == 0
    return out[0], out[1], out[2] > 1


SHAPES = [(1, 1, 1), (1, 16, 128), (2, 3, 130), (17, 33, 129), (64, 64, 256), (65, 127, 640), (128, 128, 128), (129, 130, 384), (1, 512, 2048), (5, 1000, 1920),
          (96, 2560, 1152), (200, 320, 5120), (257, 511, 512), (300, 1031, 896), (16, 4608, 3584), (1, 3584, 18944), (3, 40, 12800), (700, 640, 1280),
          (1000, 2048, 256), (2300, 300, 384), (40, 9001, 256), (513, 2816, 640), (320, 4864, 128), (1500, 1800, 128)]


@pytest.mark.parametrize("m,n,k", SHAPES)
def test_products_of_whole_numbers_are_exact(ctx, m, n, k):
    g = np.random.default_rng(m + 3 * n + 7 * k)
    a, w = whole_numbers(g, m, k, 3), whole_numbers(g, n, k, 2)
    assert 9 * 2 ** 5 * k < 2 ** 24
    out = torch.full((m * n + 16,), 5.0, dtype=torch.bfloat16, device="cuda")
    got = product(ctx, a, w, out[:m * n].view(m, n))
    want = torch.from_numpy(exact(a, w)).to(torch.float32).to(torch.bfloat16)
    assert torch.equal(got.cpu(), want) and (out[m * n:] == 5).all()


# Every tile, with and without K slices, on sizes that its edges cut.
TILES = [(64, 33000, 130, (64, 256, False)), (645, 2965, 306, (128, 128, False)), (773, 129, 12004, (128, 128, True)), (100, 33000, 200, (128, 256, False)),
         (1243, 3203, 1073, (128, 256, False)), (270, 3773, 13898, (128, 256, True)), (2291, 3616, 303, (192, 256, False)), (264, 5377, 12486, (192, 256, True)),
         (552, 7277, 1222, (256, 128, False)), (131, 5691, 10588, (256, 128, True)), (1750, 6635, 487, (256, 192, False)), (2206, 541, 18307, (256, 192, True)),
         (1559, 7785, 538, (256, 256, False)), (454, 8225, 8008, (256, 256, True)), (17, 102, 2455, (64, 128, True)), (16, 16384, 512, (16, 16, False)),
         (9, 520, 512, (16, 16, False)), (3, 3584, 3300, (16, 16, False)), (16, 2100, 2048, (16, 16, False)), (16, 300, 1000, (16, 16, False))]


@pytest.mark.parametrize("m,n,k,tile", TILES)
def test_products_on_every_tile_are_exact(ctx, m, n, k, tile):
    """As above, in 64 bits on the GPU."""
    assert plan(m, n, k) == tile
    g = torch.Generator(device="cuda").manual_seed(m + n)

    def matrix(rows, small):
        x = torch.zeros((rows, -(-k // 128) * 128), device="cuda")
        x[:, :k] = torch.randint(-3, 4, (rows, k), device="cuda", generator=g).float()
        scales = torch.randint(127, 128 + small, (x.shape[1] // 128, -(-rows // 16) * 16), dtype=torch.uint8, device="cuda", generator=g)
        value = x.double().unflatten(1, (-1, 128)) * torch.exp2(scales.T[:rows].double() - 127)[..., None]
        return x.to(torch.float8_e4m3fn).view(torch.uint8), scales, value.flatten(1)

    (a, a_scales, va), (w, w_scales, vw) = matrix(m, 3), matrix(n, 2)
    out = torch.full((m * n + 16,), 5.0, dtype=torch.bfloat16, device="cuda")
    ctx.laps_gemm_fp8(a, a_scales, w, w_scales, out=out[:m * n].view(m, n))
    want = (va @ vw.T.contiguous()).float().to(torch.bfloat16)
    assert torch.equal(out[:m * n].view(m, n), want) and (out[m * n:] == 5).all()


def test_every_k_counts_once_under_its_own_scale(ctx):
    """One code a row, a place of its own: results tell k, row and column apart."""
    k = 512
    a, w = (np.zeros((128, k), np.uint8), np.full((4, 128), 127, np.uint8)), (np.zeros((128, k), np.uint8), np.full((4, 128), 127, np.uint8))
    for lo in range(0, k, 128):
        a[0][:], w[0][:] = 0, 0
        a[0][np.arange(128), lo + np.arange(128)] = 0x38            # 1
        w[0][np.arange(128), lo + (5 * np.arange(128) + 3) % 128] = 0x3c   # 1.5
        a[1][lo // 128], w[1][lo // 128] = 127 + np.arange(128) % 7, 127 - np.arange(128) % 5
        got = wide(product(ctx, a, w))
        want = np.zeros((128, 128))
        for n in range(128):
            m = (5 * n + 3) % 128
            want[m, n] = 1.5 * 2.0 ** (m % 7 - n % 5)
        assert np.array_equal(got, want)


@pytest.mark.parametrize("m,n,k", [(1, 300, 3584), (33, 520, 5120), (150, 260, 1408), (300, 600, 18944), (520, 1100, 256)])
def test_products_within_their_roundings(ctx, m, n, k):
    """Element by element: the bf16 rounding; each of eight products side by side cut below 2^-13 of the largest (its power of two); float32
    sums, 2^-23 of the magnitudes for each of the k / 8 + 64 additions at worst.  In the mean the cuts, whose signs are the products', are
    off by what eight of them of 2^-13 / sqrt(12) each are, against sqrt(k) products' worth of result."""
    g = np.random.default_rng(n)
    x, y = g.standard_normal((m, k)) * np.exp2(g.integers(-3, 3, (m, 1))), g.standard_normal((n, k)) * 0.02
    a, w = O.quantise(x), O.quantise(y)
    got, want = wide(product(ctx, a, w)), exact(a, w)
    va, vw = O.value(*a), O.value(*w)
    size = np.abs(va) @ np.abs(vw).T
    groups = np.zeros((m, n))
    for lo in range(0, va.shape[1], 8):      # sum over groups of the largest product: at most the product of the largest factors
        groups += np.abs(va[:, lo:lo + 8]).max(1)[:, None] * np.abs(vw[:, lo:lo + 8]).max(1)[None]
    slack = ULP * np.abs(want) + (1 + ULP) * (8 * 2.0 ** -13 * groups + (k / 8 + 64) * 2.0 ** -23 * size)
    assert (np.abs(got - want) <= slack).all()
    off = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert off <= ULP / math.sqrt(3) + 2.0 ** -13, off      # bf16 roundings alone: at most ULP / sqrt(3) in the mean square


@pytest.mark.parametrize("m,n,k", [(1, 4000, 3584), (33, 520, 5120), (150, 260, 1408), (300, 600, 18944), (520, 1100, 256)])
def test_products_are_as_near_as_documented(ctx, m, n, k):
    """The cuts take 3e-5 of a result at the most, in the mean square of a row, and float32 sums a tenth of that.  So an element is off by half
    a bf16 step of its value and 8 times that; and it differs from the 64-bit value's own rounding where a border between two numbers of
    bf16 lies between the two, once in (step / error): of as many elements as the sum of these, within four standard deviations."""
    g = np.random.default_rng(m + n)
    a, w = O.quantise(g.standard_normal((m, k))), O.quantise(g.standard_normal((n, k)) * 0.02)
    got, want = wide(product(ctx, a, w)), exact(a, w)
    error = 3e-5 * np.sqrt((want ** 2).mean(1, keepdims=True))
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(want), np.abs(got)))) - 7)
    assert (np.abs(got - want) <= step / 2 + 8 * error).all()
    expected = np.minimum(1, error / step).sum()
    differ = (got != wide(torch.from_numpy(want).to(torch.float32).to(torch.bfloat16))).sum()
    assert differ <= expected + 4 * math.sqrt(expected), (differ, expected)


def test_a_nan_makes_its_row_and_its_column(ctx):
    g = np.random.default_rng(2)
    a, w = whole_numbers(g, 150, 300, 2), whole_numbers(g, 260, 300, 2)
    a[0][140, 299], w[0][7, 0], w[0][258, 130] = 0x7f, 0xff, 0x7f
    got = wide(product(ctx, a, w))
    bad = np.zeros((150, 260), bool)
    bad[140], bad[:, [7, 258]] = True, True
    assert np.array_equal(np.isnan(got), bad)
    want = exact(a, w)
    assert np.array_equal(got[~bad], wide(torch.from_numpy(want[~bad]).to(torch.bfloat16)))


@pytest.mark.parametrize("e", [(11, 246), (246, 11), (11, 11), (246, 246)])
def test_scales_at_their_ends(ctx, e):
    """2^-116 and 2^119: products that are ordinary, vanish or overflow."""
    a = np.full((3, 128), 0x38, np.uint8), np.full((1, 16), e[0], np.uint8)
    w = np.full((20, 128), 0x40, np.uint8), np.full((1, 32), e[1], np.uint8)
    got = wide(product(ctx, a, w))
    total = 256.0 * 2.0 ** (e[0] + e[1] - 254)
    assert (got == (math.inf if total > 2.0 ** 128 else total if total > 2.0 ** -126 else 0.0)).all()


@pytest.mark.parametrize("m,n,k", [(1, 3584, 3584), (1, 7, 100), (37, 640, 1000), (130, 200, 5120), (600, 300, 72), (2, 9000, 130), (8, 2000, 4096), (8, 333, 3000),
                                   (9, 2000, 4096), (16, 500, 2048), (16, 77, 1016), (5, 300, 1012), (3, 640, 40), (16, 4000, 512), (1, 8000, 136)])
def test_linear_is_quantise_then_multiply(ctx, m, n, k):
    g = np.random.default_rng(k)
    x = torch.from_numpy(g.standard_normal((m, k)).astype(np.float32)).to(torch.bfloat16).cuda()
    w = ctx.laps_fp8_quant(torch.from_numpy(g.standard_normal((n, k)).astype(np.float32)).to(torch.bfloat16).cuda())
    want = ctx.laps_gemm_fp8(*ctx.laps_fp8_quant(x), *w)
    assert torch.equal(ctx.laps_linear_fp8(x, *w), want)
    padded = torch.nn.functional.pad(x, (0, w[0].shape[1] - k))
    assert torch.equal(ctx.laps_linear_fp8(padded, *w), want)


@pytest.mark.parametrize("m,n,k", [(3, 200, 1032), (4, 64, 4096), (40, 64, 512)])
def test_linear_of_values_that_are_not_finite(ctx, m, n, k):
    """Quantised in one launch with the product or in one of its own: the scale is that of a block's finite values."""
    g = np.random.default_rng(m)
    x = bits_of(g, (m, k)) if k == 512 else torch.from_numpy(g.standard_normal((m, k)).astype(np.float32)).to(torch.bfloat16)
    x[1, 130], x[m - 1, k - 1] = math.inf, math.nan
    w = ctx.laps_fp8_quant(torch.from_numpy(g.standard_normal((n, k)).astype(np.float32)).to(torch.bfloat16).cuda())
    got, want = ctx.laps_linear_fp8(x.cuda(), *w), ctx.laps_gemm_fp8(*ctx.laps_fp8_quant(x.cuda()), *w)
    assert torch.isnan(got[1]).all() and torch.isnan(got[m - 1]).all() and torch.equal(got.view(torch.int16)[~torch.isnan(got)], want.view(torch.int16)[~torch.isnan(got)])
    assert torch.equal(torch.isnan(got), torch.isnan(want))


def test_linear_of_rows_off_their_bounds(ctx):
    """Rows two bytes off 16-byte bounds take the launch that reads them one by one."""
    g = torch.Generator(device="cuda").manual_seed(8)
    flat = torch.empty(3 * 1024 + 1, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    w = ctx.laps_fp8_quant(torch.empty((500, 1024), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g))
    x = flat[1:].view(3, 1024)
    assert torch.equal(ctx.laps_linear_fp8(x, *w), ctx.laps_linear_fp8(x.clone(), *w))


@pytest.mark.parametrize("m", [2, 40, 200])
def test_long_offsets(ctx, m):
    """Weights and rows behind 4 GiB: their last columns and rows against the same ones in matrices of their own."""
    n, k = (1 << 20) + 77, 4224
    g = torch.Generator(device="cuda").manual_seed(m)
    tail = torch.empty((77, k), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    x = torch.empty((m, k), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    few = ctx.laps_fp8_quant(tail)
    if m == 2:   # rows behind 4 GiB: of 8-bit codes and, twice as far, of bf16
        wide_w = torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
        wide_w[-77:] = tail
        codes, scales = ctx.laps_fp8_quant(wide_w)
        assert torch.equal(codes[-77:], few[0]) and torch.equal(scales[:, n - 77:n], few[1][:, :77]) and not codes[:-77].any()
        wide_w.fill_(3)
        ctx.laps_fp8_dequant(codes, scales, k, wide_w)
        assert torch.equal(wide_w[-77:], ctx.laps_fp8_dequant(*few, k)) and not wide_w[:-77].any()
        del wide_w
    else:
        codes = torch.zeros((n, k), dtype=torch.uint8, device="cuda")
        scales = torch.full((k // 128, (n + 15) // 16 * 16), 127, dtype=torch.uint8, device="cuda")
        codes[-77:], scales[:, n - 77:n] = few[0], few[1][:, :77]
    got = ctx.laps_linear_fp8(x, codes, scales)
    vx, vw = (ctx.laps_fp8_dequant(*q, k).double() for q in (ctx.laps_fp8_quant(x), few))
    want, size = vx @ vw.T, vx.abs() @ vw.abs().T
    groups = vx.abs().unflatten(1, (-1, 8)).amax(2) @ vw.abs().unflatten(1, (-1, 8)).amax(2).T
    assert not got[:, :-77].any()
    slack = ULP * want.abs() + (1 + ULP) * (8 * 2.0 ** -13 * groups + (k / 8 + 64) * 2.0 ** -23 * size)   # as above
    assert ((got[:, -77:].double() - want).abs() <= slack).all()


def test_more_rows_than_the_library_counts(ctx):
    """2^32 + 5 rows are not 5."""
    x = torch.empty(((1 << 32) + 5, 1), dtype=torch.bfloat16, device="cuda")
    w = ctx.laps_fp8_quant(torch.ones((1, 1), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(api.LapsError, match="rows"):
        ctx.laps_linear_fp8(x, *w)
    with pytest.raises(api.LapsError, match="codes|rows"):
        ctx.laps_fp8_quant(x)


def test_projections_refuse_what_their_parts_would(ctx):
    """Rows off their elements' bounds, weights and scales off 16 bytes, results off two: before any launch, on both paths."""
    L, h = api.lib(), ctx._h
    for m, n, k in ((3, 40, 256), (200, 300, 512)):
        x = torch.zeros(m * k + 1, dtype=torch.bfloat16, device="cuda")
        w, sw, ws = (torch.zeros(s, dtype=torch.uint8, device="cuda") for s in (n * k + 16, k // 128 * 304 + 16, L.laps_linear_fp8_workspace_bytes(m, n, k)))
        y = torch.full((m * n + 1,), 2.0, dtype=torch.bfloat16, device="cuda")
        ptr = [t.data_ptr() for t in (x, w, sw, y)]
        for at, off in ((0, 1), (1, 8), (2, 4), (3, 1)):
            a = [p + off * (i == at) for i, p in enumerate(ptr)]
            assert L.laps_linear_fp8(h, *a, m, n, k, ws.data_ptr(), ws.numel(), None) == -1, (m, at)
        torch.cuda.synchronize()
        assert (y == 2).all()


def test_results_repeat_on_any_stream(ctx):
    g = np.random.default_rng(3)
    a, w = O.quantise(g.standard_normal((48, 5120))), O.quantise(g.standard_normal((512, 5120)))
    t = [torch.from_numpy(v).cuda() for v in (*a, *w)]
    want = ctx.laps_gemm_fp8(*t)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [ctx.laps_gemm_fp8(*t, stream=s) for _ in range(6) for s in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got)


@pytest.mark.parametrize("m,n,k", [(1, 3584, 3584), (300, 512, 640)])
def test_captured_projections_replay(ctx, m, n, k):
    """Two graphs whose workspaces are their own, eager calls between replays."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x, wide_w = (torch.empty(s, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g) for s in ((m, k), (n, k)))
    w = ctx.laps_fp8_quant(wide_w)
    ctx.laps_linear_fp8(x, *w)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = ctx.laps_linear_fp8(x, *w)
        graphs.append((graph, out))
    for turn in range(6):
        x.normal_(0, 1, generator=g)
        graphs[turn % 2][0].replay()
        want = ctx.laps_linear_fp8(x, *w)
        torch.cuda.synchronize()
        assert torch.equal(graphs[turn % 2][1], want) and bool(want.any())


def test_refusals(ctx):
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    a, sa, w, sw = u8(3, 256), u8(2, 16), u8(40, 256), u8(2, 48)
    L, p, y = api.lib(), lambda t: t.data_ptr(), torch.full((3, 40), 2.0, dtype=torch.bfloat16, device="cuda")
    h = ctx._h
    assert L.laps_gemm_fp8(h, p(a) + 8, p(sa), p(w), p(sw), p(y), 2, 40, 256, None, 0, None) == -1
    assert L.laps_gemm_fp8(h, p(a), p(sa), p(w), p(sw) + 1, p(y), 3, 40, 256, None, 0, None) == -1
    assert L.laps_gemm_fp8(h, p(a), p(sa), p(w), p(sw), None, 3, 40, 256, None, 0, None) == -1
    assert L.laps_gemm_fp8(h, p(a), p(sa), p(w), p(sw), p(y), 0, 40, 256, None, 0, None) == -1
    big = L.laps_gemm_fp8_workspace_bytes(1, 256, 1 << 20)
    assert big > 0 and L.laps_gemm_fp8(h, p(a), p(sa), p(w), p(sw), p(y), 1, 256, 1 << 20, None, 0, None) == -2
    ws = u8(1 << 16)
    assert L.laps_linear_fp8(h, p(y), p(w), p(sw), p(y), 3, 40, 256, p(ws), 100, None) == -2
    assert L.laps_linear_fp8(h, p(y), p(w), p(sw), p(y), 3, 40, 256, p(ws) + 16, 60000, None) == -1
    assert L.laps_fp8_quant(h, p(y), 3, 40, p(a) + 4, p(sa), None) == -1 and L.laps_fp8_quant(h, p(y) + 1, 3, 40, p(a), p(sa), None) == -1
    assert L.laps_fp8_dequant(h, p(a), p(sa), 3, (1 << 22) + 1, p(y), None) == -1
    with pytest.raises(api.LapsError, match="x:"):
        ctx.laps_fp8_quant(torch.zeros((3, 4), dtype=torch.bfloat16))
    with pytest.raises(api.LapsError, match="codes|rows"):
        ctx.laps_fp8_quant(torch.zeros((0, 4), dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    assert (y == 2).all() and not a.any() and not w.any()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("cfgf", [inputs.tiny_cfg, inputs.qwen7b_cfg])
def test_a_layer_half_in_eight_bits(cfgf):
    """A chunk, then single tokens: q/k/v projection in 8 bits, keys and values into the 8-bit cache, attention over it, o projection in 8
    bits.  Each step against the definition, from what the step before handed on."""
    cfg = cfgf(1)
    ctx, g = api.LapsCtx(cfg, 64), np.random.default_rng(9)
    n_q, n_kv, hd = cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
    dev = lambda v: torch.from_numpy(np.ascontiguousarray(v, np.int32)).cuda()
    weights = [torch.from_numpy((g.standard_normal(s) * cfg.hidden ** -0.5).astype(np.float32)).to(torch.bfloat16).cuda()
               for s in (((n_q + 2 * n_kv) * hd, cfg.hidden), (cfg.hidden, n_q * hd))]
    w_qkv, w_o = (ctx.laps_fp8_quant(w) for w in weights)
    host = lambda pair: tuple(t.cpu().numpy() for t in pair)
    k8, v8 = (p[0] for p in ctx.new_kv8_pools(9, 1))
    pk, pv = k8.cpu().numpy(), v8.cpu().numpy()
    table = g.permutation(9)[None]
    at = 0

    def near(got, want, size):
        assert (np.abs(wide(got) - want) <= ULP * np.abs(want) + 2.0 ** -9 * size).all()      # roundings, and the cuts of sums (see above)

    for n in (37, 1, 1, 3):
        x = torch.from_numpy(g.standard_normal((n, cfg.hidden)).astype(np.float32)).to(torch.bfloat16).cuda()
        qkv = ctx.laps_linear_fp8(x, *w_qkv)
        vx, vw = O.value(*O.quantise(wide(x))), O.value(*host(w_qkv), cfg.hidden)
        near(qkv, vx @ vw.T, np.abs(vx) @ np.abs(vw).T)
        q, k, v = (t.contiguous() for t in qkv.split([n_q * hd, n_kv * hd, n_kv * hd], 1))
        k, v = k.view(n, n_kv, hd), v.view(n, n_kv, hd)
        ctx.laps_kv8_scatter(dev([0, n]), dev([at]), dev(table), k, v, k8, v8)
        O.write_run(pk, table[0], at, wide(k), False)
        O.write_run(pv, table[0], at, wide(v), True)
        out = ctx.laps_attention_kv8(dev([0, n]), None, dev([at]), dev(table), k8, v8, q)
        keys, values = (O.read_run(p, table[0], 0, at + n, n_kv, hd, t) for p, t in ((pk, False), (pv, True)))
        want, spread = attend(wide(q).reshape(n, n_q, hd), keys, values, at)
        assert (np.abs(wide(out).reshape(want.shape) - want) <= ULP * (spread + 2 * np.abs(want)) * (1 + 4 * ULP) + spread * 2.0 ** -14).all()
        y = ctx.laps_linear_fp8(out, *w_o)
        vx, vw = O.value(*O.quantise(wide(out))), O.value(*host(w_o), n_q * hd)
        near(y, vx @ vw.T, np.abs(vx) @ np.abs(vw).T)
        at += n
    ctx.close()
