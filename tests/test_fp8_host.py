"""8-bit floats on the CPU: their definition against hand-worked values, the library's sizes and plans, and what its entry points and
their binding refuse."""
import ctypes as C
import math
import random
import types

import numpy as np
import pytest
import torch

from oracle import fp8_oracle as O
from paper_2601_11589_amd import api, inputs

NAN = math.nan


@pytest.mark.parametrize("x, e, want", [
    ([0.0, -0.0], -116, [0.0, -0.0]),
    ([448.0, 1.0, 17.0, 19.0, 2.0 ** -9, 2.0 ** -10], 0, [448.0, 1.0, 16.0, 20.0, 2.0 ** -9, 0.0]),   # ties: to the even code
    ([449.0, 34.0, -38.0], 1, [448.0, 32.0, -40.0]),                        # above 448: the next power of two
    ([1.0, 1 / 3, -0.3], -8, [1.0, 0.34375, -0.3125]),                      # 256, 85.33 -> 88, 76.8 -> 80
    ([1.75, 3 * 2.0 ** -18, 5 * 2.0 ** -18], -8, [1.75, 4 * 2.0 ** -18, 4 * 2.0 ** -18]),   # steps of 2^-9 * 2^-8: ties at 1.5 and 2.5
    ([2.0 ** 127 * 1.9921875, 2.0 ** 127], 119, [448 * 2.0 ** 119, 2.0 ** 127]),
    ([2.0 ** -130], -116, [0.0]),
    ([math.inf, 3.0, NAN, -448.0], 0, [NAN, 3.0, NAN, -448.0]),
    ([math.inf, -math.inf], -116, [NAN, NAN]),
])
def test_definition(x, e, want):
    x = np.array(x)
    assert O.exponent(O.top(x)) == e
    got = O.decode(O.encode(x, e), e)
    assert np.array_equal(got, want, equal_nan=True) and np.array_equal(np.signbit(got)[got == 0], np.signbit(want)[got == 0])


def test_codes_are_those_of_the_type():
    all_codes = np.arange(256).astype(np.uint8)
    want = torch.from_numpy(all_codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.decode(all_codes, 0), want, equal_nan=True)
    x = np.random.default_rng(1).standard_normal(20000) * 100
    x = x[np.abs(x) <= 448]
    assert np.array_equal(O.encode(x.astype(np.float32), 0), torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_every_value_is_a_normal_bf16_number():
    for e in (O.LOWEST, 0, O.HIGHEST):
        v = O.decode(np.arange(1, 127).astype(np.uint8), e)
        assert np.array_equal(torch.from_numpy(v).to(torch.bfloat16).double().numpy(), v) and v.min() >= 2.0 ** -126


@pytest.mark.parametrize("v", [False, True])
def test_a_page_in_pieces(v):
    """Tokens written piece by piece: the larger scale wins, tokens before are rounded again; slot 0 begins anew."""
    pool = np.random.default_rng(2).integers(0, 256, (2, O.page_bytes(2, 64))).astype(np.uint8)
    rest = pool[0].copy()
    x = np.ones((16, 2, 64))
    x[3:6] = 40 * 448.0
    x[3, 1] = 1.0
    x[4, 1] = math.inf      # counts for no scale
    x[5, 1, 7] = 100.0
    O.write(pool, 1, 0, x[:3], v)
    assert np.array_equal(O.read(pool, 1, 2, 64, v)[:4], np.concatenate([x[:3], np.zeros((1, 2, 64))]))
    O.write(pool, 1, 3, x[3:6], v)
    got = O.read(pool, 1, 2, 64, v)
    # under 2^6: 280 lies between 256 and 288, 1 is 2^-6
    assert np.array_equal(got[3:6, 0], np.full((3, 64), 288 * 64.0)) and np.array_equal(got[:3, 0], np.ones((3, 64)))
    want = np.ones((3, 64))
    want[1], want[2], want[2, 7] = NAN, 288 * 64.0, 96.0      # 100 / 64 lies between 1.5 and 1.625
    assert np.array_equal(got[3:6, 1], want, equal_nan=True) and (got[6:] == 0).all()
    O.write(pool, 1, 0, x[:1], v)
    assert np.array_equal(O.read(pool, 1, 2, 64, v), np.concatenate([x[:1], np.zeros((15, 2, 64))]))
    assert np.array_equal(pool[0], rest)


def test_layout_by_hand():
    pool = np.zeros((1, O.page_bytes(3, 64)), np.uint8)
    x = np.zeros((16, 3, 64))
    x[9, 1, 22] = 448.0
    for v, at in ((False, 9 * 64 + 22), (True, 22 // 4 * 64 + 2 * 16 + 2 * 4 + 1)):
        pool[:] = 0
        O.write(pool, 0, 0, x, v)
        assert list(np.flatnonzero(pool[0][:3 * 1024])) == [1024 + at] and pool[0][1024 + at] == 0x7e
        assert list(pool[0][3 * 1024:3 * 1024 + 4]) == [11, 127, 11, 0] and pool.shape[1] == 3 * 1024 + 128


def test_matrix_by_hand():
    x = np.zeros((17, 130))
    x[16, 129], x[0, 0] = -7.0, 448.0 * 4
    codes, scales = O.quantise(x)
    assert codes.shape == (17, 256) and scales.shape == (2, 32)
    assert codes[0, 0] == 0x7e and scales[0, 0] == 129 and codes[16, 129] == 0x80 | 0x7e and scales[1, 16] == 127 - 6
    assert np.array_equal(O.value(codes, scales, 130), x) and scales[0, 17:].tolist() == [127] * 15


# ------------------------------------------------------------------------------------------------ sizes, plans
def test_sizes():
    L = api.lib()
    assert [L.laps_kv8_page_bytes(n, h) for n, h in ((2, 64), (8, 128), (129, 64), (0, 64), (4, 96), (-1, 128))] == [
        2 * 1024 + 128, 8 * 2048 + 128, 129 * 1024 + 256, 0, 0, 0]
    assert [L.laps_fp8_columns(k) for k in (1, 128, 129, 1 << 22, 0, (1 << 22) + 1, -5)] == [128, 128, 256, 1 << 22, 0, 0, 0]
    assert [L.laps_fp8_scale_pitch(r) for r in (1, 16, 17, 1 << 24, 0, (1 << 24) + 1)] == [16, 16, 32, 1 << 24, 0, 0]
    for n_kv, hd in ((2, 64), (8, 128), (129, 64)):
        assert L.laps_kv8_page_bytes(n_kv, hd) == O.page_bytes(n_kv, hd)


def product_plan(m, n, k):
    out = (C.c_int32 * 5)()
    rc = api.lib().laps_gemm_fp8_plan_info(C.c_int32(m), C.c_int32(n), C.c_int32(k), out)
    return dict(zip(("rows", "columns", "slices", "per_slice", "workgroups"), list(out))) if rc == 0 else None


def test_plans_of_products_hold_what_their_kernels_assume():
    g = random.Random(4)
    log = lambda hi: int(math.exp(g.uniform(0, math.log(hi))))
    for _ in range(4000):
        m, n, k = log(20000), log(60000), log(40000)
        p, columns = product_plan(m, n, k), -(-k // 128) * 128
        what = (m, n, k, p)
        assert p["per_slice"] % 128 == 0 and (p["slices"] - 1) * p["per_slice"] < columns <= p["slices"] * p["per_slice"], what
        assert p["workgroups"] == -(-m // p["rows"]) * -(-n // p["columns"]) * p["slices"], what
        need = api.lib().laps_gemm_fp8_workspace_bytes(m, n, k)
        assert need == 0 if p["slices"] == 1 else need >= p["slices"] * m * n * 4, what
        assert need <= 512 << 20, what
        whole = api.lib().laps_linear_fp8_workspace_bytes(m, n, k)
        assert whole >= need + m * columns + columns // 128 * (-(-m // 16) * 16), what


def test_plans_of_products_refuse():
    assert product_plan(1, 1, 1) is not None and product_plan(1 << 24, 1, 128 * 127) is not None
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, (1 << 22) + 1), ((1 << 24) + 1, 1, 1), (1, (1 << 24) + 1, 1), (1 << 24, 1 << 24, 128), (1 << 24, 1, 128 * 128), (1, 1 << 24, 1 << 22), (-1, 5, 5)):
        assert product_plan(*bad) is None and api.lib().laps_gemm_fp8_workspace_bytes(*bad) == 0, bad
        assert api.lib().laps_linear_fp8_workspace_bytes(*bad) == 0, bad


HEADS = [(4, 2, 64), (28, 4, 128), (40, 8, 128), (64, 8, 64), (8, 8, 128), (71, 1, 64)]


def test_plans_of_the_attention_hold_what_its_kernels_assume():
    g = random.Random(5)
    for _ in range(4000):
        n_seq = int(math.exp(g.uniform(0, math.log(3000))))
        tokens = max(1, int(n_seq * math.exp(g.uniform(math.log(0.5), math.log(300)))))
        (n_q, n_kv, hd), pages = g.choice(HEADS), int(math.exp(g.uniform(0, math.log(1 << 17))))
        out = (C.c_int64 * 6)()
        assert api.lib().laps_attention_kv8_plan_info(*(C.c_int32(v) for v in (n_seq, tokens, n_q, n_kv, hd, pages)), out) == 0
        rows, blocks, parts, least, shares, size = out
        what = (n_seq, tokens, n_q, n_kv, hd, pages, list(out))
        if rows > 32:      # blocks: never a split key range, whose kernel reads bf16 pools only
            assert rows in (128, 256) and parts == 1 and tokens * (n_q // n_kv) > 16 * n_seq and (shares == 0 or rows == 256), what
            assert size >= shares * 2 * 256 * (hd + 2) * 4 + blocks * 32, what
            continue
        assert rows in (16, 32) and 1 <= least <= parts <= 96 and blocks * n_seq * n_kv <= max(1 << 20, n_seq * n_kv), what
        assert size >= (tokens * n_q * parts * (hd + 2) * 4 if parts > 1 else 1) and size <= 96 << 20, what


# ------------------------------------------------------------------------------------------------ refusals
def test_entry_points_refuse_a_missing_context():
    L, n, some = api.lib(), None, 4096
    said = lambda rc, what: rc == -1 and what in L.laps_last_error()
    for f in (L.laps_kv8_scatter, L.laps_kv8_gather):
        assert said(f(n, 1, 1, some, some, some, 1, 1, some, some, some, some, n), b"kv8 move")
    assert said(L.laps_attention_kv8(n, 1, 1, some, some, some, some, 1, 1, some, some, some, some, some, 1 << 20, n), b"attention_kv8")
    assert said(L.laps_attention_kv8(some, 1, 1, some, some, some, some, 1, 0, some, some, some, some, some, 1 << 20, n), b"0 pages")
    assert L.laps_attention_kv8_workspace_bytes(n, 1, 1, 1) == 0
    assert said(L.laps_fp8_quant(n, some, 1, 1, some, some, n), b"fp8_quant")
    assert said(L.laps_fp8_dequant(n, some, some, 1, 1, some, n), b"fp8_dequant")
    assert said(L.laps_gemm_fp8(n, some, some, some, some, some, 1, 1, 1, n, 0, n), b"gemm_fp8")
    assert said(L.laps_linear_fp8(n, some, some, some, some, 1, 1, 1, some, 1 << 20, n), b"linear_fp8")


class Recorder:
    """Stands where the shared library does: takes every call, and answers sizes as the library does."""

    def __init__(self, real):
        self.real, self.asked = real, []

    def __getattr__(self, name):
        if name in ("laps_fp8_columns", "laps_fp8_scale_pitch", "laps_kv8_page_bytes", "laps_gemm_fp8_workspace_bytes", "laps_linear_fp8_workspace_bytes"):
            return getattr(self.real, name)
        if name.endswith("_bytes"):
            return lambda *a: 544
        return lambda *a: self.asked.append(name) or 0


@pytest.fixture
def ctx(monkeypatch):
    lib = Recorder(api.lib())
    monkeypatch.setattr(api, "lib", lambda: lib)
    monkeypatch.setattr(api, "_after_current", lambda stream: None)
    monkeypatch.setattr(api, "_raw_stream", lambda device: 0)
    real = api._expect

    def expect(what, t, dtype, shape, device):    # as if the tensors lay on the GPU
        if t.dtype is dtype and t.shape == shape and t.is_contiguous():
            return 4096
        return real(what, t, dtype, shape, device)

    monkeypatch.setattr(api, "_expect", expect)
    c = api.LapsCtx(inputs.tiny_cfg(1), 64)
    c.asked = lib.asked
    return c


def tensors(cfg):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    page = O.page_bytes(cfg.n_kv_heads, cfg.head_dim)
    return types.SimpleNamespace(cu=i32(3), start=i32(2), table=i32(2, 4), lens=i32(2), k8=u8(5, page), v8=u8(5, page), k=bf(3, cfg.n_kv_heads, cfg.head_dim),
                                 v=bf(3, cfg.n_kv_heads, cfg.head_dim), q=bf(3, cfg.n_q_heads * cfg.head_dim), out=bf(3, cfg.n_q_heads * cfg.head_dim),
                                 x=bf(3, 200), codes=u8(3, 256), scales=u8(2, 16), w=u8(40, 256), w_scales=u8(2, 48), y=bf(3, 40), back=bf(3, 200))


CALLS = {
    "scatter": (("cu", "start", "table", "k", "v", "k8", "v8"), lambda c, a, s: c.laps_kv8_scatter(a.cu, a.start, a.table, a.k, a.v, a.k8, a.v8, stream=s)),
    "gather": (("cu", "start", "table", "k8", "v8", "k", "v"),
               lambda c, a, s: c.laps_kv8_gather(a.cu, a.start, a.table, a.k8, a.v8, 3, a.k, a.v, stream=s)),
    "attention": (("cu", "lens", "start", "table", "k8", "v8", "q", "out"),
                  lambda c, a, s: c.laps_attention_kv8(a.cu, a.lens, a.start, a.table, a.k8, a.v8, a.q, a.out, stream=s)),
    "quant": (("x", "codes", "scales"), lambda c, a, s: c.laps_fp8_quant(a.x, a.codes, a.scales, stream=s)),
    "dequant": (("codes", "scales", "back"), lambda c, a, s: c.laps_fp8_dequant(a.codes, a.scales, 200, a.back, stream=s)),
    "gemm": (("codes", "scales", "w", "w_scales", "y"), lambda c, a, s: c.laps_gemm_fp8(a.codes, a.scales, a.w, a.w_scales, a.y, stream=s)),
    "linear": (("x", "w", "w_scales", "y"), lambda c, a, s: c.laps_linear_fp8(torch.zeros((3, 256), dtype=torch.bfloat16) if s is None else a.x2, a.w,
                                                                              a.w_scales, a.y, stream=s)),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_everything_a_side_stream_reads_or_writes_is_held(ctx, monkeypatch, name):
    held = []
    monkeypatch.setattr(api, "_held_by", lambda stream, *t: held.extend(x for x in t if x is not None))
    a = tensors(ctx.cfg)
    a.x2 = torch.zeros((3, 256), dtype=torch.bfloat16)
    names, call = CALLS[name]
    call(ctx, a, types.SimpleNamespace(cuda_stream=1))
    given = [a.x2 if (n, name) == ("x", "linear") else getattr(a, n) for n in names]
    assert ctx.asked[-1].startswith("laps_") and all(any(h is t for h in held) for t in given)
    if name in ("attention", "linear"):
        assert any(h.dtype is torch.uint8 and h.dim() == 1 for h in held)      # and the workspace


BAD = [
    ("scatter", "k", lambda t: t[:, :1], "k_src"), ("scatter", "v", lambda t: t[:2], "v_src"), ("scatter", "k8", lambda t: t[:, :-1], "k8_pool"),
    ("scatter", "v8", lambda t: t[1:], "v8_pool"), ("scatter", "start", lambda t: t[:1], "start_pos"), ("scatter", "cu", lambda t: t.long(), "cu"),
    ("gather", "v", lambda t: t.float(), "v_out"), ("gather", "table", lambda t: t[:1], "page_table"), ("gather", "k8", lambda t: t.short(), "k8_pool"),
    ("attention", "lens", lambda t: t.long(), "seq_len"), ("attention", "start", lambda t: t[:1], "prefix_len"), ("attention", "q", lambda t: t.float(), "q:"),
    ("attention", "q", lambda t: t[:, 1:], "q:"), ("attention", "out", lambda t: t[:2], "out"), ("attention", "k8", lambda t: t[..., :-1], "k8_pool"),
    ("quant", "x", lambda t: t.half(), "x:"), ("quant", "x", lambda t: t[:, 1:], "x:"), ("quant", "codes", lambda t: t[:, :200], "codes:"),
    ("quant", "codes", lambda t: t.view(torch.float8_e4m3fn), "codes:"), ("quant", "scales", lambda t: t[:1], "scales"),
    ("quant", "codes", lambda t: t[:2], "codes: need 3 rows"),
    ("dequant", "scales", lambda t: t[:, :3], "scales"), ("dequant", "back", lambda t: t[:, :199], "out"), ("dequant", "codes", lambda t: t[:, :128], "codes"),
    ("gemm", "codes", lambda t: t[:, :128].contiguous(), "a:"), ("gemm", "w_scales", lambda t: t[:, :40], "w scales"), ("gemm", "scales", lambda t: t.int(), "a scales"),
    ("gemm", "y", lambda t: t.float(), "out"), ("gemm", "y", lambda t: t[:, :39], "out"), ("linear", "w", lambda t: t[:, :128].contiguous(), "w:"),
    ("linear", "y", lambda t: t[:2], "out"), ("linear", "w_scales", lambda t: t[:1], "w scales"),
]


@pytest.mark.parametrize("name, which, change, match", BAD)
def test_binding_refuses_other_tensors(ctx, name, which, change, match):
    a = tensors(ctx.cfg)
    CALLS[name][1](ctx, a, None)                      # as they are they pass
    count = len(ctx.asked)
    setattr(a, which, change(getattr(a, which)))
    with pytest.raises(api.LapsError, match=match):
        CALLS[name][1](ctx, a, None)
    assert len(ctx.asked) == count


def test_tensors_on_the_host_are_refused():
    with pytest.raises(api.LapsError, match="k8_pool"):
        api._expect("k8_pool", torch.zeros((2, 3), dtype=torch.uint8), torch.uint8, (2, 3), -1)
