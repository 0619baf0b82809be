"""The 4-bit K/V cache on the CPU: its definition against hand-worked values, the library's sizes, and what its entry points
and their binding refuse."""
import ctypes as C
import math
import os
import random
import subprocess

import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O
from paper_2601_11589_amd import api, inputs


def group(*first):
    x = np.zeros(32)
    x[:len(first)] = first
    return x


@pytest.mark.parametrize("x, e, want", [
    (group(), -126, [0, 0]),
    (group(7.0, 0.25, 0.75, 1.25), 0, [6, 0, 1, 1]),              # ties go to the even code
    (group(7.0, 1.75, 2.5, 3.5, 5.0), 0, [6, 2, 2, 4, 4]),
    (group(7.03, 2.0, -0.5), 1, [8, 2, -0.0]),                    # one step above 7: the next power of two
    (group(3.5), -1, [3.0]),                                      # 7 * 2^-1
    (group(-1.0, 1 / 3), -2, [-1.0, 0.375]),                      # 1/3 / 2^-2 = 1.333 -> 1.5
    (group(2.0 ** 127 * 1.9921875, 2.0 ** 127), 125, [6 * 2.0 ** 125, 4 * 2.0 ** 125]),
    (group(2.0 ** -133), -126, [0.0]),
])
def test_definition(x, e, want):
    codes, scales = O.quantise(x)
    assert scales[0] == e + 127
    got = O.value(codes, scales)[:len(want)]
    assert np.array_equal(got, want) and np.array_equal(np.signbit(got), np.signbit(want))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_definition_of_a_group_that_is_not_finite(bad):
    codes, scales = O.quantise(group(1.0, bad, 2.0))
    assert scales[0] == 255 and not codes.any() and np.isnan(O.value(codes, scales)).all()


def test_definition_is_off_by_half_a_step():
    x = np.random.default_rng(1).standard_normal((64, 128)) * np.exp2(np.random.default_rng(2).integers(-30, 30, (64, 1)))
    codes, scales = O.quantise(x)
    z = np.abs(x).reshape(64, 4, 32) / np.exp2(scales.astype(float) - 127)[..., None]
    step = np.where(z < 2, 0.5, np.where(z < 4, 1.0, 2.0))
    off = np.abs(O.value(codes, scales) - x).reshape(64, 4, 32) / np.exp2(scales.astype(float) - 127)[..., None]
    assert (off <= step / 2).all() and z.max() <= 7 and (z.max(-1) > 3.5).all()


def test_pages_hold_what_was_put():
    g = np.random.default_rng(3)
    for hd in (64, 128):
        k, v = g.standard_normal((16, 2, hd)), g.standard_normal((16, 2, hd))
        kp, vp = (g.integers(0, 256, (3, 2, O.block_bytes(hd))).astype(np.uint8) for _ in range(2))
        for t in range(16):
            O.put(kp, vp, 1, t, *O.quantise(k[t]), *O.quantise(v[t]))
        for t in range(16):
            got_k, got_v = O.take(kp, vp, 1, t)
            assert np.array_equal(got_k, O.value(*O.quantise(k[t]))) and np.array_equal(got_v, O.value(*O.quantise(v[t])))


def test_block_bytes():
    L = api.lib()
    assert [int(L.laps_kv4_block_bytes(C.c_int32(h))) for h in (64, 128, 0, 32, 96, 256, -64)] == [544, 1088, 0, 0, 0, 0, 0]


def test_entry_points_refuse_a_missing_context():
    L, n, i = api.lib(), C.c_void_p(0), C.c_int32(1)
    some = C.c_void_p(4096)
    for f in (L.laps_kv4_scatter, L.laps_kv4_gather):
        assert f(n, i, i, some, some, some, i, some, some, some, some, n) == -1 and b"kv4 move" in L.laps_last_error()
    assert L.laps_attention_kv4(n, i, i, some, some, some, some, i, some, some, some, some, some, C.c_size_t(1 << 20), n) == -1
    assert b"attention_kv4" in L.laps_last_error()
    assert int(L.laps_attention_kv4_workspace_bytes(n, i, i, i)) == 0


@pytest.mark.parametrize("t", [torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int32).t()])
def test_binding_refuses_other_tensors(t):
    for device in (-1, 0):
        with pytest.raises(api.LapsError, match="page_table"):
            api._expect("page_table", t, torch.int32, (4, 2), device)      # host memory, another type, not contiguous


def test_model_shapes_have_whole_groups():
    for f in (inputs.tiny_cfg, inputs.qwen7b_cfg, inputs.qwen14b_cfg, inputs.qwen32b_cfg):
        assert f(1).head_dim % O.GROUP == 0


# ------------------------------------------------------------------------------------------------ launch plans
def plan(n_seq, n_tokens, heads, pages):
    out = (C.c_int64 * 6)()
    rc = api.lib().laps_attention_kv4_plan_info(C.c_int32(n_seq), C.c_int32(n_tokens), *(C.c_int32(h) for h in heads), C.c_int32(pages), out)
    return dict(zip(("rows", "blocks", "parts", "min_parts", "shares", "bytes"), list(out))) if rc == 0 else None


HEADS = [(4, 2, 64), (28, 4, 128), (40, 8, 128), (64, 8, 64), (8, 8, 128), (71, 1, 64)]


def shapes(n, seed):
    g = random.Random(seed)
    for _ in range(n):
        n_seq = int(math.exp(g.uniform(0, math.log(3000))))
        tokens = max(1, int(n_seq * math.exp(g.uniform(math.log(0.5), math.log(300)))))
        yield n_seq, tokens, g.choice(HEADS), int(math.exp(g.uniform(0, math.log(1 << 17))))


def test_plans_of_few_rows_hold_what_their_kernel_assumes():
    for n_seq, tokens, heads, pages in shapes(4000, 1):
        p, (n_q, n_kv, hd) = plan(n_seq, tokens, heads, pages), heads
        what = (n_seq, tokens, heads, pages, p)
        mean = tokens * (n_q // n_kv) / n_seq
        if p["rows"] > 32:      # blocks: never a split key range, whose kernel reads bf16 pools only
            assert p["rows"] in (128, 256) and p["parts"] == 1 and mean > 16, what
            assert p["shares"] == 0 or p["rows"] == 256, what
            assert p["bytes"] >= p["shares"] * 2 * 256 * (hd + 2) * 4 + p["blocks"] * 32, what
            continue
        assert p["rows"] == (16 if mean <= 16 else 32) and 1 <= p["min_parts"] <= p["parts"] <= 96, what
        assert p["blocks"] * n_seq * n_kv <= max(1 << 20, n_seq * n_kv), what
        assert p["blocks"] * p["rows"] * n_seq >= tokens * (n_q // n_kv) or p["blocks"] * n_seq * n_kv > (1 << 19), what
        assert p["bytes"] >= (tokens * n_q * p["parts"] * (hd + 2) * 4 if p["parts"] > 1 else 1), what
        assert p["bytes"] <= 64 << 20, what      # what lies between the kernels stays small


def test_plans_refuse():
    assert plan(1, 1, (40, 8, 128), 10) is not None
    for bad in ((0, 1, (40, 8, 128), 10), (1, 0, (40, 8, 128), 10), (1, 1, (40, 8, 128), 0), (1, 1, (40, 8, 96), 10), (1, 1, (40, 7, 128), 10),
                (1, 1, (40, 8, 128), (1 << 26) + 1), (1 << 15, 1 << 15, (40, 8, 128), 10)):
        assert plan(*bad) is None, bad


@pytest.fixture(scope="module")
def parts_driver(tmp_path_factory, repo_root):
    exe = str(tmp_path_factory.mktemp("parts") / "kv4_parts")
    build = subprocess.run(["/opt/rocm/bin/hipcc", "-x", "c++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                            os.path.join(repo_root, "tests", "kv4_parts_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr

    def run(lines):
        r = subprocess.run([exe], input="\n".join(" ".join(map(str, x)) for x in lines) + "\n", capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        return [tuple(map(int, x.split())) for x in r.stdout.splitlines()]

    return run


def test_parts_cover_the_keys(parts_driver):
    g = random.Random(2)
    asked = []
    for n_seq, tokens, heads, pages in shapes(600, 3):
        p = plan(n_seq, tokens, heads, pages)
        if p["rows"] <= 32:
            for kv_len in (1, pages * 16, g.randint(1, pages * 16), min(pages * 16, 128), min(pages * 16, 129)):
                asked.append((kv_len, pages, p["parts"], p["min_parts"]))
    assert len(asked) > 1000
    for (kv_len, pages, parts, least), (each, used) in zip(asked, parts_driver(asked), strict=True):
        what = (kv_len, pages, parts, least, each, used)
        rounds = -(-kv_len // 128)
        assert 1 <= used <= parts and each >= 1 and (used - 1) * each < rounds <= used * each, what
        assert used == 1 or each >= 2, what
        assert used >= min(least, rounds // 2) * 0.5, what                   # equal lengths may need fewer parts than asked for
        assert each <= max(-(-rounds // least), -(-(-(-pages // 8)) // parts), 3), what   # none longer than its share of the table
