"""What the binding does around the calls of the library (those on 4-bit pools above all), on the CPU: a library that only writes down what
it is asked."""
import threading
import time
import types

import pytest
import torch

from paper_2601_11589_amd import api, inputs

CFG = inputs.tiny_cfg(1)


class Recorder:
    """Stands where the shared library does.  Every call that sets a page count leaves other threads time to come between."""

    def __init__(self):
        self.pages, self.used = None, {}

    def __getattr__(self, name):
        def call(handle, *args):
            if "pool_pages" in name:
                self.pages = getattr(args[0], "value", args[0])
                time.sleep(0.01)
                return 0
            if name.endswith("_bytes"):
                return 544
            if name == "laps_ctx_create":
                return 0
            self.used.setdefault(threading.current_thread().name, []).append(self.pages)
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    lib = Recorder()
    monkeypatch.setattr(api, "lib", lambda: lib)
    monkeypatch.setattr(api, "_expect", lambda what, t, dtype, shape, device: t.data_ptr())
    monkeypatch.setattr(api, "_after_current", lambda stream: None)
    monkeypatch.setattr(api, "_raw_stream", lambda device: 0)
    return lib


def arguments(n_pages):
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    pool = lambda: torch.zeros((n_pages, CFG.n_kv_heads, 544), dtype=torch.uint8)
    rows = lambda: torch.zeros((3, CFG.n_kv_heads, CFG.head_dim), dtype=torch.bfloat16)
    q = lambda: torch.zeros((3, CFG.n_q_heads * CFG.head_dim), dtype=torch.bfloat16)
    return types.SimpleNamespace(cu=i32(3), start=i32(2), table=i32(2, 4), lens=i32(2), k4=pool(), v4=pool(), k=rows(), v=rows(), q=q(), out=q())


def calls(ctx, a, stream):
    return {
        "scatter": ([a.cu, a.start, a.table, a.k, a.v, a.k4, a.v4],
                    lambda: ctx.laps_kv4_scatter(a.cu, a.start, a.table, a.k, a.v, a.k4, a.v4, stream=stream)),
        "gather": ([a.cu, a.start, a.table, a.k4, a.v4, a.k, a.v],
                   lambda: ctx.laps_kv4_gather(a.cu, a.start, a.table, a.k4, a.v4, 3, a.k, a.v, stream=stream)),
        "attention": ([a.cu, a.lens, a.start, a.table, a.k4, a.v4, a.q, a.out],
                      lambda: ctx.laps_attention_kv4(a.cu, a.lens, a.start, a.table, a.k4, a.v4, a.q, a.out, stream=stream)),
    }


@pytest.mark.parametrize("name", ["scatter", "gather", "attention"])
def test_everything_a_side_stream_reads_or_writes_is_held(library, monkeypatch, name):
    held = []
    monkeypatch.setattr(api, "_held_by", lambda stream, *tensors: held.extend(t for t in tensors if t is not None))
    side = types.SimpleNamespace(cuda_stream=1)
    given, call = calls(api.LapsCtx(CFG, 64), arguments(5), side)[name]
    call()
    assert all(any(h is t for h in held) for t in given), [i for i, t in enumerate(given) if not any(h is t for h in held)]
    assert all(isinstance(t, torch.Tensor) for t in held)
    assert name != "attention" or any(h.dtype is torch.uint8 and h.dim() == 1 for h in held)      # and the workspace


@pytest.mark.parametrize("name", ["scatter", "gather", "attention"])
def test_threads_with_pools_of_different_sizes_keep_their_counts(library, name):
    ctx, sizes = api.LapsCtx(CFG, 64), (3, 50, 700)

    def run(n_pages):
        call = calls(ctx, arguments(n_pages), None)[name][1]
        for _ in range(5):
            call()

    threads = [threading.Thread(target=run, args=(n,), name=str(n)) for n in sizes]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert library.used == {str(n): [n] * 5 for n in sizes}


def test_the_4bit_page_count_refuses_a_missing_context():
    assert api.lib().laps_ctx_set_kv4_pool_pages(None, 8) == -1 and b"kv4_pool_pages" in api.lib().laps_last_error()


@pytest.mark.parametrize("epilogue", [0, 1, 2])
def test_the_workspace_of_a_product_on_a_side_stream_is_held(library, monkeypatch, epilogue):
    held = []
    monkeypatch.setattr(api, "_held_by", lambda stream, *tensors: held.extend(tensors))
    side, ctx = types.SimpleNamespace(cuda_stream=1), api.LapsCtx(CFG, 64)
    a, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((64, 64), dtype=torch.bfloat16)
    ctx.laps_gemm_epilogue_bf16(a, w, epilogue, stream=side) if epilogue else ctx.laps_gemm_bf16(a, w, 4, stream=side)
    assert any(t.dtype is torch.uint8 for t in held)
