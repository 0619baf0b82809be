"""Eight-bit serving, as measurable cases: the 8-bit K/V cache with the attention that reads it, and projections in 8-bit floating point.

Operators, each through the public binding (`paper_2601_11589_amd.api`):

* laps_kv8_scatter     token-major bf16 K/V quantised into 8-bit pools
* laps_kv8_gather      8-bit pools read back to token-major bf16 K/V
* laps_attention_kv8   ragged paged causal grouped-query attention over 8-bit pools
* laps_fp8_quant       bf16 rows to 8-bit floats with a scale for each block of 128 along the row
* laps_fp8_dequant     the way back
* laps_linear_fp8      bf16 rows times 8-bit weights: laps_fp8_quant of the rows, then
* laps_gemm_fp8        the product of two 8-bit matrices under their scales, in bf16

Both formats are floats of 4 exponent and 3 mantissa bits (largest 448, no infinity) under a scale 2^e, kept as the byte e + 127: e is the
smallest integer with amax <= 448 * 2^e, cut to [-116, 119]; x / 2^e is rounded to nearest, ties to the even code, magnitudes above 448
to 448.  amax is taken over the finite values of a block; what is not finite becomes NaN.

* Cache: a block is a page of 16 tokens of one kv head, K and V apart.  Whoever writes a page's first token begins the page anew; whoever
  writes later ones keeps the tokens of the page, under the larger of the old scale and the one that the new tokens need, and rounds
  them again where that is larger.  A page holds n_kv blocks of 16 * head_dim codes, then n_kv scale bytes, padded to 128:

      K  codes [16 tokens][head_dim]
      V  codes [head_dim / 4][4 groups of tokens][4 head_dim indices][4 tokens]

* Matrices: codes [rows][k rounded up to 128], zeros behind k; scales [blocks of 128][rows rounded up to 16].

Kinds of pass:

* store    tokens into the pools and the same tokens back out: a hand-over of finished K/V through an 8-bit cache
* attend   attention alone, the new tokens' K/V in the pools already
* step     one serving step: the new tokens' K/V into the pools, then the attention that sees them
* linear   a projection of bf16 rows by weights that were quantised once
* product  the same of rows that are quantised already (several projections share them)
* round    a matrix to 8 bits and back: weights as they are loaded, rows as they are handed on

Lengths come from the case alone (`mix` seeds them), values from the seed.  Pages lie in random order and the pools' unused slots
hold stale bytes, as in a server that has run for a while.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
BLOCK = 128
HEADS = {"tiny": (4, 2, 64), "7b": (28, 4, 128), "14b": (40, 8, 128), "32b": (40, 8, 128)}   # query heads, kv heads, head_dim
# (columns, k) of the projections: q/k/v, o, gate/up, down
WEIGHTS = {"tiny": [(512, 256), (256, 256), (1024, 256), (256, 512)],
           "7b": [(4608, 3584), (3584, 3584), (37888, 3584), (3584, 18944)],
           "14b": [(7168, 5120), (5120, 5120), (27648, 5120), (5120, 13824)],
           "32b": [(7168, 5120), (5120, 5120), (55296, 5120), (5120, 27648)]}
LOWEST, HIGHEST = 11, 246   # scale bytes


# ----------------------------------------------------------------------------------------------- the cases
def _case(name, kind, model, n_seq, new, pre, fresh=0.0, pad=False, spare=0, mix=1):
    return dict(name=name, kind=kind, model=model, n_seq=n_seq, new_lo=new[0], new_hi=new[1], pre_lo=pre[0], pre_hi=pre[1],
                fresh=fresh, pad=pad, spare=spare, mix=mix)


def _matrix(name, kind, m, n, k):
    return dict(name=name, kind=kind, m=m, n=n, k=k)


def listed():
    return [
        # the smallest call: one conversation of an idle server writes and reads one token, behind four that its page holds already
        _case("store_one_7b", "store", "7b", 1, (1, 1), (900, 900)),
        # finished prompts handed over through the 8-bit cache, beginning and ending inside pages
        _case("store_prompts_32b", "store", "32b", 8, (512, 4096), (0, 40), mix=3),
        # the small test model: ragged turns, sequences without a token, padding rows between the sequences (head_dim 64)
        _case("tiny_ragged", "attend", "tiny", 12, (0, 40), (0, 300), fresh=0.25, pad=True, mix=7),
        # one token of many conversations: the cache is all the traffic
        _case("token_batch_32b", "step", "32b", 64, (1, 1), (512, 8191), mix=9),
        # one token over two very long histories: the key axis is all the parallelism there is
        _case("token_long_7b", "attend", "7b", 2, (1, 1), (100000, 131071), mix=11),
        # the re-prefill workload of the benchmark: short turns over cached histories
        _case("reprefill_32b", "attend", "32b", 16, (17, 64), (512, 4096), mix=15),
        # ragged last chunk of the longest prompt of the benchmark
        _case("chunk_last_32b", "attend", "32b", 1, (1847, 1847), (6144, 6144)),
        # one token through one projection (o): latency
        _matrix("linear_token_7b", "linear", 1, 3584, 3584),
        # a batch of short turns (mean fill of the captured 128-row buckets) through the widest projection: the weights' stream
        _matrix("linear_turns_32b", "linear", 96, 55296, 5120),
        # a chunk of a long prompt through the same: the matrix cores
        _matrix("product_chunk_32b", "product", 2048, 55296, 5120),
        # a ragged batch of turns through the longest rows (down)
        _matrix("linear_group_7b", "linear", 573, 3584, 18944),
        # one layer's gate and up weights as a checkpoint is loaded
        _matrix("round_weights_7b", "round", 37888, 0, 3584),
    ]


MOST_STORED = 16384             # tokens of the largest store
MOST_CACHED = 131072            # cached tokens of all sequences of the largest attention
MOST_PAIRS = 11 << 20           # (new token, cached token) pairs of the largest attention
MOST_PRODUCTS = 2048 * 55296 * 5120
MOST_ROUNDED = 37888 * 3584


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    kind = rng.choice(["store", "token", "token", "few", "turn", "chunk", "mixed", "linear", "linear", "linear", "product", "round"])
    model = rng.choice(["tiny", "7b", "14b", "32b"])
    mix = rng.randrange(1 << 30)
    if kind in ("linear", "product", "round"):
        # the models' projections, and matrices of any size, odd ones among them
        n, k = rng.choice(WEIGHTS[model]) if rng.random() < 0.6 else (_log(rng, 1, 16384), _log(rng, 8, 16384))
        if kind == "round":
            c = _matrix("", kind, min(_log(rng, 1, 40000), MOST_ROUNDED // k), 0, k)
        else:
            c = _matrix("", kind, min(_log(rng, 1, 4096), MOST_PRODUCTS // (n * k)), n, k)
    elif kind == "store":
        hi = _log(rng, 1, 8192)
        n = min(_log(rng, 1, 256), max(1, MOST_STORED // hi))
        c = _case("", kind, model, n, (rng.randint(1, hi), hi), (0, rng.choice([0, 40])), mix=mix)
    else:
        new_hi = {"token": 1, "few": rng.randint(2, 8), "turn": _log(rng, 9, 200), "chunk": _log(rng, 129, 2048),
                  "mixed": _log(rng, 40, 600)}[kind]
        new_lo = {"token": 1, "few": 1, "turn": 8, "chunk": new_hi, "mixed": 0}[kind]
        n = 1 if kind == "chunk" else _log(rng, 1, 96 if kind == "token" else 48)
        pre = min(_log(rng, 16, 131072), MOST_CACHED // n, MOST_PAIRS // (n * new_hi))
        pre = max(0, pre - new_hi)
        c = _case("", rng.choice(["attend", "step"]), model, n, (new_lo, new_hi), (rng.randint(0, pre), pre),
                  fresh=rng.choice([0.0, 0.25]), pad=rng.random() < 0.25, spare=rng.choice([0, 3, 200]), mix=mix)
    c.pop("name")
    return c


# ----------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """(new, prefix, rows) of every sequence; rows > new where the batch is padded."""
    g = np.random.default_rng(case["mix"])
    n = case["n_seq"]
    new = g.integers(case["new_lo"], case["new_hi"] + 1, n)
    pre = np.where(g.random(n) < case["fresh"], 0, g.integers(case["pre_lo"], case["pre_hi"] + 1, n))
    if new.sum() == 0:
        new[0] = 1
    rows = new + g.integers(0, 4, n) if case["pad"] else new
    return new, pre, rows


def _generator(seed, what):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + what) % (1 << 62))


def _normal(g, shape):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def _tokens(case, seed):
    """All K/V that the pools will hold, token-major over the sequences' whole histories, and the new tokens' q."""
    n_q, n_kv, hd = HEADS[case["model"]]
    new, pre, rows = _lengths(case)
    total = int((new + pre).sum())
    g = _generator(seed, 1)
    k, v = _normal(g, (total, n_kv, hd)), _normal(g, (total, n_kv, hd))
    # keys of a rotated cache: a few channels stand out
    k *= 1 + 3 * (torch.rand((1, n_kv, hd), generator=g, device="cuda") > 0.95)
    q = _normal(g, (int(rows.sum()), n_q * hd)) if case["kind"] in ("attend", "step") else None
    return k, v, q


def _matrices(case, seed):
    """Rows as a norm leaves them (some channels and rows stand out), weights of a layer."""
    g = _generator(seed, 3)
    k = case["k"]
    scale = 0.02 if case["kind"] == "round" else 1.0
    x = _normal(g, (case["m"], k)) * scale
    if case["kind"] == "round":
        return x, None
    x *= 1 + 15 * (torch.rand((1, k), generator=g, device="cuda") > 0.99)
    x *= torch.exp2(torch.randint(-3, 2, (case["m"], 1), generator=g, device="cuda").float()).to(torch.bfloat16)
    return x, _normal(g, (case["n"], k)) * 0.02


def _positions(start, count):
    """(sequence, position) of every token of ragged runs, as index tensors."""
    seq = np.repeat(np.arange(len(count)), count)
    first = np.concatenate([[0], np.cumsum(count)])[:-1]
    return torch.from_numpy(seq).cuda(), torch.from_numpy(np.arange(int(count.sum())) - np.repeat(first - start, count)).cuda()


def _config(model):
    from paper_2601_11589_amd import inputs
    return {"tiny": inputs.tiny_cfg, "7b": inputs.qwen7b_cfg, "14b": inputs.qwen14b_cfg, "32b": inputs.qwen32b_cfg}[model](1)


def prepare(case, seed):
    st = _prepare_matrix(case, seed) if "k" in case else _prepare_cache(case, seed)
    if own:
        from paper_2601_11589_amd import api
        st["ctx"] = api.LapsCtx(_config(case.get("model", "tiny")), 64)
    torch.cuda.synchronize()
    return st


def _prepare_matrix(case, seed):
    x, w = _matrices(case, seed)
    st = dict(case=case, x=x)
    if w is not None:
        st["w"], st["w_scales"] = _plain_quant(w)
        st["out"] = torch.empty((case["m"], case["n"]), dtype=torch.bfloat16, device="cuda")
    if case["kind"] == "product":
        st["a"], st["a_scales"] = _plain_quant(x)
    return st


def _prepare_cache(case, seed):
    n_q, n_kv, hd = HEADS[case["model"]]
    new, pre, rows = _lengths(case)
    k, v, q = _tokens(case, seed)
    need = (new + pre + PAGE - 1) // PAGE
    width = int(need.max()) + case["spare"]
    g = np.random.default_rng([seed, case["mix"]])
    n_pages = int(need.sum()) + 7
    order = g.permutation(n_pages)
    table = np.full((len(new), max(width, 1)), -1)
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m]
        at += m
    st = dict(case=case, n_q=n_q, n_kv=n_kv, hd=hd, table=_i32(table), prefix=_i32(pre), cu=_i32(np.concatenate([[0], np.cumsum(rows)])),
              seq_len=_i32(new) if case["pad"] else None)
    gen = _generator(seed, 2)
    for name in ("k8", "v8"):
        pool = torch.empty((n_pages, n_kv * PAGE * hd + (n_kv + 127) // 128 * 128), dtype=torch.uint8, device="cuda")
        st[name] = pool.random_(0, 256, generator=gen)
    kept = pre if case["kind"] in ("step", "store") else new + pre       # what the pools hold before the pass
    seq, pos = _positions(np.zeros_like(kept), kept)
    whole = torch.from_numpy(np.concatenate([[0], np.cumsum(new + pre)])[:-1]).cuda()
    if len(seq):
        src = whole[seq] + pos
        _plain_store(st, seq, pos, k[src], v[src])
    if case["kind"] in ("step", "store"):
        seq, pos = _positions(pre, new)
        src = whole[seq] + pos
        st.update(k=k[src].contiguous(), v=v[src].contiguous(), cu_new=_i32(np.concatenate([[0], np.cumsum(new)])))
    n_tok = int(new.sum())
    if q is not None:
        st.update(q=q, out=torch.zeros_like(q))
    else:
        st.update(k_out=torch.empty((n_tok, n_kv, hd), dtype=torch.bfloat16, device="cuda"),
                  v_out=torch.empty((n_tok, n_kv, hd), dtype=torch.bfloat16, device="cuda"), n_tok=n_tok)
    return st


# ----------------------------------------------------------------------------------------------- the plain form
def _scale_byte(amax):
    """Byte e + 127 of the smallest e with amax <= 448 * 2^e, from a finite float32."""
    mantissa, exponent = torch.frexp(amax)          # amax = mantissa * 2^exponent, 448 = 0.875 * 2^9
    return (exponent - 9 + (mantissa > 0.875) + 127).masked_fill(amax == 0, 0).clamp(LOWEST, HIGHEST)


def _power(byte):
    return (byte.int() << 23).view(torch.float32)   # 2^(byte - 127)


def _encode(x, byte):
    """float32 values under scale bytes that broadcast against them -> codes."""
    y = x * _power(254 - byte)
    y = torch.where(torch.isfinite(x), y.clamp(-448, 448), float("nan"))
    return y.to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(codes, byte):
    return codes.view(torch.float8_e4m3fn).float() * _power(byte)


def _plain_quant(x):
    """bf16 [rows, k] -> codes uint8 [rows, k rounded up to 128], scale bytes uint8 [blocks, rows rounded up to 16]."""
    m, k = x.shape
    blocks = (k + BLOCK - 1) // BLOCK
    codes = torch.zeros((m, blocks * BLOCK), dtype=torch.uint8, device=x.device)
    scales = torch.full((blocks, (m + 15) // 16 * 16), 127, dtype=torch.uint8, device=x.device)
    for lo in range(0, m, 4096):
        y = torch.nn.functional.pad(x[lo:lo + 4096].float(), (0, blocks * BLOCK - k)).unflatten(-1, (blocks, BLOCK))
        byte = _scale_byte(torch.where(torch.isfinite(y), y.abs(), 0.0).amax(-1))
        codes[lo:lo + 4096] = _encode(y, byte[..., None]).flatten(-2)
        scales[:, lo:lo + len(y)] = byte.T.to(torch.uint8)
    return codes, scales


def _plain_dequant(codes, scales, lo=0, hi=None):
    """float32 [rows lo to hi, k rounded up to 128]."""
    part = codes[lo:hi].unflatten(-1, (-1, BLOCK))
    return _decode(part, scales.T[lo:lo + len(part), :, None]).flatten(-2)


def _codes_of(st, name, page):
    """Codes of whole pages, token-major [pages, 16, n_kv, hd], and scale bytes [pages, n_kv]."""
    n_kv, hd = st["n_kv"], st["hd"]
    held = st[name][page]
    codes, byte = held[:, :n_kv * PAGE * hd].unflatten(-1, (n_kv, PAGE * hd)), held[:, n_kv * PAGE * hd:n_kv * PAGE * hd + n_kv]
    if name == "k8":
        codes = codes.unflatten(-1, (PAGE, hd)).transpose(1, 2)
    else:                                                        # [hd / 4][4][hd % 4][4] -> [4][4][hd / 4][hd % 4]
        codes = codes.unflatten(-1, (hd // 4, 4, 4, 4)).permute(0, 3, 5, 1, 2, 4).flatten(1, 2).flatten(-2)
    return codes, byte


def _put_codes(st, name, page, codes, byte):
    n_kv, hd = st["n_kv"], st["hd"]
    if name == "k8":
        flat = codes.transpose(1, 2).flatten(-2)
    else:
        flat = codes.unflatten(-1, (hd // 4, 4)).unflatten(1, (4, 4)).permute(0, 3, 4, 1, 5, 2).flatten(2)
    st[name][page, :n_kv * PAGE * hd] = flat.flatten(1)
    st[name][page, n_kv * PAGE * hd:n_kv * PAGE * hd + n_kv] = byte.to(torch.uint8)


def _plain_store(st, seq, pos, k, v):
    """Tokens of runs, in order of (sequence, position)."""
    if len(seq) == 0:
        return
    place = seq * st["table"].shape[1] + pos // PAGE
    places, which = torch.unique_consecutive(place, return_inverse=True)
    for lo in range(0, len(places), 2048):
        mine = (which >= lo) & (which < lo + 2048)
        at, off = which[mine] - lo, pos[mine] % PAGE
        page = st["table"].flatten()[places[lo:lo + 2048]].long()
        first = torch.full((len(page),), PAGE, device=page.device, dtype=off.dtype).scatter_reduce(0, at, off, "amin")
        for name, x in (("k8", k[mine].float()), ("v8", v[mine].float())):
            fine = torch.isfinite(x).all(-1)                                       # a token's whole head, or none of it
            top = torch.where(fine, x.abs().amax(-1), 0.0)
            amax = torch.zeros((len(page), st["n_kv"]), device=x.device).index_reduce(0, at, top, "amax")
            byte = _scale_byte(amax)
            old, old_byte = _codes_of(st, name, page)
            old_byte = old_byte.int().clamp(LOWEST, HIGHEST)
            keeps = first > 0
            byte = torch.where(keeps[:, None], torch.maximum(byte, old_byte), byte)
            codes = torch.where(keeps[:, None, None, None], _encode(_decode(old, old_byte[:, None, :, None]), byte[:, None, :, None]), 0)
            codes[at, off] = _encode(torch.where(fine[..., None], x, float("nan")), byte[at][..., None])
            _put_codes(st, name, page, codes, byte)


def _plain_load(st, seq, pos):
    """float32 K and V of tokens that come in order of (sequence, position)."""
    place = seq * st["table"].shape[1] + pos // PAGE
    places, which = torch.unique_consecutive(place, return_inverse=True)
    page = st["table"].flatten()[places].long()
    out = []
    for name in ("k8", "v8"):
        codes, byte = _codes_of(st, name, page)
        out.append(_decode(codes[which, pos % PAGE], byte[which][..., None]))
    return out


def _ragged(start, count):
    """Sequence and position of every token of ragged runs (device index tensors)."""
    seq = torch.repeat_interleave(torch.arange(len(count), device="cuda"), count)
    first = torch.cumsum(count, 0) - count
    return seq, torch.arange(len(seq), device="cuda") - (first - start)[seq]


def _plain_matrix(st):
    case = st["case"]
    if case["kind"] == "round":
        codes, scales = _plain_quant(st["x"])
        return torch.cat([_plain_dequant(codes, scales, lo, lo + 4096)[:, :case["k"]].to(torch.bfloat16) for lo in range(0, case["m"], 4096)])
    a, a_scales = (st["a"], st["a_scales"]) if case["kind"] == "product" else _plain_quant(st["x"])
    x = _plain_dequant(a, a_scales)
    out = torch.empty_like(st["out"])
    for lo in range(0, case["n"], 8192):
        out[:, lo:lo + 8192] = (x @ _plain_dequant(st["w"], st["w_scales"], lo, lo + 8192).T).to(out.dtype)
    return out


def _plain(st):
    if "k" in st["case"]:
        return _plain_matrix(st)
    kind, n_kv, hd = st["case"]["kind"], st["n_kv"], st["hd"]
    group = st["n_q"] // n_kv
    if kind in ("store", "step"):
        seq, pos = _ragged(st["prefix"], st["cu_new"][1:] - st["cu_new"][:-1])
        _plain_store(st, seq, pos, st["k"], st["v"])
        if kind == "store":
            return tuple(t.to(torch.bfloat16) for t in _plain_load(st, seq, pos))
    cu, pre = st["cu"].tolist(), st["prefix"].tolist()
    new = [b - a for a, b in zip(cu, cu[1:])] if st["seq_len"] is None else st["seq_len"].tolist()
    out = torch.zeros_like(st["q"])
    for i, (n, h) in enumerate(zip(new, pre)):
        if n == 0:
            continue
        pos = torch.arange(h + n, device="cuda")
        k, v = _plain_load(st, torch.full_like(pos, i), pos)
        q = st["q"][cu[i]:cu[i] + n].float().view(n, n_kv, group, hd)
        hidden = pos[None, :] > (h + torch.arange(n, device="cuda"))[:, None]
        for j in range(n_kv):
            s = (q[:, j].reshape(n * group, hd) @ k[:, j].T).view(n, group, -1) * hd ** -0.5
            s = s.masked_fill(hidden[:, None], float("-inf"))
            p = torch.exp(s - s.amax(-1, keepdim=True))
            o = (p.view(n * group, -1) @ v[:, j]).view(n, group, hd) / p.sum(-1, keepdim=True)
            out.view(-1, n_kv, group, hd)[cu[i]:cu[i] + n, j] = o.to(torch.bfloat16)
    return out


# ----------------------------------------------------------------------------------------------- one pass
def run(st):
    if not own:
        return _plain(st)
    ctx, kind = st["ctx"], st["case"]["kind"]
    if kind == "linear":
        return ctx.laps_linear_fp8(st["x"], st["w"], st["w_scales"], out=st["out"])
    if kind == "product":
        return ctx.laps_gemm_fp8(st["a"], st["a_scales"], st["w"], st["w_scales"], out=st["out"])
    if kind == "round":
        codes, scales = ctx.laps_fp8_quant(st["x"])
        return ctx.laps_fp8_dequant(codes, scales, st["case"]["k"])
    if kind in ("store", "step"):
        ctx.laps_kv8_scatter(st["cu_new"], st["prefix"], st["table"], st["k"], st["v"], st["k8"], st["v8"])
    if kind == "store":
        return ctx.laps_kv8_gather(st["cu_new"], st["prefix"], st["table"], st["k8"], st["v8"], st["n_tok"], st["k_out"], st["v_out"])
    return ctx.laps_attention_kv8(st["cu"], st["seq_len"], st["prefix"], st["table"], st["k8"], st["v8"], st["q"], out=st["out"])


def work(case):
    if "k" in case:
        m, n, k = case["m"], case["n"], case["k"]
        if case["kind"] == "round":
            return {"bytes": 2 * m * (3 * k + k // BLOCK), "flops": 0}
        rows = m * k * (1 if case["kind"] == "product" else 2)
        return {"bytes": rows + n * (k + k // BLOCK) + 2 * m * n, "flops": 2 * m * n * k}
    n_q, n_kv, hd = HEADS[case["model"]]
    new, pre, _ = (np.asarray(a, dtype=np.int64) for a in _lengths(case))
    token8 = 2 * n_kv * hd           # a token of both pools, the scales aside
    token16 = 2 * n_kv * hd * 2      # the same in bf16
    stored = int(new.sum()) * (token8 + token16) if case["kind"] in ("store", "step") else 0
    if case["kind"] == "store":
        return {"bytes": 2 * stored, "flops": 0}
    live = new > 0
    cached = int((new + pre)[live].sum()) * token8
    return {"bytes": stored + cached + 4 * int(new.sum()) * n_q * hd, "flops": int(4 * hd * n_q * (new * pre + new * (new + 1) // 2).sum())}


# ----------------------------------------------------------------------------------------------- in 64 bits
def _exponent64(amax):
    """The smallest e with amax <= 448 * 2^e, cut to its range, in float64."""
    e = torch.ceil(torch.log2(amax / 448))
    e = torch.where(amax > 448 * torch.exp2(e), e + 1, e)
    e = torch.where(amax <= 448 * torch.exp2(e - 1), e - 1, e)
    return torch.nan_to_num(e, neginf=-116.0).clamp(-116, 119)


def _rounded64(x, e):
    """x under the scale 2^e to the nearest 8-bit float, ties to even, in float64."""
    y = x / torch.exp2(e)
    binade = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(binade - 3)
    return (torch.round(y / step) * step).clamp(-448, 448) * torch.exp2(e)


def _matrix64(x):
    m, k = x.shape
    out = torch.empty((m, k), dtype=torch.float64, device=x.device)
    for lo in range(0, k, BLOCK):
        part = x[:, lo:lo + BLOCK].double()
        out[:, lo:lo + BLOCK] = _rounded64(part, _exponent64(part.abs().amax(1, keepdim=True)))
    return out


def _history64(x, first):
    """What a cache holds of one sequence's tokens [n, n_kv, hd] where those from `first` on were written behind the others."""
    n = len(x)
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    whole = first // PAGE * PAGE
    head = -(-n // PAGE) * PAGE - n
    pages = torch.cat([x, x.new_zeros((head,) + x.shape[1:])]).double().unflatten(0, (-1, PAGE))
    e = _exponent64(pages.abs().amax((1, 3), keepdim=True))
    out = _rounded64(pages, e).flatten(0, 1)[:n]
    if whole < first < n:     # the page that both runs share: its first tokens were rounded for themselves before
        old, late = x[whole:first].double(), x[first:whole + PAGE].double()
        e_old = _exponent64(old.abs().amax((0, 2), keepdim=True))
        e_all = torch.maximum(e_old, _exponent64(late.abs().amax((0, 2), keepdim=True)))
        out[whole:first] = _rounded64(_rounded64(old, e_old), e_all)
        out[first:whole + PAGE] = _rounded64(late, e_all)
    return out


def exact(case, seed):
    if "k" in case:
        x, w = _matrices(case, seed)
        if case["kind"] == "round":
            return torch.cat([_matrix64(part) for part in x.split(4096)])
        x = _matrix64(x)
        return torch.cat([x @ _matrix64(part).T for part in w.split(8192)], 1)
    n_q, n_kv, hd = HEADS[case["model"]]
    new, pre, rows = _lengths(case)
    k, v, q = _tokens(case, seed)
    ends = np.cumsum(new + pre)
    split = case["kind"] in ("store", "step")
    held = []
    for e, n, h in zip(ends.tolist(), new.tolist(), pre.tolist()):
        held.append([_history64(t[e - n - h:e], h if split else n + h) for t in (k, v)])
    if q is None:
        return tuple(torch.cat([pair[i][h:] for pair, h in zip(held, pre.tolist())]) for i in (0, 1))
    out = torch.zeros((q.shape[0], n_q * hd), dtype=torch.float64, device="cuda")
    row = np.cumsum(rows) - rows
    for i in range(len(new)):
        n, h, r = int(new[i]), int(pre[i]), int(row[i])
        if n == 0:
            continue
        keys, values = held[i]
        sees = torch.tril(torch.ones((n, n + h), dtype=torch.bool, device="cuda"), diagonal=h)
        for head in range(n_q):
            at, j = slice(head * hd, (head + 1) * hd), head // (n_q // n_kv)
            s = torch.where(sees, q[r:r + n, at].double() @ keys[:, j].T / math.sqrt(hd), -math.inf)
            out[r:r + n, at] = torch.softmax(s, -1) @ values[:, j]
    return out
