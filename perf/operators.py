"""The 4-bit K/V cache and the attention that reads it, as measurable cases.

Three operators, each through the public binding (`paper_2601_11589_amd.api`):

* laps_kv4_scatter     token-major bf16 K/V quantised into 4-bit pools
* laps_kv4_gather      4-bit pools read back to token-major bf16 K/V
* laps_attention_kv4   ragged paged causal grouped-query attention over 4-bit pools

The cache holds groups of 32 values along head_dim of one token and kv head: a scale 2^e (one byte, e + 127) and 4-bit
floats with magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6.  e is the smallest integer with max |x| <= 7 * 2^e, cut to [-126, 125]; x / 2^e is
rounded to nearest, ties to the even code, magnitudes above 6 to 6.  A page of 16 tokens and one kv head is a block of
8.5 * head_dim bytes:

    K  codes [16 tokens][head_dim / 2]               scales [16 tokens][head_dim / 32]
    V  codes [head_dim / 8][16 tokens][4 bytes]      scales [head_dim / 32][16 tokens]

with two values a byte, the lower index in the lower half.

Kinds of pass:

* store    tokens into the pools and the same tokens back out: a hand-over of finished K/V through a 4-bit cache
* read     whole histories out of the pools
* attend   attention alone, the new tokens' K/V in the pools already
* step     one serving step: the new tokens' K/V into the pools, then the attention that sees them

Lengths come from the case alone (`mix` seeds them), values from the seed.  Pages lie in random order and the pools' unused slots
hold stale bytes, as in a server that has run for a while.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
GROUP = 32
HEADS = {"tiny": (4, 2, 64), "7b": (28, 4, 128), "14b": (40, 8, 128), "32b": (40, 8, 128)}   # query heads, kv heads, head_dim
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ----------------------------------------------------------------------------------------------- the cases
def _case(name, kind, model, n_seq, new, pre, fresh=0.0, pad=False, spare=0, mix=1):
    return dict(name=name, kind=kind, model=model, n_seq=n_seq, new_lo=new[0], new_hi=new[1], pre_lo=pre[0], pre_hi=pre[1],
                fresh=fresh, pad=pad, spare=spare, mix=mix)


def listed():
    return [
        # the smallest call: one conversation of an idle server writes and reads one token; launches count
        _case("store_one_7b", "store", "7b", 1, (1, 1), (900, 900)),
        # finished prompts handed over through the 4-bit cache, beginning and ending inside pages
        _case("store_prompts_32b", "store", "32b", 8, (512, 4096), (0, 40), mix=3),
        # whole conversations read back to bf16, to go on in bf16 pools
        _case("read_back_32b", "read", "32b", 8, (1024, 8192), (0, 0), mix=5),
        # the small test model: ragged turns, sequences without a token, padding rows between the sequences (head_dim 64)
        _case("tiny_ragged", "attend", "tiny", 12, (0, 40), (0, 300), fresh=0.25, pad=True, mix=7),
        # one token of one conversation: the latency of a decode step; a page table for 8192 tokens
        _case("token_one_7b", "step", "7b", 1, (1, 1), (900, 900), spare=450),
        # one token of many conversations: the cache is all the traffic
        _case("token_batch_32b", "step", "32b", 64, (1, 1), (512, 8191), mix=9),
        # one token over two very long histories: the key axis is all the parallelism there is
        _case("token_long_7b", "attend", "7b", 2, (1, 1), (100000, 131071), mix=11),
        # a few drafted tokens of each conversation verified at once
        _case("verify_14b", "attend", "14b", 16, (2, 5), (100, 6000), mix=13),
        # one short turn over a long cached history, alone
        _case("one_turn_14b", "attend", "14b", 1, (16, 16), (4000, 4000)),
        # the re-prefill workload of the benchmark: short turns over cached histories
        _case("reprefill_32b", "attend", "32b", 16, (17, 64), (512, 4096), mix=15),
        # first chunk of a long prompt
        _case("chunk_first_32b", "step", "32b", 1, (2048, 2048), (0, 0)),
        # ragged last chunk of the longest prompt of the benchmark
        _case("chunk_last_32b", "attend", "32b", 1, (1847, 1847), (6144, 6144)),
    ]


MOST_STORED = 16384     # tokens of the largest store or read
MOST_CACHED = 131072    # cached tokens of all sequences of the largest attention
MOST_PAIRS = 12 << 20   # (new token, cached token) pairs of the largest attention


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    kind = rng.choice(["store", "read", "token", "token", "few", "turn", "turn", "chunk", "mixed"])
    model = rng.choice(["tiny", "7b", "14b", "32b"])
    mix = rng.randrange(1 << 30)
    if kind in ("store", "read"):
        hi = _log(rng, 1, 8192)
        n = min(_log(rng, 1, 256), max(1, MOST_STORED // hi))
        c = _case("", kind, model, n, (rng.randint(1, hi), hi), (0, rng.choice([0, 40])) if kind == "store" else (0, 0), mix=mix)
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


def _inputs(case, seed):
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


def _positions(start, count):
    """(sequence, position) of every token of ragged runs, as index tensors."""
    seq = np.repeat(np.arange(len(count)), count)
    first = np.concatenate([[0], np.cumsum(count)])[:-1]
    return seq, np.arange(int(count.sum())) - np.repeat(first - start, count)


def prepare(case, seed):
    n_q, n_kv, hd = HEADS[case["model"]]
    new, pre, rows = _lengths(case)
    k, v, q = _inputs(case, seed)
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
    st = dict(case=case, n_q=n_q, n_kv=n_kv, hd=hd, table=_i32(table), prefix=_i32(pre), seed=seed,
              cu=_i32(np.concatenate([[0], np.cumsum(rows)])), seq_len=_i32(new) if case["pad"] else None)
    gen = _generator(seed, 2)
    for name in ("k4", "v4"):
        pool = torch.empty((n_pages, n_kv, hd // 2 * 17), dtype=torch.uint8, device="cuda")
        st[name] = pool.random_(0, 256, generator=gen)
    kept = pre if case["kind"] in ("step", "store") else new + pre       # what the pools hold before the pass
    seq, pos = _positions(np.zeros_like(kept), kept)
    whole = np.concatenate([[0], np.cumsum(new + pre)])[:-1]
    if len(seq):
        src = torch.from_numpy(whole[seq] + pos).cuda()
        _plain_store(st, torch.from_numpy(seq).cuda(), torch.from_numpy(pos).cuda(), k[src], v[src])
    if case["kind"] in ("step", "store"):
        seq, pos = _positions(pre, new)
        src = torch.from_numpy(whole[seq] + pos).cuda()
        st.update(k=k[src].contiguous(), v=v[src].contiguous(), cu_new=_i32(np.concatenate([[0], np.cumsum(new)])))
    n_tok = int(new.sum())
    if q is not None:
        st.update(q=q, out=torch.zeros_like(q))
    else:
        st.update(k_out=torch.empty((n_tok, n_kv, hd), dtype=torch.bfloat16, device="cuda"),
                  v_out=torch.empty((n_tok, n_kv, hd), dtype=torch.bfloat16, device="cuda"), n_tok=n_tok)
    if own:
        from paper_2601_11589_amd import api, inputs
        cfg = {"tiny": inputs.tiny_cfg, "7b": inputs.qwen7b_cfg, "14b": inputs.qwen14b_cfg, "32b": inputs.qwen32b_cfg}
        st["ctx"] = api.LapsCtx(cfg[case["model"]](1), 64)
    torch.cuda.synchronize()
    return st


# ----------------------------------------------------------------------------------------------- the plain form
def _quantise(x):
    """bf16 [..., hd] -> packed codes uint8 [..., hd / 2], scale bytes uint8 [..., hd / 32]."""
    y = x.float().unflatten(-1, (-1, GROUP))
    top = y.abs().amax(-1)
    bits = top.view(torch.int32)
    byte = ((bits >> 23) - 2 + (((bits >> 16) & 127) > 96)).clamp(1, 252)
    byte = torch.where((bits >> 23) == 255, 255, byte)
    inverse = ((254 - byte.clamp(max=252)) << 23).view(torch.float32)       # 2^-e
    mag = y.abs() * inverse[..., None]
    code = ((mag > 0.25).int() + (mag >= 0.75) + (mag > 1.25) + (mag >= 1.75) + (mag > 2.5) + (mag >= 3.5) + (mag > 5.0))
    code = code | (torch.signbit(y).int() << 3)
    code = torch.where((byte == 255)[..., None], 0, code).flatten(-2)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8), byte.to(torch.uint8)


def _value(codes, byte):
    """The inverse: float32 [..., hd]."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float32, device=codes.device)
    scale = torch.where(byte == 255, float("nan"), (byte.int() << 23).view(torch.float32))
    return (table[code.long()].unflatten(-1, (-1, GROUP)) * scale[..., None]).flatten(-2)


def _views(st):
    hd = st["hd"]
    cut = 8 * hd
    kc, ks = st["k4"][..., :cut].unflatten(-1, (PAGE, hd // 2)), st["k4"][..., cut:].unflatten(-1, (PAGE, hd // GROUP))
    vc, vs = st["v4"][..., :cut].unflatten(-1, (hd // 8, PAGE, 4)), st["v4"][..., cut:].unflatten(-1, (hd // GROUP, PAGE))
    return kc, ks, vc, vs


def _plain_store(st, seq, pos, k, v):
    kc, ks, vc, vs = _views(st)
    page, off = st["table"][seq, pos // PAGE].long(), pos % PAGE
    for lo in range(0, len(seq), 1 << 16):
        at = slice(lo, lo + (1 << 16))
        kc[page[at], :, off[at]], ks[page[at], :, off[at]] = _quantise(k[at])
        codes, byte = _quantise(v[at])
        vc[page[at], :, :, off[at]] = codes.unflatten(-1, (-1, 4))
        vs[page[at], :, :, off[at]] = byte


def _plain_load(st, seq, pos):
    kc, ks, vc, vs = _views(st)
    page, off = st["table"][seq, pos // PAGE].long(), pos % PAGE
    return (_value(kc[page, :, off], ks[page, :, off]),
            _value(vc[page, :, :, off].flatten(-2), vs[page, :, :, off]))


def _ragged(start, count):
    """Sequence and position of every token of ragged runs (device index tensors)."""
    seq = torch.repeat_interleave(torch.arange(len(count), device="cuda"), count)
    first = torch.cumsum(count, 0) - count
    return seq, torch.arange(len(seq), device="cuda") - (first - start)[seq]


def _plain(st):
    kind, n_kv, hd = st["case"]["kind"], st["n_kv"], st["hd"]
    group = st["n_q"] // n_kv
    if kind in ("store", "step"):
        count = st["cu_new"][1:] - st["cu_new"][:-1]
        seq, pos = _ragged(st["prefix"], count)
        _plain_store(st, seq, pos, st["k"], st["v"])
        if kind == "store":
            return tuple(t.to(torch.bfloat16) for t in _plain_load(st, seq, pos))
    if kind == "read":
        parts = [_plain_load(st, s, p) for s, p in zip(*(t.split(1 << 15) for t in _ragged(st["prefix"], st["cu"][1:] - st["cu"][:-1])))]
        return tuple(torch.cat([p[i].to(torch.bfloat16) for p in parts]) for i in (0, 1))
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
    if kind in ("store", "step"):
        ctx.laps_kv4_scatter(st["cu_new"], st["prefix"], st["table"], st["k"], st["v"], st["k4"], st["v4"])
    if kind == "store":
        return ctx.laps_kv4_gather(st["cu_new"], st["prefix"], st["table"], st["k4"], st["v4"], st["n_tok"], st["k_out"], st["v_out"])
    if kind == "read":
        return ctx.laps_kv4_gather(st["cu"], st["prefix"], st["table"], st["k4"], st["v4"], st["n_tok"], st["k_out"], st["v_out"])
    return ctx.laps_attention_kv4(st["cu"], st["seq_len"], st["prefix"], st["table"], st["k4"], st["v4"], st["q"], out=st["out"])


def work(case):
    n_q, n_kv, hd = HEADS[case["model"]]
    new, pre, _ = (np.asarray(a, dtype=np.int64) for a in _lengths(case))
    token4 = 2 * n_kv * (hd // 2 + hd // GROUP)      # a token of both pools
    token16 = 2 * n_kv * hd * 2                      # the same in bf16
    tokens = int(new.sum())
    if case["kind"] == "read":
        return {"bytes": tokens * (token4 + token16), "flops": 0}
    stored = tokens * (token4 + token16) if case["kind"] in ("store", "step") else 0
    if case["kind"] == "store":
        return {"bytes": 2 * stored, "flops": 0}
    live = new > 0
    cached = int((new + pre)[live].sum()) * token4
    return {"bytes": stored + cached + 4 * tokens * n_q * hd, "flops": int(4 * hd * n_q * (new * pre + new * (new + 1) // 2).sum())}


# ----------------------------------------------------------------------------------------------- in 64 bits
def _cached64(x):
    """What a 4-bit cache holds of x, in float64: every group over its scale to the nearest 4-bit float, ties to even."""
    y = x.double().unflatten(-1, (-1, GROUP))
    top = y.abs().amax(-1, keepdim=True)
    e = torch.frexp(top)[1].double() - 3
    e = torch.where(top > 7 * torch.exp2(e), e + 1, e).clamp(-126, 125)
    z = y / torch.exp2(e)
    step = torch.where(z.abs() < 2, 0.5, torch.where(z.abs() < 4, 1.0, 2.0))
    z = (torch.round(z / step) * step).clamp(-6, 6)
    return (z * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    n_q, n_kv, hd = HEADS[case["model"]]
    new, pre, rows = _lengths(case)
    k, v, q = _inputs(case, seed)
    ends = np.cumsum(new + pre)
    if q is None:
        mine = torch.cat([torch.arange(e - n, e) for e, n in zip(ends, new)]).cuda()
        return _cached64(k[mine]), _cached64(v[mine])
    out = torch.zeros((q.shape[0], n_q * hd), dtype=torch.float64, device="cuda")
    row = np.cumsum(rows) - rows
    for i in range(len(new)):
        n, h, r = int(new[i]), int(pre[i]), int(row[i])
        if n == 0:
            continue
        keys, values = (_cached64(t[ends[i] - n - h:ends[i]]) for t in (k, v))
        sees = torch.tril(torch.ones((n, n + h), dtype=torch.bool, device="cuda"), diagonal=h)
        for head in range(n_q):
            at, j = slice(head * hd, (head + 1) * hd), head // (n_q // n_kv)
            s = torch.where(sees, q[r:r + n, at].double() @ keys[:, j].T / math.sqrt(hd), -math.inf)
            out[r:r + n, at] = torch.softmax(s, -1) @ values[:, j]
    return out
