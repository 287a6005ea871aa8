"""Performance cases of the cache-side operators beside the compression: new tokens entering a cache with their position
rotation, attention over a sliding window with a few first tokens that stay visible, and attention for a batch whose
sequences share a long prefix.

Kinds of case:
  append  the new tokens' keys are rotated by their positions and enter the caches with their values; their queries are
          rotated on the way.  One token per sequence, or prompts of different lengths packed one after the other.
  window  attention of the new tokens over the caches that hold them already: token t sees the cached rows up to its own
          that lie among the last `window` (0: all) or among the first `sinks`.
  prefix  one decode step of a batch that was sampled from a few prompts: every sequence attends over its prompt's keys and
          values, which are stored once, and over its own cache.

Caches are [batch, kv_heads, capacity, dim], or pools of pages of 128 rows.  Keys: N(0, 1) with four outlier channels per
KV head scaled by 8; queries and values N(0, 1).  `run` computes the plain form, or the library's calls where `own` is set.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}
ESIZE = {"bf16": 2, "f32": 4, "fp8": 1}
PAGE = 128
BASE = 500000.0         # of the rotation's frequencies
E4M3_MAX = 448.0


def _case(name, kind, batch, kv_heads, q_heads, dim, dtype, cached, new, ragged=False, paged=False, window=0, sinks=0,
          rotary=None, interleaved=False, fused=False, prefix=0, prefixes=1, mix=0):
    """cached: rows of a sequence's cache before the call; new: its new tokens (ragged: at most that many of either)."""
    c = dict(kind=kind, batch=batch, kv_heads=kv_heads, q_heads=q_heads, dim=dim, dtype=dtype, cached=cached, new=new,
             ragged=ragged, paged=paged, window=window, sinks=sinks, rotary=dim if rotary is None else rotary,
             interleaved=interleaved, fused=fused, prefix=prefix, prefixes=prefixes, mix=mix)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token of a single conversation enters one layer's cache: all latency
        _case("append_step_b1", "append", 1, 8, 32, 128, "bf16", 1100, 1),
        # one token of 64 sequences of different lengths, paged caches
        _case("append_step_b64_paged", "append", 64, 4, 28, 128, "bf16", 2100, 1, ragged=True, paged=True),
        # a batch of prompts of different lengths out of a fused projection, into 8-bit pages, pairs side by side
        _case("append_prompts_fp8_paged", "append", 16, 8, 32, 128, "fp8", 0, 4096, ragged=True, paged=True, interleaved=True,
              fused=True, mix=3),
        # sixteen long prompts at once
        _case("append_prompts_b16", "append", 16, 8, 40, 128, "bf16", 0, 4096),
        # one token of a single conversation, a window of a thousand
        _case("window_step_b1", "window", 1, 8, 32, 128, "bf16", 4100, 1, window=1024, sinks=4),
        # one token of 64 sequences, seven queries per KV head, 8-bit caches
        _case("window_step_b64_fp8", "window", 64, 4, 28, 128, "fp8", 4200, 1, ragged=True, window=2048, sinks=4, mix=1),
        # prompts of different lengths, heads of 64 dimensions
        _case("window_prompts_d64", "window", 8, 8, 32, 64, "bf16", 0, 2048, ragged=True, window=512, sinks=4, mix=2),
        # the next piece of a long prompt over what is cached of it already, no window, paged
        _case("window_chunk_full", "window", 2, 4, 28, 128, "bf16", 7000, 1000, paged=True),
        # two long prompts, five queries per KV head
        _case("window_prompts_long", "window", 2, 8, 40, 128, "bf16", 0, 8192, window=2048, sinks=4),
        # a handful of samples of a short prompt
        _case("prefix_b8_short", "prefix", 8, 4, 28, 128, "bf16", 150, 1, ragged=True, prefix=333),
        # 64 samples of one question
        _case("prefix_b64", "prefix", 64, 8, 32, 128, "bf16", 1152, 1, ragged=True, prefix=2048, mix=4),
        # 256 samples of four long documents, caches compressed to a thousand tokens
        _case("prefix_b256_long", "prefix", 256, 8, 32, 128, "bf16", 1152, 1, prefix=16000, prefixes=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "window", "window", "prefix"])
    dtype = rng.choice(["bf16"] * 6 + ["fp8"] * 2 + ["f32"])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    group = rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
    q_heads = kv_heads * group
    paged, ragged, mix = rng.random() < 0.3, rng.random() < 0.6, rng.randrange(1 << 16)
    if kind == "append":
        dim = rng.choice([128] * 5 + [64] * 2 + [256])
        step = rng.random() < 0.5
        new = 1 if step else _log(rng, 2, 4096)
        cached = _log(rng, 1, 4000) if step or rng.random() < 0.3 else 0
        # at most the largest listed case's elements, new and cached
        most = 16 * 4096 * 56 * 128 // (2 if dtype == "f32" else 1)
        row = max((q_heads + 2 * kv_heads) * new, 2 * kv_heads * (new + cached)) * dim
        batch = _log(rng, 1, max(1, min(256, most // row)))
        return _case(None, kind, batch, kv_heads, q_heads, dim, dtype, cached, new, ragged, paged, rotary=rng.choice([dim, dim, dim // 2]),
                     interleaved=rng.random() < 0.3, fused=rng.random() < 0.4, mix=mix)
    dim = 64 if dtype == "bf16" and rng.random() < 0.25 else 128
    if kind == "prefix":
        # few samples of a short prompt up to what the largest listed case reads and multiplies
        small = dtype == "f32"
        prefix = _log(rng, 1, 2000 if small else 16000)
        cached = _log(rng, 1, 500 if small else 4000)
        most = 256 * 8 * 1152 // (8 if small else 1)
        batch = _log(rng, 1, max(1, min(256, most // (kv_heads * cached), (1 << 25) // (q_heads * prefix))))
        prefixes = rng.choice([p for p in (1, 1, 1, 2, 4) if batch % p == 0])
        return _case(None, kind, batch, kv_heads, q_heads, dim, dtype, cached, 1, ragged, paged, prefix=prefix, prefixes=prefixes, mix=mix)
    step = rng.random() < 0.5
    small = dtype == "f32"
    new = 1 if step else _log(rng, 2, 1000 if small else 8000)
    cached = _log(rng, 1, 7000) if step or rng.random() < 0.4 else 0
    window, sinks = rng.choice([0, _log(rng, 1, 4096), _log(rng, 16, 4096)]), rng.choice([0, 1, 4, 4, 130])
    # score entries of the plain form, and rows held
    entries = 1 << 29 if small else 9 << 27
    while q_heads * new * (new + cached) > entries:
        new, cached = (new + 1) // 2, cached // 2
    length = new + cached
    most = min(entries // (q_heads * new * length), (1 << 22) // (kv_heads * length) if step else 64)
    batch = _log(rng, 1, max(1, min(128, most)))
    return _case(None, kind, batch, kv_heads, q_heads, dim, dtype, cached, new, ragged, paged, window, sinks, mix=mix)


def _lengths(c):
    """Rows cached before the call and new tokens, per sequence; a property of the case, not of the inputs."""
    rng, n = random.Random(1000003 * c["mix"] + c["batch"]), c["batch"]
    if not c["ragged"]:
        return [c["cached"]] * n, [c["new"]] * n
    cached = [rng.randint(0 if c["new"] > 1 else min(1, c["cached"]), c["cached"]) for _ in range(n)]
    new = [c["new"] if c["new"] == 1 else rng.randint(1, c["new"]) for _ in range(n)]
    at = rng.randrange(n)
    cached[at], new[at] = c["cached"], c["new"]              # one sequence has all of it
    if c["kind"] == "window" or c["kind"] == "append" and c["new"] > 1:
        return cached, new
    if n > 2:
        cached[(at + 1) % n] = 0                             # and one an empty cache
    return cached, new


def _capacity(c):
    cap = c["cached"] + (0 if c["kind"] == "prefix" else c["new"]) + 28
    return -(-cap // PAGE) * PAGE if c["paged"] else cap


def _frequencies(c):
    return [BASE ** (-2.0 * i / c["rotary"]) for i in range(c["rotary"] // 2)]


# ---------------------------------------------------------------------------------------------------- inputs
def _normal(shape, gen, dtype):
    big = math.prod(shape) > 1 << 28
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16 if big else torch.float32)
    return x.to(dtype)


def _keys(shape, gen, dtype):
    scale = torch.ones(shape[1], shape[-1], device="cuda")
    scale.scatter_(-1, torch.rand(shape[1], shape[-1], generator=gen, device="cuda").argsort(-1)[:, :4], 8.0)
    return _normal(shape, gen, torch.bfloat16 if dtype != torch.float32 else dtype).mul_(scale[:, None].to(torch.bfloat16)).to(dtype)


def _bits(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    B, H, Hq, d, cap = c["batch"], c["kv_heads"], c["q_heads"], c["dim"], _capacity(c)
    cached, new = _lengths(c)
    store, wide = DTYPES[c["dtype"]], torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    total = sum(new)
    s = {"case": c, "cap": cap, "total": total, "longest": max(new)}
    s["k"], s["v"] = _keys((B, H, cap, d), gen, store), _normal((B, H, cap, d), gen, store)
    s["table"] = None
    if c["paged"]:                              # a head's pages lie anywhere in the pool
        table = torch.randperm(B * H * cap // PAGE, generator=gen, device="cuda")
        for x in "kv":
            pool = torch.empty(table.numel(), PAGE, d, dtype=store, device="cuda")
            _bits(pool)[table] = _bits(s[x]).view(-1, PAGE, d)
            s[x] = pool
        s["table"] = table.view(B, H, -1).to(torch.int32)
    s["offsets"] = i32([sum(new[:b]) for b in range(B + 1)])
    s["before"] = i32(cached)
    if c["kind"] == "append":
        qkv = _normal((total, Hq + 2 * H, d), gen, wide)
        parts = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        s["q_new"], s["k_new"], s["v_new"] = parts if c["fused"] else [x.contiguous() for x in parts]
        s["q_out"] = torch.empty(total, Hq, d, dtype=wide, device="cuda")
        s["lens"] = s["before"].clone()
        # a compressed cache holds fewer rows than there were tokens: positions run ahead of the rows
        ahead = torch.randint(0, 1 << 15, (B,), generator=gen, device="cuda", dtype=torch.int32)
        s["positions"] = torch.where(s["before"] > 0, s["before"] + ahead, 0).to(torch.int32)
        angle = torch.arange((1 << 15) + cap, device="cuda", dtype=torch.float64)[:, None] * torch.tensor(
            _frequencies(c), dtype=torch.float64, device="cuda")
        s["angles"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    else:
        s["q"] = _normal((total, Hq, d), gen, wide)
        s["out"] = torch.empty(total, Hq, d, dtype=wide, device="cuda")
        s["lens"] = i32([a if c["kind"] == "prefix" else a + b for a, b in zip(cached, new)])
    if c["kind"] == "prefix":
        n = c["prefixes"]
        s["pk"], s["pv"] = _keys((n, H, c["prefix"], d), gen, store), _normal((n, H, c["prefix"], d), gen, store)
        s["prefix_lens"] = i32([c["prefix"]] * n)
    if own:
        _plan(s)
    return s


def _plan(s):
    """The descriptors and the workspace that a program keeps."""
    import paper_2505_24133_b200 as rkv
    c = s["case"]
    d = rkv.rkv_desc_default()
    d.batch, d.n_kv_heads, d.n_q_heads, d.head_dim = c["batch"], c["kv_heads"], c["q_heads"], c["dim"]
    d.dtype = {"bf16": rkv.RKV_BF16, "f32": rkv.RKV_F32, "fp8": rkv.RKV_FP8_E4M3}[c["dtype"]]
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    d.device_status = s["status"].data_ptr()
    if s["table"] is not None:
        d.block_table, d.pool_pages = s["table"].data_ptr(), s["k"].shape[0]
    budget, buffer = s["cap"] - 28, 28
    s["rkv"], s["desc"], s["room"] = rkv, d, (budget, buffer)
    stride = {x + "_stride": s[x + "_new"].stride(0) for x in "qkv"} if c["fused"] else {}
    one = c["new"] == 1
    s["tokens"] = rkv.rkv_tokens(s["total"], s["longest"], None if one else s["offsets"], **stride)
    nbytes = 0
    if c["kind"] == "append":
        s["rotary"] = rkv.rkv_rotary(s["angles"], c["rotary"], s["positions"], interleaved=c["interleaved"])
    elif c["kind"] == "window":
        nbytes = rkv.rkv_window_workspace_bytes(d, budget, buffer, s["tokens"], c["window"], c["sinks"])
    else:
        s["prefix"] = rkv.rkv_prefix(s["pk"], s["pv"], s["prefix_lens"])
        nbytes = rkv.rkv_prefix_workspace_bytes(d, budget, buffer, s["prefix"])
    s["workspace"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda")
    d.workspace, d.workspace_bytes = s["workspace"].data_ptr(), s["workspace"].numel()


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    if c["kind"] == "append":
        s["lens"].copy_(s["before"])            # the same tokens enter at the same rows again
        if own:
            _ok(s, s["rkv"].rkv_append_rotary(s["desc"], s["k"], s["v"], s["k_new"], s["v_new"], s["lens"], *s["room"], s["tokens"],
                                              s["rotary"], s["q_new"], s["q_out"]))
        else:
            _append(s)
        return {"k": s["k"], "v": s["v"], "q": s["q_out"], "lens": s["lens"]}
    if own:
        if c["kind"] == "window":
            _ok(s, s["rkv"].rkv_window_attention(s["desc"], s["k"], s["v"], s["q"], s["lens"], s["out"], *s["room"], s["tokens"],
                                                 c["window"], c["sinks"]))
        else:
            _ok(s, s["rkv"].rkv_prefix_attention(s["desc"], s["k"], s["v"], s["q"], s["lens"], s["out"], *s["room"], s["prefix"]))
        return s["out"]
    return _window(s) if c["kind"] == "window" else _prefix(s)


def _ok(s, rc):
    if rc != 0:
        raise RuntimeError(s["rkv"].rkv_status_string(rc))


def _rotate(x, angles, c):
    """x [tokens, heads, dim] in 32 bits; angles [tokens, rotary]: the cosines, then the sines."""
    half = c["rotary"] // 2
    cos, sin = angles[:, None, :half], angles[:, None, half:]
    r = x[..., :c["rotary"]]
    if c["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = r[..., :half], r[..., half:]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., c["rotary"]:]], -1)


def _store(x, c):
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn) if c["dtype"] == "fp8" else x.to(DTYPES[c["dtype"]])


def _append(s):
    c = s["case"]
    H, cap = c["kv_heads"], s["cap"]
    off = s["offsets"].long()
    seq = torch.searchsorted(off[1:], torch.arange(s["total"], device="cuda"), right=True)
    nth = torch.arange(s["total"], device="cuda") - off[seq]
    angles = s["angles"][s["positions"][seq] + nth]
    row = s["before"][seq] + nth
    head = torch.arange(H, device="cuda")
    if s["table"] is None:
        at = (seq[:, None] * H + head) * cap + row[:, None]
    else:
        at = s["table"][seq[:, None], head, row[:, None] // PAGE].long() * PAGE + row[:, None] % PAGE
    at = at.flatten()
    k, v = _store(_rotate(s["k_new"].float(), angles, c), c), _store(s["v_new"].float(), c)
    _bits(s["k"]).view(-1, c["dim"])[at] = _bits(k).view(-1, c["dim"])
    _bits(s["v"]).view(-1, c["dim"])[at] = _bits(v).view(-1, c["dim"])
    s["q_out"].copy_(_rotate(s["q_new"].float(), angles, c))
    s["lens"].add_(s["offsets"].diff())


def _rows(s, name, b0, b1):
    """The caches of sequences b0 .. b1 as [n, kv_heads, capacity, dim] in 32 bits."""
    if s["table"] is None:
        return s[name][b0:b1].float()
    n = b1 - b0
    return s[name].view(torch.uint8)[s["table"][b0:b1].flatten().long()].view(s[name].dtype).view(n, s["table"].shape[1], -1, s["case"]["dim"]).float()


def _softmax(x):
    """Over the last axis, in place; a row without a visible entry (all -inf) gives zeros."""
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    return x.div_(x.sum(-1, keepdim=True).clamp_min_(1e-30))


def _window(s):
    c = s["case"]
    B, H, Hq, d, n = c["batch"], c["kv_heads"], c["q_heads"], c["dim"], s["longest"]
    G = Hq // H
    off, fresh = s["offsets"].long(), s["offsets"].diff().long()
    out = s["out"]
    step = max(1, (1 << 30) // (Hq * n * s["cap"]))
    key = torch.arange(s["cap"], device="cuda")
    for b0 in range(0, B, step):
        b1 = min(B, b0 + step)
        nth = torch.arange(n, device="cuda")
        token = (off[b0:b1, None] + nth).clamp_max_(s["total"] - 1)          # [m, n], the last ones stand for none
        there = nth < fresh[b0:b1, None]
        q = s["q"][token].float().view(b1 - b0, n, H, G, d).permute(0, 2, 1, 3, 4).reshape(b1 - b0, H, n * G, d)
        x = q @ _rows(s, "k", b0, b1).transpose(-1, -2)
        x.mul_(d ** -0.5)
        own_row = (s["lens"][b0:b1].long() - fresh[b0:b1])[:, None] + nth                # [m, n]
        seen = key <= own_row[..., None]
        if c["window"]:
            seen &= (key > own_row[..., None] - c["window"]) | (key < c["sinks"])
        x.view(b1 - b0, H, n, G, -1).masked_fill_(~seen[:, None, :, None], -math.inf)
        v = _rows(s, "v", b0, b1)
        v.masked_fill_((key >= s["lens"][b0:b1, None])[:, None, :, None], 0.0)
        y = (_softmax(x) @ v).view(b1 - b0, H, n, G, d).permute(0, 2, 1, 3, 4).reshape(b1 - b0, n, Hq, d)
        if c["ragged"]:
            # tokens that stand for none are written to a row behind the last
            room = torch.empty(s["total"] + 1, Hq, d, dtype=out.dtype, device="cuda")
            room[torch.where(there, token, s["total"])] = y.to(out.dtype)
            lo, hi = sum(_lengths(c)[1][:b0]), sum(_lengths(c)[1][:b1])
            out[lo:hi] = room[lo:hi]
        else:
            out[b0 * n:b1 * n] = y.reshape(-1, Hq, d).to(out.dtype)
    return out


def _prefix(s):
    c = s["case"]
    B, H, Hq, d, n = c["batch"], c["kv_heads"], c["q_heads"], c["dim"], c["prefixes"]
    G = Hq // H
    q = s["q"].float()
    # every sequence of a prompt against the prompt's keys at once
    shared = q.view(n, B // n, H, G, d).transpose(1, 2).reshape(n, H, B // n * G, d)
    x = shared @ s["pk"].float().transpose(-1, -2)
    x = x.view(n, H, B // n, G, -1).transpose(1, 2).reshape(B, H, G, -1)
    y = q.view(B, H, G, d) @ _rows(s, "k", 0, B).transpose(-1, -2)
    gone = (torch.arange(s["cap"], device="cuda") >= s["lens"][:, None])[:, None, :]
    y.masked_fill_(gone[:, :, None], -math.inf)
    w = _softmax(torch.cat([x, y], -1).mul_(d ** -0.5))
    v = _rows(s, "v", 0, B).masked_fill_(gone[..., None], 0.0)
    o = w[..., c["prefix"]:] @ v
    w = w[..., :c["prefix"]].view(n, B // n, H, G, -1).transpose(1, 2).reshape(n, H, B // n * G, -1)
    o += (w @ s["pv"].float()).view(n, H, B // n, G, d).transpose(1, 2).reshape(B, H, G, d)
    s["out"].copy_(o.view(B, Hq, d))
    return s["out"]


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = dict(case)
    cached, new = _lengths(c)
    H, Hq, d, e = c["kv_heads"], c["q_heads"], c["dim"], ESIZE[c["dtype"]]
    q = 4 if c["dtype"] == "f32" else 2
    total = sum(new)
    if c["kind"] == "append":
        # queries, keys and values in, queries out, keys and values into the caches, one row of angles per token
        return {"bytes": total * (2 * Hq * d * q + 2 * H * d * (q + e) + c["rotary"] * 4), "flops": total * (H + Hq) * c["rotary"] * 3}
    if c["kind"] == "prefix":
        rows, pairs = c["prefixes"] * c["prefix"] + sum(cached), c["batch"] * c["prefix"] + sum(cached)
        return {"bytes": 2 * rows * H * d * e + 2 * total * Hq * d * q, "flops": 4 * pairs * Hq * d}
    rows = pairs = 0
    for before, n in zip(cached, new):
        length, w, sinks = before + n, c["window"], c["sinks"]
        if not w:
            rows, pairs = rows + length, pairs + n * before + n * (n + 1) // 2
            continue
        least = max(0, before + 1 - w)                       # the first row that the first token's window holds
        rows += length - least + min(sinks, least)
        for at in range(before, length):
            start = max(0, at + 1 - w)
            pairs += at + 1 - start + min(sinks, start)
    return {"bytes": 2 * rows * H * d * e + 2 * total * Hq * d * q, "flops": 4 * pairs * Hq * d}


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    c = dict(case)
    cached, new = _lengths(c)
    H, Hq, d = c["kv_heads"], c["q_heads"], c["dim"]
    if c["kind"] == "append":
        return _exact_append(prepare(c, seed), c, cached, new)
    w = work(c)
    if w["flops"] > 3e13:                                    # over about 20 seconds in 64 bits
        return None
    s = prepare(c, seed)
    out = torch.zeros(sum(new), Hq, d, dtype=torch.float64, device="cuda")
    first = 0
    for b in range(c["batch"]):
        n = new[b]
        length = cached[b] + (0 if c["kind"] == "prefix" else n)
        for h in range(H):
            keys, values = (_head(s, x, b, h, length) for x in "kv")
            if c["kind"] == "prefix":
                p = b // (c["batch"] // c["prefixes"])
                keys, values = torch.cat([s["pk"][p, h].double(), keys]), torch.cat([s["pv"][p, h].double(), values])
            for g in range(h * Hq // H, (h + 1) * Hq // H):
                for t0 in range(0, n, 2048):
                    t1 = min(n, t0 + 2048)
                    x = torch.einsum("td,jd->tj", s["q"][first + t0:first + t1, g].double(), keys) / math.sqrt(d)
                    if c["kind"] == "window":
                        at = torch.arange(cached[b] + t0, cached[b] + t1, device="cuda")[:, None]
                        j = torch.arange(length, device="cuda")[None]
                        hidden = j > at
                        if c["window"]:
                            hidden |= (at - j >= c["window"]) & (j >= c["sinks"])
                        x[hidden] = -math.inf
                    out[first + t0:first + t1, g] = torch.softmax(x, 1) @ values
        first += n
    return out


def _head(s, name, b, h, length):
    if s["table"] is None:
        return s[name][b, h, :length].double()
    return s[name].view(torch.uint8)[s["table"][b, h].long()].view(s[name].dtype).reshape(-1, s["case"]["dim"])[:length].double()


def _exact_append(s, c, cached, new):
    half = c["rotary"] // 2
    freq = torch.tensor(_frequencies(c), dtype=torch.float64, device="cuda")
    where = s["positions"].tolist()
    q = torch.empty(s["total"], c["q_heads"], c["dim"], dtype=torch.float64, device="cuda")
    k, v = s["k"].double(), s["v"].double()
    first = 0
    for b, n in enumerate(new):
        pos = torch.arange(where[b], where[b] + n, device="cuda", dtype=torch.float64)
        turn = torch.polar(torch.ones(n, half, dtype=torch.float64, device="cuda"), pos[:, None] * freq)[:, None]
        for name, src in (("q", s["q_new"]), ("k", s["k_new"])):
            x = src[first:first + n].double()
            i = torch.arange(half, device="cuda")
            lo, hi = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
            z = torch.complex(x[..., lo], x[..., hi]) * turn
            x[..., lo], x[..., hi] = z.real, z.imag
            if name == "q":
                q[first:first + n] = x
            else:
                _put(s, k, b, cached[b], x)
        _put(s, v, b, cached[b], s["v_new"][first:first + n].double())
        first += n
    lens = torch.tensor([a + n for a, n in zip(cached, new)], dtype=torch.int32, device="cuda")
    return {"k": k, "v": v, "q": q, "lens": lens}


def _put(s, cache, b, row, x):
    """x [n, kv_heads, dim] into the rows from `row` on of sequence b."""
    if s["table"] is None:
        cache[b, :, row:row + x.shape[0]] = x.transpose(0, 1)
        return
    at = torch.arange(row, row + x.shape[0], device="cuda")
    cache[s["table"][b][:, at // PAGE].long(), (at % PAGE)[None]] = x.transpose(0, 1)
