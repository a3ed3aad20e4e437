"""The 8-bit paged cache next to the decoder's reduce step, as measurable cases.

A decoder that reduces its vision tokens keeps keys and values in pages of e4m3 codes with one
power-of-two scale for each page and key/value head.  Four kinds of call: ``append`` writes new
rows into pages, ``attention`` reads them (single tokens and prompts, causal, with a sliding window
and first tokens that stay visible), ``weights`` hands out the text -> vision attention that
``ficoco_l_reduce`` takes, and ``compact`` / ``copy`` rearrange pages behind a reduce step or a
forked sequence.  Inputs are made on the GPU from a seed; the sequence lengths of a ragged batch
follow from the case alone.
"""
import math
import random

import numpy as np
import torch

own = False

QMAX = 448.0                    # largest e4m3 value
SCALE_MIN = 2.0 ** -64          # smallest scale of a page
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one generated token for each of 64 requests: the smallest write, every decode step of every layer
        dict(name="append_step", kind="append", batch=64, lo=100, hi=2000, new_lo=1, new_hi=1, kv_heads=8, dim=128,
             page=64, dtype="bf16", ragged=1),
        # the prompts of a batch (576 vision + 64 text tokens each) written at once, 32 heads
        dict(name="append_prompts", kind="append", batch=16, lo=640, hi=640, new_lo=640, new_hi=640, kv_heads=32,
             dim=128, page=64, dtype="bf16", ragged=2),
        # the next token of a single request: all latency
        dict(name="step_one", kind="attention", batch=1, lo=640, hi=640, q_lo=1, q_hi=1, heads=32, kv_heads=32, dim=128,
             page=64, dtype="bf16", causal=True, window=0, sinks=0, ragged=3),
        # the next token of 64 requests of very different lengths, grouped heads: throughput serving
        dict(name="step_ragged", kind="attention", batch=64, lo=64, hi=8192, q_lo=1, q_hi=1, heads=32, kv_heads=8,
             dim=128, page=16, dtype="bf16", causal=True, window=0, sinks=0, ragged=4),
        # one long conversation in full precision: the length has to be split
        dict(name="step_long_fp32", kind="attention", batch=1, lo=65536, hi=65536, q_lo=1, q_hi=1, heads=32, kv_heads=8,
             dim=128, page=32, dtype="fp32", causal=True, window=0, sinks=0, ragged=5),
        # long conversations of which a window and the first tokens stay visible
        dict(name="step_window", kind="attention", batch=8, lo=20000, hi=40000, q_lo=1, q_hi=1, heads=32, kv_heads=8,
             dim=128, page=128, dtype="bf16", causal=True, window=8000, sinks=5, ragged=6),
        # prompts of five crops and their text, and chunks behind a cached beginning
        dict(name="prompt_multicrop", kind="attention", batch=4, lo=2944, hi=4000, q_lo=2500, q_hi=2944, heads=32,
             kv_heads=32, dim=128, page=64, dtype="bf16", causal=True, window=0, sinks=0, ragged=7),
        # what the decoder's reduce step takes: 64 text rows over 576 vision tokens, 16 sequences
        dict(name="weights_batch", kind="weights", batch=16, lo=640, hi=640, q_lo=640, q_hi=640, text=64, first=0,
             vision=576, heads=32, kv_heads=32, dim=128, page=64, dtype="bf16", causal=True, window=0, sinks=0, ragged=8),
        # one multi-crop request behind a system prompt, a short question, fp32
        dict(name="weights_one_fp32", kind="weights", batch=1, lo=2952, hi=2952, q_lo=37, q_hi=37, text=37, first=35,
             vision=2880, heads=32, kv_heads=8, dim=128, page=32, dtype="fp32", causal=True, window=0, sinks=0, ragged=9),
        # the cache behind a reduce step: 64 of 576 vision tokens and the text stay
        dict(name="compact_batch", kind="compact", batch=16, lo=640, hi=640, first=0, keep_lo=128, keep_hi=128, kv_heads=32,
             dim=128, page=64, ragged=10),
        # ragged sequences of dynamic resolution, a system prompt in front, small pages
        dict(name="compact_ragged", kind="compact", batch=48, lo=500, hi=4200, first=35, keep_lo=100, keep_hi=2000,
             kv_heads=32, dim=128, page=16, ragged=11),
        # pages of forked sequences that are written next
        dict(name="copy_fork", kind="copy", pages=400, moved=190, kv_heads=8, dim=128, page=128),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "attention", "weights", "compact", "copy"])
    kv = rng.choice([1, 2, 4, 8, 16, 32])
    page = rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    base = dict(kind=kind, kv_heads=kv, dim=rng.choice([64, 128, 128, 128]), page=page, ragged=rng.randrange(1 << 20))
    if kind == "copy":
        moved = _log_int(rng, 1, max(1, 24000 // (kv * page)))
        return dict(base, pages=2 * moved + rng.randrange(1, 50), moved=moved)
    hi = _log_int(rng, 16, 8000)
    lo = _log_int(rng, 1, hi)
    if kind == "append":
        new_hi = rng.choice([1, 1, _log_int(rng, 1, hi)])
        batch = _log_int(rng, 1, max(1, min(200, 300000 // (hi * kv))))
        return dict(base, batch=batch, lo=lo, hi=hi, new_lo=min(lo, new_hi, rng.randrange(0, 3)), new_hi=new_hi, dtype=dtype)
    if kind == "compact":
        batch = _log_int(rng, 1, max(1, min(100, 1500000 // (hi * kv))))
        keep = _log_int(rng, 1, max(1, hi // 2))
        return dict(base, batch=batch, lo=lo, hi=hi, first=rng.choice([0, 0, rng.randrange(1, 40)]), keep_lo=rng.randrange(0, keep + 1),
                    keep_hi=keep)
    heads = kv * rng.choice([1, 2, 4, 8] if kv <= 8 else [1, 2])
    mask = dict(causal=rng.random() < 0.8, window=rng.choice([0, 0, _log_int(rng, 1, hi)]), sinks=rng.choice([0, 4, 17]))
    base = dict(base, heads=heads, dtype=dtype, **mask)
    if kind == "weights":
        text = _log_int(rng, 1, 200)
        first = rng.choice([0, rng.randrange(1, 60)])
        vision = _log_int(rng, 16, 4000)
        n = first + vision + text
        batch = _log_int(rng, 1, max(1, min(16, 15000000 // (heads * text * vision))))
        return dict(base, batch=batch, lo=n, hi=n, q_lo=text, q_hi=rng.randrange(text, n + 1), text=text, first=first, vision=vision)
    if rng.random() < 0.6:      # single tokens, now and then a few drafted ones
        batch = _log_int(rng, 1, max(1, min(128, 1200000 // (hi * kv))))
        return dict(base, batch=batch, lo=lo, hi=hi, q_lo=1, q_hi=rng.choice([1, 1, 1, 4]))
    hi = min(hi, 2944)
    batch = _log_int(rng, 1, max(1, min(32, 250000000 // (hi * hi * heads))))
    return dict(base, batch=batch, lo=min(lo, hi), hi=hi, q_lo=1, q_hi=hi, dtype="bf16")


# ---- sizes that follow from the case --------------------------------------------------------------------------------
def _lengths(c):
    """(tokens in the cache, rows of this call) of every sequence."""
    rng = random.Random(c.get("ragged", 0))
    ns, ms = [], []
    for b in range(c["batch"]):
        n = _log_int(rng, c["lo"], c["hi"])
        lo, hi = ((c["new_lo"], c["new_hi"]) if c["kind"] == "append" else (c["keep_lo"], c["keep_hi"])
                  if c["kind"] == "compact" else (c["q_lo"], c["q_hi"]))
        room = n - min(n, c["first"]) if c["kind"] == "compact" else n
        ns.append(n)
        ms.append(min(room, rng.randint(lo, hi)))
    return ns, ms


def _visible(c, n, m):
    """(pairs of a row and a token it sees, tokens that some row sees) for m rows at the end of n tokens."""
    pos = np.arange(n - m, n, dtype=np.int64)
    top = pos + 1 if c["causal"] else np.full(m, n, dtype=np.int64)
    low = np.maximum(0, pos - c["window"] + 1) if c["window"] else np.zeros(m, dtype=np.int64)
    if not m:
        return 0, 0
    pairs = int((top - low + np.minimum(c["sinks"], low)).sum())
    return pairs, int(top.max() - low.min() + min(c["sinks"], int(low.min())))


def work(case):
    c = case
    kd = c["kv_heads"] * c["dim"]
    if c["kind"] == "copy":
        return {"bytes": 4 * c["moved"] * (kd * c["page"] + 4 * c["kv_heads"]), "flops": 0}
    ns, ms = _lengths(c)
    rows = sum(ms)
    e = 2 if c.get("dtype") == "bf16" else 4
    if c["kind"] == "append":
        touched = sum((n - 1) // c["page"] - (n - m) // c["page"] + 1 for n, m in zip(ns, ms) if m)
        return {"bytes": 2 * rows * kd * (e + 1) + 2 * touched * 4 * c["kv_heads"], "flops": 2 * rows * kd}
    if c["kind"] == "compact":
        kept = sum(m + min(n, c["first"]) for n, m in zip(ns, ms))
        return {"bytes": 4 * kept * kd + 4 * rows, "flops": 2 * kept * kd}
    if c["kind"] == "weights":
        out = c["batch"] * c["heads"] * c["text"] * c["vision"]
        q = c["batch"] * c["text"] * c["heads"] * (c["dim"] * e + 4)
        return {"bytes": 4 * out + q + c["batch"] * c["vision"] * kd, "flops": 2 * out * c["dim"]}
    seen = [_visible(c, n, m) for n, m in zip(ns, ms)]
    return {"bytes": sum(s for _, s in seen) * 2 * kd + 2 * rows * c["heads"] * c["dim"] * e,
            "flops": 4 * c["dim"] * c["heads"] * sum(p for p, _ in seen)}


# ---- the cache in plain torch ---------------------------------------------------------------------------------------
def _scale_of(amax):
    """The smallest power of two, SCALE_MIN at least, that brings amax to 448 or below."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), 0.0).clamp_min(SCALE_MIN)


def _codes_of(x):
    return x.clamp(-QMAX, QMAX).to(torch.float8_e4m3fn)


def _paged(c, ns, gen, spare=0):
    """A pool whose pages lie in random order, filled with keys and values of ns[b] tokens."""
    dev, P, H, D = "cuda", c["page"], c["kv_heads"], c["dim"]
    per = [max(1, -(-n // P)) for n in ns]
    used = sum(per)
    total = used + spare + 1
    order = torch.randperm(total, generator=gen, device=dev).to(torch.int32)
    table = torch.zeros((len(ns), max(per)), dtype=torch.int32)
    at = torch.tensor(np.concatenate([[0], np.cumsum(per)]).astype(np.int64))
    col = torch.arange(max(per))
    index = at[:-1, None] + col[None, :].clamp(max=used - 1)
    inside = col[None, :] < torch.tensor(per)[:, None]
    table = torch.where(inside.to(dev), order[index.clamp(max=total - 1).to(dev)], 0).contiguous()
    offset = torch.randn((1, H, 1, D), generator=gen, device=dev) * 0.7       # keys have channels of their own level
    pool = {}
    for name in ("k", "v"):
        x = torch.randn((total, H, P, D), generator=gen, device=dev)
        x = x + offset if name == "k" else x
        amax = x.abs().amax((2, 3))
        pool[name + "_scale"] = _scale_of(amax)
        pool[name + "_codes"] = _codes_of(x / pool[name + "_scale"][:, :, None, None])
        del x
    pool["table"] = table
    pool["lengths"] = torch.tensor(ns, dtype=torch.int32, device=dev)
    pool["spare"] = order[used:used + spare].contiguous()
    return pool


def _cu(ms):
    return torch.tensor(np.concatenate([[0], np.cumsum(ms)]).astype(np.int32), device="cuda")


def _handles(s, pool):
    """What a program that uses the framework keeps: a context and the cache's description."""
    if own:
        from paper_2411_17686_b200 import binding as B
        s["ctx"] = _context()
        s["cache"] = B.PagedCache(pool["k_codes"], pool["v_codes"], pool["k_scale"], pool["v_scale"], pool["table"],
                                  pool["lengths"])
    return s


_contexts = []


def _context():
    """One context for the process, as a program has it."""
    if not _contexts:
        from paper_2411_17686_b200 import binding as B
        _contexts.append(B.Context(max_tokens=1024, max_dim=128, max_batch=16, max_text=16, device=0))
    return _contexts[0]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if c["kind"] == "copy":
        pool = _paged(c, [c["page"]] * c["pages"], gen)
        order = torch.randperm(c["pages"], generator=gen, device="cuda").to(torch.int32)
        s = dict(c=c, pool=pool, src=order[:c["moved"]].contiguous(), dst=order[c["moved"]:2 * c["moved"]].contiguous())
        return _handles(s, pool)
    ns, ms = _lengths(c)
    s = dict(c=c, max_len=max(max(ns), 1), max_m=max(max(ms), 1), rows=sum(ms), cu=_cu(ms))
    dtype = DTYPES[c.get("dtype", "bf16")]
    shape = lambda h: (s["rows"], h, c["dim"])      # noqa: E731
    if c["kind"] == "append":
        pool = _paged(c, ns, gen)
        s["k"] = (torch.randn(shape(c["kv_heads"]), generator=gen, device="cuda") * 1.3).to(dtype)
        s["v"] = torch.randn(shape(c["kv_heads"]), generator=gen, device="cuda").to(dtype)
    elif c["kind"] == "compact":
        kept_n = [m + min(n, c["first"]) for n, m in zip(ns, ms)]
        per = [max(1, -(-n // c["page"])) for n in kept_n]
        pool = _paged(c, ns, gen, spare=sum(per))
        at = torch.tensor(np.concatenate([[0], np.cumsum(per)]).astype(np.int64))[:-1, None]
        index = (at + torch.arange(max(per))).clamp(max=sum(per) - 1).to("cuda")
        s["to"] = pool["spare"][index].contiguous()
        rng = np.random.RandomState(seed & 0x7FFFFFFF)
        kept = [np.sort(rng.choice(n - min(n, c["first"]), m, replace=False)) for n, m in zip(ns, ms)]
        s["kept"] = torch.tensor(np.concatenate(kept).astype(np.int32), device="cuda")
    else:
        pool = _paged(c, ns, gen)
        s["q"] = (torch.randn(shape(c["heads"]), generator=gen, device="cuda") * 1.5).to(dtype)
    s["pool"] = pool
    if c["kind"] == "weights":      # the statistics that the attention call before it has returned
        s["lse"] = _attend(s)[1]
    return _handles(s, pool)


def _gathered(s, name):
    """Dequantised keys or values, [batch, kv heads, tokens, dim]."""
    c, pool = s["c"], s["pool"]
    table = pool["table"].long()
    x = pool[name + "_codes"][table].float() * pool[name + "_scale"][table][:, :, :, None, None]
    b, n = table.shape
    x = x.permute(0, 2, 1, 3, 4).reshape(b, c["kv_heads"], n * c["page"], c["dim"])
    return x[:, :, :s["max_len"]]


def _row_places(s):
    """(sequence, place in it) of every row of q."""
    r = torch.arange(s["rows"], device="cuda", dtype=torch.int32)
    b = (torch.searchsorted(s["cu"], r, right=True) - 1).long()
    return b, (r - s["cu"][b]).long()


def _scores(s, m_rows, from_end):
    """Scaled scores [batch, kv heads, group, m_rows, tokens], -inf where a row does not see a token."""
    c, pool = s["c"], s["pool"]
    count = (s["cu"][1:] - s["cu"][:-1]).long()[:, None]
    i = torch.arange(m_rows, device="cuda")[None, :]
    i = i + (count - m_rows) if from_end else i.expand(c["batch"], -1)
    there = (i >= 0) & (i < count)
    rows = (s["cu"][:-1].long()[:, None] + i).clamp(0, max(s["rows"] - 1, 0))
    q = s["q"][rows].float().reshape(c["batch"], m_rows, c["kv_heads"], -1, c["dim"]).permute(0, 2, 3, 1, 4)
    g = q.shape[2]
    k = _gathered(s, "k")
    x = torch.matmul(q.reshape(c["batch"], c["kv_heads"], g * m_rows, c["dim"]), k.transpose(2, 3))
    x = x.reshape(c["batch"], c["kv_heads"], g, m_rows, -1) * (1.0 / math.sqrt(c["dim"]))
    pos = pool["lengths"].long()[:, None] - count + i
    j = torch.arange(x.shape[-1], device="cuda")
    see = (j < pool["lengths"].long()[:, None, None]) & there[:, :, None]
    if c["causal"]:
        see = see & (j <= pos[:, :, None])
    if c["window"]:
        see = see & ((j > pos[:, :, None] - c["window"]) | (j < c["sinks"]))
    return torch.where(see[:, None, None], x, float("-inf")), rows


def _attend(s):
    c = s["c"]
    x, _ = _scores(s, s["max_m"], False)
    top = x.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(x - top)
    del x
    total = p.sum(-1, keepdim=True)
    v = _gathered(s, "v")
    o = torch.matmul(p.reshape(c["batch"], c["kv_heads"], -1, p.shape[-1]), v).reshape(*p.shape[:-1], c["dim"])
    o = o / torch.where(total > 0, total, 1.0)
    lse = torch.where(total > 0, top + torch.log(total), float("-inf"))[..., 0]
    b, i = _row_places(s)
    o = o.permute(0, 3, 1, 2, 4).reshape(c["batch"], s["max_m"], c["heads"], c["dim"])
    lse = lse.permute(0, 3, 1, 2).reshape(c["batch"], s["max_m"], c["heads"])
    return o[b, i].to(s["q"].dtype), lse[b, i].contiguous()


def _weights(s):
    c = s["c"]
    x, rows = _scores(s, c["text"], True)
    lse = s["lse"][rows].reshape(c["batch"], c["text"], c["kv_heads"], -1).permute(0, 2, 3, 1)
    a = torch.exp(x[..., c["first"]:c["first"] + c["vision"]] - lse[..., None])
    return a.reshape(c["batch"], c["heads"], c["text"], c["vision"])


def _scale_pages(pool, values, pages, keep):
    """New scales [n, heads] of the pages that the tokens of `values` [tokens, heads, dim] go to, for each token."""
    amax = torch.zeros_like(pool).scatter_reduce(0, pages[:, None].expand(-1, pool.shape[1]), values.abs().amax(2), "amax")
    new = _scale_of(amax)
    return torch.maximum(new, torch.where(keep[:, None], pool, 0.0))


def _append(s):
    c, pool = s["c"], s["pool"]
    P = c["page"]
    count = (s["cu"][1:] - s["cu"][:-1]).long()
    b, i = _row_places(s)
    start = pool["lengths"].long() - count
    pos = start[b] + i
    page, slot = pool["table"].long()[b, pos // P], pos % P
    first = pool["table"].long().gather(1, (start // P).clamp(max=pool["table"].shape[1] - 1)[:, None])[:, 0]
    behind = (start % P > 0) & (count > 0)              # a page that holds older tokens keeps or grows its scale
    n = pool["k_scale"].shape[0]
    keep = torch.zeros(n, dtype=torch.int32, device="cuda").scatter_reduce(0, first, behind.int(), "amax") > 0
    for name in ("k", "v"):
        x, scale, codes = s[name].float(), pool[name + "_scale"], pool[name + "_codes"]
        new = _scale_pages(scale, x, page, keep)
        touched = torch.zeros(n, dtype=torch.bool, device="cuda").index_fill(0, page, True)
        old = codes[first].float() * (scale[first] / new[first])[:, :, None, None]
        there = (torch.arange(P, device="cuda")[None, :] < (start % P)[:, None]) & behind[:, None]
        at = first[:, None].expand(-1, P)[there], torch.arange(P, device="cuda")[None, :].expand(first.shape[0], -1)[there]
        codes[at[0], :, at[1]] = _codes_of(old.permute(0, 2, 1, 3)[there])
        codes[page, :, slot] = _codes_of(x / new[page][:, :, None])
        scale.copy_(torch.where(touched[:, None], new, scale))
    return {k: pool[k] for k in ("k_codes", "k_scale", "v_codes", "v_scale")}


def _compact(s):
    c, pool = s["c"], s["pool"]
    P = c["page"]
    lengths = pool["lengths"].long()
    head = lengths.clamp(max=c["first"])
    count = (s["cu"][1:] - s["cu"][:-1]).long()
    total = head + count
    cut = torch.cumsum(total, 0)
    t = torch.arange(s["rows"] + sum(min(n, c["first"]) for n in _lengths(c)[0]), device="cuda")
    b = torch.searchsorted(cut, t, right=True)
    i = t - (cut - total)[b]
    kept = s["kept"].long()[(s["cu"].long()[b] + i - head[b]).clamp(0, max(s["rows"] - 1, 0))] if s["rows"] else i
    pos = torch.where(i < head[b], i, head[b] + kept)
    src, dst = pool["table"].long()[b, pos // P], s["to"].long()[b, i // P]
    keep = torch.zeros(pool["k_scale"].shape[0], dtype=torch.bool, device="cuda")
    touched = keep.index_fill(0, dst, True)
    for name in ("k", "v"):
        scale, codes = pool[name + "_scale"], pool[name + "_codes"]
        x = codes[src, :, pos % P].float() * scale[src][:, :, None]
        new = _scale_pages(scale, x, dst, keep)
        codes[dst, :, i % P] = _codes_of(x / new[dst][:, :, None])
        scale.copy_(torch.where(touched[:, None], new, scale))
    return dict({k: pool[k] for k in ("k_codes", "k_scale", "v_codes", "v_scale")}, lengths=total.int())


def _copy(s):
    src, dst = s["src"].long(), s["dst"].long()
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        s["pool"][name][dst] = s["pool"][name][src]
    return {k: s["pool"][k] for k in ("k_codes", "k_scale", "v_codes", "v_scale")}


def run(state):
    s = state
    c = s["c"]
    kind = c["kind"]
    if own:
        ctx, cache = s["ctx"], s["cache"]
        if kind == "append":
            ctx.ficoco_cache_append(cache, s["k"], s["v"], s["cu"])
        elif kind == "attention":
            return ctx.ficoco_cache_attention(cache, s["q"], s["cu"], causal=c["causal"], window=c["window"],
                                              sinks=c["sinks"], want_lse=True)
        elif kind == "weights":
            return ctx.ficoco_cache_weights(cache, s["q"], s["lse"], s["cu"], c["text"], c["first"], c["vision"],
                                            causal=c["causal"], window=c["window"], sinks=c["sinks"])
        elif kind == "compact":
            lengths = ctx.ficoco_cache_compact(cache, s["to"], s["kept"], s["cu"], first=c["first"])
            return dict({k: s["pool"][k] for k in ("k_codes", "k_scale", "v_codes", "v_scale")}, lengths=lengths)
        else:
            ctx.ficoco_cache_copy(cache, s["src"], s["dst"])
        return {k: s["pool"][k] for k in ("k_codes", "k_scale", "v_codes", "v_scale")}
    return {"append": _append, "attention": _attend, "weights": _weights, "compact": _compact, "copy": _copy}[kind](s)


# ---- the definitions in 64 bits, one sequence after the other --------------------------------------------------------
def _round_e4m3(x):
    """Nearest multiple of 2^(e - 3) for |x| in [2^e, 2^(e+1)), e at least -6, ties to the even one."""
    e = torch.floor(torch.log2(x.abs().clamp_min(1e-300))).clamp_min(-6)
    step = torch.pow(2.0, e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_scale(amax):
    """Doubled from 2^-64 until 448 times it reaches amax."""
    s = torch.full_like(amax, 2.0 ** -64)
    while bool((448 * s < amax).any()):
        s = torch.where(448 * s < amax, 2 * s, s)
    return s


def _exact_pool(s):
    p = s["pool"]
    return {k: p[k].double() for k in ("k_codes", "k_scale", "v_codes", "v_scale")}


def exact(case, seed):
    c = dict(case)
    s = prepare(case, seed)
    P = c["page"]
    pool = _exact_pool(s)
    if c["kind"] == "copy":
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            for k in pool:
                pool[k][b] = pool[k][a]
        return pool
    ns, ms = _lengths(c)
    table = s["pool"]["table"].tolist()
    cu = [0] + np.cumsum(ms).tolist()
    if c["kind"] in ("append", "compact"):
        lengths = []
        for b, (n, m) in enumerate(zip(ns, ms)):
            if c["kind"] == "append":
                begin, total, to = n - m, n, table[b]
            else:
                head = min(n, c["first"])
                places = list(range(head)) + [head + i for i in s["kept"][cu[b]:cu[b + 1]].tolist()]
                begin, total, to = 0, len(places), s["to"][b].tolist()
                lengths.append(total)
            for g in range(begin // P, -(-total // P) if total > begin else 0):
                lo, hi = max(begin, g * P), min(total, (g + 1) * P)
                page, keep = to[g], lo - g * P
                for w in ("k", "v"):
                    if c["kind"] == "append":
                        x = s[w][cu[b] + lo - begin:cu[b] + hi - begin].double()
                    else:
                        at = torch.tensor(places[lo:hi], device="cuda")
                        src = s["pool"]["table"][b].long()[at // P]
                        x = s["pool"][w + "_codes"][src, :, at % P].double() * s["pool"][w + "_scale"][src].double()[:, :, None]
                    scale = _exact_scale(x.abs().amax((0, 2)))
                    if keep:
                        before = pool[w + "_scale"][page]
                        scale = torch.maximum(scale, before)
                        pool[w + "_codes"][page, :, :keep] = _round_e4m3(pool[w + "_codes"][page, :, :keep] *
                                                                         (before / scale)[:, None, None])
                    pool[w + "_scale"][page] = scale
                    pool[w + "_codes"][page, :, keep:keep + hi - lo] = _round_e4m3(x / scale[None, :, None]).transpose(0, 1)
        return dict(pool, lengths=None) if lengths else pool
    out, lses, group = [], [], c["heads"] // c["kv_heads"]
    for b, (n, m) in enumerate(zip(ns, ms)):
        pages = torch.tensor(table[b][:-(-n // P)], device="cuda")

        def tokens(w):
            x = pool[w + "_codes"][pages] * pool[w + "_scale"][pages][:, :, None, None]
            return x.transpose(1, 2).reshape(-1, c["kv_heads"], c["dim"])[:n]

        keys, values = tokens("k"), tokens("v")
        count = c["text"] if c["kind"] == "weights" else m
        q = s["q"][cu[b + 1] - count:cu[b + 1]].double()
        place = torch.arange(n - count, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None, :]
        hidden = j > place if c["causal"] else torch.zeros((count, n), dtype=torch.bool, device="cuda")
        if c["window"]:
            hidden = hidden | ((j <= place - c["window"]) & (j >= c["sinks"]))
        o, l = [], []
        for h in range(c["heads"]):
            x = q[:, h] @ keys[:, h // group].T / math.sqrt(c["dim"])
            x = x.masked_fill(hidden, -math.inf)
            if c["kind"] == "weights":
                lse = s["lse"][cu[b + 1] - count:cu[b + 1], h].double()
                o.append(torch.exp(x - lse[:, None])[:, c["first"]:c["first"] + c["vision"]])
            else:
                o.append(torch.softmax(x, -1) @ values[:, h // group])
                l.append(torch.logsumexp(x, -1))
        if c["kind"] == "weights":
            out.append(torch.stack(o))
        else:
            out.append(torch.stack(o, 1))
            lses.append(torch.stack(l, 1))
    return torch.stack(out) if c["kind"] == "weights" else (torch.cat(out), torch.cat(lses))
