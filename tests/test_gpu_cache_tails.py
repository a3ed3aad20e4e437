"""Attention over the 8-bit cache behind dominant tokens (attention sinks): first tokens that take nearly all of the weight and whose
values are near zero, so that the tail behind them is the result."""
import math

import numpy as np
import pytest
import torch

from paper_2411_17686_b200 import binding
from tests import cache_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(max_tokens=1024, max_dim=128, max_batch=4, max_text=16, device=0)
    yield c
    c.close()


def sunk(rng, n, page, kv, dim, above, sinks=1, beside=None):
    """A sequence whose first `sinks` tokens score about `above` more than the rest for query rows near `u`, values 0 there and near
    1 behind them.  `beside`: the token behind the sinks, with next to no weight, has values of that size and with them their page's
    scale."""
    per = -(-n // page)
    cache = R.Cache(rng, [0], page, kv, dim, spare=per + 1, max_pages=per + 1)
    cache.table[0, :per] = cache.spare[:per]
    cache.lengths = [n]
    u = np.where(rng.random(dim) < 0.5, -1.0, 1.0)
    k, v = 0.05 * rng.standard_normal((n, kv, dim)), 1 + 0.25 * rng.standard_normal((n, kv, dim))
    k[:sinks] += above / math.sqrt(dim) * u
    v[:sinks] = 0.0
    if beside:
        k[sinks], v[sinks] = -30 / math.sqrt(dim) * u, beside
    cache.write(0, 0, k, v)
    return cache, u


def expected(cache, q, kernel, causal=True, window=0, sinks=0):
    """(out, lse, tolerances) in 64 bits for rows q [m, heads, dim], the last ones of the cache's only sequence.

    A weight (times its page's value scale) is off by at most 2^-8 of itself where two e4m3 terms hold it ("step", bf16 rows), 2^-24
    where six do ("step", fp32 rows), 2^-11 where it is one fp16 number ("prompt").  The smallest steps put on top of that, by half a
    step and never by more than the weight: two terms of 256 times the weight relative to the largest of its 32 neighbours, 2^-10 / 16 /
    256 = 2^-22 of that one; six terms 2^-10 / 16^5 / 256 = 2^-38; fp16 weights whose tile of 128 tokens has its largest one at 2^-5
    or above, 2^-25 / 2^-5 = 2^-20 of that, or, in tiles more than 2^-28 below the row's largest, 2^-25 where that one is 2^23:
    2^-48 of it.  Scores are off by ds as in cache_reference.attention, each weight by 2 ds (numerator and denominator).  Sums in
    fp32: single tokens, per tile of 128 tokens four additions and one multiplication of the output and as many roundings of the
    denominator, 10 of 2^-24 each; prompts, eight products of 16 tokens and eight additions to the denominator, 16 of 2^-22 each (a
    product's own sum: measured 2^-22 of the magnitudes at 128 terms); exponentials and the joining of parts like 8 tiles more.  The
    result is rounded by half a step of its type, 2^-8 of it (bf16) or 2^-24."""
    m, heads, dim = q.shape
    n, bf16 = cache.lengths[0], q.dtype == torch.bfloat16
    rel, near, group, far = {"step": (2.0 ** -8, 2.0 ** -22, 32, 0.0) if bf16 else (2.0 ** -24, 2.0 ** -38, 32, 0.0),
                             "prompt": (2.0 ** -11, 2.0 ** -20, 128, 2.0 ** -48)}[kernel]
    x = q.double().cpu().numpy()
    scale = dim ** -0.5
    see = np.array([R.visible(n, n - m + i, causal, window, sinks) for i in range(m)])
    pad = -n % group
    chain = (n / 128 + 8) * (10 * 2.0 ** -24 if kernel == "step" else 16 * 2.0 ** -22)
    out, lse = np.zeros(x.shape), np.zeros(x.shape[:2])
    tol, ltol = np.zeros(x.shape), np.zeros(x.shape[:2])
    for h in range(heads):
        k, v, sv = cache.tokens(0, h // (heads // cache.kv))
        s = np.where(see, x[:, h] @ k.T * scale, -math.inf)
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        l = p.sum(1, keepdims=True)
        p /= l
        out[:, h] = p @ v
        lse[:, h] = top[:, 0] + np.log(l[:, 0])
        size = np.abs(np.where(see, s, 0.0)).max(1)
        ds = 2.0 ** -21 * scale * np.where(see, np.abs(x[:, h]) @ np.abs(k).T, 0.0).max(1) + 2.0 ** -21 * (1 + size)
        if bf16:
            ds += scale * np.abs(x[:, h]).max(1) * np.where(see, np.abs(k).sum(1)[None], 0.0).max(1) * 2.0 ** -17
        w = np.pad(p * sv, ((0, 0), (0, pad)))
        most = w.reshape(m, -1, group).max(2).repeat(group, 1)[:, :n]
        held = rel * p + np.minimum(p, (near * most + far * w.max(1, keepdims=True)) / sv)
        t = held @ np.abs(v) + (p @ np.abs(v)) * (2 * ds + chain)[:, None]
        tol[:, h] = t + (2.0 ** -8 if bf16 else 2.0 ** -24) * (np.abs(out[:, h]) + t)
        ltol[:, h] = ds + chain + 2.0 ** -22 * (4 + np.abs(lse[:, h]))
    return out, lse, tol, ltol


def compare(out, lse, want, want_lse, tol, ltol):
    assert (tol <= 2.0 ** -5 * np.abs(want)).all()       # (a tolerance that the fault would pass is none)
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= tol).all(), f"{np.max(off / tol)} of the tolerance, {np.max(off / np.abs(want))} of the result"
    assert (np.abs(lse.double().cpu().numpy() - want_lse) <= ltol).all()


# dim, page, heads, kv, dtype, tokens, rows, copies, above, sinks, mask.  `copies` sequences share the pages: 37 of 8 heads are one
# item per CTA of 148 SMs, which none of them cuts; one sequence is cut into many pieces.
STEPS = [
    (128, 64, 8, 8, "bf16", 30000, 1, 37, 16.0, 1, {}),
    (128, 128, 8, 8, "fp32", 9000, 1, 37, 16.0, 1, {}),
    (64, 32, 32, 8, "bf16", 9000, 1, 37, 14.0, 4, {}),
    (128, 64, 96, 8, "bf16", 9000, 1, 37, 15.0, 1, {}),
    (128, 16, 8, 2, "bf16", 30000, 1, 1, 16.0, 1, {}),
    (128, 16, 8, 2, "fp32", 30000, 1, 1, 18.0, 1, {}),
    (64, 128, 4, 4, "bf16", 12000, 2, 1, 16.0, 3, {}),
    (128, 64, 8, 8, "bf16", 12000, 1, 37, 15.0, 4, dict(window=8000, sinks=4)),
    (128, 64, 8, 2, "bf16", 12000, 3, 1, 15.0, 4, dict(window=8000, sinks=5)),
]


@pytest.mark.parametrize("dim,page,heads,kv,dtype,n,rows,copies,above,sinks,mask", STEPS)
def test_the_tail_behind_a_sink_single_tokens(ctx, dim, page, heads, kv, dtype, n, rows, copies, above, sinks, mask):
    rng = np.random.default_rng(n + heads + dim)
    cache, u = sunk(rng, n, page, kv, dim, above, sinks)
    q = torch.from_numpy(u + 0.1 * rng.standard_normal((rows, heads, dim))).to(DT[dtype]).to(DEV)
    d = cache.device()
    dc = binding.PagedCache(d.k_codes, d.v_codes, d.k_scale, d.v_scale, d.page_table.repeat(copies, 1), d.lengths.repeat(copies))
    ctx.ficoco_profile(True)
    out, lse = ctx.ficoco_cache_attention(dc, q.repeat(copies, 1, 1), R.cu([rows] * copies), want_lse=True, **mask)
    assert [name for name, _, _ in ctx.ficoco_profile_read()] == ["k_cache_step"]
    ctx.ficoco_profile(False)
    assert ctx.ficoco_status() == 0
    want = expected(cache, q, "step", **mask)
    for b in {0, copies // 2, copies - 1}:
        compare(out[b * rows:(b + 1) * rows], lse[b * rows:(b + 1) * rows], *want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_tail_behind_a_sink_whose_page_has_a_larger_scale(ctx, dtype):
    """The scale is part of what the largest weight is taken of: a sink of 2^13 times a tail token's weight in a page of 2^13 times its scale."""
    rng = np.random.default_rng(31)
    n, kv, dim, copies = 12000, 8, 128, 37
    cache, u = sunk(rng, n, 16, kv, dim, 9.0, 1, beside=2.0 ** 14)
    q = torch.from_numpy(u + 0.1 * rng.standard_normal((1, kv, dim))).to(DT[dtype]).to(DEV)
    d = cache.device()
    dc = binding.PagedCache(d.k_codes, d.v_codes, d.k_scale, d.v_scale, d.page_table.repeat(copies, 1), d.lengths.repeat(copies))
    out, lse = ctx.ficoco_cache_attention(dc, q.repeat(copies, 1, 1), R.cu([1] * copies), want_lse=True)
    assert ctx.ficoco_status() == 0
    compare(out[-1:], lse[-1:], *expected(cache, q, "step"))


# dim, page, heads, kv, tokens, rows, above, sinks, mask
PROMPTS = [
    (128, 64, 16, 8, 12000, 520, 16.0, 1, {}),
    (128, 16, 16, 8, 9000, 530, 18.0, 1, {}),
    (64, 128, 16, 8, 12000, 520, 17.0, 4, {}),
    (128, 64, 16, 8, 12000, 520, 16.0, 4, dict(window=9000, sinks=4)),
    (128, 32, 16, 8, 6000, 520, 24.0, 1, dict(causal=False)),
]


@pytest.mark.parametrize("dim,page,heads,kv,n,rows,above,sinks,mask", PROMPTS)
def test_the_tail_behind_a_sink_prompts(ctx, dim, page, heads, kv, n, rows, above, sinks, mask):
    rng = np.random.default_rng(n + heads + dim)
    cache, u = sunk(rng, n, page, kv, dim, above, sinks)
    q = torch.from_numpy(u + 0.1 * rng.standard_normal((rows, heads, dim))).to(torch.bfloat16).to(DEV)
    ctx.ficoco_profile(True)
    out, lse = ctx.ficoco_cache_attention(cache.device(), q, R.cu([rows]), want_lse=True, **mask)
    assert [name for name, _, _ in ctx.ficoco_profile_read()] == ["k_cache_prompt"]
    ctx.ficoco_profile(False)
    assert ctx.ficoco_status() == 0
    compare(out, lse, *expected(cache, q, "prompt", **mask))
