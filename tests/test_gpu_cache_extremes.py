"""The 8-bit cache at the ends of fp32's range and of its own limits."""
import numpy as np
import pytest
import torch

from paper_2411_17686_b200 import binding
from tests import cache_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(max_tokens=1024, max_dim=128, max_batch=4, max_text=16, device=0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_that_round_to_2_to_the_128(ctx, dtype):
    """The largest finite numbers become code 256 at scale 2^120; gathered they stay what they are."""
    big = torch.finfo(dtype).max
    n, page, kv, dim = 40, 16, 2, 32
    cache = R.Cache(np.random.default_rng(0), [0], page, kv, dim, spare=6, max_pages=4)
    cache.table[0, :3], to = cache.spare[:3], cache.spare[3:5]
    cache.lengths = [n]
    k = torch.randn((n, kv, dim), generator=torch.Generator().manual_seed(0)).to(dtype)
    v = k * 2.0 ** 100
    k[[3, 20], 0, 5], k[4, 1, 6], v[[7, 25], 1, 2], v[2, 0, 1] = big, -big, -big, big
    dc = cache.device()
    ctx.ficoco_cache_append(dc, k.to(DEV), v.to(DEV), R.cu([n]))
    cache.write(0, 0, k.double().numpy(), v.double().numpy())
    kept = np.array([3, 4, 2, 7, 20, 25, 1, 39, 38, 0] + list(range(8, 20)), dtype=np.int32)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)      # noqa: E731
    got = ctx.ficoco_cache_compact(dc, t(to[None].astype(np.int32)), t(kept), R.cu([len(kept)]))
    assert got.tolist() == [len(kept)] and ctx.ficoco_status() == 0
    for pi in range(2):
        at = kept[pi * page:(pi + 1) * page]
        sp = cache.table[0, at // page]
        for codes, scales in ((cache.kc, cache.ks), (cache.vc, cache.vs)):
            for h in range(kv):
                x = R.E4M3[codes[sp, h, at % page]] * scales[sp, h].astype(np.float64)[:, None]
                scales[to[pi], h] = R.scale_of(np.abs(x).max())
                codes[to[pi], h, :len(at)] = R.to_codes(x / float(scales[to[pi], h]))
    assert cache.ks[to[0], 0] == 2.0 ** 120 and 256.0 in R.E4M3[cache.kc[to[0], 0]]
    for got, want in ((dc.k_codes, cache.kc), (dc.v_codes, cache.vc)):
        assert np.array_equal(got.view(torch.uint8).cpu().numpy(), want)
    for got, want in ((dc.k_scale, cache.ks), (dc.v_scale, cache.vs)):
        assert np.array_equal(got.cpu().numpy(), want, equal_nan=True)


def test_row_offsets_that_make_the_work_too_long_to_count(ctx):
    """Every other sequence claims all rows again: 2.6e9 tiles of work, more than 31 bits count.  Nothing is done, the status tells."""
    batch, rows, heads, kv, dim, page, pages = 20000, 4096, 32, 8, 128, 128, 16
    codes = [torch.zeros((pages, kv, page, dim), dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.ones((pages, kv), device=DEV) for _ in range(2)]
    table = torch.arange(pages, dtype=torch.int32, device=DEV).repeat(batch, 1)
    dc = binding.PagedCache(*codes, *scales, table, torch.full((batch,), page * pages, dtype=torch.int32, device=DEV))
    q = torch.ones((rows, heads, dim), dtype=torch.bfloat16, device=DEV)
    out = torch.full_like(q, 7.0)
    cu = torch.zeros(batch + 1, dtype=torch.int32, device=DEV)
    cu[1::2] = rows
    ctx.ficoco_profile(True)
    ctx.ficoco_cache_attention(dc, q, cu, out=out)
    assert ctx.ficoco_status() == 16 and bool((out == 7.0).all())
    assert [name for name, _, _ in ctx.ficoco_profile_read()] == ["k_cache_step"]
    ctx.ficoco_profile(False)
    cu[2:] = rows                                        # one sequence with all rows, the rest with none
    ctx.ficoco_cache_attention(dc, q, cu, out=out)
    assert ctx.ficoco_status() == 0 and bool((out == 0.0).all())


@pytest.mark.parametrize("n,heads,kv,dim,dtype,pages,kernel", [
    (600, 16, 8, 128, "bf16", 1 << 22, "k_cache_prompt"),             # 151 blocks * 8 heads * 2^22 tiles: 5.1e9
    (70, 32, 32, 64, "bf16", 1 << 23, "k_cache_prompt"),              # 2.6e9
    (600, 16, 8, 128, "bf16", 1 << 17, "k_cache_prompt"),             # 1.6e8
    (100, 8, 8, 128, "bf16", 1 << 22, "k_cache_step"),                # 4.5e8
    (40, 8, 8, 128, "fp32", 1 << 23, "k_cache_step"),                 # 4.0e8
    (500, 8, 8, 128, "fp32", 1 << 23, "k_cache_attention_simt"),      # 4.3e9
    (30, 64, 64, 128, "bf16", 1 << 23, "k_cache_attention_simt"),     # 2.6e9, few rows
])
def test_tables_with_room_for_very_long_sequences(ctx, n, heads, kv, dim, dtype, pages, kernel):
    """A table of up to 2^30 tokens, a short sequence: which kernel is taken around the limit of 2e9 tiles, and its result."""
    rng = np.random.default_rng(n)
    cache = R.Cache(rng, [700], 128, kv, dim)
    d = cache.device()
    table = torch.full((1, pages), -7, dtype=torch.int32, device=DEV)
    table[:, :d.page_table.shape[1]] = d.page_table
    dc = binding.PagedCache(d.k_codes, d.v_codes, d.k_scale, d.v_scale, table, d.lengths)
    q = torch.from_numpy(rng.standard_normal((n, heads, dim)) * 1.5).to(dict(bf16=torch.bfloat16, fp32=torch.float32)[dtype]).to(DEV)
    ctx.ficoco_profile(True)
    out, lse = ctx.ficoco_cache_attention(dc, q, R.cu([n]), want_lse=True)
    assert [name for name, _, _ in ctx.ficoco_profile_read()] == [kernel]
    ctx.ficoco_profile(False)
    assert ctx.ficoco_status() == 0
    want, want_lse, tol, ltol = R.attention(cache, q, [n])
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    assert (np.abs(lse.double().cpu().numpy() - want_lse) <= ltol).all()


@pytest.mark.parametrize("n_text,dim,dtype,kernel", [
    (60000, 128, "bf16", "k_cache_weights"),              # (n_text * group + 64) * n_text: 3.6e9
    (70000, 128, "bf16", "k_cache_weights_simt"),         # 4.9e9: beyond 32 bits
    (5, 64, "fp32", "k_cache_weights"),
    (5, 80, "fp32", "k_cache_weights_simt"),
])
def test_weights_of_more_text_rows_than_there_are(ctx, n_text, dim, dtype, kernel):
    """Which kernel is taken around the limit of 32-bit row numbers, and its result: rows that are not there weigh nothing."""
    rng = np.random.default_rng(n_text)
    rows, heads, kv, first, count = [90, 3], 2, 2, 4, 50
    cache = R.Cache(rng, [120, 40], 32, kv, dim)
    q = torch.from_numpy(rng.standard_normal((sum(rows), heads, dim))).to(dict(bf16=torch.bfloat16, fp32=torch.float32)[dtype]).to(DEV)
    dc = cache.device()
    _, lse = ctx.ficoco_cache_attention(dc, q, R.cu(rows), want_lse=True)
    out = torch.full((2, heads, n_text, count), float("nan"), device=DEV)
    ctx.ficoco_profile(True)
    ctx.ficoco_cache_weights(dc, q, lse, R.cu(rows), n_text, first, count, out=out)
    assert [name for name, _, _ in ctx.ficoco_profile_read()] == [kernel]
    ctx.ficoco_profile(False)
    assert ctx.ficoco_status() == 0
    want, tol = R.weights(cache, q, lse, rows, n_text, first, count)
    got = out.double().cpu().numpy()
    assert (np.abs(got - want) <= tol).all() and (got[want == 0] == 0).all()
