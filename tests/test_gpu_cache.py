"""The 8-bit paged cache on the GPU against its definitions in 64 bits (tests/cache_reference.py)."""
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
    c = binding.Context(max_tokens=4096, max_dim=512, max_batch=16, max_text=128, device=0)
    yield c
    c.close()


def rows_of(rng, rows, heads, dim, dtype, factor=1.5):
    return torch.from_numpy(rng.standard_normal((sum(rows), heads, dim)) * factor).to(DT[dtype]).to(DEV)


def check_attention(ctx, cache, q, rows, **mask):
    out, lse = ctx.ficoco_cache_attention(cache.device(), q, R.cu(rows), want_lse=True, **mask)
    torch.cuda.synchronize()
    assert ctx.ficoco_status() == 0
    want, want_lse, tol, ltol = R.attention(cache, q, rows, **mask)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.isfinite(got).all()
    off = np.abs(got - want)
    assert (off <= tol).all(), f"out: {np.max(off / np.maximum(tol, 1e-300))} of the tolerance"
    inf = np.isinf(want_lse)
    assert (np.isinf(got_lse) == inf).all() and (got_lse[inf] < 0).all()
    assert (np.abs(got_lse[~inf] - want_lse[~inf]) <= ltol[~inf]).all()
    return out, lse


# dim, page, heads, kv heads, dtype, lengths, rows, mask
ATTENTION = [
    (128, 64, 4, 4, "bf16", [640], [1], {}),
    (128, 16, 8, 2, "bf16", [1, 0, 17, 300], [1, 0, 1, 1], {}),
    (128, 32, 8, 1, "fp32", [129, 128, 127, 1], [1, 1, 1, 1], {}),
    (64, 128, 16, 2, "bf16", [513, 5], [3, 5], {}),
    (128, 64, 32, 2, "bf16", [700, 33], [1, 2], {}),
    (128, 64, 10, 2, "bf16", [257, 64, 65], [1, 1, 1], {}),
    (64, 16, 6, 2, "fp32", [90, 400], [1, 3], {}),
    (128, 128, 2, 1, "fp32", [1000], [9], {}),
    (128, 16, 8, 2, "bf16", [1000, 40, 200], [1, 1, 4], dict(window=100, sinks=5)),
    (128, 32, 4, 2, "bf16", [700, 300], [1, 2], dict(window=1)),
    (128, 64, 4, 4, "fp32", [900, 129], [2, 1], dict(window=128, sinks=200)),
    (64, 32, 4, 2, "bf16", [500, 20], [2, 2], dict(window=260, sinks=129)),
    (128, 64, 4, 2, "bf16", [300, 100], [5, 7], dict(causal=False)),
    (128, 64, 4, 2, "bf16", [600], [6], dict(causal=False, window=50, sinks=3)),
    (128, 64, 4, 2, "bf16", [300, 150, 1], [300, 100, 1], {}),
    (128, 16, 8, 2, "bf16", [260, 0, 131], [130, 0, 131], dict(window=40, sinks=4)),
    (128, 128, 2, 2, "bf16", [513], [400], dict(causal=False)),
    (64, 64, 8, 2, "bf16", [200, 333], [200, 61], {}),
    (64, 64, 2, 2, "fp32", [140, 30], [140, 11], {}),
    (128, 32, 4, 1, "fp32", [150], [70], dict(window=33, sinks=2)),
    (80, 16, 4, 2, "bf16", [100, 31], [1, 31], {}),
    (256, 32, 4, 4, "fp32", [140, 3], [2, 3], {}),
    (16, 64, 3, 1, "bf16", [65, 200], [4, 1], dict(window=20, sinks=1)),
    (128, 64, 4, 2, "bf16", [3, 200], [5, 1], {}),
    (128, 64, 4, 2, "bf16", [2, 100], [90, 100], {}),
    (128, 16, 4, 1, "bf16", [9000], [1], {}),
    (128, 64, 2, 1, "fp32", [5000, 70], [1, 1], {}),
    (128, 16, 8, 8, "bf16", list(range(1, 301)), [1] * 300, {}),
    (64, 16, 40, 1, "bf16", [100, 300], [1, 2], {}),
]


@pytest.mark.parametrize("dim,page,heads,kv,dtype,lengths,rows,mask", ATTENTION)
def test_attention(ctx, dim, page, heads, kv, dtype, lengths, rows, mask):
    rng = np.random.default_rng(len(lengths) * 1000 + dim + heads)
    cache = R.Cache(rng, lengths, page, kv, dim)
    check_attention(ctx, cache, rows_of(rng, rows, heads, dim, dtype), rows, **mask)


# enough rows and heads for the kernel of prompts, which the sizes above leave to the one of single tokens
PROMPTS = [
    (128, 64, 8, 4, [1100, 700, 40, 0], [1100, 300, 40, 0], {}),
    (128, 16, 16, 16, [640, 257], [640, 129], {}),
    (128, 128, 8, 8, [1500], [1025], dict(window=300, sinks=200)),
    (128, 32, 20, 4, [515, 513, 3], [300, 250, 3], dict(window=1)),
    (128, 64, 8, 8, [1100, 130], [1000, 130], dict(causal=False)),
    (128, 16, 8, 8, [1000, 60], [1000, 60], dict(causal=False, window=77, sinks=5)),
    (64, 64, 32, 8, [777], [400], {}),
    (64, 128, 16, 8, [400, 300], [300, 200], dict(window=130, sinks=129)),
    (64, 16, 24, 8, [5, 500], [200, 450], {}),
    (128, 64, 16, 8, [2, 640, 64], [260, 256, 64], {}),
    (128, 64, 40, 8, [129] * 9, [128] * 9, {}),
]


@pytest.mark.parametrize("dim,page,heads,kv,lengths,rows,mask", PROMPTS)
def test_attention_of_prompts(ctx, dim, page, heads, kv, lengths, rows, mask):
    rng = np.random.default_rng(len(lengths) * 1000 + dim + heads)
    cache = R.Cache(rng, lengths, page, kv, dim)
    ctx.ficoco_profile(True)
    check_attention(ctx, cache, rows_of(rng, rows, heads, dim, "bf16"), rows, **mask)
    assert [name for name, _, _ in ctx.ficoco_profile_read()] == ["k_cache_prompt"]
    ctx.ficoco_profile(False)


def test_attention_of_prompts_scales_poison_and_fused_rows(ctx):
    """Pages whose scales differ by 2^40, maxima that grow late, poisoned tokens and rows, rows cut out of a fused projection."""
    rng = np.random.default_rng(17)
    for dim in (64, 128):
        heads, kv, n, m = 16, 8, 700, 400
        cache = R.Cache(rng, [n, 90], 16, kv, dim)
        for p in range(cache.vs.shape[0]):
            if not np.isnan(cache.vs[p, 0]):
                cache.vs[p] *= 2.0 ** rng.integers(-20, 21)
        for pi in range(20, 40):                         # keys that grow along the sequence
            cache.ks[cache.table[0, pi]] *= 2.0 ** ((pi - 20) // 4)
        fused = torch.from_numpy(rng.standard_normal((m + 90 + 6, (heads + 2 * kv) * dim))).to(torch.bfloat16).to(DEV)
        q = fused[:, :heads * dim].unflatten(1, (heads, dim))
        q[7, 0] *= 2.0 ** -12
        q[7, 0, 3] = 2.0
        q[8, 2] = 0.0
        out = torch.full((m + 96, heads, dim), 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((m + 96, heads), 7.0, device=DEV)
        cu = R.cu([m, 90]) + 3
        ctx.ficoco_cache_attention(cache.device(), q, cu, out=out, lse=lse)
        want, want_lse, tol, ltol = R.attention(cache, q[3:3 + m + 90], [m, 90])
        assert (np.abs(out[3:-3].double().cpu().numpy() - want) <= tol).all()
        assert (np.abs(lse[3:-3].double().cpu().numpy() - want_lse) <= ltol).all()
        for rest in (out[:3], out[-3:], lse[:3], lse[-3:]):
            assert (rest == 7.0).all()
        k, v = rng.standard_normal((m, kv, dim)), rng.standard_normal((m, kv, dim))
        v[m - 30, 1, 5] = np.nan
        cache.write(0, n - m, k, v)
        q2 = rows_of(rng, [m, 90], heads, dim, "bf16")
        q2[0, 0, 2] = float("inf")
        got = ctx.ficoco_cache_attention(cache.device(), q2, R.cu([m, 90])).float().cpu().numpy()
        bad = np.isnan(got).all(2)
        want = np.zeros((m + 90, heads), dtype=bool)
        want[0, 0] = True
        want[m - 30:m, 2:4] = True
        assert (np.isnan(got).any(2) == bad).all() and (bad == want).all()
        assert ctx.ficoco_status() == 0


@pytest.mark.parametrize("dim", [64, 128, 48])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_scales_far_apart(ctx, dim, dtype):
    """Pages whose scales differ by 2^40, sharp softmaxes, a query row of one large element and small ones."""
    rng = np.random.default_rng(7)
    cache = R.Cache(rng, [400, 33], 16, 2, dim)
    for p in range(cache.vs.shape[0]):
        if not np.isnan(cache.vs[p, 0]):
            cache.vs[p] *= 2.0 ** rng.integers(-20, 21)
            cache.ks[p] *= 2.0 ** rng.integers(-6, 3)
    q = rows_of(rng, [2, 1], 4, dim, dtype, 4.0)
    q[0, 0] *= 2.0 ** -12
    q[0, 0, 3] = 2.0
    q[1, 2] = 0.0
    check_attention(ctx, cache, q, [2, 1])


def test_attention_nan_tokens_and_rows(ctx):
    """A poisoned token reaches the rows that see it, a NaN in a query row that row alone."""
    rng = np.random.default_rng(3)
    for dim, rows in ((128, 6), (64, 6), (128, 150), (48, 6)):
        cache = R.Cache(rng, [300], 64, 2, dim)
        k, v = rng.standard_normal((rows, 2, dim)), rng.standard_normal((rows, 2, dim))
        v[rows - 3, 1, 5] = np.inf                       # the token at position 297, head 1
        cache.write(0, 300 - rows, k, v)
        q = rows_of(rng, [rows], 4, dim, "bf16")
        q[0, 0, 2] = float("nan")
        out = ctx.ficoco_cache_attention(cache.device(), q, R.cu([rows])).float().cpu().numpy()
        bad = np.isnan(out).all(2)
        assert (np.isnan(out).any(2) == bad).all()
        want = np.zeros((rows, 4), dtype=bool)
        want[0, 0] = True
        want[rows - 3:, 2:] = True
        assert (bad == want).all()
        assert ctx.ficoco_status() == 0


def test_attention_fused_rows_padding_and_out_buffers(ctx):
    """Rows cut out of a fused projection, rows behind the last sequence left as they were, cu_rows that start behind row 0."""
    rng = np.random.default_rng(11)
    for dim, heads, kv, rows in ((128, 4, 2, [1, 3]), (128, 4, 2, [70, 3]), (80, 4, 2, [1, 3])):
        cache = R.Cache(rng, [100, 40], 16, kv, dim)
        total = sum(rows)
        fused = torch.from_numpy(rng.standard_normal((total + 5, (heads + 2 * kv) * dim))).to(torch.bfloat16).to(DEV)
        q = fused[:, :heads * dim].unflatten(1, (heads, dim))
        out = torch.full((total + 5, heads, dim), 7.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((total + 5, heads), 7.0, device=DEV)
        cu = R.cu(rows) + 2
        ctx.ficoco_cache_attention(cache.device(), q, cu, out=out, lse=lse)
        want, want_lse, tol, ltol = R.attention(cache, q[2:2 + total], rows)
        assert (np.abs(out[2:2 + total].double().cpu().numpy() - want) <= tol).all()
        assert (np.abs(lse[2:2 + total].double().cpu().numpy() - want_lse) <= ltol).all()
        for rest in (out[:2], out[2 + total:], lse[:2], lse[2 + total:]):
            assert (rest == 7.0).all()
        assert ctx.ficoco_status() == 0


def test_strided_tables_and_windows_that_hide_nothing(ctx):
    """A table cut out of a wider one; the largest window and more sinks than tokens are no mask, also with more rows than tokens."""
    rng = np.random.default_rng(13)
    for heads, kv, rows in ((4, 2, [1, 40]), (16, 8, [300, 300])):
        cache = R.Cache(rng, [400, 30], 32, kv, 128)
        dc = cache.device()
        wide = torch.full((2, dc.page_table.shape[1] + 7), -3, dtype=torch.int32, device=DEV)
        wide[:, 4:4 + dc.page_table.shape[1]] = dc.page_table
        dc = binding.PagedCache(dc.k_codes, dc.v_codes, dc.k_scale, dc.v_scale, wide[:, 4:4 + dc.page_table.shape[1]], dc.lengths)
        q = rows_of(rng, rows, heads, 128, "bf16")
        cu = R.cu(rows)
        a = ctx.ficoco_cache_attention(dc, q, cu)
        assert torch.equal(a, ctx.ficoco_cache_attention(dc, q, cu, window=2 ** 31 - 1))
        assert torch.equal(a, ctx.ficoco_cache_attention(dc, q, cu, window=2 ** 31 - 1, sinks=2 ** 31 - 1))
        want, _, tol, _ = R.attention(cache, q, rows)
        assert (np.abs(a.double().cpu().numpy() - want) <= tol).all()
        want, _, tol, _ = R.attention(cache, q, rows, window=1, sinks=10 ** 6)
        got = ctx.ficoco_cache_attention(dc, q, cu, window=1, sinks=2 ** 31 - 1)
        assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()
        assert ctx.ficoco_status() == 0


def test_attention_same_bits_again_and_on_another_stream(ctx):
    rng = np.random.default_rng(5)
    cache = R.Cache(rng, [3000, 500, 17], 32, 2, 128)
    q = rows_of(rng, [1, 1, 1], 8, 128, "bf16")
    dc = cache.device()
    a = ctx.ficoco_cache_attention(dc, q, R.cu([1, 1, 1]))
    for _ in range(3):
        assert torch.equal(a, ctx.ficoco_cache_attention(dc, q, R.cu([1, 1, 1])))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = ctx.ficoco_cache_attention(dc, q, R.cu([1, 1, 1]))
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a, b)


@pytest.mark.parametrize("n_rows", [1, 80, 256])
def test_attention_in_a_graph_follows_lengths_and_tables(ctx, n_rows):
    rng = np.random.default_rng(6)
    heads, kv = (4, 2) if n_rows < 100 else (16, 8)
    cache = R.Cache(rng, [400, 300], 32, kv, 128)
    rows = [n_rows, n_rows]
    q = rows_of(rng, rows, heads, 128, "bf16")
    dc = cache.device()
    out, lse = ctx.ficoco_cache_attention(dc, q, R.cu(rows), want_lse=True)
    cu = R.cu(rows)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.ficoco_cache_attention(dc, q, cu, out=out, lse=lse)
    for lengths in ([400, 300], [129, 90], [300, 257]):
        cache.lengths = lengths
        dc.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        q.copy_(rows_of(rng, rows, heads, 128, "bf16"))
        g.replay()
        torch.cuda.synchronize()
        want, want_lse, tol, ltol = R.attention(cache, q, rows)
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
        got_lse, some = lse.double().cpu().numpy(), np.isfinite(want_lse)          # (more rows than tokens: -infinity)
        assert (np.abs(got_lse[some] - want_lse[some]) <= ltol[some]).all() and np.array_equal(got_lse[~some], want_lse[~some])
    assert ctx.ficoco_status() == 0


# dim, page, heads, kv, dtype, lengths, rows, n_text, first, count, mask
WEIGHTS = [
    (128, 64, 4, 4, "bf16", [100, 100], [100, 100], 20, 0, 80, {}),
    (128, 32, 8, 2, "fp32", [200], [37], 37, 35, 120, {}),
    (64, 16, 4, 2, "bf16", [150, 90], [40, 70], 33, 5, 300, {}),
    (64, 128, 6, 2, "fp32", [140], [9], 9, 3, 129, {}),
    (128, 16, 4, 1, "bf16", [400, 10], [70, 3], 70, 0, 333, {}),
    (128, 16, 4, 2, "bf16", [300], [50], 50, 10, 200, dict(window=60, sinks=14)),
    (128, 64, 4, 2, "bf16", [300, 0], [5, 0], 5, 0, 300, dict(causal=False)),
    (80, 16, 4, 2, "bf16", [100], [10], 10, 1, 90, {}),
    (256, 16, 4, 2, "fp32", [50], [10], 12, 1, 90, {}),
    (128, 64, 2, 2, "bf16", [700], [200], 200, 0, 1, {}),
]


@pytest.mark.parametrize("dim,page,heads,kv,dtype,lengths,rows,n_text,first,count,mask", WEIGHTS)
def test_weights(ctx, dim, page, heads, kv, dtype, lengths, rows, n_text, first, count, mask):
    rng = np.random.default_rng(dim + heads + n_text)
    cache = R.Cache(rng, lengths, page, kv, dim)
    q = rows_of(rng, rows, heads, dim, dtype)
    dc = cache.device()
    _, lse = ctx.ficoco_cache_attention(dc, q, R.cu(rows), want_lse=True, **mask)
    out = torch.full((len(rows), heads, n_text, count), float("nan"), device=DEV)
    ctx.ficoco_cache_weights(dc, q, lse, R.cu(rows), n_text, first, count, out=out, **mask)
    assert ctx.ficoco_status() == 0
    want, tol = R.weights(cache, q, lse, rows, n_text, first, count, **mask)
    got = out.double().cpu().numpy()
    assert ((np.abs(got - want) <= tol)).all(), np.max(np.abs(got - want) / tol)
    assert (got[want == 0] == 0).all()


def same_cache(dc, cache, unused=()):
    torch.cuda.synchronize()
    for got, want in ((dc.k_codes, cache.kc), (dc.v_codes, cache.vc)):
        assert np.array_equal(got.view(torch.uint8).cpu().numpy(), want)
    for got, want in ((dc.k_scale, cache.ks), (dc.v_scale, cache.vs)):
        assert np.array_equal(got.cpu().numpy(), want, equal_nan=True)


APPEND = [
    (128, 64, 2, "bf16", [100, 64, 1, 0, 65, 200], [1, 1, 1, 0, 1, 1]),
    (128, 16, 1, "fp32", [100, 33, 16], [100, 1, 15]),
    (64, 32, 3, "bf16", [70, 140, 5], [39, 140, 0]),
    (80, 128, 2, "fp32", [300, 129], [173, 1]),
    (256, 16, 2, "bf16", [50], [34]),
    (16, 128, 1, "bf16", list(range(1, 290)), [1 + i % 2 if i else 1 for i in range(289)]),
]


@pytest.mark.parametrize("dim,page,kv,dtype,lengths,rows", APPEND)
def test_append_bit_for_bit(ctx, dim, page, kv, dtype, lengths, rows):
    """Codes, scales, rescaled pages and everything that stays as it was."""
    rng = np.random.default_rng(dim + page)
    before = [n - m for n, m in zip(lengths, rows)]
    cache = R.Cache(rng, before, page, kv, dim, spare=sum(-(-n // page) for n in lengths) + 2)
    at = 0
    for b, n in enumerate(lengths):                     # pages that the new rows open
        have, need = -(-before[b] // page), -(-n // page)
        if need >= cache.table.shape[1]:
            cache.table = np.pad(cache.table, ((0, 0), (0, need - cache.table.shape[1] + 1)), constant_values=-7)
        cache.table[b, have:need] = cache.spare[at:at + need - have]
        at += need - have
    dc0 = cache.device()
    dc = binding.PagedCache(dc0.k_codes, dc0.v_codes, dc0.k_scale, dc0.v_scale, dc0.page_table,
                            torch.tensor(lengths, dtype=torch.int32, device=DEV))
    total = sum(rows)
    grow = np.repeat(2.0 ** rng.integers(-3, 6, len(rows)), rows)[:, None, None]
    k = torch.from_numpy(rng.standard_normal((total + 3, kv, dim))).to(DT[dtype])
    v = torch.from_numpy(rng.standard_normal((total + 3, kv, dim))).to(DT[dtype])
    k[:total] *= torch.from_numpy(grow).to(DT[dtype])
    v[total // 2] = 0
    if total > 4:
        k[2, 0, 3], v[total - 1, 0, 1], k[total - 2, -1, 0] = float("nan"), float("-inf"), float("inf")
        v[3, 0] = 1e-30
    k[total:] = float("nan")                            # rows behind the last sequence
    ctx.ficoco_cache_append(dc, k.to(DEV), v.to(DEV), R.cu(rows))
    assert ctx.ficoco_status() == 0
    r = 0
    for b, m in enumerate(rows):
        cache.write(b, before[b], k[r:r + m].double().numpy(), v[r:r + m].double().numpy())
        r += m
    same_cache(dc, cache)


def test_append_scale_borders(ctx):
    """Largest magnitudes at 448 * 2^e, just above it, zero, and at the ends of the range."""
    values = [448.0, 449.0, 1.75, 1.7500001, 0.0, 2.0 ** -70, 448 * 2.0 ** -64, 449 * 2.0 ** -64, 1e30, 3e38]
    cache = R.Cache(np.random.default_rng(1), [0] * len(values), 16, 1, 16, spare=len(values))
    cache.table[:, 0] = cache.spare
    cache.lengths = [1] * len(values)
    k = torch.zeros((len(values), 1, 16))
    k[:, 0, 5] = torch.tensor(values)
    k[:, 0, 6] = -torch.tensor(values) / 3
    dc = cache.device()
    ctx.ficoco_cache_append(dc, k.to(DEV), (-k).to(DEV), R.cu([1] * len(values)))
    for b in range(len(values)):
        cache.write(b, 0, k[b:b + 1].double().numpy(), -k[b:b + 1].double().numpy())
    same_cache(dc, cache)


@pytest.mark.parametrize("dim,page,kv,lengths,first,keep", [
    (128, 64, 2, [640, 100, 64, 1], 0, [128, 64, 0, 1]),
    (64, 16, 3, [300, 35, 20, 0], 35, [100, 0, 0, 0]),
    (80, 128, 1, [500, 200], 7, [129, 121]),
    (16, 32, 2, list(range(1, 270)), 3, [max(0, n - 3) // 2 for n in range(1, 270)]),
])
def test_compact_bit_for_bit(ctx, dim, page, kv, lengths, first, keep):
    rng = np.random.default_rng(dim)
    front = [min(n, first) for n in lengths]
    new = [f + m for f, m in zip(front, keep)]
    cache = R.Cache(rng, lengths, page, kv, dim, spare=sum(-(-n // page) for n in new) + 2)
    for p in range(cache.vs.shape[0]):
        cache.ks[p] *= 2.0 ** rng.integers(-8, 9)
        cache.vs[p] *= 2.0 ** rng.integers(-8, 9)
    if lengths[0] > 2:
        cache.kc[cache.table[0, 0], 0, 1], cache.vc[cache.table[0, 0], 0, 1] = 0x7F, 0        # a poisoned token
    kept = [rng.permutation(n - f)[:m].astype(np.int32) for n, f, m in zip(lengths, front, keep)]     # in any order
    to = np.full((len(lengths), max(max(-(-n // page) for n in new), 1) + 1), -5, dtype=np.int32)
    at = 0
    for b, n in enumerate(new):
        p = -(-n // page)
        to[b, :p] = cache.spare[at:at + p]
        at += p
    dc = cache.device()
    got = ctx.ficoco_cache_compact(dc, torch.from_numpy(to).to(DEV), torch.from_numpy(np.concatenate(kept + [[9999]]).astype(np.int32)).to(DEV),
                                   R.cu(keep), first=first)
    assert got.tolist() == new and ctx.ficoco_status() == 0
    for b, n in enumerate(new):
        pos = np.concatenate([np.arange(front[b]), front[b] + kept[b]]).astype(int)
        for pi in range(-(-n // page)):
            at = pos[pi * page:(pi + 1) * page]
            sp, page_to = cache.table[b, at // page], to[b, pi]
            for codes, scales in ((cache.kc, cache.ks), (cache.vc, cache.vs)):
                for h in range(kv):
                    x = R.E4M3[codes[sp, h, at % page]] * scales[sp, h].astype(np.float64)[:, None]
                    s = R.scale_of(np.nanmax(np.abs(x))) if not np.isnan(x).all() else R.scale_of(0.0)
                    scales[page_to, h] = s
                    codes[page_to, h, :len(at)] = np.where(np.isnan(x), 127, R.to_codes(x / s))
    same_cache(dc, cache)


@pytest.mark.parametrize("dim,page,kv", [(128, 64, 8), (16, 16, 1), (256, 128, 3)])
def test_copy(ctx, dim, page, kv):
    rng = np.random.default_rng(2)
    cache = R.Cache(rng, [page * 5], page, kv, dim, spare=6, garbage=False)
    own, spare = cache.table[0, :5].copy(), cache.spare
    src = [own[0], own[3], own[0], -1, own[2], own[1]]
    dst = [spare[0], spare[1], spare[2], spare[3], -1, own[1]]
    dc = cache.device()
    t = lambda x: torch.tensor(np.array(x, dtype=np.int32), device=DEV)      # noqa: E731
    ctx.ficoco_cache_copy(dc, t(src), t(dst))
    ctx.ficoco_cache_copy(dc, t([]), t([]))
    assert ctx.ficoco_status() == 0
    for a, b in zip(src, dst):
        if a >= 0 and b >= 0:
            for x in (cache.kc, cache.vc, cache.ks, cache.vs):
                x[b] = x[a]
    same_cache(dc, cache)


def test_what_only_the_device_can_see(ctx):
    """Pages, lengths, row offsets and kept indices out of range raise the status bit and stay inside the buffers."""
    rng = np.random.default_rng(4)
    t = lambda x: torch.tensor(np.array(x, dtype=np.int32), device=DEV)      # noqa: E731
    for dim, n in ((128, 1), (128, 100), (80, 1)):
        cache = R.Cache(rng, [200, 100], 64, 2, dim, garbage=False)
        q = rows_of(rng, [n, n], 4, dim, "bf16")
        k = rows_of(rng, [n, n], 2, dim, "bf16")
        for what in ("page", "negative page", "length", "negative length", "rows", "descending rows"):
            dc, cu = cache.device(), R.cu([n, n])
            if what == "page":
                dc.page_table[0, 0] = 1 << 20
                dc.page_table[1, 1] = 1 << 20
            elif what == "negative page":
                dc.page_table[:, 0] = -1
                dc.page_table[:, 1] = -1
                dc.page_table[:, 3] = -1
            elif what == "length":
                dc.page_table.clamp_(0, dc.struct.n_pages - 1)
                dc.lengths[0] = 1 << 30
            elif what == "negative length":
                dc.lengths[1] = -3
            elif what == "rows":
                cu[2] = 1 << 24
            else:
                cu[1] = -5
            _, lse = ctx.ficoco_cache_attention(dc, q, cu, want_lse=True)
            assert ctx.ficoco_status() == 16, what
            ctx.ficoco_cache_weights(dc, q, lse, cu, n, 0, 90)
            assert ctx.ficoco_status() == 16, what
            ctx.ficoco_cache_append(dc, k, k, cu)
            assert ctx.ficoco_status() == 16, what
        dc = cache.device()
        to = t([[cache.spare[0]], [cache.spare[1]]])
        for kept in ([5, -1], [5, 200]):
            ctx.ficoco_cache_compact(dc, to, t(kept), t([0, 1, 2]))
            assert ctx.ficoco_status() == 16
        # kept indices whose sum with `first` passes 32 bits: token 0 in their place, as for every other one outside
        for e in ((1 << 31) - 1, (1 << 31) - 8, -(1 << 31)):
            ctx.ficoco_cache_compact(dc, to, t([0, e]), t([0, 1, 2]), first=8)
            assert ctx.ficoco_status() == 16
            page, first_page = int(cache.spare[1]), int(dc.page_table[1, 0])
            same = dc.k_codes[page, :, 8].view(torch.uint8) == dc.k_codes[page, :, 0].view(torch.uint8)
            assert bool(same.all()) and bool((dc.k_codes[first_page, :, 0].view(torch.uint8) != 0).any()), e
        ctx.ficoco_cache_compact(dc, t([[1 << 20], [-1]]), t([1, 2]), t([0, 1, 2]))
        assert ctx.ficoco_status() == 16
        ctx.ficoco_cache_compact(dc, to, t([1, 2]), t([0, 1, 70000]))
        assert ctx.ficoco_status() == 16
        ctx.ficoco_cache_copy(dc, t([0, 1 << 20]), t([1 << 20, 0]))
        assert ctx.ficoco_status() == 16


def test_page_indexes_beyond_32_bit_offsets(ctx):
    """A pool of more than 2^31 bytes of codes: pages at its end are written, copied, gathered and read."""
    page, kv, dim = 128, 8, 128
    n_pages = (1 << 31) // (page * kv * dim) + 40
    rng = np.random.default_rng(8)
    small = R.Cache(rng, [300, 257], page, kv, dim, spare=4)
    codes = [torch.full((n_pages, kv, page, dim), 0x7F, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.full((n_pages, kv), float("nan"), device=DEV) for _ in range(2)]
    shift = n_pages - small.kc.shape[0]
    t = lambda a: torch.from_numpy(a.copy()).to(DEV)      # noqa: E731
    for big, part in zip(codes + scales, (small.kc, small.vc, small.ks, small.vs)):
        big[shift:] = t(part)
    table = t(np.where(small.table >= 0, small.table + shift, small.table).astype(np.int32))
    dc = binding.PagedCache(codes[0], codes[1], scales[0], scales[1], table, t(np.array(small.lengths, dtype=np.int32)))
    for n in (1, 100):
        rows = [n, n]
        q = rows_of(rng, rows, 8, dim, "bf16")
        out, lse = ctx.ficoco_cache_attention(dc, q, R.cu(rows), want_lse=True)
        want, _, tol, _ = R.attention(small, q, rows)
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
        w = ctx.ficoco_cache_weights(dc, q, lse, R.cu(rows), n, 0, 250)
        want, tol = R.weights(small, q, lse, rows, n, 0, 250)
        assert (np.abs(w.double().cpu().numpy() - want) <= tol).all()
    k = torch.from_numpy(rng.standard_normal((2, kv, dim)) * 9).to(DEV).float()
    ctx.ficoco_cache_append(dc, k, k, R.cu([1, 1]))
    for b in range(2):
        small.write(b, small.lengths[b] - 1, k[b:b + 1].double().cpu().numpy(), k[b:b + 1].double().cpu().numpy())
    spare = (small.spare + shift).astype(np.int32)
    got = ctx.ficoco_cache_compact(dc, t(spare[:2].reshape(2, 1)), t(np.arange(200, dtype=np.int32)), R.cu([100, 100]))
    assert got.tolist() == [100, 100]
    ctx.ficoco_cache_copy(dc, t(spare[:1]), t(spare[2:3]))
    torch.cuda.synchronize()
    assert torch.equal(codes[0][spare[0]], codes[0][spare[2]]) and ctx.ficoco_status() == 0
    first = small.table[0, 0]
    assert np.array_equal(codes[0][shift:].cpu().numpy()[first], small.kc[first])


def test_a_decoder_layer_with_its_reduce_step(ctx):
    """Prompts are appended and attended to, their text -> vision weights feed ficoco_l_reduce, the cache keeps what the step
    kept, a sequence is forked, and single tokens go on from there, with a captured step among them."""
    rng = np.random.default_rng(21)
    batch, vision, text, heads, kv, dim, page, keep = 2, 144, 20, 4, 2, 64, 16, 30
    n = vision + text
    pool = binding.PagePool(80)
    per = -(-n // page)
    pages = [pool.take(per + 1) for _ in range(batch)]
    dc = binding.PagedCache.empty(80, kv, page, dim, batch, per + 1, DEV)
    dc.page_table.copy_(torch.tensor(pages, dtype=torch.int32))
    dc.lengths.fill_(n)
    host = R.Cache(rng, [0, 0], page, kv, dim, spare=78, garbage=False)
    host.table, host.lengths = np.array(pages, dtype=np.int32), [n, n]
    host.kc[:], host.vc[:], host.ks[:], host.vs[:] = 0, 0, 1.0, 1.0
    qkv = torch.from_numpy(rng.standard_normal((batch * n, heads + 2 * kv, dim))).to(torch.bfloat16).to(DEV)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
    cu = R.cu([n, n])
    ctx.ficoco_cache_append(dc, k, v, cu)
    for b in range(batch):
        host.write(b, 0, k[b * n:(b + 1) * n].double().cpu().numpy(), v[b * n:(b + 1) * n].double().cpu().numpy())
    out, lse = ctx.ficoco_cache_attention(dc, q, cu, want_lse=True)
    want, _, tol, _ = R.attention(host, q, [n, n])
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    t2v = ctx.ficoco_cache_weights(dc, q, lse, cu, text, 0, vision)
    want, tol = R.weights(host, q, lse, [n, n], text, 0, vision)
    assert (np.abs(t2v.double().cpu().numpy() - want) <= tol).all()
    hidden = torch.from_numpy(rng.standard_normal((batch * n, 512)) / 16).to(torch.bfloat16).to(DEV)
    res = ctx.ficoco_l_reduce(hidden, t2v, keep, vision, text, heads)
    assert res.out_rows == [keep + text] * batch
    total = keep + text
    new = [pool.take(-(-total // page) + 1) for _ in range(batch)]
    to = torch.tensor(new, dtype=torch.int32, device=DEV)
    lengths = ctx.ficoco_cache_compact(dc, to, res.kept_idx, R.cu([total, total]))
    for p in pages:
        pool.give(p)
    assert pool.free_pages == 80 - sum(map(len, new))
    # the compacted layer, and its first sequence forked: a third sequence that shares the full pages
    forked, pair = pool.fork(new[0][:-(-total // page)], page, total)
    assert pair is not None and forked[:total // page] == new[0][:total // page]
    one = torch.tensor([pair[0]], dtype=torch.int32, device=DEV), torch.tensor([pair[1]], dtype=torch.int32, device=DEV)
    ctx.ficoco_cache_copy(dc, *one)
    third = forked + pool.take(1)
    table = torch.tensor(new + [third], dtype=torch.int32, device=DEV)
    after = binding.PagedCache(dc.k_codes, dc.v_codes, dc.k_scale, dc.v_scale, table, torch.cat([lengths, lengths[:1]]))
    now = R.Cache(rng, [0, 0, 0], page, kv, dim, spare=77, garbage=False)
    now.table, now.lengths = np.array(new + [third], dtype=np.int32), [total] * 3
    now.kc, now.vc = (x.view(torch.uint8).cpu().numpy().copy() for x in (dc.k_codes, dc.v_codes))
    now.ks, now.vs = dc.k_scale.cpu().numpy().copy(), dc.v_scale.cpu().numpy().copy()
    kept = res.kept_idx.cpu().numpy().reshape(batch, total)
    for b in range(batch):                              # every kept token is the one that was there, but for the second rounding
        for h in range(kv):
            was, is_ = host.tokens(b, h)[0][kept[b]], now.tokens(b, h)[0]
            assert (np.abs(was - is_) <= np.abs(was) * 2.0 ** -4 + 448 * 2.0 ** -10 * now.ks[now.table[b, 0], h]).all()
    step = R.cu([1, 1, 1])
    qs, ks, vs = (torch.zeros((3, x, dim), dtype=torch.bfloat16, device=DEV) for x in (heads, kv, kv))
    out = torch.zeros((3, heads, dim), dtype=torch.bfloat16, device=DEV)

    def decode():
        after.lengths.add_(1)
        ctx.ficoco_cache_append(after, ks, vs, step)
        ctx.ficoco_cache_attention(after, qs, step, out=out)

    graph = None
    for i in range(5):
        for x in (qs, ks, vs):
            x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape)) * (1 + i)))
        if i == 2:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                decode()
        if graph is not None:
            graph.replay()
        else:
            decode()
        torch.cuda.synchronize()
        now.lengths = [total + i + 1] * 3
        for b in range(3):
            now.write(b, total + i, ks[b:b + 1].double().cpu().numpy(), vs[b:b + 1].double().cpu().numpy())
        same = after.k_codes.view(torch.uint8).cpu().numpy()
        for b in range(3):
            assert np.array_equal(same[now.table[b]], now.kc[now.table[b]])
        want, _, tol, _ = R.attention(now, qs, [1, 1, 1])
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    assert after.lengths.tolist() == now.lengths and ctx.ficoco_status() == 0
    pool.close()


def test_a_wait_that_runs_out_ends_the_call_and_the_context_recovers():
    """A barrier that expects an arrival too many (the testing hook): the kernels give up, raise bit 2 and write nothing more, later
    calls do nothing until the status has been read, then results are the same bits as before."""
    c = binding.Context(max_tokens=1024, max_dim=128, max_batch=4, max_text=16, device=0)
    rng = np.random.default_rng(9)
    cache = R.Cache(rng, [3000, 700], 32, 4, 128)
    dc = cache.device()
    try:
        for n, heads in ((1, 8), (400, 16)):
            rows = [n, n]
            q = rows_of(rng, rows, heads, 128, "bf16")
            cu = R.cu(rows)
            good, lse = c.ficoco_cache_attention(dc, q, cu, want_lse=True)
            w = c.ficoco_cache_weights(dc, q, lse, cu, 1, 0, 600)
            torch.cuda.synchronize()
            assert c.ficoco_status() == 0
            for call in (lambda: c.ficoco_cache_attention(dc, q, cu), lambda: c.ficoco_cache_weights(dc, q, lse, cu, 1, 0, 600)):
                c.ficoco_debug_waits(200_000, 1)
                call()
                c.ficoco_debug_waits(0, 0)
                out = torch.full_like(q, 3.0)
                c.ficoco_cache_attention(dc, q, cu, out=out)
                torch.cuda.synchronize()
                assert (out == 3.0).all()
                assert c.ficoco_status() == 4
                assert torch.equal(good, c.ficoco_cache_attention(dc, q, cu))
                assert torch.equal(w, c.ficoco_cache_weights(dc, q, lse, cu, 1, 0, 600))
                assert c.ficoco_status() == 0
    finally:
        c.close()


def test_first_attention_of_a_context_is_refused_under_capture():
    c = binding.Context(max_tokens=1024, max_dim=128, max_batch=4, max_text=16, device=0)
    rng = np.random.default_rng(10)
    dc = R.Cache(rng, [50], 32, 2, 128).device()
    q = rows_of(rng, [1], 2, 128, "bf16")
    cu, out = R.cu([1]), torch.empty_like(q)
    torch.cuda.synchronize()
    try:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            with pytest.raises(binding.FicocoError) as e:
                c.ficoco_cache_attention(dc, q, cu, out=out)
            out.fill_(1.0)
        assert e.value.code == -7
        g.replay()
        torch.cuda.synchronize()
        assert (out == 1.0).all()
        a = c.ficoco_cache_attention(dc, q, cu)
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            c.ficoco_cache_attention(dc, q, cu, out=out)
        assert torch.isfinite(a).all()
    finally:
        c.close()


@pytest.mark.parametrize("dim", [128, 48])
def test_weights_of_tokens_far_behind_the_end(ctx, dim):
    """The last tokens that a call can name (the tile's end is 2^31) weigh nothing, whatever the last tile has left in shared memory."""
    rng = np.random.default_rng(12)
    dc = R.Cache(rng, [200, 64], 64, 2, dim).device()
    q, cu = rows_of(rng, [2, 2], 4, dim, "bf16"), R.cu([2, 2])
    _, lse = ctx.ficoco_cache_attention(dc, q, cu, want_lse=True)
    assert ctx.ficoco_cache_weights(dc, q, lse, cu, 2, 0, 64).abs().sum() > 0
    for first, count in (((1 << 31) - 100, 99), ((1 << 30), 300), ((1 << 31) - 2, 1)):
        w = ctx.ficoco_cache_weights(dc, q, lse, cu, 2, first, count)
        assert torch.equal(w, torch.zeros_like(w)), (first, count)
    assert ctx.ficoco_status() == 0


def test_a_prompt_prepares_the_context_for_captured_single_tokens():
    """The first attention call allocates, whatever kernel it takes: single tokens may be captured after an eager prompt."""
    c = binding.Context(max_tokens=1024, max_dim=128, max_batch=4, max_text=16, device=0)
    rng = np.random.default_rng(11)
    dc = R.Cache(rng, [2100], 64, 2, 128).device()
    q, one = rows_of(rng, [2048], 32, 128, "bf16"), rows_of(rng, [1], 32, 128, "bf16")
    cu, cu1, out = R.cu([2048]), R.cu([1]), torch.empty_like(one)
    try:
        c.ficoco_profile(True)
        c.ficoco_cache_attention(dc, q, cu)
        assert [name for name, _, _ in c.ficoco_profile_read()] == ["k_cache_prompt"]
        c.ficoco_profile(False)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.ficoco_cache_attention(dc, one, cu1, out=out)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, c.ficoco_cache_attention(dc, one, cu1))
        assert c.ficoco_status() == 0
    finally:
        c.close()


def test_empty_calls(ctx):
    rng = np.random.default_rng(12)
    cache = R.Cache(rng, [0, 30], 16, 2, 64)
    dc = cache.device()
    none = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    out, lse = ctx.ficoco_cache_attention(dc, none, R.cu([0, 0]), want_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    ctx.ficoco_cache_append(dc, none[:, :2], none[:, :2], R.cu([0, 0]))
    w = ctx.ficoco_cache_weights(dc, none, lse, R.cu([0, 0]), 3, 0, 40)
    assert w.shape == (2, 4, 3, 40) and (w == 0).all()
    kept = torch.empty((0,), dtype=torch.int32, device=DEV)
    to = torch.full((2, 2), -1, dtype=torch.int32, device=DEV)
    to[1, 0] = int(cache.spare[0])
    assert ctx.ficoco_cache_compact(dc, to, kept, R.cu([0, 0]), first=9).tolist() == [0, 9]
    assert ctx.ficoco_status() == 0
    with pytest.raises(ValueError):
        ctx.ficoco_cache_attention(dc, none.cpu(), R.cu([0, 0]))
