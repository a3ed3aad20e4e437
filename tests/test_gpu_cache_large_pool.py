"""A pool whose codes pass 2^32 bytes: pages at its end are appended to, gathered and copied, bit for bit, and nothing else changes."""
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


@pytest.mark.parametrize("page,kv,dim", [(128, 8, 128), (16, 32, 64)])
def test_pages_behind_4_gb_of_codes(ctx, page, kv, dim):
    rng = np.random.default_rng(8)
    before, rows = [300, 257], [60, 1]
    lengths = [n + m for n, m in zip(before, rows)]
    keep = [100, 33]
    small = R.Cache(rng, before, page, kv, dim, spare=40, max_pages=-(-max(lengths) // page) + 1)
    free = list(small.spare)
    for b, (n, m) in enumerate(zip(before, lengths)):
        for pi in range(-(-n // page), -(-m // page)):
            small.table[b, pi] = free.pop()
    to = np.full((2, -(-max(keep) // page)), -1, dtype=np.int32)
    for b, m in enumerate(keep):
        for pi in range(-(-m // page)):
            to[b, pi] = free.pop()
    copied = free.pop()

    n_pages = (1 << 32) // (page * kv * dim) + small.kc.shape[0]
    shift = n_pages - small.kc.shape[0]
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)      # noqa: E731
    moved = lambda a: t(np.where(a >= 0, a + shift, a).astype(np.int32))  # noqa: E731
    codes = [torch.full((n_pages, kv, page, dim), 0x2A, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.full((n_pages, kv), 0.75, device=DEV) for _ in range(2)]
    host = (small.kc, small.vc, small.ks, small.vs)
    for big, part in zip(codes + scales, host):
        big[shift:] = t(part)
    dc = binding.PagedCache(codes[0], codes[1], scales[0], scales[1], moved(small.table), t(np.array(lengths, dtype=np.int32)))

    def same():
        torch.cuda.synchronize()
        assert ctx.ficoco_status() == 0
        for big, part in zip(codes + scales, host):
            assert np.array_equal(big[shift:].cpu().numpy(), part, equal_nan=part.dtype == np.float32)
            assert bool((big[:shift] == (0x2A if part.dtype == np.uint8 else 0.75)).all())

    def differs(page_at):                                # (what the next call writes is not there yet)
        return all(not np.array_equal(big[shift + page_at].cpu().numpy(), part[page_at]) for big, part in zip(codes, host))

    same()
    k, v = (torch.from_numpy(rng.standard_normal((sum(rows), kv, dim)) * 9).float() for _ in range(2))
    r = 0
    for b, m in enumerate(rows):
        small.write(b, before[b], k[r:r + m].double().numpy(), v[r:r + m].double().numpy())
        r += m
    small.lengths = lengths
    assert all(differs(small.table[b, (lengths[b] - 1) // page]) for b in range(2))
    ctx.ficoco_cache_append(dc, k.to(DEV), v.to(DEV), R.cu(rows))
    same()

    kept = [rng.permutation(n)[:m].astype(np.int32) for n, m in zip(lengths, keep)]
    for b, m in enumerate(keep):
        for pi in range(-(-m // page)):
            at = kept[b][pi * page:(pi + 1) * page]
            sp, page_to = small.table[b, at // page], to[b, pi]
            for c, s in ((small.kc, small.ks), (small.vc, small.vs)):
                for h in range(kv):
                    x = R.E4M3[c[sp, h, at % page]] * s[sp, h].astype(np.float64)[:, None]
                    s[page_to, h] = R.scale_of(np.abs(x).max())
                    c[page_to, h, :len(at)] = R.to_codes(x / s[page_to, h])
    assert all(differs(p) for p in to[to >= 0])
    got = ctx.ficoco_cache_compact(dc, moved(to), t(np.concatenate(kept)), R.cu(keep))
    assert got.tolist() == keep
    same()

    for part in host:
        part[copied] = part[to[0, 0]]
    assert differs(copied)
    ctx.ficoco_cache_copy(dc, moved(to[0, :1]), moved(np.array([copied])))
    same()
