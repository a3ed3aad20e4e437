"""The 8-bit cache without a GPU: refusals before anything is launched, struct layouts, the page pool, the reference itself."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2411_17686_b200 import binding, build
from tests import cache_reference as R


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def test_struct_layouts():
    assert C.sizeof(binding.ficoco_cache) == 7 * 8 + 6 * 4
    assert C.sizeof(binding.ficoco_append_args) == 5 * 8 + 2 * 4
    assert C.sizeof(binding.ficoco_attention_args) == 5 * 8 + 7 * 4 + 4
    assert C.sizeof(binding.ficoco_compact_args) == 5 * 8 + 4 * 4


# Arguments are looked at before the context or the device: a context that is no context shows that none is touched.
FAKE = C.create_string_buffer(4096)
P16 = 0x10000


def cache(**over):
    a = dict(k_codes=P16, v_codes=P16 * 2, k_scale=P16 * 3, v_scale=P16 * 4, page_table=P16 * 5, lengths=P16 * 6, table_stride=8,
             n_pages=10, page_size=64, kv_heads=2, head_dim=128, batch=3, max_pages=8)
    a.update(over)
    return binding.ficoco_cache(*[a[f[0]] for f in binding.ficoco_cache._fields_])


def attention(**over):
    a = dict(q=P16 * 1000, cu_rows=P16 * 8, out=P16 * 2000, lse=P16 * 3000, q_stride=512, scale=0.1, dtype=1, rows=5, heads=4, window=0,
             sinks=0, flags=1)
    a.update(over)
    return binding.ficoco_attention_args(*[a[f[0]] for f in binding.ficoco_attention_args._fields_])


def append(**over):
    a = dict(k=P16 * 9, v=P16 * 10, cu_rows=P16 * 8, k_stride=256, v_stride=256, dtype=1, rows=5)
    a.update(over)
    return binding.ficoco_append_args(*[a[f[0]] for f in binding.ficoco_append_args._fields_])


def compact(**over):
    a = dict(to_table=P16 * 11, kept=P16 * 12, cu_kept=P16 * 13, lengths_out=P16 * 14, to_stride=4, to_pages=4, n_kept=9, first=0, reserved=0)
    a.update(over)
    return binding.ficoco_compact_args(*[a[f[0]] for f in binding.ficoco_compact_args._fields_])


BAD_CACHE = [
    (dict(k_codes=None), -1), (dict(v_scale=None), -1), (dict(page_table=None), -1), (dict(lengths=None), -1),
    (dict(k_codes=P16 + 8), -1), (dict(v_codes=P16 + 1), -1), (dict(n_pages=0), -1), (dict(batch=0), -1), (dict(max_pages=0), -1),
    (dict(table_stride=7), -1), (dict(kv_heads=0), -1), (dict(head_dim=0), -1),
    (dict(page_size=48), -2), (dict(page_size=256), -2), (dict(page_size=0), -2), (dict(head_dim=72), -2), (dict(head_dim=272), -2),
    (dict(batch=65536), -2), (dict(n_pages=1 << 26), -2), (dict(max_pages=1 << 26, table_stride=1 << 26), -2),
]


@pytest.mark.parametrize("over,code", BAD_CACHE)
def test_caches_that_are_refused(lib, over, code):
    c = cache(**over)
    assert lib.ficoco_cache_append(FAKE, c, append(), None) == code
    assert lib.ficoco_cache_attention(FAKE, c, attention(), None) == code
    assert lib.ficoco_cache_weights(FAKE, c, attention(), 2, 0, 3, P16, None) == code
    assert lib.ficoco_cache_copy(FAKE, c, P16, P16 * 2, 3, None) == code
    assert lib.ficoco_cache_compact(FAKE, c, compact(), None) == code


@pytest.mark.parametrize("over,code", [
    (dict(q=None), -1), (dict(q=P16 + 2), -1), (dict(cu_rows=None), -1), (dict(out=None), -1), (dict(out=P16 * 2000 + 4), -1), (dict(rows=-1), -1),
    (dict(heads=0), -1), (dict(heads=5, q_stride=640), -1), (dict(q_stride=511), -1), (dict(q_stride=513), -1), (dict(scale=0.0), -1),
    (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(window=-1), -1), (dict(sinks=-1), -1),
    (dict(flags=2), -1), (dict(dtype=2), -2), (dict(out=P16 * 1000), -1), (dict(out=P16 * 1000 + 1024 * 4 + 16), -1),
    (dict(heads=65536 * 2, q_stride=65536 * 256), -2), (dict(rows=1 << 30, out=1 << 62), -2),
])
def test_attention_calls_that_are_refused(lib, over, code):
    assert lib.ficoco_cache_attention(FAKE, cache(), attention(**over), None) == code
    if not set(over) & {"out"}:
        assert lib.ficoco_cache_weights(FAKE, cache(), attention(**over), 2, 0, 3, P16, None) == code


def test_other_calls_that_are_refused(lib):
    c = cache()
    for lse in (P16 * 3000 + 2, P16 * 2000 + 64, P16 * 1000 + 1024 * 4 + 1020):
        assert lib.ficoco_cache_attention(FAKE, c, attention(lse=lse), None) == -1
    assert lib.ficoco_cache_attention(None, c, attention(), None) == -1
    assert lib.ficoco_cache_attention(FAKE, None, attention(), None) == -1
    assert lib.ficoco_cache_attention(FAKE, c, None, None) == -1
    assert lib.ficoco_cache_append(FAKE, c, None, None) == -1
    assert lib.ficoco_cache_compact(FAKE, c, None, None) == -1
    for over, code in ((dict(k=None), -1), (dict(v=P16 + 4), -1), (dict(cu_rows=None), -1), (dict(rows=-2), -1), (dict(k_stride=255), -1),
                       (dict(v_stride=260 + 1), -1), (dict(dtype=7), -2)):
        assert lib.ficoco_cache_append(FAKE, c, append(**over), None) == code, over
    for args in ((0, 0, 3, P16), (2, -1, 3, P16), (2, 0, 0, P16), (2, 0, 3, None), (2, 0, 3, P16 + 2)):
        assert lib.ficoco_cache_weights(FAKE, c, attention(), *args, None) == -1, args
    assert lib.ficoco_cache_weights(FAKE, c, attention(lse=None), 2, 0, 3, P16, None) == -1
    assert lib.ficoco_cache_weights(FAKE, c, attention(), 2, 1 << 30, 1 << 30, P16, None) == -2
    assert lib.ficoco_cache_weights(FAKE, c, attention(), 1 << 30, 0, 3, P16, None) == -2
    for args in ((None, P16, 1), (P16, None, 1), (P16, P16, 1), (P16, P16 * 2, -1)):
        assert lib.ficoco_cache_copy(FAKE, c, *args, None) == -1, args
    for over, code in ((dict(to_table=None), -1), (dict(kept=None), -1), (dict(cu_kept=None), -1), (dict(n_kept=-1), -1), (dict(first=-1), -1),
                       (dict(to_pages=0), -1), (dict(to_stride=3), -1), (dict(to_table=P16 * 5), -1), (dict(lengths_out=P16 * 6), -1),
                       (dict(first=1 << 30), -2)):
        assert lib.ficoco_cache_compact(FAKE, c, compact(**over), None) == code, over


def test_binding_refuses_what_it_cannot_describe():
    with pytest.raises(ValueError):                     # not on a device
        binding.PagedCache.empty(4, 1, 16, 16, 1, 2, device="cpu")
    with pytest.raises(TypeError):
        z = torch.zeros((4, 1, 16, 16))
        binding.PagedCache(z, z, z[:, :, 0, 0], z[:, :, 0, 0], z[0, 0], z[0, 0, 0])
    with pytest.raises(ValueError):
        binding._rows3("q", torch.zeros(3, 2, 16), 32)
    with pytest.raises(ValueError):
        binding._int32("cu_rows", torch.zeros(3, dtype=torch.int32), 3)


def test_pool(lib):
    with pytest.raises(binding.FicocoError):
        binding.PagePool(0)
    p = binding.PagePool(6)
    a = p.take(3)
    assert a == [0, 1, 2] and p.free_pages == 3 and p.take(0) == []
    with pytest.raises(binding.FicocoError) as e:
        p.take(4)
    assert e.value.code == -10 and p.free_pages == 3
    forked, pair = p.fork(a, 16, 40)                    # two full pages and eight tokens
    assert forked == [0, 1, 3] and pair == (2, 3) and p.free_pages == 2
    again, pair = p.fork(a, 16, 32)
    assert again == [0, 1] and pair is None
    assert p.fork([], 16, 0) == ([], None)
    p.give(a)
    assert p.free_pages == 3                            # page 2 alone: 0 and 1 have two holders left
    with pytest.raises(binding.FicocoError):
        p.give([0, 1, 2])                               # 2 is free: nothing changes
    p.give([0, 1])
    p.give([1, 0, 3])
    assert p.free_pages == 6 and p.take(6) == list(range(6))
    with pytest.raises(binding.FicocoError):
        p.fork([0], 16, 5)                              # no page left for the partly filled one
    with pytest.raises(binding.FicocoError):
        p.give([6])
    with pytest.raises(ValueError):
        p.fork([0], 16, 17)
    p.give(range(6))
    with pytest.raises(binding.FicocoError):
        p.give([2, 2])
    b = p.take(1)
    p.fork(b, 16, 16)
    p.give([b[0], b[0]])                                # a list may hold a page once for each holder
    assert p.free_pages == 6 and sorted(p.take(6)) == list(range(6))
    p.close()
    for args in ((None, 1, None), (None, 0, None)):
        assert lib.ficoco_pool_take(*args) == -1
    assert lib.ficoco_pool_free_pages(None) == -1 and lib.ficoco_pool_destroy(None) == -1


def test_reference_codes_against_torch():
    """Every finite e4m3 value, every midpoint between two of them and random values, rounded like torch's conversion."""
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes.copy()).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.E4M3, want, equal_nan=True)
    fin = np.sort(R.E4M3[np.isfinite(R.E4M3)])
    x = np.concatenate([fin, (fin[1:] + fin[:-1]) / 2, np.random.default_rng(0).uniform(-448, 448, 4000),
                        np.random.default_rng(1).uniform(-0.05, 0.05, 4000)])
    got = R.E4M3[R.to_codes(x)]
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    ok = x == x.astype(np.float32)
    assert np.array_equal(got[ok], want[ok])
    assert R.scale_of(448.0) == 1 and R.scale_of(448.1) == 2 and R.scale_of(0) == 2.0 ** -64


def test_reference_softmax_by_hand():
    rng = np.random.default_rng(0)
    c = R.Cache(rng, [3], 16, 1, 16)
    q = torch.from_numpy(rng.standard_normal((1, 1, 16)))
    k, v, _ = c.tokens(0, 0)
    s = (k * q[0, 0].numpy()).sum(1) / 4
    w = np.exp(s) / np.exp(s).sum()
    out, lse, _, _ = R.attention(c, q, [1])
    assert np.allclose(out[0, 0], (w[:, None] * v).sum(0)) and np.isclose(lse[0, 0], np.log(np.exp(s).sum()))
    got, _ = R.weights(c, q, torch.from_numpy(lse), [1], 1, 1, 4)
    assert np.allclose(got[0, 0, 0], [w[1], w[2], 0, 0])
    out, _, _, _ = R.attention(c, q, [1], window=1, sinks=1)
    w2 = np.exp(s[[0, 2]]) / np.exp(s[[0, 2]]).sum()
    assert np.allclose(out[0, 0], w2 @ v[[0, 2]])
