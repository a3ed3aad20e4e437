"""Refusals of the 8-bit cache's calls, without a GPU: tensors that lie on another device than the cache, pointers that a kernel
could not follow."""
import types

import pytest
import torch

from paper_2411_17686_b200 import binding, build
from tests import test_cache_cpu as A

GPU, OTHER, CPU = torch.device("cuda", 0), torch.device("cuda", 1), torch.device("cpu")


class Shown:
    """What the binding looks at in a tensor, on a device that need not exist."""

    def __init__(self, shape, dtype, device=GPU):
        self.shape, self.dtype, self.device, self.is_cuda = torch.Size(shape), dtype, device, device.type == "cuda"

    def stride(self, d=None):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s) if d is None else s[d]

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000


class Reached(Exception):
    pass


class Library:
    def __getattr__(self, name):
        def call(*args):
            raise Reached(name)
        return call


@pytest.fixture
def ctx():
    c = binding.Context.__new__(binding.Context)
    c.device, c.h, c.lib = 0, None, Library()
    return c


BATCH, ROWS, HEADS, KV, DIM, TEXT, COUNT = 3, 5, 4, 2, 128, 2, 7
I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16


def tensors(**over):
    shapes = dict(q=((ROWS, HEADS, DIM), BF16), out=((ROWS, HEADS, DIM), BF16), lse=((ROWS, HEADS), F32), k=((ROWS, KV, DIM), BF16),
                  v=((ROWS, KV, DIM), BF16), cu=((BATCH + 1,), I32), weights=((BATCH, HEADS, TEXT, COUNT), F32), src=((6,), I32),
                  dst=((6,), I32), to=((BATCH, 4), I32), kept=((9,), I32), lengths=((BATCH,), I32))
    return types.SimpleNamespace(**{n: Shown(s, t, over.get(n, GPU)) for n, (s, t) in shapes.items()})


def cache():
    s = binding.ficoco_cache(*([0x10000] * 6), 8, 10, 64, KV, DIM, BATCH, 8)
    return types.SimpleNamespace(struct=s, device=GPU, scale=DIM ** -0.5)


CALLS = {
    "append": (lambda c, t: c.ficoco_cache_append(cache(), t.k, t.v, t.cu, stream=0), ("k", "v", "cu")),
    "attention": (lambda c, t: c.ficoco_cache_attention(cache(), t.q, t.cu, out=t.out, lse=t.lse, stream=0), ("q", "cu", "out", "lse")),
    "weights": (lambda c, t: c.ficoco_cache_weights(cache(), t.q, t.lse, t.cu, TEXT, 0, COUNT, out=t.weights, stream=0),
                ("q", "lse", "cu", "weights")),
    "copy": (lambda c, t: c.ficoco_cache_copy(cache(), t.src, t.dst, stream=0), ("src", "dst")),
    "compact": (lambda c, t: c.ficoco_cache_compact(cache(), t.to, t.kept, t.cu, lengths=t.lengths, stream=0),
                ("to", "kept", "cu", "lengths")),
}


@pytest.mark.parametrize("device", [CPU, OTHER], ids=str)
@pytest.mark.parametrize("call,name", [(c, n) for c, (_, names) in CALLS.items() for n in names])
def test_tensors_on_another_device_are_refused(ctx, call, name, device):
    run = CALLS[call][0]
    with pytest.raises(Reached):                         # with everything in place the library is called
        run(ctx, tensors())
    with pytest.raises(ValueError):
        run(ctx, tensors(**{name: device}))


def test_numbers_that_no_c_int_holds_are_refused(ctx):
    """Their low 32 bits would be a window of 5, token 0, ..."""
    t = tensors()
    for over in (dict(window=(1 << 32) + 5), dict(window=1 << 31), dict(window=8, sinks=(1 << 32) + 1), dict(sinks=-(1 << 33))):
        with pytest.raises(ValueError):
            ctx.ficoco_cache_attention(cache(), t.q, t.cu, out=t.out, lse=t.lse, stream=0, **over)
        with pytest.raises(ValueError):
            ctx.ficoco_cache_weights(cache(), t.q, t.lse, t.cu, TEXT, 0, COUNT, out=t.weights, stream=0, **over)
    with pytest.raises(ValueError):
        ctx.ficoco_cache_weights(cache(), t.q, t.lse, t.cu, TEXT, 1 << 32, COUNT, out=t.weights, stream=0)
    with pytest.raises(ValueError):
        ctx.ficoco_cache_compact(cache(), t.to, t.kept, t.cu, first=1 << 32, lengths=t.lengths, stream=0)
    with pytest.raises(Reached):
        ctx.ficoco_cache_attention(cache(), t.q, t.cu, out=t.out, lse=t.lse, stream=0, window=(1 << 31) - 1, sinks=(1 << 31) - 1)


# ---- the C entry points, with a context that none may touch (tests/test_cache_cpu.py) ---------------------------------------------
P = A.P16


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


@pytest.mark.parametrize("by", [1, 2, 3])
def test_misaligned_pointers_are_refused(lib, by):
    for name, at in (("k_scale", 3), ("v_scale", 4), ("page_table", 5), ("lengths", 6)):
        c = A.cache(**{name: P * at + by})
        assert lib.ficoco_cache_append(A.FAKE, c, A.append(), None) == -1, name
        assert lib.ficoco_cache_attention(A.FAKE, c, A.attention(), None) == -1, name
        assert lib.ficoco_cache_weights(A.FAKE, c, A.attention(), 2, 0, 3, P * 4000, None) == -1, name
        assert lib.ficoco_cache_copy(A.FAKE, c, P * 15, P * 16, 3, None) == -1, name
        assert lib.ficoco_cache_compact(A.FAKE, c, A.compact(), None) == -1, name
    c = A.cache()
    for name, at in (("cu_rows", 8), ("lse", 3000)):
        a = A.attention(**{name: P * at + by})
        assert lib.ficoco_cache_attention(A.FAKE, c, a, None) == -1, name
        assert lib.ficoco_cache_weights(A.FAKE, c, a, 2, 0, 3, P * 4000, None) == -1, name
    assert lib.ficoco_cache_append(A.FAKE, c, A.append(cu_rows=P * 8 + by), None) == -1
    assert lib.ficoco_cache_copy(A.FAKE, c, P * 15 + by, P * 16, 3, None) == -1
    assert lib.ficoco_cache_copy(A.FAKE, c, P * 15, P * 16 + by, 3, None) == -1
    for name, at in (("to_table", 11), ("kept", 12), ("cu_kept", 13), ("lengths_out", 14)):
        assert lib.ficoco_cache_compact(A.FAKE, c, A.compact(**{name: P * at + by}), None) == -1, name


def test_outputs_that_overlap_inputs_are_refused(lib):
    """The library's general rule.  Sizes of tests/test_cache_cpu.py's calls: 10 pages of 2 heads x 64 tokens x 128, 3 sequences, 5 rows."""
    wide = dict(k_codes=P * 100, v_codes=P * 200, k_scale=P * 300, v_scale=P * 400, page_table=P * 500, lengths=P * 600)
    c, codes = A.cache(**wide), 10 * 2 * 64 * 128
    inputs = [P * 100, P * 100 + codes - 16, P * 300, P * 300 + 76, P * 500, P * 500 + 92, P * 600 + 8, P * 8, P * 8 + 12]
    for at in inputs + [P * 200 + 1024, P * 400 + 4]:
        assert lib.ficoco_cache_attention(A.FAKE, c, A.attention(lse=at), None) == -1, hex(at)
        if at % 16 == 0:
            assert lib.ficoco_cache_attention(A.FAKE, c, A.attention(out=at), None) == -1, hex(at)
    size = 3 * 4 * 2 * 3 * 4                             # bytes of the weights
    for at in inputs + [P * 1000, P * 1000 + (4 * 512 + 512) * 2 - 4, P * 3000, P * 3000 + 76, P * 3000 - size + 4]:
        assert lib.ficoco_cache_weights(A.FAKE, c, A.attention(), 2, 0, 3, at, None) == -1, hex(at)
    for at in (P * 100, P * 200 + codes - 16, P * 300, P * 400 + 64):
        assert lib.ficoco_cache_append(A.FAKE, c, A.append(k=at), None) == -1, hex(at)
        assert lib.ficoco_cache_append(A.FAKE, c, A.append(v=at), None) == -1, hex(at)
        assert lib.ficoco_cache_append(A.FAKE, c, A.append(cu_rows=at), None) == -1, hex(at)
        assert lib.ficoco_cache_copy(A.FAKE, c, at, P * 2, 3, None) == -1, hex(at)
        assert lib.ficoco_cache_copy(A.FAKE, c, P * 2, at, 3, None) == -1, hex(at)
        for name in ("to_table", "kept", "cu_kept", "lengths_out"):
            assert lib.ficoco_cache_compact(A.FAKE, c, A.compact(**{name: at}), None) == -1, (name, hex(at))
    for at in (P * 11, P * 11 + 44, P * 12 + 32, P * 13 + 12, P * 13 - 8, P * 500 + 92, P * 600 + 8):
        assert lib.ficoco_cache_compact(A.FAKE, c, A.compact(lengths_out=at), None) == -1, hex(at)
