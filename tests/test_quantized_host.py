"""Host side of the quantised operators, without a GPU: the library exports what include/quantized_c.h declares, and every call
that is refused is refused before any launch."""
import ctypes
import os
import re

import pytest
import torch

import paper_1901_01965_amd as wg
from paper_1901_01965_amd import binding, quantized
from tests.test_native_calls_host import NoStorage

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EUNSUPPORTED, ESMALLBUF = 0, -1, -2, -3
F16, BF16, I8, F32 = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1901_01965_amd import build
        build.build()
    return wg.load_quantized()


def test_every_declared_function_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "quantized_c.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(int[48]_\w+)\s*\(", text)))
    assert names == sorted(quantized.EXPORTED_SYMBOLS)
    for n in names:
        assert hasattr(lib, n), n


def test_packed_sizes(lib):
    assert wg.int4_packed_bytes(16, 128, 128) == 256 + 1024 + 256            # header, one tile, 16 scales
    assert wg.int4_packed_bytes(17, 129, 32, True) == 256 + 4 * 1024 + 2 * 8 * 16 * 3
    for bad in ((0, 128, 128), (16, 0, 128), (16, 128, 48), (16, 128, 0), (1 << 27, 1, 32), (1 << 22, 1 << 13, 32)):
        assert wg.int4_packed_bytes(*bad) == 0
    assert wg.int4_packed_bytes(1 << 22, 1 << 12, 128) > 1 << 33


p = ctypes.c_void_p
A, B, C, D, E, G = (p(0x10000 * (i + 1)) for i in range(6))
ODD = p(0x10001)


def test_weights_are_refused_before_any_launch(lib):
    def pack(codes=A, scales=B, scale_type=F16, zeros=None, N=16, K=128, group=64, blob=C, size=1 << 40):
        return lib.int4_pack_weights(codes, scales, scale_type, zeros, N, K, group, blob, size, None)
    assert pack(codes=None) == pack(scales=None) == pack(blob=None) == EINVAL
    assert pack(scale_type=F32) == pack(N=0) == pack(K=-1) == pack(group=16) == pack(scales=ODD) == pack(blob=p(0x30010)) == EINVAL
    assert pack(N=1 << 27) == EUNSUPPORTED
    assert pack(size=wg.int4_packed_bytes(16, 128, 64) - 1) == ESMALLBUF
    assert pack(zeros=D, size=wg.int4_packed_bytes(16, 128, 64)) == ESMALLBUF


def test_products_are_refused_before_any_launch(lib):
    def call(x=A, x_type=F16, stride=128, x_scale=None, blob=B, bias=None, y=C, y_type=F16, M=4, N=16, K=128, group=64, scale_type=F16, relu=0,
             workspace=None, size=0):
        return lib.int4_linear(x, x_type, stride, x_scale, blob, bias, y, y_type, M, N, K, group, scale_type, 0, relu, workspace, size, None)
    assert call(x=None) == call(blob=None) == call(y=None) == EINVAL
    assert call(x_type=F32) == call(x_type=7) == call(y_type=I8) == call(scale_type=I8) == EINVAL
    assert call(stride=127) == call(M=-1) == call(N=0) == call(group=100) == EINVAL
    assert call(x_scale=D) == EINVAL                       # goes with int8
    assert call(x=ODD) == call(y=ODD) == call(y=p(0x30002), y_type=F32) == call(blob=p(0x20080)) == call(bias=p(0x20002)) == EINVAL
    assert call(K=1 << 27, stride=1 << 27) == EUNSUPPORTED
    assert call(M=0, x=None, y=None) == OK
    assert call(M=1 << 24) == call(M=1 << 21, N=1 << 17) == EUNSUPPORTED
    need = lambda **a: lib.int4_linear_workspace_bytes(*dict(dict(x=A, x_type=BF16, stride=128, M=300, N=8192, K=128), **a).values())
    assert need() == 300 * 128 * 2 + 1280                                                      # rows, and 300 factors in whole 256 bytes
    many = dict(M=300, N=8192, x_type=BF16)
    assert call(**many) == call(workspace=p(0x40010), size=1 << 40, **many) == EINVAL
    assert call(workspace=D, size=need() - 1, **many) == ESMALLBUF
    assert need(M=4) == need(N=16) == need(x_type=F16) == need(x_type=F32) == need(M=0) == 0   # few rows; whole, aligned tiles; invalid
    for copied in (dict(K=120), dict(stride=129), dict(x=p(0x10002))):
        assert need(x_type=F16, **copied) > 0
    assert need(x_type=F16, M=100, N=20000, K=2048, stride=2048) == 128 * 2048 * 2             # a tile's rows
    parts, rest = divmod(need(x_type=F16, M=1500, N=203, K=4096, stride=4096), 1500 * 203 * 4)
    assert parts > 1 and rest < 268                                                            # few outputs, long sums
    assert need(M=4, K=120) == 0 and need(M=4, stride=129) == 4 * 128 * 2                      # few rows: pieces, not tiles


def cache_args(**over):
    a = dict(k=A, v=B, ks=C, vs=D, blocks=8, heads=2, dim=64, block=16)
    a.update(over)
    return [a[n] for n in ("k", "v", "ks", "vs", "blocks", "heads", "dim", "block")]


def batch_args(**over):
    a = dict(table=E, width=4, sequences=3, lengths=G, starts=None)
    a.update(over)
    return [a[n] for n in ("table", "width", "sequences", "lengths", "starts")]


BAD_CACHES = [(dict(k=None), EINVAL), (dict(vs=None), EINVAL), (dict(blocks=0), EINVAL), (dict(heads=0), EINVAL), (dict(v=p(0x20008)), EINVAL),
              (dict(dim=96), EUNSUPPORTED), (dict(block=48), EUNSUPPORTED), (dict(heads=1025), EUNSUPPORTED)]
BAD_BATCHES = [(dict(table=None), EINVAL), (dict(lengths=None), EINVAL), (dict(width=0), EINVAL), (dict(sequences=-1), EINVAL),
               (dict(sequences=4), EINVAL), (dict(table=p(0x50002)), EINVAL), (dict(starts=p(0x60002)), EINVAL),
               (dict(width=1 << 27), EUNSUPPORTED)]


def append(lib, cache={}, batch={}, k=A, k_stride=128, v=B, v_stride=128, type=F16, rows=3):
    return lib.int8_cache_append(k, k_stride, v, v_stride, type, rows, *cache_args(**cache), *batch_args(**batch), None)


def attention(lib, cache={}, batch={}, q=A, q_stride=256, type=BF16, rows=3, heads=4, scale=0.1, causal=1, window=0, out=B, out_stride=256,
              workspace=C, size=1 << 40):
    return lib.int8_cache_attention(q, q_stride, type, rows, heads, *cache_args(**cache), *batch_args(**batch), scale, causal, window, out,
                                    out_stride, workspace, size, None)


@pytest.mark.parametrize("call", [append, attention])
def test_caches_and_batches_are_refused_before_any_launch(lib, call):
    for over, status in BAD_CACHES:
        assert call(lib, cache=over) == status, over
    for over, status in BAD_BATCHES:
        assert call(lib, batch=over) == status, over
    assert call(lib, rows=-1) == call(lib, type=F32) == call(lib, type=I8) == EINVAL
    assert call(lib, rows=4) == EINVAL                                      # one row per sequence, or starts
    assert call(lib, rows=0, batch=dict(sequences=0, table=None, lengths=None)) == OK
    assert call(lib, rows=0, batch=dict(starts=D)) == OK


def test_rows_and_sizes_are_refused_before_any_launch(lib):
    assert append(lib, k=None) == append(lib, v=None) == append(lib, k=ODD) == append(lib, k_stride=127) == append(lib, v_stride=0) == EINVAL
    assert attention(lib, q=None) == attention(lib, out=None) == attention(lib, q=ODD) == attention(lib, out=ODD) == EINVAL
    assert attention(lib, q_stride=255) == attention(lib, out_stride=255) == attention(lib, heads=3) == attention(lib, heads=0) == EINVAL
    assert attention(lib, window=-1) == attention(lib, window=5, causal=0) == EINVAL
    assert attention(lib, scale=float("inf")) == attention(lib, scale=float("nan")) == EINVAL
    assert attention(lib, heads=8194, q_stride=1 << 20, out_stride=1 << 20) == EUNSUPPORTED
    wide = dict(lib=lib, rows=1 << 25, heads=1024, q_stride=1 << 16, out_stride=1 << 16, batch=dict(starts=D))
    assert attention(cache=dict(heads=1024), **wide) == EUNSUPPORTED      # more workgroups than a grid's dimension
    long = dict(width=4096)
    need = lib.int8_cache_attention_workspace_bytes(3, 4, 2, 64, 16, 4096, 3, 0)
    assert need > 0
    assert attention(lib, batch=long, workspace=None) == attention(lib, batch=long, workspace=p(0x30080)) == EINVAL
    assert attention(lib, batch=long, size=need - 1) == ESMALLBUF
    assert lib.int8_cache_attention_workspace_bytes(3, 4, 2, 64, 16, 1, 3, 0) == 0
    assert lib.int8_cache_attention_workspace_bytes(3, 5, 2, 64, 16, 4096, 3, 0) == 0
    read = lambda cache={}, ids=E, count=2, k=A, v=B, type=F32: lib.int8_cache_read(*cache_args(**cache), ids, count, k, v, type, None)
    for over, status in BAD_CACHES:
        assert read(over) == status
    assert read(ids=None) == read(count=-1) == read(k=None) == read(v=p(0x20008)) == read(type=I8) == EINVAL
    assert read(count=1 << 24) == EUNSUPPORTED
    assert read(count=0) == OK


# ---- calls through the extension, with tensors that say they are on the GPU and hold nothing ---------------------

def gpu(dtype, *shape):
    return NoStorage(shape, dtype)


def packed(N=32, K=64, group=32, zeros=False, dtype=torch.float16):
    return wg.PackedInt4Weights(gpu(torch.uint8, wg.int4_packed_bytes(N, K, group, zeros)), N, K, group, dtype, zeros)


def cache(blocks=8, heads=2, block=16, dim=64):
    return wg.Int8Cache(gpu(torch.int8, blocks, heads, block, dim), gpu(torch.int8, blocks, heads, dim, block), gpu(torch.float32, blocks, heads),
                        gpu(torch.float32, blocks, heads))


H, I, F = torch.float16, torch.int32, torch.float32


@pytest.mark.parametrize("error,call", [
    (TypeError, lambda: wg.int4_linear(torch.zeros(2, 64, dtype=H), packed())),                    # not on the GPU
    (TypeError, lambda: wg.int4_linear(gpu(F, 2, 64), packed())),
    (TypeError, lambda: wg.int4_linear(gpu(H, 2, 64), gpu(torch.uint8, 100))),
    (ValueError, lambda: wg.int4_linear(gpu(H, 2, 63), packed())),
    (TypeError, lambda: wg.int4_linear(gpu(H, 2, 64), packed(), out_dtype=torch.int8)),
    (RuntimeError, lambda: wg.int4_linear(gpu(H, 2, 64), packed())),                               # no data pointer
    (ValueError, lambda: wg.int4_linear(gpu(H, 2, 0), wg.PackedInt4Weights(gpu(torch.uint8, 0), 32, 0, 32, H, False))),
])
def test_products_through_the_extension_are_refused(lib, error, call):
    with pytest.raises(error):
        call()


def test_weights_through_the_binding_are_refused(lib):
    codes, scales = gpu(torch.uint8, 32, 64), gpu(H, 32, 2)
    for error, args in ((TypeError, (gpu(torch.int8, 32, 64), scales)), (ValueError, (gpu(torch.uint8, 32, 64, 1), scales)),
                        (TypeError, (codes, gpu(F, 32, 2))), (ValueError, (codes, gpu(H, 32, 1))), (ValueError, (codes, scales, gpu(torch.uint8, 32, 1))),
                        (TypeError, (codes, scales, gpu(torch.int8, 32, 2)))):
        with pytest.raises(error):
            wg.pack_int4_weights(*args, group=32)
    with pytest.raises(ValueError):
        wg.pack_int4_weights(codes, scales, group=48)


@pytest.mark.parametrize("error,call", [
    (TypeError, lambda c: wg.int8_cache_attention(gpu(F, 3, 4, 64), c, gpu(I, 3, 4), gpu(I, 3))),
    (ValueError, lambda c: wg.int8_cache_attention(gpu(H, 3, 4, 128), c, gpu(I, 3, 4), gpu(I, 3))),
    (TypeError, lambda c: wg.int8_cache_append(gpu(F, 3, 2, 64), gpu(F, 3, 2, 64), c, gpu(I, 3, 4), gpu(I, 3))),
    (TypeError, lambda c: wg.int8_cache_append(gpu(H, 3, 2, 64), gpu(H, 3, 2, 64), None, gpu(I, 3, 4), gpu(I, 3))),
    (TypeError, lambda c: wg.int8_cache_read(c, gpu(I, 3), torch.int8)),
    (RuntimeError, lambda c: wg.int8_cache_read(c, gpu(I, 3))),
    (RuntimeError, lambda c: wg.int8_cache_attention(gpu(H, 3, 4, 64), c, gpu(I, 3, 4), gpu(I, 3))),
    (RuntimeError, lambda c: wg.int8_cache_append(gpu(H, 3, 2, 64), gpu(H, 3, 2, 64), c, gpu(I, 3, 4), gpu(I, 3))),
])
def test_the_cache_through_the_extension_is_refused(lib, error, call):
    with pytest.raises(error):
        call(cache())


def test_caches_of_other_shapes_are_refused(lib):
    k, v, s = gpu(torch.int8, 8, 2, 16, 64), gpu(torch.int8, 8, 2, 64, 16), gpu(F, 8, 2)
    for error, args in ((ValueError, (k, k, s, s)), (ValueError, (k, v, gpu(F, 8, 1), s)), (TypeError, (k, v, s, gpu(H, 8, 2))),
                        (ValueError, (gpu(torch.int8, 8, 2, 24, 64), gpu(torch.int8, 8, 2, 64, 24), s, s)), (TypeError, (gpu(torch.uint8, 8, 2, 16, 64), v, s, s))):
        with pytest.raises(error):
            wg.Int8Cache(*args)
