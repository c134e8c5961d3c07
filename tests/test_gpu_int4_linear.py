"""Products with 4-bit weights against their definition in 64 bits.

Tolerance of an element: half a step of the output's type, and what 32-bit sums lose.  Within a group of 128 inputs (or fewer)
partial sums are at most sum |x| (31/16 + 31/16) in the operands' units of scale * 16, and at most 128 products and four joins of
them are rounded, 2^-24 each: 132 * 62 * 2^-24 * sum |x| scale over all groups.  Sums over groups, waves, scale and bias add as many
roundings of at most the whole magnitude.  int8 sums are exact within a group."""
import pytest
import torch

import paper_1901_01965_amd as wg

pytestmark = pytest.mark.gpu

F16, BF16, I8, F32 = torch.float16, torch.bfloat16, torch.int8, torch.float32


def make(M, N, K, group, dtype, zeros, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    groups = -(-K // group)
    codes = torch.randint(0, 16, (N, K), dtype=torch.uint8, device="cuda", generator=gen)
    scales = (torch.rand(N, groups, device="cuda", generator=gen) * 0.1 + 0.01).to(F16 if dtype == I8 else dtype)
    zero = torch.randint(0, 16, (N, groups), dtype=torch.uint8, device="cuda", generator=gen) if zeros else None
    if dtype == I8:
        x = torch.randint(-128, 128, (M, K), dtype=torch.int16, device="cuda", generator=gen).to(I8)
    else:
        x = torch.randn(M, K, device="cuda", generator=gen).to(dtype)
    return x, codes, scales, zero


def reference(x, codes, scales, zero, group, bias=None, relu=False, x_scale=None):
    """(result, magnitude that the tolerance counts) in 64 bits."""
    K = codes.shape[1]
    wide = lambda t: t.double().repeat_interleave(group, 1)[:, :K]
    s = wide(scales)
    w = (codes.double() - (8.0 if zero is None else wide(zero))) * s
    y = x.double() @ w.t()
    size = (x.double().abs() @ s.t()) * 62
    if x_scale is not None:
        y, size = y * x_scale.double()[:, None], size * x_scale.double()[:, None]
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    return (y.clamp(min=0) if relu else y), size


def check(got, want, size, dtype, K, group):
    groups = -(-K // group)
    inner = 0 if dtype == I8 else 132
    tol = torch.finfo(got.dtype).eps / 2 * want.abs() + 2.0 ** -24 * (inner + groups + 16) * size
    tol = tol + torch.finfo(got.dtype).tiny
    over = (got.double() - want).abs() / tol
    assert torch.isfinite(got).all()
    assert over.max().item() <= 1.0, over.max().item()


@pytest.mark.parametrize("dtype", [F16, BF16, I8])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (128, False)])
@pytest.mark.parametrize("M,N,K", [(1, 16, 128), (1, 1, 1), (2, 17, 33), (16, 64, 256), (17, 40, 1000), (5, 129, 2049), (64, 48, 384),
                                   (70, 33, 136), (131, 257, 640), (1000, 17, 96)])
def test_every_size_against_64_bits(M, N, K, group, zeros, dtype):
    x, codes, scales, zero = make(M, N, K, group, dtype, zeros)
    packed = wg.pack_int4_weights(codes, scales, zero, group)
    got = wg.int4_linear(x, packed)
    assert got.dtype == (F32 if dtype == I8 else dtype) and got.shape == (M, N)
    check(got, *reference(x, codes, scales, zero, group), dtype, K, group)


@pytest.mark.parametrize("dtype", [F16, BF16, I8])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("N,K", [(4099, 2200), (9000, 1290), (16900, 650)])
@pytest.mark.parametrize("M", [1, 4, 5, 16, 31, 70])
def test_few_rows_of_many_outputs(M, N, K, group, zeros, dtype):
    """More tiles of outputs than compute units: a workgroup takes several, of fewer waves; the last ones end inside both."""
    x, codes, scales, zero = make(M, N, K, group, dtype, zeros, seed=14)
    got = wg.int4_linear(x, wg.pack_int4_weights(codes, scales, zero, group))
    check(got, *reference(x, codes, scales, zero, group), dtype, K, group)


@pytest.mark.parametrize("dtype", [F16, BF16, I8])
@pytest.mark.parametrize("group,zeros", [(32, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("M,N,K", [(1101, 8200, 384), (131, 11001, 1100), (100, 20001, 2000), (300, 5003, 1000)])
def test_enough_rows_and_outputs_for_tiles(M, N, K, group, zeros, dtype):
    """The first is large enough for the coarser tiles, the others end inside tiles of rows, outputs and inputs."""
    x, codes, scales, zero = make(M, N, K, group, dtype, zeros, seed=2)
    got = wg.int4_linear(x, wg.pack_int4_weights(codes, scales, zero, group))
    check(got, *reference(x, codes, scales, zero, group), dtype, K, group)


@pytest.mark.parametrize("dtype", [F16, BF16, I8])
@pytest.mark.parametrize("group,zeros", [(32, False), (64, True), (128, True)])
@pytest.mark.parametrize("M,N,K", [(1500, 203, 4096), (1300, 260, 3001)])
@pytest.mark.parametrize("out_dtype", [F16, F32])
def test_long_sums_of_few_outputs_in_parts(out_dtype, M, N, K, group, zeros, dtype):
    x, codes, scales, zero = make(M, N, K, group, dtype, zeros, seed=12)
    bias = torch.randn(N, device="cuda") * 3
    x_scale = torch.rand(M, device="cuda") + 0.1 if dtype == I8 else None
    packed = wg.pack_int4_weights(codes, scales, zero, group)
    got = wg.int4_linear(x, packed, bias=bias, relu=True, x_scale=x_scale, out_dtype=out_dtype)
    check(got, *reference(x, codes, scales, zero, group, bias, True, x_scale), dtype, K, group)
    other = wg.PackedInt4Weights(packed.blob, N, K, group, BF16 if packed.scale_dtype == F16 else F16, zeros)
    out = torch.full((M, N), 5.0, dtype=out_dtype, device="cuda")
    wg.int4_linear(x, other, x_scale=x_scale, out=out, out_dtype=out_dtype)
    assert (out == 5).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_many_rows_beside_each_other_and_of_unlike_sizes(dtype):
    """bfloat16 rows are held as float16 with a power of two each: rows of any size, an infinite and a NaN row, strided rows."""
    M, N, K, group = 300, 5120, 512, 64
    x, codes, scales, zero = make(M, N, K, group, dtype, True, seed=9)
    if dtype == BF16:
        x = (x.float() * 2.0 ** torch.randint(-60, 60, (M, 1), device="cuda")).to(BF16)
        x[5] = 0
    packed = wg.pack_int4_weights(codes, scales, zero, group)
    clean = wg.int4_linear(x, packed, out_dtype=F32)
    check(clean, *reference(x, codes, scales, zero, group), dtype, K, group)
    wide = torch.full((M, K + 8), float("nan"), dtype=dtype, device="cuda")
    wide[:, :K] = x
    wide[7, 5], wide[200, 0] = float("nan"), float("inf")
    got = wg.int4_linear(wide[:, :K], packed, out_dtype=F32)
    rest = [m for m in range(M) if m not in (7, 200)]
    assert torch.equal(got[rest], clean[rest])
    assert torch.isnan(got[7]).all() and not torch.isfinite(got[200]).any()


@pytest.mark.parametrize("dtype", [F16, BF16, I8])
@pytest.mark.parametrize("out_dtype", [F16, BF16, F32])
@pytest.mark.parametrize("M", [3, 40, 200])
def test_bias_relu_scales_of_rows_and_types_of_the_result(M, out_dtype, dtype):
    N, K, group = 100, 320, 64
    x, codes, scales, zero = make(M, N, K, group, dtype, True, seed=3)
    bias = torch.randn(N, device="cuda") * 3
    x_scale = torch.rand(M, device="cuda") + 0.1 if dtype == I8 else None
    packed = wg.pack_int4_weights(codes, scales, zero, group)
    out = torch.full((M, N), -7.0, dtype=out_dtype, device="cuda")
    got = wg.int4_linear(x, packed, bias=bias, relu=True, x_scale=x_scale, out_dtype=out_dtype, out=out)
    assert got.data_ptr() == out.data_ptr()
    check(got, *reference(x, codes, scales, zero, group, bias, True, x_scale), dtype, K, group)


@pytest.mark.parametrize("dtype", [F16, BF16, I8])
@pytest.mark.parametrize("M", [1, 9, 90])
def test_rows_that_lie_apart_and_off_boundaries(M, dtype):
    N, K, group = 50, 200, 32
    x, codes, scales, zero = make(M, N, K, group, dtype, False, seed=4)
    packed = wg.pack_int4_weights(codes, scales, zero, group)
    wide = torch.full((M, K + 37), 100.0, device="cuda").to(dtype)
    wide[:, 3:3 + K] = x
    # what lies beside the rows must not be looked at
    if dtype != I8:
        wide[:, :3], wide[:, 3 + K:] = float("nan"), float("inf")
    assert torch.equal(wg.int4_linear(wide[:, 3:3 + K], packed), wg.int4_linear(x, packed))
    assert torch.equal(wg.int4_linear(x.reshape(1, M, K), packed), wg.int4_linear(x, packed)[None])
    assert torch.equal(wg.int4_linear(x[0], packed), wg.int4_linear(x[:1], packed)[0])


def test_results_do_not_depend_on_the_rows_beside_and_nan_stays_in_its_row():
    x, codes, scales, zero = make(40, 70, 512, 128, F16, False, seed=5)
    packed = wg.pack_int4_weights(codes, scales, zero, 128)
    clean = wg.int4_linear(x, packed)
    bad = x.clone()
    bad[7, 5], bad[20, 0] = float("nan"), float("inf")
    got = wg.int4_linear(bad, packed)
    rows = [m for m in range(40) if m not in (7, 20)]
    assert torch.equal(got[rows], clean[rows])
    assert torch.isnan(got[7]).all() and torch.isnan(got[20]).all()


@pytest.mark.parametrize("M", [1, 16, 64, 300])
def test_extremes_of_codes_zero_points_and_int8(M):
    """All products at their largest: int32 sums of a group stay exact, 32-bit sums within the tolerance."""
    N, K, group = 32, 4096, 128
    x = torch.full((M, K), -128, dtype=I8, device="cuda")
    codes = torch.full((N, K), 15, dtype=torch.uint8, device="cuda")
    codes[1::2] = 0
    zero = torch.zeros((N, K // group), dtype=torch.uint8, device="cuda")
    zero[1::2] = 15
    scales = torch.full((N, K // group), 0.5, dtype=F16, device="cuda")
    got = wg.int4_linear(x, wg.pack_int4_weights(codes, scales, zero, group))
    want, _ = reference(x, codes, scales, zero, group)
    assert torch.equal(got.double(), want)   # multiples of a half below 2^24


def test_nothing_is_written_beside_the_result():
    x, codes, scales, zero = make(3, 19, 64, 32, BF16, True, seed=6)
    packed = wg.pack_int4_weights(codes, scales, zero, 32)
    room = torch.full((5, 19), 42.0, dtype=BF16, device="cuda")
    wg.int4_linear(x, packed, out=room[1:4])
    assert (room[0] == 42).all() and (room[4] == 42).all()
    assert torch.equal(room[1:4], wg.int4_linear(x, packed))


def test_no_rows():
    _, codes, scales, zero = make(1, 19, 64, 32, BF16, True)
    packed = wg.pack_int4_weights(codes, scales, zero, 32)
    assert wg.int4_linear(torch.empty((0, 64), dtype=BF16, device="cuda"), packed).shape == (0, 19)


def test_a_blob_of_other_weights_leaves_the_result_untouched():
    x, codes, scales, zero = make(3, 32, 64, 32, F16, False)
    packed = wg.pack_int4_weights(codes, scales, None, 32)
    other = wg.PackedInt4Weights(packed.blob, 32, 64, 32, BF16, False)
    out = torch.full((3, 32), 5.0, dtype=F16, device="cuda")
    wg.int4_linear(x, other, out=out)
    assert (out == 5).all()


@pytest.mark.parametrize("M", [1, 33, 150])
def test_captured_and_replayed_on_another_stream(M):
    x, codes, scales, zero = make(M, 96, 256, 64, F16, True, seed=8)
    packed = wg.pack_int4_weights(codes, scales, zero, 64)
    out = torch.empty((M, 96), dtype=F16, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        wg.int4_linear(x, packed, out=out)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wg.int4_linear(x, packed, out=out)
    for seed in (9, 10, 11):
        x.copy_(make(M, 96, 256, 64, F16, True, seed=seed)[0])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, wg.int4_linear(x, packed))


def test_captured_many_rows_that_are_copied_and_summed_in_parts():
    M, N, K = 1300, 250, 3000
    x, codes, scales, zero = make(M, N, K, 128, BF16, True, seed=8)
    packed = wg.pack_int4_weights(codes, scales, zero, 128)
    out, again = (torch.empty((M, N), dtype=BF16, device="cuda") for _ in range(2))
    wg.int4_linear(x, packed, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wg.int4_linear(x, packed, out=out)
        wg.int4_linear(x, packed, out=again)
    for seed in (9, 10, 11):
        x.copy_(make(M, N, K, 128, BF16, True, seed=seed)[0])
        out.zero_()
        graph.replay()
        want = wg.int4_linear(x, packed)
        assert torch.equal(out, want) and torch.equal(again, want)


def test_refusals():
    x, codes, scales, zero = make(4, 32, 64, 32, F16, False)
    packed = wg.pack_int4_weights(codes, scales, None, 32)
    f = torch.float32
    for error, call in (
            (ValueError, lambda: wg.int4_linear(x[:, :32], packed)),
            (ValueError, lambda: wg.int4_linear(x[:1].expand(4, 64), packed)),             # rows that overlap
            (ValueError, lambda: wg.int4_linear(x.t().contiguous().t(), packed)),
            (TypeError, lambda: wg.int4_linear(x, packed, bias=torch.zeros(32, dtype=F16, device="cuda"))),
            (ValueError, lambda: wg.int4_linear(x, packed, bias=torch.zeros(31, device="cuda"))),
            (TypeError, lambda: wg.int4_linear(x, packed, x_scale=torch.ones(4, device="cuda"))),
            (ValueError, lambda: wg.int4_linear(x.to(I8), packed, x_scale=torch.ones(3, device="cuda"))),
            (TypeError, lambda: wg.int4_linear(x, packed, out=torch.zeros(4, 32, dtype=f, device="cuda"))),
            (ValueError, lambda: wg.int4_linear(x, packed, out=torch.zeros(4, 33, dtype=F16, device="cuda"))),
            (ValueError, lambda: wg.int4_linear(x, wg.PackedInt4Weights(packed.blob, 33, 64, 32, F16, False))),
            (RuntimeError, lambda: wg.int4_linear(x.clone().requires_grad_(), packed))):
        with pytest.raises(error):
            call()
    with torch.no_grad():
        assert torch.equal(wg.int4_linear(x.clone().requires_grad_(), packed), wg.int4_linear(x, packed))
