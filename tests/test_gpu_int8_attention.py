"""Attention over the cache held in 8 bits against its definition in 64 bits.

Tolerance of an element, with W = sum p |v| / sum p, n visible tokens and vmax their largest |v|:
  - half a step of the output's type;
  - the weights are rounded to float16, half a step 2^-11 each: 2^-11 W;
  - the scores' error moves every weight by a factor: products of D terms summed in 32 bits, 2^-24 * (D + 8) * sum |q k| scale, the
    exponent's own rounding 2^-23 |score| at most twice and the exponential's 2^-22; twice that times W, for the weights and their sum;
  - sums over tokens in 32 bits: 2^-24 (n + 16) W at the most, n / 64 of them in turn: 2^-24 (n / 16 + 64) W is enough, as a product
    sums 32 terms and four waves and up to 64 parts are joined;
  - weights below float16's smallest step: 2^-25 each against a sum of at least 2^-1 (the largest is 2^7, or 2^8 less behind the last
    adjustment): n 2^-24 vmax."""
import math

import pytest
import torch

import paper_1901_01965_amd as wg
from tests.test_gpu_int8_cache import batch, random_cache

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def reference(q, cache, table, lengths, starts, scale, causal=True, window=0):
    """(result, tolerance without the type's own rounding), rows of nobody NaN, in 64 bits."""
    rows, heads, dim = q.shape
    group = heads // cache.kv_heads
    out = torch.full(q.shape, float("nan"), dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    for b, length in enumerate(lengths):
        n = starts[b + 1] - starts[b]
        if n == 0:
            continue
        if length == 0:
            out[starts[b]:starts[b + 1]] = 0
            continue
        count = -(-length // cache.block)
        pages = table[b, :count].long()
        good = ((pages >= 0) & (pages < cache.blocks)).repeat_interleave(cache.block)[:length]
        pages = pages.clamp(0, cache.blocks - 1)
        position = length - n + torch.arange(n, device="cuda")[:, None]
        token = torch.arange(length, device="cuda")[None, :]
        seen = (good[None, :] & (position >= 0)).expand(n, length)
        if causal:
            seen = seen & (token <= position)
        if window:
            seen = seen & (token > position - window)
        for h in range(cache.kv_heads):
            k = (cache.k[pages, h].double() * cache.k_scale[pages, h].double()[:, None, None]).reshape(-1, dim)[:length]
            v = (cache.v[pages, h].double() * cache.v_scale[pages, h].double()[:, None, None]).transpose(1, 2).reshape(-1, dim)[:length]
            some = seen.any(0)
            k, v = torch.where(some[:, None], k, 0), torch.where(some[:, None], v, 0)
            for g in range(h * group, (h + 1) * group):
                x = q[starts[b]:starts[b + 1], g].double()
                s = (x @ k.t().contiguous()) * scale
                terms = (x.abs() @ k.abs().t().contiguous()) * abs(scale)
                top = torch.where(seen, s, -math.inf).amax(1, keepdim=True)
                p = torch.where(seen, torch.exp((s - top).clamp(max=0)), 0)
                total = p.sum(1, keepdim=True).clamp(min=1e-300)
                mean, size = (p @ v) / total, (p @ v.abs()) / total
                worst = 2.0 ** -24 * (dim + 8) * torch.where(seen, terms, 0).amax(1, keepdim=True)
                worst = worst + 2 * 2.0 ** -23 * torch.where(seen, s.abs(), 0).amax(1, keepdim=True) + 2.0 ** -22
                out[starts[b]:starts[b + 1], g] = mean
                tol[starts[b]:starts[b + 1], g] = (2.0 ** -11 + 2 * worst + 2.0 ** -24 * (length / 16 + 64)) * size + length * 2.0 ** -24 * v.abs().amax()
    return out, tol


def check(got, want, tol):
    tol = tol + torch.finfo(got.dtype).eps / 2 * want.abs() + torch.finfo(got.dtype).tiny
    # what the type does not hold becomes infinite; next to its largest value either is right
    most = torch.finfo(got.dtype).max
    infinite = got.double() == want.sign() * math.inf
    assert infinite[want.abs() - tol > most].all()
    rest = ~(infinite & (want.abs() + tol > most))
    assert torch.isfinite(got[rest]).all()
    over = ((got.double() - want).abs() / tol)[rest]
    assert over.max().item() <= 1.0, over.max().item()


def queries(rows, heads, dim, dtype, seed=1, size=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, heads, dim, device="cuda", generator=gen) * size).to(dtype)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block,dim", [(16, 64), (32, 128), (64, 128), (64, 256), (128, 64), (128, 128)])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (8, 2), (3, 1), (20, 1)])
def test_single_tokens(heads, kv_heads, block, dim, dtype):
    lengths = [1, 2, 15, 16, 17, 63, 64, 65, 300, 1000, 0]
    blocks = 160
    cache = random_cache(blocks, kv_heads, dim, block, 3)
    table, on_gpu, starts, begins = batch(lengths, [1] * len(lengths), block, blocks, extra=1)
    assert starts is None
    q = queries(len(lengths), heads, dim, dtype)
    got = wg.int8_cache_attention(q, cache, table, on_gpu)
    want, tol = reference(q, cache, table, lengths, begins, 1 / math.sqrt(dim))
    check(got, want, tol)
    assert (got[-1] == 0).all()   # a sequence without tokens


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block,dim", [(16, 128), (64, 64), (64, 128), (128, 256)])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 1), (12, 2), (18, 1)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 70)])
@pytest.mark.parametrize("lengths,news", [([130, 64, 5], [3, 5, 2]), ([200, 1, 333], [200, 1, 150])])
def test_several_rows_per_sequence(lengths, news, causal, window, heads, kv_heads, block, dim, dtype):
    blocks = 60
    cache = random_cache(blocks, kv_heads, dim, block, 6)
    table, on_gpu, starts, begins = batch(lengths, news, block, blocks)
    q = queries(begins[-1], heads, dim, dtype, seed=2)
    got = wg.int8_cache_attention(q, cache, table, on_gpu, starts, scale=0.11, causal=causal, window=window)
    check(got, *reference(q, cache, table, lengths, begins, 0.11, causal, window))


@pytest.mark.parametrize("heads,kv_heads,rows", [(8, 1, 1), (4, 4, 1), (8, 2, 700)])
def test_long_sequences(heads, kv_heads, rows):
    """Long enough to be split into many parts, with one sequence beside it that is not."""
    dim, block, lengths = 128, 64, [20011, 37]
    blocks = 20011 // block + 3
    cache = random_cache(blocks, kv_heads, dim, block, 8)
    table, on_gpu, starts, begins = batch(lengths, [rows, 1], block, blocks)
    q = queries(rows + 1, heads, dim, BF16, seed=4)
    got = wg.int8_cache_attention(q, cache, table, on_gpu, starts)
    check(got, *reference(q, cache, table, lengths, begins, 1 / math.sqrt(dim)))


@pytest.mark.parametrize("dim,block", [(64, 16), (128, 64), (256, 128)])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (12, 2)])
@pytest.mark.parametrize("lengths,news,causal,window", [
    ([752], [127], True, 0), ([3589, 0, 2322], [105, 0, 90], True, 0), ([2000], [300], True, 53), ([2000, 700], [300, 70], True, 700),
    ([1537, 90], [130, 90], False, 0), ([129], [129], True, 0)])
def test_parts_of_sequences_that_many_rows_ask(lengths, news, causal, window, heads, kv_heads, dim, block):
    blocks = sum(-(-n // block) + 1 for n in lengths)
    cache = random_cache(blocks, kv_heads, dim, block, 21)
    table, on_gpu, starts, begins = batch(lengths, news, block, blocks, extra=5)
    q = queries(begins[-1], heads, dim, BF16, seed=5)
    got = wg.int8_cache_attention(q, cache, table, on_gpu, starts, causal=causal, window=window)
    check(got, *reference(q, cache, table, lengths, begins, dim ** -0.5, causal, window))


@pytest.mark.parametrize("rows", [1, 2, 90])
def test_scales_of_unlike_sizes_and_one_far_larger_score(rows):
    """Blocks whose scales differ by 2^20, rise and fall; rows whose weight lies on one token late in the sequence."""
    heads, kv_heads, dim, block, lengths = 4, 2, 64, 16, [700, 300]
    blocks = 80
    cache = random_cache(blocks, kv_heads, dim, block, 12)
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache.v_scale.copy_(2.0 ** torch.randint(-10, 11, (blocks, kv_heads), device="cuda", generator=gen).float())
    cache.v_scale[::5] = 0
    cache.k_scale.copy_(2.0 ** torch.randint(-9, -1, (blocks, kv_heads), device="cuda", generator=gen).float())
    table, on_gpu, starts, begins = batch(lengths, [rows, rows], block, blocks)
    q = queries(2 * rows, heads, dim, F16, seed=5)
    got = wg.int8_cache_attention(q, cache, table, on_gpu, starts, scale=0.3)
    check(got, *reference(q, cache, table, lengths, begins, 0.3))


@pytest.mark.parametrize("rows", [1, 3, 130])
def test_what_lies_in_hidden_places_does_not_matter(rows):
    """Scales that are NaN or infinite in blocks that no row sees, codes behind the length, numbers that name no block in front of
    a window and behind the length."""
    heads, kv_heads, dim, block, length, window = 4, 2, 64, 16, 333, 40
    blocks = 30
    cache = random_cache(blocks, kv_heads, dim, block, 13)
    table, on_gpu, starts, begins = batch([length], [rows], block, blocks, extra=3)
    q = queries(rows, heads, dim, BF16, seed=6)
    want = wg.int8_cache_attention(q, cache, table, on_gpu, starts, window=window)
    check(want, *reference(q, cache, table, [length], begins, 1 / 8, True, window))
    hidden = max(0, length - rows - window + 1) // block   # blocks that lie in front of every window
    for i in range(hidden):
        if i % 3 == 0:
            table[0, i] = (-1, 2 ** 31 - 1, blocks)[i // 3 % 3]
        else:
            cache.k_scale[table[0, i]] = float("nan")
            cache.v_scale[table[0, i]] = float("inf") if i % 2 else float("nan")
    table[0, -3:] = -7
    last = table[0, (length - 1) // block]
    cache.k[last, :, (length - 1) % block + 1:] = -128
    cache.v[last, :, :, (length - 1) % block + 1:] = -128
    assert torch.equal(wg.int8_cache_attention(q, cache, table, on_gpu, starts, window=window), want)


@pytest.mark.parametrize("rows", [1, 4, 70])
def test_blocks_without_a_number_are_not_seen(rows):
    heads, kv_heads, dim, block, length, blocks = 2, 1, 128, 32, 200, 12
    cache = random_cache(blocks, kv_heads, dim, block, 14)
    table, on_gpu, starts, begins = batch([length], [rows], block, blocks)
    table[0, 1], table[0, 4] = -1, blocks
    q = queries(rows, heads, dim, F16, seed=7)
    got = wg.int8_cache_attention(q, cache, table, on_gpu, starts)
    check(got, *reference(q, cache, table, [length], begins, 1 / math.sqrt(dim)))
    table.fill_(-1)
    assert (wg.int8_cache_attention(q, cache, table, on_gpu, starts) == 0).all()


@pytest.mark.parametrize("rows", [5, 200])
def test_rows_in_front_of_the_first_token_are_zero_and_rows_of_nobody_stay(rows):
    heads, kv_heads, dim, block, blocks = 4, 2, 64, 16, 20
    cache = random_cache(blocks, kv_heads, dim, block, 15)
    cuda = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table = torch.arange(20, dtype=torch.int32, device="cuda").reshape(2, 10)
    q = queries(2 * rows + 7, heads, dim, F16, seed=8)
    out = torch.full_like(q, 9.0)
    lengths, starts = [rows - 3 if rows < 100 else 150, 100], [2, 2 + rows, 2 + 2 * rows]
    if rows > 100:
        lengths[1] = 160
    for causal in (True, False):
        out.fill_(9.0)
        wg.int8_cache_attention(q, cache, table, cuda(lengths), cuda(starts), causal=causal, out=out)
        assert (out[:2] == 9).all() and (out[starts[-1]:] == 9).all()
        for b in range(2):
            front = max(0, rows - lengths[b])
            assert (out[starts[b]:starts[b] + front] == 0).all()
        want, tol = reference(q, cache, table, lengths, starts, 1 / 8, causal)
        own = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
        own[2:starts[-1]] = True
        check(out[own], want[own], tol[own])


@pytest.mark.parametrize("rows", [1, 6, 100])
def test_rows_that_lie_apart_and_nan_stays_in_its_row(rows):
    heads, kv_heads, dim, block, length, blocks = 6, 3, 64, 16, 150, 12
    cache = random_cache(blocks, kv_heads, dim, block, 16)
    table, on_gpu, starts, _ = batch([length], [rows], block, blocks)
    wide = queries(rows, heads + 5, dim, BF16, seed=9)
    q = wide[:, 2:2 + heads]
    want = wg.int8_cache_attention(q.contiguous(), cache, table, on_gpu, starts)
    room = torch.full((rows, heads + 1, dim), 3.0, dtype=BF16, device="cuda")
    wg.int8_cache_attention(q, cache, table, on_gpu, starts, out=room[:, :heads])
    assert torch.equal(room[:, :heads], want) and (room[:, heads] == 3).all()
    q = q.contiguous()
    q[rows // 2, 4, 7] = float("nan")
    got = wg.int8_cache_attention(q, cache, table, on_gpu, starts)
    assert torch.isnan(got[rows // 2, 4]).all()
    rest = torch.ones(rows, heads, dtype=torch.bool, device="cuda")
    rest[rows // 2, 4] = False
    assert torch.equal(got[rest], want[rest])


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** 40])
@pytest.mark.parametrize("rows", [1, 80])
def test_bfloat16_queries_beyond_float16(rows, size):
    heads, kv_heads, dim, block, length, blocks = 2, 1, 64, 32, 100, 8
    cache = random_cache(blocks, kv_heads, dim, block, 17)
    table, on_gpu, starts, begins = batch([length], [rows], block, blocks)
    q = queries(rows, heads, dim, BF16, seed=10, size=size)
    got = wg.int8_cache_attention(q, cache, table, on_gpu, starts, scale=0.1 / size)
    check(got, *reference(q, cache, table, [length], begins, 0.1 / size))


@pytest.mark.parametrize("rows", [1, 90])
def test_a_program_that_stores_and_asks_captured_and_replayed(rows):
    """Tokens are stored and asked for in one graph, lengths advanced by the host in between; two graphs in flight share nothing."""
    heads, kv_heads, dim, block, blocks, sequences = 8, 2, 128, 64, 400, 3
    cuda = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table = torch.randperm(blocks, device="cuda")[:390].to(torch.int32).reshape(sequences, 130)
    starts = None if rows == 1 else cuda([0, rows, 2 * rows, 3 * rows])

    def make():
        cache = wg.make_int8_cache(blocks, kv_heads, dim, block)
        k, v, q = (torch.zeros(rows * sequences, n, dim, dtype=BF16, device="cuda") for n in (kv_heads, kv_heads, heads))
        return cache, k, v, q, cuda([rows] * sequences), torch.empty_like(q)

    def step(cache, k, v, q, lengths, out):
        wg.int8_cache_append(k, v, cache, table, lengths, starts)
        wg.int8_cache_attention(q, cache, table, lengths, starts, out=out)

    eager, one, two = make(), make(), make()
    step(*one), step(*two)
    torch.cuda.synchronize()
    graphs = []
    for state in (one, two):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(*state)
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        gen = torch.Generator(device="cuda").manual_seed(turn)
        fresh = [torch.randn(t.shape, device="cuda", generator=gen).to(BF16) for t in eager[1:4]]
        length = rows * (turn + 1) + (2000 if turn > 1 else 0)
        for state in (eager, one, two):
            for t, f in zip(state[1:4], fresh):
                t.copy_(f)
            state[4].fill_(length)
        step(*eager)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert torch.isfinite(eager[5]).all()
        assert torch.equal(one[5], eager[5]) and torch.equal(two[5], eager[5])
        assert torch.equal(one[0].k, eager[0].k) and torch.equal(one[0].v, eager[0].v)


def test_refusals():
    cache = random_cache(8, 2, 64, 16, 1)
    cuda = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table, lengths = cuda([[0, 1], [2, 3]]), cuda([20, 30])
    q = queries(2, 4, 64, F16)
    ask = wg.int8_cache_attention
    for error, call in (
            (ValueError, lambda: ask(queries(3, 4, 64, F16), cache, table, lengths)),                      # rows without starts
            (ValueError, lambda: ask(queries(2, 3, 64, F16), cache, table, lengths)),
            (ValueError, lambda: ask(q, cache, table, cuda([20]))),
            (ValueError, lambda: ask(q, cache, table, lengths, cuda([0, 2]))),
            (TypeError, lambda: ask(q, cache, table.long(), lengths)),
            (TypeError, lambda: ask(q, cache, table.t(), lengths)),
            (ValueError, lambda: ask(q, cache, table, lengths, out=q[:, :2])),
            (ValueError, lambda: ask(q, cache, table, lengths, out=q.bfloat16())),
            (ValueError, lambda: ask(queries(2, 64, 4, F16).transpose(1, 2), cache, table, lengths)),
            (wg.WinogradError, lambda: ask(q, cache, table, lengths, causal=False, window=3)),
            (wg.WinogradError, lambda: ask(q, cache, table, lengths, scale=float("nan"))),
            (RuntimeError, lambda: ask(q.clone().requires_grad_(), cache, table, lengths)),
            (ValueError, lambda: wg.int8_cache_append(q[:, :2], q[:, :2].bfloat16(), cache, table, lengths)),
            (ValueError, lambda: wg.int8_cache_append(q, q, cache, table, lengths)),
            (ValueError, lambda: wg.int8_cache_append(q[:1, :2].expand(2, 2, 64), q[:, :2], cache, table, lengths)),
            (TypeError, lambda: wg.int8_cache_read(cache, table[0].long()))):
        with pytest.raises(error):
            call()
