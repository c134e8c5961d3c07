"""The cache held in 8 bits: codes and scales bit for bit as their definition in 64 bits gives them."""
import pytest
import torch

import paper_1901_01965_amd as wg

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def random_cache(blocks, heads, dim, block, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    codes = lambda *shape: torch.randint(-127, 128, shape, dtype=torch.int8, device="cuda", generator=gen)
    scale = lambda: torch.rand(blocks, heads, device="cuda", generator=gen) * 0.02 + 0.01
    return wg.Int8Cache(codes(blocks, heads, block, dim), codes(blocks, heads, dim, block), scale(), scale())


def copy_of(cache):
    return wg.Int8Cache(cache.k.clone(), cache.v.clone(), cache.k_scale.clone(), cache.v_scale.clone())


def reference_append(k, v, cache, table, lengths, starts):
    """The definition, block by block, on the CPU in 64 bits; cache is changed."""
    block = cache.block
    table, k, v = table.cpu(), k.cpu(), v.cpu()
    parts = [cache.k.cpu(), cache.v.cpu().transpose(2, 3).contiguous(), cache.k_scale.cpu(), cache.v_scale.cpu()]
    for b, length in enumerate(lengths):
        rows = range(starts[b], starts[b + 1])
        base = length - len(rows)
        for index in range(max(base, 0) // block, -(-length // block) if len(rows) else 0):
            begin, end = max(base, index * block), min(length, (index + 1) * block)
            if index >= table.shape[1] or not 0 <= table[b, index] < cache.blocks:
                continue
            page, lo, hi = int(table[b, index]), begin - index * block, end - index * block
            for new, codes, scales in ((k, parts[0], parts[2]), (v, parts[1], parts[3])):
                top = torch.finfo(new.dtype).max
                x = torch.nan_to_num(new[starts[b] + begin - base:starts[b] + end - base], nan=0.0, posinf=top, neginf=-top).double().transpose(0, 1)
                old = scales[page].double() * (lo > 0)
                scale = torch.maximum(old, (x.abs().amax((1, 2)) / 127.0).float().double())
                by = torch.where(scale > 0, scale, torch.ones_like(scale))[:, None, None]
                codes[page][:, :lo] = torch.round(codes[page][:, :lo].double() * old[:, None, None] / by).to(torch.int8)
                codes[page][:, lo:hi] = torch.round(x / by).clamp(-127, 127).to(torch.int8)
                scales[page] = scale.float()
    cache.k.copy_(parts[0])
    cache.v.copy_(parts[1].transpose(2, 3))
    cache.k_scale.copy_(parts[2])
    cache.v_scale.copy_(parts[3])


def equal(a, b):
    return all(torch.equal(getattr(a, n), getattr(b, n)) for n in ("k", "v", "k_scale", "v_scale"))


def batch(lengths, news, block, blocks, extra=0, seed=0):
    gen = torch.Generator().manual_seed(seed)
    counts = [max(1, -(-n // block)) for n in lengths]
    order = torch.randperm(blocks, generator=gen).tolist()
    table = torch.zeros(len(lengths), max(counts) + extra, dtype=torch.int32)
    for b, count in enumerate(counts):
        for i in range(count):
            table[b, i] = order.pop()
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    cuda = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return table.cuda(), cuda(lengths), (None if all(n == 1 for n in news) else cuda(starts)), starts


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block,dim", [(16, 64), (32, 128), (64, 128), (64, 256), (128, 64), (128, 256)])
@pytest.mark.parametrize("lengths,news", [
    ([1], [1]), ([64, 65, 130, 17], [1, 1, 1, 1]), ([200, 33, 64, 1], [200, 2, 64, 1]), ([129, 7, 300], [3, 0, 171]),
    ([5, 128, 0, 190], [5, 128, 0, 77])])
def test_codes_and_scales_are_those_of_the_definition(lengths, news, block, dim, dtype):
    heads, blocks = 3, 40
    cache = random_cache(blocks, heads, dim, block, 5)
    table, on_gpu, starts, begins = batch(lengths, news, block, blocks)
    gen = torch.Generator(device="cuda").manual_seed(7)
    rows = begins[-1]
    # slices of one tensor, magnitudes around the scales that are there
    both = (torch.randn(rows + 2, 2, heads, dim, device="cuda", generator=gen) * torch.rand(rows + 2, 1, heads, 1, device="cuda", generator=gen)).to(dtype)
    k, v = both[:rows, 0], both[:rows, 1]
    want = copy_of(cache)
    reference_append(k, v, want, table, lengths, begins)
    if starts is not None:   # rows behind the last sequence are not looked at
        both[rows:] = float("inf")
        k, v = both[:, 0], both[:, 1]
    wg.int8_cache_append(k, v, cache, table, on_gpu, starts)
    assert equal(cache, want)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_token_by_token_as_in_one_program(dtype):
    """A sequence that grows by single tokens whose sizes rise: every one may change the block's scale."""
    heads, dim, block = 2, 64, 16
    cache, want = (wg.make_int8_cache(4, heads, dim, block) for _ in range(2))
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(11)
    for length in range(1, 38):
        k, v = ((torch.randn(1, heads, dim, device="cuda", generator=gen) * (1 + 0.3 * (length % 16))).to(dtype) for _ in range(2))
        reference_append(k, v, want, table, [length], [0, 1])
        wg.int8_cache_append(k, v, cache, table, torch.tensor([length], dtype=torch.int32, device="cuda"))
    assert equal(cache, want)


def test_halves_go_to_the_even_code_and_zeros_infinities_and_small_numbers():
    heads, dim, block = 1, 64, 16
    cases = {
        "ties": [127.0] + [i + 0.5 for i in range(-30, 33)],
        "zeros": [0.0] * 64,
        "infinite": [float("inf"), float("-inf"), float("nan")] + [float(i) for i in range(61)],
        "small": [2.0 ** -24 * (i % 5) for i in range(64)],
    }
    for dtype in (F16, BF16):
        for name, row in cases.items():
            x = torch.tensor(row, device="cuda").to(dtype).reshape(1, heads, dim)
            if name == "small" and dtype == BF16:
                x = (torch.arange(64, device="cuda") * 2.0 ** -133).to(dtype).reshape(1, heads, dim)
            cache, want = (random_cache(1, heads, dim, block, 3) for _ in range(2))
            table, length = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
            reference_append(x, x, want, table, [1], [0, 1])
            wg.int8_cache_append(x, x, cache, table, length)
            assert equal(cache, want), (name, dtype)


def test_old_codes_at_halves_go_to_the_even_code():
    """The scale doubles, and grows sixfold: c / 2 and c / 6 hit halves exactly."""
    heads, dim, block = 1, 64, 16
    for grow in (2.0, 6.0):
        cache = wg.make_int8_cache(1, heads, dim, block)
        cache.k[0, 0, 0] = torch.arange(-32, 32, dtype=torch.int8)
        cache.v[0, 0, :, 0] = torch.arange(-32, 32, dtype=torch.int8)
        cache.k_scale.fill_(1.0)
        cache.v_scale.fill_(1.0)
        want = copy_of(cache)
        x = torch.zeros(1, heads, dim, dtype=F16, device="cuda")
        x[0, 0, 3] = 127.0 * grow
        table, length = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.full((1,), 2, dtype=torch.int32, device="cuda")
        reference_append(x, x, want, table, [2], [0, 1])
        wg.int8_cache_append(x, x, cache, table, length)
        assert equal(cache, want)
        assert cache.k[0, 0, 0, 0].item() == round(-32 / grow)


def test_numbers_that_name_no_block_and_lengths_beyond_the_table_are_skipped():
    heads, dim, block, blocks = 2, 64, 16, 6
    cache = random_cache(blocks, heads, dim, block, 9)
    want = copy_of(cache)
    table = torch.tensor([[1, -1, 3], [6, 4, 2147483647]], dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn(96, heads, dim, device="cuda", generator=gen).to(F16) for _ in range(2))
    lengths, starts = [48, 48], [0, 48, 96]
    reference_append(k, v, want, table, lengths, starts)
    cuda = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    wg.int8_cache_append(k, v, cache, table, cuda(lengths), cuda(starts))
    assert equal(cache, want)
    # a length beyond the table counts as the table's; starts beyond the rows as the rows
    before = copy_of(cache)
    wg.int8_cache_append(k[:1], v[:1], cache, table[:1, :1], cuda([-5]))
    wg.int8_cache_append(k[:0], v[:0], cache, table[:1, :1], cuda([1]), cuda([0, 0]))
    assert equal(cache, before)
    wg.int8_cache_append(k[:16], v[:16], cache, table[:1, :1], cuda([1000]), cuda([-3, 400]))
    reference_append(k[:16], v[:16], before, table[:1, :1], [16], [0, 16])
    assert equal(cache, before)


@pytest.mark.parametrize("block,dim", [(16, 64), (64, 128), (128, 256), (32, 256)])
@pytest.mark.parametrize("dtype", [torch.float32, F16, BF16])
def test_blocks_read_back_as_values(block, dim, dtype):
    heads, blocks = 3, 7
    cache = random_cache(blocks, heads, dim, block, 4)
    ids = torch.tensor([5, 0, -1, 5, 7, 2], dtype=torch.int32, device="cuda")
    k, v = wg.int8_cache_read(cache, ids, dtype)
    there = torch.tensor([1.0, 1, 0, 1, 0, 1], device="cuda")[:, None, None, None]
    at = ids.long().clamp(0, blocks - 1) % blocks
    want_k = cache.k[at].float() * cache.k_scale[at][:, :, None, None] * there
    want_v = (cache.v[at].float() * cache.v_scale[at][:, :, None, None] * there).transpose(2, 3)
    assert torch.equal(k, want_k.to(dtype)) and torch.equal(v, want_v.to(dtype))
    assert wg.int8_cache_read(cache, ids[:0], dtype)[0].shape == (0, heads, block, dim)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("block,dim", [(16, 64), (128, 128), (128, 256)])
@pytest.mark.parametrize("news", [1, 5])
def test_special_numbers_in_blocks_of_every_size(news, block, dim, dtype):
    """Each head holds another kind of numbers, in one token of a block whose older tokens stay."""
    heads, length = 5, block // 2 + 5
    x = torch.randn(news, heads, dim, generator=torch.Generator().manual_seed(4))
    x[-1, 0] = torch.cat((torch.tensor([127.0]), torch.arange(dim - 1) % 100 - 50.5))   # halves
    x[:, 1] = 0
    x[-1, 2, :3] = torch.tensor([float("inf"), float("-inf"), float("nan")])
    x[:, 3] *= 2.0 ** -24 if dtype == F16 else 2.0 ** -130
    x[-1, 4] = float("nan")
    x = x.to(dtype).cuda()
    cache = random_cache(2, heads, dim, block, 3)
    cache.k_scale[:, 3] = cache.v_scale[:, 3] = 2.0 ** -140
    cache.v_scale[:, 0] = 1.0
    want, table = copy_of(cache), torch.ones(1, 1, dtype=torch.int32, device="cuda")
    reference_append(x, x, want, table, [length], [0, news])
    cuda = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    wg.int8_cache_append(x, x, cache, table, cuda([length]), cuda([0, news]) if news > 1 else None)
    assert equal(cache, want)


def test_more_sequences_than_a_wave_has_lanes():
    heads, dim, block, sequences = 1, 64, 16, 200
    gen = torch.Generator().manual_seed(8)
    news = torch.randint(0, 5, (sequences,), generator=gen).tolist()
    lengths = [n + int(torch.randint(0, 30, (1,), generator=gen)) for n in news]
    table, on_gpu, starts, begins = batch(lengths, news, block, 600)
    cache = random_cache(600, heads, dim, block, 6)
    want = copy_of(cache)
    k, v = torch.randn(2, begins[-1], heads, dim, generator=gen).to(F16).cuda()
    reference_append(k, v, want, table, lengths, begins)
    wg.int8_cache_append(k, v, cache, table, on_gpu, starts)
    assert equal(cache, want)
