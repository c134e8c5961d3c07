"""A layer as a program runs it: projections with 4-bit weights, tokens into the 8-bit cache, attention, two more products."""
import pytest
import torch

import paper_1901_01965_amd as wg
from tests import test_gpu_int4_linear as products
from tests import test_gpu_int8_attention as attention
from tests import test_gpu_int8_cache as caches

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
HEADS, KV_HEADS, DIM, BLOCK, BLOCKS, GROUP = 8, 2, 64, 16, 400, 64
WIDTH = HEADS * DIM
SHAPES = {"in": (WIDTH + 2 * KV_HEADS * DIM, WIDTH), "out": (WIDTH, WIDTH), "up": (1500, WIDTH), "down": (WIDTH, 1500)}   # outputs, inputs


def weights(dtype):
    made = {}
    for seed, (name, (N, K)) in enumerate(SHAPES.items()):
        _, codes, scales, zero = products.make(1, N, K, GROUP, dtype, seed % 2 == 0, seed=seed)
        scales = (scales.float() / K ** 0.5).to(dtype)
        made[name] = (wg.pack_int4_weights(codes, scales, zero, GROUP), (codes, scales, zero, GROUP), torch.randn(N, device="cuda") * 0.1)
    return made


def layer(x, w, cache, table, lengths, starts):
    """Every step's result by name; keys, values and queries are slices of one product's."""
    r = {"in": wg.int4_linear(x, w["in"][0], bias=w["in"][2])}
    q, k, v = r["in"].split((WIDTH, KV_HEADS * DIM, KV_HEADS * DIM), 1)
    q, k, v = q.view(-1, HEADS, DIM), k.view(-1, KV_HEADS, DIM), v.view(-1, KV_HEADS, DIM)
    wg.int8_cache_append(k, v, cache, table, lengths, starts)
    r["attention"] = wg.int8_cache_attention(q, cache, table, lengths, starts)
    r["out"] = wg.int4_linear(r["attention"].flatten(1), w["out"][0], bias=w["out"][2])
    r["up"] = wg.int4_linear(r["out"], w["up"][0], bias=w["up"][2], relu=True)
    r["down"] = wg.int4_linear(r["up"], w["down"][0], bias=w["down"][2])
    return r


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_prompts_and_then_tokens_step_by_step(dtype):
    """Each step against its definition in 64 bits of what it was given; the tokens' steps from a graph, against the same made eagerly."""
    w = weights(dtype)
    prompts = [700, 1, 333]
    table, _, _, begins = caches.batch([n + 8 for n in prompts], prompts, BLOCK, BLOCKS)
    cuda = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    cache, mirror = (wg.make_int8_cache(BLOCKS, KV_HEADS, DIM, BLOCK) for _ in range(2))
    x = torch.randn(begins[-1], WIDTH, device="cuda").to(dtype)

    def checked(x, lengths, starts, begins):
        want = caches.copy_of(cache)
        r = layer(x, w, cache, table, cuda(lengths), starts)
        k, v = r["in"][:, WIDTH:].view(-1, 2, KV_HEADS, DIM).unbind(1)
        caches.reference_append(k, v, want, table, lengths, begins)
        assert caches.equal(cache, want)
        q = r["in"][:, :WIDTH].view(-1, HEADS, DIM)
        attention.check(r["attention"], *attention.reference(q, cache, table, lengths, begins, DIM ** -0.5))
        given = {"in": x, "out": r["attention"].flatten(1), "up": r["out"], "down": r["up"]}
        for name, (_, plain, bias) in w.items():
            products.check(r[name], *products.reference(given[name], *plain, bias, name == "up"), dtype, given[name].shape[1], GROUP)
        return r

    checked(x, prompts, cuda(begins), begins)
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(mirror, name).copy_(getattr(cache, name))
    token, lengths = torch.randn(3, WIDTH, device="cuda").to(dtype), cuda(prompts)
    out = torch.empty(3, WIDTH, dtype=dtype, device="cuda")
    step = lambda: out.copy_(layer(token, w, mirror, table, lengths, None)["down"])
    spare = caches.copy_of(mirror)
    step()   # once before the capture; the cache as it was afterwards
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(mirror, name).copy_(getattr(spare, name))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(1, 9):
        token.copy_(torch.randn(3, WIDTH, device="cuda"))
        lengths.add_(1)
        graph.replay()
        r = checked(token, [n + turn for n in prompts], None, [0, 1, 2, 3])
        assert torch.equal(out, r["down"]) and caches.equal(cache, mirror)
