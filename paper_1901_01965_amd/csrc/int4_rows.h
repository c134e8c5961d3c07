// y = x W^T with 4-bit weights for few rows: the weights' bytes are read once, everything else stays beside them.
//
// A workgroup takes 16 NT outputs and 16 MT rows; its waves share the inputs out by tiles of 128 and add their sums up in LDS at the
// end, in the order of the waves.  The matrix cores multiply (rows beyond the last are copies of it and are not stored): a word of
// eight codes costs seven vector instructions as float16 and three as int8 (int4_weights.h), the sum over a group of sum_k x_k that
// takes the zero points off is one more product, whose other operand is constant, and becomes the accumulator that the codes'
// products start from.
#pragma once
#include "int4_weights.h"

namespace wq {

namespace {

constexpr int kMostWaves = 8;

template <int XT, int GROUP, bool ZEROS, bool BF16, int MT, int NT, int AHEAD>
__global__ __launch_bounds__(64 * kMostWaves) void int4_rows_kernel(const typename Element<XT>::type* x, long long x_stride, Int4Weights w, Int4Output o) {
    typedef Products<XT> P;
    typedef std::conditional_t<XT == WQ_I8, v2u, v4u> Bits;
    constexpr int kGroups = kTileInputs / GROUP, kSteps = GROUP / 32;   // groups in a tile, products in a group
    __shared__ v4f sums[kMostWaves][NT * MT][64];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int tile0 = blockIdx.x * NT, m0 = blockIdx.y * (16 * MT);
    const bool fits = matches(w);

    const typename Element<XT>::type* row[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) row[mt] = x + (long long)min(m0 + 16 * mt + (lane & 15), o.M - 1) * x_stride;
    const v4u* codes[NT];
    size_t scale_at[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const size_t tile = min(tile0 + nt, w.output_tiles - 1);
        codes[nt] = reinterpret_cast<const v4u*>(w.codes + tile * w.input_tiles * kTileBytes) + lane;
        scale_at[nt] = tile * w.groups * kTileOutputs + 4 * (lane >> 4);
    }

    // what a tile of inputs needs, on its way while earlier ones are multiplied
    struct Stage {
        v4u words[NT];
        v2u scales[NT][kGroups];
        uint32_t zeros[NT][kGroups];
        Bits x[4][MT];
    };
    auto load = [&](Stage& t, int kt, bool whole) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            t.words[nt] = codes[nt][(size_t)kt * (kTileBytes / 16)];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const size_t at = scale_at[nt] + (size_t)(kt * kGroups + g) * kTileOutputs;
                t.scales[nt][g] = *reinterpret_cast<const v2u*>(w.scales + at);
                t.zeros[nt][g] = ZEROS ? *reinterpret_cast<const uint32_t*>(w.zeros + at) : 0;
            }
        }
#pragma unroll
        for (int step = 0; step < 4; ++step)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                t.x[step][mt] = load_inputs<XT>(row[mt], kt * kTileInputs + 32 * step + 8 * (lane >> 4), w.K, whole);
    };

    v4f acc[NT][MT] = {};
    const typename P::Fragment ones = P::ones(ZEROS);
    auto multiply = [&](const Stage& t) {
        typename P::Fragment xs[4][MT];
#pragma unroll
        for (int step = 0; step < 4; ++step)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) xs[step][mt] = P::activations(t.x[step][mt]);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            typename P::Sum off[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                off[mt] = typename P::Sum{};
#pragma unroll
                for (int j = 0; j < kSteps; ++j) off[mt] = P::multiply(ones, xs[g * kSteps + j][mt], off[mt]);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                typename P::Fragment ws[kSteps];
#pragma unroll
                for (int j = 0; j < kSteps; ++j) ws[j] = P::weights(t.words[nt][g * kSteps + j]);
                const v4f scale = scales_of<BF16>(t.scales[nt][g]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    typename P::Sum sum = off[mt];
                    if (ZEROS)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sum[i] = P::times_zero(off[mt][i], (int)(t.zeros[nt][g] >> (8 * i) & 255));
#pragma unroll
                    for (int j = 0; j < kSteps; ++j) sum = P::multiply(ws[j], xs[g * kSteps + j][mt], sum);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nt][mt][i] = __builtin_fmaf((float)sum[i], scale[i], acc[nt][mt][i]);
                }
            }
        }
    };

    const int whole_tiles = w.K / kTileInputs, count = max(whole_tiles - wave + waves - 1, 0) / waves;
    Stage ahead[AHEAD];
    auto tile = [&](int i) { return wave + min(i, count - 1) * waves; };
    if (count > 0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load(ahead[u], tile(u), true);
        for (int i = 0; i < count; i += AHEAD) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (i + u >= count) break;
                multiply(ahead[u]);
                load(ahead[u], tile(i + u + AHEAD), true);
            }
        }
    }
    if (whole_tiles < w.input_tiles && wave == whole_tiles % waves) {
        load(ahead[0], whole_tiles, false);
        multiply(ahead[0]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sums[wave][nt * MT + mt][lane] = acc[nt][mt];
    __syncthreads();
    if (!fits) return;
    for (int e = threadIdx.x; e < NT * MT * 64; e += blockDim.x) {
        const int tile = e >> 6, l = e & 63;
        v4f total = sums[0][tile][l];
        for (int v = 1; v < waves; ++v) total += sums[v][tile][l];
        store_outputs(o, m0 + 16 * (tile % MT) + (l & 15), (tile0 + tile / MT) * kTileOutputs + 4 * (l >> 4), total, P::kUnit);
    }
}

template <int XT, int GROUP, bool ZEROS, bool BF16, int MT, int NT>
hipError_t launch(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, hipStream_t s) {
    const dim3 grid(ceil_div(w.output_tiles, NT), ceil_div(o.M, 16 * MT));
    if (grid.y > 65535) return hipErrorInvalidValue;
    const int waves = min(kMostWaves, w.input_tiles);
    constexpr int kAhead = MT * (XT == WQ_I8 ? 1 : 2) + NT <= 4 ? 4 : MT <= 2 ? 3 : 2;
    int4_rows_kernel<XT, GROUP, ZEROS, BF16, MT, NT, kAhead><<<grid, 64 * waves, 0, s>>>(static_cast<const typename Element<XT>::type*>(x), x_stride, w, o);
    return hipGetLastError();
}

template <int XT>
hipError_t launch_rows_of(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, hipStream_t s) {
    return with_weights(w, [&](auto group, auto zeros, auto bf16) {
        const bool pairs = w.output_tiles >= 2 * kComputeUnits;
        if (o.M <= 16) return (pairs ? launch<XT, group(), zeros(), bf16(), 1, 2> : launch<XT, group(), zeros(), bf16(), 1, 1>)(x, x_stride, w, o, s);
        if (o.M <= 32) return (pairs ? launch<XT, group(), zeros(), bf16(), 2, 2> : launch<XT, group(), zeros(), bf16(), 2, 1>)(x, x_stride, w, o, s);
        return (pairs ? launch<XT, group(), zeros(), bf16(), 4, 2> : launch<XT, group(), zeros(), bf16(), 4, 1>)(x, x_stride, w, o, s);
    });
}

}  // namespace

}  // namespace wq
