// y = x W^T with 4-bit weights for many rows: the matrix cores' rate bounds it.
//
// A workgroup computes 256 outputs by 128 rows, a wave 64 of the outputs by all rows, over the inputs by tiles of 128.  Codes go from
// memory into the wave's registers as they lie (16 bytes a lane and tile of 16 outputs) and become operands there, once per workgroup;
// activations are shared by the waves through LDS, where the 16-byte piece c of a row r lies at c ^ (r & 15), which keeps the reads of
// 16 rows' pieces free of bank conflicts.  The next tile's activations travel into the other half of the LDS, and its codes into
// registers, while this one is multiplied.  A group's products are summed apart and enter the result by one multiply-add with the scale.
#pragma once
#include "int4_weights.h"

namespace wq {

namespace {

constexpr int kWaves = 4;
constexpr int kWaveOutputs = 4;                               // tiles of 16
constexpr int kOutputs = kWaves * kWaveOutputs * 16;          // of a workgroup
constexpr int kRowTiles = 8;
constexpr int kRows = kRowTiles * 16;

// Operands whose zero point is off already, in the order of the inputs.
template <int XT> struct Exact { static constexpr bool kHas = false; };

template <> struct Exact<WQ_F16> {
    static constexpr bool kHas = true;
    __device__ static uint32_t zero(int z) {   // -(16 + z) / 16, twice
        const uint32_t h = __builtin_bit_cast(uint16_t, (_Float16)(-(16 + z) * 0.0625f));
        return h | h << 16;
    }
    __device__ static v8h weights(uint32_t w, uint32_t zero) {
        const v8h v = Products<WQ_F16>::weights(w);
        const v4u z = {zero, zero, zero, zero};
        return v + __builtin_bit_cast(v8h, z);
    }
};

template <> struct Exact<WQ_I8> {
    static constexpr bool kHas = true;
    __device__ static uint32_t zero(int z) { return 0x04040404u * z; }
    // 4 (code - zero) in every byte: 128 + 4 code holds off a borrow, and its sign bit turned takes the 128 off again
    __device__ static long weights(uint32_t w, uint32_t zero) {
        const uint32_t even = (((w & 0x3c3c3c3cu) | 0x80808080u) - zero) ^ 0x80808080u;
        const uint32_t odd = (((rotate_right(w, 4) & 0x3c3c3c3cu) | 0x80808080u) - zero) ^ 0x80808080u;
        // even: inputs 0 4 1 5, odd: 2 6 3 7
        const v2u r = {__builtin_amdgcn_perm(odd, even, 0x06040200u), __builtin_amdgcn_perm(odd, even, 0x07050301u)};
        return __builtin_bit_cast(long, r);
    }
};

template <int XT, int GROUP, bool ZEROS, bool BF16, bool WHOLE>
__global__ __launch_bounds__(64 * kWaves, 2) void int4_tiles_kernel(const typename Element<XT>::type* x, long long x_stride, Int4Weights w, Int4Output o,
                                                                    int row_tiles, int tiles) {
    typedef typename Element<XT>::type T;
    typedef Products<XT> P;
    typedef Exact<XT> E;
    constexpr int kGroups = kTileInputs / GROUP, kSteps = GROUP / 32;
    constexpr int kPieces = kTileInputs * sizeof(T) / 16;          // 16-byte pieces of a row of the tile
    constexpr int kLoads = kRows * kPieces / (64 * kWaves);        // a thread's
    __shared__ v4u held[2][kRows * kPieces];
    __shared__ v4u codes[kWaves][kWaveOutputs][64];                // each wave's own

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, quarter = lane >> 4;
    // an eighth of the tiles, one behind the other, to each of the eight XCDs, which share their codes in its L2
    const int each = tiles >> 3, rest = tiles & 7, xcd = blockIdx.x & 7;
    const int tile = xcd * each + min(xcd, rest) + (blockIdx.x >> 3);
    const int m0 = tile % row_tiles * kRows, n_tile0 = tile / row_tiles * (kOutputs / 16) + wave * kWaveOutputs;
    const bool fits = matches(w);
    auto output_tile = [&](int nt) { return (size_t)min(n_tile0 + nt, w.output_tiles - 1); };

    auto fetch_codes = [&](int kt) {
#pragma unroll
        for (int nt = 0; nt < kWaveOutputs; ++nt)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(w.codes + (output_tile(nt) * w.input_tiles + kt) * kTileBytes + 16 * lane),
                                             (__attribute__((address_space(3))) void*)(codes[wave][nt]), 16, 0, 0);
    };
    // thread -> (row, piece) of the tile as it lies in LDS
    auto fetch = [&](int kt, int half) {
        const bool whole = WHOLE || (kt + 1) * kTileInputs <= w.K;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = i * 64 * kWaves + threadIdx.x, r = at / kPieces, piece = (at % kPieces) ^ (r & (kPieces - 1));
            const T* const from = x + (long long)min(m0 + r, o.M - 1) * x_stride;
            const int k = kt * kTileInputs + piece * (16 / (int)sizeof(T));
            if (WHOLE) {
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + k),
                                                 (__attribute__((address_space(3))) void*)(&held[half][i * 64 * kWaves + wave * 64]), 16, 0, 0);
            } else if constexpr (XT == WQ_I8) {
                const v2u a = load_inputs<XT>(from, k, w.K, whole), b = load_inputs<XT>(from, k + 8, w.K, whole);
                held[half][at] = v4u{a[0], a[1], b[0], b[1]};
            } else {
                held[half][at] = load_inputs<XT>(from, k, w.K, whole);
            }
        }
    };
    // eight inputs of row 16 mt + row, from 32 step + 8 quarter on
    auto inputs = [&](int half, int mt, int step) {
        const int r = 16 * mt + row;
        if constexpr (XT == WQ_I8) {
            const int piece = 2 * step + (quarter >> 1);
            const v2u* const p = reinterpret_cast<const v2u*>(&held[half][r * kPieces + (piece ^ (r & (kPieces - 1)))]) + (quarter & 1);
            return __builtin_bit_cast(long, *p);
        } else {
            const int piece = 4 * step + quarter;
            return P::activations(held[half][r * kPieces + (piece ^ (r & (kPieces - 1)))]);
        }
    };

    v4f acc[kWaveOutputs][kRowTiles] = {};
    fetch_codes(0);
    fetch(0, 0);
    for (int kt = 0; kt < w.input_tiles; ++kt) {
        const int half = kt & 1;
        __syncthreads();   // this tile is there, the other half has been read
        if (kt + 1 < w.input_tiles) fetch(kt + 1, half ^ 1);
#pragma unroll 1
        for (int g = 0; g < kGroups; ++g) {
            const size_t group = (size_t)(kt * kGroups + g) * kTileOutputs;
            typename P::Fragment ws[kWaveOutputs][kSteps];
            v4f scale[kWaveOutputs];
            uint32_t zeros[kWaveOutputs];
#pragma unroll
            for (int nt = 0; nt < kWaveOutputs; ++nt) {
                const size_t scale_at = output_tile(nt) * w.groups * kTileOutputs + group;
                scale[nt] = load_scales<XT, BF16>(w.scales + scale_at + 4 * quarter);
                uint32_t zero = 0;
                if constexpr (E::kHas) zero = E::zero(ZEROS ? w.zeros[scale_at + row] : 8);
                else if (ZEROS) zeros[nt] = *reinterpret_cast<const uint32_t*>(w.zeros + scale_at + 4 * quarter);
                const uint32_t* const words = reinterpret_cast<const uint32_t*>(&codes[wave][nt][lane]) + g * kSteps;
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    if constexpr (E::kHas) ws[nt][j] = E::weights(words[j], zero);
                    else ws[nt][j] = P::weights(words[j]);
                }
            }
            if (g == kGroups - 1 && kt + 1 < w.input_tiles) fetch_codes(kt + 1);
#pragma unroll
            for (int mt = 0; mt < kRowTiles; ++mt) {
                typename P::Fragment xs[kSteps];
#pragma unroll
                for (int j = 0; j < kSteps; ++j) xs[j] = inputs(half, mt, g * kSteps + j);
                typename P::Sum off = {};
                if constexpr (!E::kHas) {
                    const typename P::Fragment ones = P::ones(ZEROS);
#pragma unroll
                    for (int j = 0; j < kSteps; ++j) off = P::multiply(ones, xs[j], off);
                }
#pragma unroll
                for (int nt = 0; nt < kWaveOutputs; ++nt) {
                    typename P::Sum sum = off;
                    if constexpr (!E::kHas && ZEROS)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sum[i] = P::times_zero(off[i], (int)(zeros[nt] >> (8 * i) & 255));
#pragma unroll
                    for (int j = 0; j < kSteps; ++j) sum = P::multiply(ws[nt][j], xs[j], sum);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nt][mt][i] = __builtin_fmaf((float)sum[i], scale[nt][i], acc[nt][mt][i]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    if (!fits) return;
#pragma unroll
    for (int mt = 0; mt < kRowTiles; ++mt)
#pragma unroll
        for (int nt = 0; nt < kWaveOutputs; ++nt)
            store_outputs(o, m0 + 16 * mt + row, (n_tile0 + nt) * kTileOutputs + 4 * quarter, acc[nt][mt]);
}

template <int XT, int GROUP, bool ZEROS, bool BF16>
hipError_t launch(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, hipStream_t s) {
    typedef typename Element<XT>::type T;
    const int row_tiles = ceil_div(o.M, kRows);
    const long long tiles = (long long)row_tiles * ceil_div(w.N, kOutputs);
    if (tiles > (1 << 23)) return hipErrorInvalidValue;
    // loads straight into LDS move whole, aligned pieces
    const bool whole = w.K % kTileInputs == 0 && (x_stride * sizeof(T)) % 16 == 0 && aligned(x, 16);
    if (whole)
        int4_tiles_kernel<XT, GROUP, ZEROS, BF16, true><<<(unsigned)tiles, 64 * kWaves, 0, s>>>(static_cast<const T*>(x), x_stride, w, o, row_tiles, (int)tiles);
    else
        int4_tiles_kernel<XT, GROUP, ZEROS, BF16, false><<<(unsigned)tiles, 64 * kWaves, 0, s>>>(static_cast<const T*>(x), x_stride, w, o, row_tiles, (int)tiles);
    return hipGetLastError();
}

template <int XT>
hipError_t launch_tiles_of(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, hipStream_t s) {
    return with_weights(w, [&](auto group, auto zeros, auto bf16) { return launch<XT, group(), zeros(), bf16()>(x, x_stride, w, o, s); });
}

}  // namespace

}  // namespace wq
