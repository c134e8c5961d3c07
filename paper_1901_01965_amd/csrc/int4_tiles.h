// y = x W^T with 4-bit weights for many rows: the matrix cores' rate bounds it (4096 rows through 4096 x 8192, float16 in groups of 128: 232 us,
// 1.18 PFLOP/s; int8 184).
//
// A workgroup computes 64 NT outputs by 128 rows, each of its four waves 16 NT of the outputs by all rows, over the inputs by tiles
// of 128.  Codes go through the wave's own part of the LDS as they lie and become operands in registers, once per workgroup; activations
// are shared by the waves through LDS, where the 16-byte piece c of a row r lies at c ^ (r & 15), which keeps the reads of 16 rows'
// pieces free of bank conflicts.  Both travel there without registers, the next tile's while this one is multiplied.  A group's
// products are summed apart and enter the result by one multiply-add with the scale; those of 16 rows are done between the products of
// the next 16.  While a wave multiplies it goes ahead of the other one of its SIMD, which then unpacks codes meanwhile (5% of
// that time).
//
// bfloat16 activations come here as float16 (int4_linear.hip): unpacked codes then take their zero point off by a packed addition, for
// which bfloat16 has no instruction (the product with a constant that stands in for it elsewhere took a fifth of the matrix cores).
#pragma once
#include "int4_weights.h"

namespace wq {

namespace {

constexpr int kWaves = 4;
constexpr int kRowTiles = 8;
constexpr int kRows = kTileRows;
static_assert(kRows == 16 * kRowTiles, "rows of a tile");
constexpr int kBand = 8;

// Operands whose zero point is off already, in the order of the inputs.
template <int XT> struct Exact;

template <> struct Exact<WQ_F16> {
    __device__ static uint32_t zero(int z) {   // -(16 + z) / 16, twice
        const uint32_t h = __builtin_bit_cast(uint16_t, (_Float16)(-(16 + z) * 0.0625f));
        return h | h << 16;
    }
    __device__ static v8h weights(uint32_t w, uint32_t zero, uint32_t one) {
        const v8h v = Products<WQ_F16>::weights(w, one);
        const v4u z = {zero, zero, zero, zero};
        return v + __builtin_bit_cast(v8h, z);
    }
};

template <> struct Exact<WQ_I8> {
    __device__ static uint32_t zero(int z) { return 0x04040404u * z; }
    // 4 (code - zero) in every byte: 128 + 4 code holds off a borrow, and its sign bit turned takes the 128 off again
    __device__ static long weights(uint32_t w, uint32_t zero, uint32_t one) {
        const uint32_t field = 0x3c3c3c3cu, even = (((w & field) | one) - zero) ^ one, odd = (((rotate_right(w, 4) & field) | one) - zero) ^ one;
        // even: inputs 0 4 1 5, odd: 2 6 3 7
        const v2u r = {__builtin_amdgcn_perm(odd, even, 0x06040200u), __builtin_amdgcn_perm(odd, even, 0x07050301u)};
        return __builtin_bit_cast(long, r);
    }
};

template <int XT, int GROUP, bool ZEROS, bool BF16, int NT>
__global__ __launch_bounds__(64 * kWaves, 2) void int4_tiles_kernel(const typename Element<XT>::type* x, long long x_stride, Int4Weights w, Int4Output o,
                                                                    int row_tiles, int tiles) {
    typedef typename Element<XT>::type T;
    typedef Products<XT> P;
    typedef Exact<XT> E;
    constexpr int kGroups = kTileInputs / GROUP, kSteps = GROUP / 32;
    constexpr int kPieces = kTileInputs * sizeof(T) / 16;          // 16-byte pieces of a row of the tile
    constexpr int kLoads = kRows * kPieces / (64 * kWaves);        // a thread's
    // two arrays, each known by name wherever it is read or written: of one, reads would wait for what is on its way into the other half
    __shared__ v4u even[kRows * kPieces], odd[kRows * kPieces];
    typedef v4u Held[kRows * kPieces];
    __shared__ v4u codes[kWaves][NT][64];                          // each wave's own

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, quarter = lane >> 4;
    // An eighth of the tiles, one behind the other, to each of the eight XCDs, in bands of eight tiles of rows: what runs at a time there
    // is about as high as wide, which asks least of memory behind its L2.
    const int each = tiles >> 3, rest = tiles & 7, xcd = blockIdx.x & 7;
    const int tile = xcd * each + min(xcd, rest) + (blockIdx.x >> 3);
    const int across = tiles / row_tiles, band = tile / (kBand * across), height = min(kBand, row_tiles - band * kBand);
    const int in_band = tile - band * kBand * across, row_tile = band * kBand + in_band % height, column = in_band / height;
    // the last tile of rows ends with the last row: it may share rows with the one before, which get the same values twice
    const int m0 = max(min(row_tile * kRows, o.M - kRows), 0), n_tile0 = (column * kWaves + wave) * NT;
    // tiles of inputs: all, or a part of them (of few outputs only: more a wave leave no registers for it)
    const int parts = NT == 2 ? gridDim.y : 1, begin = NT == 2 ? w.input_tiles * blockIdx.y / parts : 0, end = NT == 2 ? w.input_tiles * (blockIdx.y + 1) / parts : w.input_tiles;
    const bool fits = matches(w);
    const uint32_t one = in_lanes(P::kOne);
    auto output_tile = [&](int nt) { return (size_t)min(n_tile0 + nt, w.output_tiles - 1); };

    auto fetch_codes = [&](int kt) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(w.codes + (output_tile(nt) * w.input_tiles + kt) * kTileBytes + 16 * lane),
                                             (__attribute__((address_space(3))) void*)(codes[wave][nt]), 16, 0, 0);
    };
    // thread -> (row, piece) of the tile as it lies in LDS: from load to load the same distance for all
    const int my_row = threadIdx.x / kPieces, my_piece = (threadIdx.x % kPieces) ^ (my_row & (kPieces - 1));
    const uint32_t my_bytes = (uint32_t)(my_row * x_stride * sizeof(T)) + 16 * my_piece;
    auto fetch = [&](int kt, Held& held) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const char* const from = reinterpret_cast<const char*>(x + (long long)(m0 + i * 64 * kWaves / kPieces) * x_stride + kt * kTileInputs);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + my_bytes),
                                             (__attribute__((address_space(3))) void*)(&held[i * 64 * kWaves + wave * 64]), 16, 0, 0);
        }
    };
    // eight inputs of row 16 mt + row, from 32 step + 8 quarter on
    auto inputs = [&](const Held& held, int mt, int step) {
        const int r = 16 * mt + row;
        if constexpr (XT == WQ_I8) {
            const int piece = 2 * step + (quarter >> 1);
            const v2u* const p = reinterpret_cast<const v2u*>(&held[r * kPieces + (piece ^ (r & (kPieces - 1)))]) + (quarter & 1);
            return __builtin_bit_cast(long, *p);
        } else {
            const int piece = 4 * step + quarter;
            return P::activations(held[r * kPieces + (piece ^ (r & (kPieces - 1)))]);
        }
    };

    // scales and zero points of a group, on their way while the group before is multiplied
    struct Factors {
        v2u scales[NT];
        uint32_t zeros[NT];
    };
    auto fetch_factors = [&](Factors& f, int group) {
        const size_t first = (size_t)min(group, w.input_tiles * kGroups - 1) * kTileOutputs;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const size_t at = output_tile(nt) * w.groups * kTileOutputs + first;
            f.scales[nt] = *reinterpret_cast<const v2u*>(w.scales + at + 4 * quarter);
            f.zeros[nt] = 0;
            if (ZEROS) f.zeros[nt] = w.zeros[at + row];
        }
    };

    v4f acc[NT][kRowTiles] = {};
    Factors next;
    fetch_codes(begin);
    fetch(begin, even);
    fetch_factors(next, begin * kGroups);
    auto multiply = [&](int kt, const Held& held, Held& other) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's share of the tile is there
        __syncthreads();                                   // everyone's is, and the other half has been read
        if (kt + 1 < end) fetch(kt + 1, other);
#pragma unroll 1
        for (int group = 0; group < kGroups; ++group) {
            typename P::Fragment ws[NT][kSteps];
            const Factors now = next;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const uint32_t zero = E::zero(ZEROS ? (int)now.zeros[nt] : 8);
                const uint32_t* const words = reinterpret_cast<const uint32_t*>(&codes[wave][nt][lane]) + group * kSteps;
#pragma unroll
                for (int j = 0; j < kSteps; ++j) ws[nt][j] = E::weights(words[j], zero, one);
            }
            __builtin_amdgcn_sched_barrier(0);   // the codes are read before the next ones are asked for in their place
            if (group == kGroups - 1 && kt + 1 < end) fetch_codes(kt + 1);
            v4f scale[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) scale[nt] = scales_of<BF16>(now.scales[nt]);
            fetch_factors(next, kt * kGroups + group + 1);
            typename P::Fragment xs[2][kSteps];
#pragma unroll
            for (int j = 0; j < kSteps; ++j) xs[0][j] = inputs(held, 0, group * kSteps + j);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            // the products of 16 rows, and between them the multiply-adds of the 16 before
            typename P::Sum sums[2][NT];
#pragma unroll
            for (int mt = 0; mt <= kRowTiles; ++mt) {
                if (mt + 1 < kRowTiles)
#pragma unroll
                    for (int j = 0; j < kSteps; ++j) xs[(mt + 1) & 1][j] = inputs(held, mt + 1, group * kSteps + j);
                if (mt < kRowTiles) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) sums[mt & 1][nt] = typename P::Sum{};
#pragma unroll
                    for (int j = 0; j < kSteps; ++j)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) sums[mt & 1][nt] = P::multiply(ws[nt][j], xs[mt & 1][j], sums[mt & 1][nt]);
                }
                if (mt > 0)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            acc[nt][mt - 1][i] = __builtin_fmaf((float)sums[(mt - 1) & 1][nt][i], scale[nt][i], acc[nt][mt - 1][i]);
                if (mt > 0 && mt < kRowTiles)
#pragma unroll
                    for (int i = 0; i < kSteps * NT; ++i) {
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);   // a product
                        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);   // a read of LDS
                        __builtin_amdgcn_sched_group_barrier(0x002, 4 / kSteps, 0);
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
        }
    };
    for (int kt = begin; kt < end; kt += 2) {
        multiply(kt, even, odd);
        if (kt + 1 < end) multiply(kt + 1, odd, even);
    }
    if (!fits) return;
    if (parts > 1) o.y = static_cast<float*>(o.y) + (size_t)blockIdx.y * o.M * o.N;
    if constexpr (NT == 2) {
        // (225 rows, 32 outputs of 128 inputs with bias and scales 12 us without, 8 with; for more outputs, and so more inputs as well, there are
        // no registers)
        float scale[kRowTiles];
        v4f bias[NT];
#pragma unroll
        for (int mt = 0; mt < kRowTiles; ++mt) scale[mt] = row_scale(o, m0 + 16 * mt + row, P::kUnit);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) bias[nt] = bias_of(o, (n_tile0 + nt) * kTileOutputs + 4 * quarter);
#pragma unroll
        for (int mt = 0; mt < kRowTiles; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                store_outputs(o, m0 + 16 * mt + row, (n_tile0 + nt) * kTileOutputs + 4 * quarter, acc[nt][mt], scale[mt], bias[nt]);
        return;
    }
#pragma unroll
    for (int mt = 0; mt < kRowTiles; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            store_outputs(o, m0 + 16 * mt + row, (n_tile0 + nt) * kTileOutputs + 4 * quarter, acc[nt][mt], P::kUnit);
}

template <int XT, int GROUP, bool ZEROS, bool BF16, int NT>
hipError_t launch(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, int parts, hipStream_t s) {
    const int row_tiles = ceil_div(o.M, kRows);
    const long long tiles = (long long)row_tiles * ceil_div(w.output_tiles, kWaves * NT);
    int4_tiles_kernel<XT, GROUP, ZEROS, BF16, NT><<<dim3((unsigned)tiles, parts), 64 * kWaves, 0, s>>>(static_cast<const typename Element<XT>::type*>(x), x_stride, w, o,
                                                                                        row_tiles, (int)tiles);
    return hipGetLastError();
}

// Rounds of two workgroups per compute unit that this many outputs a wave take.
inline long long rounds(const Int4Weights& w, const Int4Output& o, int nt) {
    return ((long long)ceil_div(o.M, kRows) * ceil_div(w.output_tiles, kWaves * nt) + 2 * kComputeUnits - 1) / (2 * kComputeUnits);
}

template <int XT>
hipError_t launch_tiles_of(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, int parts, hipStream_t s) {
    return with_weights(w, [&](auto group, auto zeros, auto bf16) {
        // More tiles of outputs a wave read LDS less often per product, in coarser rounds: three of float16 in groups of 128, whose operands leave no
        // room for four, which cost 1.23 of two's time a round, four otherwise, 1.84.  (Three against two: 4096 rows through 4096 x 8192
        // 237 and 250 us, 8192 through 4096 x 28672 1546 and 1735, but 2048 through 4096 x 4096 72 and 66; four against two: int8, 4096
        // through 4096 x 8192, 184 and 217, 1200 float16 rows in groups of 32 through 448 x 20000 58 and 65.)
        constexpr int kMore = XT == WQ_F16 && group() == 128 ? 3 : 4;
        constexpr double kCost = kMore == 3 ? 0.82 * 1.5 : 0.92 * 2;
        if (parts == 1 && rounds(w, o, kMore) * kCost < rounds(w, o, 2)) return launch<XT, group(), zeros(), bf16(), kMore>(x, x_stride, w, o, 1, s);
        return launch<XT, group(), zeros(), bf16(), 2>(x, x_stride, w, o, parts, s);
    });
}

}  // namespace

}  // namespace wq
