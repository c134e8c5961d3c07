// How packed 4-bit weights lie in memory, and how a wave turns them into matrix-core operands.
#pragma once
#include <type_traits>

#include "quantized_common.h"

namespace wq {

// Blob: [header][codes][scales][zero points].  Codes lie in tiles of 16 outputs by 128 inputs, 1 KB each, the tiles of 16 outputs
// one behind the other: lane l of a wave reads its 16 bytes of a tile in one load, word w of them holding the eight codes of output
// l % 16 and inputs 32 w + 8 (l / 16) ..  + 7, which is what that lane contributes to a 16x16x32 matrix-core product.  Scales and
// zero points lie in the order the same wave needs them: [tile of outputs][group][16].
//
// Within a word the code of input j (0..7) is field s = j / 2 + 4 (j % 2) of eight, field s at bits 4 s + 2 .. 4 s + 5 of the word
// taken as a ring.  So two codes of neighbouring inputs are 16 bits apart, and a field lies where a 16-bit float keeps the upper
// bits of its fraction: masked there and joined with the bits of 1.0 it reads as 1 + code / 16, exactly, without a conversion.
constexpr int kTileOutputs = 16;
constexpr int kTileInputs = 128;
constexpr int kTileRows = 128;   // of the kernel for many rows
constexpr int kTileBytes = kTileOutputs * kTileInputs / 2;

constexpr uint32_t kInt4Magic = 0x34695157u;
constexpr uint32_t kInt4Version = 1;
struct Int4Header {
    uint32_t magic, version;
    int32_t N, K, group, scale_type, has_zeros;
    uint32_t pad[57];
};
static_assert(sizeof(Int4Header) == 256, "the codes are 256-byte aligned");

struct Int4Layout {
    int output_tiles, input_tiles, groups;   // groups: those of whole input tiles
    size_t codes, scales, zeros, total;      // offsets
};
inline Int4Layout int4_layout(int N, int K, int group, int has_zeros) {
    Int4Layout l;
    l.output_tiles = ceil_div(N, kTileOutputs);
    l.input_tiles = ceil_div(K, kTileInputs);
    l.groups = l.input_tiles * (kTileInputs / group);
    l.codes = sizeof(Int4Header);
    l.scales = l.codes + (size_t)l.output_tiles * l.input_tiles * kTileBytes;
    l.zeros = l.scales + (((size_t)l.output_tiles * l.groups * kTileOutputs * 2 + 255) & ~(size_t)255);
    l.total = l.zeros + (has_zeros ? (((size_t)l.output_tiles * l.groups * kTileOutputs + 255) & ~(size_t)255) : 0);
    return l;
}

struct Int4Weights {
    const uint8_t* blob;
    const uint8_t* codes;
    const uint16_t* scales;
    const uint8_t* zeros;
    int output_tiles, input_tiles, groups;
    int N, K, group, scale_type, has_zeros;
};

__device__ inline bool matches(const Int4Weights& w) {
    const Int4Header* h = reinterpret_cast<const Int4Header*>(w.blob);
    return (h->magic == kInt4Magic) & (h->version == kInt4Version) & (h->N == w.N) & (h->K == w.K) & (h->group == w.group) &
           (h->scale_type == w.scale_type) & (h->has_zeros == w.has_zeros);
}

// A constant in a vector register, as the compiler sees it a value of each lane: (w & field) | this is one instruction only where not
// both come from scalar registers.  (Written as inline assembly, that instruction may overwrite the start value of a product under way:
// the compiler keeps the wait states in between only for instructions that it knows.)
__device__ inline uint32_t in_lanes(uint32_t constant) { return __builtin_amdgcn_mbcnt_hi(0u, constant); }

__device__ inline uint32_t rotate_right(uint32_t w, int bits) { return __builtin_amdgcn_alignbit(w, w, bits); }

// What the products of one type of activations are made of.  A code u enters as a x16 or x4 multiple of itself plus a constant:
// unit * sum_k operand(u_k) x_k = sum_k (u_k + offset) x_k; the product with `ones`, whose elements are all -kOnes, takes
// zero + offset off again.
template <int XT> struct Products;

template <> struct Products<WQ_F16> {
    typedef v8h Fragment;
    typedef v4f Sum;
    static constexpr float kUnit = 16.0f;   // operand 1 + u / 16
    static constexpr int kOffset = 16;
    static constexpr uint32_t kOne = 0x3c003c00u;
    __device__ static Fragment weights(uint32_t w, uint32_t one) {   // one: kOne in the lanes
        const uint32_t field = 0x03c003c0u;
        const v4u r = {((w << 4) & field) | one, (w & field) | one, ((w >> 4) & field) | one, (rotate_right(w, 8) & field) | one};
        return __builtin_bit_cast(Fragment, r);
    }
    // the same value in every place: -(16 + 8) / 16 where the zero point is 8 everywhere, else -1 / 16
    __device__ static Fragment ones(bool zeros) {
        const uint32_t v = zeros ? 0xac00ac00u : 0xbe00be00u;
        const v4u r = {v, v, v, v};
        return __builtin_bit_cast(Fragment, r);
    }
    __device__ static Sum multiply(const Fragment& a, const Fragment& b, const Sum& c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
    __device__ static Fragment activations(const v4u& v) { return __builtin_bit_cast(Fragment, v); }
    __device__ static float times_zero(float sum, int zero) { return sum * (float)(kOffset + zero); }
};

template <> struct Products<WQ_BF16> {
    typedef v8b Fragment;
    typedef v4f Sum;
    static constexpr float kUnit = 16.0f;
    static constexpr int kOffset = 16;
    static constexpr uint32_t kOne = 0x3f803f80u;
    __device__ static Fragment weights(uint32_t w, uint32_t one) {
        const uint32_t field = 0x00780078u;
        const v4u r = {((w << 1) & field) | one, ((w >> 3) & field) | one, ((w >> 7) & field) | one, (rotate_right(w, 11) & field) | one};
        return __builtin_bit_cast(Fragment, r);
    }
    __device__ static Fragment ones(bool zeros) {
        const uint32_t v = zeros ? 0xbd80bd80u : 0xbfc0bfc0u;
        const v4u r = {v, v, v, v};
        return __builtin_bit_cast(Fragment, r);
    }
    __device__ static Sum multiply(const Fragment& a, const Fragment& b, const Sum& c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    __device__ static Fragment activations(const v4u& v) { return __builtin_bit_cast(Fragment, v); }
    __device__ static float times_zero(float sum, int zero) { return sum * (float)(kOffset + zero); }
};

template <> struct Products<WQ_I8> {
    typedef long Fragment;
    typedef v4i Sum;
    static constexpr float kUnit = 0.25f;   // operand 4 u: fields two bits up in their bytes
    static constexpr int kOffset = 0;
    static constexpr uint32_t kOne = 0x80808080u;
    __device__ static Fragment weights(uint32_t w, uint32_t) {
        const v2u r = {w & 0x3c3c3c3cu, rotate_right(w, 4) & 0x3c3c3c3cu};
        return __builtin_bit_cast(Fragment, r);
    }
    __device__ static Fragment ones(bool zeros) {
        const uint32_t v = zeros ? 0xfcfcfcfcu : 0xe0e0e0e0u;   // -4 or -4 * 8
        const v2u r = {v, v};
        return __builtin_bit_cast(Fragment, r);
    }
    __device__ static Sum multiply(const Fragment& a, const Fragment& b, const Sum& c) {
        return __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, c, 0, 0, 0);
    }
    // eight inputs in the order in which weights() leaves their codes: 0 4 1 5, 2 6 3 7
    __device__ static Fragment activations(const v2u& v) {
        const v2u r = {__builtin_amdgcn_perm(v[1], v[0], 0x05010400u), __builtin_amdgcn_perm(v[1], v[0], 0x07030602u)};
        return __builtin_bit_cast(Fragment, r);
    }
    __device__ static int times_zero(int sum, int zero) { return __mul24(sum, zero); }
};

// Eight inputs of a row from `k` on, zeros behind the row's end.
template <int XT>
__device__ inline auto load_inputs(const typename Element<XT>::type* row, int k, int K) {
    typedef typename Element<XT>::type T;
    typedef std::conditional_t<XT == WQ_I8, v2u, v4u> Bits;
    if (k + 8 <= K) return load_unaligned<Bits, sizeof(T)>(row + k);
    union { Bits bits; T e[8]; } r;
    r.bits = Bits{};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (k + j < K) r.e[j] = row[k + j];
    return r.bits;
}

// The scales of four neighbouring outputs.
template <bool BF16>
__device__ inline v4f scales_of(v2u bits) {
    v4f s;
    if constexpr (BF16) {
        s = v4f{__builtin_bit_cast(float, bits[0] << 16), __builtin_bit_cast(float, bits[0] & 0xffff0000u),
                __builtin_bit_cast(float, bits[1] << 16), __builtin_bit_cast(float, bits[1] & 0xffff0000u)};
    } else {
        const v4h h = __builtin_bit_cast(v4h, bits);
        s = v4f{(float)h[0], (float)h[1], (float)h[2], (float)h[3]};
    }
    return s;
}

// What becomes of a finished sum: the row's scale, bias, ReLU, one rounding.
struct Int4Output {
    const float* x_scale;
    const float* bias;
    void* y;
    int type, M, N, relu;
};

__device__ inline void store_rounded(const Int4Output& o, int m, int n, const float (&r)[4]) {
    const long long at = (long long)m * o.N + n;
    const int count = min(4, o.N - n);
    if (o.type == WQ_F32) {
        float* y = static_cast<float*>(o.y) + at;
        if (count == 4) store_unaligned<4>(y, v4f{r[0], r[1], r[2], r[3]});
        else
            for (int i = 0; i < count; ++i) y[i] = r[i];
        return;
    }
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        h[i] = o.type == WQ_F16 ? __builtin_bit_cast(uint16_t, (_Float16)r[i]) : __builtin_bit_cast(uint16_t, (__bf16)r[i]);
    uint16_t* y = static_cast<uint16_t*>(o.y) + at;
    if (count == 4) store_unaligned<2>(y, v2u{h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16});
    else
        for (int i = 0; i < count; ++i) y[i] = h[i];
}

// unit: the operands'.
__device__ inline void store_outputs(const Int4Output& o, int m, int n, v4f v, float unit) {
    if (m >= o.M || n >= o.N) return;
    v *= unit;
    if (o.x_scale) v *= o.x_scale[m];
    float r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[i] = v[i];
        if (o.bias && n + i < o.N) r[i] += o.bias[n + i];
        if (o.relu) r[i] = r[i] < 0.0f ? 0.0f : r[i];   // keeps NaN
    }
    store_rounded(o, m, n, r);
}

// The same where many are stored: behind a store, every load of a scale or a bias would be waited for by itself, so they come first.
__device__ inline float row_scale(const Int4Output& o, int m, float unit) { return o.x_scale ? unit * o.x_scale[min(m, o.M - 1)] : unit; }
__device__ inline v4f bias_of(const Int4Output& o, int n) {
    v4f b = {};
    if (o.bias)
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = o.bias[min(n + i, o.N - 1)];
    return b;
}
__device__ inline void store_outputs(const Int4Output& o, int m, int n, v4f v, float scale, v4f bias) {
    if (m >= o.M || n >= o.N) return;
    float r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r[i] = v[i] * scale;
        if (o.bias) r[i] += bias[i];
        if (o.relu) r[i] = r[i] < 0.0f ? 0.0f : r[i];
    }
    store_rounded(o, m, n, r);
}

hipError_t launch_int4_pack(const uint8_t* codes, const void* scales, const uint8_t* zeros, const Int4Weights& w, uint8_t* blob, hipStream_t s);
// One translation unit per type of activations: the variants take their time to compile.
hipError_t launch_int4_rows_half(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, hipStream_t s);
hipError_t launch_int4_rows_bfloat(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, hipStream_t s);
hipError_t launch_int4_rows_int8(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, hipStream_t s);
// Many rows: x holds whole tiles (kTileInputs inputs, kTileRows rows or more) of 16-byte aligned rows.  parts > 1: that many sums of
// parts of the inputs, one y of float32 behind the other.
hipError_t launch_int4_tiles_half(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, int parts, hipStream_t s);
hipError_t launch_int4_tiles_int8(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, int parts, hipStream_t s);

// Calls launch(group, has zero points, scales are bfloat16), each as a constant, for what the weights are.
template <class F>
hipError_t with_weights(const Int4Weights& w, F&& launch) {
    auto scales = [&](auto group, auto zeros) {
        return w.scale_type == WQ_BF16 ? launch(group, zeros, std::true_type()) : launch(group, zeros, std::false_type());
    };
    auto zeros = [&](auto group) { return w.has_zeros ? scales(group, std::true_type()) : scales(group, std::false_type()); };
    return w.group == 32 ? zeros(std::integral_constant<int, 32>()) : w.group == 64 ? zeros(std::integral_constant<int, 64>()) : zeros(std::integral_constant<int, 128>());
}

}  // namespace wq
