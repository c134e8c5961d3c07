// The cache held in 8 bits: quantising new keys and values into its blocks, and reading blocks back as values.
#include "int8_cache.h"

namespace wq {

namespace {

constexpr int kThreads = 256;

__device__ inline float finite(float x, float largest) { return x != x ? 0.0f : fminf(fmaxf(x, -largest), largest); }

template <int TYPE> __device__ inline float largest_of();
template <> __device__ inline float largest_of<WQ_F16>() { return 65504.0f; }
template <> __device__ inline float largest_of<WQ_BF16>() { return 3.38953139e38f; }

template <int TYPE>
__device__ inline void load_values(const typename Element<TYPE>::type* p, float (&v)[8]) {
    typedef typename Element<TYPE>::type T;
    typedef T V __attribute__((ext_vector_type(8)));
    const V bits = load_unaligned<V, 2>(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = finite((float)bits[j], largest_of<TYPE>());
}

// The integer nearest to x / s, ties to even, exactly: a candidate from a rounded quotient is off by one at most, and what is left of
// x behind it is a multiple of the distance of floats around s / 2, so that the comparison with s / 2 sees it unrounded.
// up: a power of two that keeps 1 / s finite.
struct Quantiser {
    float s, inverse, up;
    __device__ explicit Quantiser(float scale) : up(scale < 0x1p-100f ? 0x1p64f : 1.0f) {
        s = scale * up;
        inverse = s > 0.0f ? 1.0f / s : 0.0f;
    }
    __device__ int code(float x) const {
        x *= up;
        float q = rintf(x * inverse);
        const float twice = 2.0f * fabsf(__builtin_fmaf(-q, s, x)), rest = __builtin_fmaf(-q, s, x);
        if (twice > s || (twice == s && ((int)q & 1))) q += rest < 0.0f ? -1.0f : 1.0f;
        return s > 0.0f ? min(max((int)q, -127), 127) : 0;
    }
};

// The integer nearest to c * from / to, ties to even, exactly: 31 bits of c * from and of q * to fit a double.
__device__ inline int rescaled(int c, double from, double to, double inverse) {
    const double x = c * from;
    double q = rint(x * inverse);
    const double rest = fma(-q, to, x), twice = 2.0 * fabs(rest);
    if (twice > to || (twice == to && ((int)q & 1))) q += rest < 0.0 ? -1.0 : 1.0;
    return min(max((int)q, -127), 127);
}

__device__ inline uint32_t rescaled4(uint32_t codes, double from, double to, double inverse) {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= (uint32_t)(rescaled((int8_t)(codes >> (8 * i)), from, to, inverse) & 255) << (8 * i);
    return r;
}

struct AppendArgs {
    const void* rows[2];
    long long stride[2];
    int8_t* codes[2];
    float* scales[2];
    Batch batch;
    int kv_heads;
};

// One workgroup per block that receives tokens and head, keys and values apart: the largest magnitude of the new tokens gives the
// scale, then the new tokens (a second time from the caches) become codes.  Keys are stored as they come.  Values change places
// between tokens and head_dim, through LDS by dwords of four tokens; of a dword that also holds bytes that are to stay only the others
// are stored.  Bound by the bytes of the new tokens for prompts, by the latency of its dependent steps for single tokens.
template <int TYPE, int D>
__global__ __launch_bounds__(kThreads) void int8_append_kernel(AppendArgs a) {
    typedef typename Element<TYPE>::type T;
    constexpr int kPieces = D / 8;   // of a row
    __shared__ float wave_largest[kThreads / 64];
    __shared__ uint32_t turned[D * (128 / 4 + 1)];

    const Batch& b = a.batch;
    const int item = blockIdx.x, head = blockIdx.y, is_v = blockIdx.z, P = 1 << b.shift;
    const int s = b.starts ? sequence_of_item(b, item, P, 2) : item;
    const Sequence q = sequence_of(b, s);
    const long long base = (long long)q.length - q.count;   // position of the first row
    const int local = b.starts ? item - item_base(b, s, P, 2) : 0;
    if (local < 0 || q.count <= 0 || q.length <= 0) return;
    const int index = (int)(max(base, 0ll) >> b.shift) + local;
    if (index > (q.length - 1) >> b.shift) return;
    const int page = b.table[(long long)s * b.width + index];
    if ((unsigned)page >= (unsigned)b.blocks) return;
    const long long origin = (long long)index << b.shift;
    const int lo = (int)(max(base, origin) - origin), hi = (int)(min((long long)q.length, origin + P) - origin);
    const long long first = q.first + (origin + lo - base);   // row of the block's first new token
    const T* const rows = static_cast<const T*>(a.rows[is_v]) + first * a.stride[is_v] + head * D;
    const long long stride = a.stride[is_v];
    const long long at = (long long)page * a.kv_heads + head;
    int8_t* const codes = a.codes[is_v] + at * ((long long)D << b.shift);

    float most = 0.0f;
    for (int e = threadIdx.x; e < (hi - lo) * kPieces; e += kThreads) {
        float v[8];
        load_values<TYPE>(rows + (e / kPieces) * stride + e % kPieces * 8, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(v[j]));
    }
#pragma unroll
    for (int step = 32; step > 0; step >>= 1) most = fmaxf(most, __shfl_xor(most, step));
    if ((threadIdx.x & 63) == 0) wave_largest[threadIdx.x >> 6] = most;
    const float old = lo > 0 ? a.scales[is_v][at] : 0.0f;
    __syncthreads();   // also: nobody stores the scale before all have read it
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) most = fmaxf(most, wave_largest[w]);
    const float scale = fmaxf(old, most / 127.0f);
    const bool grown = lo > 0 && scale > old;
    const double from = old, to = scale, inverse = grown ? 1.0 / to : 0.0;
    const Quantiser quantiser(scale);
    if (threadIdx.x == 0) a.scales[is_v][at] = scale;

    if (!is_v) {
        for (int e = threadIdx.x; e < (hi - lo) * kPieces; e += kThreads) {
            float v[8];
            load_values<TYPE>(rows + (e / kPieces) * stride + e % kPieces * 8, v);
            v2u packed = {};
#pragma unroll
            for (int j = 0; j < 8; ++j) packed[j / 4] |= (uint32_t)(quantiser.code(v[j]) & 255) << (8 * (j % 4));
            *reinterpret_cast<v2u*>(codes + (lo + e / kPieces) * D + e % kPieces * 8) = packed;
        }
        if (grown)
            for (int e = threadIdx.x; e < lo * (D / 4); e += kThreads) {
                uint32_t* const p = reinterpret_cast<uint32_t*>(codes) + e;
                *p = rescaled4(*p, from, to, inverse);
            }
        return;
    }

    const int quads = P / 4, line = quads + 1;   // dwords of a row of turned
    for (int e = threadIdx.x; e < ((hi + 3) / 4 - lo / 4) * kPieces; e += kThreads) {
        const int quad = lo / 4 + e / kPieces, piece = e % kPieces;
        uint32_t packed[8] = {};
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * quad + i;
            if (t < lo || t >= hi) continue;
            float v[8];
            load_values<TYPE>(rows + (t - lo) * stride + piece * 8, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) packed[j] |= (uint32_t)(quantiser.code(v[j]) & 255) << (8 * i);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) turned[(piece * 8 + j) * line + quad] = packed[j];
    }
    __syncthreads();
    const int begin = grown ? 0 : lo;   // bytes begin .. hi - 1 of every row change
    const int first_quad = begin / 4, count = (hi + 3) / 4 - first_quad;
    for (int e = threadIdx.x; e < D * count; e += kThreads) {
        const int d = e / count, quad = first_quad + e % count;
        uint32_t* const p = reinterpret_cast<uint32_t*>(codes + ((long long)d << b.shift)) + quad;
        uint32_t word = 4 * quad + 3 >= lo ? turned[d * line + quad] : 0;
        if (4 * quad < lo && grown) {
            const uint32_t older = rescaled4(*p, from, to, inverse), keep = lo - 4 * quad >= 4 ? ~0u : (1u << (8 * (lo - 4 * quad))) - 1;
            word = (older & keep) | (word & ~keep);
        }
        if (4 * quad >= begin && 4 * quad + 4 <= hi) *p = word;
        else
            for (int i = 0; i < 4; ++i)
                if (4 * quad + i >= begin && 4 * quad + i < hi) reinterpret_cast<int8_t*>(p)[i] = (int8_t)(word >> (8 * i));
    }
}

template <int TYPE, int D>
hipError_t append(const AppendArgs& a, hipStream_t s) {
    const long long items = a.batch.starts ? item_count(a.batch.rows, a.batch.sequences, 1 << a.batch.shift, 2) : a.batch.sequences;
    int8_append_kernel<TYPE, D><<<dim3((unsigned)items, a.kv_heads, 2), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

struct ReadArgs {
    const int8_t* codes[2];
    const float* scales[2];
    void* out[2];
    const int32_t* ids;
    int blocks, kv_heads, shift;
};

template <int TYPE>
__device__ inline void store_values(void* out, long long at, const float (&v)[8]) {
    if constexpr (TYPE == WQ_F32) {
        v4f* const p = reinterpret_cast<v4f*>(static_cast<float*>(out) + at);
        p[0] = v4f{v[0], v[1], v[2], v[3]};
        p[1] = v4f{v[4], v[5], v[6], v[7]};
    } else {
        typedef typename Element<TYPE>::type T;
        typedef T V __attribute__((ext_vector_type(8)));
        V r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = (T)v[j];
        *reinterpret_cast<V*>(static_cast<T*>(out) + at) = r;
    }
}

__device__ inline float value(uint32_t codes, int i, float scale) { return (float)(int8_t)(codes >> (8 * i)) * scale; }

// One workgroup per block and head, keys and values apart; values change places between tokens and head_dim through LDS.  Bound by
// the bytes written.
template <int TYPE, int D>
__global__ __launch_bounds__(kThreads) void int8_read_kernel(ReadArgs a) {
    constexpr int kPieces = D / 8;
    __shared__ uint32_t held[D * (128 / 4 + 1)];
    const int head = blockIdx.y, is_v = blockIdx.z, P = 1 << a.shift, quads = P / 4, line = quads + 1;
    const int page = a.ids[blockIdx.x];
    const bool there = (unsigned)page < (unsigned)a.blocks;
    const long long at = there ? (long long)page * a.kv_heads + head : 0;
    const float scale = there ? a.scales[is_v][at] : 0.0f;
    const uint32_t* const codes = reinterpret_cast<const uint32_t*>(a.codes[is_v] + at * ((long long)D << a.shift));
    const long long out = ((long long)blockIdx.x * a.kv_heads + head) * ((long long)D << a.shift);
    if (!is_v) {
        for (int e = threadIdx.x; e < P * kPieces; e += kThreads) {
            const v2u c = there ? reinterpret_cast<const v2u*>(codes)[e] : v2u{};
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = value(c[j / 4], j % 4, scale);
            store_values<TYPE>(a.out[0], out + 8ll * e, v);
        }
        return;
    }
    for (int e = threadIdx.x; e < D * quads; e += kThreads) held[e / quads * line + e % quads] = there ? codes[e] : 0;
    __syncthreads();
    for (int e = threadIdx.x; e < quads * kPieces; e += kThreads) {
        const int quad = e / kPieces, piece = e % kPieces;
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = held[(piece * 8 + j) * line + quad];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = value(c[j], i, scale);
            store_values<TYPE>(a.out[1], out + (long long)(4 * quad + i) * D + piece * 8, v);
        }
    }
}

template <int TYPE, int D>
hipError_t read(const ReadArgs& a, int count, hipStream_t s) {
    int8_read_kernel<TYPE, D><<<dim3(count, a.kv_heads, 2), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <int D>
hipError_t read_type(const ReadArgs& a, int count, int type, hipStream_t s) {
    return type == WQ_F32 ? read<WQ_F32, D>(a, count, s) : type == WQ_F16 ? read<WQ_F16, D>(a, count, s) : read<WQ_BF16, D>(a, count, s);
}

}  // namespace

}  // namespace wq

using namespace wq;

extern "C" {

int int8_cache_append(const void* k_dev, long long k_stride, const void* v_dev, long long v_stride, int type, int rows,
                      int8_t* cache_k_dev, int8_t* cache_v_dev, float* k_scale_dev, float* v_scale_dev, int blocks,
                      int kv_heads, int head_dim, int block, const int32_t* table_dev, int table_width, int sequences,
                      const int32_t* lengths_dev, const int32_t* starts_dev, void* hip_stream) {
    const CacheArgs c = {cache_k_dev, cache_v_dev, k_scale_dev, v_scale_dev, blocks, kv_heads, head_dim, block};
    if (int st = check_cache(c)) return st;
    bool empty;
    if (int st = check_batch(rows, table_dev, table_width, sequences, lengths_dev, starts_dev, block, empty)) return st;
    if (!is_half(type) || k_stride < (long long)kv_heads * head_dim || v_stride < (long long)kv_heads * head_dim) return WG_EINVAL;
    if (empty) return WG_OK;
    if (!k_dev || !v_dev || !aligned(k_dev, 2) || !aligned(v_dev, 2)) return WG_EINVAL;
    const Batch b = {table_dev, lengths_dev, starts_dev, table_width, sequences, rows, blocks, block_shift(block)};
    if (item_count(rows, sequences, block, 2) > kMostItems) return WG_EUNSUPPORTED;
    const AppendArgs a = {{k_dev, v_dev}, {k_stride, v_stride}, {cache_k_dev, cache_v_dev}, {k_scale_dev, v_scale_dev}, b, kv_heads};
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (type == WQ_F16)
        return status_of(head_dim == 64 ? append<WQ_F16, 64>(a, s) : head_dim == 128 ? append<WQ_F16, 128>(a, s) : append<WQ_F16, 256>(a, s));
    return status_of(head_dim == 64 ? append<WQ_BF16, 64>(a, s) : head_dim == 128 ? append<WQ_BF16, 128>(a, s) : append<WQ_BF16, 256>(a, s));
}

int int8_cache_read(const int8_t* cache_k_dev, const int8_t* cache_v_dev, const float* k_scale_dev, const float* v_scale_dev,
                    int blocks, int kv_heads, int head_dim, int block, const int32_t* ids_dev, int count, void* out_k_dev,
                    void* out_v_dev, int type, void* hip_stream) {
    const CacheArgs c = {cache_k_dev, cache_v_dev, k_scale_dev, v_scale_dev, blocks, kv_heads, head_dim, block};
    if (int st = check_cache(c)) return st;
    if (count < 0 || !(is_half(type) || type == WQ_F32)) return WG_EINVAL;
    if (count == 0) return WG_OK;
    if (!ids_dev || !out_k_dev || !out_v_dev) return WG_EINVAL;
    if (!aligned(ids_dev, 4) || !aligned(out_k_dev, 16) || !aligned(out_v_dev, 16)) return WG_EINVAL;
    if (count > kMostItems) return WG_EUNSUPPORTED;
    const ReadArgs a = {{cache_k_dev, cache_v_dev}, {k_scale_dev, v_scale_dev}, {out_k_dev, out_v_dev}, ids_dev, blocks, kv_heads, block_shift(block)};
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return status_of(head_dim == 64 ? read_type<64>(a, count, type, s) : head_dim == 128 ? read_type<128>(a, count, type, s) : read_type<256>(a, count, type, s));
}

}  // extern "C"
