// C ABI of the products with 4-bit weights: argument checks on the host, layout of the weights, choice of the kernel.
#include "int4_weights.h"

namespace wq {

namespace {

bool valid_weights(int N, int K, int group) {
    return N > 0 && K > 0 && (group == 32 || group == 64 || group == 128);
}

// Keeps every count an int and every launch below 2^32 threads: 2^34 codes, 2^22 outputs.
bool too_large(int N, int K) {
    return N > (1 << 22) || K > (1 << 26) || (long long)ceil_div(N, kTileOutputs) * ceil_div(K, kTileInputs) > (1 << 23);
}

Int4Weights weights_of(const void* blob, int N, int K, int group, int scale_type, int has_zeros) {
    const Int4Layout l = int4_layout(N, K, group, has_zeros);
    const uint8_t* b = static_cast<const uint8_t*>(blob);
    return {b, b + l.codes, reinterpret_cast<const uint16_t*>(b + l.scales), has_zeros ? b + l.zeros : nullptr,
            l.output_tiles, l.input_tiles, l.groups, N, K, group, scale_type, has_zeros};
}

// One thread per word of codes, then one per scale (with its zero point).  Places without an output or an input get code 0 and scale
// 0: inputs behind the row's end are read as zeros, outputs behind the last are not stored.
__global__ void int4_pack_kernel(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, Int4Weights w, uint8_t* blob,
                                 long long words, long long total) {
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i == 0) {
        Int4Header* h = reinterpret_cast<Int4Header*>(blob);
        h->magic = kInt4Magic; h->version = kInt4Version;
        h->N = w.N; h->K = w.K; h->group = w.group; h->scale_type = w.scale_type; h->has_zeros = w.has_zeros;
    }
    if (i < words) {
        const int word = (int)(i & 3), lane = (int)(i >> 2) & 63;
        const long long tile = i >> 8;
        const long long n = tile / w.input_tiles * kTileOutputs + (lane & 15);
        const long long k = tile % w.input_tiles * kTileInputs + 32 * word + 8 * (lane >> 4);
        uint32_t fields = 0;
        for (int j = 0; j < 8; ++j)
            if (n < w.N && k + j < w.K) fields |= (uint32_t)(codes[n * w.K + k + j] & 15) << (4 * ((j >> 1) + 4 * (j & 1)));
        reinterpret_cast<uint32_t*>(const_cast<uint8_t*>(w.codes))[i] = rotate_right(fields, 30);
    } else if (i < total) {
        const long long e = i - words;
        const long long row = e >> 4, n = row / w.groups * kTileOutputs + (e & 15), g = row % w.groups;
        const int given = ceil_div(w.K, w.group);
        const bool there = n < w.N && g < given;
        const_cast<uint16_t*>(w.scales)[e] = there ? scales[n * given + g] : 0;
        if (w.has_zeros) const_cast<uint8_t*>(w.zeros)[e] = there ? zeros[n * given + g] & 15 : 0;
    }
}

// Rows as the kernels read them: whole tiles of inputs with zeros behind the last, 16-byte aligned.  HALF, for many rows: bfloat16 becomes
// float16, brought by a power of two per row to a largest magnitude of 2^14 .. 2^15: its eight bits fit, down to 2^-28 of that, and
// `factors` takes the power off again.  One workgroup per row, bound by the bytes.
template <int XT, bool HALF>
__global__ __launch_bounds__(256) void int4_rows_in_order_kernel(const typename Element<XT>::type* x, long long x_stride, typename Element<XT>::type* out,
                                                                 float* factors, int K, int padded) {
    typedef typename Element<XT>::type T;
    typedef T V __attribute__((ext_vector_type(8)));
    __shared__ float wave_largest[4];
    const T* const row = x + (long long)blockIdx.x * x_stride;
    T* const to = out + (long long)blockIdx.x * padded;
    float up = 1.0f;
    if constexpr (HALF) {
        float most = 0.0f;
        for (int k = 8 * threadIdx.x; k < K; k += 8 * 256) {
            const V v = __builtin_bit_cast(V, load_inputs<XT>(row, k, K));
#pragma unroll
            for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf((float)v[j]));
        }
#pragma unroll
        for (int step = 32; step > 0; step >>= 1) most = fmaxf(most, __shfl_xor(most, step));
        if ((threadIdx.x & 63) == 0) wave_largest[threadIdx.x >> 6] = most;
        __syncthreads();
        for (int w = 0; w < 4; ++w) most = fmaxf(most, wave_largest[w]);
        float down;
        half_powers(most, up, down);
        if (threadIdx.x == 0) factors[blockIdx.x] = down;
    }
    for (int k = 8 * threadIdx.x; k < padded; k += 8 * 256) {
        const V v = __builtin_bit_cast(V, load_inputs<XT>(row, k, K));
        if constexpr (HALF) {
            v8h h;
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = (_Float16)((float)v[j] * up);
            *reinterpret_cast<v8h*>(to + k) = h;
        } else {
            *reinterpret_cast<V*>(to + k) = v;
        }
    }
}

hipError_t launch_rows_in_order(const void* x, int x_type, bool half, long long x_stride, void* out, float* factors, int M, int K, int padded, hipStream_t s) {
    const auto run = [&](auto type, auto as_half) {
        typedef typename Element<type()>::type T;
        int4_rows_in_order_kernel<type(), as_half()><<<M, 256, 0, s>>>(static_cast<const T*>(x), x_stride, static_cast<T*>(out), factors, K, padded);
        return hipGetLastError();
    };
    if (x_type == WQ_I8) return run(std::integral_constant<int, WQ_I8>(), std::false_type());
    // without a change of type 16 bits are 16 bits
    return half ? run(std::integral_constant<int, WQ_BF16>(), std::true_type()) : run(std::integral_constant<int, WQ_F16>(), std::false_type());
}

// Adds up the parts of the inputs, in their order, four outputs a thread.
__global__ __launch_bounds__(256) void int4_join_kernel(const float* sums, int parts, Int4Weights w, Int4Output o) {
    const int quads = ceil_div(o.N, 4), i = blockIdx.x * 256 + threadIdx.x, m = i / quads, n = 4 * (i % quads);
    if (m >= o.M || !matches(w)) return;
    const size_t each = (size_t)o.M * o.N;
    const float* const from = sums + (size_t)m * o.N + n;
    v4f total = {};
#pragma unroll 4
    for (int p = 0; p < parts; ++p) total += load_unaligned<v4f, 4>(from + p * each);   // up to 12 bytes more than a row
    store_outputs(o, m, n, total, 1.0f);
}

// Which kernel a call runs, and what it needs of a workspace: a copy of the rows, and one factor each.
struct Int4Plan {
    bool many, copy;
    int parts, padded;               // parts of the inputs whose sums are added up at the end
    size_t factors, sums, total;     // offsets of the factors and of the parts' sums, and all in bytes
};
// How long either kernel takes, in us, to about a quarter (measured at 33 to 4000 rows, 16 to 30000 outputs of 32 to 28672 inputs).  For few rows:
// a workgroup to a compute unit at a time, for 16, 32 or 64 outputs of 32 rows, whose eight waves share the tiles of inputs.
double rows_time(int M, int N, int K) {
    const int tiles = ceil_div(N, kTileOutputs), blocks = ceil_div(M, 32);
    const bool wide = tiles >= kComputeUnits && (long long)blocks * tiles >= 4 * kComputeUnits;
    const long long workgroups = (long long)blocks * (wide ? ceil_div(tiles, 4) : tiles < kComputeUnits ? tiles : ceil_div(tiles, 2));
    return 2.0 + (workgroups + kComputeUnits - 1) / kComputeUnits * (2.2 + (wide ? 1.85 : 1.05) * ceil_div(ceil_div(K, kTileInputs), 8));
}
// For many: 1.2 us a tile of inputs as long as no two workgroups share a compute unit, 1.4 times that for two, which is as many as run there at
// a time; parts of the inputs are written, read again and added up by a launch more, and a copy of the rows is another.  (Their best
// number, one, and the kernel for few rows: 1661 rows, 1024 outputs of 28672 inputs 136, 317 and 808 us; 400, 4096 of 4096 31, 40 and
// 33; 256, 8192 of 8192 50, 72 and 65; but 256, 4096 of 4096 26, 40 and 20; 300, 14336 of 4096 is best in one, 55 and 76.)
double tiles_time(int M, int N, int K, int parts, bool copy) {
    const long long workgroups = (long long)ceil_div(M, kTileRows) * ceil_div(N, 8 * kTileOutputs) * parts;
    const long long deep = (workgroups + kComputeUnits - 1) / kComputeUnits;
    const double at_a_time = 1.4 * (deep / 2) + deep % 2;
    const double inputs = (double)ceil_div(ceil_div(K, kTileInputs), parts) * 1.2 * at_a_time;
    return 3.0 + inputs + (parts > 1 ? 6.0 + 1.3e-6 * parts * M * N : 0.0) + (copy ? 4.0 : 0.0);
}
constexpr int kMostParts = 32;

Int4Plan plan_int4(const void* x, int x_type, long long x_stride, int M, int N, int K) {
    Int4Plan p = {false, false, 1, ceil_div(K, kTileInputs) * kTileInputs, 0, 0, 0};
    // both kernels read whole aligned pieces of rows, the one for many rows also whole tiles only
    const bool copy = x_type == WQ_BF16 || M < kTileRows || K % kTileInputs != 0;
    if (M > 32) {
        const long long tiles = (long long)ceil_div(M, kTileRows) * ceil_div(N, 8 * kTileOutputs);
        double least = tiles_time(M, N, K, 1, copy);
        for (int parts = 2; parts <= kMostParts && 2 * parts <= ceil_div(K, kTileInputs) && tiles * parts <= 4 * kComputeUnits; ++parts) {
            const double time = tiles_time(M, N, K, parts, copy);
            if (time >= least) continue;
            least = time;
            p.parts = parts;
        }
        p.many = least < rows_time(M, N, K) || (long long)M * N > 1ll << 30;   // a launch of fewer than 2^32 threads either way
        if (!p.many) p.parts = 1;
    }
    const size_t size = x_type == WQ_I8 ? 1 : 2;
    p.copy = (M > 1 && (x_stride * size) % 16 != 0) || !aligned(x, 16) || x_stride > (1 << 24) || (p.many && copy);
    const auto whole = [](size_t bytes) { return (bytes + 255) & ~(size_t)255; };
    if (p.copy) p.factors = whole((size_t)(p.many ? max(M, kTileRows) : M) * p.padded * size);
    p.sums = p.factors + (p.many && x_type == WQ_BF16 ? whole((size_t)M * sizeof(float)) : 0);
    p.total = p.sums + (p.parts > 1 ? whole((size_t)p.parts * M * N * sizeof(float) + 12) : 0);
    return p;
}

}  // namespace

hipError_t launch_int4_pack(const uint8_t* codes, const void* scales, const uint8_t* zeros, const Int4Weights& w, uint8_t* blob, hipStream_t s) {
    const long long words = (long long)w.output_tiles * w.input_tiles * (kTileBytes / 4);
    const long long total = words + (long long)w.output_tiles * w.groups * kTileOutputs;
    int4_pack_kernel<<<(unsigned)((total + 255) / 256), 256, 0, s>>>(codes, static_cast<const uint16_t*>(scales), zeros, w, blob, words, total);
    return hipGetLastError();
}

}  // namespace wq

using namespace wq;

extern "C" {

size_t int4_packed_bytes(int N, int K, int group, int has_zeros) {
    return valid_weights(N, K, group) && !too_large(N, K) ? int4_layout(N, K, group, has_zeros != 0).total : 0;
}

int int4_pack_weights(const uint8_t* codes_dev, const void* scales_dev, int scale_type, const uint8_t* zeros_dev, int N, int K,
                      int group, void* packed_dev, size_t packed_bytes, void* hip_stream) {
    if (!codes_dev || !scales_dev || !packed_dev || !is_half(scale_type) || !valid_weights(N, K, group)) return WG_EINVAL;
    if (!aligned(scales_dev, 2) || !aligned(packed_dev, 256)) return WG_EINVAL;
    if (too_large(N, K)) return WG_EUNSUPPORTED;
    const Int4Weights w = weights_of(packed_dev, N, K, group, scale_type, zeros_dev != nullptr);
    if (packed_bytes < int4_packed_bytes(N, K, group, zeros_dev != nullptr)) return WG_ESMALLBUF;
    return status_of(launch_int4_pack(codes_dev, scales_dev, zeros_dev, w, static_cast<uint8_t*>(packed_dev), static_cast<hipStream_t>(hip_stream)));
}

size_t int4_linear_workspace_bytes(const void* x_dev, int x_type, long long x_stride, int M, int N, int K) {
    if (!(is_half(x_type) || x_type == WQ_I8) || M <= 0 || N <= 0 || K <= 0 || too_large(N, K)) return 0;
    return plan_int4(x_dev, x_type, x_stride, M, N, K).total;
}

int int4_linear(const void* x_dev, int x_type, long long x_stride, const float* x_scale_dev, const void* packed_dev,
                const float* bias_dev, void* y_dev, int y_type, int M, int N, int K, int group, int scale_type, int has_zeros,
                int relu, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    if (!packed_dev || !valid_weights(N, K, group) || !is_half(scale_type)) return WG_EINVAL;
    if (!(is_half(x_type) || x_type == WQ_I8) || !(is_half(y_type) || y_type == WQ_F32)) return WG_EINVAL;
    if (x_scale_dev && x_type != WQ_I8) return WG_EINVAL;
    if (M < 0 || x_stride < K) return WG_EINVAL;
    if (M == 0) return WG_OK;
    if (!x_dev || !y_dev) return WG_EINVAL;
    if (!aligned(packed_dev, 256) || !aligned(y_dev, y_type == WQ_F32 ? 4 : 2) || !aligned(x_dev, x_type == WQ_I8 ? 1 : 2)) return WG_EINVAL;
    if (!aligned(x_scale_dev, 4) || !aligned(bias_dev, 4)) return WG_EINVAL;
    if (too_large(N, K) || M > (1 << 23) || (long long)M * N > 1ll << 36) return WG_EUNSUPPORTED;
    const Int4Plan p = plan_int4(x_dev, x_type, x_stride, M, N, K);
    if (p.total > 0) {
        if (!workspace_dev || !aligned(workspace_dev, 256)) return WG_EINVAL;
        if (workspace_bytes < p.total) return WG_ESMALLBUF;
    }
    const Int4Weights w = weights_of(packed_dev, N, K, group, scale_type, has_zeros != 0);
    Int4Output o = {x_scale_dev, bias_dev, y_dev, y_type, M, N, relu != 0};
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (p.copy) {
        float* const factors = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + p.factors);
        if (hipError_t e = launch_rows_in_order(x_dev, x_type, p.many && x_type == WQ_BF16, x_stride, workspace_dev, factors, M, K, p.padded, s)) return status_of(e);
        x_dev = workspace_dev;
        x_stride = p.padded;
        if (p.many && x_type == WQ_BF16) o.x_scale = factors;
    }
    if (p.many) {
        const auto launch = x_type == WQ_I8 ? launch_int4_tiles_int8 : launch_int4_tiles_half;
        if (p.parts == 1) return status_of(launch(x_dev, x_stride, w, o, 1, s));
        float* const sums = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + p.sums);
        if (hipError_t e = launch(x_dev, x_stride, w, Int4Output{nullptr, nullptr, sums, WQ_F32, M, N, 0}, p.parts, s)) return status_of(e);
        int4_join_kernel<<<(unsigned)(((long long)M * ceil_div(N, 4) + 255) / 256), 256, 0, s>>>(sums, p.parts, w, o);
        return status_of(hipGetLastError());
    }
    const auto launch = x_type == WQ_F16 ? launch_int4_rows_half : x_type == WQ_BF16 ? launch_int4_rows_bfloat : launch_int4_rows_int8;
    return status_of(launch(x_dev, x_stride, w, o, s));
}

}  // extern "C"
