// Attention over the cache held in 8 bits: what its kernels share.
#pragma once
#include "int8_cache.h"

namespace wq {

struct AttentionArgs {
    const void* q;
    long long q_stride;
    void* out;
    long long out_stride;
    const int8_t *k, *v;
    const float *k_scale, *v_scale;
    float* partial;   // sums of parts of the tokens, where a sequence is split
    Batch batch;
    int kv_heads, group;   // heads of queries per head of keys
    int causal, window, splits;
    float scale_log2;      // scale / ln 2: exponentials are taken to base 2
};

// Four codes as two pairs of float16, exactly: a byte with its sign bit turned is code + 128, and in the fraction of 1024 it counts
// ones.
__device__ inline void codes_to_half(uint32_t codes, v2h& low, v2h& high) {
    const uint32_t u = codes ^ 0x80808080u;
    const v2h off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    low = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) + off;
    high = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) + off;
}
__device__ inline v8h codes_to_half(uint32_t a, uint32_t b) {
    v2h r[4];
    codes_to_half(a, r[0], r[1]);
    codes_to_half(b, r[2], r[3]);
    return v8h{r[0][0], r[0][1], r[1][0], r[1][1], r[2][0], r[2][1], r[3][0], r[3][1]};
}

// The tokens that a row at `position` sees: low .. high - 1.
__device__ inline void visible(const AttentionArgs& a, int position, int length, int& low, int& high) {
    high = position < 0 ? 0 : a.causal ? min(position + 1, length) : length;
    low = a.window > 0 ? max(position - a.window + 1, 0) : 0;
}

// Exponents are lowered by the row's largest score only when it has grown by more than this (to base 2) since the last time; what is
// summed lies this much below float16's 2^16.
constexpr float kSlack = 8.0f;
constexpr float kRaise = 7.0f;

template <int TYPE>
__device__ inline void store4(void* out, long long at, v4f v) {
    typedef typename Element<TYPE>::type T;
    typedef T V __attribute__((ext_vector_type(4)));
    store_unaligned<2>(static_cast<T*>(out) + at, V{(T)v[0], (T)v[1], (T)v[2], (T)v[3]});
}

struct AttentionPlan {
    int tokens_shift;   // a tile of 16 rows holds 1 << tokens_shift of a sequence's rows, of up to 16 heads each
    int head_tiles;     // tiles of 16 that a group of heads needs
    long long items;    // tiles of rows, head tiles aside
    int splits;
    size_t workspace;
};
AttentionPlan plan_attention(int rows, int heads, int kv_heads, int head_dim, int block, int width, int sequences, bool has_starts);

hipError_t launch_attention_rows(const AttentionArgs& a, const AttentionPlan& p, int type, int head_dim, hipStream_t s);

}  // namespace wq
