// Internal declarations of the attention block: rotary positions, the paged
// cache and attention (attn_api.hip validates; rope.hip, cache.hip,
// attn_decode.hip and attn_prompt.hip launch).
#pragma once

#include <type_traits>

#include "common.hpp"

namespace unisvq {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Rows of activations: element d of head h of token t at p + t * ts + h * hs + d.
struct Rows {
    void* p;
    int64_t ts, hs;
};

struct Rotary {
    const float* table;  // [positions][2][rot / 2]; null: no rotation
    int64_t positions;
    int rot;
    int interleaved;
    int inverse;
};

// A paged cache and the page table it is looked up in.
struct CacheView {
    uint8_t *k, *v;
    uint32_t *ks, *vs;  // one 4-byte word a token and head
    const int32_t* table;
    int64_t sequences, width, pages;
    int page_shift;  // log2 of page_tokens
    int heads, head_dim, kind;
};

constexpr int entry_bits(int kind) { return kind == UNISVQ_CACHE_I8 ? 8 : kind == UNISVQ_CACHE_I4 ? 4 : 16; }

hipError_t launch_rope_table(int64_t positions, int rot, double theta, double factor, double low, double high,
                             double original, double magnitude, float* table, hipStream_t s);
hipError_t launch_rope(int64_t tokens, int heads, int head_dim, const Rotary& rotary, Rows x, const int32_t* positions,
                       Rows y, int dtype, hipStream_t s);
hipError_t launch_cache_append(const CacheView& c, int64_t tokens, const int32_t* seqs, const int32_t* positions,
                               Rows k, Rows v, Rows q, int q_heads, Rows q_out, int x_dtype, const Rotary& rotary,
                               hipStream_t s);
hipError_t launch_cache_read(const CacheView& c, const int32_t* starts, const int32_t* cu, int64_t tokens, Rows k,
                             Rows v, int dtype, hipStream_t s);

// Attention over the cache.  slots: parts that a row's work can be split into.
int decode_slots(int64_t sequences, int q_len, int q_heads, int kv_heads, int64_t max_len, int token_bytes);
size_t decode_workspace_bytes(int64_t sequences, int q_len, int q_heads, int head_dim, int slots);
hipError_t launch_attn_decode(const CacheView& c, const int32_t* lens, int64_t max_len, int slots, int q_len, int q_heads,
                              Rows q, int x_dtype, float scale, Rows out, float* lse, void* workspace, hipStream_t s);

struct PromptArgs {
    const int32_t *cu_q, *cu_k;
    int64_t sequences, q_tokens, k_tokens;
    int q_heads, kv_heads, head_dim;
    Rows q, k, v, out;
    int dtype, causal;
    float scale;
    float* lse;
};
size_t prompt_workspace_bytes(int64_t sequences, int64_t q_tokens, int64_t k_tokens, int q_heads, int kv_heads,
                              int head_dim);
hipError_t launch_attn_prompt(const PromptArgs& a, void* workspace, hipStream_t s);

// ---- device helpers ----

// A vector of eight 16-bit elements as floats and back (round to nearest even).
template <typename T>
struct Vec8;
template <>
struct Vec8<_Float16> {
    typedef f16x8 type;
};
template <>
struct Vec8<__bf16> {
    typedef bf16x8 type;
};

template <typename T>
__device__ inline void load8(const T* p, float (&f)[8]) {
    const typename Vec8<T>::type v = *reinterpret_cast<const typename Vec8<T>::type*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = static_cast<float>(v[i]);
}

template <typename T>
__device__ inline void store8(T* p, const float (&f)[8]) {
    typename Vec8<T>::type v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = static_cast<T>(f[i]);
    *reinterpret_cast<typename Vec8<T>::type*>(p) = v;
}

// Eight pairs rotated; products and sums are rounded one by one (a contracted
// product would differ from the plain formula in the last bit, and where the
// result is quantised, in a code).
__device__ inline void rotate8(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8]) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = a[i], y = b[i];
        const float xc = x * c[i], ys = y * s[i], yc = y * c[i], xs = x * s[i];
        a[i] = xc - ys;
        b[i] = yc + xs;
    }
}

// Sixteen dims of a head as one thread holds them: eight from d0 and eight from
// d1 on, so that neighbouring threads have whole lines of either half of what is
// rotated and of what is not.  Pairs are (d0 + i, d1 + i), or where the layout
// is interleaved neighbours of either run, which `turn` takes apart.
struct Chunk {
    int d0, d1;
    bool turned;  // whether they are rotated
};

__device__ inline Chunk chunk_of(int c, int rot, int head_dim) {
    Chunk k;
    k.turned = 16 * c < rot;
    k.d0 = k.turned ? 8 * c : rot + 8 * (c - rot / 16);
    k.d1 = k.d0 + (k.turned ? rot : head_dim - rot) / 2;
    return k;
}

// Cosines and sines of the chunk's pairs from a table row.
__device__ inline void load_angles(const float* row, int rot, int c, int interleaved, float (&cs)[8], float (&sn)[8]) {
    const float* lo = row + (interleaved ? 4 * c : 8 * c);
    const float* hi = row + (interleaved ? rot / 4 + 4 * c : 8 * c + 4);
    const f32x4 v[4] = {*reinterpret_cast<const f32x4*>(lo), *reinterpret_cast<const f32x4*>(hi),
                        *reinterpret_cast<const f32x4*>(lo + rot / 2), *reinterpret_cast<const f32x4*>(hi + rot / 2)};
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = v[0][i], cs[4 + i] = v[1][i], sn[i] = v[2][i], sn[4 + i] = v[3][i];
}

// Rotates a chunk's dims (u from d0, w from d1) with its cosines c and sines s.
__device__ inline void turn(float (&u)[8], float (&w)[8], const float (&c)[8], const float (&s)[8], int interleaved) {
    if (!interleaved) {
        rotate8(u, w, c, s);
        return;
    }
    float a[8], b[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = u[2 * i], b[i] = u[2 * i + 1], a[4 + i] = w[2 * i], b[4 + i] = w[2 * i + 1];
    rotate8(a, b, c, s);
#pragma unroll
    for (int i = 0; i < 4; ++i) u[2 * i] = a[i], u[2 * i + 1] = b[i], w[2 * i] = a[4 + i], w[2 * i + 1] = b[4 + i];
}

// ---- values that are not finite ----
// A product on the matrix cores takes 0 * inf and 0 * NaN to NaN, so a value
// that is not finite would reach rows that do not see it.  Where rows of a
// tile see different keys and the tile holds such values, they are added to
// the sums of the rows that see them one by one, and zeros take their places
// before the product.
template <typename T>
__device__ constexpr uint32_t exponent_bits() { return std::is_same_v<T, _Float16> ? 0x7c00u : 0x7f80u; }

// Whether one of the two values in w is not finite.
template <typename T>
__device__ inline bool not_finite(uint32_t w) {
    constexpr uint32_t e = exponent_bits<T>();
    return (w & e) == e || (w >> 16 & e) == e;
}

// Weights of 16-bit values are 2^(s - m) with m so far (log2) below the maximum
// as f16's range allows beside what scores may exceed it by (2^8): a weight keeps
// all its bits down to 2^-21 of the largest and vanishes below 2^-32.  bf16 has
// fp32's range and needs none.
template <typename T>
__device__ constexpr float weight_lift() { return std::is_same_v<T, _Float16> ? 7.0f : 0.0f; }

// w with zeros in place of what is not finite.
template <typename T>
__device__ inline uint32_t finite_only(uint32_t w) {
    constexpr uint32_t e = exponent_bits<T>();
    if ((w & e) == e) w &= 0xffff0000u;
    if ((w >> 16 & e) == e) w &= 0xffffu;
    return w;
}

// A word that no kernel running now writes, from an address that is the same in
// all lanes: by a scalar load, also where the compiler cannot see that the
// kernel's own stores leave it alone.
__device__ inline int32_t load_uniform(const int32_t* p) {
    return *(const __attribute__((address_space(4))) int32_t*)reinterpret_cast<uintptr_t>(p);
}

// Sum, or the largest (of what is not negative), over the lanes up to this one.
template <typename F>
__device__ inline int scan64(int x, F op) {
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));  // row_shr
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));  // row_bcast
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
    return x;
}
__device__ inline int scan64(int x) { return scan64(x, [](int a, int b) { return a + b; }); }
__device__ inline int scan64_max(int x) { return scan64(x, [](int a, int b) { return max(a, b); }); }

// The sequence that packed row r belongs to: the last b with cu[b] <= r, found
// by a whole wave together (64 entries a step; r is the same in all lanes).
// Returns n where r >= cu[n].
__device__ inline int sequence_of(const int32_t* cu, int n, int64_t r) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int i = 0; i < n; i += 64) {
        const bool past = i + lane < n && cu[i + lane + 1] <= r;
        const int count = __popcll(__ballot(past));
        before += count;
        if (count < 64) break;
    }
    return before;
}

}  // namespace unisvq
