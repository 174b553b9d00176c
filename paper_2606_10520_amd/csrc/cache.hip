// The paged key/value cache: writing new tokens (with the rotation of keys and
// queries) and reading tokens back, on gfx950.
//
// Both are bound by memory.  A head's quantisation needs the largest magnitude
// of its values, which eight (head_dim 128) or four (64) neighbouring threads
// find together, sixteen values each, so everything is read and written once.
#include "attn.hpp"

namespace unisvq {
namespace {

constexpr int kThreads = 256;

struct Append {
    CacheView c;
    uint32_t count;  // threads with work: tokens * heads * chunks
    const int32_t *seqs, *positions;
    Rows k, v, q, q_out;
    int q_heads;
    Rotary rotary;
};

// The place of a token: its page (or -1) and the token of that page.
__device__ inline int64_t page_of(const CacheView& c, int64_t seq, int64_t pos) {
    if (seq < 0 || seq >= c.sequences || pos < 0) return -1;
    const int64_t col = pos >> c.page_shift;
    if (col >= c.width) return -1;
    const int64_t page = c.table[seq * c.width + col];
    return page >= 0 && page < c.pages ? page : -1;
}

// Largest magnitude as the bits of |x|: ordered like the magnitudes, inf and
// NaN above them all.
__device__ inline uint32_t magnitude8(const float (&f)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
    return m;
}

template <int LANES>
__device__ inline uint32_t max_over(uint32_t m) {
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), d)));
    return m;
}

constexpr uint32_t kInfBits = 0x7f800000u;
constexpr float kSmallest = 1e-30f;

// Eight codes of f, round to even, |code| <= top.
__device__ inline void codes8(const float (&f)[8], float inv, float top, int (&q)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = static_cast<int>(fminf(fmaxf(rintf(f[i] * inv), -top), top));
}

// A token's page, token of the page and head: the index of its entry.
__device__ inline int64_t entry_of(const CacheView& c, int64_t page, int64_t pos, int head) {
    return ((page * c.heads + head) << c.page_shift) + (pos & ((int64_t{1} << c.page_shift) - 1));
}

// Store a chunk (u from dim k.d0, w from k.d1) of entry e; `lane` 0 of the
// head's threads stores the scales.  All threads of a head take part.
template <int KIND, int D, typename T>
__device__ inline void store_entry(uint8_t* pool, uint32_t* scales, int64_t e, bool write, const Chunk& k, int c,
                                   const float (&u)[8], const float (&w)[8]) {
    constexpr int LANES = D / 16;
    if constexpr (KIND == UNISVQ_CACHE_F16 || KIND == UNISVQ_CACHE_BF16) {
        if (!write) return;
        T* row = reinterpret_cast<T*>(pool) + e * D;
        store8(row + k.d0, u);
        store8(row + k.d1, w);
    } else if constexpr (KIND == UNISVQ_CACHE_I8) {
        const uint32_t m = max_over<LANES>(max(magnitude8(u), magnitude8(w)));
        const float a = __uint_as_float(m);
        const bool finite = m < kInfBits;
        const float scale = !finite ? __builtin_nanf("") : a < kSmallest ? 0.0f : a / 127.0f;
        const float inv = finite && scale > 0.0f ? 1.0f / scale : 0.0f;
        if (!write) return;
        int q[2][8];
        codes8(u, inv, 127.0f, q[0]);
        codes8(w, inv, 127.0f, q[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint2 b = {0u, 0u};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                b.x |= (finite ? static_cast<uint32_t>(q[i][j]) & 255u : 0u) << 8 * j;
                b.y |= (finite ? static_cast<uint32_t>(q[i][4 + j]) & 255u : 0u) << 8 * j;
            }
            *reinterpret_cast<uint2*>(pool + e * D + (i ? k.d1 : k.d0)) = b;
        }
        if (c == 0) scales[e] = __float_as_uint(scale);
    } else {
        // a run of eight dims lies in one half of the head
        const int hu = k.d0 >= D / 2, hw = k.d1 >= D / 2;
        const uint32_t mu = magnitude8(u), mw = magnitude8(w);
        const uint32_t m0 = max_over<LANES>(max(hu ? 0u : mu, hw ? 0u : mw));
        const uint32_t m1 = max_over<LANES>(max(hu ? mu : 0u, hw ? mw : 0u));
        float scale[2], inv[2];
        bool finite[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t m = i ? m1 : m0;
            const float a = __uint_as_float(m);
            finite[i] = m < kInfBits;
            scale[i] = !finite[i] ? __builtin_nanf("") : a < kSmallest ? 0.0f : static_cast<float>(static_cast<__bf16>(a / 7.0f));
            inv[i] = finite[i] && scale[i] > 0.0f ? 1.0f / scale[i] : 0.0f;
        }
        if (!write) return;
        int q[2][8];
        codes8(u, hu ? inv[1] : inv[0], 7.0f, q[0]);
        codes8(w, hw ? inv[1] : inv[0], 7.0f, q[1]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool fin = (i ? hw : hu) ? finite[1] : finite[0];
            uint32_t b = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) b |= (fin ? static_cast<uint32_t>(q[i][j] + 8) & 15u : 8u) << 4 * j;
            *reinterpret_cast<uint32_t*>(pool + e * (D / 2) + (i ? k.d1 : k.d0) / 2) = b;
        }
        if (c == 0)
            scales[e] = (__float_as_uint(scale[0]) >> 16) | (__float_as_uint(scale[1]) & 0xffff0000u);
    }
}

// Thread i: chunk i % chunks of a head of a token; a token's heads are those
// of q, then of k, then of v.
template <int KIND, int D, typename T>
__global__ __launch_bounds__(kThreads) void append_kernel(Append a) {
    constexpr int LANES = D / 16;
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= a.count) return;  // count is a multiple of LANES: a head's threads leave together
    const uint32_t heads = a.q_heads + 2 * a.c.heads;
    const int c = i % LANES;
    const uint32_t th = i / LANES, t = th / heads;
    int h = th % heads;
    const int64_t pos = a.positions[t];
    const int role = h < a.q_heads ? 0 : h < a.q_heads + a.c.heads ? 1 : 2;
    h -= role == 0 ? 0 : role == 1 ? a.q_heads : a.q_heads + a.c.heads;
    const Rows& from = role == 0 ? a.q : role == 1 ? a.k : a.v;
    Chunk k = chunk_of(c, role == 2 || !a.rotary.table ? 0 : a.rotary.rot, a.rotary.interleaved);
    const T* x = static_cast<const T*>(from.p) + t * from.ts + h * from.hs;
    float u[8], w[8];
    load8(x + k.d0, u);
    load8(x + k.d1, w);
    if (k.turned) {
        float cs[8], sn[8];
        if (pos >= 0 && pos < a.rotary.positions) {
            const float* row = a.rotary.table + pos * a.rotary.rot + 8 * c;
            load8(row, cs);
            load8(row + a.rotary.rot / 2, sn);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) cs[j] = sn[j] = __builtin_nanf("");
        }
        turn(u, w, cs, sn, a.rotary.interleaved);
    }
    if (role == 0) {
        T* y = static_cast<T*>(a.q_out.p) + t * a.q_out.ts + h * a.q_out.hs;
        store8(y + k.d0, u);
        store8(y + k.d1, w);
        return;
    }
    const int64_t page = page_of(a.c, a.seqs ? a.seqs[t] : static_cast<int64_t>(t), pos);
    const int64_t e = entry_of(a.c, page < 0 ? 0 : page, pos < 0 ? 0 : pos, h);
    store_entry<KIND, D, T>(role == 1 ? a.c.k : a.c.v, role == 1 ? a.c.ks : a.c.vs, e, page >= 0, k, c, u, w);
}

// ---- reading back ----

// Sixteen values, dims 16c .. 16c + 15, of entry e.
template <int KIND, int D, typename T>
__device__ inline void load_entry(const uint8_t* pool, const uint32_t* scales, int64_t e, int c, float (&u)[8],
                                  float (&w)[8]) {
    if constexpr (KIND == UNISVQ_CACHE_F16 || KIND == UNISVQ_CACHE_BF16) {
        typedef std::conditional_t<KIND == UNISVQ_CACHE_F16, _Float16, __bf16> P;
        const P* row = reinterpret_cast<const P*>(pool) + e * D + 16 * c;
        load8(row, u);
        load8(row + 8, w);
    } else if constexpr (KIND == UNISVQ_CACHE_I8) {
        const uint4 b = *reinterpret_cast<const uint4*>(pool + e * D + 16 * c);
        const float scale = __uint_as_float(scales[e]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u[j] = static_cast<float>(static_cast<int8_t>(b.x >> 8 * j)) * scale;
            u[4 + j] = static_cast<float>(static_cast<int8_t>(b.y >> 8 * j)) * scale;
            w[j] = static_cast<float>(static_cast<int8_t>(b.z >> 8 * j)) * scale;
            w[4 + j] = static_cast<float>(static_cast<int8_t>(b.w >> 8 * j)) * scale;
        }
    } else {
        const uint2 b = *reinterpret_cast<const uint2*>(pool + e * (D / 2) + 8 * c);
        const uint32_t both = scales[e];
        const float scale = __uint_as_float(16 * c < D / 2 ? both << 16 : both & 0xffff0000u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u[j] = static_cast<float>(static_cast<int>(b.x >> 4 * j & 15u) - 8) * scale;
            w[j] = static_cast<float>(static_cast<int>(b.y >> 4 * j & 15u) - 8) * scale;
        }
    }
}

// A wave reads rows one after the other, all heads of a row together: the
// row's place is the same for all its lanes.
constexpr int kRowsPerWave = 2;

template <int KIND, int D, typename T>
__global__ __launch_bounds__(kThreads) void read_kernel(CacheView c, const int32_t* starts, const int32_t* cu,
                                                        int64_t tokens, Rows k, Rows v) {
    constexpr int LANES = D / 16;
    const int lane = threadIdx.x & 63;
    const int64_t first = (static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6)) * kRowsPerWave;
    for (int64_t r = first; r < first + kRowsPerWave && r < tokens; ++r) {
        const int seq = sequence_of(cu, static_cast<int>(c.sequences), r);
        if (seq >= c.sequences) return;
        const int64_t pos = (starts ? starts[seq] : 0) + r - cu[seq];
        const int64_t page = page_of(c, seq, pos);
        for (int i = lane; i < 2 * c.heads * LANES; i += 64) {
            const int h2 = i / LANES, part = i % LANES;
            const bool key = h2 < c.heads;
            const int h = key ? h2 : h2 - c.heads;
            float u[8], w[8];
            if (page >= 0) {
                load_entry<KIND, D, T>(key ? c.k : c.v, key ? c.ks : c.vs, entry_of(c, page, pos, h), part, u, w);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = w[j] = __builtin_nanf("");
            }
            const Rows& to = key ? k : v;
            T* y = static_cast<T*>(to.p) + r * to.ts + h * to.hs + 16 * part;
            store8(y, u);
            store8(y + 8, w);
        }
    }
}

template <int D, typename T>
hipError_t append_with(const Append& a, hipStream_t s) {
    const uint32_t blocks = (a.count + kThreads - 1) / kThreads;
    switch (a.c.kind) {
        case UNISVQ_CACHE_I8: append_kernel<UNISVQ_CACHE_I8, D, T><<<blocks, kThreads, 0, s>>>(a); break;
        case UNISVQ_CACHE_I4: append_kernel<UNISVQ_CACHE_I4, D, T><<<blocks, kThreads, 0, s>>>(a); break;
        default:  // a 16-bit kind is the activations' own
            append_kernel<UNISVQ_CACHE_F16, D, T><<<blocks, kThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

template <int D, typename T>
hipError_t read_with(const CacheView& c, const int32_t* starts, const int32_t* cu, int64_t tokens, Rows k, Rows v,
                     hipStream_t s) {
    const int64_t per = kThreads / 64 * kRowsPerWave;
    const uint32_t blocks = static_cast<uint32_t>((tokens + per - 1) / per);
    switch (c.kind) {
        case UNISVQ_CACHE_F16: read_kernel<UNISVQ_CACHE_F16, D, T><<<blocks, kThreads, 0, s>>>(c, starts, cu, tokens, k, v); break;
        case UNISVQ_CACHE_BF16: read_kernel<UNISVQ_CACHE_BF16, D, T><<<blocks, kThreads, 0, s>>>(c, starts, cu, tokens, k, v); break;
        case UNISVQ_CACHE_I8: read_kernel<UNISVQ_CACHE_I8, D, T><<<blocks, kThreads, 0, s>>>(c, starts, cu, tokens, k, v); break;
        default: read_kernel<UNISVQ_CACHE_I4, D, T><<<blocks, kThreads, 0, s>>>(c, starts, cu, tokens, k, v);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheView& c, int64_t tokens, const int32_t* seqs, const int32_t* positions,
                               Rows k, Rows v, Rows q, int q_heads, Rows q_out, int x_dtype, const Rotary& rotary,
                               hipStream_t s) {
    Append a{c, static_cast<uint32_t>(tokens * (q_heads + 2 * c.heads) * (c.head_dim / 16)), seqs, positions, k, v, q,
             q_out, q_heads, rotary};
    if (c.head_dim == 128)
        return x_dtype == UNISVQ_F16 ? append_with<128, _Float16>(a, s) : append_with<128, __bf16>(a, s);
    return x_dtype == UNISVQ_F16 ? append_with<64, _Float16>(a, s) : append_with<64, __bf16>(a, s);
}

hipError_t launch_cache_read(const CacheView& c, const int32_t* starts, const int32_t* cu, int64_t tokens, Rows k,
                             Rows v, int dtype, hipStream_t s) {
    if (c.head_dim == 128)
        return dtype == UNISVQ_F16 ? read_with<128, _Float16>(c, starts, cu, tokens, k, v, s)
                                   : read_with<128, __bf16>(c, starts, cu, tokens, k, v, s);
    return dtype == UNISVQ_F16 ? read_with<64, _Float16>(c, starts, cu, tokens, k, v, s)
                               : read_with<64, __bf16>(c, starts, cu, tokens, k, v, s);
}

}  // namespace unisvq
