// The paged key/value cache: writing new tokens (with the rotation of keys and
// queries) and reading tokens back, on gfx950.
//
// Both are bound by memory; at a few tokens, by the latency of a launch.  A
// head's quantisation needs the largest magnitude of its values, which eight
// (head_dim 128) or four (64) neighbouring threads find together, sixteen
// values each, so everything is read and written once.
#include "attn.hpp"

namespace unisvq {
namespace {

constexpr int kThreads = 256;

struct Append {
    CacheView c;
    int64_t tokens;
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

// Codes of f * inv, rounded to even, in BITS bits each at an offset of half
// their range.  A sum with 1.5 * 2^23 rounds to an integer in the low bits of
// a float; the integers are put in place by adding them up shifted, and what
// the exponents add is known, so it is taken off once.  No code can pass its
// top: |f| <= a, and scale is a / top but for a rounding of 2^-9 at most, which
// is far from a half even at 127 (whose scale is rounded to 2^-24).
template <int BITS>
__device__ inline uint32_t codes(const float* f, float inv) {
#pragma clang fp contract(off)
    constexpr float kMagic = 12582912.0f + (1 << (BITS - 1));
    uint32_t b = 0, base = 0;
#pragma unroll
    for (int i = 0; i < 32 / BITS; ++i) {
        const float product = f[i] * inv;
        b += __float_as_uint(product + kMagic) << BITS * i;
        base += 0x4b400000u << BITS * i;
    }
    return b - base;
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
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float* f = i ? w : u;
            const uint2 b = {codes<8>(f, inv) ^ 0x80808080u, codes<8>(f + 4, inv) ^ 0x80808080u};
            *reinterpret_cast<uint2*>(pool + e * D + (i ? k.d1 : k.d0)) = finite ? b : uint2{0u, 0u};
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
        *reinterpret_cast<uint32_t*>(pool + e * (D / 2) + k.d0 / 2) =
            finite[hu] ? codes<4>(u, hu ? inv[1] : inv[0]) : 0x88888888u;
        *reinterpret_cast<uint32_t*>(pool + e * (D / 2) + k.d1 / 2) =
            finite[hw] ? codes<4>(w, hw ? inv[1] : inv[0]) : 0x88888888u;
        if (c == 0)
            scales[e] = (__float_as_uint(scale[0]) >> 16) | (__float_as_uint(scale[1]) & 0xffff0000u);
    }
}

// A block: one head of kThreads / LANES tokens, a thread sixteen dims.
// Neighbouring threads are neighbouring tokens of the head because that is what
// lies together in a page: a block's codes are whole lines (each of its two
// stores writes halves of the rows) and its scales are one line, where a token's
// heads side by side would leave 64-byte and 4-byte pieces to different dies'
// caches.
//
// 2048 tokens of 64 + 2 * 8 heads into 8-bit pages: 17.6 us, 4.5 TB/s; 2000
// tokens of 3 * 32 heads into 4-bit pages: 23 us, 3.2 TB/s.  In both a thread
// waits for its position and then for its table row and page; two heads a thread
// take as long, four 1-2 us longer (fewer waves fit).  What holds the 4-bit form
// below the 8-bit one is not known; its stores are of 4 bytes a lane, in 32-byte
// halves of rows of 64.
template <int KIND, int D, typename T>
__global__ __launch_bounds__(kThreads) void append_kernel(Append a) {
    constexpr int LANES = D / 16;
    const uint32_t heads = static_cast<uint32_t>(a.q_heads + 2 * a.c.heads);
    const int64_t t = static_cast<int64_t>(blockIdx.x / heads) * (kThreads / LANES) + threadIdx.x / LANES;
    if (t >= a.tokens) return;  // a head's threads leave together
    // a token's heads are those of q, then of k, then of v
    const int h = static_cast<int>(blockIdx.x % heads), c = threadIdx.x % LANES;
    const int role = h < a.q_heads ? 0 : h < a.q_heads + a.c.heads ? 1 : 2;
    const int at = h - (role == 0 ? 0 : role == 1 ? a.q_heads : a.q_heads + a.c.heads);
    const Rows& from = role == 0 ? a.q : role == 1 ? a.k : a.v;
    const int64_t pos = a.positions[t];
    const Chunk k = chunk_of(c, role != 2 && a.rotary.table ? a.rotary.rot : 0, D);
    const T* row = static_cast<const T*>(from.p) + t * from.ts + at * from.hs;
    float u[8], w[8];
    load8(row + k.d0, u);
    load8(row + k.d1, w);
    if (k.turned) {
        float cs[8], sn[8];
        if (pos >= 0 && pos < a.rotary.positions) {
            load_angles(a.rotary.table + pos * a.rotary.rot, a.rotary.rot, c, a.rotary.interleaved, cs, sn);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) cs[j] = sn[j] = __builtin_nanf("");
        }
        turn(u, w, cs, sn, a.rotary.interleaved);
    }
    if (role == 0) {
        T* y = static_cast<T*>(a.q_out.p) + t * a.q_out.ts + at * a.q_out.hs;
        store8(y + k.d0, u);
        store8(y + k.d1, w);
        return;
    }
    const int64_t page = page_of(a.c, a.seqs ? a.seqs[t] : t, pos);
    const int64_t e = page < 0 ? 0 : entry_of(a.c, page, pos, at);
    store_entry<KIND, D, T>(role == 1 ? a.c.k : a.c.v, role == 1 ? a.c.ks : a.c.vs, e, page >= 0, k, c, u, w);
}

// ---- reading back ----

// Sixteen values of entry e as they are stored: dims 8c .. 8c + 7 of both
// halves of the head, so that a head's threads write whole lines.
template <int KIND, int D>
struct Stored {
    static constexpr int kWords = KIND == UNISVQ_CACHE_I8 ? 2 : KIND == UNISVQ_CACHE_I4 ? 1 : 4;
    uint32_t b[2][kWords], scale;

    __device__ inline void load(const uint8_t* pool, const uint32_t* scales, int64_t e, int c) {
        typedef uint32_t Words __attribute__((ext_vector_type(kWords)));
        const Words* p = reinterpret_cast<const Words*>(pool) + e * (D / 8) + c;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const Words v = p[i * (D / 16)];
#pragma unroll
            for (int j = 0; j < kWords; ++j) b[i][j] = v[j];
        }
        if constexpr (kWords < 4) scale = scales[e];
    }

    __device__ inline void values(int i, float (&f)[8]) const {
        const uint32_t* x = b[i];
        if constexpr (KIND == UNISVQ_CACHE_F16) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                f[j] = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(x[j / 2] >> 16 * (j % 2))));
        } else if constexpr (KIND == UNISVQ_CACHE_BF16) {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(x[j / 2] >> 16 * (j % 2) << 16);
        } else if constexpr (KIND == UNISVQ_CACHE_I8) {
            const float s = __uint_as_float(scale);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = static_cast<float>(static_cast<int8_t>(x[j / 4] >> 8 * (j % 4))) * s;
        } else {
            const float s = __uint_as_float(i ? scale & 0xffff0000u : scale << 16);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t four = (j % 2 ? x[0] >> 4 : x[0]) & 0x0f0f0f0fu;  // its bytes convert as they are
                f[j] = (static_cast<float>(four >> 8 * (j / 2) & 255u) - 8.0f) * s;
            }
        }
    }
};

// A block: one head of kThreads / LANES rows, keys and values; neighbours as
// in append_kernel, for the same reason.  3808 rows of 32 heads out of 4-bit
// pages: 18 us, 4.7 TB/s; 16 rows of 32 heads: 4 us.
template <int KIND, int D, typename T>
__global__ __launch_bounds__(kThreads) void read_kernel(CacheView c, const int32_t* starts, const int32_t* cu,
                                                        int64_t tokens, Rows k, Rows v) {
    constexpr int LANES = D / 16;
    const uint32_t heads = static_cast<uint32_t>(c.heads);
    const int h = static_cast<int>(blockIdx.x % heads), part = threadIdx.x % LANES;
    const int64_t first = static_cast<int64_t>(blockIdx.x / heads) * (kThreads / LANES) +
                          __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (64 / LANES);
    const int64_t r = first + (threadIdx.x & 63) / LANES;
    int seq = sequence_of(cu, static_cast<int>(c.sequences), first);
    if (r >= tokens) return;
    while (seq < c.sequences && cu[seq + 1] <= r) ++seq;
    if (seq >= c.sequences) return;
    const int64_t pos = (starts ? starts[seq] : 0) + r - cu[seq];
    const int64_t page = page_of(c, seq, pos);
    Stored<KIND, D> in[2];
    if (page >= 0) {
        const int64_t e = entry_of(c, page, pos, h);
        in[0].load(c.k, c.ks, e, part);
        in[1].load(c.v, c.vs, e, part);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const Rows& to = i ? v : k;
        T* y = static_cast<T*>(to.p) + r * to.ts + h * to.hs + 8 * part;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            float f[8];
            if (page >= 0) {
                in[i].values(half, f);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = __builtin_nanf("");
            }
            store8(y + half * (D / 2), f);
        }
    }
}

// A block for each head of the rows that a block holds.
uint32_t blocks_of(int64_t tokens, int heads, int head_dim) {
    const int64_t rows = kThreads / (head_dim / 16);
    return static_cast<uint32_t>((tokens + rows - 1) / rows * heads);
}

template <int D, typename T>
hipError_t append_with(const Append& a, hipStream_t s) {
    const uint32_t blocks = blocks_of(a.tokens, a.q_heads + 2 * a.c.heads, D);
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
    const uint32_t blocks = blocks_of(tokens, c.heads, D);
    switch (c.kind) {
        case UNISVQ_CACHE_F16:
            read_kernel<UNISVQ_CACHE_F16, D, T><<<blocks, kThreads, 0, s>>>(c, starts, cu, tokens, k, v);
            break;
        case UNISVQ_CACHE_BF16:
            read_kernel<UNISVQ_CACHE_BF16, D, T><<<blocks, kThreads, 0, s>>>(c, starts, cu, tokens, k, v);
            break;
        case UNISVQ_CACHE_I8:
            read_kernel<UNISVQ_CACHE_I8, D, T><<<blocks, kThreads, 0, s>>>(c, starts, cu, tokens, k, v);
            break;
        default:
            read_kernel<UNISVQ_CACHE_I4, D, T><<<blocks, kThreads, 0, s>>>(c, starts, cu, tokens, k, v);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheView& c, int64_t tokens, const int32_t* seqs, const int32_t* positions,
                               Rows k, Rows v, Rows q, int q_heads, Rows q_out, int x_dtype, const Rotary& rotary,
                               hipStream_t s) {
    const Append a{c, tokens, seqs, positions, k, v, q, q_out, q_heads, rotary};
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
