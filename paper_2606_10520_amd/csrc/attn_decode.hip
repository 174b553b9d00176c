// Attention of a few new tokens per sequence over a paged cache, on gfx950.
//
//   s_t = scale (q . k_t),  p_t = exp(s_t - m),  out = sum_t p_t v_t / sum_t p_t
//
// Bound: HBM (keys and values are read for two products of at most sixteen rows:
// once where the new tokens times the heads that share a key head are sixteen or
// fewer, else once for every sixteen of them).  So nothing is staged: a wave
// reads 32 tokens at a time
// straight into the registers that the matrix cores take their operands from,
// and the products are arranged so that this works without moving data
// between lanes:
//   S^T = K Q^T   (16 tokens x 16 query rows): lane (i, g) = (lane % 16,
//                 lane / 16) holds dims of token i; the order of the dims
//                 along the product's inner axis is free, so each kind takes
//                 the order in which 16 bytes of a token's row come.
//   O^T = V^T P^T (16 dims x 16 query rows, 32 tokens inner): the result of
//                 the first product leaves lane (i, g) with tokens 4g .. 4g+3
//                 of query i, and the inner order of the second is chosen to
//                 be just that: V comes as, for each of these tokens, D/16
//                 consecutive dims a lane; row i of dim tile e is dim (D/16) i + e,
//                 and pairs of tokens are put together by byte permutes.
// Query rows are the q_len tokens of the q_heads / kv_heads heads that share a
// key head.
//
// Codes.  A byte u in the low bits of an f16 is the (subnormal) number u 2^-24,
// a nibble in bits 6 to 9 u 2^-18, exactly, and the matrix cores multiply
// subnormals too.  So codes become operands with a mask or a byte permute each,
// without arithmetic: u = code + 128 (i8, the sign bit turned) or code + 8
// (i4).  The bias is taken off sums, not elements: the scores start from -bias
// sum(q), and the values' sums lose bias sum(p), which one more product with a
// constant keeps.  (A sum's last bit is that of its largest product as if its
// subnormal factor had all its bits: what is lost of 24 bits are the zeros
// before u, two or three for bytes, one for nibbles; with nibbles in bits 0 to
// 3, one operation a word less, seven were, and it showed in the results.)  The keys' scales multiply the scores and the
// values' scales the weights, both in fp32; queries are scaled by a power of
// two into f16's range.
//
// Work.  An item is a sequence's rows on one key head (sixteen of them), in
// units of 128 tokens.  The units of all items are dealt out evenly, so that a
// ragged batch loads the GPU as evenly as one of equal lengths; the lengths are
// on the device, so every workgroup finds its share by a scan over them.  There
// are as many workgroups as the GPU holds at once, two a CU, since one costs
// about what three units do before it has its first tile (16 x 8192 tokens of
// 8-bit cache, 8 heads: 512 workgroups 53 us, 768 62 us, 1024 59 us; 16 ragged
// sequences up to 8192 tokens: 24 us, 43 us where each was cut into as many
// parts).  Where a share of up to two units more allows it, items are rounded up
// to whole shares, so that no workgroup has parts of two, which costs it a start
// more (the 16 ragged sequences 22 us for 24, 32 up to 4096 tokens 25 for 33;
// batches of equal lengths lose 0.4 us to the search).  Else a share may begin
// and end within items.  An item within one share is finished there, others are
// joined by a second launch.  Short sequences are not split (form_of).
// A workgroup's four waves take every fourth 32-token tile of its part of an
// item, the next tile's loads under way while one is computed, each with its
// own running maximum m, sum and outputs, joined through LDS.  m is raised only
// when a score exceeds it by 2^8 (the weights then stay inside f16), so most tiles
// need no exchange between lanes and no rescaling.
//
// Measured a call among others, with the launch that joins: 4 x 32768 tokens of
// 4-bit cache, 32 heads, 117 us (4.9 TB/s); 4 x 16384 of 8-bit 94 us (5.9 TB/s);
// 4 x 8192 of f16 87 us (6.1 TB/s), where a plain read has 7.1 TB/s: the order is
// that of the bytes that a wave has under way, a tile of 4.5, 8 or 16 KB.  Rows
// beyond sixteen: 16 x 8192 tokens of 8-bit cache, 64 heads on 8, 53 us for one
// new token and 97 us for four, whose 32 rows read everything twice.  One sequence
// of 1001 tokens of f16, 32 heads: launches of 8.5 and 3.9 us, in the first 1 us to
// find the share, 2.6 until the queries and the first tile are there, 1.4 for a
// tile, 0.8 to join the waves; 512 tokens 9.0 us, one launch with whole items.
#include <algorithm>
#include <cfloat>

#include "attn_join.hpp"

namespace unisvq {
namespace {

constexpr int kWaves = 4, kTile = 32, kRows = 16;
constexpr int kUnit = kWaves * kTile;  // tokens
constexpr int kGrid = 512;             // workgroups at most: what the GPU holds at once, two a CU
constexpr int kSlots = 66;             // parts of a row at most, of which two are not whole shares
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kSlack = 8.0f;  // log2 of how far scores may exceed the running maximum
// For codes (see Running): a bound of the sum of a tile's 32 operands, so that
// none passes f16's range and one of at least 2^10 is there where it is passed;
// and (log2) where the largest one starts, how far apart halves may share a unit,
// bounds of units.
constexpr int kLarge = 24;  // log2 of what scores of very large queries on codes are times besides
constexpr float kMostSum = 0x1p15f, kAim = 4.0f, kApart = 6.0f, kMostUnit = 95.0f, kLeastShift = -60.0f;

struct Decode {
    CacheView c;
    const int32_t* lens;
    Rows q, out;
    float* lse;
    float* part;      // [rows][slots][D] sums, where slots > 1
    float2* part_ml;  // [rows][slots] maximum (log2) and sum
    int32_t* before;  // [sequences + 1] (rounded) units of an item of the sequences before, and the share after them
    int slots;        // parts a row can have; 1: a workgroup has an item
    int q_len, q_heads, group, row_tiles;
    float scale;      // of the scores, times log2 e
};

__device__ inline f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }

// Nibbles of w in the order 0 4 1 5 2 6 3 7, as u 2^-18.
__device__ inline u32x4 nibbles(uint32_t w) {
    const uint32_t m = 0x03c003c0u;
    return u32x4{w << 6 & m, w << 2 & m, w >> 2 & m, w >> 6 & m};
}

// What a lane reads of 16 tokens' keys (K) and of one token's values (V).
template <int KIND, int D>
struct Geometry {
    static constexpr int bits = entry_bits(KIND);
    static constexpr int row = D * bits / 8;      // bytes of an entry
    static constexpr int E = D / 16;              // dims of a token's values a lane holds
    static constexpr int vbytes = E * bits / 8;   // 2, 4, 8 or 16
    static constexpr int kword = bits == 16 || bits == 8 ? 16 : D / 16;  // bytes a key load: 16, or 8 / 4 (half a head of 4-bit codes over 4 lanes)
    static constexpr int kloads = row / (4 * kword);
    static constexpr bool scaled = bits < 16;
    static constexpr int halves = bits == 4 ? 2 : 1;  // scales of a head
    static constexpr uint32_t bias = bits == 4 ? 8 << 6 : 128;  // as an operand's bits
    static constexpr float unit = bits == 4 ? 0x1p18f : 0x1p24f;  // what operands are to be times for their codes
};

template <int BYTES>
struct Word;
template <> struct Word<16> { typedef u32x4 type; };
template <> struct Word<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };

template <int KIND, int D>
struct TileRegs {
    typedef Geometry<KIND, D> G;
    typename Word<G::kword>::type k[2][G::kloads];
    typename Word<G::vbytes>::type v[2][4];
    u32x4 ks[2], vs[2];  // the scale words of tokens 4g .. 4g + 3
    bool there[2];       // whether the 16 tokens have a page (the same in all lanes)
};

template <typename T>
__device__ inline T load_stream(const uint8_t* p) { return __builtin_nontemporal_load(reinterpret_cast<const T*>(p)); }

// The pages of the 16 tokens from p and from p + 16 on, -1 where there is none.
struct Pages {
    int at[2];
};
__device__ inline Pages look_up(const Decode& a, const int32_t* row, int p, int len) {
    Pages r;
#pragma unroll
    for (int t = 0; t < 2; ++t) r.at[t] = p + 16 * t < len ? load_uniform(row + ((p + 16 * t) >> a.c.page_shift)) : -1;
    return r;
}

template <int KIND, int D>
__device__ __forceinline__ void load_tile(const Decode& a, const Pages& pages, int h, int pos, int i, int g, TileRegs<KIND, D>& r) {
    typedef Geometry<KIND, D> G;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int p = pos + 16 * t;
        int64_t page = pages.at[t];
        r.there[t] = page >= 0 && page < a.c.pages;
        if (!r.there[t]) page = 0;
        const int64_t e = ((page * a.c.heads + h) << a.c.page_shift) + (p & ((1 << a.c.page_shift) - 1));
        const uint8_t* kp = a.c.k + e * G::row;
        const uint8_t* vp = a.c.v + e * G::row;
#pragma unroll
        for (int n = 0; n < G::kloads; ++n)
            r.k[t][n] = load_stream<typename Word<G::kword>::type>(kp + (i * G::row + n * 4 * G::kword + g * G::kword));
        if constexpr (G::scaled) r.ks[t] = *reinterpret_cast<const u32x4*>(a.c.ks + e + 4 * g);
#pragma unroll
        for (int n = 0; n < 4; ++n)
            r.v[t][n] = load_stream<typename Word<G::vbytes>::type>(vp + ((4 * g + n) * G::row + i * G::vbytes));
        if constexpr (G::scaled) r.vs[t] = *reinterpret_cast<const u32x4*>(a.c.vs + e + 4 * g);
    }
}

// The dims of query operand step n for lane group g: eight from first on, in
// natural order or as nibbles() has them.
template <int KIND, int D>
__device__ inline int query_dim(int n, int g) {
    if constexpr (KIND == UNISVQ_CACHE_I8) return 64 * (n / 2) + 16 * g + 8 * (n % 2);
    if constexpr (KIND == UNISVQ_CACHE_I4) return (n / (D / 64)) * (D / 2) + g * (D / 8) + 8 * (n % (D / 64));
    return 32 * n + 8 * g;
}

// Scores of 16 tokens (without scales; one sum for each half of the head where
// the scales differ), from `start`.
template <int KIND, int D, typename C8>
__device__ __forceinline__ void scores16(const TileRegs<KIND, D>& r, int t, const C8 (&q)[D / 32],
                                         const float (&start)[Geometry<KIND, D>::halves], f32x4 (&s)[Geometry<KIND, D>::halves]) {
#pragma unroll
    for (int h = 0; h < Geometry<KIND, D>::halves; ++h) s[h] = f32x4{start[h], start[h], start[h], start[h]};
    if constexpr (KIND == UNISVQ_CACHE_I8) {
#pragma unroll
        for (int n = 0; n < D / 32; ++n) {
            const uint32_t w0 = r.k[t][n / 2][2 * (n % 2)] ^ 0x80808080u, w1 = r.k[t][n / 2][2 * (n % 2) + 1] ^ 0x80808080u;
            const u32x4 a = {perm(0, w0, 0x0c010c00u), perm(0, w0, 0x0c030c02u), perm(0, w1, 0x0c010c00u), perm(0, w1, 0x0c030c02u)};
            s[0] = mfma(__builtin_bit_cast(C8, a), q[n], s[0]);
        }
    } else if constexpr (KIND == UNISVQ_CACHE_I4) {
#pragma unroll
        for (int n = 0; n < D / 32; ++n) {
            constexpr int per = D / 64;
            uint32_t w;
            if constexpr (per == 2) w = r.k[t][n / per][n % per];
            else w = r.k[t][n];
            s[n / per] = mfma(__builtin_bit_cast(C8, nibbles(w)), q[n], s[n / per]);
        }
    } else {
#pragma unroll
        for (int n = 0; n < D / 32; ++n) s[0] = mfma(__builtin_bit_cast(C8, r.k[t][n]), q[n], s[0]);
    }
}

// 32-bit word w of a lane's values of one token.
template <int KIND, int D>
__device__ inline uint32_t vword(const TileRegs<KIND, D>& r, int t, int n, int w) {
    if constexpr (Geometry<KIND, D>::vbytes <= 4) return r.v[t][n];
    else return r.v[t][n][w];
}

// The A operand of dim tile e: dim (D/16) i + e of the lane's eight tokens.
template <int KIND, int D, typename C8>
__device__ __forceinline__ void value_operands(const TileRegs<KIND, D>& r, C8 (&v)[D / 16]) {
    constexpr int E = D / 16;
    uint32_t w[E][4];  // [dim][token pair]
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < 4; n += 2) {
            const int pair = 2 * t + n / 2;
            if constexpr (KIND == UNISVQ_CACHE_I8) {
#pragma unroll
                for (int x = 0; x < E / 4; ++x) {
                    const uint32_t a = vword<KIND, D>(r, t, n, x) ^ 0x80808080u, b = vword<KIND, D>(r, t, n + 1, x) ^ 0x80808080u;
                    w[4 * x + 0][pair] = perm(b, a, 0x0c040c00u);
                    w[4 * x + 1][pair] = perm(b, a, 0x0c050c01u);
                    w[4 * x + 2][pair] = perm(b, a, 0x0c060c02u);
                    w[4 * x + 3][pair] = perm(b, a, 0x0c070c03u);
                }
            } else if constexpr (KIND == UNISVQ_CACHE_I4) {
                const uint32_t a = vword<KIND, D>(r, t, n, 0), b = vword<KIND, D>(r, t, n + 1, 0);
#pragma unroll
                for (int x = 0; x < E / 4; ++x) {
                    const uint32_t both = perm(b, a, x ? 0x07060302u : 0x05040100u);  // four nibbles of each token
                    const u32x4 d = nibbles(both);
#pragma unroll
                    for (int y = 0; y < 4; ++y) w[4 * x + y][pair] = d[y];
                }
            } else {
#pragma unroll
                for (int x = 0; x < E / 2; ++x) {
                    const uint32_t a = vword<KIND, D>(r, t, n, x), b = vword<KIND, D>(r, t, n + 1, x);
                    w[2 * x][pair] = perm(b, a, 0x05040100u);
                    w[2 * x + 1][pair] = perm(b, a, 0x07060302u);
                }
            }
        }
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = __builtin_bit_cast(C8, u32x4{w[e][0], w[e][1], w[e][2], w[e][3]});
}

// Adds the tile's values that are not finite to the sums of the rows that see
// them, and puts zeros in their places (see not_finite).
template <int KIND, int D, typename CT>
__device__ inline void only_where_seen(TileRegs<KIND, D>& r, int pos, int limit, int g, f32x4 (&o)[D / 16]) {
    constexpr int words = D / 32;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int x = 0; x < words; ++x) {
                const uint32_t w = vword<KIND, D>(r, t, n, x);
                uint64_t left = __ballot(not_finite<CT>(w));
                while (left) {  // rare
                    const int lane = __ffsll(static_cast<unsigned long long>(left)) - 1;
                    left &= left - 1;
                    const uint32_t both = __builtin_amdgcn_readlane(w, lane);
                    const bool mine = (lane & 15) >> 2 == g && pos + 16 * t + 4 * (lane >> 4) + n < limit;
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const uint16_t bits = static_cast<uint16_t>(both >> 16 * y);
                        const float add = mine && (bits & exponent_bits<CT>()) == exponent_bits<CT>()
                                              ? static_cast<float>(__builtin_bit_cast(CT, bits)) : 0.0f;
#pragma unroll
                        for (int c = 0; c < 4; ++c) o[2 * x + y][c] += (lane & 3) == c ? add : 0.0f;
                    }
                }
                r.v[t][n][x] = finite_only<CT>(w);
            }
}

__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The scale of a token in half h of the head.
template <int KIND>
__device__ inline float scale_of(uint32_t word, int h) {
    if constexpr (KIND == UNISVQ_CACHE_I4) return __uint_as_float(h ? word & 0xffff0000u : word << 16);
    return __uint_as_float(word);
}

// A scale word times a factor each; what is finite stays finite.
template <int KIND, int HV>
__device__ inline uint32_t scaled_word(uint32_t word, const float (&factor)[2]) {
    uint32_t half[HV];
#pragma unroll
    for (int x = 0; x < HV; ++x) {
        const float was = scale_of<KIND>(word, x), is = was * factor[x];
        half[x] = is == INFINITY && was < INFINITY ? 0x7f7f0000u : __float_as_uint(is);
    }
    if constexpr (KIND == UNISVQ_CACHE_I4) return half[0] >> 16 | (half[HV - 1] & 0xffff0000u);
    return half[0];
}

// One wave's running result.  Weights are 2^(s - m + shift), l their sum.  o: the
// sums of the values' codes times operands; for codes these are the weights
// times the values' scales in f16, in a unit 2^u that is the half of the head's
// own.  u follows from the row's own products weight * scale, whatever scales
// there are and whatever the row does not see: the largest one starts at 2^kAim
// and may grow to 2^10 and more.  A f16 has all its bits down to 2^-14 and some
// down to 2^-25.  u is lowered where a tile's operands sum up to 2^15 (which the
// product for the bias shows), and raised with m and as much, so that o stays.
// The weights' shift is the lower u, which costs nothing; the other half has it
// too while they are 2^kApart or less apart, else its scales are multiplied (as
// all are below kLeastShift, where l would lose weights; kMostUnit keeps l in
// range).  Beside units set by the largest scale met, which lost what a row
// sees to a token of large scale and no weight, 8-bit caches take as long and
// 4-bit ones 1 to 2.5% longer (16 x 8192 tokens 40.2 us for 39.1).
template <int KIND, int D, typename CT>
struct Running {
    typedef Geometry<KIND, D> G;
    typedef typename Vec8<CT>::type C8;
    static constexpr int E = D / 16, HV = G::halves;
    static constexpr float lift = G::scaled ? 0.0f : weight_lift<CT>();
    C8 q[D / 32];
    float start[HV];       // of the scores
    float qscale;          // of the scores to log2 units
    float m, l;
    float u[HV];           // units (log2, whole numbers) that the halves ask for
    bool apart;            // whether scales of a lane are multiplied (the same in all lanes)
    bool large = false;    // whether scores are times 2^kLarge besides (the same in all lanes)
    f32x4 o[HV][E];
    float b[HV];           // sums of the operands times the bias
    int seen;              // tokens below it are seen by the lane's row

    __device__ __forceinline__ float least() const { return HV == 1 ? u[0] : fminf(u[0], u[HV - 1]); }
    __device__ __forceinline__ float shift() const { return G::scaled ? fmaxf(least(), kLeastShift) : 0.0f; }
    // The unit that half x of o has.
    __device__ __forceinline__ float used(int x) const { return HV > 1 && u[x] - least() > kApart ? u[x] : least(); }

    __device__ __forceinline__ void begin() {
        m = -FLT_MAX;
        l = 0.0f;
        apart = large;
#pragma unroll
        for (int x = 0; x < HV; ++x) {
            u[x] = kMostUnit;
#pragma unroll
            for (int e = 0; e < E; ++e) o[x][e] = f32x4{0, 0, 0, 0};
            b[x] = 0.0f;
        }
    }

    // Changes the units, where m has risen by `up`.
    __device__ __forceinline__ void set_units(const float (&to)[HV], float up) {
        float was[HV];
        const float shift_was = shift();
#pragma unroll
        for (int x = 0; x < HV; ++x) was[x] = used(x);
#pragma unroll
        for (int x = 0; x < HV; ++x) u[x] = to[x];
        l *= exp2_(shift() - shift_was - up);
        bool far = false;
#pragma unroll
        for (int x = 0; x < HV; ++x) {
            const float c = exp2_(used(x) - was[x] - up);
            far = far || used(x) != shift();
            b[x] *= c;
#pragma unroll
            for (int e = 0; e < E; ++e) o[x][e] *= c;
        }
        apart = large || __any(far);
    }

    // Raises the maximum (`top`: the lane's largest score of the tile) and finds
    // new units, where an operand would be 2^10 or more and where the row has none.
    __device__ __forceinline__ void renew(const float (&s)[2][4], float top, TileRegs<KIND, D>& r) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m2 = fmaxf(m, top - lift), up = m2 - m;
        if constexpr (G::scaled) {
            float to[HV];
#pragma unroll
            for (int x = 0; x < HV; ++x) {
                float largest = 0.0f;  // product, of those that are finite, times 2^-16
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const float p = exp2_(__builtin_fmaf(s[t][n], qscale, -m2)) * (scale_of<KIND>(r.vs[t][n], x) * 0x1p-16f);
                        largest = fmaxf(largest, p < INFINITY ? p : 0.0f);
                    }
                largest = fmaxf(largest, __shfl_xor(largest, 16));
                largest = fmaxf(largest, __shfl_xor(largest, 32));
                const float log = static_cast<float>(static_cast<int>(__float_as_uint(largest) >> 23) - 127 + 16);
                to[x] = fminf(u[x] + floorf(up), kMostUnit);
                if (m == -FLT_MAX || log + to[x] >= 10.0f) to[x] = fminf(kAim - log, kMostUnit);
            }
            m = m2;
            set_units(to, up);
            if (apart) {
                const float factor[2] = {exp2_(used(0) - shift()), exp2_(used(HV - 1) - shift())};
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int n = 0; n < 4; ++n) r.vs[t][n] = scaled_word<KIND, HV>(r.vs[t][n], factor);
            }
        } else {
            const float c = exp2_(-up);
            m = m2;
            l *= c;
#pragma unroll
            for (int e = 0; e < E; ++e) o[0][e] *= c;
        }
    }
};

template <int KIND, int D, typename CT>
__device__ __forceinline__ void attend(const Decode& a, TileRegs<KIND, D>& r, int pos, int len, int g, Running<KIND, D, CT>& w) {
    typedef Geometry<KIND, D> G;
    typedef typename Vec8<CT>::type C8;
    constexpr int E = G::E, HV = G::halves;
    float s[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        f32x4 acc[HV];
        scores16<KIND, D>(r, t, w.q, w.start, acc);
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            if constexpr (KIND == UNISVQ_CACHE_I4)
                s[t][n] = acc[0][n] * scale_of<KIND>(r.ks[t][n], 0) + acc[HV - 1][n] * scale_of<KIND>(r.ks[t][n], 1);
            else if constexpr (KIND == UNISVQ_CACHE_I8)
                s[t][n] = acc[0][n] * scale_of<KIND>(r.ks[t][n], 0);
            else
                s[t][n] = acc[0][n];
        }
    }
    // whether all 32 tokens are seen by all rows
    const bool full = pos + kTile <= len - a.q_len + 1 && r.there[0] && r.there[1];
    if (!full) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int p = pos + 16 * t + 4 * g + n;
                if (!(p < w.seen && r.there[t])) {
                    s[t][n] = -INFINITY;
                    if constexpr (G::scaled) r.vs[t][n] = 0;  // (the lane's copy, which serves its row alone)
                }
                // what no row sees may hold anything
                if constexpr (!G::scaled)
                    if (!(p < len && r.there[t])) r.v[t][n] = {};
            }
    }
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int n = 0; n < 4; ++n) top = fmaxf(top, s[t][n]);
    top *= w.qscale;
    C8 p[HV], values[E];
    float sum;
    f32x4 bias[HV];  // the operands' sum times the codes' bias, in all four
#pragma nounroll
    for (bool again = false;; again = true) {
        const bool renew = again || (G::scaled && w.apart) || __any(top > w.m + (kSlack + w.lift));
        if (renew) {
            if (G::scaled && w.large) {  // (then every tile comes here, and once)
                top *= ldexpf(1.0f, kLarge);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int n = 0; n < 4; ++n) s[t][n] *= ldexpf(1.0f, kLarge);
            }
            w.renew(s, top, r);
        }
        const float m = w.m - w.shift();
        sum = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float v = exp2_(__builtin_fmaf(s[t][n], w.qscale, -m));
                sum += v;
#pragma unroll
                for (int x = 0; x < HV; ++x)
                    p[x][4 * t + n] = static_cast<CT>(G::scaled ? v * scale_of<KIND>(r.vs[t][n], x) : v);
            }
        if constexpr (!G::scaled) break;
        constexpr uint32_t word = G::bias | G::bias << 16;
        bool over = false;
#pragma unroll
        for (int x = 0; x < HV; ++x) {
            bias[x] = mfma(__builtin_bit_cast(C8, u32x4{word, word, word, word}), p[x], f32x4{0, 0, 0, 0});
            over = over || bias[x][0] > static_cast<float>(G::bias) * 0x1p-24f * kMostSum;
        }
        value_operands<KIND, D>(r, values);
        if (renew || !__any(over)) break;
    }
    w.l += sum;
    if constexpr (!G::scaled) {  // codes are finite, and a scale that is not is the weight's matter
        if (!full && a.q_len > 1) only_where_seen<KIND, D, CT>(r, pos, w.seen, g, w.o[0]);
    }
    if constexpr (!G::scaled) value_operands<KIND, D>(r, values);
#pragma unroll
    for (int x = 0; x < HV; ++x) {
        if constexpr (G::scaled) w.b[x] += bias[x][0];
#pragma unroll
        for (int e = 0; e < E; ++e) w.o[x][e] = mfma(values[e], p[x], w.o[x][e]);
    }
}

// Units of a sequence's items: one also where there is nothing to see (its rows
// are to become zeros).
__device__ inline int units_of(int len) { return max(1, (len + kUnit - 1) / kUnit); }

__device__ inline int padded(int units, int pad) { return pad == 1 ? units : (units + pad - 1) / pad * pad; }

__device__ inline int length_of(const Decode& a, int64_t b) {
    const int64_t room = a.c.width << a.c.page_shift;
    return static_cast<int>(min(static_cast<int64_t>(max(0, a.lens[b])), room));
}

// Units begin .. end - 1 of item (b, hr), for sequences of length len.  `slot`:
// of the part, or -1 where the item is all here.
template <int KIND, int D, typename XT, int WAVES>
__device__ __forceinline__ void attend_item(const Decode& a, int b, int hr, int len, int begin, int end, int slot, int wave, int lane) {
    typedef Geometry<KIND, D> G;
    typedef std::conditional_t<G::scaled, _Float16, XT> CT;
    constexpr int E = G::E, HV = G::halves, kPad = 4, kStep = WAVES * kTile;
    const int h = hr / a.row_tiles, row0 = hr % a.row_tiles * kRows;
    const int i = lane & 15, g = lane >> 4;
    end = min(len, end * kUnit);

    // the lane's query row: token j, head hq of the group
    const int rows = a.q_len * a.group;
    const int row = row0 + i;
    const bool live = row < rows;
    const int j = live ? row / a.group : 0, hq = h * a.group + (live ? row % a.group : 0);
    const int64_t token = static_cast<int64_t>(b) * a.q_len + j;
    // the queries, then the first tile: loads return in their order, so the
    // queries are made ready while the tile is on its way
    const int32_t* row_pages = a.c.table + static_cast<int64_t>(b) * a.c.width;
    int pos = begin * kUnit + wave * kTile;
    Pages pages = look_up(a, row_pages, pos, end);
    typename Vec8<XT>::type raw[D / 32];
    {
        const XT* x = static_cast<const XT*>(a.q.p) + token * a.q.ts + hq * a.q.hs;
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
            raw[n] = *reinterpret_cast<const typename Vec8<XT>::type*>(x + query_dim<KIND, D>(n, g));
    }
    TileRegs<KIND, D> r0, r1;
    if (pos < end) load_tile<KIND, D>(a, pages, h, pos, i, g, r0);
    pages = look_up(a, row_pages, pos + kStep, end);

    Running<KIND, D, CT> w;
    w.seen = live ? len - a.q_len + 1 + j : 0;
    w.qscale = a.scale;
#pragma unroll
    for (int x = 0; x < HV; ++x) w.start[x] = 0.0f;
    {
#pragma unroll
        for (int n = 0; n < D / 32; ++n) {
            if (!live)
#pragma unroll
                for (int y = 0; y < 8; ++y) raw[n][y] = static_cast<XT>(0.0f);
        }
        if constexpr (!G::scaled) {
#pragma unroll
            for (int n = 0; n < D / 32; ++n) w.q[n] = raw[n];
        } else {
            // times a power of two that brings the row's largest into [2^14,
            // 2^15): exact for what is within 2^28 of it
            uint32_t most = 0;
#pragma unroll
            for (int n = 0; n < D / 32; ++n)
#pragma unroll
                for (int y = 0; y < 8; ++y) most = max(most, __float_as_uint(static_cast<float>(raw[n][y])) & 0x7fffffffu);
            most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 16)));
            most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 32)));
            const int exponent = static_cast<int>(most >> 23) - 127;
            int up = most == 0 || exponent == 128 ? 0 : 14 - exponent;
            // The scores' factor is scale * unit * 2^-up.  Where it is past fp32's
            // range for a row, scores take kLarge of it apart (see attend); where it
            // would be subnormal, the queries are smaller instead (which costs
            // nothing: what f16 loses of them is far below the scores' last bit).
            constexpr int unit = KIND == UNISVQ_CACHE_I4 ? 18 : 24;
            const int factor = (static_cast<int>(__float_as_uint(a.scale) >> 23) - 127) + unit;
            w.large = __any(factor - up > 126);
            const int apart = w.large ? kLarge : 0;
            up = min(up, factor - apart + 126);
            constexpr bool nibble = KIND == UNISVQ_CACHE_I4;
#pragma unroll
            for (int n = 0; n < D / 32; ++n)
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    const float v = ldexpf(static_cast<float>(raw[n][nibble ? y / 2 + y % 2 * 4 : y]), up);
                    w.start[n / (D / 32 / HV)] += v;
                    w.q[n][y] = static_cast<CT>(v);
                }
#pragma unroll
            for (int n = 0; n < HV; ++n) {
                w.start[n] += __shfl_xor(w.start[n], 16);
                w.start[n] += __shfl_xor(w.start[n], 32);
                w.start[n] *= -static_cast<float>(G::bias) * 0x1p-24f;
            }
            w.qscale = fminf(ldexpf(a.scale, unit - up - apart), FLT_MAX);
        }
    }
    w.begin();

    while (pos < end) {
        if (pos + kStep < end) load_tile<KIND, D>(a, pages, h, pos + kStep, i, g, r1);
        pages = look_up(a, row_pages, pos + 2 * kStep, end);
        attend<KIND, D, CT>(a, r0, pos, len, g, w);
        pos += kStep;
        if (pos >= end) break;
        if (pos + kStep < end) load_tile<KIND, D>(a, pages, h, pos + kStep, i, g, r0);
        pages = look_up(a, row_pages, pos + 2 * kStep, end);
        attend<KIND, D, CT>(a, r1, pos, len, g, w);
        pos += kStep;
    }

    // join the waves: dim E (4g + n) + e of query i
    w.l += __shfl_xor(w.l, 16);
    w.l += __shfl_xor(w.l, 32);
    __shared__ float so[WAVES][kRows][D + kPad];
    __shared__ float sm[WAVES][kRows], sl[WAVES][kRows];
    if (live) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float v = HV == 2 && g >= 2 ? w.o[HV - 1][e][n] : w.o[0][e][n];
                if constexpr (G::scaled) {
                    const float bias = HV == 2 && g >= 2 ? w.b[HV - 1] : w.b[0];
                    const float u = w.used(HV == 2 && g >= 2 ? HV - 1 : 0);
                    v = (v - bias) * G::unit * exp2_(-u);
                }
                so[wave][i][E * (4 * g + n) + e] = v;
            }
        if (g == 0) sm[wave][i] = w.m, sl[wave][i] = w.l * exp2_(-w.shift());
    }
    __syncthreads();
    const int y = threadIdx.x / (D / 8), d = threadIdx.x % (D / 8) * 8;
    if (y >= kRows || row0 + y >= rows) return;
    float mt = sm[0][y], lt = 0.0f, f[8];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) mt = fmaxf(mt, sm[w][y]);
#pragma unroll
    for (int n = 0; n < 8; ++n) f[n] = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float c = exp2_(sm[w][y] - mt);
        lt += c * sl[w][y];
#pragma unroll
        for (int n = 0; n < 8; ++n) f[n] += c * so[w][y][d + n];
    }
    const int jy = (row0 + y) / a.group, hy = h * a.group + (row0 + y) % a.group;
    const int64_t ty = static_cast<int64_t>(b) * a.q_len + jy, r_out = ty * a.q_heads + hy;
    if (slot < 0) {
        const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
#pragma unroll
        for (int n = 0; n < 8; ++n) f[n] *= inv;
        store8(static_cast<XT*>(a.out.p) + ty * a.out.ts + hy * a.out.hs + d, f);
        if (a.lse && d == 0) a.lse[r_out] = (mt + log2f(lt)) * kLn2;
    } else {
        float* to = a.part + (r_out * a.slots + slot) * D + d;
        *reinterpret_cast<f32x4*>(to) = f32x4{f[0], f[1], f[2], f[3]};
        *reinterpret_cast<f32x4*>(to + 4) = f32x4{f[4], f[5], f[6], f[7]};
        if (d == 0) a.part_ml[r_out * a.slots + slot] = float2{mt, lt};
    }
}

// With eight waves, one a CU: whole items only.
template <int KIND, int D, typename XT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void decode_kernel(Decode a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int items = a.c.heads * a.row_tiles, sequences = static_cast<int>(a.c.sequences);
    int first = 0, unit, last;  // units of the sequences before b, and those of this workgroup
    int b = 0, share, pad = 1;  // (units of items are rounded up to multiples of pad)
    if (WAVES > kWaves || a.slots == 1) {  // an item, whatever its length
        b = blockIdx.x / items;
        share = units_of(length_of(a, b));
        unit = blockIdx.x % items * share;
        last = unit + share;
    } else {
        const int mine = lane < sequences ? units_of(length_of(a, lane)) : 0;
        const auto units_at = [&](int base) {
            return base == 0 ? mine : base + lane < sequences ? units_of(length_of(a, base + lane)) : 0;
        };
        int all = 0, most = 0;
        for (int base = 0; base < sequences; base += 64) {
            const int units = units_at(base);
            all += __builtin_amdgcn_readlane(scan64(units), 63);
            most = max(most, __builtin_amdgcn_readlane(scan64_max(units), 63));
        }
        // even shares, and rows have slots for their parts
        const int grid = gridDim.x;
        share = max((all * items + grid - 1) / grid, (most + a.slots - 3) / (a.slots - 2));
        if (sequences * items <= grid) {
            bool found = false;
            for (int s = share; s < share + 3 && !found; ++s) {
                int parts = 0;
                for (int base = 0; base < sequences; base += 64)
                    parts += __builtin_amdgcn_readlane(scan64((units_at(base) + s - 1) / s), 63);
                found = parts * items <= grid;
                if (found) share = pad = s;
            }
        }
        if (pad > 1) {
            all = 0;
            for (int base = 0; base < sequences; base += 64) all += __builtin_amdgcn_readlane(scan64(padded(units_at(base), pad)), 63);
        }
        if (blockIdx.x == 0 && wave == 0) {
            int sum = 0;
            for (int base = 0; base < sequences; base += 64) {
                const int units = padded(units_at(base), pad), here = scan64(units);
                if (base + lane < sequences) a.before[base + lane] = sum + here - units;
                sum += __builtin_amdgcn_readlane(here, 63);
            }
            if (lane == 0) a.before[sequences] = all, a.before[sequences + 1] = share;
        }
        const int n = all * items;
        if (static_cast<int64_t>(blockIdx.x) * share >= n) return;
        unit = blockIdx.x * share;
        last = min(unit + share, n);
        // (this search and the loop below end, and stay inside, also where another
        // stream writes the lengths meanwhile)
        for (int base = 0;; base += 64) {
            if (base >= sequences) return;
            const int units = padded(units_at(base), pad);
            const int sum = scan64(units);
            const uint64_t in = __ballot(unit < (first + sum) * items);
            if (in) {
                const int l = __ffsll(static_cast<unsigned long long>(in)) - 1;
                b = base + l;
                first += __builtin_amdgcn_readlane(sum - units, l);
                break;
            }
            first += __builtin_amdgcn_readlane(sum, 63);
        }
    }
    while (unit < last && b < sequences) {
        const int64_t room = a.c.width << a.c.page_shift;
        const int len = static_cast<int>(min(static_cast<int64_t>(max(0, load_uniform(a.lens + b))), room));
        const int n = padded(units_of(len), pad);
        const int hr = (unit - first * items) / n, item = first * items + hr * n;
        if (hr >= items) return;
        const int begin = unit - item, end = min(n, last - item);
        const Shares s = shares_of(item, n, share);
        attend_item<KIND, D, XT, WAVES>(a, b, hr, len, begin, end, s.count == 1 ? -1 : static_cast<int>(blockIdx.x) - s.first, wave, lane);
        unit += end - begin;
        if (hr == items - 1 && end == n) first += n, ++b;
        __syncthreads();  // (LDS is used again)
    }
}

// Workgroups: as many as there are units if all sequences have max_len tokens.
int decode_grid(int64_t sequences, int items, int64_t max_len) {
    const int64_t count = std::min<int64_t>(sequences * items, kGrid);  // (their product with the units may pass 64 bits)
    return static_cast<int>(std::min<int64_t>(count * std::max<int64_t>(1, (max_len + kUnit - 1) / kUnit), kGrid));
}

int row_tiles_of(int q_len, int q_heads, int kv_heads) { return (q_len * (q_heads / kv_heads) + kRows - 1) / kRows; }

// How items are worked on.  A workgroup has a whole one, whatever its length,
// where that takes less than joining parts costs (4 us on the GPU, and a
// launch): where none has more than a unit; and where all workgroups are
// resident and none has more than eight units, with eight waves each where
// there is a CU for each.  Of these, few that have much to read take longer,
// a CU reading 40 GB/s: items above 256 KB on half the CUs or fewer are split.
// Calls, with the launches: 32 heads of f16, 512 tokens 10 us whole and 16
// split, 1001 tokens 18 and 16; 8 heads of 8 bits, 1001 tokens 11 and 16, 2000
// tokens 18 and 16; 32 heads of 8 bits, 8 sequences of 1001 tokens 15 and 20,
// 16 of them 25 and 28, 16 ragged ones 15 and 22.
enum Form { kSplit, kWhole, kWholeWide };
Form form_of(int64_t sequences, int items, int64_t max_len, int token_bytes) {
    const int64_t count = sequences * items;
    if (max_len <= kUnit) return kWhole;
    if (max_len > 8 * kUnit || count > kGrid) return kSplit;
    if (count > kGrid / 2) return kWhole;
    return count > kGrid / 4 || max_len * token_bytes <= 1 << 18 ? kWholeWide : kSplit;
}

template <int D, typename XT, int WAVES>
void launch(const Decode& a, uint32_t blocks, hipStream_t s) {
    constexpr int raw = std::is_same_v<XT, _Float16> ? UNISVQ_CACHE_F16 : UNISVQ_CACHE_BF16;
    if (a.c.kind == UNISVQ_CACHE_I8)
        decode_kernel<UNISVQ_CACHE_I8, D, XT, WAVES><<<blocks, 64 * WAVES, 0, s>>>(a);
    else if (a.c.kind == UNISVQ_CACHE_I4)
        decode_kernel<UNISVQ_CACHE_I4, D, XT, WAVES><<<blocks, 64 * WAVES, 0, s>>>(a);
    else
        decode_kernel<raw, D, XT, WAVES><<<blocks, 64 * WAVES, 0, s>>>(a);
}

template <int D, typename XT>
hipError_t run(const Decode& a, int64_t max_len, hipStream_t s) {
    const int items = a.c.heads * a.row_tiles;
    const uint32_t blocks = a.slots == 1 ? static_cast<uint32_t>(a.c.sequences * items) : decode_grid(a.c.sequences, items, max_len);
    if (form_of(a.c.sequences, items, max_len, D * entry_bits(a.c.kind) / 4) == kWholeWide)
        launch<D, XT, 2 * kWaves>(a, blocks, s);
    else
        launch<D, XT, kWaves>(a, blocks, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.slots == 1) return e;
    Join j{};
    j.part = a.part;
    j.part_ml = a.part_ml;
    j.rows = a.c.sequences * a.q_len * a.q_heads;
    j.slots = a.slots;
    j.expected = static_cast<int>(blocks / (a.c.sequences * items));
    j.q_heads = a.q_heads;
    j.out = a.out;
    j.lse = a.lse;
    j.before = a.before;
    j.share = a.before + a.c.sequences + 1;
    j.q_len = a.q_len;
    j.group = a.group;
    j.items = items;
    j.row_tiles = a.row_tiles;
    j.tile = kRows;
    return launch_join<D, XT>(j, s);
}

}  // namespace

// Parts a row can have (a share is made large enough for it); one: workgroups
// have whole items.
int decode_slots(int64_t sequences, int q_len, int q_heads, int kv_heads, int64_t max_len, int token_bytes) {
    const int items = kv_heads * row_tiles_of(q_len, q_heads, kv_heads);
    if (form_of(sequences, items, max_len, token_bytes) != kSplit) return 1;
    return std::min(kSlots, std::max(1, decode_grid(sequences, items, max_len) / items) + 2);
}

size_t decode_workspace_bytes(int64_t sequences, int q_len, int q_heads, int head_dim, int slots) {
    if (slots == 1) return 0;
    return static_cast<size_t>(sequences * q_len * q_heads) * slots * (head_dim + 2) * 4 + static_cast<size_t>(sequences + 2) * 4;
}

hipError_t launch_attn_decode(const CacheView& c, const int32_t* lens, int64_t max_len, int slots, int q_len, int q_heads,
                              Rows q, int x_dtype, float scale, Rows out, float* lse, void* workspace, hipStream_t s) {
    Decode a{};
    a.c = c;
    a.lens = lens;
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.slots = slots;
    a.q_len = q_len;
    a.q_heads = q_heads;
    a.group = q_heads / c.heads;
    a.row_tiles = row_tiles_of(q_len, q_heads, c.heads);
    a.scale = scale * kLog2e;
    if (slots > 1) {
        const int64_t parts = c.sequences * q_len * q_heads * slots;
        a.part = static_cast<float*>(workspace);
        a.part_ml = reinterpret_cast<float2*>(a.part + parts * c.head_dim);
        a.before = reinterpret_cast<int32_t*>(a.part_ml + parts);
    }
    if (c.head_dim == 128) return x_dtype == UNISVQ_F16 ? run<128, _Float16>(a, max_len, s) : run<128, __bf16>(a, max_len, s);
    return x_dtype == UNISVQ_F16 ? run<64, _Float16>(a, max_len, s) : run<64, __bf16>(a, max_len, s);
}

}  // namespace unisvq
