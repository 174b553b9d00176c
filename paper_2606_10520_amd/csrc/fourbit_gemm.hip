// Products with 4-bit weights on gfx950.
//   y[t][n] = sum_g S[n][g] sum_{k in g} x[t][k] (c[n][k] - 8)
// over groups g of 128 columns, codes c 0..15, x of 16 bits or, with a scale a
// token, of 8.
//
// Codes go to the matrix cores as they are: a byte 0..15 is c as an i8, and as
// an e4m3 it is c * 2^-9 (the format is linear through its subnormals and its
// first binade), which one instruction turns into two exact f16 or bf16.  The
// -8 of all codes of a group is sum x * -8, one more product with a constant
// operand, which the groups' sums start from; so every product is exact, sums of
// a group are fp32 (i8: exact integers), and scales multiply them in fp32: no
// weight is ever rounded.
#include <algorithm>

#include "layer.hpp"

namespace unisvq {
namespace {

constexpr int64_t kCUs = 256;
constexpr int kMostLds = 160 * 1024;  // of a CU

struct Prob {
    const uint8_t* packed;
    const void* x;
    const float* x_scales;
    void* y;
    int64_t N;
    int K, wg_begin, wgs;
};

struct Batch {
    Prob p[kMaxBatch];
    int count, y_dtype;
    int64_t M;
};

// What differs between the types of activations: an operand's 16 bytes, the
// products of a group's tile (16 rows x 128 columns), and the sums' unit.
template <typename T>
struct Kind {
    static constexpr bool kI8 = false;
    typedef typename Vec8<T>::type Operand;
    typedef f32x4 Sum;
    static constexpr int kSteps = 4, kBytes = 2;      // products a slot of codes, bytes an element
    static constexpr float kUnit = 512.0f;            // codes are c * 2^-9
    __device__ static Operand minus8() {
        Operand v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<T>(-8.0f / kUnit);
        return v;
    }
    // operands of steps 0..3 (a word of codes each)
    __device__ static void decode(uint4 q, Operand (&w)[kSteps]) {
        const uint32_t word[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = word[j] & 0x0f0f0f0fu, hi = word[j] >> 4 & 0x0f0f0f0fu;
            uint4 v;
            if constexpr (std::is_same_v<T, _Float16>) {
                v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false));
                v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true));
                v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false));
                v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
            } else {
                v.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
                v.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
                v.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
                v.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
            }
            w[j] = __builtin_bit_cast(Operand, v);
        }
    }
    __device__ static Sum mma(Operand x, Operand w, Sum c) {
        if constexpr (std::is_same_v<T, _Float16>)
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, c, 0, 0, 0);
    }
    // byte offset of step s's operand in a token's group, for chunk c of the lane
    __device__ static constexpr uint32_t at(int s) { return 128 * (s >> 1) + 16 * (s & 1); }
    static constexpr uint32_t kChunk = 32;
};

template <>
struct Kind<int8_t> {
    static constexpr bool kI8 = true;
    typedef i32x4 Operand;
    typedef i32x4 Sum;
    static constexpr int kSteps = 2, kBytes = 1;
    static constexpr float kUnit = 1.0f;
    __device__ static Operand minus8() {
        const int b = static_cast<int>(0xf8f8f8f8u);
        return i32x4{b, b, b, b};
    }
    __device__ static void decode(uint4 q, Operand (&w)[kSteps]) {
        constexpr uint32_t m = 0x0f0f0f0fu;
        w[0] = __builtin_bit_cast(i32x4, uint4{q.x & m, q.x >> 4 & m, q.y & m, q.y >> 4 & m});
        w[1] = __builtin_bit_cast(i32x4, uint4{q.z & m, q.z >> 4 & m, q.w & m, q.w >> 4 & m});
    }
    __device__ static Sum mma(Operand x, Operand w, Sum c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(x, w, c, 0, 0, 0); }
    __device__ static constexpr uint32_t at(int s) { return 64 * s; }
    static constexpr uint32_t kChunk = 16;
};

// ---- few tokens ----
// Bound by the weights' read: x has to come from somewhere near.  A workgroup's
// waves share K out in runs of groups; every wave keeps its part of x in LDS (TOK
// tokens, 16-byte chunks turned by the token so that those that are read together
// lie in different banks) and -8 times its groups' sums, and passes over blocks of
// sixteen rows with them, as far apart as its problem has workgroups, DEEP tiles of
// codes on their way.  The waves' sums of a block meet in LDS, one of the waves adds and
// stores them while the others go on.  One token, 57344 rows of 8192: 40.6 us (5.9 TB/s);
// 4096 rows of 4096: 5.0; four tokens, 22016 rows of 4096: 13.2 (two sets of tiles on
// their way: 42.8, 5.7, 15.3).
template <typename X, int TOK, int WAVES, int DEEP>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(const Batch b) {
    typedef Kind<X> Q;
    constexpr int kRow = kGroup * Q::kBytes, kChunks = kRow / 16, kGroupBytes = TOK * kRow + 64;
    extern __shared__ __attribute__((aligned(16))) uint8_t few_lds[];
    f32x4(*parts)[WAVES][64] = reinterpret_cast<f32x4(*)[WAVES][64]>(few_lds);
    Prob p = b.p[0];
#pragma unroll
    for (int i = 1; i < kMaxBatch; ++i)
        if (i < b.count && static_cast<int>(blockIdx.x) >= b.p[i].wg_begin) p = b.p[i];
    const int wgs = p.wgs;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, c = lane >> 4, tok = n & (TOK - 1);
    const int blocks = static_cast<int>(p.N / kRowBlock), first = static_cast<int>(blockIdx.x) - p.wg_begin;
    const int K = p.K, groups = K / kGroup, quads = (groups + 3) / 4;
    const int g0 = __builtin_amdgcn_readfirstlane(groups * wave / WAVES), g1 = __builtin_amdgcn_readfirstlane(groups * (wave + 1) / WAVES);
    const int share = g1 - g0;
    uint8_t* mine = few_lds + 2 * WAVES * 1024 + g0 * kGroupBytes;

    // a tile: codes and scale of (block, group), by running offsets
    const uint8_t* tail = p.packed + p.N * (K / 2);
    struct Tile {
        uint4 q;
        uint32_t s;
    } ring[DEEP];
    // (a block's tiles are taken DEEP at a time; those past the share read nothing:
    // their scales are zeros)
    const int padded = max((share + DEEP - 1) / DEEP * DEEP, DEEP);
    int rb = first, next = 0;  // of the next tile to ask for
    const auto ask = [&](Tile& t) {
        const uint32_t out = rb < blocks && next < share ? 0u : kOutOfRange;
        const int g = g0 + next;
        const int64_t at = min(rb, blocks - 1);
        const __amdgpu_buffer_rsrc_t rw = make_rsrc(p.packed + at * groups * kFourbitTile, groups * kFourbitTile);
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(tail + at * quads * kFourbitQuad, quads * kFourbitQuad);
        t.q = ld128_stream(rw, out | static_cast<uint32_t>(g * kFourbitTile + 16 * lane));
        t.s = ld16(rs, out | static_cast<uint32_t>((g >> 2) * kFourbitQuad + 8 * n + 2 * (g & 3)));
        const bool last = next + 1 >= padded;
        next = last ? 0 : next + 1;
        rb += last ? wgs : 0;
    };
#pragma unroll
    for (int i = 0; i < DEEP; ++i) ask(ring[i]);

    // x and the sums
    {
        const __amdgpu_buffer_rsrc_t rx = make_rsrc(p.x, static_cast<uint32_t>(b.M) * K * Q::kBytes);
        for (int i = lane; i < share * TOK * kChunks; i += 64) {
            const int chunk = i % kChunks, t = i / kChunks % TOK, h = i / (kChunks * TOK);
            const int turn = Q::kI8 ? (t >> 1 & 1) << 2 | t >> 2 : (t & 1) | (t >> 1 & 1) << 3 | (t >> 2) << 1;
            const uint4 v = ld128(rx, t < b.M ? static_cast<uint32_t>((t * K + (g0 + h) * kGroup) * Q::kBytes + 16 * chunk) : kOutOfRange);
            *reinterpret_cast<uint4*>(mine + h * kGroupBytes + t * kRow + 16 * (chunk ^ turn)) = v;
        }
    }
    const int turn = Q::kI8 ? (tok >> 1 & 1) << 2 | tok >> 2 : (tok & 1) | (tok >> 1 & 1) << 3 | (tok >> 2) << 1;
    const uint8_t* at[Q::kSteps];
#pragma unroll
    for (int j = 0; j < Q::kSteps; ++j) at[j] = mine + tok * kRow + 16 * (((Q::kChunk * c + Q::at(j)) / 16) ^ turn);
    {
        const typename Q::Operand minus8 = Q::minus8();
        for (int h = 0; h < share; ++h) {
            typename Q::Sum bias{};
#pragma unroll
            for (int j = 0; j < Q::kSteps; ++j)
                bias = Q::mma(*reinterpret_cast<const typename Q::Operand*>(at[j] + h * kGroupBytes), minus8, bias);
            if (n == 0) *reinterpret_cast<typename Q::Sum*>(mine + h * kGroupBytes + TOK * kRow + 16 * c) = bias;
        }
    }
    __builtin_amdgcn_wave_barrier();  // (a wave reads what it wrote itself)

    int block = first, turnover = 0, h0 = 0;
    f32x4 acc{};
    const auto pass = [&](Tile(&r)[DEEP]) {
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            const int h = max(min(h0 + i, share - 1), 0);
            typename Q::Operand w[Q::kSteps];
            Q::decode(r[i].q, w);
            const float s = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(r[i].s)));
            ask(r[i]);
            typename Q::Sum sum = *reinterpret_cast<const typename Q::Sum*>(mine + h * kGroupBytes + TOK * kRow + 16 * c);
#pragma unroll
            for (int j = 0; j < Q::kSteps; ++j)
                sum = Q::mma(*reinterpret_cast<const typename Q::Operand*>(at[j] + h * kGroupBytes), w[j], sum);
            if (share > 0)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(s, static_cast<float>(sum[e]), acc[e]);
        }
        h0 += DEEP;
        if (h0 < padded) return;
        h0 = 0;
        parts[turnover & 1][wave][lane] = acc;
        acc = f32x4{};
        __syncthreads();
        if (wave == turnover % WAVES && 4 * c < b.M) {
            f32x4 sum = parts[turnover & 1][0][lane];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) sum += parts[turnover & 1][w][lane];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (4 * c + i < b.M) {
                    const float unit = Q::kI8 ? p.x_scales[4 * c + i] : Q::kUnit;
                    store_out(p.y, (4 * c + i) * p.N + block * kRowBlock + n, sum[i] * unit, b.y_dtype);
                }
        }
        block += wgs, ++turnover;
    };
    while (block < blocks) pass(ring);
}

// Bytes of LDS: two rounds of the waves' sums, x and its groups' sums.
int64_t few_lds_bytes(int64_t K, int tok, int waves, int size) {
    return 2 * waves * 1024 + K / kGroup * (tok * kGroup * size + 64);
}

// How few tokens' work is shared out: waves of a workgroup, tiles that a wave asks for
// together, and blocks of rows that a workgroup passes over.
struct FewPlan {
    int waves, deep, passes;
};

// The variants there are.  (Eight tokens come with 16 to 32 groups of 16 bits alone, which
// take these by the plan below.)
constexpr bool few_variant(int tok, int waves, int deep) {
    if (tok == 8) return waves == 16 ? deep == 2 : deep >= 2 && deep <= 4;
    return waves == 16 ? deep >= 2 && deep <= 4 : deep >= 1 && deep <= 5;
}

// A wave's share of the groups is taken DEEP tiles at a time, the last ones empty where
// DEEP does not divide it: as few empty ones as can be (40 groups, 22016 rows, one token:
// five of eight waves 13.5 us, threes of sixteen 14.0, fours of sixteen 18.0; 20 groups,
// threes 9.2, fours 10.3).  Eight waves, two workgroups to a CU, or sixteen: 16 bits, more
// than 32 groups: sixteen are faster by 3 to 8% where both have as many empty tiles (48
// groups, one token: 14.6 us for 15.0), 8 bits slower by 6 to 10% (48 groups, four
// tokens: 19.6 for 17.7); few rows, one block a workgroup: sixteen, by 10% (28 groups, 4096
// rows, 8 bits: 5.3 us for 5.8), and no more than three at a time (64 groups: twos 6.7,
// fours 7.0).
FewPlan few_plan(const Batch& b, int64_t K, int tok, int size) {
    const int groups = static_cast<int>(K / kGroup);
    FewPlan best{};
    double least = 1e30;
    for (const int waves : {8, 16}) {
        const int64_t lds = few_lds_bytes(K, tok, waves, size);
        if (lds > (waves == 8 ? kMostLds / 2 : kMostLds)) continue;
        // as many workgroups as the GPU holds, every one with as many blocks as any
        const int64_t places = kCUs * 16 / waves;
        int64_t total = 0;
        for (int i = 0; i < b.count; ++i) total += b.p[i].N / kRowBlock;
        int64_t passes = (total + places - 1) / places;
        for (int64_t wgs = places + 1; wgs > places; ++passes) {
            wgs = 0;
            for (int i = 0; i < b.count; ++i) wgs += (b.p[i].N / kRowBlock + passes - 1) / passes;
            if (wgs <= places) break;
        }
        const bool few_rows = total <= kCUs;
        double factor = 1.0;
        if (few_rows)
            factor = waves == 8 ? 1.25 : 1.0;
        else if (size == 1)
            factor = waves == 16 ? 1.1 : 1.0;
        else if (groups > 32)
            factor = waves == 8 ? 1.1 : 1.0;
        const int share = (groups + waves - 1) / waves;
        for (int deep = waves == 8 ? share > 1 ? 5 : 1 : few_rows ? 3 : 4; deep >= (share > 1 ? 2 : 1); --deep) {
            if (!few_variant(tok, waves, deep)) continue;
            const double cost = (share + deep - 1) / deep * deep * waves * factor;
            if (cost < least) least = cost, best = FewPlan{waves, deep, static_cast<int>(passes)};
        }
    }
    return best;
}

template <typename X, int TOK, int WAVES, int DEEP>
int launch_few(Batch b, int64_t K, int64_t passes, hipStream_t s) {
    const int lds = static_cast<int>(few_lds_bytes(K, TOK, WAVES, Kind<X>::kBytes));
    static std::atomic<uint64_t> done{0};
    if (lds > 65536) {
        const int st = ensure_lds_limit(reinterpret_cast<const void*>(few_kernel<X, TOK, WAVES, DEEP>), kMostLds, done);
        if (st != UNISVQ_OK) return st;
    }
    int64_t blocks = 0;
    for (int i = 0; i < b.count; ++i) {
        b.p[i].wg_begin = static_cast<int>(blocks);
        b.p[i].wgs = static_cast<int>((b.p[i].N / kRowBlock + passes - 1) / passes);
        blocks += b.p[i].wgs;
    }
    few_kernel<X, TOK, WAVES, DEEP><<<static_cast<uint32_t>(blocks), 64 * WAVES, lds, s>>>(b);
    return hipGetLastError() == hipSuccess ? UNISVQ_OK : UNISVQ_EHIP;
}

template <typename X, int TOK, int WAVES, int DEEP = 1>
int launch_deep(const Batch& b, int64_t K, const FewPlan& p, hipStream_t s) {
    if constexpr (DEEP <= 5) {
        if constexpr (few_variant(TOK, WAVES, DEEP))
            if (p.deep == DEEP) return launch_few<X, TOK, WAVES, DEEP>(b, K, p.passes, s);
        return launch_deep<X, TOK, WAVES, DEEP + 1>(b, K, p, s);
    }
    return UNISVQ_EUNSUP;
}

template <typename X, int TOK>
int launch_few(const Batch& b, int64_t K, hipStream_t s) {
    const FewPlan p = few_plan(b, K, TOK, Kind<X>::kBytes);
    return p.waves == 16 ? launch_deep<X, TOK, 16>(b, K, p, s) : launch_deep<X, TOK, 8>(b, K, p, s);
}

int tok_of(int64_t M) { return M == 1 ? 1 : M == 2 ? 2 : M <= 4 ? 4 : 8; }

// Up to sixteen tokens and not many rows: a workgroup has a block of sixteen rows, its
// waves share K out in runs of groups and read x from the L2, and their sums meet
// in LDS; one launch, where tiles would have to be joined by a second.
constexpr int kSomeWaves = 8;  // (16 tokens, 4096 x 4096: 7.6 us, four waves 8.4, sixteen 8.2)

template <typename X>
__global__ __launch_bounds__(64 * kSomeWaves) void some_kernel(const Batch b) {
    typedef Kind<X> Q;
    __shared__ f32x4 parts[kSomeWaves][64];
    Prob p = b.p[0];
#pragma unroll
    for (int i = 1; i < kMaxBatch; ++i)
        if (i < b.count && static_cast<int>(blockIdx.x) >= b.p[i].wg_begin) p = b.p[i];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, c = lane >> 4;
    const int64_t rb = static_cast<int>(blockIdx.x) - p.wg_begin;
    const int K = p.K, groups = K / kGroup, quads = (groups + 3) / 4;
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(p.packed + rb * groups * kFourbitTile, groups * kFourbitTile);
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(p.packed + p.N * (K / 2) + rb * quads * kFourbitQuad, quads * kFourbitQuad);
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(p.x, static_cast<uint32_t>(b.M) * K * Q::kBytes);
    const int g0 = groups * wave / kSomeWaves, g1 = groups * (wave + 1) / kSomeWaves;

    struct Step {
        uint4 q, x[Q::kSteps];
        uint32_t s;
    };
    const auto load = [&](int g, Step& t) {
        const uint32_t out = g < g1 ? 0u : kOutOfRange;
        t.q = ld128_stream(rw, out | static_cast<uint32_t>(g * kFourbitTile + 16 * lane));
        t.s = ld16(rs, out | static_cast<uint32_t>((g >> 2) * kFourbitQuad + 8 * n + 2 * (g & 3)));
#pragma unroll
        for (int j = 0; j < Q::kSteps; ++j)
            t.x[j] = ld128(rx, out | (static_cast<uint32_t>(n * K + g * kGroup) * Q::kBytes + Q::kChunk * c + Q::at(j)));
    };
    f32x4 acc{};
    const typename Q::Operand minus8 = Q::minus8();
    const auto use = [&](const Step& t) {
        typename Q::Operand x[Q::kSteps], w[Q::kSteps];
        typename Q::Sum sum{};
#pragma unroll
        for (int j = 0; j < Q::kSteps; ++j) {
            x[j] = __builtin_bit_cast(typename Q::Operand, t.x[j]);
            sum = Q::mma(x[j], minus8, sum);
        }
        Q::decode(t.q, w);
#pragma unroll
        for (int j = 0; j < Q::kSteps; ++j) sum = Q::mma(x[j], w[j], sum);
        const float s = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(t.s)));
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = fmaf(s, static_cast<float>(sum[i]), acc[i]);
    };
    Step even, odd;
    load(g0, even);
    for (int g = g0; g < g1; g += 2) {
        load(g + 1, odd);
        use(even);
        load(g + 2, even);
        if (g + 1 < g1) use(odd);
    }

    parts[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < kSomeWaves; ++w) acc += parts[w][lane];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t t = 4 * c + i;
        if (t < b.M) store_out(p.y, t * p.N + rb * kRowBlock + n, acc[i] * (Q::kI8 ? p.x_scales[t] : Q::kUnit), b.y_dtype);
    }
}

template <typename X>
int launch_some(Batch b, hipStream_t s) {
    int blocks = 0;
    for (int i = 0; i < b.count; ++i) {
        b.p[i].wg_begin = blocks;
        blocks += static_cast<int>(b.p[i].N / kRowBlock);
    }
    some_kernel<X><<<blocks, 64 * kSomeWaves, 0, s>>>(b);
    return hipGetLastError() == hipSuccess ? UNISVQ_OK : UNISVQ_EHIP;
}

// ---- many tokens ----
// -8 times the sums of every token's groups, bias[token / 16][group][token % 16]
// (fp32, or i8's integers), sixteen lanes a sum: what the tiled product's sums of
// a group start from.  Bound by memory; 2048 tokens of 4096 bf16: 5 us.
constexpr int kSumTile = 16;

struct Sums {
    const void* x;
    void* bias;
    int64_t M;
    int groups;
};

template <typename X>
__global__ __launch_bounds__(256) void sums_kernel(Sums a) {
    const int64_t count = a.M * a.groups;
    const int lane = threadIdx.x & 15;
    for (int64_t i0 = blockIdx.x * 16ll; i0 < count; i0 += gridDim.x * 16ll) {
        const int64_t i = i0 + (threadIdx.x >> 4), at = min(i, count - 1), t = at / a.groups, g = at - t * a.groups;
        const int64_t to = (t / kSumTile * a.groups + g) * kSumTile + t % kSumTile;
        const X* x = static_cast<const X*>(a.x) + at * kGroup + 8 * lane;
        if constexpr (Kind<X>::kI8) {
            const uint2 v = *reinterpret_cast<const uint2*>(x);
            int sum = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) sum += static_cast<int8_t>(v.x >> 8 * b) + static_cast<int8_t>(v.y >> 8 * b);
            sum = over_lanes(sum, 4, [](int p, int q) { return p + q; });
            if (lane == 0 && i < count) static_cast<int*>(a.bias)[to] = -8 * sum;
        } else {
            float f[8], sum = 0.0f;
            load8(x, f);
#pragma unroll
            for (int b = 0; b < 8; ++b) sum += f[b];
            sum = over_lanes(sum, 4, [](float p, float q) { return p + q; });
            if (lane == 0 && i < count) static_cast<float*>(a.bias)[to] = -8.0f / Kind<X>::kUnit * sum;
        }
    }
}

struct TileProb {
    const uint8_t* packed;
    const void* x;
    const void* bias;
    const float* x_scales;
    void* y;
    float* partial;  // [split][M][N], or null
    int64_t N;
    int K, splits, wg_begin;
};

struct TileBatch {
    TileProb p[kMaxBatch];
    int count, y_dtype, m_tiles;
    int64_t M;
};

// Loads of 16 bytes a lane that go to LDS, 1 KB a wave and load: to `to` and
// every STEP bytes on, from the buffer at off[i] + at.  (In asm, as the compiler
// would wait for a load that it knows of before any read of LDS.  What it puts
// between its own instructions has to be done here: a load that goes to LDS by M0
// comes a wait state after the write of M0, and one that reads scalar registers
// five after vector instructions that wrote them.)
template <int STEP, int LOADS>
__device__ __forceinline__ void load_lds(uint32_t to, const uint32_t (&off)[LOADS], __amdgpu_buffer_rsrc_t r, uint32_t at) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to + i * STEP),
                     "v"(off[i]), "s"(r), "s"(at)
                     : "memory");
}

// A workgroup has 16 MT tokens and four waves, a wave 16 NB rows for all of them;
// two workgroups share a CU.  A group of columns at a time goes to LDS by direct
// loads: activations, which all waves read, in rows whose 16-byte chunks are
// turned by the row (so that sixteen rows' same chunk lies in sixteen places),
// and every wave's own codes and scales.  A wave turns its rows' codes into
// operands once and passes over the tokens with them.
//
// SUMS: the sums that a group starts from are made here, by one product more for
// every NB; else they come from sums_kernel.
//
// 2048 tokens, 22016 rows of 4096: bf16 335 to 360 us (1.03 to 1.10 PFLOP/s; the matrix
// cores are busy 51% of the cycles at the clock that the power leaves, and products
// wait for their operands' conversion); 8 bits 215 to 225 us (1.7 POP/s): the two waves
// of a SIMD issue in 98% of the cycles, five vector instructions a product, most of
// them a sum's conversion and its product with the scale.  61 tokens, 10240 rows of
// 8192: 21 us, of which a wave lives 14, a third of that waiting for loads.
template <typename X, int MT, int NB, bool SUMS>
struct Tiled {
    typedef Kind<X> Q;
    static constexpr int kWaves = 4, kThreads = 64 * kWaves;
    static constexpr int BM = 16 * MT, BN = 16 * NB * kWaves;
    static constexpr int kRow = kGroup * Q::kBytes;  // bytes of a token's group
    // bytes of activations, of sums (whole loads: what is behind the tokens becomes
    // zeros), and of a wave's codes and scales
    static constexpr int kX = (BM * kRow + 16 * kThreads - 1) / (16 * kThreads) * (16 * kThreads);
    static constexpr int kBias = SUMS ? 0 : 1024, kCodes = NB * 1024, kScales = 1024;
    static constexpr int kShared = kX + kBias, kOwn = kCodes + kScales;
    // Groups in LDS; where there is no room for two of everything, codes and
    // scales are one deep: their next ones are asked for when they have been read.
    static constexpr int kRoom = kMostLds / 2, kGroups = kRoom / (kShared + kWaves * kOwn);
    static constexpr int kStages = kGroups < 2 ? 2 : kGroups < 3 ? kGroups : 3, kCodeStages = kGroups < 2 ? 1 : kStages;
    static constexpr int kLds = kStages * kShared + kWaves * kCodeStages * kOwn;
    static_assert(kLds <= kRoom, "");
    static constexpr int kLoadsX = kX / (16 * kThreads), kLoadsCodes = kCodes / 1024;
    static_assert(BM <= 256, "");
    // a wave's outputs of one tile of tokens, staged for whole-line stores
    static constexpr int kPitch = 16 * NB * 4 + 16;
    static_assert(kWaves * 16 * kPitch <= kLds, "");
};

// A wave's outputs, acc[m][j][i] of token 16 m + 4 (lane / 16) + i and row 16 j +
// lane % 16, to y[token][row]: a tile of sixteen tokens at a time through the
// wave's own LDS, and from there in pieces of 16 bytes of tokens' rows.
template <int MT, int NB, typename Y>
__device__ __forceinline__ void store_tiles(Y* y, int64_t pitch, const f32x4 (&acc)[MT][NB], int toks, int rows, uint8_t* mine, int lane) {
    const int n = lane & 15, c = lane >> 4;
    if ((reinterpret_cast<uintptr_t>(y) & 15) != 0) {  // (rows are of sixteen elements and more: one row's place says it all)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    if (16 * m + 4 * c + i < toks && 16 * j < rows)
                        y[(16 * m + 4 * c + i) * pitch + 16 * j + n] = static_cast<Y>(acc[m][j][i]);
        return;
    }
    constexpr int kPieces = 16 * NB * sizeof(Y) / 16, kRow = 16 * NB + 16 / sizeof(Y);
    Y* stage = reinterpret_cast<Y*>(mine);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) stage[(4 * c + i) * kRow + 16 * j + n] = static_cast<Y>(acc[m][j][i]);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < 16 * kPieces / 64; ++e) {
            const int piece = e * 64 + lane, t = piece / kPieces, at = piece % kPieces * (16 / static_cast<int>(sizeof(Y)));
            const uint4 v = *reinterpret_cast<const uint4*>(stage + t * kRow + at);
            if (16 * m + t < toks && at < rows) *reinterpret_cast<uint4*>(y + (16 * m + t) * pitch + at) = v;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename X, int MT, int NB, bool SUMS>
__global__ __launch_bounds__(256, 2) void tiled_kernel(const TileBatch tb) {
    typedef Tiled<X, MT, NB, SUMS> C;
    typedef typename C::Q Q;
    __shared__ __attribute__((aligned(16))) uint8_t lds[C::kLds];
    TileProb p = tb.p[0];
#pragma unroll
    for (int i = 1; i < kMaxBatch; ++i)
        if (i < tb.count && static_cast<int>(blockIdx.x) >= tb.p[i].wg_begin) p = tb.p[i];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, c = lane >> 4;
    const int K = p.K, groups = K / kGroup, quads = (groups + 3) / 4;
    const int64_t blocks = p.N / kRowBlock;

    // Tile: token tile fastest, so that what runs at once shares rows of weights;
    // an XCD has a contiguous run of tiles.
    const int n_tiles = static_cast<int>((blocks * kRowBlock + C::BN - 1) / C::BN);
    const int T = tb.m_tiles * n_tiles * p.splits;
    int L = static_cast<int>(blockIdx.x) - p.wg_begin;
    if ((T & 7) == 0) L = (L & 7) * (T >> 3) + (L >> 3);
    // (divisions leave the scalar registers)
    const int nt_sp = __builtin_amdgcn_readfirstlane(L / tb.m_tiles), mt = L - nt_sp * tb.m_tiles;
    const int sp = __builtin_amdgcn_readfirstlane(nt_sp / n_tiles), nt = nt_sp - sp * n_tiles;
    const int64_t tok0 = static_cast<int64_t>(mt) * C::BM, rb0 = nt * (C::BN / 16) + wave * NB;
    const int toks = static_cast<int>(min(static_cast<int64_t>(C::BM), tb.M - tok0));
    // row blocks of the wave's that are there (a wave with none goes along)
    const int rbs = max(min(NB, static_cast<int>(blocks - rb0)), 0);
    const int64_t rb_at = __builtin_amdgcn_readfirstlane(static_cast<int>(min(rb0, blocks - 1)));
    const int g0 = __builtin_amdgcn_readfirstlane(groups * sp / p.splits);
    const int g1 = __builtin_amdgcn_readfirstlane(groups * (sp + 1) / p.splits);

    const __amdgpu_buffer_rsrc_t rx = make_rsrc(static_cast<const uint8_t*>(p.x) + tok0 * K * Q::kBytes,
                                                static_cast<uint32_t>(toks) * K * Q::kBytes);
    const uint32_t here = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(max(rbs, 1)));
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(p.packed + rb_at * groups * kFourbitTile, here * groups * kFourbitTile);
    const __amdgpu_buffer_rsrc_t rs =
        make_rsrc(p.packed + p.N * (K / 2) + rb_at * quads * kFourbitQuad, here * quads * kFourbitQuad);
    const __amdgpu_buffer_rsrc_t rb = make_rsrc(static_cast<const uint8_t*>(p.bias) + tok0 * groups * 4,
                                                static_cast<uint32_t>((toks + kSumTile - 1) / kSumTile * groups * kSumTile * 4));

    // Places past the last token or row read the last one again: they are not stored.
    constexpr int kChunks = C::kRow / 16, kTurn = Q::kI8 ? 1 : 0;  // a row's chunk j lies at j ^ ((row >> kTurn) % kChunks)
    uint32_t off_x[C::kLoadsX];
#pragma unroll
    for (int i = 0; i < C::kLoadsX; ++i) {
        const int at = i * C::kThreads + threadIdx.x, row = at / kChunks, chunk = at % kChunks ^ (row >> kTurn) % kChunks;
        off_x[i] = row < C::BM ? static_cast<uint32_t>(min(row, toks - 1)) * K * Q::kBytes + 16 * chunk : kOutOfRange;
    }
    const uint32_t at16[1] = {16u * lane};
    const uint32_t off_s[1] = {lane >> 3 < NB ? min(static_cast<uint32_t>(lane) >> 3, here - 1) * quads * kFourbitQuad + 16 * (lane & 7)
                                                  : kOutOfRange};
    const uint32_t off_b[1] = {4 * lane < C::BM ? static_cast<uint32_t>(lane / 4 * groups * kSumTile * 4 + 16 * (lane % 4)) : kOutOfRange};
    static_assert(kSumTile == 16, "");
    const bool has_bias = !SUMS && wave == 0;
    const uint32_t base = __builtin_amdgcn_readfirstlane(
        static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)&lds[0])));
    constexpr int kOwnAt = C::kStages * C::kShared;
    const auto issue_shared = [&](int g, int stage) {
        const uint32_t to = base + stage * C::kShared;
        load_lds<16 * C::kThreads>(to + wave * 1024, off_x, rx, static_cast<uint32_t>(g) * C::kRow);
        if (has_bias) load_lds<0>(to + C::kX, off_b, rb, static_cast<uint32_t>(g) * (kSumTile * 4));
    };
    const auto issue_own = [&](int g, int stage) {
        const uint32_t to = base + kOwnAt + (wave * C::kCodeStages + stage) * C::kOwn;
#pragma unroll
        for (uint32_t i = 0; i < C::kLoadsCodes; ++i)
            load_lds<0>(to + i * 1024, at16, rw, __builtin_amdgcn_readfirstlane((min(i, here - 1) * groups + g) * kFourbitTile));
        load_lds<0>(to + C::kCodes, off_s, rs, static_cast<uint32_t>(g >> 2) * kFourbitQuad);
    };

    typename Q::Operand minus8 = Q::minus8();
    f32x4 acc[MT][NB] = {};
    // groups under way, and this wave's loads of one
    constexpr int kAhead = C::kStages - 1, kAheadOwn = C::kCodeStages == 1 ? 1 : kAhead;
    constexpr int kLoads = C::kLoadsX + C::kLoadsCodes + 1;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (g0 + i < g1) {
            issue_shared(g0 + i, i);
            issue_own(g0 + i, C::kCodeStages == 1 ? 0 : i);
        }
    int stage = 0;
    for (int g = g0; g < g1; ++g) {
        // this group is there, and the last one has been read by all
        __builtin_amdgcn_sched_barrier(0);
        if (kAhead == 1 || g + kAhead > g1)
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else if (has_bias)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kAhead - 1) * (kLoads + 1)) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((kAhead - 1) * kLoads) : "memory");
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        const int before = stage ? stage - 1 : kAhead;
        if (g + kAhead < g1) issue_shared(g + kAhead, before);
        const uint8_t* own = lds + kOwnAt + (wave * C::kCodeStages + (C::kCodeStages == 1 ? 0 : stage)) * C::kOwn;
        typename Q::Operand w[NB][Q::kSteps];
        float s[NB];
        uint4 q[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            q[j] = *reinterpret_cast<const uint4*>(own + j * 1024 + 16 * lane);
            s[j] = static_cast<float>(*reinterpret_cast<const _Float16*>(own + C::kCodes + j * 128 + 8 * n + 2 * (g & 3)));
        }
        if constexpr (C::kCodeStages == 1) {  // (read before they are overwritten)
#pragma unroll
            for (int j = 0; j < NB; ++j) asm volatile("" : "+v"(s[j]));
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        if (g + kAheadOwn < g1) issue_own(g + kAheadOwn, C::kCodeStages == 1 ? 0 : before);
        // Tokens' operands are read one tile ahead (instructions on LDS stay where they
        // are put, all others may move over them): 333 tokens through 3 x 4096 x 4096,
        // 8 bits, 36 us for 39.
        const uint8_t* from = lds + stage * C::kShared;
        typename Q::Operand x[2][Q::kSteps];
        typename Q::Sum bias[2];
        const auto read = [&](int m) {
            const int row = 16 * m + n;
#pragma unroll
            for (int k = 0; k < Q::kSteps; ++k) {
                const int chunk = (Q::kChunk * c + Q::at(k)) / 16;
                x[m & 1][k] = *reinterpret_cast<const typename Q::Operand*>(from + row * C::kRow + 16 * (chunk ^ (row >> kTurn) % kChunks));
            }
            bias[m & 1] = typename Q::Sum{};
            if constexpr (!SUMS) bias[m & 1] = *reinterpret_cast<const typename Q::Sum*>(from + C::kX + 4 * (row - n + 4 * c));
            __builtin_amdgcn_sched_barrier(0x1f);
        };
        read(0);
#pragma unroll
        for (int j = 0; j < NB; ++j) Q::decode(q[j], w[j]);
        // (before a wave that turns codes: 2048 tokens of 8 bits 222 us for 226; of 16 no gain)
        if (Q::kI8) __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            if (m + 1 < MT) read(m + 1);
            typename Q::Sum sum[NB];
            if constexpr (SUMS)
#pragma unroll
                for (int k = 0; k < Q::kSteps; ++k) bias[m & 1] = Q::mma(x[m & 1][k], minus8, bias[m & 1]);
#pragma unroll
            for (int k = 0; k < Q::kSteps; ++k)
#pragma unroll
                for (int j = 0; j < NB; ++j) sum[j] = Q::mma(x[m & 1][k], w[j][k], k ? sum[j] : bias[m & 1]);
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][j][i] = fmaf(s[j], static_cast<float>(sum[j][i]), acc[m][j][i]);
        }
        if (Q::kI8) __builtin_amdgcn_s_setprio(0);
        stage = stage == kAhead ? 0 : stage + 1;
    }
    __syncthreads();

    // Outputs (all scales asked for at once)
    const bool partial = p.partial != nullptr;
    f32x4 unit[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            unit[m][i] = Q::kI8 ? (partial ? 1.0f : p.x_scales[tok0 + min(16 * m + 4 * c + i, toks - 1)]) : Q::kUnit;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[m][j] *= unit[m];
    const int64_t at = tok0 * p.N + rb0 * 16;
    uint8_t* mine = lds + wave * 16 * C::kPitch;
    if (partial)
        store_tiles<MT, NB>(p.partial + sp * tb.M * p.N + at, p.N, acc, toks, 16 * rbs, mine, lane);
    else if (tb.y_dtype == UNISVQ_F32)
        store_tiles<MT, NB>(static_cast<float*>(p.y) + at, p.N, acc, toks, 16 * rbs, mine, lane);
    else if (tb.y_dtype == UNISVQ_F16)
        store_tiles<MT, NB>(static_cast<_Float16*>(p.y) + at, p.N, acc, toks, 16 * rbs, mine, lane);
    else
        store_tiles<MT, NB>(static_cast<__bf16*>(p.y) + at, p.N, acc, toks, 16 * rbs, mine, lane);
}

// Sums of the parts of a K that was split, in their order; four columns a thread,
// four parts asked for at a time (one after the other 16 tokens of 8192 rows in
// four parts took 4.5 us, now 4.0).
struct JoinBatch {
    TileProb p[kMaxBatch];
    int64_t begin[kMaxBatch];
    int count, y_dtype, i8;
    int64_t M;
};

__global__ __launch_bounds__(256) void join_kernel(const JoinBatch b) {
    TileProb p = b.p[0];
    int64_t begin = b.begin[0];
#pragma unroll
    for (int i = 1; i < kMaxBatch; ++i)
        if (i < b.count && blockIdx.x >= b.begin[i]) p = b.p[i], begin = b.begin[i];
    const int64_t at = ((blockIdx.x - begin) * 256 + threadIdx.x) * 4, part = b.M * p.N;
    if (at >= part) return;
    const float unit = b.i8 ? p.x_scales[at / p.N] : 1.0f;  // (N is a multiple of four)
    f32x4 sum{};
    for (int s = 0; s < p.splits; s += 4) {
        f32x4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const f32x4*>(p.partial + min(s + i, p.splits - 1) * part + at);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (s + i < p.splits) sum += v[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) store_out(p.y, at + i, sum[i] * unit, b.y_dtype);
}

// How a batch is split: tokens and rows of a workgroup, and parts of K.
struct Plan {
    int mt, nb;  // a workgroup has 16 mt tokens and 64 nb rows
    int splits[kMaxBatch];
    bool split, sums;  // whether any K is split, and the product makes its own sums
    double us;
};

// Times of a group of columns in us where memory does not hold it up, [i8][sums made
// here, given][nb 2, 4][mt 1, 2, 3, 4, 5, 6, 8]: a CU with one workgroup (the slope over K of
// calls with 128 workgroups), and with two (of calls whose token tiles share weights).
// 0: not a variant, as other tiles or sums were faster on all or nearly all shapes.
constexpr int kTileTokens[] = {1, 2, 3, 4, 5, 6, 8};
constexpr float kAlone[2][2][2][7] = {
    {{{0.43f, 0.54f, 0.67f, 0.77f, 0.90f, 1.01f, 0}, {0.62f, 0.77f, 0.97f, 1.18f, 1.39f, 1.60f, 0}},
     {{0, 0, 0.66f, 0.75f, 0.87f, 0, 0}, {0, 0, 0.92f, 1.06f, 1.37f, 1.44f, 0}}},
    {{{0.37f, 0.46f, 0.54f, 0.57f, 0.69f, 0.73f, 0}, {0.55f, 0.65f, 0.73f, 0.87f, 1.00f, 1.12f, 0}},
     {{0, 0, 0, 0.60f, 0.68f, 0.75f, 0}, {0, 0, 0, 0.82f, 0.94f, 1.06f, 1.28f}}}};
constexpr float kPaired[2][2][2][7] = {
    {{{0.60f, 0.85f, 1.05f, 1.28f, 1.50f, 1.80f, 0}, {1.10f, 1.40f, 1.70f, 2.10f, 2.60f, 3.05f, 0}},
     {{0, 0, 0.92f, 1.05f, 1.25f, 0, 0}, {0, 0, 1.50f, 1.92f, 2.40f, 2.65f, 0}}},
    {{{0.50f, 0.55f, 0.62f, 0.75f, 0.85f, 1.05f, 0}, {0.80f, 0.90f, 1.02f, 1.25f, 1.55f, 1.85f, 0}},
     {{0, 0, 0, 0.70f, 0.80f, 0.95f, 0}, {0, 0, 0, 1.20f, 1.50f, 1.80f, 2.36f}}}};

// The plan with the least expected time: what the workgroups take, two to a CU, or
// the weights' read (4.2 TB/s to 256 workgroups, 5.0 to 384, 5.8 above); 3 to 9 us to
// start and end; a launch for the sums of activations, where they are given; parts of K
// and the launch that joins them.  Of 162 calls of 17 to 4096 tokens the plan took at most
// 5% more than the fastest of up to 24 others on 134, at most 10% more on 146.  The rest are
// mostly of 1025 to 1535 workgroups, whose third round costs more than the share of a round
// that is counted (12 of the 17 such calls more than 10%): 256 tokens of 8 bits, 22016 rows
// of 4096, 1032 workgroups 65.9 us, tiles of 64 x 256 with given sums 41.7; of 16 bits 80.6
// and 61.5.
Plan plan_of(const FourbitProblem* probs, int count, int64_t M, bool i8) {
    Plan best{};
    best.us = 1e30;
    double read = 0, weights = 0;
    for (int i = 0; i < count; ++i) {
        read = std::max(read, static_cast<double>(M * probs[i].K) * (i8 ? 1 : 2));
        weights += static_cast<double>(fourbit_bytes(probs[i].N, probs[i].K));
    }
    for (int n = 0; n < 2; ++n)
        for (int m = 0; m < (i8 ? 7 : 6); ++m) {
            const int mt = kTileTokens[m], nb = 2 * (n + 1);
            const int64_t BM = 16 * mt, BN = 64 * nb, m_tiles = (M + BM - 1) / BM;
            if (m && 16 * kTileTokens[m - 1] >= M) break;  // (a smaller one has all tokens)
            int64_t tiles = 0;
            for (int i = 0; i < count; ++i) tiles += (probs[i].N + BN - 1) / BN * m_tiles;
            for (int splits = 1; splits == 1 || (splits <= 12 && tiles * splits <= 2 * kCUs); ++splits) {
                Plan p{mt, nb, {}, false, false, 0};
                int64_t wgs = 0;
                int groups = 0;
                double parts = 0;
                for (int i = 0; i < count; ++i) {
                    const int g = static_cast<int>(probs[i].K / kGroup);
                    p.splits[i] = std::max(1, std::min(splits, g / 4));
                    p.split |= p.splits[i] > 1;
                    wgs += (probs[i].N + BN - 1) / BN * m_tiles * p.splits[i];
                    groups = std::max(groups, (g + p.splits[i] - 1) / p.splits[i]);
                    if (p.splits[i] > 1) parts += 8.0 * p.splits[i] * static_cast<double>(M * probs[i].N);
                }
                // up to two rounds are rounds; of more, workgroups begin as others end
                const int64_t rest = wgs % (2 * kCUs);
                const double rate = wgs > 3 * kCUs / 2 ? 5.8e6 : wgs > kCUs ? 5.0e6 : 4.2e6;
                for (int given = 0; given < 2; ++given) {
                    const double alone = kAlone[i8][given][n][m], paired = kPaired[i8][given][n][m];
                    if (alone == 0) continue;
                    const double last = rest > kCUs ? paired : rest ? alone : 0.0;
                    const double rounds = wgs > 4 * kCUs ? 0.97 * static_cast<double>(wgs) / (2 * kCUs) * paired
                                                         : static_cast<double>(wgs / (2 * kCUs)) * paired + last;
                    p.sums = given == 0;
                    p.us = 2.8 + 0.2 * mt * nb + std::max(groups * rounds, weights / rate) +
                           (given ? 2.6 + read / 4e6 : 0.0) + (p.split ? 2.5 + parts / 6e6 : 0.0);
                    if (p.us < best.us) best = p;
                }
            }
        }
    return best;
}

// No output shares memory with another operand of the batch, nor does the workspace.
// (Looked at once its size is known; a batch that fits a grid has less than 2^42 bytes of outputs.)
bool apart(const FourbitProblem* probs, int count, int64_t M, int size, int y_dtype, const void* workspace, size_t room) {
    const int64_t out = y_dtype == UNISVQ_F32 ? 4 : 2, ws = static_cast<int64_t>(room);
    for (int i = 0; i < count; ++i) {
        const int64_t y_bytes = M * probs[i].N * out;
        if (bytes_meet(probs[i].y, y_bytes, workspace, ws)) return false;
        for (int j = 0; j < count; ++j) {
            const FourbitProblem& p = probs[j];
            if (bytes_meet(probs[i].y, y_bytes, p.x, M * p.K * size) || bytes_meet(probs[i].y, y_bytes, p.x_scales, 4 * M) ||
                bytes_meet(probs[i].y, y_bytes, p.packed, fourbit_bytes(p.N, p.K)) ||
                (i < j && bytes_meet(probs[i].y, y_bytes, p.y, M * p.N * out)))
                return false;
        }
        if (bytes_meet(workspace, ws, probs[i].x, M * probs[i].K * size) || bytes_meet(workspace, ws, probs[i].x_scales, 4 * M) ||
            bytes_meet(workspace, ws, probs[i].packed, fourbit_bytes(probs[i].N, probs[i].K)))
            return false;
    }
    return true;
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

// A batch's workspace: sums of each distinct x, then parts of the problems whose K is split.
struct Places {
    size_t bias[kMaxBatch], partial[kMaxBatch], bytes;
    bool first[kMaxBatch];
};

Places places_of(const FourbitProblem* probs, int count, int64_t M, const Plan& plan) {
    Places p{};
    for (int i = 0; i < count; ++i) {
        // (without addresses, for the size alone, every x counts as another)
        int same = i;
        for (int j = i - 1; j >= 0; --j)
            if (probs[i].x && probs[j].x == probs[i].x && probs[j].K == probs[i].K) same = j;
        p.first[i] = same == i;
        p.bias[i] = p.first[i] ? p.bytes : p.bias[same];
        if (p.first[i] && !plan.sums) p.bytes += static_cast<size_t>((M + kSumTile - 1) / kSumTile * (probs[i].K / kGroup)) * kSumTile * 4;
    }
    for (int i = 0; i < count; ++i)
        if (plan.splits[i] > 1) {
            p.partial[i] = p.bytes;
            p.bytes += up256(static_cast<size_t>(plan.splits[i]) * M * probs[i].N * 4);
        }
    return p;
}

template <typename X, int MT, int NB, bool SUMS>
int launch_tiles(const TileBatch& tb, uint32_t wgs, hipStream_t s) {
    tiled_kernel<X, MT, NB, SUMS><<<wgs, Tiled<X, MT, NB, SUMS>::kThreads, 0, s>>>(tb);
    return hipGetLastError() == hipSuccess ? UNISVQ_OK : UNISVQ_EHIP;
}

template <typename X, int NB, bool SUMS, int I = 0>
int launch_tokens(int mt, const TileBatch& tb, uint32_t wgs, hipStream_t s) {
    if constexpr (I < 7) {
        if constexpr (kAlone[Kind<X>::kI8][!SUMS][NB / 2 - 1][I] > 0)
            if (mt == kTileTokens[I]) return launch_tiles<X, kTileTokens[I], NB, SUMS>(tb, wgs, s);
        return launch_tokens<X, NB, SUMS, I + 1>(mt, tb, wgs, s);
    }
    return UNISVQ_EUNSUP;
}

template <typename X>
int launch_tiled(const FourbitProblem* probs, int count, int64_t M, int y_dtype, uint8_t* workspace, size_t room, hipStream_t s) {
    const Plan plan = plan_of(probs, count, M, Kind<X>::kI8);
    const Places at = places_of(probs, count, M, plan);
    if (at.bytes && (!workspace || room < at.bytes)) return UNISVQ_EWORKSPACE;
    if (at.bytes && (reinterpret_cast<uintptr_t>(workspace) & 15) != 0) return UNISVQ_EALIGN;
    TileBatch tb{};
    tb.count = count, tb.y_dtype = y_dtype, tb.M = M;
    const int64_t BM = 16 * plan.mt, BN = 64 * plan.nb, m_tiles = (M + BM - 1) / BM;
    int64_t wgs = 0;
    for (int i = 0; i < count; ++i) {
        tb.p[i] = TileProb{probs[i].packed, probs[i].x, workspace + at.bias[i], probs[i].x_scales, probs[i].y,
                           plan.splits[i] > 1 ? reinterpret_cast<float*>(workspace + at.partial[i]) : nullptr, probs[i].N,
                           static_cast<int>(probs[i].K), plan.splits[i], static_cast<int>(wgs)};
        wgs += (probs[i].N + BN - 1) / BN * m_tiles * plan.splits[i];
        if (wgs >= int64_t{1} << 24) return UNISVQ_EUNSUP;  // (a grid has below 2^32 threads)
    }
    if (!apart(probs, count, M, Kind<X>::kBytes, y_dtype, at.bytes ? workspace : nullptr, at.bytes)) return UNISVQ_EINVAL;
    tb.m_tiles = static_cast<int>(m_tiles);
    for (int i = 0; i < count; ++i)
        if (at.first[i] && !plan.sums) {
            const int groups = static_cast<int>(probs[i].K / kGroup);
            const Sums a{probs[i].x, workspace + at.bias[i], M, groups};
            sums_kernel<X><<<static_cast<uint32_t>(std::min<int64_t>((M * groups + 15) / 16, 1 << 20)), 256, 0, s>>>(a);
        }
    const uint32_t grid = static_cast<uint32_t>(wgs);
    int st;
    if (plan.nb == 2)
        st = plan.sums ? launch_tokens<X, 2, true>(plan.mt, tb, grid, s) : launch_tokens<X, 2, false>(plan.mt, tb, grid, s);
    else
        st = plan.sums ? launch_tokens<X, 4, true>(plan.mt, tb, grid, s) : launch_tokens<X, 4, false>(plan.mt, tb, grid, s);
    if (st != UNISVQ_OK || !plan.split) return st;
    JoinBatch jb{};
    jb.y_dtype = y_dtype, jb.i8 = Kind<X>::kI8, jb.M = M;
    wgs = 0;
    for (int i = 0; i < count; ++i)
        if (plan.splits[i] > 1) {
            jb.p[jb.count] = tb.p[i];
            jb.begin[jb.count++] = wgs;
            wgs += (M * probs[i].N / 4 + 255) / 256;
        }
    if (!jb.count) return UNISVQ_OK;
    join_kernel<<<static_cast<uint32_t>(wgs), 256, 0, s>>>(jb);
    return hipGetLastError() == hipSuccess ? UNISVQ_OK : UNISVQ_EHIP;
}

// Which kernel serves a batch.
// x in LDS: up to four tokens, where it fits; up to eight of 16 bits on 2048 to 4096
// columns, of 4097 to 24576 rows (8 tokens, 8192 rows of 4096: 7.8 us, tiles 9.7; 22016
// rows: 14.0, 16.4; 28672 rows of 2048: 10.8, 9.9; 22016 of 5120: 17.1, 16.5; 22016 of 2048:
// 9.6, 9.9, of 1920 9.6, 9.5, and of 2176, a share of threes with a third empty, 11.2, 10.4;
// 11008 of 2048: 7.9, 8.9, of 1920 8.0, 9.0).
// Else up to sixteen tokens without a second launch, every workgroup with x from the L2:
// 4096 rows while x is at most 128 KB (16 bits, 1024 rows: 16 tokens of 4096 columns 7.2 us,
// tiles 7.0, of 6144 9.7 and 7.6; 8 of 8192 8.7 and 8.2; 8 bits, 16 of 8192 7.9 and 8.3, of
// 12288 10.1 and 9.1), and 8192 rows, two workgroups to a CU, while it is at most 32 KB, of
// 8 bits 64 (16 tokens of 16 bits, 1024 columns 5.5 us, tiles 5.9, 2048 8.2 and 7.7; of 8
// bits, 4096 8.9 and 10.1, 6144 11.5 and 11.0).
// Else tiles.
enum Way { kFew, kSome, kTiled };

Way way_of(const FourbitProblem* probs, int count, int64_t M, int size) {
    int64_t most = 0, blocks = 0;
    for (int i = 0; i < count; ++i) most = std::max(most, probs[i].K), blocks += probs[i].N / kRowBlock;
    const bool eight = M <= 8 && size == 2 && blocks > kCUs && blocks <= 6 * kCUs && most >= 2048 && most <= 4096;
    if ((M <= 4 || eight) && blocks < (1 << 30) && few_lds_bytes(most, tok_of(M), 16, size) <= kMostLds) return kFew;
    if (M > 16 || blocks > 2 * kCUs) return kTiled;
    return M * most * size <= (blocks <= kCUs ? 131072 : size == 1 ? 65536 : 32768) ? kSome : kTiled;
}

template <typename X>
int launch_kind(const FourbitProblem* probs, int count, int64_t M, int y_dtype, uint8_t* workspace, size_t room, hipStream_t s) {
    const Way way = way_of(probs, count, M, Kind<X>::kBytes);
    if (way == kTiled) return launch_tiled<X>(probs, count, M, y_dtype, workspace, room, s);
    if (!apart(probs, count, M, Kind<X>::kBytes, y_dtype, nullptr, 0)) return UNISVQ_EINVAL;
    Batch b{};
    b.count = count, b.y_dtype = y_dtype, b.M = M;
    int64_t most = 0;
    for (int i = 0; i < count; ++i) {
        b.p[i] = Prob{probs[i].packed, probs[i].x, probs[i].x_scales, probs[i].y, probs[i].N, static_cast<int>(probs[i].K), 0, 0};
        most = std::max(most, probs[i].K);
    }
    if (way == kSome) return launch_some<X>(b, s);
    const int tok = tok_of(M);
    if constexpr (!Kind<X>::kI8)
        if (tok == 8) return launch_few<X, 8>(b, most, s);
    return tok == 1 ? launch_few<X, 1>(b, most, s) : tok == 2 ? launch_few<X, 2>(b, most, s) : launch_few<X, 4>(b, most, s);
}

}  // namespace

size_t fourbit_workspace_bytes(const FourbitProblem* probs, int count, int64_t M, int x_dtype) {
    const bool i8 = x_dtype == UNISVQ_I8;
    if (way_of(probs, count, M, i8 ? 1 : 2) != kTiled) return 0;
    return places_of(probs, count, M, plan_of(probs, count, M, i8)).bytes;
}

int launch_fourbit_batch(const FourbitProblem* probs, int count, int64_t M, int x_dtype, int y_dtype, void* workspace,
                         size_t workspace_bytes, hipStream_t s) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (x_dtype == UNISVQ_F16) return launch_kind<_Float16>(probs, count, M, y_dtype, ws, workspace_bytes, s);
    if (x_dtype == UNISVQ_BF16) return launch_kind<__bf16>(probs, count, M, y_dtype, ws, workspace_bytes, s);
    return launch_kind<int8_t>(probs, count, M, y_dtype, ws, workspace_bytes, s);
}

}  // namespace unisvq
