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

struct Prob {
    const uint8_t* packed;
    const void* x;
    const float* x_scales;
    void* y;
    int64_t N;
    int K, wg_begin;
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
    static constexpr int kSteps = 4, kBytes = 2;      // products a group, bytes an element
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

// Few tokens: a workgroup has RB blocks of 16 rows and MT tiles of 16 tokens, its
// waves share K out in runs of groups, and their sums meet in LDS.
template <typename X, int MT, int RB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(const Batch b) {
    typedef Kind<X> Q;
    __shared__ f32x4 parts[WAVES][RB * MT][64];
    Prob p = b.p[0];
#pragma unroll
    for (int i = 1; i < kMaxBatch; ++i)
        if (i < b.count && static_cast<int>(blockIdx.x) >= b.p[i].wg_begin) p = b.p[i];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, c = lane >> 4;
    const int64_t blocks = p.N / kRowBlock;
    const int64_t L = static_cast<int>(blockIdx.x) - p.wg_begin, across = (blocks + RB - 1) / RB;
    const int64_t rb0 = L % across * RB, tok0 = L / across * (16 * MT);
    const int K = p.K, groups = K / kGroup, quads = (groups + 3) / 4;
    const int rbs = static_cast<int>(min(static_cast<int64_t>(RB), blocks - rb0));
    const int toks = static_cast<int>(min(static_cast<int64_t>(16 * MT), b.M - tok0));
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(p.packed + rb0 * groups * kFourbitTile, static_cast<uint32_t>(rbs) * groups * kFourbitTile);
    const __amdgpu_buffer_rsrc_t rs =
        make_rsrc(p.packed + p.N * (K / 2) + rb0 * quads * kFourbitQuad, static_cast<uint32_t>(rbs) * quads * kFourbitQuad);
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(static_cast<const uint8_t*>(p.x) + tok0 * K * Q::kBytes,
                                                static_cast<uint32_t>(toks) * K * Q::kBytes);
    const int g0 = groups * wave / WAVES, g1 = groups * (wave + 1) / WAVES;

    struct Step {
        uint4 q[RB], x[MT][Q::kSteps];
        uint32_t s[RB];
    };
    const auto load = [&](int g, Step& t) {
        const uint32_t out = g < g1 ? 0u : kOutOfRange;
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            t.q[r] = ld128_stream(rw, out | static_cast<uint32_t>((r * groups + g) * kFourbitTile + 16 * lane));
            t.s[r] = ld16(rs, out | static_cast<uint32_t>((r * quads + (g >> 2)) * kFourbitQuad + 8 * n + 2 * (g & 3)));
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < Q::kSteps; ++j)
                t.x[m][j] = ld128(rx, out | (static_cast<uint32_t>((16 * m + n) * K + g * kGroup) * Q::kBytes + Q::kChunk * c + Q::at(j)));
    };
    f32x4 acc[RB][MT] = {};
    const typename Q::Operand minus8 = Q::minus8();
    const auto compute = [&](const Step& t) {
        typename Q::Sum bias[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            bias[m] = typename Q::Sum{};
#pragma unroll
            for (int j = 0; j < Q::kSteps; ++j)
                bias[m] = Q::mma(__builtin_bit_cast(typename Q::Operand, t.x[m][j]), minus8, bias[m]);
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            typename Q::Operand w[Q::kSteps];
            Q::decode(t.q[r], w);
            const float s = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(t.s[r])));
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                typename Q::Sum sum = bias[m];
#pragma unroll
                for (int j = 0; j < Q::kSteps; ++j) sum = Q::mma(__builtin_bit_cast(typename Q::Operand, t.x[m][j]), w[j], sum);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[r][m][i] = fmaf(s, static_cast<float>(sum[i]), acc[r][m][i]);
            }
        }
    };
    Step even, odd;
    load(g0, even);
    for (int g = g0; g < g1; g += 2) {
        load(g + 1, odd);
        compute(even);
        load(g + 2, even);
        if (g + 1 < g1) compute(odd);
    }

#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) parts[wave][r * MT + m][lane] = acc[r][m];
    __syncthreads();
    for (int i = threadIdx.x; i < RB * MT * 64; i += 64 * WAVES) {
        const int tile = i >> 6, at = i & 63;
        f32x4 sum = parts[0][tile][at];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += parts[w][tile][at];
        const int r = tile / MT, row = at & 15, t0 = 16 * (tile % MT) + 4 * (at >> 4);
        if (r >= rbs) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (t0 + j < toks) {
                const int64_t t = tok0 + t0 + j;
                const float unit = Q::kI8 ? p.x_scales[t] : Q::kUnit;
                store_out(p.y, t * p.N + (rb0 + r) * kRowBlock + row, sum[j] * unit, b.y_dtype);
            }
    }
}

template <typename X, int MT, int RB, int WAVES>
int launch_few(Batch b, hipStream_t s) {
    int64_t blocks = 0;
    for (int i = 0; i < b.count; ++i) {
        b.p[i].wg_begin = static_cast<int>(blocks);
        blocks += (b.p[i].N / kRowBlock + RB - 1) / RB * ((b.M + 16 * MT - 1) / (16 * MT));
        if (blocks > (int64_t{1} << 32) / (64 * WAVES) - 1) return UNISVQ_EUNSUP;
    }
    few_kernel<X, MT, RB, WAVES><<<static_cast<uint32_t>(blocks), 64 * WAVES, 0, s>>>(b);
    return hipGetLastError() == hipSuccess ? UNISVQ_OK : UNISVQ_EHIP;
}

// ---- many tokens ----
// -8 times the sums of every token's groups, bias[token / 32][group][token % 32]
// (fp32, or i8's integers), sixteen lanes a sum: what the tiled product's sums of
// a group start from.
constexpr int kSumTile = 32;

struct Sums {
    const void* x;
    void* bias;
    int64_t M;
    int groups;
};

template <typename X>
__global__ __launch_bounds__(256) void sums_kernel(Sums a) {
    const int64_t i = blockIdx.x * 16ll + (threadIdx.x >> 4), count = a.M * a.groups;
    const int64_t at = min(i, count - 1), t = at / a.groups, g = at - t * a.groups;
    const int64_t to = (t / kSumTile * a.groups + g) * kSumTile + t % kSumTile;
    const int64_t from = t * a.groups * kGroup + g * kGroup + 8 * (threadIdx.x & 15);
    if constexpr (std::is_same_v<X, int8_t>) {
        const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(a.x) + from);
        int sum = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) sum += static_cast<int8_t>(v.x >> 8 * b) + static_cast<int8_t>(v.y >> 8 * b);
        sum = over_lanes(sum, 4, [](int p, int q) { return p + q; });
        if ((threadIdx.x & 15) == 0 && i < count) static_cast<int*>(a.bias)[to] = -8 * sum;
    } else {
        float f[8], sum = 0.0f;
        load8(static_cast<const X*>(a.x) + from, f);
#pragma unroll
        for (int b = 0; b < 8; ++b) sum += f[b];
        sum = over_lanes(sum, 4, [](float p, float q) { return p + q; });
        if ((threadIdx.x & 15) == 0 && i < count)
            static_cast<float*>(a.bias)[to] = -8.0f / Kind<X>::kUnit * sum;
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

// A workgroup has WM x WN waves, a wave 16 MT tokens x 16 NB rows.  A group of
// columns at a time goes to LDS by direct loads, two groups deep: activations in
// rows whose 16-byte chunks are turned by the row (so that sixteen rows' same
// chunk lies in sixteen places), codes as they are, scales and sums.  A wave turns
// its rows' codes into operands once and passes over its tokens with them.
template <typename X, int MT, int NB, int WM, int WN>
struct Tiled {
    typedef Kind<X> Q;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int BM = 16 * MT * WM, BN = 16 * NB * WN;
    static constexpr int kRow = kGroup * Q::kBytes;            // bytes of a token's group
    static constexpr int kX = BM * kRow, kCodes = BN * 64, kScales = BN * 8;
    static constexpr int kBias = (BM * 4 + 1023) / 1024 * 1024;  // (whole loads: what is behind the tokens becomes zeros)
    static constexpr int kStage = kX + kCodes + kScales + kBias;
    static constexpr int kLoadsX = kX / (16 * kThreads), kLoadsCodes = kCodes / (16 * kThreads);
    static_assert(kX % (16 * kThreads) == 0 && kCodes % (16 * kThreads) == 0, "");
    static constexpr int kWavesScales = kScales / 1024, kWavesBias = kBias / 1024;
    static_assert(kScales % 1024 == 0 && kWavesScales + kWavesBias <= kWaves, "");
    // a wave's outputs of one tile of tokens, staged for whole-line stores
    static constexpr int kPitch = 16 * NB * 4 + 16;
    static_assert(kWaves * 16 * kPitch <= 2 * kStage, "");
};

template <typename X, int MT, int NB, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void tiled_kernel(const TileBatch tb) {
    typedef Tiled<X, MT, NB, WM, WN> C;
    typedef typename C::Q Q;
    __shared__ __attribute__((aligned(16))) uint8_t lds[2][C::kStage];
    TileProb p = tb.p[0];
#pragma unroll
    for (int i = 1; i < kMaxBatch; ++i)
        if (i < tb.count && static_cast<int>(blockIdx.x) >= tb.p[i].wg_begin) p = tb.p[i];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, c = lane >> 4, wm = wave % WM, wn = wave / WM;
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
    const int64_t tok0 = static_cast<int64_t>(mt) * C::BM, rb0 = static_cast<int64_t>(nt) * (C::BN / 16);
    const int toks = static_cast<int>(min(static_cast<int64_t>(C::BM), tb.M - tok0));
    const int rbs = static_cast<int>(min(static_cast<int64_t>(C::BN / 16), blocks - rb0));
    const int g0 = __builtin_amdgcn_readfirstlane(groups * sp / p.splits);
    const int g1 = __builtin_amdgcn_readfirstlane(groups * (sp + 1) / p.splits);

    const __amdgpu_buffer_rsrc_t rx = make_rsrc(static_cast<const uint8_t*>(p.x) + tok0 * K * Q::kBytes,
                                                static_cast<uint32_t>(toks) * K * Q::kBytes);
    const __amdgpu_buffer_rsrc_t rw = make_rsrc(p.packed + rb0 * groups * kFourbitTile, static_cast<uint32_t>(rbs) * groups * kFourbitTile);
    const __amdgpu_buffer_rsrc_t rs =
        make_rsrc(p.packed + p.N * (K / 2) + rb0 * quads * kFourbitQuad, static_cast<uint32_t>(rbs) * quads * kFourbitQuad);
    const __amdgpu_buffer_rsrc_t rb = make_rsrc(static_cast<const uint8_t*>(p.bias) + tok0 * groups * 4,
                                                static_cast<uint32_t>((toks + kSumTile - 1) / kSumTile * groups * kSumTile * 4));

    // Places past the last token or row read the last one again: they are not stored.
    constexpr int kChunks = C::kRow / 16, kTurn = Q::kI8 ? 1 : 0;  // a row's chunk j lies at j ^ ((row >> kTurn) % kChunks)
    uint32_t off_x[C::kLoadsX];
#pragma unroll
    for (int i = 0; i < C::kLoadsX; ++i) {
        const int at = i * C::kThreads + threadIdx.x, row = at / kChunks, chunk = at % kChunks ^ (row >> kTurn) % kChunks;
        off_x[i] = static_cast<uint32_t>(min(row, toks - 1)) * K * Q::kBytes + 16 * chunk;
    }
    const uint32_t at16[1] = {16u * lane};
    uint32_t off_s[1], off_b[1];
    const bool has_scales = wave < C::kWavesScales, has_bias = wave >= C::kWaves - C::kWavesBias;
    {
        const int at = wave * 1024 + 16 * lane, r = at >> 7;
        off_s[0] = static_cast<uint32_t>(min(r, rbs - 1)) * quads * kFourbitQuad + (at & 127);
        const int t = (wave - (C::kWaves - C::kWavesBias)) * 256 + 4 * lane;
        off_b[0] = t < C::BM ? static_cast<uint32_t>(t / kSumTile * groups * kSumTile + t % kSumTile) * 4u : kOutOfRange;
    }
    const uint32_t base = __builtin_amdgcn_readfirstlane(
        static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)&lds[0][0])));
    const auto issue = [&](int g, int stage) {
        const uint32_t to = base + stage * C::kStage;
        load_lds<16 * C::kThreads>(to + wave * 1024, off_x, rx, static_cast<uint32_t>(g) * C::kRow);
#pragma unroll
        for (int i = 0; i < C::kLoadsCodes; ++i) {
            const int r = i * C::kWaves + wave;
            load_lds<0>(to + C::kX + r * 1024, at16, rw, static_cast<uint32_t>(min(r, rbs - 1) * groups + g) * kFourbitTile);
        }
        if (has_scales) load_lds<0>(to + C::kX + C::kCodes + wave * 1024, off_s, rs, static_cast<uint32_t>(g >> 2) * kFourbitQuad);
        if (has_bias)
            load_lds<0>(to + C::kX + C::kCodes + C::kScales + (wave - (C::kWaves - C::kWavesBias)) * 1024, off_b, rb,
                        static_cast<uint32_t>(g * kSumTile * 4));
    };

    f32x4 acc[MT][NB] = {};
    if (g0 < g1) issue(g0, 0);
    for (int g = g0; g < g1; ++g) {
        const int stage = (g - g0) & 1;
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");  // this group is there, the last one read by all
        __builtin_amdgcn_sched_barrier(0);
        if (g + 1 < g1) issue(g + 1, stage ^ 1);
        const uint8_t* from = lds[stage];
        typename Q::Operand w[NB][Q::kSteps];
        float s[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int r = wn * NB + j;
            Q::decode(*reinterpret_cast<const uint4*>(from + C::kX + r * 1024 + 16 * lane), w[j]);
            s[j] = static_cast<float>(*reinterpret_cast<const _Float16*>(from + C::kX + C::kCodes + r * 128 + 8 * n + 2 * (g & 3)));
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int row = (wm * MT + m) * 16 + n;
            typename Q::Operand x[Q::kSteps];
#pragma unroll
            for (int k = 0; k < Q::kSteps; ++k) {
                const int chunk = (Q::kChunk * c + Q::at(k)) / 16;
                x[k] = *reinterpret_cast<const typename Q::Operand*>(from + row * C::kRow + 16 * (chunk ^ (row >> kTurn) % kChunks));
            }
            const typename Q::Sum bias = *reinterpret_cast<const typename Q::Sum*>(
                from + C::kX + C::kCodes + C::kScales + 4 * ((wm * MT + m) * 16 + 4 * c));
            typename Q::Sum sum[NB];
#pragma unroll
            for (int k = 0; k < Q::kSteps; ++k)
#pragma unroll
                for (int j = 0; j < NB; ++j) sum[j] = Q::mma(x[k], w[j][k], k ? sum[j] : bias);
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][j][i] = fmaf(s[j], static_cast<float>(sum[j][i]), acc[m][j][i]);
        }
    }
    __syncthreads();

    // Outputs: a tile of sixteen tokens at a time through the wave's own part of
    // LDS, and from there in pieces of 16 bytes of tokens' rows.
    const bool partial = p.partial != nullptr, wide = partial || tb.y_dtype == UNISVQ_F32;
    void* out = partial ? p.partial + sp * tb.M * p.N : p.y;
    const int y_dtype = partial ? UNISVQ_F32 : tb.y_dtype;
    const bool whole = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
    const int rows = min(16 * NB, (rbs - wn * NB) * 16);  // of the wave's that are there
    uint8_t* mine = &lds[0][0] + wave * 16 * C::kPitch;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int t0 = (wm * MT + m) * 16;
        float unit[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = min(t0 + 4 * c + i, toks - 1);
            unit[i] = Q::kI8 ? (partial ? 1.0f : p.x_scales[tok0 + t]) : Q::kUnit;
        }
        const int64_t at = (tok0 + t0) * p.N + (rb0 + wn * NB) * 16;
        if (!whole) {
#pragma unroll
            for (int j = 0; j < NB; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (16 * j < rows && t0 + 4 * c + i < toks)
                        store_out(out, at + (4 * c + i) * p.N + 16 * j + n, acc[m][j][i] * unit[i], y_dtype);
            continue;
        }
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) store_out(mine + (4 * c + i) * C::kPitch, 16 * j + n, acc[m][j][i] * unit[i], y_dtype);
        __builtin_amdgcn_wave_barrier();
        const int size = wide ? 4 : 2, pieces = 16 * NB * size / 16;  // of 16 bytes, a token
        for (int e = lane; e < 16 * pieces; e += 64) {
            const int t = e / pieces, piece = e % pieces;
            if (t0 + t < toks && piece * 16 < rows * size)
                *reinterpret_cast<uint4*>(static_cast<uint8_t*>(out) + (at + t * p.N) * size + 16 * piece) =
                    *reinterpret_cast<const uint4*>(mine + t * C::kPitch + 16 * piece);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Sums of the parts of a K that was split, in their order; four columns a thread.
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
    const int64_t at = ((blockIdx.x - begin) * 256 + threadIdx.x) * 4;
    if (at >= b.M * p.N) return;
    f32x4 sum = *reinterpret_cast<const f32x4*>(p.partial + at);
    for (int s = 1; s < p.splits; ++s) sum += *reinterpret_cast<const f32x4*>(p.partial + s * b.M * p.N + at);
    if (b.i8) sum *= p.x_scales[at / p.N];  // (N is a multiple of four)
#pragma unroll
    for (int i = 0; i < 4; ++i) store_out(p.y, at + i, sum[i], b.y_dtype);
}

// How a batch is split: tokens and rows of a workgroup, and parts of K.
constexpr int64_t kCUs = 256;
constexpr int64_t kFewTokens = 64;

struct Plan {
    int mt;      // token tiles of a wave: 2 mt tiles of 16 a workgroup, 256 rows
    int splits[kMaxBatch];
    bool split;
};

Plan plan_of(const FourbitProblem* probs, int count, int64_t M, bool i8) {
    Plan best{};
    double least = 1e30;
    for (int mt : {2, 4, 6, 8}) {
        if (mt == 8 && !i8) continue;  // (LDS)
        int64_t tiles = 0;
        for (int i = 0; i < count; ++i) tiles += (probs[i].N + 255) / 256 * ((M + 32 * mt - 1) / (32 * mt));
        for (int splits = 1; splits <= 8 && (splits == 1 || tiles < 2 * kCUs); ++splits) {
            int64_t wgs = 0;
            int groups = 0;
            Plan p{mt, {}, splits > 1};
            for (int i = 0; i < count; ++i) {
                const int g = static_cast<int>(probs[i].K / kGroup);
                p.splits[i] = std::max(1, std::min(splits, g / 4));
                wgs += (probs[i].N + 255) / 256 * ((M + 32 * mt - 1) / (32 * mt)) * p.splits[i];
                groups = std::max(groups, (g + p.splits[i] - 1) / p.splits[i]);
            }
            const double rounds = static_cast<double>((wgs + kCUs - 1) / kCUs);
            double outs = 0;
            for (int i = 0; i < count; ++i) outs += static_cast<double>(M * probs[i].N) * (p.splits[i] > 1 ? 8.0 * p.splits[i] : 0.0);
            const double us = rounds * (2.0 + groups * (0.4 + 0.25 * mt)) + (splits > 1 ? 3.0 + outs / 4e6 : 0.0);
            if (us < least) least = us, best = p;
        }
    }
    return best;
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
        if (p.first[i]) p.bytes += static_cast<size_t>((M + kSumTile - 1) / kSumTile * (probs[i].K / kGroup)) * kSumTile * 4;
    }
    for (int i = 0; i < count; ++i)
        if (plan.splits[i] > 1) {
            p.partial[i] = p.bytes;
            p.bytes += up256(static_cast<size_t>(plan.splits[i]) * M * probs[i].N * 4);
        }
    return p;
}

template <typename X, int MT>
int launch_tiles(TileBatch& tb, hipStream_t s) {
    typedef Tiled<X, MT, 4, 2, 4> C;
    int64_t wgs = 0;
    tb.m_tiles = static_cast<int>((tb.M + C::BM - 1) / C::BM);
    for (int i = 0; i < tb.count; ++i) {
        tb.p[i].wg_begin = static_cast<int>(wgs);
        wgs += (tb.p[i].N + C::BN - 1) / C::BN * tb.m_tiles * tb.p[i].splits;
        if (wgs > (int64_t{1} << 32) / C::kThreads - 1) return UNISVQ_EUNSUP;
    }
    tiled_kernel<X, MT, 4, 2, 4><<<static_cast<uint32_t>(wgs), C::kThreads, 0, s>>>(tb);
    return hipGetLastError() == hipSuccess ? UNISVQ_OK : UNISVQ_EHIP;
}

template <typename X>
int launch_most(int mt, TileBatch& tb, hipStream_t s) {
    if constexpr (Kind<X>::kI8)
        if (mt == 8) return launch_tiles<X, 8>(tb, s);
    return launch_tiles<X, 6>(tb, s);
}

template <typename X>
int launch_tiled(const FourbitProblem* probs, int count, int64_t M, int y_dtype, uint8_t* workspace, hipStream_t s) {
    const Plan plan = plan_of(probs, count, M, Kind<X>::kI8);
    const Places at = places_of(probs, count, M, plan);
    TileBatch tb{};
    tb.count = count, tb.y_dtype = y_dtype, tb.M = M;
    for (int i = 0; i < count; ++i) {
        const int groups = static_cast<int>(probs[i].K / kGroup);
        tb.p[i] = TileProb{probs[i].packed, probs[i].x, workspace + at.bias[i], probs[i].x_scales, probs[i].y,
                           plan.splits[i] > 1 ? reinterpret_cast<float*>(workspace + at.partial[i]) : nullptr, probs[i].N,
                           static_cast<int>(probs[i].K), plan.splits[i], 0};
        if (at.first[i]) {
            const Sums a{probs[i].x, workspace + at.bias[i], M, groups};
            sums_kernel<X><<<static_cast<uint32_t>((M * groups + 15) / 16), 256, 0, s>>>(a);
        }
    }
    const int st = plan.mt == 2 ? launch_tiles<X, 2>(tb, s) : plan.mt == 4 ? launch_tiles<X, 4>(tb, s)
                 : launch_most<X>(plan.mt, tb, s);
    if (st != UNISVQ_OK || !plan.split) return st;
    JoinBatch jb{};
    jb.y_dtype = y_dtype, jb.i8 = Kind<X>::kI8, jb.M = M;
    int64_t wgs = 0;
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

template <typename X>
int launch_kind(const FourbitProblem* probs, int count, int64_t M, int y_dtype, uint8_t* workspace, hipStream_t s) {
    if (M > kFewTokens) return launch_tiled<X>(probs, count, M, y_dtype, workspace, s);
    Batch b{};
    b.count = count, b.y_dtype = y_dtype, b.M = M;
    for (int i = 0; i < count; ++i)
        b.p[i] = Prob{probs[i].packed, probs[i].x, probs[i].x_scales, probs[i].y, probs[i].N, static_cast<int>(probs[i].K), 0};
    if (M <= 16) return launch_few<X, 1, 1, 8>(b, s);
    if (M <= 32) return launch_few<X, 2, 2, 8>(b, s);
    return launch_few<X, 4, 2, 8>(b, s);
}

}  // namespace

size_t fourbit_workspace_bytes(const FourbitProblem* probs, int count, int64_t M, int x_dtype) {
    return M > kFewTokens ? places_of(probs, count, M, plan_of(probs, count, M, x_dtype == UNISVQ_I8)).bytes : 0;
}

int launch_fourbit_batch(const FourbitProblem* probs, int count, int64_t M, int x_dtype, int y_dtype, void* workspace,
                         hipStream_t s) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    if (x_dtype == UNISVQ_F16) return launch_kind<_Float16>(probs, count, M, y_dtype, ws, s);
    if (x_dtype == UNISVQ_BF16) return launch_kind<__bf16>(probs, count, M, y_dtype, ws, s);
    return launch_kind<int8_t>(probs, count, M, y_dtype, ws, s);
}

}  // namespace unisvq
