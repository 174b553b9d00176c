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

template <typename X>
int launch_kind(const Batch& b, hipStream_t s) {
    if (b.M <= 16) return launch_few<X, 1, 1, 8>(b, s);
    if (b.M <= 32) return launch_few<X, 2, 2, 8>(b, s);
    return launch_few<X, 4, 2, 8>(b, s);
}

}  // namespace

size_t fourbit_workspace_bytes(const FourbitProblem*, int, int64_t, int) { return 0; }

int launch_fourbit_batch(const FourbitProblem* probs, int count, int64_t M, int x_dtype, int y_dtype, void*, hipStream_t s) {
    Batch b{};
    b.count = count, b.y_dtype = y_dtype, b.M = M;
    for (int i = 0; i < count; ++i)
        b.p[i] = Prob{probs[i].packed, probs[i].x, probs[i].x_scales, probs[i].y, probs[i].N, static_cast<int>(probs[i].K), 0};
    if (x_dtype == UNISVQ_F16) return launch_kind<_Float16>(b, s);
    if (x_dtype == UNISVQ_BF16) return launch_kind<__bf16>(b, s);
    return launch_kind<int8_t>(b, s);
}

}  // namespace unisvq
