// Internal declarations of what a decoder layer does beside attention and the
// products on 2- and 3-bit weights: norm, gated activations, and products on
// 4-bit weights (layer_api.hip validates; norm.hip, gated.hip, fourbit_pack.hip and
// fourbit_gemm.hip launch).
#pragma once

#include "attn.hpp"

namespace unisvq {

struct NormArgs {
    int64_t tokens;
    int n;
    const void *x, *w, *r;  // r: the residual stream, or null
    void *h, *y;            // h: the stream after the addition, null with r
    int64_t x_stride, r_stride, h_stride, y_stride;
    int x_dtype, w_dtype, r_dtype, y_dtype;
    float offset, eps;
    float* scales;  // of an I8 output
};
hipError_t launch_rmsnorm(const NormArgs& a, hipStream_t s);

struct GatedArgs {
    int64_t tokens;
    int n;
    const void *gate, *up;
    void* y;
    int64_t gate_stride, up_stride, y_stride;
    int x_dtype, y_dtype, act;
    float* scales;  // of an I8 output
};
hipError_t launch_gated(const GatedArgs& a, hipStream_t s);

// Longest row that a workgroup takes.
constexpr int kMaxRow = 65536;

// 4-bit weights: tiles of 16 rows x 128 columns of 1 KB, [row block][group],
// then the scales, 128 bytes a row block and four groups (see unisvq.h).
constexpr int kFourbitTile = 1024;
constexpr int kFourbitQuad = 128;
inline int64_t fourbit_code_bytes(int64_t N, int64_t K) { return N * (K / 2); }
inline int64_t fourbit_quads(int64_t K) { return (K / kGroup + 3) / 4; }
inline int64_t fourbit_bytes(int64_t N, int64_t K) { return fourbit_code_bytes(N, K) + N / kRowBlock * fourbit_quads(K) * kFourbitQuad; }

hipError_t launch_fourbit_pack(int64_t N, int64_t K, const uint8_t* codes, const uint16_t* scales, uint8_t* packed,
                          int32_t* bad, hipStream_t s);
hipError_t launch_fourbit_unpack(int64_t N, int64_t K, const uint8_t* packed, uint8_t* codes, uint16_t* scales,
                            hipStream_t s);
hipError_t launch_fourbit_quantize(int64_t N, int64_t K, const void* W, int w_dtype, uint8_t* packed, hipStream_t s);

// Whether na bytes at a and nb at b have one in common (absent operands have none).
inline bool bytes_meet(const void* a, int64_t na, const void* b, int64_t nb) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return p && q && p < q + static_cast<uintptr_t>(nb) && q < p + static_cast<uintptr_t>(na);
}

struct FourbitProblem {
    const uint8_t* packed;
    const void* x;
    const float* x_scales;  // of I8 activations
    void* y;
    int64_t N, K;
};
size_t fourbit_workspace_bytes(const FourbitProblem* probs, int count, int64_t M, int x_dtype);
// UNISVQ_OK, UNISVQ_EWORKSPACE or UNISVQ_EALIGN (the workspace), UNISVQ_EUNSUP where
// the launch would be too large, UNISVQ_EINVAL where an output or the workspace shares
// memory with another operand, or UNISVQ_EHIP.
int launch_fourbit_batch(const FourbitProblem* probs, int count, int64_t M, int x_dtype, int y_dtype, void* workspace,
                         size_t workspace_bytes, hipStream_t s);

// ---- device helpers ----

__device__ inline void load8(const float* p, float (&f)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = a[i], f[4 + i] = b[i];
}
__device__ inline void store8(float* p, const float (&f)[8]) {
    *reinterpret_cast<f32x4*>(p) = f32x4{f[0], f[1], f[2], f[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
}

// x combined with the same of the lanes that differ in the low bits of the
// lane number, 1 << steps lanes in all; every lane gets the result.
template <typename V, typename F>
__device__ inline V over_lanes(V x, int steps, F op) {
    const auto moved = [](V v, auto ctrl) {
        const int b = __builtin_bit_cast(int, v);
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(b, b, decltype(ctrl)::value, 0xf, 0xf, false));
    };
    if (steps > 0) x = op(x, moved(x, std::integral_constant<int, 0xb1>{}));   // the neighbour
    if (steps > 1) x = op(x, moved(x, std::integral_constant<int, 0x4e>{}));   // the other pair of four
    if (steps > 2) x = op(x, moved(x, std::integral_constant<int, 0x141>{}));  // the other four, mirrored
    if (steps > 3) x = op(x, moved(x, std::integral_constant<int, 0x140>{}));  // the other eight, mirrored
    if (steps > 4) {
        const unsigned b = __builtin_bit_cast(unsigned, x);
        const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
        const unsigned p = r[0], q = r[1];
        x = op(__builtin_bit_cast(V, p), __builtin_bit_cast(V, q));
    }
    if (steps > 5) {
        const unsigned b = __builtin_bit_cast(unsigned, x);
        const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
        const unsigned p = r[0], q = r[1];
        x = op(__builtin_bit_cast(V, p), __builtin_bit_cast(V, q));
    }
    return x;
}

// The same over all threads of a workgroup of whole waves, by way of sixteen
// words of LDS (other ones for each use); of operations that zero does not change.
template <typename V, typename F>
__device__ inline V over_block(V x, V* words, F op) {
    x = over_lanes(x, 6, op);
    const int waves = blockDim.x >> 6, lane = threadIdx.x & 15;
    if (waves == 1) return x;
    if ((threadIdx.x & 63) == 0) words[threadIdx.x >> 6] = x;
    __syncthreads();
    return over_lanes(lane < waves ? words[lane] : V{}, 4, op);
}

// A row held in 8 bits: code * scale, scale = a / 127 with a the largest
// magnitude; scale 0 where a < 1e-30, NaN (codes 0) where a value is not
// finite.  The same rule as the cache's.
struct RowScale {
    float scale, inv;
};
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }  // NaN above infinity
__device__ inline RowScale row_scale(uint32_t most) {
    const float a = __uint_as_float(most);
    const bool finite = most < 0x7f800000u, some = finite && a >= 1e-30f;
    const float scale = !finite ? __builtin_nanf("") : some ? a / 127.0f : 0.0f;
    return RowScale{scale, some ? 1.0f / scale : 0.0f};
}

// round-to-even(f * inv) of eight values in [-127, 127], as bytes: the sum with
// 1.5 * 2^23 rounds, and its low byte is the code in two's complement.  (The
// product is rounded by itself, as the rule has it.)
__device__ inline uint2 codes_of(const float (&f)[8], float inv) {
#pragma clang fp contract(off)
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float p = f[i] * inv;
        b[i] = inv > 0.0f ? __float_as_uint(p + 12582912.0f) : 0u;
    }
    uint2 q;
    q.x = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
    q.y = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[7], b[6], 0x0c0c0400u), __builtin_amdgcn_perm(b[5], b[4], 0x0c0c0400u), 0x05040100u);
    return q;
}

// Eight values stored as dtype (16 bits or 32).
template <typename T>
__device__ inline void store_row8(void* y, int64_t i, const float (&f)[8], bool wide) {
    if (wide)
        store8(static_cast<float*>(y) + i, f);
    else
        store8(static_cast<T*>(y) + i, f);
}

}  // namespace unisvq
