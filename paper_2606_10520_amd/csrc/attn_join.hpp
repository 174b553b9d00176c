// Joining the parts of split attention rows: every part has a maximum m_p
// (log2), a sum l_p and the sums o_p of its weighted values, and
//   m = max m_p,  l = sum 2^(m_p - m) l_p,  out = sum 2^(m_p - m) o_p / l.
// Bound by reading the parts.  Sixteen lanes have a row (eight or four dims
// each), in the order of the parts, so a result does not depend on timing.
#pragma once

#include <cfloat>

#include "attn.hpp"

namespace unisvq {

struct Join {
    const float* part;      // [rows][splits][D]
    const float2* part_ml;  // [rows][splits]
    int64_t rows;           // tokens * q_heads
    int splits, q_heads;
    Rows out;
    float* lse;             // [rows] or null
    const int32_t* tokens;  // rows of tokens from *tokens on are left alone; null: there are none
    // Parts that there are of a row: those that begin before the length of its
    // sequence (of q_len tokens); null: all.
    const int32_t* lens;
    int q_len, chunk;
};

namespace {

constexpr float kJoinLn2 = 0.69314718055994530942f;

template <int D, typename T>
__global__ __launch_bounds__(256) void join_kernel(Join j) {
    constexpr int kDims = D / 16;
    const int64_t r = static_cast<int64_t>(blockIdx.x) * 16 + threadIdx.x / 16;
    if (r >= j.rows) return;
    const int at = threadIdx.x % 16;
    const int64_t token = r / j.q_heads;
    const int head = static_cast<int>(r - token * j.q_heads);
    if (j.tokens && token >= *j.tokens) return;
    int n = j.splits;
    if (j.lens) n = min(n, max(0, j.lens[token / j.q_len] - 1) / j.chunk + 1);
    const float2* ml = j.part_ml + r * j.splits;
    float m = -FLT_MAX;
    for (int x = at; x < n; x += 16) m = fmaxf(m, ml[x].x);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    const float* part = j.part + r * j.splits * D + at * kDims;
    float l = 0.0f, f[kDims] = {};
#pragma unroll 4
    for (int x = 0; x < n; ++x) {
        const float2 here = ml[x];
        float v[kDims];
#pragma unroll
        for (int y = 0; y < kDims; y += 4) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(part + static_cast<int64_t>(x) * D + y);
#pragma unroll
            for (int z = 0; z < 4; ++z) v[y + z] = q[z];
        }
        // (a part that saw nothing has written no sums)
        const bool some = here.y != 0.0f;
        const float c = some ? __builtin_amdgcn_exp2f(here.x - m) : 0.0f;
        l += c * here.y;
#pragma unroll
        for (int y = 0; y < kDims; ++y) f[y] += some ? c * v[y] : 0.0f;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    typedef T TN __attribute__((ext_vector_type(kDims)));
    TN out;
#pragma unroll
    for (int y = 0; y < kDims; ++y) out[y] = static_cast<T>(f[y] * inv);
    *reinterpret_cast<TN*>(static_cast<T*>(j.out.p) + token * j.out.ts + head * j.out.hs + at * kDims) = out;
    if (j.lse && at == 0) j.lse[r] = (m + log2f(l)) * kJoinLn2;
}

template <int D, typename T>
hipError_t launch_join(const Join& j, hipStream_t s) {
    join_kernel<D, T><<<static_cast<uint32_t>((j.rows + 15) / 16), 256, 0, s>>>(j);
    return hipGetLastError();
}

}  // namespace

}  // namespace unisvq
