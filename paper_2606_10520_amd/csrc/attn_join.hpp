// Joining the parts of split attention rows: every part has a maximum m_p
// (log2), a sum l_p and the sums o_p of its weighted values, and
//   m = max m_p,  l = sum 2^(m_p - m) l_p,  out = sum 2^(m_p - m) o_p / l.
// Bound by the latency of a launch and, for many rows, by reading the parts.
// Sixteen lanes have a part of a row (eight or four dims each).  Where rows
// have more than sixteen parts (and so are few), sixteen such groups share a
// row, every sixteenth part each, and are joined through LDS: 64 rows of 64
// parts 6 us instead of 14, but 32 rows of 8 parts 5.2 us instead of 3.9.  The
// order goes by the parts alone, so a result does not depend on timing.
#pragma once

#include <cfloat>

#include "attn.hpp"

namespace unisvq {

struct Join {
    const float* part;      // [rows][slots][D]
    const float2* part_ml;  // [rows][slots]
    int64_t rows;           // tokens * q_heads
    int slots, q_heads;
    int expected;           // parts of a row, as the host knows lengths
    Rows out;
    float* lse;             // [rows] or null
    const int32_t* tokens;  // rows of tokens from *tokens on are left alone; null: there are none
    // Where rows have different numbers of parts (else null, and all slots are
    // theirs): before[b] counts the units of work of an item of sequences 0 ..
    // b - 1, and an item is the q_len tokens' `tile` rows of one of `items`
    // (key heads times row tiles).  Units are dealt out `share` a workgroup, in
    // order; an item within one share needs no joining.
    const int32_t* before;
    const int32_t* share;
    int q_len, group, items, row_tiles, tile;
};

// The shares that units first .. first + n - 1 lie in: the first, and how many.
struct Shares {
    int first, count;
};
__device__ inline Shares shares_of(int first, int n, int share) {
    const int a = first / share;
    return Shares{a, (first + n - 1) / share - a + 1};
}

namespace {

constexpr float kJoinLn2 = 0.69314718055994530942f;

template <int D, typename T, int GROUPS>
__global__ __launch_bounds__(256) void join_kernel(Join j) {
    constexpr int kDims = D / 16;
    const int64_t r = static_cast<int64_t>(blockIdx.x) * (16 / GROUPS) + threadIdx.x / (16 * GROUPS);
    const int group = threadIdx.x / 16 % GROUPS, at = threadIdx.x % 16;
    if (r >= j.rows) return;  // (with GROUPS > 1 a block has one row)
    const int64_t token = r / j.q_heads;
    const int head = static_cast<int>(r - token * j.q_heads);
    if (j.tokens && token >= *j.tokens) return;
    int n = j.slots;
    if (j.before) {
        const int64_t b = token / j.q_len;
        const int units = j.before[b + 1] - j.before[b];
        const int item = head / j.group * j.row_tiles + (static_cast<int>(token - b * j.q_len) * j.group + head % j.group) / j.tile;
        n = shares_of(j.before[b] * j.items + item * units, units, *j.share).count;
        if (n == 1) return;
    }
    const float2* ml = j.part_ml + r * j.slots;
    float m = -FLT_MAX;
    for (int x = at; x < n; x += 16) m = fmaxf(m, ml[x].x);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
    const float* part = j.part + r * j.slots * D + at * kDims;
    float l = 0.0f, f[kDims] = {};
#pragma unroll 4
    for (int x = group; x < n; x += GROUPS) {
        const float2 here = ml[x];
        float v[kDims];
#pragma unroll
        for (int y = 0; y < kDims; y += 4) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(part + static_cast<int64_t>(x) * D + y);
#pragma unroll
            for (int z = 0; z < 4; ++z) v[y + z] = q[z];
        }
        const float c = __builtin_amdgcn_exp2f(here.x - m);
        l += c * here.y;
#pragma unroll
        for (int y = 0; y < kDims; ++y) f[y] += c * v[y];
    }
    if constexpr (GROUPS > 1) {
        __shared__ float so[GROUPS][16][kDims + 1];
#pragma unroll
        for (int y = 0; y < kDims; ++y) so[group][at][y] = f[y];
        so[group][at][kDims] = l;
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int x = 1; x < GROUPS; ++x) {
#pragma unroll
            for (int y = 0; y < kDims; ++y) f[y] += so[x][at][y];
            l += so[x][at][kDims];
        }
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
    if (j.expected > 16)
        join_kernel<D, T, 16><<<static_cast<uint32_t>(j.rows), 256, 0, s>>>(j);
    else
        join_kernel<D, T, 1><<<static_cast<uint32_t>((j.rows + 15) / 16), 256, 0, s>>>(j);
    return hipGetLastError();
}

}  // namespace

}  // namespace unisvq
