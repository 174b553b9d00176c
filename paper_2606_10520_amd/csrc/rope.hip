// Rotary positions on gfx950.
//   table[p][0][i] = m cos(p f_i), table[p][1][i] = m sin(p f_i)
//   (a, b) -> (a c - b s, b c + a s) for the pairs of the rotated dims
//
// The table is made once, in fp64: an angle p f_i reaches 10^5 and more, where
// an fp32 product would be off by a hundredth of a turn.
#include <algorithm>
#include <cmath>

#include "attn.hpp"

namespace unisvq {
namespace {

constexpr int kThreads = 256;

__global__ __launch_bounds__(kThreads) void rope_table_kernel(int64_t count, int half, double log_theta, double factor,
                                                              double low, double high, double original,
                                                              double magnitude, float* table) {
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < count;
         i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t p = i / half;
        const int j = static_cast<int>(i - p * half);
        double f = exp(-log_theta * j / half);
        double g = 0.0;
        if (original > 0) {
            const double turns = original * f * 0.15915494309189533577;  // 1 / (2 pi)
            g = fmin(fmax((turns - low) / (high - low), 0.0), 1.0);
        }
        f = (1.0 - g) * f / factor + g * f;
        double s, c;
        sincos(static_cast<double>(p) * f, &s, &c);
        table[2 * p * half + j] = static_cast<float>(magnitude * c);
        table[(2 * p + 1) * half + j] = static_cast<float>(magnitude * s);
    }
}

// Bound by memory: x is read and y written once.  A thread rotates sixteen dims
// (eight pairs) of kHeads heads of one token, so that it reads the sixteen table
// entries once for all of them, and every access is 16 bytes.  It reads and
// writes the same dims, so y may be x.
// 8192 tokens of 64 heads of 128, half of each rotated: 55 us, 4.9 TB/s, what a
// large copy reaches; 4 tokens of 32 heads: 3.3 us, a launch and its latency.
constexpr int kHeads = 4;

template <typename T>
__global__ __launch_bounds__(kThreads) void rope_kernel(uint32_t count, int heads, int chunks, Rotary rotary, Rows x,
                                                        const int32_t* positions, Rows y) {
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= count) return;
    const uint32_t groups = (heads + kHeads - 1) / kHeads;
    const uint32_t c = i % chunks, th = i / chunks, t = th / groups;
    const int h0 = static_cast<int>(th % groups) * kHeads;
    const Chunk k = chunk_of(c, rotary.rot, 16 * chunks);
    float cs[8], sn[8];
    if (k.turned) {
        const int64_t p = positions[t];
        if (p >= 0 && p < rotary.positions) {
            load_angles(rotary.table + p * rotary.rot, rotary.rot, c, rotary.interleaved, cs, sn);
            if (rotary.inverse)
#pragma unroll
                for (int j = 0; j < 8; ++j) sn[j] = -sn[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) cs[j] = sn[j] = __builtin_nanf("");
        }
    }
    const T* from = static_cast<const T*>(x.p) + t * x.ts;
    T* to = static_cast<T*>(y.p) + t * y.ts;
#pragma unroll
    for (int j = 0; j < kHeads; ++j) {
        const int h = h0 + j;
        if (h >= heads) break;
        float u[8], w[8];
        load8(from + h * x.hs + k.d0, u);
        load8(from + h * x.hs + k.d1, w);
        if (k.turned) turn(u, w, cs, sn, rotary.interleaved);
        store8(to + h * y.hs + k.d0, u);
        store8(to + h * y.hs + k.d1, w);
    }
}

}  // namespace

hipError_t launch_rope_table(int64_t positions, int rot, double theta, double factor, double low, double high,
                             double original, double magnitude, float* table, hipStream_t s) {
    const int64_t count = positions * (rot / 2);
    // (a launch has fewer than 2^32 threads, the largest table twice as many entries)
    const uint32_t blocks = static_cast<uint32_t>(std::min<int64_t>((count + kThreads - 1) / kThreads, 1 << 20));
    rope_table_kernel<<<blocks, kThreads, 0, s>>>(count, rot / 2, std::log(theta), factor, low, high, original,
                                                  magnitude, table);
    return hipGetLastError();
}

hipError_t launch_rope(int64_t tokens, int heads, int head_dim, const Rotary& rotary, Rows x, const int32_t* positions,
                       Rows y, int dtype, hipStream_t s) {
    const int chunks = head_dim / 16;
    const uint32_t count = static_cast<uint32_t>(tokens * ((heads + kHeads - 1) / kHeads) * chunks);
    const uint32_t blocks = (count + kThreads - 1) / kThreads;
    if (dtype == UNISVQ_F16)
        rope_kernel<_Float16><<<blocks, kThreads, 0, s>>>(count, heads, chunks, rotary, x, positions, y);
    else
        rope_kernel<__bf16><<<blocks, kThreads, 0, s>>>(count, heads, chunks, rotary, x, positions, y);
    return hipGetLastError();
}

}  // namespace unisvq
