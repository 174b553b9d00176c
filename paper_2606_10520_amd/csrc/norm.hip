// Root-mean-square norm with the residual's addition on gfx950.
//   h = x + r, rounded to the stream's type (h = x without a stream)
//   y = h / sqrt(mean(h^2) + eps) * (w + offset), as 16 bits, fp32, or 8 bits
//   with a scale a row
#include <algorithm>

#include "layer.hpp"

namespace unisvq {
namespace {

// Bound by memory: x, r, h and y pass once, so a row stays in registers from its
// loads to its stores, V runs of eight a thread.  WIDE: a workgroup a row, else
// 2^steps lanes of a wave.  Runs past the row's end read its last run again and
// count as zeros, so that no load waits behind a branch.  h, rounded to the stream's
// type, is what a later layer reads, and so what is normalised; y is rounded once.
// 4096 rows of 8192 bf16: 45 us (5.9 TB/s), with an fp32 stream 73 us (5.5 TB/s);
// one row of 4096 2.4 us.
template <typename T, int V, bool WIDE>
__global__ __launch_bounds__(WIDE ? 1024 : 256) void norm_kernel(NormArgs a, int steps) {
    __shared__ float sums[16];
    __shared__ uint32_t tops[16];
    const int lanes = WIDE ? blockDim.x : 1 << steps;
    const int lane = WIDE ? threadIdx.x : threadIdx.x & (lanes - 1);
    const int64_t rows = WIDE ? 1 : 256 >> steps;
    const int64_t t0 = WIDE ? blockIdx.x : blockIdx.x * rows + (threadIdx.x >> steps);
    const int runs = a.n / 8;
    for (int64_t t = t0; WIDE ? t < a.tokens : t - (threadIdx.x >> steps) < a.tokens; t += gridDim.x * rows) {
        const bool there = WIDE || t < a.tokens;  // (lanes of rows past the end go along, and store nothing)
        const int64_t tt = there ? t : a.tokens - 1;
        float h[V][8];
        int at[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            at[v] = 8 * min(lane + v * lanes, runs - 1);
            load8(static_cast<const T*>(a.x) + tt * a.x_stride + at[v], h[v]);
        }
        float w[V][8];
        if (a.w_dtype == UNISVQ_F32) {
#pragma unroll
            for (int v = 0; v < V; ++v) load8(static_cast<const float*>(a.w) + at[v], w[v]);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) load8(static_cast<const T*>(a.w) + at[v], w[v]);
        }
        if (a.r) {
            float r[V][8];
            if (a.r_dtype == UNISVQ_F32) {
#pragma unroll
                for (int v = 0; v < V; ++v) load8(static_cast<const float*>(a.r) + tt * a.r_stride + at[v], r[v]);
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[v][i] += r[v][i];
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) load8(static_cast<const T*>(a.r) + tt * a.r_stride + at[v], r[v]);
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[v][i] = static_cast<float>(static_cast<T>(h[v][i] + r[v][i]));
            }
            // (in place: every thread has read what it overwrites)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (there && lane + v * lanes < runs)
                    store_row8<T>(a.h, t * a.h_stride + at[v], h[v], a.r_dtype == UNISVQ_F32);
        }
        float sum = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const bool in = lane + v * lanes < runs;
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(h[v][i], h[v][i], s);
            sum += in ? s : 0.0f;
        }
        const auto add = [](float p, float q) { return p + q; };
        if constexpr (WIDE)
            sum = over_block(sum, sums, add);
        else
            sum = over_lanes(sum, steps, add);
        const float f = __builtin_amdgcn_rsqf(sum / static_cast<float>(a.n) + a.eps);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * f * (w[v][i] + a.offset);
        if (a.y_dtype != UNISVQ_I8) {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (there && lane + v * lanes < runs)
                    store_row8<T>(a.y, t * a.y_stride + at[v], h[v], a.y_dtype == UNISVQ_F32);
        } else {
            // (runs past the end are left out: where the stream is written in place another
            // wave may have stored its last run before they read it)
            uint32_t most = 0;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) most = max(most, lane + v * lanes < runs ? magnitude(h[v][i]) : 0u);
            const auto larger = [](uint32_t p, uint32_t q) { return max(p, q); };
            if constexpr (WIDE)
                most = over_block(most, tops, larger);
            else
                most = over_lanes(most, steps, larger);
            const RowScale k = row_scale(most);
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (there && lane + v * lanes < runs)
                    *reinterpret_cast<uint2*>(static_cast<int8_t*>(a.y) + t * a.y_stride + at[v]) = codes_of(h[v], k.inv);
            if (there && lane == 0) a.scales[t] = k.scale;
        }
        if constexpr (WIDE) __syncthreads();  // (the words of LDS serve the next row)
    }
}

// Rows too long for registers (1024 threads have 128 each): a thread's runs four at
// a time, read again from the L2 for the result, and once more for 8 bits (with four
// and eight runs a thread the registers went to memory instead).  The stream is read
// back from where it was stored, by the thread that stored it (or, past the row's end,
// by one whose value is not used).
template <typename T>
__device__ __forceinline__ void load_four(const void* p, int64_t row, bool wide, const int (&at)[4], float (&f)[4][8]) {
    if (wide) {
#pragma unroll
        for (int v = 0; v < 4; ++v) load8(static_cast<const float*>(p) + row + at[v], f[v]);
    } else {
#pragma unroll
        for (int v = 0; v < 4; ++v) load8(static_cast<const T*>(p) + row + at[v], f[v]);
    }
}

template <typename T>
__global__ __launch_bounds__(1024) void long_norm_kernel(NormArgs a) {
    __shared__ float sums[16];
    __shared__ uint32_t tops[16];
    const int lane = threadIdx.x, runs = a.n / 8;
    const bool wide = a.r && a.r_dtype == UNISVQ_F32;
    const auto places = [&](int r0, int (&at)[4]) {
#pragma unroll
        for (int v = 0; v < 4; ++v) at[v] = 8 * min(r0 + v * 1024 + lane, runs - 1);
    };
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        float sum = 0.0f;
        for (int r0 = 0; r0 < runs; r0 += 4096) {
            int at[4];
            float h[4][8];
            places(r0, at);
            load_four<T>(a.x, t * a.x_stride, false, at, h);
            if (a.r) {
                float r[4][8];
                load_four<T>(a.r, t * a.r_stride, wide, at, r);
#pragma unroll
                for (int v = 0; v < 4; ++v) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        h[v][i] += r[v][i];
                        if (!wide) h[v][i] = static_cast<float>(static_cast<T>(h[v][i]));
                    }
                    if (r0 + v * 1024 + lane < runs) store_row8<T>(a.h, t * a.h_stride + at[v], h[v], wide);
                }
            }
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(h[v][i], h[v][i], s);
                sum += r0 + v * 1024 + lane < runs ? s : 0.0f;
            }
        }
        sum = over_block(sum, sums, [](float p, float q) { return p + q; });
        const float f = __builtin_amdgcn_rsqf(sum / static_cast<float>(a.n) + a.eps);
        const void* from = a.r ? a.h : a.x;
        const int64_t row = t * (a.r ? a.h_stride : a.x_stride);
        const auto result = [&](const int(&at)[4], float(&h)[4][8]) {
            float w[4][8];
            load_four<T>(from, row, wide, at, h);
            load_four<T>(a.w, 0, a.w_dtype == UNISVQ_F32, at, w);
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * f * (w[v][i] + a.offset);
        };
        RowScale k{};
        if (a.y_dtype == UNISVQ_I8) {
            uint32_t most = 0;
            for (int r0 = 0; r0 < runs; r0 += 4096) {
                int at[4];
                float h[4][8];
                places(r0, at);
                result(at, h);
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                    for (int i = 0; i < 8; ++i) most = max(most, r0 + v * 1024 + lane < runs ? magnitude(h[v][i]) : 0u);
            }
            k = row_scale(over_block(most, tops, [](uint32_t p, uint32_t q) { return max(p, q); }));
            if (lane == 0) a.scales[t] = k.scale;
        }
        for (int r0 = 0; r0 < runs; r0 += 4096) {
            int at[4];
            float h[4][8];
            places(r0, at);
            result(at, h);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                if (r0 + v * 1024 + lane >= runs) continue;
                if (a.y_dtype == UNISVQ_I8)
                    *reinterpret_cast<uint2*>(static_cast<int8_t*>(a.y) + t * a.y_stride + at[v]) = codes_of(h[v], k.inv);
                else
                    store_row8<T>(a.y, t * a.y_stride + at[v], h[v], a.y_dtype == UNISVQ_F32);
            }
        }
        __syncthreads();  // (the words of LDS serve the next row)
    }
}

template <typename T>
void launch(const NormArgs& a, hipStream_t s) {
    constexpr int64_t kMostBlocks = 1 << 20;  // the rest of the rows in turn
    const int runs = a.n / 8;
    if (runs <= 64) {
        int steps = 3;
        while ((1 << steps) < runs) ++steps;
        const int64_t rows = 256 >> steps;
        const uint32_t blocks = static_cast<uint32_t>(std::min((a.tokens + rows - 1) / rows, kMostBlocks));
        norm_kernel<T, 1, false><<<blocks, 256, 0, s>>>(a, steps);
        return;
    }
    const uint32_t blocks = static_cast<uint32_t>(std::min(a.tokens, kMostBlocks));
    const auto threads = [&](int v) { return static_cast<uint32_t>((runs + 64 * v - 1) / (64 * v) * 64); };
    if (runs <= 1024)
        norm_kernel<T, 1, true><<<blocks, threads(1), 0, s>>>(a, 0);
    else if (runs <= 2048)
        norm_kernel<T, 2, true><<<blocks, threads(2), 0, s>>>(a, 0);
    else
        long_norm_kernel<T><<<blocks, 1024, 0, s>>>(a);
}

}  // namespace

hipError_t launch_rmsnorm(const NormArgs& a, hipStream_t s) {
    if (a.x_dtype == UNISVQ_F16)
        launch<_Float16>(a, s);
    else
        launch<__bf16>(a, s);
    return hipGetLastError();
}

}  // namespace unisvq
