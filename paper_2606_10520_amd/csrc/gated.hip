// Gated activations on gfx950: y = act(gate) * up, as 16 bits, fp32, or 8 bits
// with a scale a row.
//   silu(g) = g s(g);  gelu(g) = g (1 + tanh(t / 2)) / 2 = g s(t),
//   t = sqrt(8 / pi) (g + 0.044715 g^3),  s(t) = 1 / (1 + exp(-t))
#include <algorithm>

#include "layer.hpp"

namespace unisvq {
namespace {

constexpr int kThreads = 256;

// (the exponential and the reciprocal are off by 2^-22 together, and the exponential by
// |t| 2^-24 more from its argument's product with log2(e), a quarter of that from the constant)
__device__ inline float gated(float g, float u, bool gelu) {
    const float t = gelu ? 1.5957691216057308f * fmaf(0.044715f * g * g, g, g) : g;
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896340736f * t)) * u;
}

// Bound by memory: every value passes once, a run of eight a thread.  2048 rows of
// 28672 bf16: 62 us (5.7 TB/s); 16 of 11008 2.8 us.
template <typename T>
__global__ __launch_bounds__(kThreads) void gated_kernel(GatedArgs a, uint32_t count, uint32_t runs) {
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= count) return;
    const uint32_t t = i / runs, c = 8 * (i - t * runs);
    float g[8], u[8];
    load8(static_cast<const T*>(a.gate) + t * a.gate_stride + c, g);
    load8(static_cast<const T*>(a.up) + t * a.up_stride + c, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = gated(g[j], u[j], a.act == UNISVQ_GELU);
    store_row8<T>(a.y, t * a.y_stride + c, g, a.y_dtype == UNISVQ_F32);
}

// 8 bits: a workgroup a row, kept in registers until its scale is known.
template <typename T, int V>
__global__ __launch_bounds__(1024) void gated_i8_kernel(GatedArgs a) {
    __shared__ uint32_t tops[16];
    const int runs = a.n / 8, lane = threadIdx.x, lanes = blockDim.x;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        float g[V][8], u[V][8];
        int at[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            at[v] = 8 * min(lane + v * lanes, runs - 1);
            load8(static_cast<const T*>(a.gate) + t * a.gate_stride + at[v], g[v]);
            load8(static_cast<const T*>(a.up) + t * a.up_stride + at[v], u[v]);
        }
        uint32_t most = 0;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[v][i] = gated(g[v][i], u[v][i], a.act == UNISVQ_GELU);
                most = max(most, magnitude(g[v][i]));
            }
        most = over_block(most, tops, [](uint32_t p, uint32_t q) { return max(p, q); });
        const RowScale k = row_scale(most);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (lane + v * lanes < runs)
                *reinterpret_cast<uint2*>(static_cast<int8_t*>(a.y) + t * a.y_stride + at[v]) = codes_of(g[v], k.inv);
        if (lane == 0) a.scales[t] = k.scale;
        __syncthreads();  // (the words of LDS serve the next row)
    }
}

// Rows past 32768 (eight runs a thread do not fit 128 registers): gated twice, from the
// L2 the second time, for the scale and for the codes.
template <typename T>
__global__ __launch_bounds__(1024) void long_gated_i8_kernel(GatedArgs a) {
    __shared__ uint32_t tops[16];
    const int runs = a.n / 8, lane = threadIdx.x;
    for (int64_t t = blockIdx.x; t < a.tokens; t += gridDim.x) {
        const auto run = [&](int r, float(&g)[8]) {
            float u[8];
            load8(static_cast<const T*>(a.gate) + t * a.gate_stride + 8 * r, g);
            load8(static_cast<const T*>(a.up) + t * a.up_stride + 8 * r, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = gated(g[i], u[i], a.act == UNISVQ_GELU);
        };
        uint32_t most = 0;
#pragma unroll 4
        for (int r = lane; r < runs; r += 1024) {
            float g[8];
            run(r, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, magnitude(g[i]));
        }
        const RowScale k = row_scale(over_block(most, tops, [](uint32_t p, uint32_t q) { return max(p, q); }));
        if (lane == 0) a.scales[t] = k.scale;
#pragma unroll 4
        for (int r = lane; r < runs; r += 1024) {
            float g[8];
            run(r, g);
            *reinterpret_cast<uint2*>(static_cast<int8_t*>(a.y) + t * a.y_stride + 8 * r) = codes_of(g, k.inv);
        }
        __syncthreads();  // (the words of LDS serve the next row)
    }
}

template <typename T>
void launch(const GatedArgs& a, hipStream_t s) {
    const int runs = a.n / 8;
    if (a.y_dtype != UNISVQ_I8) {
        const uint32_t count = static_cast<uint32_t>(a.tokens * runs);
        gated_kernel<T><<<(count + kThreads - 1) / kThreads, kThreads, 0, s>>>(a, count, runs);
        return;
    }
    const uint32_t blocks = static_cast<uint32_t>(std::min<int64_t>(a.tokens, 1 << 20));
    const auto threads = [&](int v) { return static_cast<uint32_t>((runs + 64 * v - 1) / (64 * v) * 64); };
    if (runs <= 1024)
        gated_i8_kernel<T, 1><<<blocks, threads(1), 0, s>>>(a);
    else if (runs <= 2048)
        gated_i8_kernel<T, 2><<<blocks, threads(2), 0, s>>>(a);
    else if (runs <= 4096)
        gated_i8_kernel<T, 4><<<blocks, threads(4), 0, s>>>(a);
    else
        long_gated_i8_kernel<T><<<blocks, 1024, 0, s>>>(a);
}

}  // namespace

hipError_t launch_gated(const GatedArgs& a, hipStream_t s) {
    if (a.x_dtype == UNISVQ_F16)
        launch<_Float16>(a, s);
    else
        launch<__bf16>(a, s);
    return hipGetLastError();
}

}  // namespace unisvq
