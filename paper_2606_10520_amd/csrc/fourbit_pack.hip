// 4-bit weights on gfx950: packing, its inverse, and rounding to the nearest
// codes.  Set-up work, once for a model's weights: simple kernels, a word of eight
// codes a thread.  8192 x 28672: pack 105 + 11 us, unpack 152, rounding from f16 225 to
// 250 (2.5 TB/s; words of a line are written by threads far apart, and an exact division
// for each weight).  A copy of the same bytes: 70, 70 and 116.
#include <algorithm>

#include "layer.hpp"

namespace unisvq {
namespace {

constexpr int kThreads = 256;

// Word w of the packed codes: its row and the first of its eight columns.
struct Place {
    int64_t row;
    int64_t col;
};
__device__ inline Place place_of(int64_t w, int64_t groups) {
    const int j = static_cast<int>(w & 3), slot = static_cast<int>(w >> 2 & 63);
    const int64_t tile = w >> 8;  // row block * groups + group
    const int64_t rb = tile / groups;
    return Place{rb * kRowBlock + (slot & 15), (tile - rb * groups) * kGroup + 64 * (j >> 1) + 16 * (slot >> 4) + 8 * (j & 1)};
}

// Place of the scale of (row, group): f16 index behind the codes.
__device__ inline int64_t scale_at(int64_t row, int64_t group, int64_t quads) {
    return ((row >> 4) * quads + (group >> 2)) * (kFourbitQuad / 2) + (row & 15) * 4 + (group & 3);
}

__global__ __launch_bounds__(kThreads) void pack_kernel(int64_t N, int64_t K, const uint8_t* codes, uint32_t* out, int32_t* bad) {
    const int64_t groups = K / kGroup, words = N * (K / 8);
    int wrong = 0;
    for (int64_t w = blockIdx.x * static_cast<int64_t>(kThreads) + threadIdx.x; w < words;
         w += static_cast<int64_t>(gridDim.x) * kThreads) {
        const Place p = place_of(w, groups);
        const uint8_t* c = codes + p.row * K + p.col;
        uint32_t q = 0;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            wrong += c[b] > 15;
            q |= static_cast<uint32_t>(c[b] & 15) << (b < 4 ? 8 * b : 8 * b - 28);
        }
        out[w] = q;
    }
    if (bad && wrong) atomicAdd(bad, wrong);
}

__global__ __launch_bounds__(kThreads) void pack_scales_kernel(int64_t N, int64_t K, const uint16_t* scales, uint16_t* out) {
    const int64_t groups = K / kGroup, quads = (groups + 3) / 4, count = N * quads * 4;
    for (int64_t i = blockIdx.x * static_cast<int64_t>(kThreads) + threadIdx.x; i < count;
         i += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t row = i / (quads * 4), g = i - row * quads * 4;
        out[scale_at(row, g, quads)] = g < groups ? scales[row * groups + g] : 0;
    }
}

__global__ __launch_bounds__(kThreads) void unpack_kernel(int64_t N, int64_t K, const uint32_t* packed, const uint16_t* tail,
                                                          uint8_t* codes, uint16_t* scales) {
    const int64_t groups = K / kGroup, quads = (groups + 3) / 4, words = N * (K / 8);
    for (int64_t w = blockIdx.x * static_cast<int64_t>(kThreads) + threadIdx.x; w < words;
         w += static_cast<int64_t>(gridDim.x) * kThreads) {
        const Place p = place_of(w, groups);
        const uint32_t q = packed[w];
        uint8_t* c = codes + p.row * K + p.col;
#pragma unroll
        for (int b = 0; b < 8; ++b) c[b] = q >> (b < 4 ? 8 * b : 8 * b - 28) & 15;
        if (p.col % kGroup == 0) scales[p.row * groups + p.col / kGroup] = tail[scale_at(p.row, p.col / kGroup, quads)];
    }
}

// Sixteen neighbouring threads have a row's group: its largest magnitude a, the
// scale a / 7 rounded to f16, and the nearest codes to w / scale.
template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_kernel(int64_t N, int64_t K, const T* W, uint32_t* out, uint16_t* tail) {
    const int64_t groups = K / kGroup, quads = (groups + 3) / 4, runs = N * (K / 8);
    for (int64_t i0 = blockIdx.x * static_cast<int64_t>(kThreads); i0 < runs; i0 += static_cast<int64_t>(gridDim.x) * kThreads) {
        const int64_t i = i0 + threadIdx.x;  // (a multiple of 256 runs: 16 rows of 128 columns and more)
        const int64_t row = i / (K / 8), run = i - row * (K / 8), g = run >> 4;
        const int r = static_cast<int>(run & 15);
        float w[8];
        load8(W + row * K + 8 * run, w);
        uint32_t most = 0;
#pragma unroll
        for (int b = 0; b < 8; ++b) most = max(most, magnitude(w[b]));
        most = over_lanes(most, 4, [](uint32_t p, uint32_t q) { return max(p, q); });
        const bool finite = most < 0x7f800000u;
        const _Float16 scale = finite ? static_cast<_Float16>(fminf(__uint_as_float(most) / 7.0f, 65504.0f))
                                      : static_cast<_Float16>(__builtin_nanf(""));
        const float s = static_cast<float>(scale);
        uint32_t q = 0x88888888u;
        if (s > 0.0f) {
            q = 0;
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const int c = static_cast<int>(fminf(fmaxf(rintf(w[b] / s), -8.0f), 7.0f)) + 8;
                q |= static_cast<uint32_t>(c) << (b < 4 ? 8 * b : 8 * b - 28);
            }
        }
        // run r of the group: 64 (r / 8) + 16 (r / 2 % 4) + 8 (r % 2)
        const int j = 2 * (r >> 3) + (r & 1), slot = (r >> 1 & 3) * 16 + static_cast<int>(row & 15);
        out[(((row >> 4) * groups + g) * 64 + slot) * 4 + j] = q;
        if (r == 0) {
            tail[scale_at(row, g, quads)] = __builtin_bit_cast(uint16_t, scale);
            if (g == groups - 1)
                for (int64_t e = groups; e < 4 * quads; ++e) tail[scale_at(row, e, quads)] = 0;
        }
    }
}

uint32_t blocks_for(int64_t count) {
    return static_cast<uint32_t>(std::min<int64_t>((count + kThreads - 1) / kThreads, 1 << 20));
}

}  // namespace

hipError_t launch_fourbit_pack(int64_t N, int64_t K, const uint8_t* codes, const uint16_t* scales, uint8_t* packed,
                          int32_t* bad, hipStream_t s) {
    pack_kernel<<<blocks_for(N * (K / 8)), kThreads, 0, s>>>(N, K, codes, reinterpret_cast<uint32_t*>(packed), bad);
    pack_scales_kernel<<<blocks_for(N * fourbit_quads(K) * 4), kThreads, 0, s>>>(
        N, K, scales, reinterpret_cast<uint16_t*>(packed + fourbit_code_bytes(N, K)));
    return hipGetLastError();
}

hipError_t launch_fourbit_unpack(int64_t N, int64_t K, const uint8_t* packed, uint8_t* codes, uint16_t* scales,
                            hipStream_t s) {
    unpack_kernel<<<blocks_for(N * (K / 8)), kThreads, 0, s>>>(
        N, K, reinterpret_cast<const uint32_t*>(packed), reinterpret_cast<const uint16_t*>(packed + fourbit_code_bytes(N, K)),
        codes, scales);
    return hipGetLastError();
}

hipError_t launch_fourbit_quantize(int64_t N, int64_t K, const void* W, int w_dtype, uint8_t* packed, hipStream_t s) {
    uint32_t* out = reinterpret_cast<uint32_t*>(packed);
    uint16_t* tail = reinterpret_cast<uint16_t*>(packed + fourbit_code_bytes(N, K));
    const uint32_t blocks = blocks_for(N * (K / 8));
    if (w_dtype == UNISVQ_F16)
        quantize_kernel<<<blocks, kThreads, 0, s>>>(N, K, static_cast<const _Float16*>(W), out, tail);
    else if (w_dtype == UNISVQ_BF16)
        quantize_kernel<<<blocks, kThreads, 0, s>>>(N, K, static_cast<const __bf16*>(W), out, tail);
    else
        quantize_kernel<<<blocks, kThreads, 0, s>>>(N, K, static_cast<const float*>(W), out, tail);
    return hipGetLastError();
}

}  // namespace unisvq
