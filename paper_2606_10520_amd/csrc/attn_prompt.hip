// Attention over packed prompts on gfx950.
//
//   s = scale (q . k),  p = exp(s - m),  out = sum p v / sum p
//
// Bound: the matrix cores (4 D operations a visible pair).  A workgroup of
// four waves has 128 queries of one head, 32 a wave; keys and values come in
// tiles of 64 through LDS, two tiles deep, loaded there directly.  The products
// are 32x32x16 ones, arranged so that the scores never leave their lanes:
//   S^T = K Q^T   (32 keys x 32 queries): lane (i, h) = (lane % 32, lane / 32)
//                 ends with keys 8x + 4h .. + 3 of query i.
//   O^T = V^T P^T (32 dims x 32 queries, 16 keys inner): P^T's operand wants
//                 eight keys of query i, in any order that V^T's has too: the
//                 ones the lane has.  V^T comes from LDS through the
//                 transposing read, four keys of one dim a lane.
// So a query's maximum and sum need one exchange between the halves of a wave,
// the maximum's only when a score exceeds it by 2^8 (the weights stay below
// 2^8, so nothing overflows, and most tiles need no rescaling).
#include <cfloat>

#include "attn.hpp"

namespace unisvq {
namespace {

constexpr int kThreads = 256, kWaves = 4, kKeys = 64;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kSlack = 8.0f;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline f32x16 mfma(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// LDS rows of D elements are held in 16-byte chunks whose place is turned by
// the row, so that the lanes that read together hit all banks: the keys' rows
// are read 16 rows of one chunk at a time, the values' 4 rows of four chunks.
template <int D>
__device__ inline int turn_k(int row) { return D == 128 ? row & 15 : row >> 1 & 7; }
template <int D>
__device__ inline int turn_v(int row) { return D == 128 ? 4 * (row & 3) : 4 * (row >> 1 & 1); }

// Bring rows of the tile at `p` (of `rows` rows, ts elements apart) to LDS; rows
// past the end become zeros.  Thread i brings the 16 bytes that are to be at
// 16 (256 n + i).
template <int D, typename T, bool VALUES>
__device__ inline void load_tile(const T* p, int64_t ts, int rows, T* lds, int wave, int lane) {
    constexpr int chunks = D / 8;
    const uint32_t bytes = static_cast<uint32_t>((rows - 1) * ts * 2 + D * 2);
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, bytes);
#pragma unroll
    for (int n = 0; n < kKeys * chunks / kThreads; ++n) {
        const int at = n * kThreads + wave * 64 + lane, row = at / chunks, place = at % chunks;
        const int chunk = place ^ (VALUES ? turn_v<D>(row) : turn_k<D>(row));
        const uint32_t off = row < rows ? static_cast<uint32_t>(row * static_cast<int>(ts) * 2 + chunk * 16) : kOutOfRange;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            r, (__attribute__((address_space(3))) void*)(lds + (n * kThreads + wave * 64) * 8), 16, off, 0, 0, 0);
    }
}

// Adds the values of the tile at `vs` that are not finite to the sums o of the
// queries that see their keys (k0 + row < limit; see not_finite).
template <int D, typename T>
__device__ inline void add_not_finite(const T* vs, int k0, int limit, int lane, f32x16 (&o)[D / 32]) {
    constexpr int chunks = D / 8;
    for (int at = lane; at < kKeys * chunks; at += 64) {
        const u32x4 w = reinterpret_cast<const u32x4*>(vs)[at];
        uint64_t left = __ballot(not_finite<T>(w[0]) || not_finite<T>(w[1]) || not_finite<T>(w[2]) || not_finite<T>(w[3]));
        while (left) {
            const int from = __ffsll(static_cast<unsigned long long>(left)) - 1;
            left &= left - 1;
            const int place = at - lane + from, row = place / chunks;
            const bool seen = k0 + row < limit;
            const int dim = ((place % chunks) ^ turn_v<D>(row)) * 8;
            uint64_t lo = __builtin_amdgcn_readlane(w[0], from) | static_cast<uint64_t>(__builtin_amdgcn_readlane(w[1], from)) << 32;
            uint64_t hi = __builtin_amdgcn_readlane(w[2], from) | static_cast<uint64_t>(__builtin_amdgcn_readlane(w[3], from)) << 32;
#pragma nounroll
            for (int e = 0; e < 8; ++e) {
                const uint16_t bits = static_cast<uint16_t>(lo);
                lo = lo >> 16 | hi << 48;
                hi >>= 16;
                if ((bits & exponent_bits<T>()) != exponent_bits<T>()) continue;
                const float add = seen ? static_cast<float>(__builtin_bit_cast(T, bits)) : 0.0f;
#pragma unroll
                for (int d = 0; d < D / 32; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        o[d][r] += 32 * d + 8 * (r / 4) + 4 * (lane >> 5) + r % 4 == dim + e ? add : 0.0f;
            }
        }
    }
}

template <int D, typename T>
__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(PromptArgs a, float scale_log2) {
    typedef typename Vec8<T>::type T8;
    constexpr int kQ = 32, kTileQ = kQ * kWaves;
    __shared__ __attribute__((aligned(16))) T sk[2][kKeys * D];
    __shared__ __attribute__((aligned(16))) T sv[2][kKeys * D];
    __shared__ int bad_tile;  // 1 + the last tile found to hold values that are not finite, of those checked
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int i = lane & 31, hf = lane >> 5;

    // heads of one key head go to one XCD (workgroups go round the eight)
    int head = blockIdx.x % a.q_heads;
    if (a.q_heads % 8 == 0) head = head % 8 * (a.q_heads / 8) + head / 8;
    int64_t tile = gridDim.x / a.q_heads - 1 - blockIdx.x / a.q_heads;  // late tiles see most keys: first
    // the sequence of the tile
    int b = 0;
    int64_t first = 0;
    bool found = false;
    for (int base = 0; base < a.sequences && !found; base += 64) {
        int tiles = 0;
        if (base + lane < a.sequences) {
            const int64_t q0 = min(static_cast<int64_t>(max(0, a.cu_q[base + lane])), a.q_tokens);
            const int64_t q1 = min(static_cast<int64_t>(max(0, a.cu_q[base + lane + 1])), a.q_tokens);
            tiles = q1 > q0 ? static_cast<int>((q1 - q0 + kTileQ - 1) / kTileQ) : 0;
        }
        int sum = tiles;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int up = __shfl_up(sum, d);
            if (lane >= d) sum += up;
        }
        const uint64_t in = __ballot(tile < first + sum);
        if (in) {
            const int l = __ffsll(static_cast<unsigned long long>(in)) - 1;
            b = base + l;
            first += __shfl(sum - tiles, l);
            found = true;
        } else {
            first += __shfl(sum, 63);
        }
    }
    if (!found) return;
    b = __builtin_amdgcn_readfirstlane(b);
    const int64_t q_first = max(0, a.cu_q[b]);
    const int nq = static_cast<int>(min(static_cast<int64_t>(a.cu_q[b + 1]), a.q_tokens) - q_first);
    const int64_t k_first = min(static_cast<int64_t>(max(0, a.cu_k[b])), a.k_tokens);
    const int nk = static_cast<int>(max(int64_t{0}, min(static_cast<int64_t>(a.cu_k[b + 1]), a.k_tokens) - k_first));
    const int q0 = __builtin_amdgcn_readfirstlane(static_cast<int>(tile - first)) * kTileQ;
    const int kv = head / (a.q_heads / a.kv_heads);

    // the lane's query: keys below `limit` are seen
    const int qi = q0 + wave * kQ + i;
    const bool live = qi < nq;
    const int limit = !live ? 0 : a.causal ? qi + nk - nq + 1 : nk;
    const int wave_first = q0 + wave * kQ;
    const int wave_low = wave_first + kQ > nq ? 0 : a.causal ? wave_first + nk - nq + 1 : nk;  // seen by all its queries
    const int wave_high = wave_first >= nq ? 0 : a.causal ? min(nk, min(wave_first + kQ, nq) + nk - nq) : nk;
    const int block_low = a.causal ? q0 + nk - nq + 1 : nk;  // seen by all queries of the tile
    const int keys = a.causal ? min(nk, min(q0 + kTileQ, nq) + nk - nq) : nk;  // seen by any query of the tile
    T8 q[D / 16];
    {
        const T* x = static_cast<const T*>(a.q.p) + (q_first + min(qi, nq - 1)) * a.q.ts + head * a.q.hs + 8 * hf;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) q[n] = *reinterpret_cast<const T8*>(x + 16 * n);
    }
    const T* kp = static_cast<const T*>(a.k.p) + k_first * a.k.ts + kv * a.k.hs;
    const T* vp = static_cast<const T*>(a.v.p) + k_first * a.v.ts + kv * a.v.hs;

    float m = -FLT_MAX, l = 0.0f;
    f32x16 o[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d) o[d] = f32x16{};

    if (threadIdx.x == 0) bad_tile = 0;
    const int tiles = keys > 0 ? (keys + kKeys - 1) / kKeys : 0;
    if (tiles > 0) {
        load_tile<D, T, false>(kp, a.k.ts, min(kKeys, nk), sk[0], wave, lane);
        load_tile<D, T, true>(vp, a.v.ts, min(kKeys, nk), sv[0], wave, lane);
    }
    for (int t = 0; t < tiles; ++t) {
        __syncthreads();  // the tile is there, and its predecessor's buffer free
        const int k0 = t * kKeys;
        if (a.causal && k0 + kKeys > block_low) {  // queries see different keys
            bool bad = false;
            u32x4* w = reinterpret_cast<u32x4*>(sv[t & 1]) + threadIdx.x;
#pragma unroll
            for (int n = 0; n < kKeys * D / 8 / kThreads; ++n)
#pragma unroll
                for (int x = 0; x < 4; ++x) bad |= not_finite<T>(w[n * kThreads][x]);
            if (bad) bad_tile = t + 1;
            __syncthreads();
            if (bad_tile == t + 1) {
                add_not_finite<D, T>(sv[t & 1], k0, limit, lane, o);
                __syncthreads();
#pragma unroll
                for (int n = 0; n < kKeys * D / 8 / kThreads; ++n)
#pragma unroll
                    for (int x = 0; x < 4; ++x) w[n * kThreads][x] = finite_only<T>(w[n * kThreads][x]);
                __syncthreads();
            }
        }
        if (t + 1 < tiles) {
            const int k1 = (t + 1) * kKeys;
            load_tile<D, T, false>(kp + k1 * a.k.ts, a.k.ts, min(kKeys, nk - k1), sk[(t + 1) & 1], wave, lane);
            load_tile<D, T, true>(vp + k1 * a.v.ts, a.v.ts, min(kKeys, nk - k1), sv[(t + 1) & 1], wave, lane);
        }
        if (k0 >= wave_high) continue;
        const T* ks = sk[t & 1];
        const T* vs = sv[t & 1];
        f32x16 s[2] = {};
#pragma unroll
        for (int n = 0; n < D / 16; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int row = 32 * x + i;
                const T8 k8 = *reinterpret_cast<const T8*>(ks + row * D + ((2 * n + hf) ^ turn_k<D>(row)) * 8);
                s[x] = mfma(k8, q[n], s[x]);
            }
        if (k0 + kKeys > wave_low) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (k0 + 32 * x + 8 * (r / 4) + 4 * hf + r % 4 >= limit) s[x][r] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[x][r]);
        top *= scale_log2;
        if (__any(top > m + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m2 = fmaxf(m, top), c = exp2_(m - m2);
            m = m2;
            l *= c;
#pragma unroll
            for (int d = 0; d < D / 32; ++d) o[d] *= c;
        }
        T8 p[4];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float w = exp2_(__builtin_fmaf(s[x][r], scale_log2, -m));
                l += w;
                p[2 * x + r / 8][r % 8] = static_cast<T>(w);
            }
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int d = 0; d < D / 32; ++d) {
                // keys 16n + 4hf + 0..3 and + 8..11 of dim 32d + i
                s16x4 part[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int row = 16 * n + 8 * x + 4 * hf + (i & 15) / 4;
                    const int dim = 32 * d + (i & 16) + 4 * (i & 3);
                    const T* at = vs + row * D + ((dim / 8) ^ turn_v<D>(row)) * 8 + dim % 8;
                    part[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
                }
                const T8 v8 = __builtin_bit_cast(T8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
                o[d] = mfma(v8, p[n], o[d]);
            }
    }

    l += __shfl_xor(l, 32);
    if (!live) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    T* to = static_cast<T*>(a.out.p) + (q_first + qi) * a.out.ts + head * a.out.hs + 4 * hf;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            typedef T T4 __attribute__((ext_vector_type(4)));
            T4 v;
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = static_cast<T>(o[d][4 * r + x] * inv);
            *reinterpret_cast<T4*>(to + 32 * d + 8 * r) = v;
        }
    if (a.lse && hf == 0) a.lse[(q_first + qi) * a.q_heads + head] = (m + log2f(l)) * kLn2;
}

template <int D, typename T>
hipError_t run(const PromptArgs& a, hipStream_t s) {
    const int64_t tiles = a.q_tokens / 128 + a.sequences;
    prompt_kernel<D, T><<<static_cast<uint32_t>(tiles * a.q_heads), kThreads, 0, s>>>(a, a.scale * kLog2e);
    return hipGetLastError();
}

}  // namespace

size_t prompt_workspace_bytes(int64_t, int64_t, int64_t, int, int, int) { return 0; }

hipError_t launch_attn_prompt(const PromptArgs& a, void*, hipStream_t s) {
    if (a.head_dim == 128) return a.dtype == UNISVQ_F16 ? run<128, _Float16>(a, s) : run<128, __bf16>(a, s);
    return a.dtype == UNISVQ_F16 ? run<64, _Float16>(a, s) : run<64, __bf16>(a, s);
}

}  // namespace unisvq
