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
constexpr uint32_t kResident = 512;  // workgroups that the GPU holds at once

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

// The offset from a tile's first row of what thread i of a group brings to
// place 16 (256 n + i) of the tile in LDS.
template <int D, bool VALUES>
__device__ inline uint32_t load_offset(int n, int i, int64_t ts) {
    constexpr int chunks = D / 8;
    const int at = n * kThreads + i, row = at / chunks, place = at % chunks;
    const int chunk = place ^ (VALUES ? turn_v<D>(row) : turn_k<D>(row));
    return static_cast<uint32_t>(row * static_cast<int>(ts) * 2 + chunk * 16);
}

// Bring the tile at `p` (of `rows` rows, ts elements apart) to LDS.  What is
// past the last row is past the buffer's end, and becomes zeros.
template <int D, typename T>
__device__ __forceinline__ void load_tile(const T* p, int64_t ts, int rows, const uint32_t (&off)[kKeys * D / 8 / kThreads],
                                          T* lds, int wave) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, static_cast<uint32_t>((rows - 1) * ts * 2 + D * 2));
#pragma unroll
    for (int n = 0; n < kKeys * D / 8 / kThreads; ++n) {
        const uint32_t to = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(
            (__attribute__((address_space(3))) void*)(lds + (n * kThreads + wave * 64) * 8))));
        // (the compiler would wait for a load that it knows of before any read of LDS that might be of its place)
        asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(off[n]), "s"(r) : "memory");
    }
}

// Which of a lane's sums have met +inf or NaN, and which -inf or NaN (bit 16 d + r: o[d][r]).
struct Spoiled {
    uint64_t up, down;
};

// Marks the sums that values of the tile at `vs` that are not finite belong to,
// for queries that see their keys (k0 + row < limit; see not_finite).
template <int D, typename T>
__device__ inline void mark_not_finite(const T* vs, int k0, int limit, int lane, Spoiled& spoiled) {
    constexpr int chunks = D / 8;
#pragma nounroll
    for (int at = lane; at < kKeys * chunks; at += 64) {
        const u32x4 w = reinterpret_cast<const u32x4*>(vs)[at];
        uint64_t left = __ballot(not_finite<T>(w[0]) || not_finite<T>(w[1]) || not_finite<T>(w[2]) || not_finite<T>(w[3]));
        while (left) {
            const int from = __ffsll(static_cast<unsigned long long>(left)) - 1;
            left &= left - 1;
            const int place = at - lane + from, row = place / chunks;
            const int dim = ((place % chunks) ^ turn_v<D>(row)) * 8;
            uint64_t lo = __builtin_amdgcn_readlane(w[0], from) | static_cast<uint64_t>(__builtin_amdgcn_readlane(w[1], from)) << 32;
            uint64_t hi = __builtin_amdgcn_readlane(w[2], from) | static_cast<uint64_t>(__builtin_amdgcn_readlane(w[3], from)) << 32;
#pragma nounroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t bits = static_cast<uint32_t>(lo & 0xffffu);
                lo = lo >> 16 | hi << 48;
                hi >>= 16;
                if ((bits & exponent_bits<T>()) != exponent_bits<T>()) continue;
                if (k0 + row < limit && (lane >> 5) == e / 4) {
                    const uint64_t here = uint64_t{1} << (dim / 32 * 16 + dim % 32 / 8 * 4 + e % 4);
                    if (bits != (0x8000u | exponent_bits<T>())) spoiled.up |= here;
                    if (bits != exponent_bits<T>()) spoiled.down |= here;
                }
            }
        }
    }
}

// Whether the tile at `vs` holds a value that is not finite (the whole wave's answer).
template <int D, typename T>
__device__ inline bool any_not_finite(const T* vs, int lane) {
    bool bad = false;
#pragma unroll 4
    for (int at = lane; at < kKeys * D / 8; at += 64) {
        const u32x4 w = reinterpret_cast<const u32x4*>(vs)[at];
#pragma unroll
        for (int x = 0; x < 4; ++x) bad |= not_finite<T>(w[x]);
    }
    return __any(bad);
}

// A barrier of all waves that waits for no loads in flight.
__device__ inline void phase() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

template <int N>
__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// The order of values() and scores() in one phase: reads of LDS four products ahead.
template <int D>
__device__ __forceinline__ void schedule_products() {
    constexpr int kProducts = D / 8, kAhead = 4;  // of either kind; two reads for one of values', one for one of scores'
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * kAhead, 0);
#pragma unroll
    for (int n = 0; n < kProducts - kAhead; ++n) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
#pragma unroll
    for (int n = 0; n < kProducts; ++n) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
}

template <int D, typename T>
struct Wave {
    typedef typename Vec8<T>::type T8;
    T8 q[D / 16];
    f32x16 o[D / 32];
    f32x16 s[2];
    T8 p[4];
    float m, l, scale;
    int hf;
    int at_k;           // keys: row i of a tile, chunk hf as it is turned (chunk 2n + hf is at_k ^ 16n)
    int at_v[D / 32];   // values: row 4hf + (i % 16) / 4, the lane's four dims of dim tile d

    // o += V^T P^T for the tile at vs; CLEAN: values that are not finite count as zero.
    template <bool CLEAN>
    __device__ __forceinline__ void values(const T* vs) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int d = 0; d < D / 32; ++d) {
                // keys 16n + 4hf + 0..3 and + 8..11 of dim 32d + i
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4*)(vs + at_v[d] + 16 * n * D));
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4*)(vs + at_v[d] + (16 * n + 8) * D));
                u32x4 v4 = __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                if constexpr (CLEAN)
#pragma unroll
                    for (int x = 0; x < 4; ++x) v4[x] = finite_only<T>(v4[x]);
                const T8 v8 = __builtin_bit_cast(T8, v4);
                o[d] = mfma(v8, p[n], o[d]);
            }
    }

    // s = K Q^T for the tile at ks.
    __device__ __forceinline__ void scores(const T* ks) {
#pragma unroll
        for (int n = 0; n < D / 16; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const T8 k8 = *reinterpret_cast<const T8*>(ks + (at_k ^ 16 * n) + 32 * x * D);
                s[x] = mfma(k8, q[n], n ? s[x] : f32x16{});
            }
    }

    // Hides keys from `limit` on, in the tile from key k0.
    __device__ __forceinline__ void mask(int k0, int limit) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (32 * x + 8 * (r / 4) + r % 4 >= limit - k0 - 4 * hf) s[x][r] = -INFINITY;
    }

    // The tile's weights from its scores.
    __device__ __forceinline__ void weights() {
        float top = s[0][0];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[x][r]);
        top *= scale;
        if (__any(top > m + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m2 = fmaxf(m, top), c = exp2_(m - m2);
            m = m2;
            l *= c;
#pragma unroll
            for (int d = 0; d < D / 32; ++d) o[d] *= c;
        }
        float sum[4] = {};
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float w = exp2_(__builtin_fmaf(s[x][r], scale, -m));
                sum[r % 4] += w;
                p[2 * x + r / 8][r % 8] = static_cast<T>(w);
            }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
};

template <int D, typename T>
__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(PromptArgs a, float scale_log2) {
    typedef typename Vec8<T>::type T8;
    constexpr int kQ = 32, kTileQ = kQ * kWaves, kTile = kKeys * D;
    constexpr int kLoads = kTile * 2 / (16 * kThreads);  // loads a thread of a tile of keys or values
    __shared__ __attribute__((aligned(16))) T sk[2][kTile];  // two tiles of keys
    __shared__ __attribute__((aligned(16))) T sv[2][kTile];  // and of values
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
    const int i = lane & 31, hf = lane >> 5;

    // heads of one key head go to one XCD (workgroups go round the eight)
    int head = blockIdx.x % a.q_heads;
    if (a.q_heads % 8 == 0) head = head % 8 * (a.q_heads / 8) + head / 8;
    // Late tiles see most keys, so they go first.  Where all workgroups are
    // resident at once, two a CU, those that come second on a CU go from the
    // fewest keys up, to share it with the most.
    const int64_t rank = blockIdx.x / a.q_heads, count = gridDim.x / a.q_heads;
    int64_t tile = count - 1 - rank;
    if (gridDim.x <= kResident && rank >= (count + 1) / 2) tile = rank - (count + 1) / 2;
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
    const int wave_low = a.causal ? wave_first + nk - nq + 1 : nk;  // seen by all its queries
    const int wave_high = wave_first >= nq ? 0 : a.causal ? min(nk, min(wave_first + kQ, nq) + nk - nq) : nk;
    const int keys = a.causal ? min(nk, min(q0 + kTileQ, nq) + nk - nq) : nk;  // seen by any query of the tile
    Wave<D, T> w;
    w.hf = hf;
    w.at_k = i * D + (hf ^ turn_k<D>(i)) * 8;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
        const int row = 4 * hf + (i & 15) / 4, dim = 32 * d + (i & 16) + 4 * (i & 3);
        w.at_v[d] = row * D + ((dim / 8) ^ turn_v<D>(row)) * 8 + dim % 8;
    }
    w.scale = scale_log2;
    w.m = -FLT_MAX;
    w.l = 0.0f;
    {
        const T* x = static_cast<const T*>(a.q.p) + (q_first + min(qi, nq - 1)) * a.q.ts + head * a.q.hs + 8 * hf;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) w.q[n] = *reinterpret_cast<const T8*>(x + 16 * n);
    }
#pragma unroll
    for (int d = 0; d < D / 32; ++d) w.o[d] = f32x16{};
    const T* kp = static_cast<const T*>(a.k.p) + k_first * a.k.ts + kv * a.k.hs;
    const T* vp = static_cast<const T*>(a.v.p) + k_first * a.v.ts + kv * a.v.hs;
    uint32_t off_k[kLoads], off_v[kLoads];
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
        off_k[n] = load_offset<D, false>(n, threadIdx.x, a.k.ts);
        off_v[n] = load_offset<D, true>(n, threadIdx.x, a.v.ts);
    }
    const auto load_k = [&](int t) __attribute__((always_inline)) {
        const int k0 = t * kKeys;
        load_tile<D, T>(kp + k0 * a.k.ts, a.k.ts, min(kKeys, nk - k0), off_k, sk[t & 1], wave);
    };
    const auto load_v = [&](int t) __attribute__((always_inline)) {
        const int k0 = t * kKeys;
        load_tile<D, T>(vp + k0 * a.v.ts, a.v.ts, min(kKeys, nk - k0), off_v, sv[t & 1], wave);
    };

    // Tiles: those before `plain` are seen whole by all the workgroup's
    // queries (the last is not counted), before `whole` by the wave's, and
    // those from `over` on by none of the wave's.
    const int tiles = keys > 0 ? (keys + kKeys - 1) / kKeys : 0;
    const int block_low = a.causal ? q0 + nk - nq + 1 : nk;
    const int plain = min(tiles - 1, max(0, block_low) / kKeys);
    const int whole = max(0, wave_low) / kKeys;
    const int over = (max(0, wave_high) + kKeys - 1) / kKeys;
    Spoiled spoiled{0, 0};

    // Tile t's weights; then its values and the next tile's scores in one go,
    // with the loads of the tiles after them: one barrier a tile.
    if (tiles > 0) {
        load_k(0);
        load_v(0);
        if (tiles > 1) load_k(1);
        wait_loads<0>();
        // (the queries too: the compiler would go on waiting for them in the loop)
#pragma unroll
        for (int n = 0; n < D / 16; ++n) asm volatile("" : "+v"(w.q[n]));
        phase();
        if (over > 0) w.scores(sk[0]);
        int t = 0;
        for (; t < plain; ++t) {
            w.weights();
            wait_loads<0>();
            phase();  // keys t + 1 and values t are there; keys t and values t - 1 are done with
            if (t + 2 < tiles) load_k(t + 2);
            load_v(t + 1);
            w.template values<false>(sv[t & 1]);
            w.scores(sk[(t + 1) & 1]);
            schedule_products<D>();
        }
        for (; t < tiles; ++t) {
            const T* const v_now = sv[t & 1];
            const int k0 = t * kKeys;
            if (t < over) {
                if (t >= whole) w.mask(k0, limit);
                w.weights();
            }
            wait_loads<0>();
            phase();
            if (t + 2 < tiles) load_k(t + 2);
            if (t + 1 < tiles) load_v(t + 1);
            if (t < over) {
                if (a.causal && t >= whole && any_not_finite<D, T>(v_now, lane)) {
                    mark_not_finite<D, T>(v_now, k0, limit, lane, spoiled);
                    w.template values<true>(v_now);
                } else {
                    w.template values<false>(v_now);
                }
            }
            if (t + 1 < over) w.scores(sk[(t + 1) & 1]);
        }
    }

    if (__any((spoiled.up | spoiled.down) != 0)) {
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const bool up = spoiled.up >> (16 * d + r) & 1, down = spoiled.down >> (16 * d + r) & 1;
                w.o[d][r] += up && down ? __builtin_nanf("") : up ? INFINITY : down ? -INFINITY : 0.0f;
            }
    }

    w.l += __shfl_xor(w.l, 32);
    if (!live) return;
    const float inv = w.l == 0.0f ? 0.0f : 1.0f / w.l;
    T* to = static_cast<T*>(a.out.p) + (q_first + qi) * a.out.ts + head * a.out.hs + 4 * hf;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            typedef T T4 __attribute__((ext_vector_type(4)));
            T4 v;
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = static_cast<T>(w.o[d][4 * r + x] * inv);
            *reinterpret_cast<T4*>(to + 32 * d + 8 * r) = v;
        }
    if (a.lse && hf == 0) a.lse[(q_first + qi) * a.q_heads + head] = (w.m + log2f(w.l)) * kLn2;
}

template <int D, typename T>
hipError_t run(const PromptArgs& a, hipStream_t s) {
    const int64_t tiles = (a.q_tokens + 127 * a.sequences) / 128;  // at most, of sequences that fill their last one anyhow
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
