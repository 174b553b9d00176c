// Attention over packed prompts on gfx950.
//
//   s = scale (q . k),  p = exp(s - m),  out = sum p v / sum p
//
// Bound: the matrix cores (4 D operations a visible pair), and under long
// prompts the power that they draw.  A workgroup of four waves has 128 rows, 32
// a wave; a row is a query of one of the heads that share a key head, so heads
// that share keys share the tiles.  Keys and values come in tiles of 64 through
// LDS, two tiles deep, loaded there directly; two workgroups fit a CU, and the
// one's vector work runs under the other's products.  The products are 32x32x16
// ones, arranged so that the scores never leave their lanes:
//   S^T = K Q^T   (32 keys x 32 queries): lane (i, h) = (lane % 32, lane / 32)
//                 ends with keys 8x + 4h .. + 3 of query i.
//   O^T = V^T P^T (32 dims x 32 queries, 16 keys inner): P^T's operand wants
//                 eight keys of query i, in any order that V^T's has too: the
//                 ones the lane has.  V^T comes from LDS through the
//                 transposing read, four keys of one dim a lane.
// So a query's maximum and sum need one exchange between the halves of a wave,
// the maximum's only when a score exceeds it by 2^8 (the weights stay below
// 2^8, or 2^15 in f16's range, so nothing overflows, and most tiles need no
// rescaling).  The weights are rounded to the type of v, which is what the matrix
// cores multiply; their sum is of the unrounded ones, in fp32.
//
// A tile's weights are followed by one run of 32 products, its values' and the
// next tile's scores', with one barrier a tile; a wave in its products goes
// before one in its vector work (16384 tokens of 32 heads 1.90 ms for 2.00; the
// other way round 2.01).
//
// 16384 tokens of 32 heads of 128, causal: 1.90 ms (1.96 on another card), 1155
// TFLOP/s, matrix cores busy 67-71% of the cycles at up to 1.6 GHz (8192^3
// library products under the same power: 1280-1560 TFLOP/s at 86-90%).  2048
// tokens: 51 us, of which 4 us pass before the first products (512 workgroups ask
// for all of q at once), 3-4 us with the first two tiles, and the rest with tiles
// of 1.1 us for a workgroup alone on its CU, 0.93 us for each of two.  64 on 8
// heads, 8 prompts of 1 to 1500 tokens: 75 us, three workgroups in turn on each
// place, and for each 5 us before its first product and 4 from its last to the
// next one's start.  Slower were (against the form of the time): one wave a SIMD
// with three tiles under way (8192 tokens 1270 us for 980: a lone wave issues at
// most one instruction in four to five cycles), eight waves that take turns at
// products and vector work, a tile's weights between the next tile's products
// (2.10 ms for 1.95, 2048 tokens 62 us for 54), and sums of weights by dot
// products (2.09 ms for 2.00).
#include <algorithm>
#include <cfloat>

#include "attn_join.hpp"

namespace unisvq {
namespace {

constexpr int kThreads = 256, kWaves = 4, kKeys = 64, kTileQ = 128;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kSlack = 8.0f;
constexpr int kCUs = 256, kResident = 2 * kCUs;  // workgroups that the GPU holds at once: two a CU

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
struct TileLoad {
    __amdgpu_buffer_rsrc_t r;
    uint32_t to;

    __device__ __forceinline__ TileLoad(const T* p, int64_t ts, int rows, T* lds, int wave)
        : r(make_rsrc(p, rows > 0 ? static_cast<uint32_t>((rows - 1) * ts * 2 + D * 2) : 0u)),
          to(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(
              reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)(lds + wave * 64 * 8))))) {}

    // (In asm, as the compiler would wait for a load that it knows of before any
    // read of LDS that might be of its place.)  What the compiler does elsewhere
    // has to be done here: a load that goes to LDS by M0 comes a wait state after
    // the write of M0, and one that reads scalar registers five after vector
    // instructions that wrote them.
    template <int LOADS>
    __device__ __forceinline__ void issue(const uint32_t (&off)[LOADS]) const {
        static_assert(LOADS == 2 || LOADS == 4, "");
        if constexpr (LOADS == 4)
            asm volatile(
                "s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
                "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %5, 0 offen lds\n\t"
                "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %5, 0 offen lds\n\t"
                "s_add_u32 m0, m0, %6\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %5, 0 offen lds" ::"s"(to),
                "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(r), "n"(kThreads * 16)
                : "scc");
        else
            asm volatile(
                "s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
                "s_add_u32 m0, m0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds" ::"s"(to),
                "v"(off[0]), "v"(off[1]), "s"(r), "n"(kThreads * 16)
                : "scc");
    }
};

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
            const auto word = [&](int x) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(w[x], from)); };
            uint64_t lo = word(0) | static_cast<uint64_t>(word(1)) << 32;
            uint64_t hi = word(2) | static_cast<uint64_t>(word(3)) << 32;
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

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Whether the wave's quarter of the tile at `vs` holds a value that is not finite.
template <int D, typename T>
__device__ inline bool any_not_finite(const T* vs, int wave, int lane) {
    u16x2 top = {0, 0};  // largest magnitudes: exponents of all ones are above every finite one
    const u32x4* at = reinterpret_cast<const u32x4*>(vs) + wave * (kKeys * D / 8 / kWaves) + lane;
#pragma unroll
    for (int n = 0; n < kKeys * D / 8 / kThreads; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, at[64 * n][x] & 0x7fff7fffu));
    return __any(top[0] >= exponent_bits<T>() || top[1] >= exponent_bits<T>());
}

// Zeros in place of them.
template <int D, typename T>
__device__ inline void drop_not_finite(T* vs, int wave, int lane) {
    u32x4* at = reinterpret_cast<u32x4*>(vs) + wave * (kKeys * D / 8 / kWaves) + lane;
#pragma nounroll
    for (int n = 0; n < kKeys * D / 8 / kThreads; ++n)
        for (int x = 0; x < 4; ++x) at[64 * n][x] = finite_only<T>(at[64 * n][x]);
}

// A barrier of all waves that waits for no loads in flight.
__device__ inline void phase() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// One that waits for the wave's own reads and writes of LDS.
__device__ inline void local_phase() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
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
    T8 p[4];
    float m, l, scale;
    int hf;
    int at_k;           // keys: row i of a tile, chunk hf as it is turned (chunk 2n + hf is at_k ^ 16n)
    int at_v[D / 32];   // values: row 4hf + (i % 16) / 4, the lane's four dims of dim tile d

    // o += V^T P^T for the tile at vs.
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
                o[d] = mfma(__builtin_bit_cast(T8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), p[n], o[d]);
            }
    }

    // s = K Q^T for the tile at ks.
    __device__ __forceinline__ void scores(const T* ks, f32x16 (&s)[2]) const {
#pragma unroll
        for (int n = 0; n < D / 16; ++n)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const T8 k8 = *reinterpret_cast<const T8*>(ks + (at_k ^ 16 * n) + 32 * x * D);
                s[x] = mfma(k8, q[n], n ? s[x] : f32x16{});
            }
    }

    // Hides keys from `limit` on, in the tile from key k0.
    __device__ __forceinline__ void mask(f32x16 (&s)[2], int k0, int limit) const {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (32 * x + 8 * (r / 4) + r % 4 >= limit - k0 - 4 * hf) s[x][r] = -INFINITY;
    }

    // Raises the maximum m where scores of the tile exceed it by 2^kSlack.
    __device__ __forceinline__ void raise(const f32x16 (&s)[2]) {
        float top = s[0][0];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[x][r]);
        top *= scale;
        if (!__any(top > m + (kSlack + weight_lift<T>()))) return;
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m2 = fmaxf(m, top - weight_lift<T>()), c = exp2_(m - m2);
        m = m2;
        l *= c;
#pragma unroll
        for (int d = 0; d < D / 32; ++d) o[d] *= c;
    }

    // The tile's weights from its scores.
    __device__ __forceinline__ void weights(const f32x16 (&s)[2]) {
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

// Division of n < 2^31 by d as a product and a shift: (mulhi(n, magic) + n) >>
// shift with 2^shift >= d and magic = floor(2^32 (2^shift - d) / d) + 1.
struct Divisor {
    uint32_t magic, shift;
};

Divisor divisor(uint32_t d) {
    uint32_t shift = 0;
    while ((uint64_t{1} << shift) < d) ++shift;
    return {static_cast<uint32_t>((((uint64_t{1} << shift) - d) << 32) / d + 1), shift};
}

__device__ inline int quotient(int n, Divisor d) {
    return static_cast<int>((__umulhi(static_cast<uint32_t>(n), d.magic) + static_cast<uint32_t>(n)) >> d.shift);
}

// (Divisions are made ready on the host: they were 350 of 900 instructions
// before the first product, 0.3 to 0.5 us of a workgroup's 5.)
struct Prompt {
    PromptArgs a;
    float scale_log2;
    int group;        // query heads of a key head
    int splits;       // parts that a tile's keys are split into, a workgroup each
    int parts;        // workgroups of a tile: key heads times splits
    int spread;       // key heads of an XCD; 0: they do not go evenly
    int at_once;      // tiles of the first kCUs workgroups ...
    int order;        // ... and of all, where those that share a CU are paired, else 0
    Divisor by_parts, by_group, by_heads;
    float* part;      // [query][head][splits][D] sums of the parts, where there are several
    float2* part_ml;  // and their maximum (log2) and sum
};

template <int D, typename T>
__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(Prompt g) {
    typedef typename Vec8<T>::type T8;
    const PromptArgs& a = g.a;
    constexpr int kQ = 32, kTile = kKeys * D, kChunks = D / 8;
    constexpr int kLoads = kTile * 2 / (16 * kThreads);  // loads a thread of a tile of keys or values
    __shared__ __attribute__((aligned(16))) T sk[2][kTile];
    __shared__ __attribute__((aligned(16))) T sv[2][kTile];
    __shared__ int64_t row_at[kTileQ];
    __shared__ int bad_tile;  // 1 + the last tile found to hold values that are not finite
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
    const int i = lane & 31, hf = lane >> 5;

    // workgroups of a key head go to one XCD (they go round the eight)
    int tile = quotient(blockIdx.x, g.by_parts);
    int kv = blockIdx.x - tile * g.parts, part = 0;
    if (g.splits > 1) {
        part = quotient(kv, g.by_heads);
        kv -= part * a.kv_heads;
    }
    if (g.spread) kv = kv % 8 * g.spread + kv / 8;
    // Tiles go in the order of their work, most first: sequences with most
    // keys first (of 64 at a time), and of a sequence the late tiles, which
    // see most.  Workgroups i and i + kCUs share a CU: where all are resident,
    // those with most work have a CU to themselves or share it with those with
    // least (2048 tokens of 32 heads 53.7 us for 55, 1536 tokens 36 for 37).
    if (g.order) {
        const int alone = 2 * g.at_once - g.order;
        tile = tile >= g.at_once ? g.order - 1 - (tile - g.at_once)
                                 : tile + alone < g.at_once ? tile + alone : tile + alone - g.at_once;
    }
    // the sequence of the tile: its tiles are its queries times the group's heads, 128 a tile
    int first = 0, q_first = 0, nq = 0, k_first = 0, nk = 0;
    for (int base = 0;; base += 64) {
        if (base >= a.sequences) return;
        int c0 = 0, c1 = 0, d0 = 0, d1 = 0;
        if (base + lane < a.sequences) {
            c0 = a.cu_q[base + lane], c1 = a.cu_q[base + lane + 1];
            d0 = a.cu_k[base + lane], d1 = a.cu_k[base + lane + 1];
        }
        const int most_q = static_cast<int>(a.q_tokens), most_k = static_cast<int>(a.k_tokens);
        c0 = min(max(c0, 0), most_q), c1 = min(max(c1, c0), most_q), d0 = min(max(d0, 0), most_k), d1 = min(max(d1, d0), most_k);
        if (a.sequences > 1) {
            const int many = min(64, static_cast<int>(a.sequences) - base);
            int before = 0;  // sequences that go before the lane's
            for (int j = 0; j < many; ++j) {
                const int other = __builtin_amdgcn_readlane(d1 - d0, j);
                before += other > d1 - d0 || (other == d1 - d0 && j < lane);
            }
            if (lane >= many) before = lane;
            c0 = __builtin_amdgcn_ds_permute(4 * before, c0), c1 = __builtin_amdgcn_ds_permute(4 * before, c1);
            d0 = __builtin_amdgcn_ds_permute(4 * before, d0), d1 = __builtin_amdgcn_ds_permute(4 * before, d1);
        }
        const int tiles = ((c1 - c0) * g.group + kTileQ - 1) / kTileQ;
        const int sum = scan64(tiles);
        const uint64_t in = __ballot(tile < first + sum);
        if (in) {
            const int l = __ffsll(static_cast<unsigned long long>(in)) - 1;
            tile = first + __builtin_amdgcn_readlane(sum, l) - 1 - tile;
            q_first = __builtin_amdgcn_readlane(c0, l);
            nq = __builtin_amdgcn_readlane(c1, l) - q_first;
            k_first = __builtin_amdgcn_readlane(d0, l);
            nk = __builtin_amdgcn_readlane(d1, l) - k_first;
            break;
        }
        first += __builtin_amdgcn_readlane(sum, 63);
    }
    // rows are (query, head of the group)
    const int rows = nq * g.group, row0 = tile * kTileQ, wave_row = row0 + wave * kQ;
    const int row = min(wave_row + i, rows - 1);
    const bool live = wave_row + i < rows;
    const int qi = quotient(max(row, 0), g.by_group), head = kv * g.group + row - qi * g.group;

    // the lane's row: keys below `limit` are seen
    const int more = nk - nq + 1;
    const int limit = !live ? 0 : a.causal ? qi + more : nk;
    const int wave_low = a.causal ? quotient(wave_row, g.by_group) + more : nk;  // seen by all its rows
    const int block_low = a.causal ? quotient(row0, g.by_group) + more : nk;  // seen by all rows of the tile
    const int keys = a.causal ? min(nk, quotient(min(row0 + kTileQ, rows) - 1, g.by_group) + more) : nk;  // seen by any
    Wave<D, T> w;
    w.hf = hf;
    w.at_k = i * D + (hf ^ turn_k<D>(i)) * 8;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
        const int r = 4 * hf + (i & 15) / 4, dim = 32 * d + (i & 16) + 4 * (i & 3);
        w.at_v[d] = r * D + ((dim / 8) ^ turn_v<D>(r)) * 8 + dim % 8;
    }
    w.scale = g.scale_log2;
    w.m = -FLT_MAX;
    w.l = 0.0f;
    {
        const T* x = static_cast<const T*>(a.q.p) + static_cast<int64_t>(q_first + qi) * a.q.ts + head * a.q.hs + 8 * hf;
#pragma unroll
        for (int n = 0; n < D / 16; ++n) w.q[n] = *reinterpret_cast<const T8*>(x + 16 * n);
    }
#pragma unroll
    for (int d = 0; d < D / 32; ++d) w.o[d] = f32x16{};

    // The part's tiles of keys: those before `plain` are seen whole by all the
    // workgroup's rows, before `whole` by the wave's.
    const int all_tiles = keys > 0 ? (keys + kKeys - 1) / kKeys : 0;
    int from = 0, tiles = all_tiles;
    if (g.splits > 1) {  // (at most 32, of at most 2^24 tiles)
        from = all_tiles * part / g.splits;
        tiles = all_tiles * (part + 1) / g.splits - from;
    }
    const int plain = max(0, block_low) / kKeys - from;
    const int whole = max(0, wave_low) / kKeys - from;
    const int key0 = from * kKeys;
    const T* kp = static_cast<const T*>(a.k.p) + static_cast<int64_t>(k_first + key0) * a.k.ts + kv * a.k.hs;
    const T* vp = static_cast<const T*>(a.v.p) + static_cast<int64_t>(k_first + key0) * a.v.ts + kv * a.v.hs;
    uint32_t off_k[kLoads], off_v[kLoads];
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
        off_k[n] = load_offset<D, false>(n, threadIdx.x, a.k.ts);
        off_v[n] = load_offset<D, true>(n, threadIdx.x, a.v.ts);
    }
    // tiles are loaded in turn; past the end, zeros
    int left_k = nk - key0, left_v = left_k;  // rows from the next tile on
    const auto next_k = [&](int slot) __attribute__((always_inline)) {
        const TileLoad<D, T> l(kp, a.k.ts, min(kKeys, left_k), sk[slot], wave);
        kp += kKeys * a.k.ts;
        left_k -= kKeys;
        return l;
    };
    const auto next_v = [&](int slot) __attribute__((always_inline)) {
        const TileLoad<D, T> l(vp, a.v.ts, min(kKeys, left_v), sv[slot], wave);
        vp += kKeys * a.v.ts;
        left_v -= kKeys;
        return l;
    };
    Spoiled spoiled{0, 0};
    if (threadIdx.x == 0) bad_tile = 0;

    f32x16 s[2];
    // Before the values of tile t: where rows see different keys, those that
    // are not finite are taken out and marked.
    const auto check_values = [&](int t, T* vs) __attribute__((always_inline)) {
        if (!a.causal || t < plain) return;
        if (any_not_finite<D, T>(vs, wave, lane)) bad_tile = t + 1;
        local_phase();
        if (bad_tile == t + 1) {
            mark_not_finite<D, T>(vs, key0 + t * kKeys, limit, lane, spoiled);
            local_phase();
            drop_not_finite<D, T>(vs, wave, lane);
            local_phase();
        }
    };
    // Tile t's weights; then its values and the next tile's scores in one run
    // of products, with the loads of the tiles after them: one barrier a tile.
    if (tiles > 0) {
        next_k(0).issue(off_k);
        next_v(0).issue(off_v);
        next_k(1).issue(off_k);
        wait_loads<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        // (the queries too: the compiler would go on waiting for them in the loop)
#pragma unroll
        for (int n = 0; n < D / 16; ++n) asm volatile("" : "+v"(w.q[n]));
        phase();
        w.scores(sk[0], s);
        for (int t = 0; t < tiles; ++t) {
            const int slot = t & 1;
            if (t >= whole) w.mask(s, key0 + t * kKeys, limit);
            w.raise(s);
            w.weights(s);
            wait_loads<0>();
            phase();  // keys t + 1 and values t are there; keys t and values t - 1 are done with
            next_k(slot).issue(off_k);
            next_v(slot ^ 1).issue(off_v);
            check_values(t, sv[slot]);
            __builtin_amdgcn_s_setprio(1);
            w.values(sv[slot]);
            w.scores(sk[slot ^ 1], s);  // (after the last tile: zeros or what was there, and not used)
            schedule_products<D>();
            __builtin_amdgcn_s_setprio(0);
        }
        wait_loads<0>();  // none may come to LDS after this
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
    const int64_t out_row = static_cast<int64_t>(q_first + qi) * a.q_heads + head;
    if (g.splits > 1) {
        if (!live) return;
        float* to = g.part + (out_row * g.splits + part) * D + 4 * hf;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<f32x4*>(to + 32 * d + 8 * r) =
                    f32x4{w.o[d][4 * r], w.o[d][4 * r + 1], w.o[d][4 * r + 2], w.o[d][4 * r + 3]};
        if (hf == 0) g.part_ml[out_row * g.splits + part] = float2{w.m, w.l};
        return;
    }
    // Results go out through LDS, so that a row leaves as a whole.
    const float inv = w.l == 0.0f ? 0.0f : 1.0f / w.l;
    if (a.lse && live && hf == 0) a.lse[out_row] = (w.m + log2f(w.l)) * kLn2;
    phase();  // all waves are done with the tiles
    T* mine = sk[0] + wave * kQ * D;
    if (hf == 0) row_at[wave * kQ + i] = live ? static_cast<int64_t>(q_first + qi) * a.out.ts + head * a.out.hs : -1;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            typedef T T4 __attribute__((ext_vector_type(4)));
            T4 v;
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = static_cast<T>(w.o[d][4 * r + x] * inv);
            *reinterpret_cast<T4*>(mine + i * D + ((4 * d + r) ^ (i & (kChunks - 1))) * 8 + 4 * hf) = v;
        }
    __builtin_amdgcn_wave_barrier();  // a wave reads its own rows only
#pragma unroll
    for (int n = 0; n < kQ * kChunks / 64; ++n) {
        const int r = (n * 64 + lane) / kChunks, place = lane % kChunks;
        const T8 v = *reinterpret_cast<const T8*>(mine + r * D + place * 8);
        const int64_t at = row_at[wave * kQ + r];
        if (at >= 0) *reinterpret_cast<T8*>(static_cast<T*>(a.out.p) + at + (place ^ (r & (kChunks - 1))) * 8) = v;
    }
}

// Workgroups without a split, at most (every sequence may end with a part of a tile).
int64_t prompt_blocks(int64_t sequences, int64_t q_tokens, int q_heads, int kv_heads) {
    return (q_tokens * (q_heads / kv_heads) + (kTileQ - 1) * sequences) / kTileQ * kv_heads;
}

// Few rows before many keys: the keys are split, so that there are up to two
// workgroups a CU, if that is expected to take less time than it costs.  A tile
// of keys takes a workgroup about 1.1 us, the launch that joins the parts 5 us
// and what their sums (written and read) take at 3.5 TB/s.  (These are measured
// with head_dim 128, and taken for 64 too, where a tile costs less: 2048 tokens of
// 32 heads 36 us for 51.)  Of a batch's
// lengths only the mean is known here: its longest sequence is taken to have
// twice that.
int prompt_splits(int64_t sequences, int64_t q_tokens, int64_t k_tokens, int q_heads, int kv_heads, int head_dim) {
    const int64_t blocks = std::max<int64_t>(1, prompt_blocks(sequences, q_tokens, q_heads, kv_heads));
    const double tiles = static_cast<double>(std::min(k_tokens, 2 * k_tokens / sequences)) / kKeys;
    const double sums = 8e-6 / 3.5 * static_cast<double>(q_tokens) * q_heads * head_dim;  // us a part
    int best = 1;
    double least = 1.1 * tiles;
    for (int n = 2; n <= 32 && n * blocks <= kResident && n * 2 <= tiles; ++n) {
        const double us = 1.1 * tiles / n + 5.0 + sums * n;
        if (us < least) least = us, best = n;
    }
    return best;
}

template <int D, typename T>
hipError_t run(const PromptArgs& a, void* workspace, hipStream_t s) {
    Prompt g{};
    g.a = a;
    g.scale_log2 = a.scale * kLog2e;
    g.group = a.q_heads / a.kv_heads;
    g.splits = prompt_splits(a.sequences, a.q_tokens, a.k_tokens, a.q_heads, a.kv_heads, D);
    g.parts = a.kv_heads * g.splits;
    g.spread = a.kv_heads % 8 == 0 ? a.kv_heads / 8 : 0;
    g.by_parts = divisor(g.parts);
    g.by_group = divisor(g.group);
    g.by_heads = divisor(a.kv_heads);
    const uint32_t blocks = static_cast<uint32_t>(prompt_blocks(a.sequences, a.q_tokens, a.q_heads, a.kv_heads) * g.splits);
    if (blocks > kCUs && blocks <= kResident && kCUs % g.parts == 0) {
        g.at_once = kCUs / g.parts;
        g.order = static_cast<int>(blocks) / g.parts;
    }
    const int64_t rows = a.q_tokens * a.q_heads;
    if (g.splits > 1) {
        g.part = static_cast<float*>(workspace);
        g.part_ml = reinterpret_cast<float2*>(g.part + rows * g.splits * D);
    }
    prompt_kernel<D, T><<<blocks, kThreads, 0, s>>>(g);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || g.splits == 1) return e;
    Join j{};
    j.part = g.part;
    j.part_ml = g.part_ml;
    j.rows = rows;
    j.slots = g.splits;
    j.expected = g.splits;
    j.q_heads = a.q_heads;
    j.out = a.out;
    j.lse = a.lse;
    j.tokens = a.cu_q + a.sequences;
    return launch_join<D, T>(j, s);
}

}  // namespace

size_t prompt_workspace_bytes(int64_t sequences, int64_t q_tokens, int64_t k_tokens, int q_heads, int kv_heads,
                              int head_dim) {
    const int n = prompt_splits(sequences, q_tokens, k_tokens, q_heads, kv_heads, head_dim);
    return n == 1 ? 0 : static_cast<size_t>(q_tokens * q_heads) * n * (head_dim + 2) * 4;
}

hipError_t launch_attn_prompt(const PromptArgs& a, void* workspace, hipStream_t s) {
    if (a.head_dim == 128)
        return a.dtype == UNISVQ_F16 ? run<128, _Float16>(a, workspace, s) : run<128, __bf16>(a, workspace, s);
    return a.dtype == UNISVQ_F16 ? run<64, _Float16>(a, workspace, s) : run<64, __bf16>(a, workspace, s);
}

}  // namespace unisvq
