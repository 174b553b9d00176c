// C entry points of the attention block: argument validation (host only,
// before any HIP call) and dispatch to the kernels.
#include <cmath>

#include "attn.hpp"

namespace {

using unisvq::CacheView;
using unisvq::Rotary;
using unisvq::Rows;

constexpr int64_t kMost = (int64_t{1} << 31) - 1;
constexpr int64_t kMostGroups = (int64_t{1} << 24) - 1;  // of 256 threads: a launch has fewer than 2^32
// Tokens that a page table may span: positions and the kernels' counts along a
// sequence are 32-bit integers.
constexpr int64_t kMaxContext = int64_t{1} << 30;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int status(hipError_t e) { return e == hipSuccess ? UNISVQ_OK : UNISVQ_EHIP; }
bool dtype_ok(int t) { return t == UNISVQ_F16 || t == UNISVQ_BF16; }

// Rows that the kernels read and write 16 bytes at a time.
bool rows_aligned(const void* p, int64_t ts, int64_t hs) { return aligned(p, 16) && ts % 8 == 0 && hs % 8 == 0; }
Rows rows(const void* p, int64_t ts, int64_t hs) { return Rows{const_cast<void*>(p), ts, hs}; }

int check_rotary(const float* table, int64_t positions, int64_t rot, int64_t head_dim) {
    if (positions < 1 || positions > kMost) return UNISVQ_EINVAL;
    if (rot < 16 || rot % 16 != 0 || rot > head_dim) return UNISVQ_EUNSUP;
    return aligned(table, 16) ? UNISVQ_OK : UNISVQ_EALIGN;
}

// A cache and its page table; `sequences` may be 0 (nothing to do).
int check_cache(const unisvq_cache* c, const int32_t* page_table, int64_t sequences, int64_t width, CacheView* out) {
    if (!c || sequences < 0 || sequences > kMost || width < 0) return UNISVQ_EINVAL;
    if (c->kind < UNISVQ_CACHE_F16 || c->kind > UNISVQ_CACHE_I4) return UNISVQ_EINVAL;
    if (c->pages < 1 || c->pages > kMost || c->kv_heads < 1 || c->kv_heads > 65535) return UNISVQ_EINVAL;
    int shift = 4;
    while (shift < 8 && (int64_t{1} << shift) != c->page_tokens) ++shift;
    if ((int64_t{1} << shift) != c->page_tokens || (c->head_dim != 64 && c->head_dim != 128)) return UNISVQ_EUNSUP;
    const bool scaled = c->kind == UNISVQ_CACHE_I8 || c->kind == UNISVQ_CACHE_I4;
    if (!c->k || !c->v || (scaled && (!c->k_scales || !c->v_scales))) return UNISVQ_EINVAL;
    if (sequences && width && !page_table) return UNISVQ_EINVAL;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(page_table, 4)) return UNISVQ_EALIGN;
    if (scaled && (!aligned(c->k_scales, 16) || !aligned(c->v_scales, 16))) return UNISVQ_EALIGN;
    if (width > kMaxContext >> shift) return UNISVQ_EUNSUP;
    *out = CacheView{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), static_cast<uint32_t*>(c->k_scales),
                     static_cast<uint32_t*>(c->v_scales), page_table, sequences, width, c->pages, shift,
                     static_cast<int>(c->kv_heads), static_cast<int>(c->head_dim), c->kind};
    return UNISVQ_OK;
}

// A 16-bit kind holds the activations' own type.
bool kind_serves(int kind, int dtype) {
    return kind == UNISVQ_CACHE_F16 ? dtype == UNISVQ_F16 : kind == UNISVQ_CACHE_BF16 ? dtype == UNISVQ_BF16 : true;
}

// Scores are multiplied by scale * log2(e) in fp32.
bool scale_ok(float scale) { return scale > 0 && std::isfinite(scale * 1.44269504088896340736f); }

bool heads_ok(int64_t q_heads, int64_t kv_heads) {
    return kv_heads >= 1 && q_heads >= kv_heads && q_heads <= 65535 && q_heads % kv_heads == 0;
}

}  // namespace

extern "C" {

int unisvq_rope_table(int64_t positions, int64_t rot, double theta, double factor, double low, double high,
                      double original, double magnitude, float* table, void* stream) {
    if (!table || positions < 1 || positions > (int64_t{1} << 24) || rot < 2 || rot > 1024 || rot % 2 != 0)
        return UNISVQ_EINVAL;
    if (!(theta > 0) || !(factor > 0) || !(original >= 0) || !std::isfinite(theta) || !std::isfinite(factor) ||
        !std::isfinite(original) || !std::isfinite(magnitude))
        return UNISVQ_EINVAL;
    if (original > 0 && !(high > low && std::isfinite(high - low))) return UNISVQ_EINVAL;
    if (!aligned(table, 16)) return UNISVQ_EALIGN;
    return status(unisvq::launch_rope_table(positions, static_cast<int>(rot), theta, factor, low, high, original,
                                            magnitude, table, static_cast<hipStream_t>(stream)));
}

int unisvq_rope(int64_t tokens, int64_t heads, int64_t head_dim, int64_t rot, int interleaved, int inverse,
                const void* x, int64_t x_token_stride, int64_t x_head_stride, const int32_t* positions,
                const float* table, int64_t table_positions, void* y, int64_t y_token_stride, int64_t y_head_stride,
                int dtype, void* stream) {
    if (tokens < 0 || heads < 1 || !dtype_ok(dtype)) return UNISVQ_EINVAL;
    if (head_dim < 16 || head_dim > 1024 || head_dim % 16 != 0) return UNISVQ_EUNSUP;
    if (tokens > 0 && (!x || !positions || !table || !y)) return UNISVQ_EINVAL;
    const int st = check_rotary(table, table_positions, rot, head_dim);
    if (st != UNISVQ_OK) return st;
    if (!rows_aligned(x, x_token_stride, x_head_stride) || !rows_aligned(y, y_token_stride, y_head_stride) ||
        !aligned(positions, 4))
        return UNISVQ_EALIGN;
    if (tokens > kMost || heads > kMost / 64 || tokens * heads > kMost / (head_dim / 16)) return UNISVQ_EUNSUP;
    if (tokens == 0) return UNISVQ_OK;
    const Rotary rotary{table, table_positions, static_cast<int>(rot), interleaved != 0, inverse != 0};
    return status(unisvq::launch_rope(tokens, static_cast<int>(heads), static_cast<int>(head_dim), rotary,
                                      rows(x, x_token_stride, x_head_stride), positions,
                                      rows(y, y_token_stride, y_head_stride), dtype, static_cast<hipStream_t>(stream)));
}

int unisvq_cache_append(const unisvq_cache* cache, const int32_t* page_table, int64_t sequences, int64_t table_width,
                        int64_t tokens, const int32_t* seqs, const int32_t* positions, const void* k,
                        int64_t k_token_stride, int64_t k_head_stride, const void* v, int64_t v_token_stride,
                        int64_t v_head_stride, const void* q, int64_t q_heads, int64_t q_token_stride,
                        int64_t q_head_stride, void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride,
                        int x_dtype, const float* rope_table, int64_t table_positions, int64_t rot, int interleaved,
                        void* stream) {
    CacheView c;
    int st = check_cache(cache, page_table, sequences, table_width, &c);
    if (st != UNISVQ_OK) return st;
    if (tokens < 0 || tokens > kMost || !dtype_ok(x_dtype) || q_heads < 0 || q_heads > 65535) return UNISVQ_EINVAL;
    if (!kind_serves(c.kind, x_dtype)) return UNISVQ_EUNSUP;
    if (tokens > 0 && (!positions || !k || !v || (q_heads > 0 && (!q || !q_out)))) return UNISVQ_EINVAL;
    if (rope_table) {
        st = check_rotary(rope_table, table_positions, rot, c.head_dim);
        if (st != UNISVQ_OK) return st;
    }
    if (!rows_aligned(k, k_token_stride, k_head_stride) || !rows_aligned(v, v_token_stride, v_head_stride) ||
        (q_heads > 0 && (!rows_aligned(q, q_token_stride, q_head_stride) ||
                         !rows_aligned(q_out, q_out_token_stride, q_out_head_stride))) ||
        !aligned(seqs, 4) || !aligned(positions, 4))
        return UNISVQ_EALIGN;
    if (tokens > kMost / ((q_heads + 2 * c.heads) * (c.head_dim / 16))) return UNISVQ_EUNSUP;
    if (tokens == 0) return UNISVQ_OK;
    const Rotary rotary{rope_table, table_positions, static_cast<int>(rot), interleaved != 0, 0};
    return status(unisvq::launch_cache_append(
        c, tokens, seqs, positions, rows(k, k_token_stride, k_head_stride), rows(v, v_token_stride, v_head_stride),
        rows(q, q_token_stride, q_head_stride), static_cast<int>(q_heads),
        rows(q_out, q_out_token_stride, q_out_head_stride), x_dtype, rotary, static_cast<hipStream_t>(stream)));
}

int unisvq_cache_read(const unisvq_cache* cache, const int32_t* page_table, int64_t sequences, int64_t table_width,
                      const int32_t* starts, const int32_t* cu, int64_t tokens, void* k_out, int64_t k_token_stride,
                      int64_t k_head_stride, void* v_out, int64_t v_token_stride, int64_t v_head_stride, int dtype,
                      void* stream) {
    CacheView c;
    const int st = check_cache(cache, page_table, sequences, table_width, &c);
    if (st != UNISVQ_OK) return st;
    if (tokens < 0 || tokens > kMost || !dtype_ok(dtype)) return UNISVQ_EINVAL;
    if (tokens > 0 && (!cu || !k_out || !v_out)) return UNISVQ_EINVAL;
    if (!rows_aligned(k_out, k_token_stride, k_head_stride) || !rows_aligned(v_out, v_token_stride, v_head_stride) ||
        !aligned(starts, 4) || !aligned(cu, 4))
        return UNISVQ_EALIGN;
    if (tokens > kMost / (c.heads * (c.head_dim / 16))) return UNISVQ_EUNSUP;
    if (tokens == 0 || sequences == 0) return UNISVQ_OK;
    return status(unisvq::launch_cache_read(c, starts, cu, tokens, rows(k_out, k_token_stride, k_head_stride),
                                            rows(v_out, v_token_stride, v_head_stride), dtype,
                                            static_cast<hipStream_t>(stream)));
}

namespace {

bool decode_shape_ok(int64_t sequences, int64_t q_len, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                     int64_t max_len) {
    return sequences >= 0 && sequences <= kMost && q_len >= 1 && q_len <= 16 && heads_ok(q_heads, kv_heads) &&
           (head_dim == 64 || head_dim == 128) && max_len >= 0 && max_len <= kMaxContext;
}

}  // namespace

size_t unisvq_attn_decode_workspace_bytes(int64_t sequences, int64_t q_len, int64_t q_heads, int64_t kv_heads,
                                          int64_t head_dim, int64_t max_len) {
    if (!decode_shape_ok(sequences, q_len, q_heads, kv_heads, head_dim, max_len) || sequences == 0) return 0;
    if (max_len == 0) max_len = kMaxContext;  // any page table's width: more is never needed for less
    // for the 16-bit kinds, which are split first
    const int slots = unisvq::decode_slots(sequences, static_cast<int>(q_len), static_cast<int>(q_heads),
                                           static_cast<int>(kv_heads), max_len, static_cast<int>(4 * head_dim));
    return unisvq::decode_workspace_bytes(sequences, static_cast<int>(q_len), static_cast<int>(q_heads),
                                          static_cast<int>(head_dim), slots);
}

int unisvq_attn_decode(const unisvq_cache* cache, const int32_t* page_table, int64_t sequences, int64_t table_width,
                       const int32_t* lens, int64_t max_len, int64_t q_len, int64_t q_heads, const void* q,
                       int64_t q_token_stride, int64_t q_head_stride, int x_dtype, float scale, void* out,
                       int64_t out_token_stride, int64_t out_head_stride, float* lse, void* workspace,
                       size_t workspace_bytes, void* stream) {
    CacheView c;
    const int st = check_cache(cache, page_table, sequences, table_width, &c);
    if (st != UNISVQ_OK) return st;
    const int64_t room = table_width * cache->page_tokens;
    if (max_len == 0 || max_len > room) max_len = room;
    if (!dtype_ok(x_dtype) || !scale_ok(scale) ||
        !decode_shape_ok(sequences, q_len, q_heads, c.heads, c.head_dim, max_len))
        return UNISVQ_EINVAL;
    if (!kind_serves(c.kind, x_dtype)) return UNISVQ_EUNSUP;
    if (sequences == 0) return UNISVQ_OK;
    if (!lens || !q || !out) return UNISVQ_EINVAL;
    if (!rows_aligned(q, q_token_stride, q_head_stride) || !rows_aligned(out, out_token_stride, out_head_stride) ||
        !aligned(lens, 4) || !aligned(lse, 4))
        return UNISVQ_EALIGN;
    const int slots = unisvq::decode_slots(sequences, static_cast<int>(q_len), static_cast<int>(q_heads), c.heads,
                                           max_len, c.head_dim * unisvq::entry_bits(c.kind) / 4);
    // workgroups and units of work are counted in 32 bits
    const int64_t row_tiles = (q_len * (q_heads / c.heads) + 15) / 16;
    if (sequences > kMostGroups / (c.heads * row_tiles) || c.heads * row_tiles > kMost / 2 / (room / 128 + 1) ||
        sequences > kMost / 2 / (c.heads * row_tiles * (room / 128 + 1)))
        return UNISVQ_EUNSUP;
    const size_t need = unisvq::decode_workspace_bytes(sequences, static_cast<int>(q_len), static_cast<int>(q_heads),
                                                       c.head_dim, slots);
    if (need) {
        if (!workspace || workspace_bytes < need) return UNISVQ_EWORKSPACE;
        if (!aligned(workspace, 16)) return UNISVQ_EALIGN;
    }
    return status(unisvq::launch_attn_decode(c, lens, max_len, slots, static_cast<int>(q_len),
                                             static_cast<int>(q_heads), rows(q, q_token_stride, q_head_stride),
                                             x_dtype, scale, rows(out, out_token_stride, out_head_stride), lse,
                                             workspace, static_cast<hipStream_t>(stream)));
}

size_t unisvq_attn_prompt_workspace_bytes(int64_t sequences, int64_t q_tokens, int64_t k_tokens, int64_t q_heads,
                                          int64_t kv_heads, int64_t head_dim) {
    if (sequences < 1 || sequences > kMost || q_tokens < 1 || q_tokens > kMost || k_tokens < 0 || k_tokens > kMost ||
        !heads_ok(q_heads, kv_heads) || (head_dim != 64 && head_dim != 128))
        return 0;
    return unisvq::prompt_workspace_bytes(sequences, q_tokens, k_tokens, static_cast<int>(q_heads),
                                          static_cast<int>(kv_heads), static_cast<int>(head_dim));
}

int unisvq_attn_prompt(int64_t sequences, int64_t q_tokens, int64_t k_tokens, const int32_t* cu_q,
                       const int32_t* cu_k, int64_t q_heads, int64_t kv_heads, int64_t head_dim, const void* q,
                       int64_t q_token_stride, int64_t q_head_stride, const void* k, int64_t k_token_stride,
                       int64_t k_head_stride, const void* v, int64_t v_token_stride, int64_t v_head_stride, int dtype,
                       int causal, float scale, void* out, int64_t out_token_stride, int64_t out_head_stride,
                       float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (sequences < 0 || sequences > kMost || q_tokens < 0 || q_tokens > kMaxContext || k_tokens < 0 ||
        k_tokens > kMaxContext || !dtype_ok(dtype) || !scale_ok(scale) || !heads_ok(q_heads, kv_heads))
        return UNISVQ_EINVAL;
    if (head_dim != 64 && head_dim != 128) return UNISVQ_EUNSUP;
    if (sequences == 0 || q_tokens == 0) return UNISVQ_OK;
    if (!cu_q || !cu_k || !q || !out || (k_tokens > 0 && (!k || !v))) return UNISVQ_EINVAL;
    if (!rows_aligned(q, q_token_stride, q_head_stride) || !rows_aligned(k, k_token_stride, k_head_stride) ||
        !rows_aligned(v, v_token_stride, v_head_stride) || !rows_aligned(out, out_token_stride, out_head_stride) ||
        !aligned(cu_q, 4) || !aligned(cu_k, 4) || !aligned(lse, 4))
        return UNISVQ_EALIGN;
    // tiles of keys and values are addressed with 32-bit offsets from their first row, and end with their last
    const int64_t wide = int64_t{1} << 22;
    if (k_token_stride < head_dim || k_token_stride > wide || v_token_stride < head_dim || v_token_stride > wide)
        return UNISVQ_EUNSUP;
    // rows are counted in 32 bits
    if (q_tokens > kMost / q_heads || q_tokens * q_heads / 128 + sequences * kv_heads > kMostGroups) return UNISVQ_EUNSUP;
    const size_t need = unisvq::prompt_workspace_bytes(sequences, q_tokens, k_tokens, static_cast<int>(q_heads),
                                                       static_cast<int>(kv_heads), static_cast<int>(head_dim));
    if (need) {
        if (!workspace || workspace_bytes < need) return UNISVQ_EWORKSPACE;
        if (!aligned(workspace, 16)) return UNISVQ_EALIGN;
    }
    const unisvq::PromptArgs a{cu_q, cu_k, sequences, q_tokens, k_tokens, static_cast<int>(q_heads),
                               static_cast<int>(kv_heads), static_cast<int>(head_dim),
                               rows(q, q_token_stride, q_head_stride), rows(k, k_token_stride, k_head_stride),
                               rows(v, v_token_stride, v_head_stride), rows(out, out_token_stride, out_head_stride),
                               dtype, causal != 0, scale, lse};
    return status(unisvq::launch_attn_prompt(a, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
