// C entry points of the norm, the gated activation and the 4-bit products:
// argument validation (host only, before any HIP call) and dispatch.
#include <algorithm>
#include <cmath>
#include <limits>

#include "layer.hpp"

namespace {

using unisvq::FourbitProblem;
using unisvq::bytes_meet;

constexpr int64_t kMost = (int64_t{1} << 31) - 1;
// Columns of 4-bit weights: 128 tokens' rows stay within 32-bit offsets.
constexpr int64_t kMostColumns = int64_t{1} << 20;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int status(hipError_t e) { return e == hipSuccess ? UNISVQ_OK : UNISVQ_EHIP; }
int size_of(int t) { return t == UNISVQ_I8 ? 1 : t == UNISVQ_F32 ? 4 : 2; }
bool half_type(int t) { return t == UNISVQ_F16 || t == UNISVQ_BF16; }
// (a single row's stride says nothing)
bool row_aligned(const void* p, int64_t stride, int64_t tokens) { return aligned(p, 16) && (tokens <= 1 || stride % 8 == 0); }

// Rows of an output lie apart.
bool rows_apart(int64_t stride, int64_t n, int64_t tokens) { return tokens <= 1 || stride >= n || stride <= -n; }

// An operand of rows, in bytes: `count` of `width`, `stride` apart.
struct Rows {
    __int128 at, stride, width, count;
};
Rows rows_of(const void* p, int64_t stride, int64_t n, int64_t tokens, int size) {
    Rows r{static_cast<__int128>(reinterpret_cast<uintptr_t>(p)), static_cast<__int128>(stride) * size,
           static_cast<__int128>(n) * size, tokens};
    if (r.count == 1) r.stride = r.width;
    if (r.stride < 0) r.at += (r.count - 1) * r.stride, r.stride = -r.stride;  // (their order is of no matter)
    return r;
}
Rows row_of(const void* p, int64_t n, int size) { return rows_of(p, 0, n, 1, size); }

// Whether the bytes from..to have one in common with a row of r.
bool row_meets(__int128 from, __int128 to, const Rows& r) {
    if (to <= r.at) return false;
    // the last row that begins before `to`
    const __int128 last = r.stride ? std::min(r.count - 1, (to - 1 - r.at) / r.stride) : 0;
    return r.at + last * r.stride + r.width > from;
}

// Whether two operands have a byte in common (absent ones have none).  Rows of the same
// stride meet as the first of one does with those of the other; of different ones, where
// one operand lies about the other, they are gone through.
bool meet(const Rows& a, const Rows& b) {
    const __int128 a_end = a.at + (a.count - 1) * a.stride + a.width, b_end = b.at + (b.count - 1) * b.stride + b.width;
    if (!a.at || !b.at || a_end <= b.at || b_end <= a.at) return false;
    if (a.stride == b.stride) return row_meets(a.at, a.at + a.width, b) || row_meets(b.at, b.at + b.width, a);
    const Rows &wide = a.stride > b.stride ? a : b, &other = a.stride > b.stride ? b : a;
    const __int128 end = &other == &b ? b_end : a_end;
    for (__int128 t = std::max<__int128>(0, (other.at - wide.at - wide.width) / wide.stride); t < wide.count; ++t) {
        const __int128 from = wide.at + t * wide.stride;
        if (from >= end) break;
        if (row_meets(from, from + wide.width, other)) return true;
    }
    return false;
}

// An output lies apart from an input, or is the same rows of the same type.
bool in_place_ok(const void* out, int out_type, int64_t out_stride, const void* in, int type, int64_t stride, int64_t n, int64_t tokens) {
    if (out == in && out_type == type && (tokens <= 1 || out_stride == stride)) return true;
    return !meet(rows_of(out, out_stride, n, tokens, size_of(out_type)), rows_of(in, stride, n, tokens, size_of(type)));
}

// Rows of outputs: as x, fp32, or bytes with a scale a row.
int check_output(const void* y, int64_t stride, int64_t tokens, int y_dtype, int x_dtype, const float* scales) {
    if (y_dtype != x_dtype && y_dtype != UNISVQ_F32 && y_dtype != UNISVQ_I8)
        return half_type(y_dtype) ? UNISVQ_EUNSUP : UNISVQ_EINVAL;
    if (!row_aligned(y, stride, tokens) || !aligned(scales, 4)) return UNISVQ_EALIGN;
    return UNISVQ_OK;
}

bool fourbit_shape_ok(int64_t N, int64_t K) {
    return N >= unisvq::kRowBlock && K >= unisvq::kGroup && N % unisvq::kRowBlock == 0 && K % unisvq::kGroup == 0 &&
           N <= kMost && K <= kMost;
}

int check_fourbit(const unisvq_fourbit_problem& p, int64_t M, int x_dtype, int y_dtype) {
    if (!p.packed || !p.x || !p.y || (x_dtype == UNISVQ_I8) != (p.x_scales != nullptr)) return UNISVQ_EINVAL;
    if (M < 1 || M > kMost) return UNISVQ_EINVAL;
    if (!half_type(x_dtype) && x_dtype != UNISVQ_I8) return UNISVQ_EINVAL;
    if (!half_type(y_dtype) && y_dtype != UNISVQ_F32) return UNISVQ_EINVAL;
    if (!fourbit_shape_ok(p.N, p.K)) return UNISVQ_ESHAPE;
    if (!aligned(p.packed, 16) || !aligned(p.x, 16) || !aligned(p.x_scales, 4) || !aligned(p.y, y_dtype == UNISVQ_F32 ? 4 : 2))
        return UNISVQ_EALIGN;
    return p.K > kMostColumns ? UNISVQ_EUNSUP : UNISVQ_OK;
}

void fourbit_batch(const unisvq_fourbit_problem* problems, int count, FourbitProblem* out) {
    for (int i = 0; i < count; ++i)
        out[i] = FourbitProblem{static_cast<const uint8_t*>(problems[i].packed), problems[i].x, problems[i].x_scales,
                           problems[i].y, problems[i].N, problems[i].K};
}

}  // namespace

extern "C" {

int unisvq_rmsnorm(int64_t tokens, int64_t n, const void* x, int64_t x_stride, int x_dtype, const void* weight,
                   int weight_dtype, float weight_offset, float eps, const void* residual, int64_t residual_stride,
                   void* residual_out, int64_t residual_out_stride, int residual_dtype, void* y, int64_t y_stride,
                   int y_dtype, float* y_scales, void* stream) {
    if (tokens < 0 || tokens > kMost || n < 1 || !half_type(x_dtype)) return UNISVQ_EINVAL;
    if (!(eps >= std::numeric_limits<float>::min()) || !std::isfinite(eps) || !std::isfinite(weight_offset)) return UNISVQ_EINVAL;
    if ((residual == nullptr) != (residual_out == nullptr)) return UNISVQ_EINVAL;
    if (tokens > 0 && (!x || !weight || !y || (y_dtype == UNISVQ_I8 && !y_scales))) return UNISVQ_EINVAL;
    if (weight_dtype != x_dtype && weight_dtype != UNISVQ_F32) return half_type(weight_dtype) ? UNISVQ_EUNSUP : UNISVQ_EINVAL;
    if (residual && residual_dtype != x_dtype && residual_dtype != UNISVQ_F32)
        return half_type(residual_dtype) ? UNISVQ_EUNSUP : UNISVQ_EINVAL;
    const int st = check_output(y, y_stride, tokens, y_dtype, x_dtype, y_scales);
    if (st != UNISVQ_OK) return st;
    if (!row_aligned(x, x_stride, tokens) || !aligned(weight, 16) || !row_aligned(residual, residual ? residual_stride : 0, tokens) ||
        !row_aligned(residual_out, residual ? residual_out_stride : 0, tokens))
        return UNISVQ_EALIGN;
    if (n % 8 != 0 || n > unisvq::kMaxRow) return UNISVQ_EUNSUP;
    if (tokens == 0) return UNISVQ_OK;
    if (!rows_apart(y_stride, n, tokens) || !in_place_ok(y, y_dtype, y_stride, x, x_dtype, x_stride, n, tokens)) return UNISVQ_EINVAL;
    const Rows y_rows = rows_of(y, y_stride, n, tokens, size_of(y_dtype)), w_row = row_of(weight, n, size_of(weight_dtype));
    if (meet(y_rows, w_row)) return UNISVQ_EINVAL;
    if (residual) {
        const Rows h_rows = rows_of(residual_out, residual_out_stride, n, tokens, size_of(residual_dtype));
        if (!rows_apart(residual_out_stride, n, tokens) || meet(y_rows, h_rows) || meet(h_rows, w_row) ||
            !in_place_ok(y, y_dtype, y_stride, residual, residual_dtype, residual_stride, n, tokens) ||
            !in_place_ok(residual_out, residual_dtype, residual_out_stride, residual, residual_dtype, residual_stride, n, tokens) ||
            !in_place_ok(residual_out, residual_dtype, residual_out_stride, x, x_dtype, x_stride, n, tokens))
            return UNISVQ_EINVAL;
    }
    if (y_dtype == UNISVQ_I8) {
        const Rows scales = row_of(y_scales, tokens, 4);
        if (meet(scales, y_rows) || meet(scales, w_row) || meet(scales, rows_of(x, x_stride, n, tokens, size_of(x_dtype))) ||
            (residual && (meet(scales, rows_of(residual, residual_stride, n, tokens, size_of(residual_dtype))) ||
                          meet(scales, rows_of(residual_out, residual_out_stride, n, tokens, size_of(residual_dtype))))))
            return UNISVQ_EINVAL;
    }
    return status(unisvq::launch_rmsnorm(
        unisvq::NormArgs{tokens, static_cast<int>(n), x, weight, residual, residual_out, y, x_stride, residual_stride,
                         residual_out_stride, y_stride, x_dtype, weight_dtype, residual_dtype, y_dtype, weight_offset,
                         eps, y_scales},
        static_cast<hipStream_t>(stream)));
}

int unisvq_gated(int64_t tokens, int64_t n, const void* gate, int64_t gate_stride, const void* up, int64_t up_stride,
                 int x_dtype, int activation, void* y, int64_t y_stride, int y_dtype, float* y_scales, void* stream) {
    if (tokens < 0 || tokens > kMost || n < 1 || !half_type(x_dtype)) return UNISVQ_EINVAL;
    if (activation != UNISVQ_SILU && activation != UNISVQ_GELU) return UNISVQ_EINVAL;
    if (tokens > 0 && (!gate || !up || !y || (y_dtype == UNISVQ_I8 && !y_scales))) return UNISVQ_EINVAL;
    const int st = check_output(y, y_stride, tokens, y_dtype, x_dtype, y_scales);
    if (st != UNISVQ_OK) return st;
    if (!row_aligned(gate, gate_stride, tokens) || !row_aligned(up, up_stride, tokens)) return UNISVQ_EALIGN;
    if (n % 8 != 0 || (y_dtype == UNISVQ_I8 ? n > unisvq::kMaxRow : n > kMost || tokens * (n / 8) > kMost))
        return UNISVQ_EUNSUP;
    if (tokens == 0) return UNISVQ_OK;
    if (!rows_apart(y_stride, n, tokens) || !in_place_ok(y, y_dtype, y_stride, gate, x_dtype, gate_stride, n, tokens) ||
        !in_place_ok(y, y_dtype, y_stride, up, x_dtype, up_stride, n, tokens))
        return UNISVQ_EINVAL;
    if (y_dtype == UNISVQ_I8) {
        const Rows scales = row_of(y_scales, tokens, 4);
        if (meet(scales, rows_of(y, y_stride, n, tokens, 1)) || meet(scales, rows_of(gate, gate_stride, n, tokens, 2)) ||
            meet(scales, rows_of(up, up_stride, n, tokens, 2)))
            return UNISVQ_EINVAL;
    }
    return status(unisvq::launch_gated(unisvq::GatedArgs{tokens, static_cast<int>(n), gate, up, y, gate_stride, up_stride,
                                                         y_stride, x_dtype, y_dtype, activation, y_scales},
                                       static_cast<hipStream_t>(stream)));
}

size_t unisvq_fourbit_bytes(int64_t N, int64_t K) {
    if (!fourbit_shape_ok(N, K) || K > kMostColumns) return 0;
    return static_cast<size_t>(unisvq::fourbit_bytes(N, K));
}

int unisvq_fourbit_pack(int64_t N, int64_t K, const uint8_t* codes, const uint16_t* scales, void* packed,
                   int32_t* bad_codes, void* stream) {
    if (!codes || !scales || !packed) return UNISVQ_EINVAL;
    if (!fourbit_shape_ok(N, K)) return UNISVQ_ESHAPE;
    if (!aligned(packed, 16) || !aligned(scales, 2) || !aligned(bad_codes, 4)) return UNISVQ_EALIGN;
    if (K > kMostColumns) return UNISVQ_EUNSUP;
    const int64_t size = unisvq::fourbit_bytes(N, K);
    if (bytes_meet(packed, size, codes, N * K) || bytes_meet(packed, size, scales, N * (K / unisvq::kGroup) * 2) ||
        bytes_meet(packed, size, bad_codes, 4) || bytes_meet(bad_codes, 4, codes, N * K) ||
        bytes_meet(bad_codes, 4, scales, N * (K / unisvq::kGroup) * 2))
        return UNISVQ_EINVAL;
    return status(unisvq::launch_fourbit_pack(N, K, codes, scales, static_cast<uint8_t*>(packed), bad_codes,
                                         static_cast<hipStream_t>(stream)));
}

int unisvq_fourbit_unpack(int64_t N, int64_t K, const void* packed, uint8_t* codes, uint16_t* scales, void* stream) {
    if (!codes || !scales || !packed) return UNISVQ_EINVAL;
    if (!fourbit_shape_ok(N, K)) return UNISVQ_ESHAPE;
    if (!aligned(packed, 16) || !aligned(scales, 2)) return UNISVQ_EALIGN;
    if (K > kMostColumns) return UNISVQ_EUNSUP;
    const int64_t size = unisvq::fourbit_bytes(N, K), scale_bytes = N * (K / unisvq::kGroup) * 2;
    if (bytes_meet(packed, size, codes, N * K) || bytes_meet(packed, size, scales, scale_bytes) ||
        bytes_meet(codes, N * K, scales, scale_bytes))
        return UNISVQ_EINVAL;
    return status(unisvq::launch_fourbit_unpack(N, K, static_cast<const uint8_t*>(packed), codes, scales,
                                           static_cast<hipStream_t>(stream)));
}

int unisvq_fourbit_quantize(int64_t N, int64_t K, const void* W, int w_dtype, void* packed, void* stream) {
    if (!W || !packed || (!half_type(w_dtype) && w_dtype != UNISVQ_F32)) return UNISVQ_EINVAL;
    if (!fourbit_shape_ok(N, K)) return UNISVQ_ESHAPE;
    if (!aligned(packed, 16) || !aligned(W, 16)) return UNISVQ_EALIGN;
    if (K > kMostColumns) return UNISVQ_EUNSUP;
    if (bytes_meet(packed, unisvq::fourbit_bytes(N, K), W, N * K * (w_dtype == UNISVQ_F32 ? 4 : 2))) return UNISVQ_EINVAL;
    return status(unisvq::launch_fourbit_quantize(N, K, W, w_dtype, static_cast<uint8_t*>(packed),
                                             static_cast<hipStream_t>(stream)));
}

size_t unisvq_fourbit_gemm_batched_workspace_bytes(const unisvq_fourbit_problem* problems, int count, int64_t M, int x_dtype) {
    if (!problems || count < 1 || count > UNISVQ_MAX_BATCH || M < 1 || M > kMost) return 0;
    if (!half_type(x_dtype) && x_dtype != UNISVQ_I8) return 0;
    for (int i = 0; i < count; ++i)
        if (!fourbit_shape_ok(problems[i].N, problems[i].K) || problems[i].K > kMostColumns) return 0;
    FourbitProblem p[UNISVQ_MAX_BATCH];
    fourbit_batch(problems, count, p);
    return unisvq::fourbit_workspace_bytes(p, count, M, x_dtype);
}

int unisvq_fourbit_gemm_batched(const unisvq_fourbit_problem* problems, int count, int64_t M, int x_dtype, int y_dtype,
                           void* workspace, size_t workspace_bytes, void* stream) {
    if (!problems || count < 1 || count > UNISVQ_MAX_BATCH) return UNISVQ_EINVAL;
    for (int i = 0; i < count; ++i) {
        const int st = check_fourbit(problems[i], M, x_dtype, y_dtype);
        if (st != UNISVQ_OK) return st;
    }
    FourbitProblem p[UNISVQ_MAX_BATCH];
    fourbit_batch(problems, count, p);
    return unisvq::launch_fourbit_batch(p, count, M, x_dtype, y_dtype, workspace, workspace_bytes,
                                        static_cast<hipStream_t>(stream));
}

size_t unisvq_fourbit_gemm_workspace_bytes(int64_t N, int64_t K, int64_t M, int x_dtype) {
    const unisvq_fourbit_problem p{N, K, nullptr, nullptr, nullptr, nullptr};
    return unisvq_fourbit_gemm_batched_workspace_bytes(&p, 1, M, x_dtype);
}

int unisvq_fourbit_gemm(int64_t N, int64_t K, const void* packed, int64_t M, const void* x, int x_dtype,
                   const float* x_scales, void* y, int y_dtype, void* workspace, size_t workspace_bytes, void* stream) {
    const unisvq_fourbit_problem p{N, K, packed, x, x_scales, y};
    return unisvq_fourbit_gemm_batched(&p, 1, M, x_dtype, y_dtype, workspace, workspace_bytes, stream);
}

}  // extern "C"
