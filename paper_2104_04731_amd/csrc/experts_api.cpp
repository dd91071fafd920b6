// C ABI of include/experts_fp8.h: arguments are validated here, the work is in the kernels.
#include "experts.h"

using namespace xp8;

namespace {

constexpr long long MOST_GRID = 0x7fffff;   // workgroups of 256 lanes, half of what a launch holds

bool is_type(int t) { return t == EXPERTS_F32 || t == EXPERTS_BF16 || t == EXPERTS_F16; }
// The kernels read elements at their own alignment at least.
bool on(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
int done(hipError_t e) { return e == hipSuccess ? CONV_OK : e == TOO_LARGE ? CONV_ERR_UNSUPPORTED : CONV_ERR_DEVICE; }
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

int check_quantize(const QuantizeProblem &p)
{
    if (p.rows < 0 || p.cols < 0 || p.count < 0 || !is_type(p.type)) return CONV_ERR_INVALID_ARG;
    if (p.take && (p.per_row <= 0 || p.src_rows < 0 || !on(p.take, 4))) return CONV_ERR_INVALID_ARG;
    if ((long long)p.cols * (p.gate ? 2 : 1) > p.lds || p.cols > 0x3fffffff) return CONV_ERR_INVALID_ARG;
    const bool empty = p.take && p.src_rows == 0;   // (no row of the list is one then, and the source need not be there)
    if ((!p.src && !empty) || !on(p.src, size_of(p.type))) return CONV_ERR_INVALID_ARG;
    if (p.rows > 0x3fffffff) return CONV_ERR_UNSUPPORTED;
    return CONV_OK;
}

}  // namespace

extern "C" {

int quantize_fp8_rows(int rows, int cols, const void *src, int type, long long lds, int gate, const int32_t *take, int per_row, int src_rows, uint8_t *q,
                      long long ldq, float *scales, void *stream)
{
    QuantizeProblem p{src, lds, type, rows, cols, gate != 0, take, per_row, src_rows, q, nullptr, ldq, 0, scales, nullptr, 1, 0};
    if (rows == 0 || cols == 0) return rows < 0 || cols < 0 || !is_type(type) ? CONV_ERR_INVALID_ARG : CONV_OK;
    if (const int rc = check_quantize(p)) return rc;
    if (!q || !scales || ldq < cols || !on(scales, 4)) return CONV_ERR_INVALID_ARG;
    return done(launch_quantize_rows(p, static_cast<hipStream_t>(stream)));
}

int quantize_fp8_columns(int rows, int cols, const void *src, int type, long long lds, int gate, const int32_t *take, int per_row, int src_rows,
                         uint8_t *qt, long long ldqt, float *scales_t, uint8_t *q, long long ldq, float *scales, void *stream)
{
    QuantizeProblem p{src, lds, type, rows, cols, gate != 0, take, per_row, src_rows, q, qt, ldq, ldqt, scales, scales_t, 1, 0};
    if (rows == 0 || cols == 0) return rows < 0 || cols < 0 || !is_type(type) ? CONV_ERR_INVALID_ARG : CONV_OK;
    if (const int rc = check_quantize(p)) return rc;
    if (!qt || !scales_t || ldqt < rows || !on(scales_t, 4)) return CONV_ERR_INVALID_ARG;
    if (q && (!scales || ldq < cols || !on(scales, 4))) return CONV_ERR_INVALID_ARG;
    return done(launch_quantize_columns(p, static_cast<hipStream_t>(stream)));
}

int quantize_fp8_tiles(int count, int rows, int cols, const void *src, int type, long long lds, int transpose, uint8_t *q, long long ldq, float *scales,
                       void *stream)
{
    QuantizeProblem p{src, lds, type, rows, cols, 0, nullptr, 1, rows, q, nullptr, ldq, 0, scales, nullptr, count, transpose != 0};
    if (rows == 0 || cols == 0 || count == 0) return rows < 0 || cols < 0 || count < 0 || !is_type(type) ? CONV_ERR_INVALID_ARG : CONV_OK;
    if (const int rc = check_quantize(p)) return rc;
    if (!q || !scales || ldq < (transpose ? rows : cols) || !on(scales, 4)) return CONV_ERR_INVALID_ARG;
    return done(launch_quantize_tiles(p, static_cast<hipStream_t>(stream)));
}

int silu_gate_backward(int rows, int cols, const void *x, long long ldx, const void *dh, long long ldh, void *dx, long long lddx, int type, void *stream)
{
    if (rows < 0 || cols < 0 || !is_type(type)) return CONV_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return CONV_OK;
    const int size = size_of(type);
    if (cols > 0x3fffffff || ldx < 2ll * cols || ldh < cols || lddx < 2ll * cols || !x || !dh || !dx || !on(x, size) || !on(dh, size) || !on(dx, size))
        return CONV_ERR_INVALID_ARG;
    if (ceil_div((long long)rows * ceil_div(cols, 8), 256) > MOST_GRID) return CONV_ERR_UNSUPPORTED;
    return done(launch_gate_backward({rows, cols, x, dh, dx, ldx, ldh, lddx, type}, static_cast<hipStream_t>(stream)));
}

int gemm_fp8_nt(int M, int N, int K, const uint8_t *A, long long lda, const float *sa, const uint8_t *B, long long ldb, const float *sb, int b_rows, void *C,
                long long ldc, int out_type, int fast_sums, void *stream)
{
    if (M < 0 || N < 0 || K < 0 || !is_type(out_type)) return CONV_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return CONV_OK;
    if (lda < K || ldb < K || ldc < N || !C || !on(C, size_of(out_type))) return CONV_ERR_INVALID_ARG;
    if (K > 0 && (!A || !sa || !B || !sb || !on(sa, 4) || !on(sb, 4))) return CONV_ERR_INVALID_ARG;
    if (M > 0x3fffffff || N > 0x3fffffff || K > 0x7fffff00) return CONV_ERR_UNSUPPORTED;
    Fp8Problem p{A, B, lda, ldb, ldc, sa, sb, C, M, N, K, M, b_rows != 0, out_type, 1, nullptr, nullptr, 1, fast_sums != 0};
    return done(launch_fp8_gemm(p, GEMM_DENSE, static_cast<hipStream_t>(stream)));
}

int gemm_fp8_experts(int R, int a_rows, int E, int N, int K, const uint8_t *A, long long lda, const float *sa, const uint8_t *W, long long ldw,
                     const float *sw, const int32_t *offsets, const int32_t *rows, int per_row, void *C, long long ldc, int out_type, int fast_sums, void *stream)
{
    if (R < 0 || a_rows < 0 || E <= 0 || E > EXPERTS_MOST || N < 0 || K < 0 || !is_type(out_type) || !offsets) return CONV_ERR_INVALID_ARG;
    if (rows ? per_row <= 0 : a_rows != R) return CONV_ERR_INVALID_ARG;
    if (!on(offsets, 4) || !on(rows, 4)) return CONV_ERR_INVALID_ARG;
    if (R == 0 || N == 0) return CONV_OK;
    if (lda < K || ldw < K || ldc < N || !C || !on(C, size_of(out_type))) return CONV_ERR_INVALID_ARG;
    if (a_rows == 0) K = 0;   // no row of the list is one: zeros, and no operand is read
    if (K > 0 && (!A || !sa || !W || !sw || !on(sa, 4) || !on(sw, 4))) return CONV_ERR_INVALID_ARG;
    if (R > 0x3fffffff || N > 0x3fffffff || a_rows > 0x3fffffff || K > 0x7fffff00) return CONV_ERR_UNSUPPORTED;
    Fp8Problem p{A, W, lda, ldw, ldc, sa, sw, C, R, N, K, a_rows, 0, out_type, E, offsets, rows, rows ? per_row : 1, fast_sums != 0};
    return done(launch_fp8_gemm(p, GEMM_EXPERTS, static_cast<hipStream_t>(stream)));
}

int gemm_fp8_experts_grad(int R, int E, int N, int K, const uint8_t *A, long long lda, const float *sa, const uint8_t *B, long long ldb, const float *sb,
                          const int32_t *offsets, void *C, long long ldc, int out_type, int fast_sums, void *stream)
{
    if (R < 0 || E <= 0 || E > EXPERTS_MOST || N < 0 || K < 0 || !is_type(out_type) || !offsets) return CONV_ERR_INVALID_ARG;
    if (!on(offsets, 4)) return CONV_ERR_INVALID_ARG;
    if (N == 0 || K == 0) return CONV_OK;
    if (lda < R || ldb < R || ldc < K || !C || !on(C, size_of(out_type))) return CONV_ERR_INVALID_ARG;
    if (R > 0 && (!A || !sa || !B || !sb || !on(sa, 4) || !on(sb, 4))) return CONV_ERR_INVALID_ARG;
    if (R > 0x7fffff00 || N > 0x3fffffff || K > 0x3fffffff) return CONV_ERR_UNSUPPORTED;
    Fp8Problem p{A, B, lda, ldb, ldc, sa, sb, C, N, K, R, N, 1, out_type, E, offsets, nullptr, 1, fast_sums != 0};
    return done(launch_fp8_gemm(p, GEMM_GRAD, static_cast<hipStream_t>(stream)));
}

static int check_route(const RouteProblem &p)
{
    if (p.T < 0 || p.E <= 0 || p.E > EXPERTS_MOST || p.k <= 0 || p.k > EXPERTS_MOST_CHOICES || p.k > p.E || !is_type(p.type)) return CONV_ERR_INVALID_ARG;
    if (p.T == 0) return CONV_OK;
    if (p.ldl < p.E || !p.logits || !on(p.logits, size_of(p.type))) return CONV_ERR_INVALID_ARG;
    return CONV_OK;
}

int route_experts(int T, int E, int k, const void *logits, int type, long long ldl, const float *bias, int sigmoid, int groups, int kept, int group_top,
                  int renormalise, float factor, int32_t *ids, float *weights, void *stream)
{
    RouteProblem p{T, E, k, logits, ldl, type, bias, sigmoid != 0, groups, kept, group_top, renormalise != 0, factor, ids, weights, nullptr, nullptr, nullptr, 0};
    if (const int rc = check_route(p)) return rc;
    if (groups <= 0 || groups > 64 || E % groups || kept <= 0 || kept > groups || (group_top != 1 && group_top != 2)) return CONV_ERR_INVALID_ARG;
    if (T == 0) return CONV_OK;
    if (!ids || !weights || !on(ids, 4) || !on(weights, 4) || (bias && !on(bias, 4))) return CONV_ERR_INVALID_ARG;
    if (ceil_div(T, 4) > MOST_GRID) return CONV_ERR_UNSUPPORTED;
    return done(launch_route(p, static_cast<hipStream_t>(stream)));
}

int route_experts_backward(int T, int E, int k, const void *logits, int type, long long ldl, const int32_t *ids, const float *dweights, int sigmoid,
                           int renormalise, float factor, void *dlogits, long long lddl, void *stream)
{
    RouteProblem p{T, E, k, logits, ldl, type, nullptr, sigmoid != 0, 1, 1, 1, renormalise != 0, factor, nullptr, nullptr, ids, dweights, dlogits, lddl};
    if (const int rc = check_route(p)) return rc;
    if (T == 0) return CONV_OK;
    if (!ids || !dweights || !dlogits || lddl < E || !on(ids, 4) || !on(dweights, 4) || !on(dlogits, size_of(type))) return CONV_ERR_INVALID_ARG;
    if (ceil_div(T, 4) > MOST_GRID) return CONV_ERR_UNSUPPORTED;
    return done(launch_route_backward(p, static_cast<hipStream_t>(stream)));
}

int expert_rows_capacity(int pairs, int E, int align)
{
    if (pairs < 0 || E <= 0 || E > EXPERTS_MOST || align <= 0 || align > 1024) return 0;
    const long long rows = ceil_div(pairs + (long long)E * (align - 1), align) * align;
    return rows > 0x3fffffff ? 0 : (int)rows;
}

int expert_rows(int pairs, int E, int align, const int32_t *ids, int32_t *offsets, int32_t *rows, int32_t *place, void *stream)
{
    if (pairs < 0 || E <= 0 || E > EXPERTS_MOST || align <= 0 || align > 1024) return CONV_ERR_INVALID_ARG;
    const int R = expert_rows_capacity(pairs, E, align);
    if (R == 0 && (pairs > 0 || align > 1)) return CONV_ERR_UNSUPPORTED;
    if (!offsets || (pairs > 0 && (!ids || !place)) || (R > 0 && !rows)) return CONV_ERR_INVALID_ARG;
    if (!on(offsets, 4) || !on(ids, 4) || !on(place, 4) || !on(rows, 4)) return CONV_ERR_INVALID_ARG;
    return done(launch_expert_rows({pairs, E, align, R, ids, offsets, rows, place}, static_cast<hipStream_t>(stream)));
}

int combine_experts(int T, int k, int N, int R, const void *y, long long ldy, int type, const int32_t *place, const float *weights, void *out,
                    long long ldo, void *stream)
{
    if (T < 0 || k <= 0 || N < 0 || R < 0 || !is_type(type)) return CONV_ERR_INVALID_ARG;
    if (T == 0 || N == 0) return CONV_OK;
    const int size = size_of(type);
    if (ldo < N || (R > 0 && (!y || ldy < N || !on(y, size))) || !out || !place || !on(out, size) || !on(place, 4) || (weights && !on(weights, 4)))
        return CONV_ERR_INVALID_ARG;
    if ((long long)T * N > 1ll << 40) return CONV_ERR_UNSUPPORTED;
    CombineProblem p{T, k, N, R, type, y, nullptr, out, nullptr, ldy, 0, ldo, 0, place, nullptr, weights, nullptr};
    return done(launch_combine(p, static_cast<hipStream_t>(stream)));
}

int combine_experts_backward(int T, int k, int N, int R, const void *dout, long long ldd, const void *y, long long ldy, int type, const int32_t *place,
                             const int32_t *rows, const float *weights, void *dy, long long lddy, float *dweights, void *stream)
{
    if (T < 0 || k <= 0 || N < 0 || R < 0 || !is_type(type)) return CONV_ERR_INVALID_ARG;
    const long long pairs = (long long)T * k;
    if (pairs > 0x3fffffff) return CONV_ERR_UNSUPPORTED;
    if (pairs == 0 && R == 0) return CONV_OK;
    const int size = size_of(type);
    if (pairs > 0 && (!place || !dweights || !on(place, 4) || !on(dweights, 4) || (N > 0 && (!dout || ldd < N || !on(dout, size))))) return CONV_ERR_INVALID_ARG;
    if (R > 0 && (!rows || !on(rows, 4) || (N > 0 && (!y || !dy || ldy < N || lddy < N || !on(y, size) || !on(dy, size))))) return CONV_ERR_INVALID_ARG;
    if (weights && !on(weights, 4)) return CONV_ERR_INVALID_ARG;
    if (ceil_div(pairs > R ? pairs : R, 4) > MOST_GRID) return CONV_ERR_UNSUPPORTED;
    CombineProblem p{T, k, N, R, type, y, dout, nullptr, dy, ldy, ldd, 0, lddy, place, rows, weights, dweights};
    return done(launch_combine_backward(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
