// What the experts' kernels share: element types, lane reductions, and the launches that experts_api.cpp makes.
#pragma once
#include "../../include/experts_fp8.h"

#include <hip/hip_runtime.h>

#include <type_traits>

namespace xp8 {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));

constexpr int BLOCK = EXPERTS_BLOCK;
__host__ __device__ inline int blocks_of(int n) { return (n + BLOCK - 1) / BLOCK; }

// f(T{}) for the element type that `type` names
template <typename F>
auto with_type(int type, F &&f)
{
    return type == EXPERTS_F32 ? f(float{}) : type == EXPERTS_BF16 ? f(__bf16{}) : f(_Float16{});
}
inline int size_of(int type) { return type == EXPERTS_F32 ? 4 : 2; }

#if defined(__HIPCC__)
// Maximum or sum over 16 neighbouring lanes (rotations within a DPP row: every lane has the result), or over the wave.
template <int N>
__device__ __forceinline__ float row_rotate(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, true));
}
__device__ __forceinline__ float max16(float v)
{
    v = fmaxf(v, row_rotate<8>(v));
    v = fmaxf(v, row_rotate<4>(v));
    v = fmaxf(v, row_rotate<2>(v));
    return fmaxf(v, row_rotate<1>(v));
}
__device__ __forceinline__ float sum16(float v)
{
    v += row_rotate<8>(v);
    v += row_rotate<4>(v);
    v += row_rotate<2>(v);
    return v + row_rotate<1>(v);
}
__device__ __forceinline__ float lane_of(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }
__device__ __forceinline__ float max64(float v)
{
    v = max16(v);
    return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
__device__ __forceinline__ float sum64(float v)
{
    v = sum16(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
// Whole numbers in the order of the floats that they are made of (no NaN), which need no canonical form before a maximum.
__device__ __forceinline__ int order_key(float v)
{
    const int b = __builtin_bit_cast(int, v);
    return b ^ (b >> 31 & 0x7fffffff);
}
template <int N>
__device__ __forceinline__ int row_max(int v)
{
    return max(v, __builtin_amdgcn_update_dpp(0, v, 0x120 + N, 0xf, 0xf, true));
}
__device__ __forceinline__ int max64(int v)   // uniform
{
    v = row_max<1>(row_max<2>(row_max<4>(row_max<8>(v))));
    return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)), max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

// Running sum over a wave's lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, true); }
__device__ __forceinline__ int running_sum(int v)
{
    v = dpp_add<0x111, 0xf>(v);   // one, two, four, eight lanes up within a row of 16
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);   // a row's last lane to the next row, then of the first half to the second
    return dpp_add<0x143, 0xc>(v);
}

template <typename T>
__device__ __forceinline__ float to_float(T v)
{
    return (float)v;
}

// N elements of T as the 16-byte pieces that hold them
template <typename T, int N>
struct Vec {
    static constexpr int BYTES = (int)sizeof(T) * N;
    alignas(BYTES < 16 ? BYTES : 16) T v[N];
};
#endif

// ---- launches ---------------------------------------------------------------------------------------------------------
// A launch holds fewer than 2^32 lanes; what a problem that asks for more returns (CONV_ERR_UNSUPPORTED to the caller).
constexpr hipError_t TOO_LARGE = hipErrorNotSupported;
inline bool fits_launch(long long workgroups, int threads) { return workgroups <= 0xffffffffll / threads; }

struct QuantizeProblem {
    const void *src;
    long long lds;
    int type, rows, cols, gate;
    const int32_t *take;
    int per_row, src_rows;
    uint8_t *q, *qt;
    long long ldq, ldqt;
    float *scales, *scales_t;
    int count, transpose;   // tiles: matrices, and whether stored transposed
};
hipError_t launch_quantize_rows(const QuantizeProblem &p, hipStream_t st);
hipError_t launch_quantize_columns(const QuantizeProblem &p, hipStream_t st);
hipError_t launch_quantize_tiles(const QuantizeProblem &p, hipStream_t st);

struct GateProblem {
    int rows, cols;
    const void *x, *dh;
    void *dx;
    long long ldx, ldh, lddx;
    int type;
};
hipError_t launch_gate_backward(const GateProblem &p, hipStream_t st);

enum GemmKind : int { GEMM_DENSE = 0, GEMM_EXPERTS = 1, GEMM_GRAD = 2 };
struct Fp8Problem {
    const uint8_t *a, *b;
    long long lda, ldb, ldc;
    const float *sa, *sb;
    void *c;
    int M, N, K;              // EXPERTS: M rows in all; GRAD: M x N results of an expert, K the depth of all experts
    int a_rows;               // rows that A and sa have
    int b_rows, out_type;
    int E;
    const int32_t *offsets, *rows;
    int per_row;
    int fast_sums;            // blocks summed by the 8-bit matrix instruction
};
hipError_t launch_fp8_gemm(const Fp8Problem &p, GemmKind kind, hipStream_t st);

struct RouteProblem {
    int T, E, k;
    const void *logits;
    long long ldl;
    int type;
    const float *bias;
    int sigmoid, groups, kept, group_top, renormalise;
    float factor;
    int32_t *ids;
    float *weights;
    const int32_t *given;      // backward: ids
    const float *dweights;
    void *dlogits;
    long long lddl;
};
hipError_t launch_route(const RouteProblem &p, hipStream_t st);
hipError_t launch_route_backward(const RouteProblem &p, hipStream_t st);

struct OrderProblem {
    int pairs, E, align, R;
    const int32_t *ids;
    int32_t *offsets, *rows, *place;
};
hipError_t launch_expert_rows(const OrderProblem &p, hipStream_t st);

struct CombineProblem {
    int T, k, N, R, type;
    const void *y, *dout;
    void *out, *dy;
    long long ldy, ldd, ldo, lddy;
    const int32_t *place, *rows;
    const float *weights;
    float *dweights;
};
hipError_t launch_combine(const CombineProblem &p, hipStream_t st);
hipError_t launch_combine_backward(const CombineProblem &p, hipStream_t st);

}  // namespace xp8
