// Quantisation to e4m3 with a power-of-two scale for each block of 128 values, and the gradient of the gated activation.
// All of it is bound by memory: every source value is read once, its 8 bits written once.
//
// A power of two as the scale: x / scale and scale_a * scale_b are exact, so the only rounding is the one to 8 bits, and a
// floating format loses nothing by a scale that is up to twice what it need be, but for values 2^-14 of the block's largest.
#include "experts.h"
#include "launch.h"

namespace xp8 {
namespace {

// Bits of the largest magnitude (of a float, finite) -> scale.  amax = m 2^E, 1 <= m < 2, and 448 = 1.75 * 2^8: the least power of two that
// reaches amax / 448 is 2^(E-8) up to m = 1.75, else 2^(E-7).
__device__ __forceinline__ float power_scale(unsigned bits)
{
    int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    e = e < -126 ? -126 : e;
    if (bits == 0) e = 0;
    return __builtin_bit_cast(float, (127 + e) << 23);
}
constexpr unsigned INF_BITS = 0x7f800000;

// (reciprocal of the hardware's: a step of the last place, which the rounding to 8 bits swallows)
__device__ __forceinline__ float silu_gate(float g, float u) { return g * __builtin_amdgcn_rcpf(1.f + expf(-g)) * u; }

typedef unsigned short v2us __attribute__((ext_vector_type(2)));
typedef short v2s __attribute__((ext_vector_type(2)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// Two of four e4m3 values of a word from two numbers / scale (a power of two), rounded to nearest even: one instruction on the numbers as they lie in
// memory.  Exact for quotients up to 448 (all 65536 patterns of each type at scales from 2^-126 to 2^120); beyond, and for NaN, NaN.
template <typename T>
__device__ __forceinline__ unsigned two_e4m3(unsigned old, unsigned pair, float scale, bool upper)
{
    const v2s o = __builtin_bit_cast(v2s, old);
    v2s q;
    if constexpr (std::is_same<T, __bf16>::value)
        q = upper ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(v2b, pair), scale, true)
                  : __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(o, __builtin_bit_cast(v2b, pair), scale, false);
    else
        q = upper ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(o, __builtin_bit_cast(v2h, pair), scale, true)
                  : __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(o, __builtin_bit_cast(v2h, pair), scale, false);
    return __builtin_bit_cast(unsigned, q);
}
__device__ __forceinline__ unsigned two_e4m3(unsigned old, float a, float b, float scale, bool upper)
{
    const v2s o = __builtin_bit_cast(v2s, old);
    return __builtin_bit_cast(unsigned, upper ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, a, b, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(o, a, b, scale, false));
}

// Eight neighbouring values of a row: 16-bit types stay as they are, two to a word; 32-bit ones and gated activations are floats.
template <typename T, bool GATE>
struct Eight {
    static constexpr bool PAIRS = sizeof(T) == 2 && !GATE;
    static constexpr int WORDS = PAIRS ? 4 : 8;
    unsigned w[WORDS];

    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    // from column c of a source row on, zeros past the end.  VEC: rows begin on 16 bytes and are whole pieces of eight
    template <bool VEC>
    __device__ __forceinline__ void load(const T *row, int c, int cols)
    {
        zero();
        if (row == nullptr || c >= cols) return;
        Vec<T, 8> v = {}, u = {};
        if constexpr (VEC) {
            constexpr int PIECES = sizeof(T) * 8 / 16;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                reinterpret_cast<v4u *>(&v)[i] = reinterpret_cast<const v4u *>(row + c)[i];
                if constexpr (GATE) reinterpret_cast<v4u *>(&u)[i] = reinterpret_cast<const v4u *>(row + cols + c)[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < cols) {
                    v.v[i] = row[c + i];
                    if constexpr (GATE) u.v[i] = row[cols + c + i];
                }
        }
        if constexpr (PAIRS) {
            const v4u x = *reinterpret_cast<const v4u *>(&v);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = x[i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = to_float(v.v[i]);
                w[i] = __builtin_bit_cast(unsigned, GATE ? silu_gate(x, to_float(u.v[i])) : x);
            }
        }
    }
    // magnitudes in an order of their own (16 bits each, or 32): the largest of two, as float bits, and without those that are not finite
    static __device__ __forceinline__ unsigned magnitude(unsigned x) { return PAIRS ? x & 0x7fff7fffu : x & 0x7fffffffu; }
    static __device__ __forceinline__ unsigned larger(unsigned a, unsigned b)
    {
        if constexpr (PAIRS) return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(v2us, a), __builtin_bit_cast(v2us, b)));
        else return a > b ? a : b;
    }
    static __device__ __forceinline__ unsigned finite(unsigned m)   // magnitudes -> 0 where not finite
    {
        if constexpr (PAIRS) {
            constexpr unsigned LIMIT = std::is_same<T, __bf16>::value ? 0x7f80 : 0x7c00;
            return ((m & 0xffff) < LIMIT ? m & 0xffff : 0) | ((m >> 16) < LIMIT ? m & 0xffff0000u : 0);
        } else {
            return m < INF_BITS ? m : 0;
        }
    }
    static __device__ __forceinline__ unsigned float_bits(unsigned m16)   // of one magnitude
    {
        if constexpr (!PAIRS) return m16;
        else if constexpr (std::is_same<T, __bf16>::value) return m16 << 16;
        else return __builtin_bit_cast(unsigned, (float)__builtin_bit_cast(_Float16, (unsigned short)m16));
    }
    static __device__ __forceinline__ unsigned top_of_word(unsigned m)   // the larger of a word's magnitudes, as float bits
    {
        if constexpr (PAIRS) return float_bits(max(m & 0xffff, m >> 16));
        else return m;
    }
    __device__ __forceinline__ unsigned top(bool only_finite) const
    {
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const unsigned x = magnitude(w[i]);
            m = larger(m, only_finite ? finite(x) : x);
        }
        return top_of_word(m);
    }
    // value i as a float's bits
    __device__ __forceinline__ unsigned value(int i) const
    {
        if constexpr (!PAIRS) return w[i];
        else {
            const unsigned h = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffff;
            if constexpr (std::is_same<T, __bf16>::value) return h << 16;
            else return __builtin_bit_cast(unsigned, (float)__builtin_bit_cast(_Float16, (unsigned short)h));
        }
    }
    __device__ __forceinline__ v2u quantized(float scale) const
    {
        v2u q = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (PAIRS) q[i >> 1] = two_e4m3<T>(q[i >> 1], w[i], scale, i & 1);
            else q[i >> 1] = two_e4m3(q[i >> 1], __builtin_bit_cast(float, w[2 * i]), __builtin_bit_cast(float, w[2 * i + 1]), scale, i & 1);
        }
        return q;
    }
};

// Infinities are +-448: in byte i of the eight (rare: only where a block has one).
__device__ __forceinline__ void mend_infinity(v2u &q, int i, unsigned bits)
{
    if ((bits & 0x7fffffffu) == INF_BITS) q[i >> 2] = (q[i >> 2] & ~(0xffu << (8 * (i & 3)))) | (0x7eu | (bits >> 31) << 7) << (8 * (i & 3));
}

template <int N>
__device__ __forceinline__ unsigned rotated_max(unsigned v) { return (unsigned)row_max<N>((int)v); }   // (magnitudes: never negative)
__device__ __forceinline__ unsigned top16(unsigned v) { return rotated_max<1>(rotated_max<2>(rotated_max<4>(rotated_max<8>(v)))); }

// A row's eight values within its block of 128, which 16 neighbouring lanes hold: quantised, and the block's scale.
template <typename T, bool GATE>
__device__ __forceinline__ v2u quantize_row(const Eight<T, GATE> &x, float *scale)
{
    unsigned top = top16(x.top(false));
    if (__any(top >= INF_BITS)) {
        top = top16(x.top(true));
        *scale = power_scale(top);
        v2u q = x.quantized(*scale);
#pragma unroll
        for (int i = 0; i < 8; ++i) mend_infinity(q, i, x.value(i));
        return q;
    }
    *scale = power_scale(top);
    return x.quantized(*scale);
}

// Source row of row r, null where it has none.
template <typename T>
__device__ __forceinline__ const T *source_row(const QuantizeProblem &p, int r)
{
    const T *src = static_cast<const T *>(p.src);
    if (r >= p.rows) return nullptr;
    if (!p.take) return src + (long long)r * p.lds;
    const int at = p.take[r];
    if (at < 0 || at / p.per_row >= p.src_rows) return nullptr;
    return src + (long long)(at / p.per_row) * p.lds;
}

__device__ __forceinline__ void store8(uint8_t *row, int c, int cols, bool whole, v2u q)
{
    if (whole && c + 8 <= cols) {
        *reinterpret_cast<v2u *>(row + c) = q;
    } else {
        const unsigned long long w = q[0] | (unsigned long long)q[1] << 32;
        for (int i = 0; i < 8 && c + i < cols; ++i) row[c + i] = (uint8_t)(w >> (8 * i));
    }
}
__device__ __forceinline__ bool rows_begin_on(const void *base, long long ld, int bytes)
{
    return ((reinterpret_cast<uintptr_t>(base) | (uintptr_t)ld) & (bytes - 1)) == 0;
}

// Rows: 16 lanes hold a block of 128 (eight values each), a wave four neighbouring blocks of EACH rows, a workgroup 4 * EACH rows x 512 columns:
// its scales leave for 4 * EACH rows at a time, since they lie [block][row].
constexpr int ROWS_COLS = 512;

// Bound by memory: 8192 x 4096 bfloat16 in 22.7 us (101 MB, 4.4 TB/s), gated 41 (168 MB, 4.1 TB/s); 517 x 2056 gated, one round of loads, 3.8 us.
template <typename T, bool VEC, bool GATE, int EACH>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeProblem p)
{
    constexpr int ROWS = 4 * EACH;
    __shared__ float scale_of[4][ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int across = (p.cols + ROWS_COLS - 1) / ROWS_COLS, bx = (int)(blockIdx.x % across), by = (int)(blockIdx.x / across);
    const int r0 = by * ROWS, c = bx * ROWS_COLS + lane * 8;
    const bool whole = rows_begin_on(p.q, p.ldq, 8);
    Eight<T, GATE> x[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) x[i].template load<VEC>(source_row<T>(p, r0 + wave * EACH + i), c, p.cols);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        float scale;
        const v2u q = quantize_row(x[i], &scale);
        const int r = r0 + wave * EACH + i;
        if ((lane & 15) == 0) scale_of[lane >> 4][wave * EACH + i] = scale;
        if (r < p.rows && c < p.cols) store8(p.q + (long long)r * p.ldq, c, p.cols, whole, q);
    }
    __syncthreads();
    if (threadIdx.x < 4 * ROWS) {
        const int b = bx * 4 + threadIdx.x / ROWS, r = r0 + threadIdx.x % ROWS;
        if (b < blocks_of(p.cols) && r < p.rows) p.scales[(long long)b * p.rows + r] = scale_of[threadIdx.x / ROWS][threadIdx.x % ROWS];
    }
}

// Tiles: a workgroup of four waves on 128 x 128 values, lane (r, c) of 16 x 16 holding rows 8r ... 8r + 7 and columns 8c ... 8c + 7,
// so that eight rows of one column are eight neighbouring bytes of the transposed result.  Those go through LDS, in pieces of
// eight bytes, piece r of column 8c + j in place r ^ c: lanes of one r write to all places, and the lanes that read 16 bytes
// of eight columns do as well.
// COLUMNS: a scale for 128 rows of a column (stored transposed), with p.q the rows' too; else one for the tile.
// Bound by memory: 8192 x 4096 bfloat16, rows and columns, in 28.4 us (136 MB, 4.8 TB/s), a scale for each tile 17.2.
template <typename T, bool VEC, bool GATE, bool COLUMNS>
__global__ __launch_bounds__(256) void quantize_tile_kernel(QuantizeProblem p)
{
    using E = Eight<T, GATE>;
    __shared__ alignas(16) unsigned char turned[128 * 128];
    __shared__ unsigned top_of[4][128];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tc = threadIdx.x & 15, tr = threadIdx.x >> 4;
    const int cb = blocks_of(p.cols), rb = blocks_of(p.rows);
    const int bx = (int)(blockIdx.x % cb), by = (int)(blockIdx.x / cb % rb), bz = (int)(blockIdx.x / cb / rb);
    const int r0 = by * 128 + tr * 8, c0 = bx * 128 + tc * 8;
    E x[8];
    const T *base = static_cast<const T *>(p.src);
    if constexpr (!COLUMNS) base += (long long)bz * p.rows * p.lds;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = r0 + i;
        const T *row;
        if constexpr (COLUMNS) row = source_row<T>(p, r);
        else row = r < p.rows ? base + (long long)r * p.lds : nullptr;
        x[i].template load<VEC>(row, c0, p.cols);
    }
    float scale[8];   // of the columns, or of the tile (scale[0])
    bool mend = false;
    // magnitudes of the columns (words of one or two), or of the tile, over the workgroup
    auto tops = [&](bool only_finite) {
        unsigned m[E::WORDS];
#pragma unroll
        for (int k = 0; k < E::WORDS; ++k) {
            m[k] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const unsigned v = E::magnitude(x[i].w[k]);
                m[k] = E::larger(m[k], only_finite ? E::finite(v) : v);
            }
        }
        if constexpr (COLUMNS) {
#pragma unroll
            for (int k = 0; k < E::WORDS; ++k) {
                m[k] = E::larger(m[k], (unsigned)__shfl_xor((int)m[k], 16));
                m[k] = E::larger(m[k], (unsigned)__shfl_xor((int)m[k], 32));
                if (lane < 16) top_of[wave][tc * E::WORDS + k] = m[k];
            }
        } else {
            unsigned all = m[0];
#pragma unroll
            for (int k = 1; k < E::WORDS; ++k) all = E::larger(all, m[k]);
            const int top = max64((int)E::top_of_word(all));
            if (lane == 0) top_of[0][wave] = (unsigned)top;
        }
        __syncthreads();
        unsigned worst = 0;
        if constexpr (COLUMNS) {
#pragma unroll
            for (int k = 0; k < E::WORDS; ++k) {
                const int at = tc * E::WORDS + k;
                const unsigned top = E::larger(E::larger(top_of[0][at], top_of[1][at]), E::larger(top_of[2][at], top_of[3][at]));
                constexpr int PER = 8 / E::WORDS;
#pragma unroll
                for (int h = 0; h < PER; ++h) {
                    const unsigned bits = E::float_bits(PER == 1 ? top : h ? top >> 16 : top & 0xffff);
                    scale[k * PER + h] = power_scale(bits);
                    worst = max(worst, bits);
                }
            }
        } else {
            worst = max(max(top_of[0][0], top_of[0][1]), max(top_of[0][2], top_of[0][3]));
            scale[0] = power_scale(worst);
        }
        return worst >= INF_BITS;
    };
    if (__syncthreads_or(tops(false))) {   // (the same for the whole workgroup)
        mend = true;
        tops(true);
    }
    if constexpr (COLUMNS) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (tr == 0 && c0 + j < p.cols) p.scales_t[(long long)by * p.cols + c0 + j] = scale[j];
        if (p.q) {   // the rows' own, from the same values
            const bool whole = rows_begin_on(p.q, p.ldq, 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float s;
                const v2u q = quantize_row(x[i], &s);
                if (r0 + i < p.rows) {
                    if (tc == 0) p.scales[(long long)bx * p.rows + r0 + i] = s;
                    if (c0 < p.cols) store8(p.q + (long long)(r0 + i) * p.ldq, c0, p.cols, whole, q);
                }
            }
        }
    } else {
#pragma unroll
        for (int j = 1; j < 8; ++j) scale[j] = scale[0];
        if (threadIdx.x == 0) p.scales[(long long)bz * rb * cb + (p.transpose ? bx * rb + by : by * cb + bx)] = scale[0];
        if (!p.transpose) {
            uint8_t *q = p.q + (long long)bz * p.rows * p.ldq;
            const bool whole = rows_begin_on(q, p.ldq, 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v2u w = x[i].quantized(scale[0]);
                if (mend)
#pragma unroll
                    for (int j = 0; j < 8; ++j) mend_infinity(w, j, x[i].value(j));
                if (r0 + i < p.rows && c0 < p.cols) store8(q + (long long)(r0 + i) * p.ldq, c0, p.cols, whole, w);
            }
            return;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {   // eight rows of column j
        v2u w = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            if constexpr (E::PAIRS) {
                const unsigned pair = __builtin_amdgcn_perm(x[i + 1].w[j >> 1], x[i].w[j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
                w[i >> 2] = two_e4m3<T>(w[i >> 2], pair, scale[j], i >> 1 & 1);
            } else {
                w[i >> 2] = two_e4m3(w[i >> 2], __builtin_bit_cast(float, x[i].w[j]), __builtin_bit_cast(float, x[i + 1].w[j]), scale[j], i >> 1 & 1);
            }
        }
        if (mend)
#pragma unroll
            for (int i = 0; i < 8; ++i) mend_infinity(w, i, x[i].value(j));
        *reinterpret_cast<v2u *>(turned + (tc * 8 + j) * 128 + ((tr ^ tc) * 8)) = w;
    }
    __syncthreads();
    uint8_t *qt = COLUMNS ? p.qt : p.q + (long long)bz * p.cols * p.ldq;
    const long long ld = COLUMNS ? p.ldqt : p.ldq;
    const bool whole = rows_begin_on(qt, ld, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = i * 32 + (threadIdx.x >> 3), piece = threadIdx.x & 7;   // 16 bytes: rows 16 piece ... of column c
        const int turn = c >> 3;
        const v2u lo = *reinterpret_cast<const v2u *>(turned + c * 128 + ((2 * piece) ^ turn) * 8);
        const v2u hi = *reinterpret_cast<const v2u *>(turned + c * 128 + ((2 * piece + 1) ^ turn) * 8);
        const int col = bx * 128 + c, r = by * 128 + piece * 16;
        if (col >= p.cols || r >= p.rows) continue;
        uint8_t *to = qt + (long long)col * ld + r;
        if (whole && r + 16 <= p.rows) {
            *reinterpret_cast<v4u *>(to) = v4u{lo.x, lo.y, hi.x, hi.y};
        } else {
            const unsigned w[4] = {lo.x, lo.y, hi.x, hi.y};
            for (int b = 0; b < 16 && r + b < p.rows; ++b) to[b] = (uint8_t)(w[b >> 2] >> (8 * (b & 3)));
        }
    }
}

// d silu(g) u: dg = dh u s (1 + g (1 - s)), du = dh g s, with s = 1 / (1 + exp(-g)).  A thread on 16 bytes of each of the five; bound by memory:
// 8192 x 4096 bfloat16 (335 MB) in 52 us, 6.4 TB/s with what the last level cache still holds.
template <typename T>
__global__ __launch_bounds__(256) void gate_backward_kernel(GateProblem p, int pieces, int vec)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    const int r = (int)(at / pieces), c = (int)(at % pieces) * 8;
    if (r >= p.rows) return;
    const T *x = static_cast<const T *>(p.x) + r * p.ldx, *dh = static_cast<const T *>(p.dh) + r * p.ldh;
    T *dx = static_cast<T *>(p.dx) + r * p.lddx;
    Eight<T, false> gv, uv, dv;
    if (vec) {
        gv.template load<true>(x, c, p.cols);
        uv.template load<true>(x + p.cols, c, p.cols);
        dv.template load<true>(dh, c, p.cols);
    } else {
        gv.template load<false>(x, c, p.cols);
        uv.template load<false>(x + p.cols, c, p.cols);
        dv.template load<false>(dh, c, p.cols);
    }
    Vec<T, 8> dg, du;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float g = __builtin_bit_cast(float, gv.value(i)), u = __builtin_bit_cast(float, uv.value(i)), d = __builtin_bit_cast(float, dv.value(i));
        const float s = __builtin_amdgcn_rcpf(1.f + expf(-g));
        dg.v[i] = (T)(d * u * s * (1.f + g * (1.f - s)));
        du.v[i] = (T)(d * g * s);
    }
    if (vec) {
        constexpr int PIECES = sizeof(T) * 8 / 16;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            reinterpret_cast<v4u *>(dx + c)[i] = reinterpret_cast<const v4u *>(&dg)[i];
            reinterpret_cast<v4u *>(dx + p.cols + c)[i] = reinterpret_cast<const v4u *>(&du)[i];
        }
    } else {
        for (int i = 0; i < 8 && c + i < p.cols; ++i) {
            dx[c + i] = dg.v[i];
            dx[p.cols + c + i] = du.v[i];
        }
    }
}

// Whether every row begins on 16 bytes and is whole pieces of eight values.
bool in_pieces(const void *base, long long ld, int cols, int size)
{
    return (reinterpret_cast<uintptr_t>(base) & 15) == 0 && (ld * size) % 16 == 0 && cols % 8 == 0 && (cols * (long long)size) % 16 == 0;
}

template <typename F>
hipError_t for_source(const QuantizeProblem &p, F &&f)
{
    const bool vec = in_pieces(p.src, p.lds, p.cols, size_of(p.type));
    return with_type(p.type, [&](auto t) {
        if (vec) return p.gate ? f(t, std::true_type{}, std::true_type{}) : f(t, std::true_type{}, std::false_type{});
        return p.gate ? f(t, std::false_type{}, std::true_type{}) : f(t, std::false_type{}, std::false_type{});
    });
}

}  // namespace

hipError_t launch_quantize_rows(const QuantizeProblem &p, hipStream_t st)
{
    const long long across = (p.cols + ROWS_COLS - 1) / ROWS_COLS;
    const long long large = across * ((p.rows + 15) / 16);
    if (!fits_launch(large, 256)) return TOO_LARGE;
    return for_source(p, [&](auto t, auto vec, auto gate) {
        using T = decltype(t);
        // four rows a wave hide the loads' time; until there are four workgroups for every compute unit one row, so that there are more of them
        if (large >= 1024)
            return c2i8::launch(quantize_rows_kernel<T, vec.value, gate.value, 4>, dim3((unsigned)large), dim3(256), 0, st, p);
        return c2i8::launch(quantize_rows_kernel<T, vec.value, gate.value, 1>, dim3((unsigned)(across * ((p.rows + 3) / 4))), dim3(256), 0, st, p);
    });
}

hipError_t launch_quantize_columns(const QuantizeProblem &p, hipStream_t st)
{
    const long long tiles = (long long)blocks_of(p.cols) * blocks_of(p.rows);
    if (!fits_launch(tiles, 256)) return TOO_LARGE;
    const dim3 grid((unsigned)tiles);
    return for_source(p, [&](auto t, auto vec, auto gate) {
        return c2i8::launch(quantize_tile_kernel<decltype(t), vec.value, gate.value, true>, grid, dim3(256), 0, st, p);
    });
}

hipError_t launch_quantize_tiles(const QuantizeProblem &p, hipStream_t st)
{
    const long long tiles = (long long)blocks_of(p.cols) * blocks_of(p.rows);
    if (!fits_launch(tiles, 256) || !fits_launch(tiles * p.count, 256)) return TOO_LARGE;
    const dim3 grid((unsigned)(tiles * p.count));
    const bool vec = in_pieces(p.src, p.lds, p.cols, size_of(p.type));
    return with_type(p.type, [&](auto t) {
        using T = decltype(t);
        return vec ? c2i8::launch(quantize_tile_kernel<T, true, false, false>, grid, dim3(256), 0, st, p)
                   : c2i8::launch(quantize_tile_kernel<T, false, false, false>, grid, dim3(256), 0, st, p);
    });
}

hipError_t launch_gate_backward(const GateProblem &p, hipStream_t st)
{
    const int size = size_of(p.type), pieces = (p.cols + 7) / 8;
    const int vec = in_pieces(p.x, p.ldx, p.cols, size) && in_pieces(p.dh, p.ldh, p.cols, size) && in_pieces(p.dx, p.lddx, p.cols, size);
    const long long blocks = ((long long)p.rows * pieces + 255) / 256;
    return with_type(p.type, [&](auto t) { return c2i8::launch(gate_backward_kernel<decltype(t)>, dim3((unsigned)blocks), dim3(256), 0, st, p, pieces, vec); });
}

}  // namespace xp8
