// Products of block-scaled e4m3 operands, C[m][n] = sum over 128-deep blocks b of sa[b][m] sb (sum over k of A[m][k] B[n][k]): dense, with a
// weight matrix for each expert (ragged groups of rows), and the experts' weight gradients (the depth cut by expert).
//
// A block's sum starts from zero in the matrix units and is scaled and added to 32-bit sums by the vector unit: four fused multiply-adds a
// lane to 16 x 16 results.  B's rows are the instruction's rows and A's its columns: a lane's results then belong to one row m, whose
// scale is one number a lane and a block, and to neighbouring columns n, which leave in 16-byte stores.
// How a block is summed: the 8-bit instruction (v_mfma_f32_16x16x128_f8f6f4) aligns each eight neighbouring products to the largest of them and cuts
// the others towards zero 13 bits below its power of two: beside 256 * 256 a 7.5 is lost and a 15 becomes 8, in the next eight a 0.0625 is kept (measured).  So a
// result is up to 7 * 2^-13 of the sum of its terms' magnitudes off, and always towards zero; sums of 128 normal values 1.5e-5 in the mean.  That is a
// hundredth of what rounding to bfloat16 costs but not a 32-bit sum, so it is the caller's
// choice (FAST); without it the values are widened to bfloat16, exactly, for v_mfma_f32_16x16x32_bf16, whose sums are 32-bit ones (8.5e-9), at half the rate.
// Two kernels: tiles through LDS, bound by the matrix units; and, for few rows of not too large weights, one that streams B from memory into
// registers with the depth shared among the waves of a workgroup, bound by B's bytes or the latency of one round of loads.
#include "experts.h"
#include "launch.h"

namespace xp8 {
namespace {

// ---- where a workgroup works -------------------------------------------------------------------------------------------
struct Place {
    int e;            // expert (0 without)
    int m0, m_end;    // its rows: from m0 on, ending at m_end (the group's end)
    bool zeros;       // no expert's rows: m0 ... are to be zeros
};

// Slots of TM rows each, an expert's rows in as many as they need: what slot number pick(all of them) is, 0 ... all - 1 an expert's, from there on
// one of the rows of no expert (e: how many before it, m0: the first of these rows).  64 experts at a time, one to a lane; offsets are held to
// 0 ... R and to rise.
template <int TM, typename F>
__device__ __forceinline__ Place place_of(const int32_t *offsets, int E, int R, int lane, F &&pick)
{
    int lo = 0, hi = 0, sum = 0, before = 0, end = 0;
    auto look = [&](int e0) {
        const int e = e0 + lane;
        lo = hi = 0;
        if (e < E) {
            lo = min(max(offsets[e], 0), R);
            hi = min(max(offsets[e + 1], lo), R);
        }
        sum = running_sum((hi - lo + TM - 1) / TM);
    };
    for (int e0 = 0; e0 < E; e0 += 64) {
        look(e0);
        end = max(end, max64(hi));
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    const int slot = pick(before);
    if (slot >= before) return {slot - before, end, R, true};
    before = 0;
    for (int e0 = 0;; e0 += 64) {
        if (E > 64) look(e0);
        const unsigned long long who = __ballot(slot < before + sum);
        if (who || e0 + 64 >= E) {
            const int l = __builtin_ctzll(who | 1ull << 63);   // the first lane whose running sum passes the slot
            const int n = (hi - lo + TM - 1) / TM;
            const int first = before + __builtin_amdgcn_readlane(sum - n, l);
            return {e0 + l, __builtin_amdgcn_readlane(lo, l) + (slot - first) * TM, __builtin_amdgcn_readlane(hi, l), false};
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
}

// The rows of no expert, counted: those ahead of the first expert's, then those behind the last one's (of a place that is `zeros`).
struct NoRows {
    int ahead, behind, count;
    __device__ __forceinline__ NoRows(const Fp8Problem &p, const Place &at) : ahead(min(max(p.offsets[0], 0), p.M)), behind(at.m0), count(ahead + at.m_end - at.m0) {}
    __device__ __forceinline__ int operator[](int i) const { return i < ahead ? i : behind + i - ahead; }
};

__device__ __forceinline__ int xcd_contiguous(int id, int n)
{
    const int x = id & 7, q = n >> 3, rem = n & 7;
    return x * q + (x < rem ? x : rem) + (id >> 3);
}

// A's row of row r of the result (EXPERTS: through rows[]), -1 where it has none.
template <GemmKind KIND>
__device__ __forceinline__ int a_row_of(const Fp8Problem &p, int r)
{
    if constexpr (KIND == GEMM_EXPERTS) {
        if (r >= p.M) return -1;
        if (!p.rows) return r;
        const int at = p.rows[r];
        return at < 0 || at / p.per_row >= p.a_rows ? -1 : at / p.per_row;
    } else {
        return r < p.M ? r : -1;
    }
}

// ---- results -----------------------------------------------------------------------------------------------------------
template <int N, typename OUT>
__device__ __forceinline__ void store_run(OUT *row, int n, int N_all, bool whole, const float (&v)[N])
{
    constexpr int W = 16 / sizeof(OUT) < N ? 16 / sizeof(OUT) : N;
#pragma unroll
    for (int i = 0; i < N; i += W) {
        Vec<OUT, W> o;
#pragma unroll
        for (int j = 0; j < W; ++j) o.v[j] = (OUT)v[i + j];
        if (whole && n + i + W <= N_all) *reinterpret_cast<Vec<OUT, W> *>(row + n + i) = o;
        else
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (n + i + j < N_all) row[n + i + j] = o.v[j];
    }
}
// N neighbouring results of a row, from column n on
template <int N>
__device__ __forceinline__ void store_results(const Fp8Problem &p, long long row, int n, const float (&v)[N])
{
    const int size = p.out_type == EXPERTS_F32 ? 4 : 2;
    const bool whole = ((reinterpret_cast<uintptr_t>(p.c) | (uintptr_t)(p.ldc * size)) & (N * size < 16 ? N * size - 1 : 15)) == 0;
    if (p.out_type == EXPERTS_F32) store_run<N>(static_cast<float *>(p.c) + row * p.ldc, n, p.N, whole, v);
    else if (p.out_type == EXPERTS_BF16) store_run<N>(static_cast<__bf16 *>(p.c) + row * p.ldc, n, p.N, whole, v);
    else store_run<N>(static_cast<_Float16 *>(p.c) + row * p.ldc, n, p.N, whole, v);
}

// 16 bytes of a row of n bytes from k on, whatever the row's alignment (one load where global memory is read unaligned, as here),
// zeros outside [lo, hi).
__device__ __forceinline__ v4u load_any(const uint8_t *at)
{
    v4u v;
    __builtin_memcpy(&v, at, 16);
    return v;
}
__device__ __forceinline__ v4u load_masked(const uint8_t *row, int k, int lo, int hi, int n)
{
    if (k >= lo && k + 16 <= hi) return load_any(row + k);
    v4u v = {0, 0, 0, 0};
    if (k + 16 <= lo || k >= hi) return v;
    if (n >= 16) {   // the row's last 16 bytes at most, moved down
        const int from = min(k, n - 16), by = k - from;
        v = load_any(row + from);
        if (by & 8) v = v4u{v[2], v[3], 0, 0};
        if (by & 4) v = v4u{v[1], v[2], v[3], 0};
        if (by & 3)
            v = v4u{__builtin_amdgcn_alignbyte(v[1], v[0], by & 3), __builtin_amdgcn_alignbyte(v[2], v[1], by & 3), __builtin_amdgcn_alignbyte(v[3], v[2], by & 3),
                    __builtin_amdgcn_alignbyte(0, v[3], by & 3)};
    } else {
        unsigned long long low = 0, high = 0;
#pragma unroll 1
        for (int i = k; i < n; ++i) (i - k < 8 ? low : high) |= (unsigned long long)row[i] << (8 * ((i - k) & 7));
        v = v4u{(unsigned)low, (unsigned)(low >> 32), (unsigned)high, (unsigned)(high >> 32)};
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {   // of a dword's bytes, those within [lo, hi)
        const int first = min(max(lo - (k + 4 * w), 0), 4), end = min(max(hi - (k + 4 * w), 0), 4);
        const unsigned below = end < 4 ? (1u << (8 * end)) - 1 : ~0u, above = first < 4 ? ~0u << (8 * first) : 0u;
        v[w] &= below & above;
    }
    return v;
}

// A lane's 32 values of a block, as the matrix instructions take them: the order of the depth is the lane's own, alike in both operands.
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
template <bool FAST>
struct Fragment;
template <>
struct Fragment<true> {
    v8i v;
    __device__ __forceinline__ void set(v8i x) { v = x; }
};
template <>
struct Fragment<false> {
    v8b v[4];
    __device__ __forceinline__ void set(v8i x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v2b h[4];
            h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[2 * i], 1.f, false);
            h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[2 * i], 1.f, true);
            h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[2 * i + 1], 1.f, false);
            h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)x[2 * i + 1], 1.f, true);
            v[i] = v8b{h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
        }
    }
};
__device__ __forceinline__ v4f block_sum(const Fragment<true> &a, const Fragment<true> &b)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, v4f{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ v4f block_sum(const Fragment<false> &a, const Fragment<false> &b)
{
    v4f c = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}

// ---- tiles -------------------------------------------------------------------------------------------------------------
// 16 (4) bytes per lane from base + off to LDS byte address lds + 16 (4) * lane (base and lds wave-uniform); counted by vmcnt, the
// compiler does not see the LDS write.
__device__ __forceinline__ void dma16(const void *base, unsigned off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void dma4(const void *base, unsigned off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory");
}
template <int NEWER>
__device__ __forceinline__ void landed()   // all transfers of this wave but the NEWER last ones
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NEWER) : "memory");
}
__device__ __forceinline__ void barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): this wave's LDS accesses are done
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// TM rows x TN columns of C, WM x WN waves on TM/WM x TN/WN each (PARTS times as many: each on its part of the depth, in its part of LDS).
// Stages of 128 deep, two of them: rows of 128 bytes in eight 16-byte chunks, chunk c of row r at place c ^ turn(r), so that the 16 rows of a fragment
// read take all banks alike.
// A wave's columns are dealt to the matrix instruction's rows, tile t, row i: 32 (t / 2) + 8 (i / 4) + 4 (t % 2) + i % 4, such that a lane ends up
// with eight neighbouring ones in two tiles and the four lanes of a row of C with 32.
template <int TM, int TN, int WM, int WN, GemmKind KIND, bool BROWS>
struct Tile {
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int MT = TM / WM / 16, NT = TN / WN / 16;
    static constexpr int STAGE = (TM + TN) * 128 + (TM + (BROWS ? TN : 0)) * 4;
    static constexpr int LOADS_A = TM / 8 / WAVES, LOADS_B = TN / 8 / WAVES;   // transfers of a wave: eight rows each
    static_assert(LOADS_A * 8 * WAVES == TM && LOADS_B * 8 * WAVES == TN && TM / 64 <= WAVES && TN / 64 <= WAVES && TN / WN <= 128);
    // Transfer j of a wave: which eight rows.  B's first half of the transfers are the rows of the first half of a wave's tiles, which are free
    // sooner.
    static __device__ __forceinline__ int a_rows(int wave, int j) { return (j * WAVES + wave) * 8; }
    static __device__ __forceinline__ int b_rows(int wave, int j)
    {
        const int q = j * WAVES + wave, h = q % (TN / 16);   // (eights of rows: NT to a wave's half)
        return (h / NT * 2 * NT + (q >= TN / 16 ? NT : 0) + h % NT) * 8;
    }
    static __device__ __forceinline__ int turn(int i) { return ((i >> 3 ^ i >> 2) & 1) << 2 | (i >> 1 & 1) << 1 | (i >> 3 & 1); }   // of the fragment's row i
    static __device__ __forceinline__ int turn_a(int r) { return turn(r & 15); }
    static __device__ __forceinline__ int turn_b(int r) { return turn((r & 3) | (r >> 3 & 3) << 2); }
};

// How whole blocks come into LDS: by transfers past the registers (rows on 16 bytes), through registers (any rows), both with 32-bit offsets from
// the tile's first row (with rows[], whose rows may be any: from A's first); or row by row.
enum Way : int { WAY_ROWS = 0, WAY_REGISTERS = 1, WAY_TRANSFERS = 2 };

// Bound by the matrix units, and those by the power they may take.  bfloat16 results with 8-bit sums: 8192 x 8192, depth 4096, in 279 us one after another (1.97 PFLOP/s;
// 243, 2.26, between other work; 229 of zeros) and 8192 x 4096, depth 4096, in 144; 32768 rows of 64 experts, 2048 x 2048, in 222 (1.24 PFLOP/s: a fifth of the tiles' rows
// are no expert's, and start and results are a quarter of 16 steps).  In 32-bit sums 8192 x 4096, depth 4096, in 287 us (0.96 PFLOP/s: the widening of both
// operands goes through the vector units of the same waves); 16 weight gradients of 1024 x 2048 over 10000 rows in 102 (134 MB of results).  Of few rows it is the weights'
// bytes that count: 16 tokens of 4 experts each of 64, 2048 x 2048, in 26 to 38 us (173 MB, of which the last level cache holds more or less; 42 where it holds nothing).
template <int TM, int TN, int WM, int WN, int PARTS, GemmKind KIND, bool BROWS, bool FAST>
__global__ __launch_bounds__(64 * WM * WN * PARTS, TM * TN <= 64 * 64 && (FAST || !BROWS || PARTS > 1) ? 4 : 2) void fp8_tile_kernel(Fp8Problem p, int slots, int tiles_n, Way way)
{
    using L = Tile<TM, TN, WM, WN, KIND, BROWS>;
    constexpr int MT = L::MT, NT = L::NT;
    __shared__ alignas(1024) unsigned char all_mem[PARTS * 2 * L::STAGE];
    const int lane = threadIdx.x & 63, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = any_wave % L::WAVES, part = any_wave / L::WAVES, tid = threadIdx.x % L::THREADS;   // within the part of the depth that a wave works on
    unsigned char *const mem = all_mem + part * 2 * L::STAGE;
    const int wm = wave % WM, wn = wave / WM;
    const int l16 = lane & 15, g = lane >> 4;

    // the tile, and the depth it sums over
    int id;
    Place at{0, 0, p.M, false};
    int n0, k_lo = 0, k_hi = p.K;
    if constexpr (KIND == GEMM_EXPERTS) {
        // the host knows how many slots there may be, the offsets how many there are: those are dealt to the XCDs, a contiguous part to each
        // (of all that there may be, the last XCDs would get the empty ones); the other workgroups share the rows of no expert
        int tiles = 0;
        at = place_of<TM>(p.offsets, p.E, p.M, lane, [&](int all) {
            tiles = all * tiles_n;
            id = (int)blockIdx.x < tiles ? xcd_contiguous(blockIdx.x, tiles) : tiles;
            return id / tiles_n;
        });
        n0 = id % tiles_n * TN;
        if (at.zeros) {
            const float none[8] = {};
            const int pieces = (p.N + 7) / 8;
            const NoRows rows(p, at);
            for (int i = (int)blockIdx.x - tiles; i < rows.count; i += gridDim.x - tiles)
                for (int j = threadIdx.x; j < pieces; j += L::THREADS * PARTS) store_results<8>(p, rows[i], j * 8, none);
            return;
        }
    } else {
        id = xcd_contiguous(blockIdx.x, gridDim.x);
        if constexpr (KIND == GEMM_GRAD) {
            at.e = id / (slots * tiles_n);
            id %= slots * tiles_n;
            k_lo = min(max(p.offsets[at.e], 0), p.K);
            k_hi = min(max(p.offsets[at.e + 1], k_lo), p.K);
        }
        // eight rows of tiles at a time: what one XCD has in work is a block of C
        const int group = id / (8 * tiles_n), left = min(8, slots - group * 8), in = id - group * 8 * tiles_n;
        at.m0 = (group * 8 + in % left) * TM;
        n0 = in / left * TN;
    }
    const long long e_rows = KIND == GEMM_EXPERTS ? (long long)at.e * p.N : 0;
    const int kb_lo = k_lo / BLOCK, kb_hi = blocks_of(k_hi);          // blocks that the depth touches
    const int all_blocks = blocks_of(p.K);
    // whole blocks, and how many others: those that the depth's ends cut
    int f_lo = (k_lo + BLOCK - 1) / BLOCK, f_hi = k_hi / BLOCK;
    if (way == WAY_ROWS || f_hi < f_lo) f_hi = f_lo = kb_lo;
    if (k_hi <= k_lo) f_hi = f_lo = 0;
    const int n_slow = k_hi > k_lo ? (kb_hi - kb_lo) - (f_hi - f_lo) : 0;

    // the whole blocks are dealt to the parts in turn; all parts take as many steps, the last one of some on a block that is another's, scaled by zero
    const int n_steps = (f_hi - f_lo + PARTS - 1) / PARTS;
    auto block = [&](int i) { return PARTS == 1 ? f_lo + i : min(f_lo + i * PARTS + part, f_hi - 1); };
    auto live = [&](int i) { return PARTS == 1 || f_lo + i * PARTS + part < f_hi; };

    // this wave's transfers: eight rows each, lane / 8, in chunk lane % 8 of the row's place
    const bool listed = KIND == GEMM_EXPERTS && p.rows;
    const uint8_t *a_base = listed ? p.a : p.a + (long long)at.m0 * p.lda, *b_base = p.b + (e_rows + n0) * p.ldb;
    // the tile's row r, and rows past the group's end as one that there is: from a_base on
    auto a_row_at = [&](int r) { return listed ? max(0, at.m0 + r < at.m_end ? a_row_of<KIND>(p, at.m0 + r) : 0) : min(r, at.m_end - 1 - at.m0); };
    unsigned a_off[L::LOADS_A], b_off[L::LOADS_B], sa_off = 0, sb_off = 0;
#pragma unroll
    for (int j = 0; j < L::LOADS_A; ++j) {
        const int r = L::a_rows(wave, j) + (lane >> 3);
        a_off[j] = (unsigned)(a_row_at(r) * p.lda) + ((lane & 7) ^ L::turn_a(r)) * 16;
    }
#pragma unroll
    for (int j = 0; j < L::LOADS_B; ++j) {
        const int r = L::b_rows(wave, j) + (lane >> 3);
        b_off[j] = (unsigned)((long long)min(r, p.N - 1 - n0) * p.ldb) + ((lane & 7) ^ L::turn_b(r)) * 16;
    }
    if (wave < TM / 64) sa_off = 4u * (unsigned)((listed ? 0 : at.m0) + a_row_at(wave * 64 + lane));
    if (BROWS && wave < TN / 64) sb_off = 4u * (unsigned)min(n0 + wave * 64 + lane, p.N - 1);
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void *)mem;
    constexpr int PIECES = L::LOADS_A + L::LOADS_B + 1;   // the last: scales
    constexpr int FIRST = L::LOADS_A + L::LOADS_B / 2;    // those of A, and of B the half that is read first
    auto transfer = [&](int j, int kb, int stage) {
        const unsigned to = lds + stage * L::STAGE;
        if (j < L::LOADS_A) {
            dma16(a_base + (long long)kb * BLOCK, a_off[j], to + L::a_rows(wave, j) * 128);
        } else if (j < L::LOADS_A + L::LOADS_B) {
            dma16(b_base + (long long)kb * BLOCK, b_off[j - L::LOADS_A], to + (TM + L::b_rows(wave, j - L::LOADS_A)) * 128);
        } else {
            if (wave < TM / 64) dma4(p.sa + (long long)kb * p.a_rows, sa_off, to + (TM + TN) * 128 + wave * 256);
            if (BROWS && wave < TN / 64) dma4(p.sb + (long long)kb * p.N, sb_off, to + (TM + TN) * 128 + TM * 4 + wave * 256);
        }
    };
    // a lane's 16-byte chunks of a stage, A's first: chunk threadIdx % 8 of the rows row_of(i)
    constexpr int CHUNKS = (TM + TN) * 8 / L::THREADS, CHUNKS_A = TM * 8 / L::THREADS;
    static_assert(CHUNKS * L::THREADS == (TM + TN) * 8 && CHUNKS_A * L::THREADS == TM * 8);
    auto row_of = [&](int i) { return (i * L::THREADS + tid) >> 3; };
    auto place_chunk = [&](int stage, int i, v4u v) {
        const int r = row_of(i), c = tid & 7;
        *reinterpret_cast<v4u *>(mem + stage * L::STAGE + r * 128 + (c ^ (i < CHUNKS_A ? L::turn_a(r) : L::turn_b(r - TM))) * 16) = v;
    };
    auto scale_at = [&](int stage) { return reinterpret_cast<float *>(mem + stage * L::STAGE + (TM + TN) * 128); };
    // a block that the depth's ends cut, or one of any other trouble: row by row into the second stage, zeros outside the depth
    auto fill = [&](int kb) {
        constexpr int AT_ONCE = CHUNKS < 8 ? CHUNKS : 8;
        static_assert(CHUNKS % AT_ONCE == 0);
        const int k = kb * BLOCK + (tid & 7) * 16;
#pragma unroll 1
        for (int i0 = 0; i0 < CHUNKS; i0 += AT_ONCE) {
            v4u v[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int r = row_of(i0 + i);
                v[i] = v4u{0, 0, 0, 0};
                if (r < TM) {
                    const int row = at.m0 + r < at.m_end ? a_row_of<KIND>(p, at.m0 + r) : -1;
                    if (row >= 0) v[i] = load_masked(p.a + row * p.lda, k, k_lo, k_hi, p.K);
                } else if (n0 + r - TM < p.N) {
                    v[i] = load_masked(p.b + (e_rows + n0 + r - TM) * p.ldb, k, k_lo, k_hi, p.K);
                }
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int r = row_of(i0 + i), c = tid & 7;
                *reinterpret_cast<v4u *>(mem + L::STAGE + r * 128 + (c ^ (r < TM ? L::turn_a(r) : L::turn_b(r - TM))) * 16) = v[i];
            }
        }
        float *s = scale_at(1);
        for (int r = tid; r < TM; r += L::THREADS) {
            const int row = at.m0 + r < at.m_end ? a_row_of<KIND>(p, at.m0 + r) : -1;
            s[r] = row < 0 ? 0.f : p.sa[(long long)kb * p.a_rows + row];
        }
        if constexpr (BROWS)
            for (int r = tid; r < TN; r += L::THREADS) s[TM + r] = n0 + r < p.N ? p.sb[(long long)kb * p.N + n0 + r] : 0.f;
    };

    v4f acc[NT][MT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int u = 0; u < MT; ++u) acc[t][u] = v4f{0, 0, 0, 0};

    // a wave's scales of B, block after block
    const int nb = min((n0 + wn * (TN / WN)) / BLOCK, blocks_of(p.N) - 1);
    const float *sb_row = BROWS ? nullptr : p.sb + ((KIND == GEMM_EXPERTS ? (long long)at.e * blocks_of(p.N) : 0) + nb) * all_blocks;

    // fragments: places within a stage
    const int a_at = (wm * (TM / WM) + l16) * 128, b_at = TM * 128 + (wn * (TN / WN) + (l16 >> 2) * 8 + (l16 & 3)) * 128;
    const int c0 = ((2 * g) ^ L::turn(l16)) * 16, c1 = ((2 * g + 1) ^ L::turn(l16)) * 16;
    auto read_a = [&](int stage, int u, Fragment<FAST> &f) {
        const unsigned char *s = mem + stage * L::STAGE + a_at + u * 2048;
        f.set(__builtin_shufflevector(*reinterpret_cast<const v4i *>(s + c0), *reinterpret_cast<const v4i *>(s + c1), 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto read_b = [&](int stage, int t, Fragment<FAST> &f) {
        const unsigned char *s = mem + stage * L::STAGE + b_at + (t >> 1) * 4096 + (t & 1) * 512;
        f.set(__builtin_shufflevector(*reinterpret_cast<const v4i *>(s + c0), *reinterpret_cast<const v4i *>(s + c1), 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto read_sa = [&](int stage, int u) { return reinterpret_cast<const float *>(mem + stage * L::STAGE + (TM + TN) * 128)[wm * (TM / WM) + u * 16 + l16]; };
    auto read_sb = [&](int stage, int t) {   // BROWS: of the four columns that a lane has of tile t
        v4f v = {};
        if constexpr (BROWS) v = *reinterpret_cast<const v4f *>(mem + stage * L::STAGE + (TM + TN) * 128 + TM * 4 + (wn * (TN / WN) + (t >> 1) * 32 + g * 8 + (t & 1) * 4) * 4);
        return v;
    };
    auto scale_add = [&](v4f &sum, const v4f &r, float by, const v4f &sbv) {
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += (BROWS ? by * sbv[i] : by) * r[i];
    };
    typedef const __attribute__((address_space(4))) float *Constant;   // (read by scalar loads)
    const Constant sb_of = reinterpret_cast<Constant>(reinterpret_cast<uintptr_t>(sb_row));

    auto multiply = [&](int stage, float sb) {   // a stage as it stands
        Fragment<FAST> a[MT], b;
#pragma unroll
        for (int u = 0; u < MT; ++u) read_a(stage, u, a[u]);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            read_b(stage, t, b);
            const v4f sbv = read_sb(stage, t);
#pragma unroll
            for (int u = 0; u < MT; ++u) scale_add(acc[t][u], block_sum(b, a[u]), read_sa(stage, u) * sb, sbv);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // The cut blocks first: their loads and the first transfers are under way together.
    if (way == WAY_TRANSFERS && f_lo < f_hi)
#pragma unroll
        for (int j = 0; j < PIECES; ++j) transfer(j, block(0), 0);
#pragma unroll 1
    for (int i = 0; i < n_slow; ++i) {
        const int kb = kb_lo + i < f_lo ? kb_lo + i : kb_lo + i + (f_hi - f_lo);
        if (i > 0) barrier();
        if (part == 0) fill(kb);
        barrier();
        if (part == 0) multiply(1, BROWS ? 1.f : sb_of[kb]);
    }
    if constexpr (TM * TN <= 128 * 128) {
        // Rows of any alignment: the next block's chunks are on their way into registers while this one's are multiplied; a barrier a block,
        // for a stage is written again only behind the next one's.
        if (way == WAY_REGISTERS && f_lo < f_hi) {
            unsigned off[CHUNKS];
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) {
                const int r = row_of(i);
                const long long row = i >= CHUNKS_A ? min(r - TM, p.N - 1 - n0) : a_row_at(r);
                off[i] = (unsigned)(row * (i < CHUNKS_A ? p.lda : p.ldb)) + (tid & 7) * 16;
            }
            v4u v[CHUNKS];
            float s_a = 0.f, s_b = 0.f;
            auto load = [&](int kb) {
                const long long k = (long long)kb * BLOCK;
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i) v[i] = load_any((i < CHUNKS_A ? a_base : b_base) + k + off[i]);
                if (wave < TM / 64) s_a = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p.sa + (long long)kb * p.a_rows) + sa_off);
                if (BROWS && wave < TN / 64) s_b = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(p.sb + (long long)kb * p.N) + sb_off);
            };
            load(block(0));
            int stage = 0;
#pragma unroll 1
            for (int step = 0; step < n_steps; ++step, stage ^= 1) {
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i) place_chunk(stage, i, v[i]);
                if (wave < TM / 64) scale_at(stage)[tid] = s_a;
                if (BROWS && wave < TN / 64) scale_at(stage)[TM + tid] = s_b;
                if (step + 1 < n_steps) load(block(step + 1));
                barrier();
                if (live(step)) multiply(stage, BROWS ? 1.f : sb_of[block(step)]);
            }
        }
    }

    // The whole blocks, software-pipelined: B's fragment of tile t + 1 is read, and tile t - 1's results are scaled and added, while the matrix
    // units work on tile t.  A step has two barriers.  HALF: every wave has A's fragments and the first half of B's in registers, so the
    // transfers of the step after next may replace them; END, in the last tile but one: every wave has the others too, and the
    // next stage, whose transfers went out a whole step ago, has landed.  The transfers are dealt over the tiles: all at once they
    // hold up the wave that issues them, and a compute unit takes in no more than 45 bytes a cycle.
    if (way == WAY_TRANSFERS && f_lo < f_hi) {
        constexpr int HALF = NT / 2 - 2, END = NT - 2;   // (NT == 2: no HALF)
        Fragment<FAST> a[MT], b;
        float by[MT], by_last[MT];
        v4f r_last[MT], sb_last = {}, sbv;
        float sb = BROWS ? 1.f : sb_of[block(0)], sb_next = sb;
        landed<0>();
        barrier();
        if (n_steps > 1)
#pragma unroll
            for (int j = 0; j < PIECES; ++j) transfer(j, block(1), 1);
#pragma unroll
        for (int u = 0; u < MT; ++u) {
            read_a(0, u, a[u]);
            by[u] = live(0) ? read_sa(0, u) * sb : 0.f;
            by_last[u] = 0.f;
            r_last[u] = v4f{0, 0, 0, 0};
        }
        read_b(0, 0, b);
        sbv = live(0) ? read_sb(0, 0) : v4f{0, 0, 0, 0};
        int stage = 0;
        auto step = [&](int i, auto last) {
            constexpr bool more = !last.value;
            const bool more2 = i + 2 < n_steps;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                Fragment<FAST> b_next;
                v4f sb_after = {};
                if (t + 1 < NT) {
                    read_b(stage, t + 1, b_next);
                    if (live(i)) sb_after = read_sb(stage, t + 1);
                }
                if (!BROWS && t == 0) sb_next = sb_of[block(i + more)];
                if (NT > 2 && t > HALF && t <= END && more2) {
                    constexpr int SPAN = NT > 2 ? END - HALF : 1;
#pragma unroll
                    for (int j = (t - HALF - 1) * FIRST / SPAN; j < (t - HALF) * FIRST / SPAN; ++j) transfer(j, block(i + 2), stage);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int u = 0; u < MT; ++u) {
                    const v4f r = block_sum(b, a[u]);
                    scale_add(acc[(t + NT - 1) % NT][u], r_last[u], t == 0 ? by_last[u] : by[u], sb_last);
                    asm volatile("" : "+v"(acc[(t + NT - 1) % NT][u]));   // (here, and not behind the branches below)
                    r_last[u] = r;
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (NT > 2 && t == HALF) barrier();
                if (t == END) {
                    if (NT > 2 && more2) landed<FIRST>();
                    else landed<0>();
                    barrier();
                }
                if (t >= END && more2) {
                    constexpr int REST = NT > 2 ? FIRST : 0;
#pragma unroll
                    for (int j = t == END ? REST : (REST + PIECES) / 2; j < (t == END ? (REST + PIECES) / 2 : PIECES); ++j) transfer(j, block(i + 2), stage);
                }
                if (t == NT - 1) {
#pragma unroll
                    for (int u = 0; u < MT; ++u) by_last[u] = by[u];
                    if (more) {
#pragma unroll
                        for (int u = 0; u < MT; ++u) {
                            read_a(stage ^ 1, u, a[u]);
                            by[u] = live(i + 1) ? read_sa(stage ^ 1, u) * sb_next : 0.f;
                        }
                        read_b(stage ^ 1, 0, b_next);
                        if (live(i + 1)) sb_after = read_sb(stage ^ 1, 0);
                    }
                }
                sb_last = sbv;
                sbv = sb_after;
                b = b_next;
                __builtin_amdgcn_sched_barrier(0);
            }
        };
#pragma unroll 1
        for (int i = 0; i + 1 < n_steps; ++i, stage ^= 1) step(i, std::false_type{});
        step(n_steps - 1, std::true_type{});
#pragma unroll
        for (int u = 0; u < MT; ++u) scale_add(acc[NT - 1][u], r_last[u], by_last[u], sb_last);
    }
    if constexpr (PARTS > 1) {   // the parts' sums, in their order
        static_assert(NT * MT * 1024 * L::WAVES <= 2 * L::STAGE);
        auto sums = [&](int of) { return reinterpret_cast<v4f *>(all_mem + of * 2 * L::STAGE) + wave * NT * MT * 64 + lane; };
        barrier();
        if (part > 0)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int u = 0; u < MT; ++u) sums(part)[(t * MT + u) * 64] = acc[t][u];
        barrier();
        if (part > 0) return;
#pragma unroll
        for (int of = 1; of < PARTS; ++of)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int u = 0; u < MT; ++u) acc[t][u] += sums(of)[(t * MT + u) * 64];
    }
    const long long c_rows = KIND == GEMM_GRAD ? (long long)at.e * p.M : 0;
#pragma unroll
    for (int u = 0; u < MT; ++u) {
        const int m = at.m0 + wm * (TM / WM) + u * 16 + l16;
        if (m >= at.m_end) continue;
        const bool there = KIND != GEMM_EXPERTS || a_row_of<KIND>(p, m) >= 0;
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = there ? acc[t + i / 4][u][i & 3] : 0.f;
            store_results<8>(p, c_rows + m, n0 + wn * (TN / WN) + t * 16 + g * 8, v);
        }
    }
}

// ---- few rows ----------------------------------------------------------------------------------------------------------
// Eight waves on 16 * MT rows x 16 * 8 / SPLIT columns of C: a wave has 16 columns and sums every SPLIT-th block of the depth, its operands
// straight from memory into registers (16 rows of B x 128 bytes, whole cache lines, several blocks in flight); the partial sums of
// a column's SPLIT waves meet in LDS, in the waves' order.  32-bit sums throughout: they cost nothing here.
// Bound by B's bytes where there are enough: one row by 32768 x 4096 in 30 us (134 MB, 4.5 TB/s); by one round of loads where there are not: one row by
// 4096 x 4096 (17 MB, which the last level cache holds) in 5.1 to 5.9 us.
constexpr int FEW_WAVES = 8;

template <int MT, int SPLIT, GemmKind KIND, bool BROWS>
__global__ __launch_bounds__(64 * FEW_WAVES) void fp8_few_kernel(Fp8Problem p, int slots, int tiles_n)
{
    __shared__ v4f part[SPLIT > 1 ? FEW_WAVES : 1][MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4, turn = wave % SPLIT;
    constexpr int WIDTH = 16 * FEW_WAVES / SPLIT;
    const int id = blockIdx.x, n0 = id % tiles_n * WIDTH + wave / SPLIT * 16;
    Place at{0, id / tiles_n * 16 * MT, p.M, false};
    if constexpr (KIND == GEMM_EXPERTS) {
        at = place_of<16 * MT>(p.offsets, p.E, p.M, lane, [&](int) { return id / tiles_n; });
        if (at.zeros) {
            const float none[4] = {};
            const NoRows rows(p, at);
            const int step = (slots - (id / tiles_n - at.e)) * 16 * MT;
            for (int r = at.e * 16 * MT; r < rows.count; r += step)
                for (int i = threadIdx.x; i < 16 * MT * (WIDTH / 4); i += 64 * FEW_WAVES)
                    if (r + i / (WIDTH / 4) < rows.count) store_results<4>(p, rows[r + i / (WIDTH / 4)], id % tiles_n * WIDTH + i % (WIDTH / 4) * 4, none);
            return;
        }
    }
    const long long e_rows = KIND == GEMM_EXPERTS ? (long long)at.e * p.N : 0;
    const int all_blocks = blocks_of(p.K), f_hi = p.K / BLOCK;
    v4f acc[MT];
#pragma unroll
    for (int u = 0; u < MT; ++u) acc[u] = v4f{0, 0, 0, 0};
    if (n0 < p.N) {
        const uint8_t *b_row = p.b + (e_rows + min(n0 + l16, p.N - 1)) * p.ldb;
        const uint8_t *a_row[MT];
        const float *sa[MT];
#pragma unroll
        for (int u = 0; u < MT; ++u) {
            const int m = at.m0 + u * 16 + l16;
            const long long row = max(0, m < at.m_end ? a_row_of<KIND>(p, m) : 0);
            a_row[u] = p.a + row * p.lda;
            sa[u] = p.sa + row;
        }
        const float *sb = BROWS ? p.sb : p.sb + ((KIND == GEMM_EXPERTS ? (long long)at.e * blocks_of(p.N) : 0) + n0 / BLOCK) * all_blocks;
        struct Block {   // a lane's part of one
            v8i b, a[MT];
            v4f sb;
            float sa[MT];
        };
        auto scales = [&](int kb, Block &v) {
            if constexpr (BROWS) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v.sb[i] = sb[(long long)kb * p.N + min(n0 + 4 * g + i, p.N - 1)];
            } else {
                v.sb[0] = sb[kb];
            }
#pragma unroll
            for (int u = 0; u < MT; ++u) v.sa[u] = sa[u][(long long)kb * p.a_rows];
        };
        auto add = [&](const Block &v) {
            Fragment<false> bw, aw;
            bw.set(v.b);
#pragma unroll
            for (int u = 0; u < MT; ++u) {
                aw.set(v.a[u]);
                const v4f r = block_sum(bw, aw);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[u][i] += v.sa[u] * v.sb[BROWS ? i : 0] * r[i];
            }
        };
        auto load32 = [&](const uint8_t *from) { return __builtin_bit_cast(v8i, __builtin_shufflevector(load_any(from), load_any(from + 16), 0, 1, 2, 3, 4, 5, 6, 7)); };
        constexpr int AT_ONCE = MT == 1 ? 4 : 2;   // blocks in flight
#pragma unroll 1
        for (int kb0 = turn; kb0 < f_hi; kb0 += AT_ONCE * SPLIT) {
            Block v[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int kb = kb0 + i * SPLIT;
                if (i > 0 && kb >= f_hi) continue;
                const long long k = (long long)kb * BLOCK + g * 32;
                v[i].b = load32(b_row + k);
#pragma unroll
                for (int u = 0; u < MT; ++u) v[i].a[u] = load32(a_row[u] + k);
                scales(kb, v[i]);
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                if (i == 0 || kb0 + i * SPLIT < f_hi) add(v[i]);
        }
        if (f_hi < all_blocks && turn == f_hi % SPLIT) {   // the rest of the depth, less than a block
            const int k = f_hi * BLOCK + g * 32;
            auto load32m = [&](const uint8_t *row) {
                return __builtin_bit_cast(v8i, __builtin_shufflevector(load_masked(row, k, 0, p.K, p.K), load_masked(row, k + 16, 0, p.K, p.K), 0, 1, 2, 3, 4, 5, 6, 7));
            };
            Block v;
            v.b = load32m(b_row);
#pragma unroll
            for (int u = 0; u < MT; ++u) v.a[u] = load32m(a_row[u]);
            scales(f_hi, v);
            add(v);
        }
    }
    auto store = [&](int u, const v4f &sum) {
        const int m = at.m0 + u * 16 + l16;
        if (m >= at.m_end || n0 >= p.N) return;
        const bool there = KIND != GEMM_EXPERTS || a_row_of<KIND>(p, m) >= 0;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = there ? sum[i] : 0.f;
        store_results<4>(p, m, n0 + 4 * g, v);
    };
    if constexpr (SPLIT == 1) {
#pragma unroll
        for (int u = 0; u < MT; ++u) store(u, acc[u]);
    } else {
#pragma unroll
        for (int u = 0; u < MT; ++u) part[wave][u][lane] = acc[u];
        __syncthreads();
        for (int u = turn; u < MT; u += SPLIT) {
            const int first = wave - turn;
            v4f sum = part[first][u][lane];
#pragma unroll
            for (int w = 1; w < SPLIT; ++w) sum += part[first + w][u][lane];
            store(u, sum);
        }
    }
}

// Slots of `rows` rows that cover E ragged groups of R rows in all, and one at least for rows of no expert.
long long slots_for(int R, int E, int rows)
{
    const long long most = (long long)R / rows + E;
    return (most < R ? most : R) + 1;
}

long long slots_of(const Fp8Problem &p, GemmKind kind, int rows) { return kind == GEMM_EXPERTS ? slots_for(p.M, p.E, rows) : (p.M + rows - 1) / rows; }
long long tiles_of(const Fp8Problem &p, GemmKind kind, int rows, int cols) { return slots_of(p, kind, rows) * ((p.N + cols - 1) / cols) * (kind == GEMM_GRAD ? p.E : 1); }

template <int TM, int TN, int WM, int WN, int PARTS, bool FAST>
hipError_t launch_tiles(const Fp8Problem &p, GemmKind kind, Way way, hipStream_t st)
{
    const int tiles_n = (p.N + TN - 1) / TN;
    const long long slots = slots_of(p, kind, TM), grid = tiles_of(p, kind, TM, TN);
    if (!fits_launch(grid, 64 * WM * WN * PARTS)) return TOO_LARGE;
    const dim3 g((unsigned)grid), b(64 * WM * WN * PARTS);
    const int s = (int)slots;
    if (kind == GEMM_EXPERTS) return c2i8::launch(fp8_tile_kernel<TM, TN, WM, WN, PARTS, GEMM_EXPERTS, false, FAST>, g, b, 0, st, p, s, tiles_n, way);
    if (kind == GEMM_GRAD) return c2i8::launch(fp8_tile_kernel<TM, TN, WM, WN, PARTS, GEMM_GRAD, true, FAST>, g, b, 0, st, p, s, tiles_n, way);
    if (p.b_rows) return c2i8::launch(fp8_tile_kernel<TM, TN, WM, WN, PARTS, GEMM_DENSE, true, FAST>, g, b, 0, st, p, s, tiles_n, way);
    return c2i8::launch(fp8_tile_kernel<TM, TN, WM, WN, PARTS, GEMM_DENSE, false, FAST>, g, b, 0, st, p, s, tiles_n, way);
}

template <int MT, int SPLIT>
hipError_t launch_few(const Fp8Problem &p, GemmKind kind, long long slots, hipStream_t st)
{
    constexpr int WIDTH = 16 * FEW_WAVES / SPLIT;
    const int tiles_n = (p.N + WIDTH - 1) / WIDTH;
    if (!fits_launch(slots * tiles_n, 64 * FEW_WAVES)) return TOO_LARGE;
    const dim3 g((unsigned)(slots * tiles_n)), b(64 * FEW_WAVES);
    const int s = (int)slots;
    if (kind == GEMM_EXPERTS) return c2i8::launch(fp8_few_kernel<MT, SPLIT, GEMM_EXPERTS, false>, g, b, 0, st, p, s, tiles_n);
    if (p.b_rows) return c2i8::launch(fp8_few_kernel<MT, SPLIT, GEMM_DENSE, true>, g, b, 0, st, p, s, tiles_n);
    return c2i8::launch(fp8_few_kernel<MT, SPLIT, GEMM_DENSE, false>, g, b, 0, st, p, s, tiles_n);
}
template <int MT>
hipError_t launch_few(const Fp8Problem &p, GemmKind kind, hipStream_t st)
{
    const long long slots = slots_of(p, kind, 16 * MT);
    // the depth is shared out until there are 4096 waves, or as far as it goes
    const long long waves = slots * ((p.N + 15) / 16);
    if (waves >= 4096 || p.K <= 2 * BLOCK) return launch_few<MT, 1>(p, kind, slots, st);
    if (waves >= 1024 || p.K <= 4 * BLOCK) return launch_few<MT, 4>(p, kind, slots, st);
    return launch_few<MT, 8>(p, kind, slots, st);
}

}  // namespace

hipError_t launch_fp8_gemm(const Fp8Problem &p, GemmKind kind, hipStream_t st)
{
    const bool on16 = ((reinterpret_cast<uintptr_t>(p.a) | reinterpret_cast<uintptr_t>(p.b) | (uintptr_t)p.lda | (uintptr_t)p.ldb) & 15) == 0;
    const bool near = 256 * p.ldb < 0xffffffffll && (p.rows ? (long long)p.a_rows : 256) * p.lda < 0xffffffffll;
    const Way way = !near ? WAY_ROWS : on16 ? WAY_TRANSFERS : WAY_REGISTERS;
    const double area = (double)p.M * p.N * (kind == GEMM_GRAD ? p.E : 1);
    const double rows = kind == GEMM_EXPERTS ? (double)p.M / p.E : p.M;   // of a weight matrix, in the mean
    const int depth = blocks_of(p.K) / (kind == GEMM_GRAD ? p.E : 1);
    // Few rows: the kernel without tiles has the shorter start and step, but reads A again for 16 columns each and moves bytes more slowly; so it is for
    // weights that take no longer than a tile's steps.  Where that ends depends on where the weights are, since the tiles move bytes faster from the last level cache: from memory
    // at a cost (below) of some 4.5e6 a step, from the cache at 2e6 with fast sums and 3e6 in 32 bits; 2.5e6 lies between (us, few | tiles in 32-bit sums, weights from memory, then from the
    // cache; rows x N, depth, or tokens, experts of each and of all, N, depth):
    //   1.1e6   1, 4 of 64, 2048, 2048    7.8 | 13.9    6.2 | 12.3       3.1e6   12 x 16384, 4096         18.1 | 21.3   16.8 | 15.7
    //   2.1e6   2, 4 of 64, 2048, 2048   10.7 | 14.4    9.6 | 13.7       4.2e6   8 x 32768, 4096          30.1 | 35.5   27.6 | 25.6
    //   2.1e6   8 x 16384, 4096          17.8 | 21.5   15.9 | 15.9       5.2e6   20 x 16384, 4096         22.7 | 21.6   21.2 | 16.2
    //   3.1e6   64, 2 of 16, 1024, 2048  12.0 | 14.2   11.3 | 11.7       9.1e6   8, 6 of 64, 1408, 2048   28.7 | 27.3   27.1 | 24.0
    // Rows that are not on 16 bytes cost it twice as much: 64, 2 of 16, 512, 1981 (1.5e6) 12.9 | 17.6, 128 of them (2.0e6) 22.5 | 19.0.  Of over 32 rows tiles are level or better
    // (33 x 16384, 4096  37 | 15) but for the smallest (33 x 300, 777  6.5 | 8.8).
    if (kind != GEMM_GRAD && rows <= 32) {
        const double weights = (kind == GEMM_EXPERTS ? fmin(p.M, p.E) : 1.) * p.N * p.K;   // bytes of those asked for
        const double cost = kind == GEMM_EXPERTS ? weights * (1 + rows / 16) : weights * rows / 8;
        if (cost <= (on16 ? 2.5e6 : 1.25e6) * depth) return rows <= 16 ? launch_few<1>(p, kind, st) : launch_few<2>(p, kind, st);
    }
    // How large a tile: a large one moves fewer bytes for its work, a small one fills the chip sooner and starts and stores in less time (200 sizes with
    // every tile; us, fast sums: 256 x 256 | 128 x 128 | 64 x 64, 32-bit sums: 128 x 128 | 64 x 64):
    //   2048 x 2048, depth 2048  28 | 16.8 | 15.0   28 | 24      4096 x 4096, depth 2048   34 | 40 | 52    71 | 82
    //   2048 x 4096, depth 2048  30 | 22.6 | 27.3   38 | 43      8192 x 8192, depth 512    58 | 55 | 70   100 | 107
    // (of weight gradients, whose depth is an expert's rows, 256 x 256 pays sooner: 16 of 2048 x 1408, 320 rows each, 53 | 58).  An expert's rows have to fill it: 64 experts of
    // 2048 x 2048 with 72 rows each 98 | 77 | 88, with 140 106 | 98 | 125, with 300 148 | 158 | 211.
    if (p.fast_sums && area >= 14e6 && rows >= 160 && depth >= (kind == GEMM_GRAD ? 4 : 8) && way == WAY_TRANSFERS)
        return launch_tiles<256, 256, 4, 2, 1, true>(p, kind, way, st);
    // (and a launch need not hold as many of the smaller: 1024 weight gradients of 8192 x 8192 ask for 2^24)
    if ((area >= (kind == GEMM_EXPERTS ? 6e6 : 8e6) && rows > 64 && (p.fast_sums || depth >= 4)) || !fits_launch(tiles_of(p, kind, 64, 64), 256))
        return p.fast_sums ? launch_tiles<128, 128, 2, 2, 1, true>(p, kind, way, st) : launch_tiles<128, 128, 2, 2, 1, false>(p, kind, way, st);
    // Tiles for no more than the compute units and a deep sum: in four parts to a workgroup, which bring in more at a time; of more tiles one part (1000 x 2048, depth 2048
    // 10.0 | 13.9).  From which depth on four take less depends on what a step costs: 16 waves leave 128 registers each, of which 32-bit sums spill 17 where B has a scale
    // for each row and 7 in weight gradients, and rows off 16 bytes come in through registers (us, one part | four; depth in blocks):
    //   blocks                          8            12           16           32
    //   512 x 512, fast sums        5.5 |  5.5   6.8 |  6.5   8.1 |  7.3  13.2 | 10.1      off 16 bytes   7.0 |  6.9   8.9 |  9.1  10.8 | 10.7  18.8 | 17.3
    //   32-bit sums                 7.2 |  7.0   9.3 |  8.1  11.3 |  9.1  19.7 | 13.4                     8.5 |  8.7  11.3 | 10.5  14.0 | 12.2  25.0 | 19.3
    //   B with a scale for a row    7.2 |  7.8   9.3 |  9.1  11.4 | 10.4  19.9 | 15.6                     8.4 | 10.1  11.1 | 11.8  13.7 | 13.4  24.6 | 20.5
    //   gradients, 2 of 512 x 512   7.7 |  9.5               11.9 | 12.6  20.6 | 18.7                     9.0 | 10.8               14.8 | 14.0  25.5 | 20.9
    // Rows too far apart for either go row by row, which is one part's work.
    const double tiles = ((p.M + 63) / 64 + (kind == GEMM_EXPERTS ? p.E / 2 : 0)) * (double)((p.N + 63) / 64) * (kind == GEMM_GRAD ? p.E : 1);
    const int from = way == WAY_ROWS ? 0x7fffffff : way == WAY_TRANSFERS ? (p.fast_sums ? 12 : kind == GEMM_GRAD ? 32 : p.b_rows ? 12 : 8) : p.fast_sums ? 32 : p.b_rows ? 16 : 12;
    if (tiles <= 256 && depth >= from)
        return p.fast_sums ? launch_tiles<64, 64, 2, 2, 4, true>(p, kind, way, st) : launch_tiles<64, 64, 2, 2, 4, false>(p, kind, way, st);
    return p.fast_sums ? launch_tiles<64, 64, 2, 2, 1, true>(p, kind, way, st) : launch_tiles<64, 64, 2, 2, 1, false>(p, kind, way, st);
}

}  // namespace xp8
