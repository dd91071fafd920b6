// Routing: choice of experts, its gradient, the order of the experts' rows, and the combination of their results.
#include "experts.h"
#include "launch.h"

#include <float.h>

namespace xp8 {
namespace {

constexpr float NEG_INF = -__builtin_inff();

// A wave on a token, lane l holding the V neighbouring experts V l ... V l + V - 1 (V: the least power of two that covers E): the
// lowest lane with the largest value then holds the lowest index, and a wave-wide maximum is four DPP steps and four lane reads.
// 4 tokens to a workgroup; no LDS but for groups.
template <typename T, int V>
__device__ __forceinline__ void load_logits(const RouteProblem &p, int t, int lane, float (&x)[V], bool (&there)[V])
{
    const T *row = static_cast<const T *>(p.logits) + t * p.ldl;
    constexpr int BYTES = sizeof(T) * V;
    // rows of whole pieces, aligned: one load a lane
    if (BYTES <= 16 && p.E == 64 * V && ((reinterpret_cast<uintptr_t>(p.logits) | (uintptr_t)(p.ldl * sizeof(T))) & (BYTES - 1)) == 0) {
        struct alignas(BYTES <= 16 ? BYTES : 16) Piece {
            T v[V];
        } w = reinterpret_cast<const Piece *>(row)[lane];
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = to_float(w.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = lane * V + i < p.E ? to_float(row[lane * V + i]) : NEG_INF;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        there[i] = x[i] > NEG_INF;           // neither NaN
        x[i] = fminf(x[i], FLT_MAX);
    }
}

// x -> scores; experts not to be had have 0.  (Reciprocals of the hardware's, one step of the last place off at most.)
template <int V>
__device__ __forceinline__ void scores(bool sigmoid, float (&x)[V], const bool (&there)[V])
{
    if (sigmoid) {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = there[i] ? __builtin_amdgcn_rcpf(1.f + expf(-x[i])) : 0.f;
        return;
    }
    float top = NEG_INF, sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) top = there[i] ? fmaxf(top, x[i]) : top;
    top = max64(top);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        x[i] = there[i] ? expf(x[i] - top) : 0.f;
        sum += x[i];
    }
    const float by = __builtin_amdgcn_rcpf(fmaxf(sum64(sum), 1e-30f));   // (0 only where no expert is to be had: the largest adds 1)
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] *= by;
}

// k rounds of a maximum over what each lane has sorted before.  Bound by vector instructions, some 600 a token: 8192 tokens, 8 of 256 experts, 4 of 8 groups, in
// 11.2 us; one token, 6 of 64, 2.3.
template <typename T, int V>
__global__ __launch_bounds__(256) void route_kernel(RouteProblem p)
{
    extern __shared__ int choice_of[];   // [4][64 V], with groups
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x * 4 + wave;
    const bool mine = t < p.T;
    float s[V];
    int c[V];   // choice scores, as whole numbers in their order
    bool there[V];
    const int none = order_key(NEG_INF);
    load_logits<T, V>(p, mine ? t : p.T - 1, lane, s, there);
    scores<V>(p.sigmoid, s, there);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float v = there[i] && p.bias ? s[i] + p.bias[lane * V + i] : s[i];
        c[i] = there[i] && v > NEG_INF ? order_key(v) : none;   // (a NaN is not to be had)
    }
    if (p.groups > 1) {
        // 64 / groups lanes (rounded down to a power of two) scan a group and join their best two; then the groups' rank, counted; those left
        // out lose their scores.  All in the wave's own part of LDS.
        const int each = p.E / p.groups, shift = 31 - __builtin_clz(64 / p.groups), width = 1 << shift;
        int *mem = choice_of + wave * 64 * V;
        auto settled = [] {   // (a wave's LDS accesses are in order; the compiler is to keep it)
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        };
#pragma unroll
        for (int i = 0; i < V; ++i) mem[lane * V + i] = c[i];
        settled();
        const int g = lane >> shift;
        int a = none, b = none;
        if (g < p.groups)
            for (int i = lane & (width - 1); i < each; i += width) {
                const int v = mem[g * each + i];
                b = max(b, min(a, v));
                a = max(a, v);
            }
        for (int m = 1; m < width; m *= 2) {
            const int a2 = __shfl_xor(a, m), b2 = __shfl_xor(b, m);
            b = max(min(a, a2), max(b, b2));
            a = max(a, a2);
        }
        if (p.group_top == 2 && b > none) {   // (of two that are to be had)
            auto value = [](int key) { return __builtin_bit_cast(float, key ^ (key >> 31 & 0x7fffffff)); };
            a = order_key(fmaxf(value(a) + value(b), -FLT_MAX));   // (of two lowest numbers: not -infinity, which is a group of none)
        }
        int ahead = 0;   // groups that come before mine
        for (int o = 0; o < p.groups; ++o) {
            const int other = __builtin_amdgcn_readlane(a, o << shift);
            ahead += other > a || (other == a && o < g) ? 1 : 0;
        }
        if (g < p.groups && ahead >= p.kept)
            for (int i = lane & (width - 1); i < each; i += width) mem[g * each + i] = none;
        settled();
#pragma unroll
        for (int i = 0; i < V; ++i) c[i] = mem[lane * V + i];
    }
    // Each lane's values in falling order (lower index first among equals), their places two to four bits each in `order`: then the largest of all, k
    // times, is the largest of the lanes' first ones; the lowest lane that has it holds the lowest index and moves up by one.
    using Order = std::conditional_t<(V > 8), unsigned long long, unsigned>;
    Order order = 0;
    {
        int at[V];
#pragma unroll
        for (int i = 0; i < V; ++i) at[i] = i;
        // odd-even transposition: neighbours change places only if out of order, so equals keep theirs
#pragma unroll
        for (int pass = 0; pass < V; ++pass)
#pragma unroll
            for (int i = pass & 1; i + 1 < V; i += 2) {
                const bool swap = c[i + 1] > c[i];
                const int hi = swap ? c[i + 1] : c[i], lo = swap ? c[i] : c[i + 1];
                const int hi_at = swap ? at[i + 1] : at[i], lo_at = swap ? at[i] : at[i + 1];
                c[i] = hi, c[i + 1] = lo, at[i] = hi_at, at[i + 1] = lo_at;
            }
#pragma unroll
        for (int i = 0; i < V; ++i) order |= (Order)at[i] << (4 * i);
    }
    int id = -1;
    for (int j = 0; j < p.k; ++j) {
        const int best = max64(c[0]);
        if (best == none) break;
        const int owner = __builtin_ctzll(__ballot(c[0] == best));
        const int chosen = owner * V + (__builtin_amdgcn_readlane((int)order, owner) & 15);
        if (lane == j) id = chosen;
        if (lane == owner) {
#pragma unroll
            for (int i = 0; i + 1 < V; ++i) c[i] = c[i + 1];
            c[V - 1] = none;
            order >>= 4;
        }
    }
    float w = 0.f;   // the score of my choice, from the lane that holds it
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float v = __shfl(s[i], id < 0 ? 0 : id / V);
        if (id >= 0 && id % V == i) w = v;
    }
    const float total = sum64(w);
    if (mine && lane < p.k) {
        p.ids[(long long)t * p.k + lane] = id;
        p.weights[(long long)t * p.k + lane] = (p.renormalise ? w / (total + 1e-20f) : w) * p.factor;
    }
}

// With the chosen scores' sum S: w = factor s / S, so ds_j = factor (dw_j - sum_i dw_i s_i / S) / S; then the scores' own derivative,
// dl = s (1 - s) ds or s (ds - sum s ds) over all experts to be had.  The scores are made again from the logits, which is cheaper than to have kept them.
// 8192 tokens of 256 experts in 6.7 us (17 MB), bound by vector instructions.
template <typename T, int V>
__global__ __launch_bounds__(256) void route_backward_kernel(RouteProblem p)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x * 4 + wave;
    if (t >= p.T) return;
    float s[V], d[V];
    bool there[V];
    load_logits<T, V>(p, t, lane, s, there);
    scores<V>(p.sigmoid, s, there);
    const int id = lane < p.k ? p.given[(long long)t * p.k + lane] : -1;
    const bool valid = id >= 0 && id < p.E;
    const float dw = valid ? p.dweights[(long long)t * p.k + lane] * p.factor : 0.f;
    // the score of choice j, from the lane that holds it
    float sj = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float v = __shfl(s[i], valid ? id / V : 0);
        if (valid && id % V == i) sj = v;
    }
    float ds = dw;
    if (p.renormalise) {
        const float total = sum64(sj) + 1e-20f, mean = sum64(dw * (sj / total));
        ds = valid ? (dw - mean) / total : 0.f;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = 0.f;
    for (int j = 0; j < p.k; ++j) {
        const int at = __builtin_amdgcn_readlane(valid ? id : -1, j) - lane * V;
        const float add = lane_of(ds, j);
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] += at == i ? add : 0.f;
    }
    if (p.sigmoid) {
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] = d[i] * s[i] * (1.f - s[i]);
    } else {
        float dot = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) dot += d[i] * s[i];
        dot = sum64(dot);
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] = s[i] * (d[i] - dot);
    }
    T *row = static_cast<T *>(p.dlogits) + t * p.lddl;
    constexpr int BYTES = sizeof(T) * V;
    if (BYTES <= 16 && p.E == 64 * V && ((reinterpret_cast<uintptr_t>(p.dlogits) | (uintptr_t)(p.lddl * sizeof(T))) & (BYTES - 1)) == 0) {
        struct alignas(BYTES <= 16 ? BYTES : 16) Piece {
            T v[V];
        } o;
#pragma unroll
        for (int i = 0; i < V; ++i) o.v[i] = (T)(there[i] ? d[i] : 0.f);
        reinterpret_cast<Piece *>(row)[lane] = o;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (lane * V + i < p.E) row[lane * V + i] = (T)(there[i] ? d[i] : 0.f);
    }
}

// Order of the experts' rows: a stable counting sort in one launch without a workspace.  Every workgroup counts ALL ids (they come
// from the L2; counts do not depend on the order of the LDS additions), those before its own segment apart, so it knows where its
// segment's pairs of each expert begin; then it ranks its pairs, a workgroup's lanes at a time: within a wave by ballots over the bits of the
// expert's number, across the waves by their counts.  Bound by instructions, about eight and one LDS addition to 64 ids in every workgroup: 65536 ids of 256
// experts in 10.3 us, six ids in 2.4 (wider loads 10.6; counters in 32 copies over the banks 12.9).
// READY: the numbers before[] lie at the beginning of the workgroup's own segment of place[], from the two kernels below, and only the ranking is left.
template <int WAVES, bool READY>
__global__ __launch_bounds__(64 * WAVES) void expert_rows_kernel(OrderProblem p, int segment, int bits)
{
    constexpr int THREADS = 64 * WAVES;
    extern __shared__ int order_mem[];
    const int E = p.E, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int *before = order_mem;                                 // [E]: pairs of an expert ahead of mine, then: its next row
    int *count = order_mem + E;                              // [E]: pairs in all
    int *start = order_mem + 2 * E;                          // [E + 1]
    unsigned short *of_wave = reinterpret_cast<unsigned short *>(order_mem + (3 * E + 4) / 4 * 4);   // [E][WAVES], 16-byte pieces
    const int from = blockIdx.x * segment, to = READY && blockIdx.x + 1 == gridDim.x ? p.pairs : min(p.pairs, from + segment);
    if constexpr (READY) {
        for (int e = tid; e < E; e += THREADS) before[e] = p.place[from + e];
        if (tid == 0) start[E] = p.offsets[E];
        __syncthreads();
    } else {
        for (int e = tid; e < E; e += THREADS) before[e] = count[e] = 0;
        __syncthreads();
        // (segments are whole rounds of the lanes, so a round is all before mine or none of it is; eight ids a lane in flight)
        auto tally = [&](int round, unsigned e) {
            if (e < (unsigned)E) atomicAdd((round < from ? before : count) + e, 1);
        };
        int i0 = 0;
        for (; i0 + 8 * THREADS <= p.pairs; i0 += 8 * THREADS) {
            int e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = p.ids[i0 + j * THREADS + tid];
#pragma unroll
            for (int j = 0; j < 8; ++j) tally(i0 + j * THREADS, (unsigned)e[j]);
        }
        for (; i0 < p.pairs; i0 += THREADS)
            if (i0 + tid < p.pairs) tally(i0, (unsigned)p.ids[i0 + tid]);
        __syncthreads();
        if (wave == 0) {   // starts: a running sum of the rounded counts, 64 experts at a time
            int carry = 0;
            for (int e0 = 0; e0 < E; e0 += 64) {
                const int e = e0 + lane, n = e < E ? before[e] + count[e] : 0;
                const int padded = p.align == 1 ? n : (n + p.align - 1) / p.align * p.align;
                const int sum = running_sum(padded);
                if (e < E) {
                    start[e] = carry + sum - padded;
                    before[e] += carry + sum - padded;
                    count[e] = n;
                }
                carry += __builtin_amdgcn_readlane(sum, 63);
            }
            if (lane == 0) start[E] = carry;
        }
        __syncthreads();
        if (blockIdx.x == 0)
            for (int e = tid; e <= E; e += THREADS) p.offsets[e] = start[e];
        // rows of no pair: behind each expert's (a wave to an expert), and behind the last expert's
        if (p.align > 1)
            for (int e = blockIdx.x * WAVES + wave; e < E; e += gridDim.x * WAVES)
                for (int r = start[e] + count[e] + lane; r < start[e + 1]; r += 64) p.rows[r] = -1;
    }
    for (int r = start[E] + blockIdx.x * THREADS + tid; r < p.R; r += gridDim.x * THREADS) p.rows[r] = -1;
    for (int base = from; base < to; base += THREADS) {
        const int i = base + tid;
        int e = i < to ? p.ids[i] : -1;
        if (e < 0 || e >= E) e = -1;
        unsigned long long same = __ballot(e >= 0);
        for (int b = 0; b < bits; ++b) {
            const unsigned long long set = __ballot(e >> b & 1);
            same &= (e >> b & 1) ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        for (int x = tid; x < E; x += THREADS) {
#pragma unroll
            for (int w = 0; w < WAVES / 8; ++w) reinterpret_cast<v4i *>(of_wave + x * WAVES)[w] = v4i{0, 0, 0, 0};
        }
        __syncthreads();
        if (e >= 0 && rank == 0) of_wave[e * WAVES + wave] = (unsigned short)__popcll(same);
        __syncthreads();
        for (int x = tid; x < E; x += THREADS) {   // counts -> pairs of the waves ahead
            int sum = 0;
#pragma unroll
            for (int w = 0; w < WAVES / 8; ++w) {
                v4i v = reinterpret_cast<const v4i *>(of_wave + x * WAVES)[w];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const int lo = v[h] & 0xffff, hi = (int)((unsigned)v[h] >> 16);
                    v[h] = sum | (sum + lo) << 16;
                    sum += lo + hi;
                }
                reinterpret_cast<v4i *>(of_wave + x * WAVES)[w] = v;
            }
            count[x] = sum;
        }
        __syncthreads();
        if (i < to) {
            const int r = e >= 0 ? before[e] + of_wave[e * WAVES + wave] + rank : -1;
            if (e >= 0) p.rows[r] = i;
            p.place[i] = r;
        }
        if (base + THREADS < to) {
            __syncthreads();
            for (int x = tid; x < E; x += THREADS) before[x] += count[x];
        }
    }
}

// Of many pairs, counts first: a workgroup's own segment's, left at the beginning of its part of place[], which nobody else reads or writes but ...
__global__ __launch_bounds__(1024) void count_pairs_kernel(OrderProblem p, int segment)
{
    extern __shared__ int order_mem[];
    const int from = blockIdx.x * segment, to = blockIdx.x + 1 == gridDim.x ? p.pairs : from + segment, tid = threadIdx.x;
    for (int e = tid; e < p.E; e += 1024) order_mem[e] = 0;
    __syncthreads();
#pragma unroll 4
    for (int i = from + tid; i < to; i += 1024) {
        const unsigned e = (unsigned)p.ids[i];
        if (e < (unsigned)p.E) atomicAdd(order_mem + e, 1);
    }
    __syncthreads();
    for (int e = tid; e < p.E; e += 1024) p.place[from + e] = order_mem[e];
}
// ... one workgroup, which makes of them the first rows of each segment's pairs; and the offsets and the rows of no pair behind an expert's.  A lane to one of
// `wide` experts (E, rounded up to whole waves and a power of two), as many parts of the segments as the lanes give.
__global__ __launch_bounds__(1024) void start_rows_kernel(OrderProblem p, int segment, int segments, int wide)
{
    __shared__ int of_part[1024], of_wave[16];
    const int tid = threadIdx.x, e = tid & (wide - 1), part = tid / wide, parts = 1024 / wide, lane = tid & 63, wave = tid >> 6;
    const int each = (segments + parts - 1) / parts, lo = min(segments, part * each), hi = min(segments, lo + each);
    const int32_t *mine = p.place + min(e, p.E - 1);
    constexpr int AT_ONCE = 16;
    int sum = 0;
    for (int s0 = lo; s0 < hi; s0 += AT_ONCE) {
        int c[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) c[j] = mine[min(s0 + j, hi - 1) * segment];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) sum += s0 + j < hi ? c[j] : 0;
    }
    of_part[tid] = sum = e < p.E ? sum : 0;
    __syncthreads();
    int n = 0, ahead = 0;
    for (int q = 0; q < parts; ++q) {
        const int c = of_part[q * wide + e];
        n += c;
        ahead += q < part ? c : 0;
    }
    const int padded = (n + p.align - 1) / p.align * p.align;
    const int up_to = running_sum(padded);
    if (lane == 63) of_wave[wave] = up_to;
    __syncthreads();
    int row = up_to - padded;
    for (int w = wave & ~(wide / 64 - 1); w < wave; ++w) row += of_wave[w];
    if (p.align > 1)
        for (int l = part; l < 64; l += parts) {
            const int end = __builtin_amdgcn_readlane(row + padded, l);
            for (int r = __builtin_amdgcn_readlane(row + n, l) + lane; r < end; r += 64) p.rows[r] = -1;
        }
    if (e >= p.E) return;
    if (part == 0) {
        p.offsets[e] = row;
        if (e + 1 == p.E) p.offsets[p.E] = row + padded;
    }
    row += ahead;
    for (int s0 = lo; s0 < hi; s0 += AT_ONCE) {
        int c[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) c[j] = mine[min(s0 + j, hi - 1) * segment];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
            if (s0 + j < hi) {
                p.place[(s0 + j) * segment + e] = row;
                row += c[j];
            }
    }
}

// Combination: a thread on VEC neighbouring columns of a token; bound by the rows' bytes: 8192 tokens, 4 rows of 2048 bfloat16 each, in 40 us (168 MB, 4.2 TB/s), 32
// tokens 3.8.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void combine_kernel(CombineProblem p, int pieces, unsigned first)
{
    const long long at = ((long long)first + blockIdx.x) * 256 + threadIdx.x;
    if (at >= (long long)p.T * pieces) return;
    const int t = (int)(at / pieces), c = (int)(at % pieces) * VEC;
    const int32_t *place = p.place + (long long)t * p.k;
    const float *w = p.weights ? p.weights + (long long)t * p.k : nullptr;
    float sum[VEC] = {};
#pragma unroll 4
    for (int j = 0; j < p.k; ++j) {
        const int r = place[j];
        if (r < 0 || r >= p.R) continue;
        const float by = w ? w[j] : 1.f;
        const Vec<T, VEC> y = *reinterpret_cast<const Vec<T, VEC> *>(static_cast<const T *>(p.y) + r * p.ldy + c);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] += by * to_float(y.v[i]);
    }
    Vec<T, VEC> o;
#pragma unroll
    for (int i = 0; i < VEC; ++i) o.v[i] = (T)sum[i];
    *reinterpret_cast<Vec<T, VEC> *>(static_cast<T *>(p.out) + t * p.ldo + c) = o;
}

// Both gradients: a wave on a pair, in token order, so that a token's gradient comes from the caches for all but its first pair; the
// same wave looks after row number `wave` in case it has no pair.  Bound by memory: 8192 tokens, 4 rows of 2048 bfloat16, in 54.7 us (302 MB, 5.5 TB/s).
template <typename T, int VEC>
__global__ __launch_bounds__(256) void combine_backward_kernel(CombineProblem p)
{
    const int lane = threadIdx.x & 63;
    const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at < p.R && p.dy) {
        const int pair = p.rows[at];
        const bool has = pair >= 0 && pair < p.T * p.k && p.place[pair] == (int)at;
        if (!has) {
            T *row = static_cast<T *>(p.dy) + at * p.lddy;
            Vec<T, VEC> zero = {};
            for (int c = lane * VEC; c < p.N; c += 64 * VEC) *reinterpret_cast<Vec<T, VEC> *>(row + c) = zero;
        }
    }
    if (at >= (long long)p.T * p.k) return;
    const int r = p.place[at];
    if (r < 0 || r >= p.R) {
        if (lane == 0) p.dweights[at] = 0.f;
        return;
    }
    const bool its = p.rows[r] == (int)at;   // (a row that two pairs claim belongs to the one that it names)
    const float w = p.weights ? p.weights[at] : 1.f;
    const T *d = static_cast<const T *>(p.dout) + at / p.k * p.ldd, *y = static_cast<const T *>(p.y) + r * p.ldy;
    T *dy = static_cast<T *>(p.dy) + r * p.lddy;
    float dot = 0.f;
    for (int c = lane * VEC; c < p.N; c += 64 * VEC) {
        const Vec<T, VEC> dv = *reinterpret_cast<const Vec<T, VEC> *>(d + c), yv = *reinterpret_cast<const Vec<T, VEC> *>(y + c);
        Vec<T, VEC> o;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            dot += to_float(dv.v[i]) * to_float(yv.v[i]);
            o.v[i] = (T)(w * to_float(dv.v[i]));
        }
        if (its) *reinterpret_cast<Vec<T, VEC> *>(dy + c) = o;
    }
    dot = sum64(dot);
    if (lane == 0) p.dweights[at] = dot;
}

bool in_pieces(const void *base, long long ld, int cols, int size)
{
    return (reinterpret_cast<uintptr_t>(base) & 15) == 0 && (ld * size) % 16 == 0 && (cols * (long long)size) % 16 == 0;
}

// f(type, V) with V experts to a lane
template <typename F>
hipError_t for_experts(const RouteProblem &p, F &&f)
{
    return with_type(p.type, [&](auto t) {
        if (p.E <= 64) return f(t, std::integral_constant<int, 1>{});
        if (p.E <= 128) return f(t, std::integral_constant<int, 2>{});
        if (p.E <= 256) return f(t, std::integral_constant<int, 4>{});
        if (p.E <= 512) return f(t, std::integral_constant<int, 8>{});
        return f(t, std::integral_constant<int, 16>{});
    });
}

}  // namespace

hipError_t launch_route(const RouteProblem &p, hipStream_t st)
{
    return for_experts(p, [&](auto t, auto v) {
        return c2i8::launch(route_kernel<decltype(t), v.value>, dim3((p.T + 3) / 4), dim3(256), p.groups > 1 ? 4u * 64 * v.value * 4 : 0, st, p);
    });
}

hipError_t launch_route_backward(const RouteProblem &p, hipStream_t st)
{
    return for_experts(p, [&](auto t, auto v) { return c2i8::launch(route_backward_kernel<decltype(t), v.value>, dim3((p.T + 3) / 4), dim3(256), 0, st, p); });
}

hipError_t launch_expert_rows(const OrderProblem &p, hipStream_t st)
{
    // From how many pairs on counting once, in three launches, takes less time than counting all of them in every workgroup: the three begin at 10 us and grow with the
    // experts' number, the one grows with the pairs'.  us, one | three (random ids, one call after another in a graph; 2^20 pairs of 64, 256 and 1000 experts 123 | 24,
    // 113 | 32, 123 | 58):
    //   pairs     64 experts   128          256          384          512          1024
    //    65536   10.0 | 10.5    9.6 | 10.8   9.5 | 11.1   9.9 | 13.5  10.3 | 13.5  11.9 | 18.9
    //    81920   12.9 | 10.6   12.6 | 10.8  12.2 | 13.0  12.7 | 15.5  13.1 | 15.8  15.4 | 21.7
    //   131072   17.7 | 10.7   16.9 | 11.1  16.1 | 13.6  16.5 | 18.4  16.8 | 18.6  18.8 | 29.0
    //   163840   22.2 | 12.2   21.2 | 12.7  20.2 | 14.9  20.5 | 17.8  20.8 | 18.1  23.1 | 24.2
    //   262144   32.8 | 12.5   31.1 | 13.2  29.1 | 15.8  29.5 | 20.8  30.2 | 21.1  33.2 | 31.7
    const int many = p.E <= 128 ? 1 << 16 : 49152 + 192 * p.E;
    int bits = 0;
    while ((1 << bits) < p.E) ++bits;
    const auto lds = [&](int waves) { return 4u * ((3 * p.E + 4) / 4 * 4) + 2u * waves * p.E; };
    if (p.pairs > many) {
        // segments of whole rounds, each longer than E; the last one has what is left
        const int segment = ((p.pairs + 127) / 128 + 1023) / 1024 * 1024, grid = p.pairs / segment;
        if (const hipError_t e = c2i8::launch(count_pairs_kernel, dim3(grid), dim3(1024), 4u * p.E, st, p, segment)) return e;
        if (const hipError_t e = c2i8::launch(start_rows_kernel, dim3(1), dim3(1024), 0, st, p, segment, grid, bits < 6 ? 64 : 1 << bits)) return e;
        return c2i8::launch(expert_rows_kernel<16, true>, dim3(grid), dim3(1024), lds(16), st, p, segment, bits);
    }
    auto go = [&](auto waves) {
        constexpr int W = waves.value;
        // segments of a workgroup's lanes until there are 64 workgroups, each of which counts every id
        const int segment = ((p.pairs + 63) / 64 + 64 * W - 1) / (64 * W) * (64 * W);
        const int grid = p.pairs ? (p.pairs + segment - 1) / segment : 1;
        return c2i8::launch(expert_rows_kernel<W, false>, dim3(grid), dim3(64 * W), lds(W), st, p, segment, bits);
    };
    if (p.pairs <= 512) return go(std::integral_constant<int, 8>{});
    return go(std::integral_constant<int, 16>{});
}

hipError_t launch_combine(const CombineProblem &p, hipStream_t st)
{
    const int size = size_of(p.type);
    const bool vec = in_pieces(p.y, p.ldy, p.N, size) && in_pieces(p.out, p.ldo, p.N, size);
    return with_type(p.type, [&](auto t) {
        using T = decltype(t);
        constexpr int W = 16 / sizeof(T);
        const int pieces = vec ? p.N / W : p.N;
        const long long blocks = ((long long)p.T * pieces + 255) / 256;
        constexpr long long MOST = 1 << 22;   // workgroups of a launch, 2^30 lanes; larger results take several
        for (long long first = 0; first < blocks; first += MOST) {
            const dim3 grid((unsigned)(blocks - first < MOST ? blocks - first : MOST));
            const hipError_t e = vec ? c2i8::launch(combine_kernel<T, W>, grid, dim3(256), 0, st, p, pieces, (unsigned)first)
                                     : c2i8::launch(combine_kernel<T, 1>, grid, dim3(256), 0, st, p, pieces, (unsigned)first);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
}

hipError_t launch_combine_backward(const CombineProblem &p, hipStream_t st)
{
    const int size = size_of(p.type);
    const bool vec = in_pieces(p.y, p.ldy, p.N, size) && in_pieces(p.dout, p.ldd, p.N, size) && in_pieces(p.dy, p.lddy, p.N, size);
    const long long waves = (long long)p.T * p.k > p.R ? (long long)p.T * p.k : p.R;
    return with_type(p.type, [&](auto t) {
        using T = decltype(t);
        return vec ? c2i8::launch(combine_backward_kernel<T, 16 / sizeof(T)>, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, p)
                   : c2i8::launch(combine_backward_kernel<T, 1>, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, p);
    });
}

}  // namespace xp8
