// Operators on rows of logits for gfx950 (CDNA4): the largest logits of each row, and two losses with their
// gradients: distillation from a teacher's top logits, and the clipped policy loss.
//
// All three read a row of `vocab` logits z once for its softmax statistics, q_j = exp(z_j / tau) / sum, and are bound
// by that read (a few operations and one exponential per logit), the gradient by the read and the write.
//
// Exponents are taken in base 2, with c = float(log2(e) / tau).  A thread keeps a running reference m (the largest z * c it
// has seen, rounded) and s = sum exp2(z * c - m): per logit one fused multiply-add, one exp2 and one addition (and for bf16
// one operation to unpack it).  The sum is f32: 150 thousand positive terms in several hundred partial sums keep its
// relative error below 1e-5 at worst, near 1e-8 in the middle.  What comes after the sums, a few values per row and per
// teacher entry, is in f64, because the losses are small differences of logarithms (a divergence of 1e-3 from logarithms
// near 10 keeps four digits in f32); there the reference counts as m * (c_exact / c), which takes c's rounding back.
// Rows whose products with c do not fit f32 (a mask of the type's lowest value over all of a row) are taken again with
// differences before products, out of the way of the others.
//
// A row is cut into 16-byte vectors on the addresses' own 16-byte grid, so that rows of any stride and start are read
// with aligned wide loads: vector i holds elements [i * W - lead, (i + 1) * W - lead), W = 4 (f32) or 8 (bf16), and the
// partial vectors at both ends are read element by element.
#include "nld_internal.h"

#include <math.h>

#include <algorithm>

namespace nld {
namespace {

constexpr uint32_t DEV_BAD_TOKEN = 0x1u;

template <bool BF>
struct Elem;
template <>
struct Elem<false> {
    typedef float type;
    static constexpr int W = 4;
};
template <>
struct Elem<true> {
    typedef uint16_t type;
    static constexpr int W = 8;
};

template <bool BF>
__device__ __forceinline__ float to_float(typename Elem<BF>::type v) {
    if constexpr (BF) return bf16_to_f32(v);
    else return v;
}
template <bool BF>
__device__ __forceinline__ float load_elem(const typename Elem<BF>::type* p) { return to_float<BF>(*p); }
template <bool BF>
__device__ __forceinline__ void store_elem(typename Elem<BF>::type* p, float v) {
    if constexpr (BF) *p = (uint16_t)f32_to_bf16(v);
    else *p = v;
}
template <bool BF>
__device__ __forceinline__ void unpack(const uint4& v, float* z) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (BF) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            z[2 * q] = __uint_as_float(w[q] << 16);
            z[2 * q + 1] = __uint_as_float(w[q] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) z[q] = __uint_as_float(w[q]);
    }
}

// One row, or a chunk of it, on the 16-byte grid.
template <bool BF>
struct Span {
    typedef typename Elem<BF>::type T;
    static constexpr int W = Elem<BF>::W;
    const T* row;     // element 0
    const T* grid;    // vector 0 (at or before element 0; its elements before 0 are never touched)
    int lead, n;      // elements between grid and row; elements of the row
    int v0, v1;       // this chunk's vectors
    int f0, f1;       // the full ones among them
    __device__ __forceinline__ Span(const LogitRows& a, int r, int chunk, int cv) {
        const int b = r / a.rows, j = r - b * a.rows;
        row = (const T*)a.z + (long long)b * a.seq_stride + (long long)j * a.row_stride;
        lead = (int)(((uintptr_t)row & 15u) / sizeof(T));
        grid = row - lead;
        n = a.vocab;
        const int nv = (lead + n + W - 1) / W;
        v0 = min(chunk * cv, nv);
        v1 = min(v0 + cv, nv);
        f0 = max(v0, lead ? 1 : 0);
        f1 = max(f0, min(v1, (lead + n) / W));
    }
    __device__ __forceinline__ uint4 load(int i) const { return ((const uint4*)grid)[i]; }
    // the elements of a partial vector that lie in the row, -inf for the others
    __device__ __forceinline__ void load_edge(int i, float* z) const {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const int j = i * W + e - lead;
            z[e] = j >= 0 && j < n ? load_elem<BF>(row + j) : -INFINITY;
        }
    }
    __device__ __forceinline__ bool full(int i) const { return i >= f0 && i < f1; }
    // partial vectors of this chunk: at most one before f0 and one from f1 on
    __device__ __forceinline__ int n_edges() const { return (f0 - v0) + (v1 - f1); }
    __device__ __forceinline__ int edge(int k) const { return k < f0 - v0 ? v0 + k : f1 + (k - (f0 - v0)); }
};

// a value that every lane holds alike, in scalar registers: rows are held in the vector registers meanwhile
__device__ __forceinline__ float uniform(float v) {
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v)));
}
__device__ __forceinline__ double uniform(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}

// z / tau * log2(e), rounded: equal logits of any size have a difference of 0, which a product fused into the difference
// would not give (rows of the type's lowest value)
__device__ __forceinline__ double base2(float z, double c_exact) {
#pragma clang fp contract(off)
    return (double)z * c_exact;
}

// Reductions over a wavefront by cross-lane moves of the vector unit (an LDS permute takes several times as long, and these
// stand one after the other at the end of every row): within rows of 16 lanes by shifts of 1, 2, 4 and 8, then lane 15 of
// a row into the next one and lane 31 into the upper half; lane 63 has the whole.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_move(uint32_t none, uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS, class T>
__device__ __forceinline__ T lane_from(T none, T v) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, lane_move<CTRL, ROWS>(__builtin_bit_cast(uint32_t, none), __builtin_bit_cast(uint32_t, v)));
    } else {
        const uint2 n = __builtin_bit_cast(uint2, none), x = __builtin_bit_cast(uint2, v);
        return __builtin_bit_cast(T, uint2{lane_move<CTRL, ROWS>(n.x, x.x), lane_move<CTRL, ROWS>(n.y, x.y)});
    }
}
template <class T>
__device__ __forceinline__ T lane63(T v) {
    if constexpr (sizeof(T) == 4) {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
    } else {
        const uint2 x = __builtin_bit_cast(uint2, v);
        return __builtin_bit_cast(T, uint2{(uint32_t)__builtin_amdgcn_readlane((int)x.x, 63), (uint32_t)__builtin_amdgcn_readlane((int)x.y, 63)});
    }
}
// op over all lanes, in every lane; none: op's neutral value
template <class T, class Op>
__device__ __forceinline__ T wave_reduce(T v, T none, const Op& op) {
    v = op(v, lane_from<0x111, 0xF>(none, v));
    v = op(v, lane_from<0x112, 0xF>(none, v));
    v = op(v, lane_from<0x114, 0xF>(none, v));
    v = op(v, lane_from<0x118, 0xF>(none, v));
    v = op(v, lane_from<0x142, 0xA>(none, v));
    v = op(v, lane_from<0x143, 0xC>(none, v));
    return lane63(v);
}
template <class T>
__device__ __forceinline__ T wave_sum(T v) {
    return wave_reduce(v, (T)0, [](T a, T b) __attribute__((always_inline)) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {
    return wave_reduce(v, -INFINITY, [](float a, float b) __attribute__((always_inline)) { return fmaxf(a, b); });
}
__device__ __forceinline__ double wave_max(double v) {
    return wave_reduce(v, -(double)INFINITY, [](double a, double b) __attribute__((always_inline)) { return fmax(a, b); });
}

// ---------------------------------------------------------------- softmax statistics
struct Stat {
    float m, s;   // reference and sum of exp2(z * c - m)
};
constexpr float STAT_EMPTY = -3.0e38f;   // the reference of no logit: finite, so that -inf adds nothing to a sum of it
// adds N logits and returns the largest of them; NaN, +inf or a product past f32 among them makes the sum NaN
template <int N>
__device__ __forceinline__ float stat_add(Stat& t, const float* z, float c) {
    float top = z[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, z[e]);
    const float m = top * c;
    if (m > t.m) {
        t.s *= __builtin_amdgcn_exp2f(t.m - m);
        t.m = m;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) t.s += __builtin_amdgcn_exp2f(fmaf(z[e], c, -t.m));
    return top;
}
// the same with differences first: m is the largest logit itself (-inf: none yet), s = sum of exp2((z - m) * c)
__device__ __forceinline__ Stat wide_merge(Stat a, Stat b, float c) {
    Stat o;
    o.m = fmaxf(a.m, b.m);
    const float ref = o.m == -INFINITY ? 0.f : o.m;   // both empty: the sums are 0 (or NaN, which stays)
    o.s = a.s * __builtin_amdgcn_exp2f((a.m - ref) * c) + b.s * __builtin_amdgcn_exp2f((b.m - ref) * c);
    return o;
}

// every thread's statistics -> the workgroup's, in every thread, and the same of the maximum *top (optional); red: two
// times NT / 64 pairs.  WIDE: as wide_merge takes them.
template <int NT, bool WIDE>
__device__ __forceinline__ Stat stat_block(Stat t, Stat* red, float c, float* top) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the largest reference first, then every sum is scaled once
    auto all = [&](Stat x) __attribute__((always_inline)) {
        const float m = wave_max(x.m), ref = WIDE && m == -INFINITY ? 0.f : m;
        return Stat{m, wave_sum(x.s * __builtin_amdgcn_exp2f(WIDE ? (x.m - ref) * c : x.m - ref))};
    };
    t = all(t);
    if (top) *top = wave_max(*top);
    __syncthreads();
    if (lane == 0) {
        red[wave] = t;
        if (top) red[NT / 64 + wave].m = *top;
    }
    __syncthreads();
    t = all(lane < NT / 64 ? red[lane] : Stat{WIDE ? -INFINITY : STAT_EMPTY, 0.f});
    if (top) *top = wave_max(lane < NT / 64 ? red[NT / 64 + lane].m : -INFINITY);
    return t;
}

// The statistics of a row or a chunk of it: sum of exp2(z / tau * log2(e) - ref) = s.
typedef ChunkStat RowStat;
constexpr float WIDE_FROM = 1e8f;
// From every thread's share; `again` takes the thread's logits once more, by wide_merge of Stat{z, 1}, where products with c
// do not fit f32 or are so large that their rounding costs many binary orders.
template <int NT, class Again>
__device__ __forceinline__ RowStat row_stat(Stat t, Stat* red, float c, double c_exact, float* top, const Again& again) {
    t = stat_block<NT, false>(t, red, c, top);
    if (t.s > 0.f && t.s < INFINITY && fabsf(t.m) < WIDE_FROM) return RowStat{uniform((double)t.m * (c_exact / (double)c)), t.s};
    t = stat_block<NT, true>(again(), red, c, nullptr);
    return RowStat{t.m == -INFINITY ? 0.0 : uniform(base2(t.m, c_exact)), t.s};
}
// all chunks of row r, in every thread: a lane takes every 64th chunk, then the wavefront's lanes are added in a tree
__device__ __forceinline__ RowStat merge_chunks(const ChunkStat* part, int r, int chunks) {
    const int lane = threadIdx.x & 63;
    const ChunkStat* p = part + (long long)r * chunks;
    double ref = -(double)INFINITY;
    for (int c = lane; c < chunks; c += 64)
        if (p[c].s != 0.f) ref = fmax(ref, p[c].ref);
    ref = wave_max(ref);
    if (ref == -(double)INFINITY) ref = 0.0;   // nothing anywhere
    double s = 0.0;
    for (int c = lane; c < chunks; c += 64)
        if (p[c].s != 0.f) s += (double)p[c].s * exp2(p[c].ref - ref);
    return RowStat{ref, uniform((float)wave_sum(s))};
}
// log2 of the sum of exp(z / tau)
__device__ __forceinline__ double stat_log2(RowStat t) { return t.s == 0.f ? -(double)INFINITY : t.ref + log2((double)t.s); }

// ---------------------------------------------------------------- the largest logits of a row
// Order-preserving key of a logit at column n: larger value first, then lower column; -0.0 counts as +0.0 and a NaN
// of either sign stands above +inf.
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t u = __float_as_uint(v + 0.f);
    if (v != v) return 0xFFFFFFFFu;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t ord) {
    return __uint_as_float((ord & 0x80000000u) ? (ord & 0x7FFFFFFFu) : ~ord);   // 0xFFFFFFFF: a NaN
}
__device__ __forceinline__ unsigned long long key_of(uint32_t ord, int n) {
    return ((unsigned long long)ord << 32) | (unsigned long long)(0xFFFFFFFFu - (uint32_t)n);
}
constexpr uint32_t ORD_POS_INF = 0xFF800000u, ORD_NEG_INF = 0x007FFFFFu;

constexpr int TOP_SEGS = 16;     // a thread's vectors are cut into at most this many segments, each with its maximum
constexpr int TOP_AHEAD = 4;     // vectors requested at once; a segment is a multiple of it
constexpr int TOP_CAND = 2048;   // candidates that one ranking holds

template <int NT>
struct TopShared {
    uint16_t seg[TOP_SEGS][NT];          // largest key of each thread's segments, its upper half
    uint16_t hits[4 * NT];               // segments that may hold one of the largest
    alignas(16) unsigned long long cand[TOP_CAND];
    alignas(16) uint32_t hist[256];
    Stat red[2 * NT / 64];
    uint32_t lo[NT / 64], hi[NT / 64];
    int n_hits, n_cand;
};

// The highest of 256 bins from which on there are at least k (hist), in every wavefront alike: *from: the count from it on,
// *past: from the next one on.  -1: there are not so many.
__device__ __forceinline__ int bin_from_top(const uint32_t* hist, int k, int* from, int* past) {
    const int lane = threadIdx.x & 63;
    const uint4 h = ((const uint4*)hist)[63 - lane];   // lane 0: the last four bins
    int n[4] = {(int)h.w, (int)h.z, (int)h.y, (int)h.x};
    n[1] += n[0];
    n[2] += n[1];
    n[3] += n[2];
    int before = n[3];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int o = __shfl_up(before, off);
        before += lane >= off ? o : 0;
    }
    before -= n[3];   // in the bins of the lanes below
    const unsigned long long reach = __ballot(before + n[3] >= k);
    if (reach == 0ull) return -1;
    const int l = __ffsll((long long)reach) - 1;
    int q = 3;
#pragma unroll
    for (int i = 2; i >= 0; --i) q = before + n[i] >= k ? i : q;
    const int here = before + (q == 0 ? n[0] : q == 1 ? n[1] : q == 2 ? n[2] : n[3]);
    const int prev = before + (q == 0 ? 0 : q == 1 ? n[0] : q == 2 ? n[1] : n[2]);
    *from = __shfl(here, l);
    *past = __shfl(prev, l);
    return 255 - 4 * l - __shfl(q, l);
}

// A key that at least k threads' maxima reach, and not many more: the keys from the least to the largest are cut into 256
// bins, and the bin of the k-th again while it holds many more than are wanted.  0 when fewer than k threads have
// anything.  At least k elements of the row reach it, so the k largest all do.
template <int NT>
__device__ __forceinline__ uint32_t bound_below(uint32_t mine, int k, TopShared<NT>& sh) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t lo = mine ? mine : 0xFFFFFFFFu, hi = mine;
    auto least = [](uint32_t a, uint32_t b) __attribute__((always_inline)) { return min(a, b); };
    auto most = [](uint32_t a, uint32_t b) __attribute__((always_inline)) { return max(a, b); };
    lo = wave_reduce(lo, 0xFFFFFFFFu, least);
    hi = wave_reduce(hi, 0u, most);
    if (lane == 0) {
        sh.lo[wave] = lo;
        sh.hi[wave] = hi;
    }
    if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0u;
    __syncthreads();
    lo = wave_reduce(sh.lo[lane & (NT / 64 - 1)], 0xFFFFFFFFu, least);
    hi = wave_reduce(sh.hi[lane & (NT / 64 - 1)], 0u, most);
    int above = 0;   // threads beyond hi
    while (lo <= hi) {
        const int shift = max(0, 24 - __clz((int)(hi - lo)));
        if (mine >= lo && mine <= hi) atomicAdd(&sh.hist[(mine - lo) >> shift], 1u);
        __syncthreads();
        int from = 0, past = 0;
        const int bin = bin_from_top(sh.hist, k - above, &from, &past);
        if (bin < 0) return 0u;
        const uint32_t bound = lo + ((uint32_t)bin << shift);
        if (shift == 0 || above + from <= k + (k >> 2) + 8) return bound;
        above += past;
        lo = bound;
        hi = bound + min(hi - bound, (1u << shift) - 1u);
        __syncthreads();
        if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0u;
        __syncthreads();
    }
    return 0u;
}

// The k largest of n distinct keys, whatever their order and ties: radix selection from the top byte down, each byte
// one pass over the keys.  Leaves them in sh.cand (any order).  For rows whose bound lets too many candidates through
// (many equal logits, a vocabulary masked down to few tokens, NaN).
template <int NT, class Keys>
__device__ void select_exact(const Keys& key, int n, int k, TopShared<NT>& sh) {
    unsigned long long prefix = 0ull;
    int need = k;
    int shift = 56;
    for (; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0u;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += NT) {
            const unsigned long long x = key(i);
            const bool in = shift == 56 || (x >> (shift + 8)) == prefix;
            const int d = (int)((x >> shift) & 255u);
            // equal logits share their digits: lanes that agree with the first one count once
            const unsigned long long act = __ballot(in);
            if (act == 0ull) continue;
            const int d0 = __shfl(d, __ffsll((long long)act) - 1);
            const unsigned long long same = __ballot(in && d == d0);
            if (in && d != d0) atomicAdd(&sh.hist[d], 1u);
            if ((threadIdx.x & 63) == __ffsll((long long)act) - 1) atomicAdd(&sh.hist[d0], (uint32_t)__popcll(same));
        }
        __syncthreads();
        int from = 0, past = 0;
        const int digit = max(bin_from_top(sh.hist, need, &from, &past), 0);
        const int in_bin = (int)sh.hist[digit];
        need -= past;
        prefix = (prefix << 8) | (unsigned long long)digit;
        if (in_bin == need) break;   // the whole bin belongs to the k largest
    }
    const unsigned long long least = prefix << (shift < 0 ? 0 : shift);
    __syncthreads();
    if (threadIdx.x == 0) sh.n_cand = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
        const unsigned long long x = key(i);
        if (x >= least) {
            const int at = atomicAdd(&sh.n_cand, 1);
            if (at < TOP_CAND) sh.cand[at] = x;
        }
    }
    __syncthreads();
}

// Ranks the n candidates (distinct keys) by counting, for each, the larger ones, and hands those of rank < k to
// `emit(rank, key)`.  SHARE threads count for a candidate, each AT keys at once; places past the last one are filled up
// with keys below all.
template <int NT, class Emit>
__device__ __forceinline__ void rank_candidates(int n, int k, TopShared<NT>& sh, const Emit& emit) {
    constexpr int AT = 8, SHARE = 8;
    static_assert(TOP_CAND % (AT * SHARE) == 0, "room to fill up");
    const int filled = (n + AT * SHARE - 1) / (AT * SHARE) * (AT * SHARE);
    if (n + (int)threadIdx.x < filled) sh.cand[n + threadIdx.x] = 0ull;
    __syncthreads();
    for (int c0 = 0; c0 < n; c0 += NT / SHARE) {
        const int c = c0 + (int)threadIdx.x / SHARE, part = (int)threadIdx.x & (SHARE - 1);
        const unsigned long long mine = c < n ? sh.cand[c] : 0ull;
        int rank = 0;
        for (int j = part; j < filled; j += AT * SHARE) {
            unsigned long long x[AT];
#pragma unroll
            for (int u = 0; u < AT; ++u) x[u] = sh.cand[j + u * SHARE];
#pragma unroll
            for (int u = 0; u < AT; ++u) rank += x[u] > mine ? 1 : 0;
        }
#pragma unroll
        for (int off = SHARE >> 1; off >= 1; off >>= 1) rank += __shfl_xor(rank, off);
        if (c < n && part == 0 && rank < k) emit(rank, mine);
    }
}

template <bool BF>
struct RowKeys {   // a chunk of a row, element by element
    const Span<BF>& sp;
    int e0;
    __device__ __forceinline__ unsigned long long operator()(int i) const {
        return key_of(order_of(load_elem<BF>(sp.row + e0 + i)), e0 + i);
    }
};
struct ListKeys {
    const unsigned long long* p;
    __device__ __forceinline__ unsigned long long operator()(int i) const { return p[i]; }
};

__device__ __forceinline__ void emit_top(const TopArgs& a, int r, int rank, unsigned long long key) {
    const uint32_t ord = (uint32_t)(key >> 32);
    a.values[(long long)r * a.n_top + rank] = value_of(ord);
    a.ids[(long long)r * a.n_top + rank] = (int32_t)(0xFFFFFFFFu - (uint32_t)key);
}
// the row's log-sum-exp, from the largest key and the statistics (whose sum is NaN where +inf or NaN took part)
__device__ __forceinline__ float lse_of(RowStat t, uint32_t top) {
    if (top == 0xFFFFFFFFu) return NAN;
    if (top == ORD_POS_INF) return INFINITY;
    if (top == ORD_NEG_INF) return -INFINITY;
    return (float)(stat_log2(t) * 0.69314718055994530942);
}

// One pass over the row for the statistics and for the maximum of every thread's segments; then a lower bound of the
// k-th largest from the threads' maxima; then a second look at the few segments that reach it (about k of some
// thousands, a few per cent of the row, which the first pass left in L2 or the memory-side cache); then the candidates
// are ranked.
template <bool BF, int NT>
__global__ void __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(8))) top_kernel(TopArgs a) {
    constexpr int W = Elem<BF>::W;
    __shared__ TopShared<NT> sh;
    const int r = blockIdx.x / a.plan.chunks, chunk = blockIdx.x % a.plan.chunks, tid = threadIdx.x;
    const Span<BF> sp(a.in, r, chunk, a.plan.cv);
    const int nf = sp.f1 - sp.f0, iters = (nf + NT - 1) / NT;   // full vectors of the chunk, and of a thread
    const int len = (iters + TOP_SEGS * TOP_AHEAD - 1) / (TOP_SEGS * TOP_AHEAD) * TOP_AHEAD;   // vectors per segment
    const int segs = len ? (iters + len - 1) / len : 0;
    if (tid == 0) {
        sh.n_hits = 0;
        sh.n_cand = 0;
    }
    Stat part{STAT_EMPTY, 0.f};
    float best_z = -INFINITY;
    bool any = false;
    float edge[W];
    if (tid < sp.n_edges()) {
        sp.load_edge(sp.edge(tid), edge);
        best_z = stat_add<W>(part, edge, a.c);
        any = true;
    }
    for (int s = 0; s < segs; ++s) {
        float top = -INFINITY;
        for (int u0 = 0; u0 < len; u0 += TOP_AHEAD) {
            const int i0 = tid + (s * len + u0) * NT;   // among the full vectors
            uint4 v[TOP_AHEAD];
#pragma unroll
            for (int u = 0; u < TOP_AHEAD; ++u) v[u] = load_stream((const uint4*)sp.grid + sp.f0 + min(i0 + u * NT, nf - 1));
#pragma unroll
            for (int u = 0; u < TOP_AHEAD; ++u)
                if (i0 + u * NT < nf) {
                    float z[W];
                    unpack<BF>(v[u], z);
                    top = fmaxf(top, stat_add<W>(part, z, a.c));
                    any = true;
                }
        }
        sh.seg[s][tid] = tid + s * len * NT < nf ? (uint16_t)(order_of(top) >> 16) : (uint16_t)0;
        best_z = fmaxf(best_z, top);
    }
    const RowStat st = row_stat<NT>(part, sh.red, a.c, a.c_exact, nullptr, [&]() {
        Stat t{-INFINITY, 0.f};
        for (int i = sp.v0 + tid; i < sp.v1; i += NT) {
            float z[W];
            if (sp.full(i)) unpack<BF>(sp.load(i), z);
            else sp.load_edge(i, z);
#pragma unroll
            for (int e = 0; e < W; ++e) t = wide_merge(t, Stat{z[e], 1.f}, a.c);
        }
        return t;
    });
    const int e0 = max(0, sp.v0 * W - sp.lead), e1 = min(sp.n, sp.v1 * W - sp.lead), n = max(0, e1 - e0);
    const int k = min(a.n_top, n);
    bool exact = !(st.s < INFINITY);   // NaN or +inf: the maxima above do not order these
    if (!exact) {
        const uint32_t bound = bound_below(any ? order_of(best_z) : 0u, k, sh);
        auto take = [&](const float* z, int i) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const int j = i * W + e - sp.lead;
                const uint32_t o = order_of(z[e]);
                if (o >= bound && j >= 0 && j < sp.n) {
                    const int at = atomicAdd(&sh.n_cand, 1);
                    if (at < TOP_CAND) sh.cand[at] = key_of(o, j);
                }
            }
        };
        __syncthreads();
        if (tid < sp.n_edges()) take(edge, sp.edge(tid));
        for (int s = 0; s < segs; ++s)
            if (sh.seg[s][tid] != 0u && sh.seg[s][tid] >= bound >> 16) {
                const int at = atomicAdd(&sh.n_hits, 1);
                if (at < 4 * NT) sh.hits[at] = (uint16_t)(s * NT + tid);
            }
        __syncthreads();
        const int items = min(sh.n_hits, 4 * NT) * len;
        for (int it = tid; it < items; it += TOP_AHEAD * NT) {
            int at[TOP_AHEAD];
            uint4 v[TOP_AHEAD];
#pragma unroll
            for (int u = 0; u < TOP_AHEAD; ++u) {
                const int x = it + u * NT, h = x < items ? sh.hits[x / len] : 0;
                at[u] = x < items ? h % NT + (h / NT * len + x % len) * NT : nf;
                v[u] = sp.load(sp.f0 + min(at[u], nf - 1));
            }
#pragma unroll
            for (int u = 0; u < TOP_AHEAD; ++u)
                if (at[u] < nf) {
                    float z[W];
                    unpack<BF>(v[u], z);
                    take(z, sp.f0 + at[u]);
                }
        }
        __syncthreads();
        exact = sh.n_cand > TOP_CAND || sh.n_hits > 4 * NT;
    }
    if (exact) select_exact(RowKeys<BF>{sp, e0}, n, k, sh);
    const int nc = sh.n_cand;
    if (a.plan.chunks == 1) {
        rank_candidates(nc, k, sh, [&](int rank, unsigned long long key) {
            emit_top(a, r, rank, key);
            if (rank == 0 && a.lse) a.lse[r] = lse_of(st, (uint32_t)(key >> 32));
        });
    } else {
        // the merge does not mind their order, so that only more candidates than there are places are ranked
        const int places = top_places(a.n_top);
        unsigned long long* out = a.keys + ((long long)r * a.plan.chunks + chunk) * places;
        if (nc <= places) {
            for (int i = tid; i < places; i += NT) out[i] = i < nc ? sh.cand[i] : 0ull;
        } else {
            for (int i = k + tid; i < places; i += NT) out[i] = 0ull;
            rank_candidates(nc, k, sh, [&](int rank, unsigned long long key) { out[rank] = key; });
        }
        if (tid == 0) a.part[(long long)r * a.plan.chunks + chunk] = st;
    }
}

// The chunks' largest keys -> the row's.  As many as MERGE_HELD per thread are read once, side by side.
constexpr int MERGE_HELD = 8;
__global__ void __launch_bounds__(1024) top_merge_kernel(TopArgs a) {
    constexpr int NT = 1024;
    __shared__ TopShared<NT> sh;
    const int r = blockIdx.x, tid = threadIdx.x, n = a.plan.chunks * top_places(a.n_top);
    const ListKeys key{a.keys + (long long)r * n};
    if (tid == 0) sh.n_cand = 0;
    unsigned long long held[MERGE_HELD];
    uint32_t best = 0u;
#pragma unroll
    for (int u = 0; u < MERGE_HELD; ++u) held[u] = tid + u * NT < n ? key(tid + u * NT) : 0ull;
#pragma unroll
    for (int u = 0; u < MERGE_HELD; ++u) best = max(best, (uint32_t)(held[u] >> 32));
    for (int i = tid + MERGE_HELD * NT; i < n; i += NT) best = max(best, (uint32_t)(key(i) >> 32));
    const RowStat st = merge_chunks(a.part, r, a.plan.chunks);
    const uint32_t bound = max(bound_below(best, a.n_top, sh), 1u);   // 0: an empty place
    auto take = [&](unsigned long long x) __attribute__((always_inline)) {
        if ((uint32_t)(x >> 32) < bound) return;
        const int at = atomicAdd(&sh.n_cand, 1);
        if (at < TOP_CAND) sh.cand[at] = x;
    };
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MERGE_HELD; ++u) take(held[u]);
    for (int i = tid + MERGE_HELD * NT; i < n; i += NT) take(key(i));
    __syncthreads();
    if (sh.n_cand > TOP_CAND) select_exact(key, n, a.n_top, sh);
    rank_candidates(sh.n_cand, a.n_top, sh, [&](int rank, unsigned long long x) {
        emit_top(a, r, rank, x);
        if (rank == 0 && a.lse) a.lse[r] = lse_of(st, (uint32_t)(x >> 32));
    });
}

// ---------------------------------------------------------------- losses with their gradients
// Both losses see a row as its entries (the teacher's tokens; the action) and the rest of the vocabulary:
//   statistics   (m, s) over the rest, the entries apart, so that neither a rest that has next to nothing nor an entry
//                that has next to all loses its digits in a difference from the row's sum;
//   row values   in f64 from the entries' logits and (m, s): the loss, and the coefficients of the gradient, which is
//                the column's share of the rest times one number for every column outside the entries, and a value of its
//                own for each entry;
//   gradient     one more pass over the row.
constexpr int LOSS_NT = TOP_MAX;   // threads: at least one per teacher entry

template <int NT>
struct LossShared {
    Stat red[2 * NT / 64];
    double sum[5][TOP_MAX / 64][2];   // the entries' sums, one place for each of a row's reductions
    double rest;                      // RowGrad's, from the wavefronts that work it out
    int none;
    int32_t ids[TOP_MAX];
    uint32_t mark[NT];   // per thread: which of its held vectors have an entry among their columns
    int repeated;
};

// The values of a row, all in f64, are worked out by the wavefronts that have teacher entries (n_top threads), while the
// others wait: with all of them at it, each with the row's values, the few vector units would do the same work many times
// (2.7 us of a row on 16 wavefronts).  A reduction over the entries: post_sums in these wavefronts, meet in all, take_sums in
// these again.
template <int NT>
struct Entries {
    const int waves, wave, lane;
    LossShared<NT>& sh;
    __device__ __forceinline__ Entries(int n_top, LossShared<NT>& s)
        : waves((n_top + 63) >> 6), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63), sh(s) {}
    __device__ __forceinline__ bool here() const { return wave < waves; }
    template <int N, bool MAX>
    __device__ __forceinline__ void post(double* v, int slot) const {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = MAX ? wave_max(v[i]) : wave_sum(v[i]);
        if (waves > 1 && lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) sh.sum[slot][wave][i] = v[i];
    }
    __device__ __forceinline__ void meet() const {
        if (waves > 1) __syncthreads();
    }
    template <int N, bool MAX>
    __device__ __forceinline__ void take(double* v, int slot) const {
        if (waves == 1) return;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = sh.sum[slot][0][i];
#pragma unroll 1   // one at a time: the row is held in registers meanwhile
        for (int w = 1; w < waves; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = MAX ? fmax(v[i], sh.sum[slot][w][i]) : v[i] + sh.sum[slot][w][i];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = uniform(v[i]);
    }
};

// What a row's gradient needs: a column outside the entries gets its share of the rest, exp2(z / tau * log2(e) - ref) / s,
// times `rest`; `entry` is what this thread's entry gets.
struct RowGrad {
    RowStat st;
    double rest;
    float entry;
    bool none;   // the gradient is zero throughout
};

// Distillation.  p: the teacher's probabilities of its entries and, with its log-sum-exp given, of everything else (the
// rest, R); q: the student's.
//   loss = w (lambda KL + (1 - lambda) TV),  KL = sum p log(p / q),  TV = 1/2 sum |p - q|,
//   lambda = kl_share exp(-eta alpha), alpha = sum min(p, q), held constant in the gradient;
//   d loss / d z_j = w / tau (q_j (lambda P + (1 - lambda) / 2 (s_j - mean)) - lambda p_j) for an entry, with P = sum p,
//   s = sign(q - p), mean = sum s q, all sums over entries and rest, and in the rest, where every q_j has the same share
//   of what the rest gets, w / tau q_j (lambda P + (1 - lambda) / 2 (s_R - mean) - lambda p_R / q_R).
// KL is taken as sum p log p - sum p y + P log(sum of the student's exponentials), y = z / tau, so that all of the teacher's side is
// done while the row is on its way, and TV as (P + 1) / 2 - alpha.

// The teacher's side: this thread's p, and for the row the sums (base-2 logarithms) over entries and rest; in the
// wavefronts with entries, and its first half.
struct Teacher {
    double p, entries, rest, plogp;   // plogp: without the rest's
    double slack;   // what the rounding of an f32 log-sum-exp can leave of 1 - sum p
    bool none;      // no token at all
    bool tail;      // the log-sum-exp is given, and counts
};
// A log-sum-exp of this size is rounded to f32 by half a unit and more, so that it says nothing of the entries.  At or below
// -LSE_ROUNDED it is that of a row masked throughout by a finite value, and counts as -inf; from LSE_ROUNDED on the entries
// alone are the teacher, as where none is given.
constexpr float LSE_ROUNDED = (float)(1 << 24);
template <int NT>
__device__ __forceinline__ Teacher teacher_side(const LossArgs& a, float t, float t_lse, bool counts, LossShared<NT>& sh) {
    const Entries<NT> en(a.n_top, sh);
    const double none = -(double)INFINITY;
    const double x = counts ? base2(t, a.c_exact) : none;
    double lse = none, more = 0.0;   // the log-sum-exp in two parts: beside a large one the other would be lost
    t_lse = uniform(t_lse);
    const bool tail = a.lse && !(t_lse >= LSE_ROUNDED && t_lse < INFINITY);
    if (tail) {
        lse = t_lse <= -LSE_ROUNDED ? none : uniform((double)t_lse * 1.44269504088896340736);
    } else {
        double top[1] = {x}, tot[1] = {0.0};
        if (en.here()) en.template post<1, true>(top, 0);
        en.meet();
        if (en.here()) {
            en.template take<1, true>(top, 0);
            tot[0] = x == none ? 0.0 : exp2(x - top[0]);
            en.template post<1, false>(tot, 1);
        }
        en.meet();
        if (en.here()) {
            en.template take<1, false>(tot, 1);
            lse = tot[0] == 0.0 ? none : top[0];
            more = uniform(log2(tot[0]));
        }
    }
    Teacher o{0.0, 0.0, 0.0, 0.0, fabs(lse) * (0.69314718055994530942 / (1 << 24)) + 1.0 / (1 << 22), lse == none, tail};
    if (en.here()) {
        const double log_p = x - lse - more;
        o.p = x == none ? 0.0 : exp2(log_p);
        double sums[2] = {o.p + 0.0 * lse, o.p > 0.0 ? o.p * log_p : 0.0};   // an infinite lse, or NaN, of no entry too
        en.template post<2, false>(sums, 2);
        o.entries = sums[0];
        o.plogp = sums[1];
    }
    return o;
}
// and the second half of it, with a barrier between: the statistics have some, and the wavefronts without entries need not
// wait for one before them.  whole: the entries are every column.
template <int NT>
__device__ __forceinline__ void teacher_sums(const LossArgs& a, Teacher& o, bool whole, const Entries<NT>& en) {
    double sums[2] = {o.entries, o.plogp};
    en.template take<2, false>(sums, 2);
    o.entries = sums[0];
    o.rest = o.tail && !whole ? uniform(fmax(0.0, 1.0 - sums[0])) : 0.0;
    o.plogp = sums[1];
    if (!(sums[0] < (double)INFINITY)) o.entries = o.plogp = (double)NAN;
}

// The rest: every thread with its entry's logit z, the statistics of the columns outside the entries, and the largest
// logit among the entries.
template <int NT>
__device__ __forceinline__ RowGrad distill_row(const LossArgs& a, int r, Teacher t, bool counts, bool whole, float z, float z_top,
                                               RowStat st, double weight, LossShared<NT>& sh) {
    const Entries<NT> en(a.n_top, sh);
    double ref = 0.0, er = 0.0, ey = 0.0, q = 0.0, q_rest = 0.0, sgn = 0.0, total = 0.0;
    double sums[2] = {0.0, 0.0}, both[2] = {0.0, 0.0};
    if (en.here()) {
        teacher_sums<NT>(a, t, whole, en);
        const double y_top = uniform(base2(z_top, a.c_exact));   // -inf: no entry has a probability
        ref = st.s == 0.f ? (z_top == -INFINITY ? 0.0 : y_top) : uniform(fmax(st.ref, y_top));
        er = st.s == 0.f ? 0.0 : uniform((double)st.s * exp2(st.ref - ref));
        const double y = base2(z, a.c_exact) - ref;
        ey = counts ? exp2(y) : 0.0;
        sums[0] = ey;
        sums[1] = t.p > 0.0 ? t.p * y : 0.0;
        en.template post<2, false>(sums, 3);
    }
    en.meet();
    if (en.here()) {
        en.template take<2, false>(sums, 3);
        total = er + sums[0];
        const double inv = uniform(1.0 / total);
        q = ey * inv;
        q_rest = uniform(er * inv);
        sgn = q > t.p ? 1.0 : (q < t.p ? -1.0 : 0.0);
        both[0] = q == q && t.p == t.p ? fmin(t.p, q) : q + t.p;
        both[1] = sgn * q;
        en.template post<2, false>(both, 4);
    }
    en.meet();
    float entry = 0.f;
    if (en.here()) {
        en.template take<2, false>(both, 4);
        const bool none = t.none || total == 0.0;   // a teacher or a student without any token: nothing to learn
        // Teacher and student masked down to the same tokens: what rounding left of the teacher's rest is no rest
        if (q_rest == 0.0 && t.rest <= t.slack) t.rest = 0.0;
        const double log_total = uniform(log2(total)), rest_y = st.s == 0.f ? -(double)INFINITY : uniform(st.ref - ref + log2((double)st.s));
        const double mass = t.entries + t.rest;
        const double kl = (t.plogp - sums[1] + (t.rest > 0.0 ? t.rest * (log2(t.rest) - rest_y) : 0.0) + mass * log_total) * 0.69314718055994530942;
        const double alpha = mass < (double)INFINITY ? both[0] + (q_rest == q_rest ? fmin(t.rest, q_rest) : q_rest) : (double)NAN;
        const double tv = 0.5 * (mass + 1.0) - alpha;
        const double lambda = uniform((double)a.kl_share * exp2(-(double)a.eta * 1.44269504088896340736 * alpha));
        const double s_rest = q_rest > t.rest ? 1.0 : (q_rest < t.rest ? -1.0 : 0.0);
        const double mean = both[1] + s_rest * q_rest, half = 0.5 * (1.0 - lambda), f = weight * a.inv_tau;
        entry = (float)(f * (q * (lambda * mass + half * (sgn - mean)) - lambda * t.p));
        if (threadIdx.x == 0) {
            a.loss[r] = none ? 0.f : (float)(weight * ((lambda > 0.0 ? lambda * kl : 0.0) + (1.0 - lambda) * tv));
            if (a.aux) a.aux[r] = none ? 0.f : (float)alpha;
            sh.rest = f * (q_rest * (lambda * mass + half * (s_rest - mean)) - lambda * t.rest);
            sh.none = none;
        }
    }
    __syncthreads();
    return RowGrad{st, uniform(sh.rest), entry, sh.none != 0};
}

// Clipped policy loss of the action's log-probability.  rho = exp(logp - old),
//   loss = w (-min(rho A, clip(rho, 1 - low, 1 + high) A) + beta (exp(d) - d - 1)),  d = ref - logp,
//   d loss / d logp = w (-[rho A is the minimum] rho A + beta (1 - exp(d))),  d logp / d z_j = ([j = action] - q_j) / tau.
// With the action apart, 1 - q of a likely action is the rest's share itself.
struct Rollout {
    float advantage, old_logp, ref_logp;
};
template <int NT>
__device__ __forceinline__ RowGrad policy_row(const LossArgs& a, int r, const Rollout& in, float z, RowStat st, double weight,
                                              LossShared<NT>& sh) {
    float entry = 0.f;
    if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) == 0) {   // one wavefront, as above
        const double y = base2(z, a.c_exact), y_rest = st.s == 0.f ? -(double)INFINITY : st.ref, ref = uniform(fmax(y_rest, y));
        const bool none = ref == -(double)INFINITY && z == z;   // no token is possible
        const double er = uniform((double)st.s * exp2(y_rest - ref)), ey = uniform(exp2(y - ref)), all = uniform(er + ey);
        // log(ey / all), by the rest's share where that is the small part
        const double logp = ey >= er ? -log1p(er / ey) : (y - ref) * 0.69314718055994530942 - log(all);
        const double adv = in.advantage;
        const double rho = a.old_logp ? exp(logp - (double)in.old_logp) : (logp == logp ? 1.0 : logp);
        const double free_ = adv == 0.0 && rho == rho ? 0.0 : rho * adv;   // also of an infinite ratio
        const double held = fmin(fmax(rho, 1.0 - (double)a.clip_low), 1.0 + (double)a.clip_high) * adv;
        double loss = free_ <= held ? -free_ : (free_ > held ? -held : (double)NAN);
        double dl = free_ <= held ? -free_ : (free_ > held ? 0.0 : (double)NAN);
        if (a.ref_logp && a.kl_coef > 0.f) {
            const double d = (double)in.ref_logp - logp, beta = a.kl_coef, e = expm1(d);
            loss += beta * (d == (double)INFINITY ? d : e - d);
            dl -= beta * e;
        }
        const double f = weight * a.inv_tau * dl;
        entry = (float)(f * (er / all));
        if (threadIdx.x == 0) {
            a.loss[r] = none ? 0.f : (float)(weight * loss);
            if (a.aux) a.aux[r] = none ? 0.f : (float)logp;
            sh.rest = -f * (er / all);
            sh.none = none || f == 0.0;   // 0: clipped
        }
    }
    __syncthreads();
    return RowGrad{st, uniform(sh.rest), entry, sh.none != 0};
}

// What a row's loss needs besides its logits, requested at once: the loads of the logits follow them, and what was
// asked for later would be waited for together with these.
struct RowInputs {
    float weight, t, t_lse;
    int last, id, action;
    Rollout rollout;
};
template <LossKind KIND>
__device__ __forceinline__ RowInputs row_inputs(const LossArgs& a, int r) {
    const int b = r / a.in.rows, tid = threadIdx.x;
    RowInputs v{};
    v.weight = a.weight ? a.weight[r] : 1.f;
    v.last = a.last_row ? a.last_row[b] : a.in.rows;
    v.id = v.action = -1;
    if constexpr (KIND == LOSS_DISTILL) {
        const long long row = (long long)b * a.t_seq_rows + (r - b * a.in.rows), e = row * a.n_top + min(tid, a.n_top - 1);
        v.id = a.ids[e];
        v.t = a.values[e];
        v.t_lse = a.lse ? a.lse[row] : 0.f;
    } else {
        v.action = a.actions[r];
        v.rollout = Rollout{a.advantage[r], a.old_logp ? a.old_logp[r] : 0.f, a.ref_logp ? a.ref_logp[r] : 0.f};
    }
    return v;
}
// does the row take part
template <LossKind KIND>
__device__ __forceinline__ bool row_counts(const LossArgs& a, int r, int chunk, const RowInputs& v) {
    if (v.weight == 0.f || r % a.in.rows > v.last) return false;
    if (KIND == LOSS_POLICY && (v.action < 0 || v.action >= a.in.vocab)) {
        if (v.action != -1 && chunk == 0 && threadIdx.x == 0) atomicOr(a.status, DEV_BAD_TOKEN);
        return false;
    }
    return true;
}

// Waits for the row's inputs, before the loads of the logits are issued: a later wait for an input, on a path where the
// compiler cannot count the loads in between, would wait for all of these.
__device__ __forceinline__ void inputs_here() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
}

// A teacher's entries in this chunk: membership bits of its vectors' columns, the marks of the threads that hold them (the
// first `held` full vectors of each), and this thread's entry.  list_entries, then (a barrier lies between) mark_entries.
template <bool BF, int NT>
__device__ __forceinline__ void list_entries(const LossArgs& a, int id, uint32_t* bits, LossShared<NT>& sh) {
    const int tid = threadIdx.x, words = (a.plan.cv * Elem<BF>::W + 31) / 32;
    if (tid < a.n_top) sh.ids[tid] = id;
    for (int w = tid; w < words; w += NT) bits[w] = 0u;
    sh.mark[tid] = 0u;
    if (tid == 0) sh.repeated = 0;
}
// Returns whether the entry counts; *here: it lies in this chunk (an entry that counts nowhere is chunk 0's to report);
// *z: its logit as stored, asked for but not looked at.
template <bool BF, int NT>
__device__ __forceinline__ bool mark_entries(const LossArgs& a, const Span<BF>& sp, int id, int chunk, int held, uint32_t* bits,
                                             LossShared<NT>& sh, typename Elem<BF>::type* z, bool* here) {
    constexpr int W = Elem<BF>::W;
    const int tid = threadIdx.x;
    __syncthreads();
    const bool entry = tid < a.n_top, valid = entry && id >= 0 && id < sp.n;
    const int v = valid ? (id + sp.lead) / W : 0;
    *here = valid ? v >= sp.v0 && v < sp.v1 : entry && chunk == 0;
    bool counts = valid && *here;
    if (counts) {
        *z = sp.row[id];
        const int bit = id + sp.lead - sp.v0 * W, at = v - sp.f0;
        if (atomicOr(&bits[bit >> 5], 1u << (bit & 31)) >> (bit & 31) & 1u) sh.repeated = 1;
        if (sp.full(v) && at < held * NT) atomicOr(&sh.mark[at % NT], 1u << (at / NT));   // a partial vector is nobody's to hold
    }
    __syncthreads();
    bool bad = entry && chunk == 0 && !valid && id != -1;
    if (sh.repeated && counts) {   // of equal ids the first counts
        for (int i = 0; i < tid; ++i)
            if (sh.ids[i] == id) counts = false;
        bad = bad || !counts;
    }
    if (bad) atomicOr(a.status, DEV_BAD_TOKEN);
    return counts;
}

// membership of vector i's columns: one bit per element
template <bool BF, LossKind KIND>
__device__ __forceinline__ uint32_t members(const Span<BF>& sp, const uint32_t* bits, int action, int i) {
    constexpr int W = Elem<BF>::W;
    if constexpr (KIND == LOSS_POLICY) {
        const int e = action + sp.lead - i * W;
        return e >= 0 && e < W ? 1u << e : 0u;
    } else {
        const int bit = (i - sp.v0) * W;
        return (bits[bit >> 5] >> (bit & 31)) & ((1u << W) - 1u);
    }
}

// One pass over this thread's vectors of a chunk for the statistics of the columns outside the entries, and a second
// one, through the same object, for their gradient.  The first CAP vectors of each thread stay in registers from the
// one to the other; the rest of a longer chunk is read again.  STREAM: held vectors, and with CAP 0 all, are loaded past the
// caches: those are for what is read again (125 us with it, 131 without, for 512 rows of 151936 f32 logits with gradient;
// 97 and 110 us for 992 rows without).
template <bool BF, LossKind KIND, int NT, int CAP, bool STREAM>
struct Columns {
    static constexpr int W = Elem<BF>::W;
    const Span<BF>& sp;
    const uint32_t* bits;
    int action;
    uint32_t mark;   // which held vectors have an entry among their columns
    static constexpr int AHEAD = CAP ? (CAP < 8 ? CAP : 8) : 4;   // vectors asked for before the first is worked on
    uint4 held[CAP ? CAP : AHEAD];   // CAP 0: a ring
    static_assert(CAP <= 32, "a bit per held vector");
    __device__ __forceinline__ Columns(const Span<BF>& s, const uint32_t* b, int act) : sp(s), bits(b), action(act), mark(0u) {
        if constexpr (KIND == LOSS_POLICY) {
            const int v = (act + s.lead) / W, at = v - s.f0;
            if (s.full(v) && at < CAP * NT && at % NT == (int)threadIdx.x) mark = 1u << (at / NT);
        }
    }
    // Asks for held vector u, without a branch (a thread's last ones may be the chunk's last vector again), so that a wait
    // for an earlier load does not wait for this one.  f1 > f0.
    __device__ __forceinline__ void ask(int u) {
        held[u] = get(min(sp.f0 + (int)threadIdx.x + u * NT, sp.f1 - 1));
    }
    __device__ __forceinline__ uint4 get(int i) const { return STREAM ? load_stream((const uint4*)sp.grid + i) : sp.load(i); }
    // The first vectors; `each` asks for the others as it goes, AHEAD ahead: with all of them asked for at once a wavefront is
    // held up until the memory has taken them, about as long as the row takes to come, and starts to work on it after that
    // (4096 rows of 151936 bf16 logits, distillation with gradient: 593 us, and 539 with 8 ahead).
    __device__ __forceinline__ void fetch() {
        if (sp.f1 <= sp.f0) return;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) ask(u);
    }
    __device__ __forceinline__ uint32_t mem(int i) const { return members<BF, KIND>(sp, bits, action, i); }
    // f(vector index, its values, is it a full one, has it an entry, its place in `held` or -1) for every vector; FIRST: the
    // pass that loads them.  The number of vectors is made opaque in each pass: the compiler would keep the comparisons with it, a
    // register pair per vector, from the one to the other.
    template <bool FIRST, class F>
    __device__ __forceinline__ void each(const F& f) {
        if ((int)threadIdx.x < sp.n_edges()) {
            float z[W];
            const int i = sp.edge(threadIdx.x);
            sp.load_edge(i, z);
            f(i, z, false, mem(i) != 0u, -1);
        }
        int count = sp.f1 - sp.f0 - (int)threadIdx.x;   // vectors from this thread's first on
        asm volatile("" : "+v"(count));
        if (CAP > 0 && sp.f1 > sp.f0) {
#pragma unroll
            for (int u = 0; u < CAP; ++u) {
                if (FIRST && u + AHEAD < CAP) {
                    ask(u + AHEAD);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (count > u * NT) {
                    float z[W];
                    unpack<BF>(held[u], z);
                    f(sp.f0 + (int)threadIdx.x + u * NT, z, true, (mark >> u & 1u) != 0u, u);
                }
            }
        }
        if constexpr (CAP == 0) {
            if (sp.f1 <= sp.f0) return;
            if (!FIRST) fetch();
            const int rounds = (sp.f1 - sp.f0 + NT - 1) / NT;
            for (int u0 = 0; u0 < rounds; u0 += AHEAD)
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int i = sp.f0 + (int)threadIdx.x + (u0 + u) * NT;
                    if (count > (u0 + u) * NT) {
                        float z[W];
                        unpack<BF>(held[u], z);
                        f(i, z, true, mem(i) != 0u, -1);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    held[u] = get(min(i + AHEAD * NT, sp.f1 - 1));
                }
            return;
        }
        constexpr int U = 2;
        int i = sp.f0 + (int)threadIdx.x + CAP * NT;
        for (; i + (U - 1) * NT < sp.f1; i += U * NT) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = sp.load(i + u * NT);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float z[W];
                unpack<BF>(v[u], z);
                f(i + u * NT, z, true, mem(i + u * NT) != 0u, -1);
            }
        }
        for (; i < sp.f1; i += NT) {
            float z[W];
            unpack<BF>(sp.load(i), z);
            f(i, z, true, mem(i) != 0u, -1);
        }
    }
    // the vectors of this thread one after the other, for what rarely runs: f(vector index, its values, entries among them)
    template <class F>
    __device__ __forceinline__ void each_slowly(const F& f) const {
#pragma unroll 1
        for (int i = sp.v0 + (int)threadIdx.x; i < sp.v1; i += NT) {
            float z[W];
            if (sp.full(i)) unpack<BF>(sp.load(i), z);
            else sp.load_edge(i, z);
            f(i, z, mem(i));
        }
    }
    // entry(): this thread's entry's logit, whose maximum goes to *z_top (NULL: neither)
    template <class E>
    __device__ __forceinline__ RowStat stats(const LossArgs& a, LossShared<NT>& sh, const E& entry_logit, float* z_top) {
        Stat st{STAT_EMPTY, 0.f};
        each<true>([&](int i, float* z, bool, bool entry, int) __attribute__((always_inline)) {
            if (entry) {
                const uint32_t m = mem(i);
#pragma unroll
                for (int e = 0; e < W; ++e) z[e] = (m >> e) & 1u ? -INFINITY : z[e];
            }
            stat_add<W>(st, z, a.c);
        });
        if (z_top) *z_top = entry_logit();
        return row_stat<NT>(st, sh.red, a.c, a.c_exact, z_top, [&]() __attribute__((always_inline)) {
            Stat t{-INFINITY, 0.f};
            each_slowly([&](int, float* z, uint32_t m) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < W; ++e) t = wide_merge(t, Stat{(m >> e) & 1u ? -INFINITY : z[e], 1.f}, a.c);
            });
            return t;
        });
    }
};

template <bool BF>
struct GradRow {
    typedef typename Elem<BF>::type T;
    static constexpr int W = Elem<BF>::W;
    T* out;   // column 0
    __device__ __forceinline__ GradRow(const LossArgs& a, int r) {
        const int b = r / a.in.rows, j = r - b * a.in.rows;
        out = (T*)a.grad + (long long)b * a.grad_seq_stride + (long long)j * a.grad_row_stride;
    }
    // All columns of vector i (of the logits' grid; the gradient's rows may lie otherwise, and global stores of any
    // alignment are one instruction).  STREAM: past the caches.  Many rows' gradients are more than these hold, and would
    // drive out the part of the logits that is read again: 512 rows of 151936 f32 logits take 131 us with it and 163 without,
    // 4096 of bf16, which stay in registers, 424 and 438.
    template <bool STREAM>
    __device__ __forceinline__ void put(const Span<BF>& sp, int i, const float* g) const {
        uint4 v;
        if constexpr (BF) v = uint4{pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]), pack_bf16x2(g[4], g[5]), pack_bf16x2(g[6], g[7])};
        else v = uint4{__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3])};
        T* at = out + ((long long)i * W - sp.lead);
        if constexpr (STREAM) {
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
            __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, (u32x4*)at);
        } else {
            __builtin_memcpy(at, &v, 16);
        }
    }
    // those that lie in the row and not in `skip`
    __device__ __forceinline__ void put_some(const Span<BF>& sp, int i, const float* g, uint32_t skip) const {
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const int col = i * W + e - sp.lead;
            if (col >= 0 && col < sp.n && !((skip >> e) & 1u)) store_elem<BF>(out + col, g[e]);
        }
    }
    template <int NT>
    __device__ __forceinline__ void zero(const Span<BF>& sp) const {
        float g[W] = {};
        if ((int)threadIdx.x < sp.n_edges()) put_some(sp, sp.edge(threadIdx.x), g, 0u);
        for (int i = sp.f0 + (int)threadIdx.x; i < sp.f1; i += NT) put<true>(sp, i, g);
    }
};

// The gradient of a chunk's columns: the rest's from `cols`, and the entry of this thread (col, where `mine`).  A thread
// has read a vector when it writes the same columns, and the entries' logits were read before, so the gradient may
// take the logits' place.  The few full vectors with an entry among their columns are written column by column, after the
// others: they are read once more for it, which keeps that code out of the unrolled part.  The partial ones at the row's
// ends are written with the others, by the thread that reads them element by element, and only there: a second look at
// them would find gradients where the logits were.
template <bool BF, LossKind KIND, int NT, int CAP, bool STREAM>
__device__ __forceinline__ void write_grad(const LossArgs& a, const Span<BF>& sp, Columns<BF, KIND, NT, CAP, STREAM>& cols, int r,
                                           const RowGrad& g, bool mine, int col) {
    constexpr int W = Elem<BF>::W;
    const GradRow<BF> out(a, r);
    if (g.none) {
        out.template zero<NT>(sp);
        return;
    }
    if (!(fabs(g.st.ref) < (double)WIDE_FROM)) {   // differences first, as in the statistics; m is the row's largest logit
        const float m = (float)(g.st.ref / a.c_exact);
        const float scale = g.st.s == 0.f ? (float)(0.0 * g.rest) : (float)(g.rest / (double)g.st.s * exp2(base2(m, a.c_exact) - g.st.ref));
        cols.each_slowly([&](int i, float* z, uint32_t mem) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < W; ++e) z[e] = __builtin_amdgcn_exp2f((z[e] - m) * a.c) * scale;
            out.put_some(sp, i, z, mem);
        });
    } else {
        // exp2(z c - m) * scale; m is the reference rounded to f32 (c's rounding taken back), and what it is off by belongs to
        // scale
        const float m = uniform((float)(g.st.ref * ((double)a.c / a.c_exact)));
        const float scale = uniform(g.st.s == 0.f ? (float)(0.0 * g.rest) : (float)(g.rest / (double)g.st.s * exp2((double)m * (a.c_exact / (double)a.c) - g.st.ref)));
        auto value = [&](float z) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(fmaf(z, a.c, -m)) * scale; };
        cols.template each<false>([&](int i, float* z, bool full, bool entry, int u) __attribute__((always_inline)) {
            if (full && !entry) {
#pragma unroll
                for (int e = 0; e < W; ++e) z[e] = value(z[e]);
                out.template put<STREAM>(sp, i, z);
            } else if (u < 0) {
#pragma unroll
                for (int e = 0; e < W; ++e) z[e] = value(z[e]);
                out.put_some(sp, i, z, cols.mem(i));
            }
        });
#pragma unroll 1
        for (uint32_t later = cols.mark; later; later &= later - 1u) {
            const int i = sp.f0 + (int)threadIdx.x + NT * (__ffs(later) - 1);
            float z[W];
            unpack<BF>(sp.load(i), z);
#pragma unroll
            for (int e = 0; e < W; ++e) z[e] = value(z[e]);
            out.put_some(sp, i, z, cols.mem(i));
        }
    }
    if (mine) store_elem<BF>(out.out + col, g.entry);
}

// a row that takes no part, or has nothing to learn from
template <bool BF, int NT>
__device__ __forceinline__ void empty_row(const LossArgs& a, const Span<BF>& sp, int r, int chunk) {
    if (chunk == 0 && threadIdx.x == 0) {
        a.loss[r] = 0.f;
        if (a.aux) a.aux[r] = 0.f;
    }
    if (a.grad) GradRow<BF>(a, r).template zero<NT>(sp);
}

// A workgroup takes a whole row and keeps it, or the first CAP * NT vectors of it, in registers from the statistics to
// the gradient.
template <bool BF, LossKind KIND, int NT, int CAP>
__global__ void __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(CAP ? 4 : 8))) loss_row_kernel(LossArgs a) {
    typedef typename Elem<BF>::type T;
    extern __shared__ uint32_t bits[];
    __shared__ LossShared<NT> sh;
    const int r = blockIdx.x, tid = threadIdx.x;
    const Span<BF> sp(a.in, r, 0, a.plan.cv);
    const RowInputs in = row_inputs<KIND>(a, r);
    if (!row_counts<KIND>(a, r, 0, in)) {
        empty_row<BF, NT>(a, sp, r, 0);
        return;
    }
    Columns<BF, KIND, NT, CAP, true> cols(sp, bits, in.action);
    RowGrad g;
    bool mine = tid == 0;
    if constexpr (KIND == LOSS_DISTILL) {
        list_entries<BF, NT>(a, in.id, bits, sh);
        inputs_here();
        cols.fetch();
        T raw = 0;
        bool here;
        const bool counts = mark_entries<BF, NT>(a, sp, in.id, 0, CAP, bits, sh, &raw, &here);
        cols.mark = sh.mark[tid];
        const bool whole = __syncthreads_count(counts) == sp.n;
        const Teacher te = teacher_side<NT>(a, in.t, in.t_lse, counts, sh);
        __builtin_amdgcn_sched_barrier(0);
        // (z as stored is looked at after the row's vectors, which were asked for before it)
        float z = -INFINITY, z_top;
        const RowStat st = cols.stats(a, sh, [&]() __attribute__((always_inline)) { return z = counts ? to_float<BF>(raw) : -INFINITY; }, &z_top);
        g = distill_row<NT>(a, r, te, counts, whole, z, z_top, st, (double)in.weight, sh);
        mine = counts;
    } else {
        const T raw = sp.row[in.action];
        cols.fetch();
        const RowStat st = cols.stats(a, sh, [] { return 0.f; }, nullptr);
        g = policy_row(a, r, in.rollout, to_float<BF>(raw), st, (double)in.weight, sh);
    }
    if (a.grad) write_grad(a, sp, cols, r, g, mine, KIND == LOSS_POLICY ? in.action : mine ? sh.ids[tid] : -1);
}

// Few rows are shared by several workgroups.  STEP 1 leaves every chunk's statistics and entries in the workspace, STEP 2
// takes them together, each workgroup for itself, and writes its chunk of the gradient.
template <bool BF, LossKind KIND, int STEP, bool STREAM>
__global__ void __launch_bounds__(LOSS_NT) loss_chunk_kernel(LossArgs a) {
    typedef typename Elem<BF>::type T;
    constexpr int NT = LOSS_NT;
    extern __shared__ uint32_t bits[];
    __shared__ LossShared<NT> sh;
    const int per_row = STEP == 2 && !a.grad ? 1 : a.plan.chunks;   // workgroups of a row in this launch
    const int r = blockIdx.x / per_row, chunk = blockIdx.x % per_row, tid = threadIdx.x;
    const int n_entries = KIND == LOSS_DISTILL ? a.n_top : 1;
    const Span<BF> sp(a.in, r, chunk, a.plan.cv);
    const RowInputs in = row_inputs<KIND>(a, r);
    if (!row_counts<KIND>(a, r, chunk, in)) {
        if (STEP == 2) empty_row<BF, NT>(a, sp, r, chunk);
        return;
    }
    Columns<BF, KIND, NT, 0, STREAM> cols(sp, bits, in.action);
    T raw = 0;
    bool counts = false, here = false;
    if constexpr (KIND == LOSS_DISTILL) {
        if (STEP == 1 || a.grad) {
            list_entries<BF, NT>(a, in.id, bits, sh);
            if (STEP == 1) {
                inputs_here();
                cols.fetch();
            }
            counts = mark_entries<BF, NT>(a, sp, in.id, STEP == 1 ? chunk : -1, 0, bits, sh, &raw, &here);
        }
    } else {
        const int v = (in.action + sp.lead) / Elem<BF>::W;
        here = v >= sp.v0 && v < sp.v1;
        counts = true;
        if (STEP == 1 && here) raw = sp.row[in.action];
        if (STEP == 1) cols.fetch();
    }
    if constexpr (STEP == 1) {
        const RowStat st = cols.stats(a, sh, [] { return 0.f; }, nullptr);
        if (tid == 0) a.part[(long long)r * a.plan.chunks + chunk] = st;
        if (here && tid < n_entries)
            a.saved[(long long)r * n_entries + tid] = uint2{__float_as_uint(to_float<BF>(raw)), counts ? 1u : 0u};
    } else {
        const RowStat st = merge_chunks(a.part, r, a.plan.chunks);
        RowGrad g;
        bool mine = here && tid == 0;
        if constexpr (KIND == LOSS_DISTILL) {
            const uint2 e = tid < a.n_top ? a.saved[(long long)r * a.n_top + tid] : uint2{0u, 0u};
            counts = e.y != 0u;
            const bool whole = __syncthreads_count(counts) == sp.n;
            const Teacher te = teacher_side<NT>(a, in.t, in.t_lse, counts, sh);
            const float z = counts ? __uint_as_float(e.x) : -INFINITY;
            float z_top = z;
            stat_block<NT, false>(Stat{STAT_EMPTY, 0.f}, sh.red, a.c, &z_top);
            g = distill_row<NT>(a, r, te, counts, whole, z, z_top, st, (double)in.weight, sh);
            mine = here && counts;
        } else {
            g = policy_row(a, r, in.rollout, __uint_as_float(a.saved[r].x), st, (double)in.weight, sh);
        }
        if (a.grad) write_grad(a, sp, cols, r, g, mine, KIND == LOSS_POLICY ? in.action : mine ? sh.ids[tid] : -1);
    }
}

template <bool BF, LossKind KIND>
void launch_loss_as(const LossArgs& a, hipStream_t s) {
    constexpr int HELD = KIND == LOSS_DISTILL ? 19 : 21;   // vectors of a thread that stay in registers
    const int n = a.in.batch * a.in.rows;
    const size_t lds = KIND == LOSS_DISTILL ? (size_t)cdiv(a.plan.cv * Elem<BF>::W, 32) * 4 : 0;
    if (a.plan.chunks == 1) {
        const int nt = a.plan.threads;
        if (a.grad) {
            if (nt == 1024) loss_row_kernel<BF, KIND, 1024, HELD><<<n, 1024, lds, s>>>(a);
            else if (nt == 512) loss_row_kernel<BF, KIND, 512, HELD><<<n, 512, lds, s>>>(a);
            else loss_row_kernel<BF, KIND, 256, HELD><<<n, 256, lds, s>>>(a);
        } else if (nt == 1024) {
            loss_row_kernel<BF, KIND, 1024, 0><<<n, 1024, lds, s>>>(a);
        } else if (nt == 512) {
            loss_row_kernel<BF, KIND, 512, 0><<<n, 512, lds, s>>>(a);
        } else {
            loss_row_kernel<BF, KIND, 256, 0><<<n, 256, lds, s>>>(a);
        }
        return;
    }
    if (a.grad) {   // the second step reads what the first left in the caches
        loss_chunk_kernel<BF, KIND, 1, false><<<n * a.plan.chunks, LOSS_NT, lds, s>>>(a);
        loss_chunk_kernel<BF, KIND, 2, false><<<n * a.plan.chunks, LOSS_NT, lds, s>>>(a);
    } else {
        loss_chunk_kernel<BF, KIND, 1, true><<<n * a.plan.chunks, LOSS_NT, lds, s>>>(a);
        loss_chunk_kernel<BF, KIND, 2, true><<<n, LOSS_NT, lds, s>>>(a);
    }
}

}  // namespace

int row_vectors(int bf16, int vocab) {
    const int W = bf16 ? 8 : 4;
    return cdiv(vocab + W - 1, W);
}

// chunks so that the launch has about `target` workgroups, each with at least `least` vectors
static RowPlan spread(int nv, int n_rows, int target, int least) {
    const int c = std::max(1, std::min(std::min(target / std::max(n_rows, 1), nv / least), 64));
    RowPlan p;
    p.cv = cdiv(nv, c);
    p.chunks = cdiv(nv, p.cv);
    return p;
}

// Rows shared by several workgroups, in two launches, or one each.  us for n rows, top 200 of 151936 columns (50 of fewer),
// shared and one each: f32 151936 columns 1 row 17 and 31, 64 rows 25 and 31, 128 rows 32 and 31, 50257 columns 1 row 13 and 17,
// 128 rows 19 and 17, 16877 columns 13 and 11; bf16 151936 columns 1 row 17 and 25, 64 rows 23 and 25, 128 rows 27 and 26.
// Threads of one: as many as keep a segment at TOP_AHEAD vectors, since each of these lies on a line of its own when it is looked
// at again (4096 bf16 rows of 50257 columns 106 us on 512, 136 on 1024; f32 of 151936 527 and 451).  NLD_TOP_CHUNKS (1: one each,
// else: shared) and NLD_TOP_THREADS (512, 1024) override.
RowPlan plan_top(int bf16, int n_rows, int vocab, int n_top, int cus) {
    const int nv = row_vectors(bf16, vocab);
    const double n = (double)n_rows * 256 / cus;
    bool share = nv * ((bf16 ? 7e-4 : 5e-4) - 3.7e-6 * n) > 5.0;
    const int forced = env_int("NLD_TOP_CHUNKS", 0);
    if (forced) share = forced > 1;
    RowPlan p{1, nv, 0};
    if (share) p = spread(nv, n_rows, SHARED_WGS * cus / 2, std::max(2048, n_top * 16 / (bf16 ? 8 : 4)));
    p.threads = env_int("NLD_TOP_THREADS", p.cv <= 512 * TOP_SEGS * TOP_AHEAD ? 512 : 1024);
    if (p.threads != 512 || n_top > 256) p.threads = 1024;   // the bound on the n_top-th comes from the threads' maxima
    return p;
}

// Rows shared by several workgroups, in two launches, or one each; and the threads of one.  us for n rows of 151936 columns,
// shared and one each: with gradient f32 1 row 14 and 28, 32 rows 25 and 35, 64 rows 35 and 36, 128 rows 59 and 48, bf16 14.6 and 25,
// 21 and 28, 27 and 29, 38 and 31; without, f32 1 row 11 and 21, 64 rows 18 and 22, 128 rows 24 and 25, bf16 64 rows 16 and 18,
// 128 rows 19 and 19; of 16877 columns one each is never slower (1 f32 row with gradient 12 and 14).  Within
// 2 us of these and of 50257 and 100000 columns, with nv vectors a row, n rows take
//     with gradient    shared 13.5 + 1e-5 n nv,   one each 8 + 8e-4 nv,
//     without          shared 11.3 + 2.7e-6 n nv, one each 8.3 + 4e-4 nv     (n of up to half the CUs)
// Threads: smaller workgroups hide each other's latencies, larger ones hold more of a row.  With gradient, 4096 rows of 4000 bf16
// columns take 60, 99 and 200 us on 256, 512 and 1024 threads, of 16877 106, 138 and 249, of 50257 214, 209 and 314, 1024 rows of
// 100000 f32 columns 204 and 157 on 512 and 1024; without, 4096 rows of 50257 bf16 columns 95, 112 and 160, 64 of 151936 f32
// columns 32, 22 and 23.
// NLD_LOSS_CHUNKS (1: one each, else: shared) and NLD_LOSS_THREADS (256, 512, 1024) override.
RowPlan plan_loss(int bf16, int n_rows, int vocab, int n_top, bool grad, int cus) {
    const int W = bf16 ? 8 : 4, nv = row_vectors(bf16, vocab);
    const double n = (double)n_rows * 256 / cus;
    bool share = grad ? 5.5 + 1e-5 * n * nv < 8e-4 * nv : 3.0 + 2.7e-6 * n * nv < 4e-4 * nv;
    const int forced = env_int("NLD_LOSS_CHUNKS", 0);
    if (forced) share = forced > 1;
    RowPlan p{1, nv, 0};
    if (share) p = spread(nv, n_rows, SHARED_WGS * cus, 1024);
    if (p.cv * W > LOSS_MAX_COLS) {
        p.cv = LOSS_MAX_COLS / W;
        p.chunks = cdiv(nv, p.cv);   // at most vocab / LOSS_MAX_COLS + 2
    }
    if (grad) p.threads = nv <= 256 * 19 ? 256 : (nv <= 512 * 26 ? 512 : 1024);
    else p.threads = nv > 2048 && n_rows < 2 * cus ? 512 : 256;
    p.threads = env_int("NLD_LOSS_THREADS", p.threads);
    if (p.threads != 256 && p.threads != 1024) p.threads = 512;
    if (p.threads == 256 && n_top > 256) p.threads = 512;   // a thread per entry
    return p;
}

hipError_t launch_top(const TopArgs& a, hipStream_t s) {
    const int n = a.in.batch * a.in.rows;
    const int wgs = n * a.plan.chunks;
    if (a.plan.threads == 512) {
        if (a.in.bf16) top_kernel<true, 512><<<wgs, 512, 0, s>>>(a);
        else top_kernel<false, 512><<<wgs, 512, 0, s>>>(a);
    } else {
        if (a.in.bf16) top_kernel<true, 1024><<<wgs, 1024, 0, s>>>(a);
        else top_kernel<false, 1024><<<wgs, 1024, 0, s>>>(a);
    }
    if (a.plan.chunks > 1) top_merge_kernel<<<n, 1024, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_loss(LossKind kind, const LossArgs& a, hipStream_t s) {
    if (kind == LOSS_DISTILL) {
        if (a.in.bf16) launch_loss_as<true, LOSS_DISTILL>(a, s);
        else launch_loss_as<false, LOSS_DISTILL>(a, s);
    } else {
        if (a.in.bf16) launch_loss_as<true, LOSS_POLICY>(a, s);
        else launch_loss_as<false, LOSS_POLICY>(a, s);
    }
    return hipGetLastError();
}

}  // namespace nld
