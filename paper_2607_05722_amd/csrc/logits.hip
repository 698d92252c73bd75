// Operators on rows of logits for gfx950 (CDNA4): the largest logits of each row, and two losses with their
// gradients: distillation from a teacher's top logits, and the clipped policy loss.
//
// All three read a row of `vocab` logits z once for its softmax statistics, q_j = exp(z_j / tau) / sum, and are bound
// by that read (a few operations and one exponential per logit), the gradient by the read and the write.
//
// Exponents are taken in base 2, with c = log2(e) / tau.  A thread keeps a running reference m (the largest logit it
// has seen) and s = sum exp2((z - m) * c); pairs (m, s) merge as s1 * exp2((m1 - m) * c) + s2 * exp2((m2 - m) * c).  The
// difference is taken before the product, so that a row of the type's lowest values does not overflow.  The sum is f32:
// 150 thousand positive terms in several hundred partial sums keep its relative error below 1e-5 at worst, near 1e-8
// in the middle.  What comes after the sums, a few values per row and per teacher entry, is in f64, because the losses
// are small differences of logarithms (a divergence of 1e-3 from logarithms near 10 keeps four digits in f32).
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

inline int cdiv(int a, int b) { return (a + b - 1) / b; }

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
__device__ __forceinline__ float load_elem(const typename Elem<BF>::type* p) {
    if constexpr (BF) return bf16_to_f32(*p);
    else return *p;
}
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

// ---------------------------------------------------------------- softmax statistics
struct Stat {
    float m, s;   // reference (-inf: nothing yet) and sum of exp2((z - m) * c)
};
__device__ __forceinline__ Stat stat_merge(Stat a, Stat b, float c) {
    Stat o;
    o.m = fmaxf(a.m, b.m);
    const float ref = o.m == -INFINITY ? 0.f : o.m;   // both empty: the sums are 0 (or NaN, which stays)
    o.s = a.s * __builtin_amdgcn_exp2f((a.m - ref) * c) + b.s * __builtin_amdgcn_exp2f((b.m - ref) * c);
    return o;
}
// adds N logits; a NaN or +inf among them makes the sum NaN
template <int N>
__device__ __forceinline__ void stat_add(Stat& t, const float* z, float c) {
    float top = z[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, z[e]);
    if (top > t.m) {
        t.s *= __builtin_amdgcn_exp2f((t.m - top) * c);
        t.m = top;
    }
    const float ref = t.m == -INFINITY ? 0.f : t.m;
#pragma unroll
    for (int e = 0; e < N; ++e) t.s += __builtin_amdgcn_exp2f((z[e] - ref) * c);
}
// every thread's statistics -> the workgroup's, in every thread; red: NT / 64 pairs
template <int NT>
__device__ __forceinline__ Stat stat_block(Stat t, Stat* red, float c) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) t = stat_merge(t, Stat{__shfl_xor(t.m, off), __shfl_xor(t.s, off)}, c);
    if (lane == 0) red[wave] = t;
    __syncthreads();
    t = red[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) t = stat_merge(t, red[w], c);
    return t;
}
// log2 of the sum of exp(z / tau)
__device__ __forceinline__ double stat_log2(Stat t, double c_exact) {
    return t.s == 0.f ? -(double)INFINITY : (double)t.m * c_exact + log2((double)t.s);
}

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

constexpr int TOP_NT = 1024;     // threads
constexpr int TOP_SEGS = 8;      // a thread's vectors are cut into this many segments, each with its maximum
constexpr int TOP_CAND = 2048;   // candidates that one ranking holds

struct TopShared {
    uint32_t seg[TOP_SEGS][TOP_NT];          // largest key of each thread's segments
    uint16_t hits[TOP_SEGS * TOP_NT];        // segments that may hold one of the largest
    unsigned long long cand[TOP_CAND];
    uint32_t hist[256];
    Stat red[TOP_NT / 64];
    int cnt[2][TOP_NT / 64];
    int n_hits, n_cand, digit, above;
};

// threads with `in`, summed over the workgroup (which: two buffers used in turn, so that one barrier does)
__device__ __forceinline__ int count_block(bool in, TopShared& sh, int which) {
    const int n = __popcll(__ballot(in));
    if ((threadIdx.x & 63) == 0) sh.cnt[which][threadIdx.x >> 6] = n;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int w = 0; w < TOP_NT / 64; ++w) t += sh.cnt[which][w];
    return t;
}

// A key that at least k threads' maxima reach, and not many more: bisection over the keys.  0 when fewer than k
// threads have anything.  At least k elements of the row reach it, so the k largest all do.
__device__ __forceinline__ uint32_t bound_below(uint32_t mine, int k, TopShared& sh) {
    uint32_t lo = 0u, hi = 0xFFFFFFFFu;   // k threads reach lo
    int which = 0;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2 + 1;
        const int n = count_block(mine >= mid, sh, which);
        which ^= 1;
        if (n >= k) {
            lo = mid;
            if (n <= k + (k >> 3) + 4) break;
        } else {
            hi = mid - 1;
        }
    }
    return lo;
}

// The k largest of n distinct keys, whatever their order and ties: radix selection from the top byte down, each byte
// one pass over the keys.  Leaves them in sh.cand (any order).  For rows whose bound lets too many candidates through
// (many equal logits, a vocabulary masked down to few tokens, NaN).
template <class Keys>
__device__ void select_exact(const Keys& key, int n, int k, TopShared& sh) {
    unsigned long long prefix = 0ull;
    int need = k;
    int shift = 56;
    for (; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0u;
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += TOP_NT) {
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
        if (threadIdx.x == 0) {
            int above = 0, d = 255;
            while (d > 0 && above + (int)sh.hist[d] < need) above += (int)sh.hist[d--];
            sh.digit = d;
            sh.above = above;
        }
        __syncthreads();
        need -= sh.above;
        prefix = (prefix << 8) | (unsigned long long)sh.digit;
        if ((int)sh.hist[sh.digit] == need) break;   // the whole bin belongs to the k largest
    }
    const unsigned long long least = prefix << (shift < 0 ? 0 : shift);
    __syncthreads();
    if (threadIdx.x == 0) sh.n_cand = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += TOP_NT) {
        const unsigned long long x = key(i);
        if (x >= least) {
            const int at = atomicAdd(&sh.n_cand, 1);
            if (at < TOP_CAND) sh.cand[at] = x;
        }
    }
    __syncthreads();
}

// Ranks the candidates (distinct keys) by counting, for each, the larger ones, and hands those of rank < k to
// `emit(rank, key)`.  Several threads share a candidate where there are few.
template <class Emit>
__device__ __forceinline__ void rank_candidates(int n, int k, TopShared& sh, const Emit& emit) {
    int share = 1;   // threads per candidate, a power of two up to 16
    while (share < 16 && n * share * 2 <= TOP_NT) share *= 2;
    for (int c0 = 0; c0 < n; c0 += TOP_NT / share) {
        const int c = c0 + (int)threadIdx.x / share, part = (int)threadIdx.x & (share - 1);
        const unsigned long long mine = c < n ? sh.cand[c] : 0ull;
        int rank = 0;
        if (c < n)
            for (int j = part; j < n; j += share) rank += sh.cand[j] > mine ? 1 : 0;
        for (int off = share >> 1; off >= 1; off >>= 1) rank += __shfl_xor(rank, off);
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
__device__ __forceinline__ float lse_of(Stat t, uint32_t top, const TopArgs& a) {
    if (top == 0xFFFFFFFFu) return NAN;
    if (top == ORD_POS_INF) return INFINITY;
    if (top == ORD_NEG_INF) return -INFINITY;
    return (float)(stat_log2(t, a.c_exact) * 0.69314718055994530942);
}

// One pass over the row for the statistics and for the maximum of every thread's segments; then a lower bound of the
// k-th largest from the threads' maxima; then a second look at the few segments that reach it (about k of 8192, a few
// per cent of the row, which the first pass left in L2 or the memory-side cache); then the candidates are ranked.
template <bool BF>
__global__ void __launch_bounds__(TOP_NT) top_kernel(TopArgs a) {
    constexpr int W = Elem<BF>::W;
    __shared__ TopShared sh;
    const int r = blockIdx.x / a.plan.chunks, chunk = blockIdx.x % a.plan.chunks, tid = threadIdx.x;
    const Span<BF> sp(a.in, r, chunk, a.plan.cv);
    const int iters = (sp.v1 - sp.v0 + TOP_NT - 1) / TOP_NT, len = (iters + TOP_SEGS - 1) / TOP_SEGS;   // vectors per segment
    if (tid == 0) {
        sh.n_hits = 0;
        sh.n_cand = 0;
    }
    Stat st{-INFINITY, 0.f};
    uint32_t best = 0u;
    for (int s = 0; s < TOP_SEGS; ++s) {
        float top = -INFINITY;
        bool any = false;
        for (int u = s * len; u < min(iters, (s + 1) * len); ++u) {
            const int i = sp.v0 + u * TOP_NT + tid;
            if (i >= sp.v1) break;
            float z[W];
            if (sp.full(i)) unpack<BF>(sp.load(i), z);
            else sp.load_edge(i, z);
            stat_add<W>(st, z, a.c);
#pragma unroll
            for (int e = 0; e < W; ++e) top = fmaxf(top, z[e]);
            any = true;
        }
        const uint32_t o = any ? order_of(top) : 0u;
        sh.seg[s][tid] = o;
        best = max(best, o);
    }
    st = stat_block<TOP_NT>(st, sh.red, a.c);
    const int e0 = max(0, sp.v0 * W - sp.lead), e1 = min(sp.n, sp.v1 * W - sp.lead), n = max(0, e1 - e0);
    const int k = min(a.n_top, n);
    uint32_t bound = 0u;
    bool exact = st.s != st.s;   // NaN or +inf: the maxima above do not order these
    if (!exact) {
        bound = bound_below(best, k, sh);
        __syncthreads();
#pragma unroll
        for (int s = 0; s < TOP_SEGS; ++s)
            if (sh.seg[s][tid] != 0u && sh.seg[s][tid] >= bound) sh.hits[atomicAdd(&sh.n_hits, 1)] = (uint16_t)(s * TOP_NT + tid);
        __syncthreads();
        const int items = sh.n_hits * len;
        for (int it = tid; it < items; it += TOP_NT) {
            const int h = sh.hits[it / len], s = h / TOP_NT, u = s * len + it % len, i = sp.v0 + u * TOP_NT + h % TOP_NT;
            if (u >= iters || i >= sp.v1) continue;
            float z[W];
            if (sp.full(i)) unpack<BF>(sp.load(i), z);
            else sp.load_edge(i, z);
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const int j = i * W + e - sp.lead;
                const uint32_t o = order_of(z[e]);
                if (j >= 0 && j < sp.n && o >= bound) {
                    const int at = atomicAdd(&sh.n_cand, 1);
                    if (at < TOP_CAND) sh.cand[at] = key_of(o, j);
                }
            }
        }
        __syncthreads();
        exact = sh.n_cand > TOP_CAND;
    }
    if (exact) select_exact(RowKeys<BF>{sp, e0}, n, k, sh);
    const int nc = sh.n_cand;
    if (a.plan.chunks == 1) {
        rank_candidates(nc, k, sh, [&](int rank, unsigned long long key) {
            emit_top(a, r, rank, key);
            if (rank == 0 && a.lse) a.lse[r] = lse_of(st, (uint32_t)(key >> 32), a);
        });
    } else {
        unsigned long long* out = a.keys + ((long long)r * a.plan.chunks + chunk) * a.n_top;
        for (int i = k + tid; i < a.n_top; i += TOP_NT) out[i] = 0ull;
        rank_candidates(nc, k, sh, [&](int rank, unsigned long long key) { out[rank] = key; });
        if (tid == 0) a.part[(long long)r * a.plan.chunks + chunk] = float2{st.m, st.s};
    }
}

// The chunks' largest keys -> the row's.
__global__ void __launch_bounds__(TOP_NT) top_merge_kernel(TopArgs a) {
    __shared__ TopShared sh;
    const int r = blockIdx.x, tid = threadIdx.x, n = a.plan.chunks * a.n_top;
    const ListKeys key{a.keys + (long long)r * n};
    if (tid == 0) sh.n_cand = 0;
    Stat st{-INFINITY, 0.f};
    for (int p = tid; p < a.plan.chunks; p += TOP_NT) {
        const float2 v = a.part[(long long)r * a.plan.chunks + p];
        st = stat_merge(st, Stat{v.x, v.y}, a.c);
    }
    uint32_t best = 0u;
    for (int i = tid; i < n; i += TOP_NT) best = max(best, (uint32_t)(key(i) >> 32));
    st = stat_block<TOP_NT>(st, sh.red, a.c);
    const uint32_t bound = max(bound_below(best, a.n_top, sh), 1u);   // 0: an empty place of a short chunk
    __syncthreads();
    for (int i = tid; i < n; i += TOP_NT) {
        const unsigned long long x = key(i);
        if ((uint32_t)(x >> 32) < bound) continue;
        const int at = atomicAdd(&sh.n_cand, 1);
        if (at < TOP_CAND) sh.cand[at] = x;
    }
    __syncthreads();
    if (sh.n_cand > TOP_CAND) select_exact(key, n, a.n_top, sh);
    rank_candidates(sh.n_cand, a.n_top, sh, [&](int rank, unsigned long long x) {
        emit_top(a, r, rank, x);
        if (rank == 0 && a.lse) a.lse[r] = lse_of(st, (uint32_t)(x >> 32), a);
    });
}

// ---------------------------------------------------------------- losses with their gradients
// Both losses see a row as its entries (the teacher's tokens; the action) and the rest of the vocabulary:
//   statistics   (m, s) over the rest, the entries apart, so that neither a rest that has next to nothing nor an entry
//                that has next to all loses its digits in a difference from the row's sum;
//   row values   in f64 from the entries' logits and (m, s): the loss, and the coefficients of the gradient, which is
//                rest * exp2((z_j - m) * c) for every column outside the entries and a value of its own for each entry;
//   gradient     one more pass over the row.
constexpr int LOSS_NT = 512;   // a thread per entry
static_assert(LOSS_NT >= TOP_MAX, "a thread per teacher entry");

struct LossShared {
    Stat red[LOSS_NT / 64];
    double sum[LOSS_NT / 64][5];
    int32_t ids[TOP_MAX];
    int repeated;
};

// sums (or maxima) of N values over the workgroup, in every thread; wavefronts without a teacher entry hold `none`
template <int N, bool MAX>
__device__ __forceinline__ void reduce_block(double* v, bool mine, LossShared& sh) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const double none = MAX ? -(double)INFINITY : 0.0;
    if (mine) {
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const double o = __shfl_xor(v[i], off);
                v[i] = MAX ? fmax(v[i], o) : v[i] + o;
            }
    }
    __syncthreads();
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) sh.sum[wave][i] = mine ? v[i] : none;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        double t = sh.sum[0][i];
        for (int w = 1; w < LOSS_NT / 64; ++w) t = MAX ? fmax(t, sh.sum[w][i]) : t + sh.sum[w][i];
        v[i] = t;
    }
}

// what a row's gradient needs: rest * exp2((z - m) * c) outside the entries, `entry` at this thread's entry
struct RowGrad {
    float m, rest, entry;
    bool none;   // the gradient is zero throughout
};

// Distillation.  p: the teacher's probabilities of its entries and, with its log-sum-exp given, of everything else (the
// rest, R); q: the student's.  Every thread calls this with its entry (counts: it is one).
//   loss = w (lambda KL + (1 - lambda) TV),  KL = sum p log(p / q),  TV = 1/2 sum |p - q|,
//   lambda = kl_share exp(-eta alpha), alpha = sum min(p, q), held constant in the gradient;
//   d loss / d z_j = w / tau (q_j (lambda P + (1 - lambda) / 2 (s_j - mean)) - lambda p_j) for an entry, with P = sum p,
//   s = sign(q - p), mean = sum s q, all sums over entries and rest, and in the rest, where every q_j has the same share
//   of what the rest gets, w / tau q_j (lambda P + (1 - lambda) / 2 (s_R - mean) - lambda p_R / q_R).
__device__ __forceinline__ RowGrad distill_row(const LossArgs& a, int r, int trow, bool counts, float z, float t, bool whole,
                                               Stat st, double weight, LossShared& sh) {
    const bool mine = (int)(threadIdx.x & ~63u) < a.n_top;   // a wavefront with entries
    const double none = -(double)INFINITY;
    const double x = counts ? (double)t * a.c_exact : none, y = counts ? (double)z * a.c_exact : none;   // base-2 exponents
    double top[2] = {x, y};
    reduce_block<2, true>(top, mine, sh);
    double tot[2];
    tot[0] = x == none ? 0.0 : exp2(x - top[0]);
    tot[1] = y == none ? 0.0 : exp2(y - top[1]);
    reduce_block<2, false>(tot, mine, sh);
    const double log_rest = stat_log2(st, a.c_exact);
    const double ref = fmax(log_rest, top[1]);
    const double lse = a.lse ? (double)a.lse[trow] * 1.44269504088896340736 : top[0] + log2(tot[0]);
    RowGrad g{st.m == -INFINITY ? 0.f : st.m, 0.f, 0.f, true};
    // a teacher or a student without any token: nothing to learn
    if (lse == none || (ref == none && st.s == 0.f && tot[1] == 0.0)) {
        if (threadIdx.x == 0) {
            a.loss[r] = 0.f;
            if (a.aux) a.aux[r] = 0.f;
        }
        return g;
    }
    const double log_all = ref + log2(exp2(log_rest - ref) + (top[1] > none ? tot[1] * exp2(top[1] - ref) : tot[1]));
    const double lp = x - lse, lq = y - log_all;
    const double p = counts ? exp2(lp) : 0.0, q = counts ? exp2(lq) : 0.0;
    const double sgn = q > p ? 1.0 : (q < p ? -1.0 : 0.0);
    double sums[5] = {p, p > 0.0 ? p * (lp - lq) : 0.0, fmin(p, q), fabs(p - q), sgn * q};
    if (counts && !(p == p && q == q)) sums[2] = p + q;   // fmin would drop a NaN
    reduce_block<5, false>(sums, mine, sh);
    const double p_rest = a.lse && !whole ? fmax(0.0, 1.0 - sums[0]) : 0.0;
    const double lq_rest = log_rest - log_all, q_rest = exp2(lq_rest);
    const double s_rest = q_rest > p_rest ? 1.0 : (q_rest < p_rest ? -1.0 : 0.0);
    const double kl = (sums[1] + (p_rest > 0.0 ? p_rest * (log2(p_rest) - lq_rest) : 0.0)) * 0.69314718055994530942;
    const double tv = 0.5 * (sums[3] + fabs(p_rest - q_rest));
    const double alpha = sums[2] + (q_rest == q_rest ? fmin(p_rest, q_rest) : q_rest);
    const double mean = sums[4] + s_rest * q_rest, mass = sums[0] + p_rest;
    const double lambda = (double)a.kl_share * exp2(-(double)a.eta * 1.44269504088896340736 * alpha);
    if (threadIdx.x == 0) {
        a.loss[r] = (float)(weight * ((lambda > 0.0 ? lambda * kl : 0.0) + (1.0 - lambda) * tv));
        if (a.aux) a.aux[r] = (float)alpha;
    }
    const double f = weight * a.inv_tau, half = 0.5 * (1.0 - lambda);
    g.none = false;
    g.entry = (float)(f * (q * (lambda * mass + half * (sgn - mean)) - lambda * p));
    // exp2((z - m) c) / s is a column's share of the rest
    if (st.s != 0.f) g.rest = (float)(f * (q_rest * (lambda * mass + half * (s_rest - mean)) - lambda * p_rest) / (double)st.s);
    return g;
}

// Clipped policy loss of the action's log-probability.  rho = exp(logp - old),
//   loss = w (-min(rho A, clip(rho, 1 - low, 1 + high) A) + beta (exp(d) - d - 1)),  d = ref - logp,
//   d loss / d logp = w (-[rho A is the minimum] rho A + beta (1 - exp(d))),  d logp / d z_j = ([j = action] - q_j) / tau.
// With the action apart, 1 - q of a likely action is the rest's share itself.
__device__ __forceinline__ RowGrad policy_row(const LossArgs& a, int r, float z, Stat st, double weight) {
    RowGrad g{st.m == -INFINITY ? 0.f : st.m, 0.f, 0.f, true};
    const double y = (double)z * a.c_exact, log_rest = stat_log2(st, a.c_exact);
    const double ref = fmax(log_rest, y);
    if (ref == -(double)INFINITY && st.s == 0.f && z == z) {   // no token is possible
        if (threadIdx.x == 0) {
            a.loss[r] = 0.f;
            if (a.aux) a.aux[r] = 0.f;
        }
        return g;
    }
    const double er = exp2(log_rest - ref), ey = exp2(y - ref), all = er + ey;
    // log(ey / all), by the rest's share where that is the small part
    const double logp = y >= log_rest ? -log1p(er / ey) : (y - ref) * 0.69314718055994530942 - log(all);
    const double adv = a.advantage[r];
    const double rho = a.old_logp ? exp(logp - (double)a.old_logp[r]) : (logp == logp ? 1.0 : logp);
    const double free_ = adv == 0.0 ? 0.0 : rho * adv;
    const double held = fmin(fmax(rho, 1.0 - (double)a.clip_low), 1.0 + (double)a.clip_high) * adv;
    double loss = free_ <= held ? -free_ : (free_ > held ? -held : (double)NAN);
    double dl = free_ <= held ? -free_ : (free_ > held ? 0.0 : (double)NAN);
    if (a.ref_logp) {
        const double d = (double)a.ref_logp[r] - logp, beta = a.kl_coef;
        loss += beta * (expm1(d) - d);
        dl -= beta * expm1(d);
    }
    if (threadIdx.x == 0) {
        a.loss[r] = (float)(weight * loss);
        if (a.aux) a.aux[r] = (float)logp;
    }
    const double f = weight * a.inv_tau * dl;
    g.none = f == 0.0;   // clipped
    g.entry = (float)(f * (er / all));
    if (st.s != 0.f) g.rest = (float)(-f * (er / all) / (double)st.s);
    return g;
}

// does row r take part, and with what weight
__device__ __forceinline__ bool row_counts(const LossArgs& a, int r, double* weight) {
    const float w = a.weight ? a.weight[r] : 1.f;
    *weight = (double)w;
    const int b = r / a.in.rows;
    return w != 0.f && !(a.last_row && r - b * a.in.rows > a.last_row[b]);
}

// The entries of this chunk: membership bits of its vectors' columns (distillation), and this thread's entry: *z its
// logit where it lies in the chunk.  Returns whether the entry counts; *here: it lies in this chunk (an entry that
// counts nowhere is chunk 0's to report).
template <bool BF>
__device__ __forceinline__ bool find_entries(const LossArgs& a, const Span<BF>& sp, long long trow, int chunk, uint32_t* bits,
                                             LossShared& sh, float* z, bool* here) {
    constexpr int W = Elem<BF>::W;
    const int tid = threadIdx.x, words = (a.plan.cv * W + 31) / 32;
    for (int w = tid; w < words; w += LOSS_NT) bits[w] = 0u;
    if (tid == 0) sh.repeated = 0;
    const int id = tid < a.n_top ? a.ids[trow * a.n_top + tid] : -1;
    if (tid < a.n_top) sh.ids[tid] = id;
    __syncthreads();
    const bool valid = id >= 0 && id < sp.n;
    const int v = valid ? (id + sp.lead) / W : 0;
    *here = valid ? v >= sp.v0 && v < sp.v1 : tid < a.n_top && chunk == 0;
    bool counts = valid && *here;
    if (counts) {
        *z = load_elem<BF>(sp.row + id);
        const int bit = id + sp.lead - sp.v0 * W;
        if (atomicOr(&bits[bit >> 5], 1u << (bit & 31)) >> (bit & 31) & 1u) sh.repeated = 1;
    }
    __syncthreads();
    bool bad = tid < a.n_top && chunk == 0 && !valid && id != -1;
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

template <bool BF, LossKind KIND>
__device__ __forceinline__ Stat rest_stats(const Span<BF>& sp, const uint32_t* bits, int action, float c) {
    constexpr int W = Elem<BF>::W, U = 4;
    Stat st{-INFINITY, 0.f};
    auto add = [&](float* z, int i) __attribute__((always_inline)) {
        const uint32_t mem = members<BF, KIND>(sp, bits, action, i);
        if (mem)
#pragma unroll
            for (int e = 0; e < W; ++e) z[e] = (mem >> e) & 1u ? -INFINITY : z[e];
        stat_add<W>(st, z, c);
    };
    if ((int)threadIdx.x < sp.n_edges()) {
        float z[W];
        const int i = sp.edge(threadIdx.x);
        sp.load_edge(i, z);
        add(z, i);
    }
    int i = sp.f0 + threadIdx.x;
    for (; i + (U - 1) * LOSS_NT < sp.f1; i += U * LOSS_NT) {
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = sp.load(i + u * LOSS_NT);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float z[W];
            unpack<BF>(v[u], z);
            add(z, i + u * LOSS_NT);
        }
    }
    for (; i < sp.f1; i += LOSS_NT) {
        float z[W];
        unpack<BF>(sp.load(i), z);
        add(z, i);
    }
    return st;
}

// The gradient of this chunk's columns outside the entries (none: zeros in all its columns).  A thread reads a
// vector before it writes the same columns, so the gradient may take the logits' place.
template <bool BF, LossKind KIND>
__device__ __forceinline__ void write_rest(const LossArgs& a, const Span<BF>& sp, int r, const uint32_t* bits, int action,
                                           RowGrad g) {
    const bool zero = g.none;
    typedef typename Elem<BF>::type T;
    constexpr int W = Elem<BF>::W;
    const int b = r / a.in.rows, j = r - b * a.in.rows;
    T* out = (T*)a.grad + (long long)b * a.grad_seq_stride + (long long)j * a.grad_row_stride;
    const bool wide = (((uintptr_t)out ^ (uintptr_t)sp.row) & 15u) == 0u;   // vectors line up with the logits'
    auto put = [&](float* z, int i, bool full) __attribute__((always_inline)) {
        const uint32_t mem = zero ? 0u : members<BF, KIND>(sp, bits, action, i);
#pragma unroll
        for (int e = 0; e < W; ++e) z[e] = zero ? 0.f : __builtin_amdgcn_exp2f((z[e] - g.m) * a.c) * g.rest;
        if (full && wide && mem == 0u) {
            uint4 v;
            if constexpr (BF) v = uint4{pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3]), pack_bf16x2(z[4], z[5]), pack_bf16x2(z[6], z[7])};
            else v = uint4{__float_as_uint(z[0]), __float_as_uint(z[1]), __float_as_uint(z[2]), __float_as_uint(z[3])};
            *(uint4*)(out + ((long long)i * W - sp.lead)) = v;
        } else {
#pragma unroll
            for (int e = 0; e < W; ++e) {
                const int col = i * W + e - sp.lead;
                if (col >= 0 && col < sp.n && !((mem >> e) & 1u)) store_elem<BF>(out + col, z[e]);
            }
        }
    };
    if ((int)threadIdx.x < sp.n_edges()) {
        float z[W];
        const int i = sp.edge(threadIdx.x);
        if (!zero) sp.load_edge(i, z);
        put(z, i, false);
    }
    for (int i = sp.f0 + threadIdx.x; i < sp.f1; i += LOSS_NT) {
        float z[W];
        if (!zero) unpack<BF>(sp.load(i), z);
        put(z, i, true);
    }
}

template <bool BF>
__device__ __forceinline__ void write_entry(const LossArgs& a, int r, int col, float v) {
    typedef typename Elem<BF>::type T;
    const int b = r / a.in.rows, j = r - b * a.in.rows;
    store_elem<BF>((T*)a.grad + (long long)b * a.grad_seq_stride + (long long)j * a.grad_row_stride + col, v);
}

// STEP 0: a workgroup takes a whole row.  Rows that several workgroups share: STEP 1 leaves every chunk's statistics and
// entries in the workspace, STEP 2 takes them together, each workgroup for itself, and writes its chunk of the gradient.
template <bool BF, LossKind KIND, int STEP>
__global__ void __launch_bounds__(LOSS_NT) loss_kernel(LossArgs a) {
    extern __shared__ uint32_t bits[];
    __shared__ LossShared sh;
    const int per_row = STEP == 2 && !a.grad ? 1 : a.plan.chunks;   // workgroups of a row in this launch
    const int r = blockIdx.x / per_row, chunk = blockIdx.x % per_row, tid = threadIdx.x;
    const Span<BF> sp(a.in, r, chunk, a.plan.cv);
    double weight;
    bool on = row_counts(a, r, &weight);
    int action = -1;
    if (KIND == LOSS_POLICY && on) {
        action = a.actions[r];
        if (action < 0 || action >= sp.n) {
            if (action != -1 && chunk == 0 && tid == 0) atomicOr(a.status, DEV_BAD_TOKEN);
            on = false;
        }
    }
    if (!on) {
        if (STEP == 1) return;
        if (chunk == 0 && tid == 0) {
            a.loss[r] = 0.f;
            if (a.aux) a.aux[r] = 0.f;
        }
        if (a.grad) write_rest<BF, KIND>(a, sp, r, bits, -1, RowGrad{0.f, 0.f, 0.f, true});
        return;
    }
    const int b = r / a.in.rows;
    const long long trow = (long long)b * a.t_seq_rows + (r - b * a.in.rows);
    float z = -INFINITY;
    bool counts = false, here = false;
    if constexpr (KIND == LOSS_DISTILL) {
        if (STEP != 2 || a.grad) counts = find_entries<BF>(a, sp, trow, STEP == 2 ? -1 : chunk, bits, sh, &z, &here);
    } else {
        const int v = (action + sp.lead) / Elem<BF>::W;
        counts = true;
        here = v >= sp.v0 && v < sp.v1;
        if (STEP != 2 && here) z = load_elem<BF>(sp.row + action);
    }
    Stat st;
    if constexpr (STEP != 2) {
        st = stat_block<LOSS_NT>(rest_stats<BF, KIND>(sp, bits, action, a.c), sh.red, a.c);
        if constexpr (STEP == 1) {
            const int n_entries = KIND == LOSS_DISTILL ? a.n_top : 1;
            if (tid == 0) a.part[(long long)r * a.plan.chunks + chunk] = float2{st.m, st.s};
            if (here && tid < n_entries) a.saved[(long long)r * n_entries + tid] = uint2{__float_as_uint(z), counts ? 1u : 0u};
            return;
        }
    } else {
        st = Stat{-INFINITY, 0.f};
        for (int p = 0; p < a.plan.chunks; ++p) {
            const float2 v = a.part[(long long)r * a.plan.chunks + p];
            st = stat_merge(st, Stat{v.x, v.y}, a.c);
        }
        if constexpr (KIND == LOSS_DISTILL) {
            const uint2 e = tid < a.n_top ? a.saved[(long long)r * a.n_top + tid] : uint2{0u, 0u};
            z = __uint_as_float(e.x);
            here = here && e.y != 0u;
            counts = e.y != 0u;
        } else {
            z = __uint_as_float(a.saved[r].x);
        }
    }
    RowGrad g;
    if constexpr (KIND == LOSS_DISTILL) {
        const int n_counts = __syncthreads_count(counts);
        const float t = tid < a.n_top ? a.values[trow * a.n_top + tid] : 0.f;
        g = distill_row(a, r, (int)trow, counts, z, t, n_counts == sp.n, st, weight, sh);
    } else {
        g = policy_row(a, r, z, st, weight);
    }
    if (!a.grad) return;
    write_rest<BF, KIND>(a, sp, r, bits, action, g);
    if (g.none) return;
    if (KIND == LOSS_DISTILL ? counts && (STEP == 0 || here) : here && tid == 0)
        write_entry<BF>(a, r, KIND == LOSS_DISTILL ? sh.ids[tid] : action, g.entry);
}

template <bool BF, LossKind KIND>
void launch_loss_as(const LossArgs& a, hipStream_t s) {
    const int n = a.in.batch * a.in.rows;
    const size_t lds = KIND == LOSS_DISTILL ? (size_t)cdiv(a.plan.cv * Elem<BF>::W, 32) * 4 : 0;
    if (a.plan.chunks == 1) {
        loss_kernel<BF, KIND, 0><<<n, LOSS_NT, lds, s>>>(a);
        return;
    }
    loss_kernel<BF, KIND, 1><<<n * a.plan.chunks, LOSS_NT, lds, s>>>(a);
    loss_kernel<BF, KIND, 2><<<a.grad ? n * a.plan.chunks : n, LOSS_NT, lds, s>>>(a);
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

RowPlan plan_top(int bf16, int n_rows, int vocab, int n_top, int cus) {
    return spread(row_vectors(bf16, vocab), n_rows, SHARED_WGS * cus / 2, std::max(2048, n_top * 16 / (bf16 ? 8 : 4)));
}

constexpr int LOSS_MAX_COLS = 1 << 18;   // columns of one workgroup: their membership bits are 32 KB

RowPlan plan_loss(int bf16, int n_rows, int vocab, int cus) {
    const int W = bf16 ? 8 : 4, nv = row_vectors(bf16, vocab);
    RowPlan p = spread(nv, n_rows, SHARED_WGS * cus, 1024);
    if (p.cv * W > LOSS_MAX_COLS) {
        p.cv = LOSS_MAX_COLS / W;
        p.chunks = cdiv(nv, p.cv);
    }
    return p;
}

hipError_t launch_top(const TopArgs& a, hipStream_t s) {
    const int n = a.in.batch * a.in.rows;
    if (a.in.bf16) top_kernel<true><<<n * a.plan.chunks, TOP_NT, 0, s>>>(a);
    else top_kernel<false><<<n * a.plan.chunks, TOP_NT, 0, s>>>(a);
    if (a.plan.chunks > 1) top_merge_kernel<<<n, TOP_NT, 0, s>>>(a);
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
