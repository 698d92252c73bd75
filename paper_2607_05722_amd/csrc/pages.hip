// Paged key/value cache: writing and reading rows, the attention of a chunk of new rows over the pages, and the selection
// of pages by a cheap score.
//
// A page holds 64 positions of one layer: per KV head the keys, then (another array) the values, in the order in which the
// matrix instructions take them, so that a wavefront's operand is whole cache lines, 16 bytes per lane, and nothing is
// shuffled on the way.  Keys are the A operand of S^T = K Q^T, values that of O^T = V^T P^T.  The first product leaves a lane with
// one row and the keys 16 s + 8 j + 4 hf + i of 32 (i = 0..3, j = 0, 1; with rows in tiles of 32 hf = lane / 32 and both s, with
// tiles of 16 s = lane / 32, hf = lane / 16 % 2); the values' blocks hold 8 keys of a dim in that order, so the weights P
// need no exchange between lanes.
#include <type_traits>

#include "nld_internal.h"

namespace nld {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(16))) int i32x16_t;
typedef __attribute__((ext_vector_type(4))) int i32x4_t;

namespace {

// status bits, as in nld.h
constexpr uint32_t ST_CAPACITY = 2u, ST_LENGTH = 4u, ST_PAGE = 16u, ST_ROWS = 32u;

__device__ __forceinline__ void flag(uint32_t* status, uint32_t bit) { atomicOr(status, bit); }

// ---------------------------------------------------------------- places in a page
// Element offset of (key, dim) in a head's keys.  Blocks of 64 lanes x 16 bytes: 16 keys (of a group of 32 those with
// key / 8 even, then the others) x 4 pieces of 8 dims (bf16) or 16 (e4m3).
template <int D, bool E4M3>
__device__ __forceinline__ int key_at(int key, int d) {
    const int tile = (key >> 5) * 2 + ((key >> 3) & 1), m = ((key >> 4) & 1) * 8 + (key & 7);
    return E4M3 ? ((tile * (D / 64) + (d >> 6)) * 64 + ((d >> 4) & 3) * 16 + m) * 16 + (d & 15)
                : ((tile * (D / 32) + (d >> 5)) * 64 + ((d >> 3) & 3) * 16 + m) * 8 + (d & 7);
}
// of (key, dim) in a head's values: blocks of 16 dims x 4 pieces of 8 keys, of one group of 32 (bf16) or of both (e4m3)
template <int D, bool E4M3>
__device__ __forceinline__ int value_at(int key, int d) {
    const int piece = ((key >> 4) & 1) * 2 + ((key >> 2) & 1), e = ((key >> 3) & 1) * 4 + (key & 3), at = piece * 16 + (d & 15);
    return E4M3 ? ((d >> 4) * 64 + at) * 16 + (key >> 5) * 8 + e : (((key >> 5) * (D / 16) + (d >> 4)) * 64 + at) * 8 + e;
}
// key, of a group of 32, of element e of the piece (s, hf) of values
__device__ __forceinline__ int value_key(int s, int hf, int e) { return 16 * s + 4 * hf + (e & 3) + ((e & 4) << 1); }

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// two e4m3 numbers (the low or the high half of a word) times a power of two -> bf16 pair, exact
template <bool HI>
__device__ __forceinline__ uint32_t pair_bf16(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, scale, HI));
}
__device__ __forceinline__ uint4 eight_bf16(uint32_t a, uint32_t b, float scale) {
    return uint4{pair_bf16<false>(a, scale), pair_bf16<true>(a, scale), pair_bf16<false>(b, scale), pair_bf16<true>(b, scale)};
}

__device__ __forceinline__ f32x16_t mfma_32x32x16(uint4 a, uint4 b, f32x16_t c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// ---------------------------------------------------------------- rows of a chunk
struct SeqRows {
    int r0, n;   // first packed row, rows
};
__device__ __forceinline__ SeqRows seq_rows(const PageChunk& c, int b, uint32_t* status) {
    if (!c.row_start) return SeqRows{b * c.max_rows, c.max_rows};
    const int s = c.row_start[b], e = c.row_start[b + 1];
    const int r0 = min(max(s, 0), c.rows), n = min(min(max(e, r0), c.rows) - r0, c.max_rows);   // e before the difference: it may be any number
    if (status && (r0 != s || r0 + n != e)) flag(status, ST_ROWS);
    return SeqRows{r0, n};
}

// committed length; of a block of new rows, no position past what the table has room for
__device__ __forceinline__ int seq_length(const PageCache& c, int b, uint32_t* status) {
    const int p = c.lengths[b];
    if (p >= 0 && p <= c.max_pages * 64) return p;
    if (status) flag(status, p < 0 ? ST_LENGTH : ST_CAPACITY);
    return p < 0 ? 0 : c.max_pages * 64;
}

__device__ __forceinline__ int page_id(const PageCache& c, int b, int page) {
    const int id = c.table[(size_t)b * c.max_pages + page];
    return (unsigned)id < (unsigned)c.n_pages ? id : -1;
}

// 8 adjacent elements of a row as f32; vec: 16-byte aligned rows
__device__ __forceinline__ void load8(const HeadRows& r, long long row, int head, int d, float* x) {
    const size_t at = (size_t)(row * r.row_stride + head * r.head_stride + d);
    if (r.f32) {
        const float* p = (const float*)r.data + at;
        if (r.vec) {
            const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = p[i];
        }
    } else {
        const uint16_t* p = (const uint16_t*)r.data + at;
        if (r.vec) {
            const uint4 a = *(const uint4*)p;
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) x[2 * i] = bf16_to_f32(w[i] & 0xFFFFu), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = bf16_to_f32(p[i]);
        }
    }
}
__device__ __forceinline__ void store4(const HeadRows& r, long long row, int head, int d, const float* x) {
    const size_t at = (size_t)(row * r.row_stride + head * r.head_stride + d);
    if (r.f32) {
        float* p = (float*)r.data + at;
        if (r.vec) {
            *(float4*)p = float4{x[0], x[1], x[2], x[3]};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = x[i];
        }
    } else {
        uint16_t* p = (uint16_t*)r.data + at;
        if (r.vec) {
            *(uint2*)p = uint2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = (uint16_t)f32_to_bf16(x[i]);
        }
    }
}

__device__ __forceinline__ void store8(const HeadRows& r, long long row, int head, int d, uint4 s) {   // eight bf16 numbers
    const uint32_t w[4] = {s.x, s.y, s.z, s.w};
    if (!r.f32 && r.vec) {
        *(uint4*)((uint16_t*)r.data + (size_t)(row * r.row_stride + head * r.head_stride + d)) = s;
        return;
    }
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    store4(r, row, head, d, x);
    store4(r, row, head, d + 4, x + 4);
}

// ---------------------------------------------------------------- writing rows
// One workgroup per page that a sequence's new rows touch, and KV head.  A thread takes 8 dims of a row: the keys go to
// their place at once, the values through LDS, where a lane's 8 keys of one dim meet.  e4m3: the row's power of two is the
// least by which no finite magnitude is over 448 (at least 2^-100); a row's codes hang on nothing but the row, so a
// row written alone and one written in a chunk are the same.  NaN and infinities become NaN, e4m3 has no others.
// Bounds: the least and largest stored key of each dim among the page's positions up to the last one written, rounded
// outwards to 8 bits; earlier positions are read back.  The bound scale of a page with a key that is not finite is +inf.
// A page per workgroup because its bounds are of all its positions: nobody else writes them.  8 x up to 512 rows, 8 heads, bf16 to e4m3
// (11 MB read, 6 MB written): 12.4 us, latency: three dependent turns, loads, LDS and the bounds' sums.  One token: 4.4 us.
struct KvSource {        // the rows to write: strided tensors, or the split block K/V of a pass
    HeadRows k, v;
    const uint16_t* blk_k;   // [unit][hi, lo][64][D]
    const uint16_t* blk_v;   // [unit][hi, lo][D][64]
};

template <int D>
__device__ __forceinline__ void load_kv8(const KvSource& src, bool value, long long row, int t, int b, int head, int heads, int d, float* x) {
    if (!src.blk_k) {
        load8(value ? src.v : src.k, row, head, d, x);
        return;
    }
    const size_t unit = (size_t)(b * heads + head) * 2 * 64 * D;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint16_t* p = value ? src.blk_v + unit + (d + i) * 64 + t : src.blk_k + unit + t * D + d + i;
        x[i] = bf16_to_f32(p[0]) + bf16_to_f32(p[64 * D]);
    }
}

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// four values as e4m3 numbers of x * 2^-e, at most `most`
__device__ __forceinline__ uint32_t four_e4m3(const float* x, float inv, float most) {
    uint32_t w = 0;
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = finite(x[i]) ? fminf(fmaxf(x[i] * inv, -most), most) : __uint_as_float(0x7FC00000u);
    w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], (int)w, false);
    w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], (int)w, true);
    return w;
}

// biased exponent of a row's power of two
__device__ __forceinline__ uint32_t row_exponent(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u);   // 448 = 1.75 * 2^8
    return (uint32_t)max(e, 27);
}

template <int D, bool E4M3>
__global__ void __launch_bounds__(256) pages_write_kernel(PageCache c, KvSource src, PageChunk ch, int touched, uint32_t* status) {
    constexpr int C = D / 8, TOK = 256 / C;   // threads per row, rows per turn
    using Elem = typename std::conditional<E4M3, uint8_t, uint16_t>::type;
    __shared__ __align__(16) Elem vt[64][D + (E4M3 ? 16 : 8)];
    __shared__ float red[2][TOK][D];
    __shared__ float top[4];
    __shared__ int bad;

    const int h = blockIdx.x % c.n_kv_heads, i = blockIdx.x / c.n_kv_heads % touched, b = blockIdx.x / c.n_kv_heads / touched;
    const int tid = threadIdx.x, chunk = tid % C, d0 = chunk * 8;
    const bool tell = h == 0 && i == 0 && tid == 0;
    const SeqRows sr = seq_rows(ch, b, tell ? status : nullptr);
    const int P = seq_length(c, b, tell && sr.n ? status : nullptr);
    if (tell && sr.n && P + sr.n > c.max_pages * 64) flag(status, ST_CAPACITY);
    const int page = P / 64 + i, end = min(min(P + sr.n, c.max_pages * 64) - page * 64, 64);   // positions of the page
    const int begin = max(P - page * 64, 0);
    if (begin >= end) return;
    const int id = page_id(c, b, page);
    if (id < 0) {
        if (tid == 0 && h == 0) flag(status, ST_PAGE);
        return;
    }
    const size_t head = (size_t)id * c.n_kv_heads + h;
    Elem* kp = (Elem*)c.k + head * 64 * D;
    Elem* vp = (Elem*)c.v + head * 64 * D;
    if (tid == 0) bad = 0;

    float lo[8], hi[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) lo[e] = INFINITY, hi[e] = -INFINITY;
    bool odd = false;   // a stored key that is not finite

    // every row of this thread is requested before any is worked on
    constexpr int TURNS = 64 / TOK;
    float rows[TURNS][2][8];
#pragma unroll
    for (int u = 0; u < TURNS; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int t = u * TOK + tid / C;
#pragma unroll
            for (int e = 0; e < 8; ++e) rows[u][w][e] = 0.0f;
            if (t >= begin && t < end) load_kv8<D>(src, w == 1, sr.r0 + (page * 64 + t - P), page * 64 + t - P, b, h, c.n_kv_heads, d0, rows[u][w]);
        }
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        const int t = u * TOK + tid / C;
        const bool there = t >= begin && t < end;
        float (&x)[2][8] = rows[u];
        float amax[2] = {0.0f, 0.0f};
        if constexpr (E4M3)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
#pragma unroll
                for (int e = 0; e < 8; ++e) amax[w] = fmaxf(amax[w], finite(x[w][e]) ? fabsf(x[w][e]) : 0.0f);
#pragma unroll
                for (int m = 1; m < C; m <<= 1) amax[w] = fmaxf(amax[w], __shfl_xor(amax[w], m));
            }
        if (!there) continue;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            if constexpr (E4M3) {
                const uint32_t ex = row_exponent(amax[w]);
                const float inv = __uint_as_float((254u - ex) << 23), sc = scale_of(ex);
                const float most = ex == 247u ? 240.0f : 448.0f;   // 256 * 2^120 would not be finite
                const uint2 q{four_e4m3(x[w], inv, most), four_e4m3(x[w] + 4, inv, most)};
                if (chunk == 0) c.scale[(head * 2 + w) * 64 + t] = (uint8_t)ex;
                if (w == 0) {
                    *(uint2*)(kp + key_at<D, true>(t, d0)) = q;
                    if (c.bounds) {
                        const uint4 s = eight_bf16(q.x, q.y, sc);
                        const uint32_t u[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float f = __uint_as_float(e & 1 ? u[e / 2] & 0xFFFF0000u : u[e / 2] << 16);
                            odd |= !finite(f);
                            lo[e] = fminf(lo[e], f), hi[e] = fmaxf(hi[e], f);
                        }
                    }
                } else {
                    *(uint2*)&vt[t][d0] = q;
                }
            } else {
                uint32_t u[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = pack_bf16x2(x[w][2 * e], x[w][2 * e + 1]);
                if (w == 0) {
                    *(uint4*)(kp + key_at<D, false>(t, d0)) = uint4{u[0], u[1], u[2], u[3]};
                    if (c.bounds) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float f = __uint_as_float(e & 1 ? u[e / 2] & 0xFFFF0000u : u[e / 2] << 16);
                            odd |= !finite(f);
                            lo[e] = fminf(lo[e], f), hi[e] = fmaxf(hi[e], f);
                        }
                    }
                } else {
                    *(uint4*)&vt[t][d0] = uint4{u[0], u[1], u[2], u[3]};
                }
            }
        }
    }
    __syncthreads();

    // values: a lane's 8 keys of one dim, whole where all of them are new
    for (int at = tid; at < 64 * D / 8; at += 256) {
        const int blk = at >> 6, kt = blk / (D / 16), d = blk % (D / 16) * 16 + (at & 15), s = (at >> 5) & 1, hf = (at >> 4) & 1;
        const int k0 = kt * 32 + value_key(s, hf, 0), k1 = kt * 32 + value_key(s, hf, 7);
        if (k1 < begin || k0 >= end) continue;
        Elem* to = vp + value_at<D, E4M3>(k0, d);
        if (k0 >= begin && k1 < end) {
            Elem g[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = vt[kt * 32 + value_key(s, hf, e)][d];
            if constexpr (E4M3)
                *(uint2*)to = uint2{(uint32_t)g[0] | (uint32_t)g[1] << 8 | (uint32_t)g[2] << 16 | (uint32_t)g[3] << 24,
                                    (uint32_t)g[4] | (uint32_t)g[5] << 8 | (uint32_t)g[6] << 16 | (uint32_t)g[7] << 24};
            else
                *(uint4*)to = uint4{(uint32_t)g[0] | (uint32_t)g[1] << 16, (uint32_t)g[2] | (uint32_t)g[3] << 16,
                                    (uint32_t)g[4] | (uint32_t)g[5] << 16, (uint32_t)g[6] | (uint32_t)g[7] << 16};
        } else {
            for (int e = 0; e < 8; ++e) {
                const int k = kt * 32 + value_key(s, hf, e);
                if (k >= begin && k < end) to[e] = vt[k][d];
            }
        }
    }
    if (!c.bounds) return;

    // earlier positions of the page, as they are stored
    for (int t = tid / C; t < begin; t += TOK) {
        uint32_t u[4];
        if constexpr (E4M3) {
            const uint2 q = *(const uint2*)(kp + key_at<D, true>(t, d0));
            const uint4 s = eight_bf16(q.x, q.y, scale_of(c.scale[head * 2 * 64 + t]));
            u[0] = s.x, u[1] = s.y, u[2] = s.z, u[3] = s.w;
        } else {
            const uint4 q = *(const uint4*)(kp + key_at<D, false>(t, d0));
            u[0] = q.x, u[1] = q.y, u[2] = q.z, u[3] = q.w;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float f = __uint_as_float(e & 1 ? u[e / 2] & 0xFFFF0000u : u[e / 2] << 16);
            odd |= !finite(f);
            lo[e] = fminf(lo[e], f), hi[e] = fmaxf(hi[e], f);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) red[0][tid / C][d0 + e] = lo[e], red[1][tid / C][d0 + e] = hi[e];
    if (odd) atomicOr(&bad, 1);
    __syncthreads();
    float a = 0.0f, l = 0.0f, g = 0.0f;
    if (tid < D) {
        l = red[0][0][tid], g = red[1][0][tid];
        for (int r = 1; r < TOK; ++r) l = fminf(l, red[0][r][tid]), g = fmaxf(g, red[1][r][tid]);
        a = fmaxf(fabsf(l), fabsf(g));
    }
    for (int m = 32; m; m >>= 1) a = fmaxf(a, __shfl_xor(a, m));
    if ((tid & 63) == 0) top[tid >> 6] = a;
    __syncthreads();
    if (tid >= D) return;
    a = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    const float sc = bad ? INFINITY : a / 127.0f, by = sc > 0.0f ? sc : 1.0f;
    int8_t* bd = c.bounds + head * 2 * D;
    bd[tid] = bad ? 0 : (int8_t)fmaxf(-127.0f, fminf(127.0f, floorf(l / by)));
    bd[D + tid] = bad ? 0 : (int8_t)fmaxf(-127.0f, fminf(127.0f, ceilf(g / by)));
    if (tid == 0) c.bound_scale[head] = sc;
}

// ---------------------------------------------------------------- reading rows
// One workgroup per page that the positions first[b] .. first[b] + n_b touch, and KV head.  Every stored value is a bf16
// number, also a scaled 8-bit one, so rows of either type are exact.  Bound by memory: 8 x up to 16384 positions, 8 heads, e4m3 to bf16,
// 154 MB read and 304 written in 96 us, 4.8 TB/s (a large copy: 4.9).
template <int D, bool E4M3>
__global__ void __launch_bounds__(256) pages_read_kernel(PageCache c, HeadRows k, HeadRows v, PageChunk ch, const int32_t* first, int touched,
                                                         uint32_t* status) {
    using Elem = typename std::conditional<E4M3, uint8_t, uint16_t>::type;
    constexpr int C = D / 8, TOK = 256 / C;
    __shared__ __align__(16) uint16_t vt[64][D + 8];
    const int h = blockIdx.x % c.n_kv_heads, i = blockIdx.x / c.n_kv_heads % touched, b = blockIdx.x / c.n_kv_heads / touched;
    const int tid = threadIdx.x, d0 = tid % C * 8;
    const bool tell = h == 0 && i == 0 && tid == 0;
    const SeqRows sr = seq_rows(ch, b, tell ? status : nullptr);
    int P = first ? first[b] : 0;
    if (P < 0) {
        if (tell && sr.n) flag(status, ST_LENGTH);
        return;
    }
    P = min(P, c.max_pages * 64);
    if (tell && P + sr.n > c.max_pages * 64) flag(status, ST_CAPACITY);
    const int page = P / 64 + i, end = min(min(P + sr.n, c.max_pages * 64) - page * 64, 64), begin = max(P - page * 64, 0);
    if (begin >= end) return;
    const int id = page_id(c, b, page);
    if (id < 0) {
        if (tid == 0 && h == 0) flag(status, ST_PAGE);
        return;
    }
    const size_t head = (size_t)id * c.n_kv_heads + h;
    const Elem* kp = (const Elem*)c.k + head * 64 * D;
    const Elem* vp = (const Elem*)c.v + head * 64 * D;
    const long long row0 = sr.r0 + (page * 64 - P);   // row of the page's first position

    // everything is requested before any of it is worked on
    constexpr int PIECES = 64 * D / 8 / 256, TURNS = 64 / TOK;
    uint4 vq[PIECES], kq[TURNS];
    uint32_t vs[PIECES][2], ks[TURNS];
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
        const int at = tid + u * 256, blk = at >> 6, kt = blk / (D / 16), d = blk % (D / 16) * 16 + (at & 15), s = (at >> 5) & 1, hf = (at >> 4) & 1;
        const int k0 = kt * 32 + value_key(s, hf, 0);
        if constexpr (E4M3) {
            const uint2 q = *(const uint2*)(vp + value_at<D, true>(k0, d));
            vq[u] = uint4{q.x, q.y, 0u, 0u};
            const uint32_t* sc = (const uint32_t*)(c.scale + (head * 2 + 1) * 64 + k0);
            vs[u][0] = sc[0], vs[u][1] = sc[2];
        } else {
            vq[u] = *(const uint4*)(vp + value_at<D, false>(k0, d));
        }
    }
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        const int t = u * TOK + tid / C;
        if (t < begin || t >= end) continue;
        if constexpr (E4M3) {
            const uint2 q = *(const uint2*)(kp + key_at<D, true>(t, d0));
            kq[u] = uint4{q.x, q.y, 0u, 0u};
            ks[u] = c.scale[head * 2 * 64 + t];
        } else {
            kq[u] = *(const uint4*)(kp + key_at<D, false>(t, d0));
        }
    }
#pragma unroll
    for (int u = 0; u < PIECES; ++u) {
        const int at = tid + u * 256, blk = at >> 6, kt = blk / (D / 16), d = blk % (D / 16) * 16 + (at & 15), s = (at >> 5) & 1, hf = (at >> 4) & 1;
        const uint32_t w[4] = {vq[u].x, vq[u].y, vq[u].z, vq[u].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t x;
            if constexpr (E4M3) x = pair_bf16<false>((w[e / 4] >> (8 * (e & 3))) & 0xFFu, scale_of((vs[u][e / 4] >> (8 * (e & 3))) & 0xFFu));
            else x = w[e / 2] >> (16 * (e & 1));
            vt[kt * 32 + value_key(s, hf, e)][d] = (uint16_t)x;
        }
    }
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        const int t = u * TOK + tid / C;
        if (t < begin || t >= end) continue;
        uint4 s = kq[u];
        if constexpr (E4M3) s = eight_bf16(s.x, s.y, scale_of(ks[u]));
        store8(k, row0 + t, h, d0, s);
    }
    __syncthreads();
    for (int t = begin + tid / C; t < end; t += TOK) {
        store8(v, row0 + t, h, d0, *(const uint4*)&vt[t][d0]);
    }
}

// ---------------------------------------------------------------- work of the attention
// An entry is a block of a sequence's rows: block_rows rows (token, query head of the group) of a KV head, or the
// rows of a group of tokens that share a list of pages.  A unit is an entry and a KV head; its work is counted in steps of
// 8 KB of keys and 8 KB of values at 128 dims (32 bf16 positions, 64 in 8 bits).  All units' steps, one behind the other, are cut into
// equal shares, one per workgroup, whatever the lengths are: the committed lengths live on the device, so the kernels work
// the shares out themselves, and a unit that lies in one share is finished there.  The others' parts meet in a second launch.
struct Entry {
    int b, blk;         // sequence, block of its rows
    int r0, n, P;       // packed rows, committed length
    int t0, t1;         // its tokens (first, past the last)
    int rows0, rows1;   // its rows (t * G + g)
    int steps;          // per KV head
};

template <int STEP>
__device__ __forceinline__ Entry entry_of(const PagesAttnArgs& a, int e, uint32_t* status) {
    Entry x;
    x.b = e / a.n_blk;
    x.blk = e % a.n_blk;
    const SeqRows sr = seq_rows(a.ch, x.b, status);
    x.r0 = sr.r0, x.n = sr.n;
    x.P = seq_length(a.c, x.b, sr.n ? status : nullptr);
    const int G = a.group_heads;
    if (a.list) {
        x.t0 = min(x.blk * a.group, x.n), x.t1 = min(x.t0 + a.group, x.n);
        x.rows0 = x.t0 * G, x.rows1 = x.t1 * G;
    } else {
        x.rows0 = min(x.blk * a.block_rows, x.n * G), x.rows1 = min(x.rows0 + a.block_rows, x.n * G);
        x.t0 = x.rows0 / G, x.t1 = (x.rows1 + G - 1) / G;
    }
    x.steps = 0;
    if (x.rows1 > x.rows0) {
        const int sees = a.draft && x.t1 > a.bidir_from ? x.n : x.t1;
        if (status && x.P + sees > a.c.max_pages * 64) flag(status, ST_CAPACITY);
        x.steps = a.list ? a.n_list * (64 / STEP) : (min(x.P + sees, a.c.max_pages * 64) + STEP - 1) / STEP;
    }
    return x;
}

// how many positions a token sees
__device__ __forceinline__ int sees_of(const PagesAttnArgs& a, int P, int n, int t) {
    return min(P + (a.draft && t >= a.bidir_from ? n : t + 1), a.c.max_pages * 64);
}

__device__ __forceinline__ long long block_sum(long long v, long long* lds) {
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int i = 0; i < (int)blockDim.x / 64; ++i) v += lds[i];
    return v;
}

struct Share {
    long long total;   // steps of all units
    int wgs;           // shares
    __device__ long long begin(int w) const { return total * w / wgs; }
    // the share that step s is in
    __device__ int of(long long s) const {
        int w = (int)(s * wgs / total);
        while (w + 1 < wgs && begin(w + 1) <= s) ++w;
        while (begin(w) > s) --w;
        return w;
    }
};
// shares of `total` steps, of `units` units: at least `least` steps each, but not fewer shares than units
__device__ __forceinline__ Share share_of(long long total, long long units, int grid, int least) {
    return Share{total, (int)max(1LL, min((long long)grid, max(units, total / least)))};
}

// Sum of all entries' steps (per KV head), and the number of entries that have rows.
template <int STEP>
__device__ __forceinline__ void sum_entries(const PagesAttnArgs& a, long long* lds, long long* all, long long* live, uint32_t* status) {
    long long mine = 0, some = 0;
    for (int e = threadIdx.x; e < a.n_entries; e += blockDim.x) {
        const int s = entry_of<STEP>(a, e, status).steps;
        mine += s;
        some += s > 0;
    }
    *all = block_sum(mine, lds);
    *live = block_sum(some, lds);
}

// A workgroup's way through its share.  Steps are numbered KV head by KV head, in each entry by entry: with the shares of one
// XCD side by side (workgroup w runs on XCD w % 8) the workgroups that read the same keys mostly share an L2.  What hangs on lengths and
// row_start is looked up by one thread and handed to the others, so that all go the same way whatever is written to these meanwhile.
struct Walk {
    Entry en;
    int e, h, share;
    long long at, last;   // the share's steps left: [at, last)
    long long before;     // steps of the entries before e
    long long per_head, live;
    bool first_unit;
    bool odd, careful;    // the present unit has sums that are not finite; it is worked on a second time
};

// inclusive sum over the workgroup's threads, and over all of them
__device__ __forceinline__ long long block_scan(long long v, long long* lds, long long* all) {
    for (int m = 1; m < 64; m <<= 1) {
        const long long o = __shfl_up(v, m);
        if ((int)(threadIdx.x & 63) >= m) v += o;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 63) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    long long sum = 0;
    for (int i = 0; i < (int)blockDim.x / 64; ++i) {
        if (i < (int)threadIdx.x / 64) v += lds[i];
        sum += lds[i];
    }
    *all = sum;
    return v;
}

// false: nothing to do.  Up to as many entries as threads are looked at once, all of them side by side.
template <int STEP>
__device__ __forceinline__ bool walk_start(const PagesAttnArgs& a, Walk* w, long long* lds) {
    const int heads = a.c.n_kv_heads;
    uint32_t* status = blockIdx.x == 0 ? a.status : nullptr;
    const bool once = a.n_entries <= (int)blockDim.x;
    Entry en{};
    if ((int)threadIdx.x < a.n_entries) en = entry_of<STEP>(a, threadIdx.x, status);
    constexpr long long LIVE = 1LL << 40;   // the entries that have rows are counted above the steps, of which 512 entries have at most 2^34
    long long per_head, live, upto = 0;
    if (once) {
        upto = block_scan(en.steps + (en.steps > 0 ? LIVE : 0), lds, &per_head);
        live = per_head >> 40;
        per_head &= LIVE - 1, upto &= LIVE - 1;
    } else {
        sum_entries<STEP>(a, lds, &per_head, &live, status);
    }
    if (per_head == 0) return false;
    const Share sh = share_of(per_head * heads, live * heads, gridDim.x, a.least_steps);
    // the shares in use, dealt to the XCDs in eight runs of adjacent ones
    const int run = sh.wgs / 8, x = blockIdx.x & 7, i = blockIdx.x >> 3;
    const int share = i < run ? x * run + i : (int)blockIdx.x;
    if (share >= sh.wgs) return false;
    const long long first = sh.begin(share);
    const int h = (int)(first / per_head);
    const long long s = first - h * per_head;
    if (threadIdx.x == 0) {
        w->e = a.n_entries;
        w->h = h, w->share = share, w->at = first, w->last = sh.begin(share + 1), w->per_head = per_head, w->live = live, w->first_unit = true;
        w->odd = w->careful = false;
    }
    // the entry that holds step s of its KV head
    __syncthreads();
    if (once) {
        if (s < upto && s >= upto - en.steps) w->en = en, w->e = threadIdx.x, w->before = upto - en.steps;
    } else {
        long long base = 0;
        for (int e0 = 0;; e0 += blockDim.x) {
            const int e = e0 + threadIdx.x;
            const Entry x2 = e < a.n_entries ? entry_of<STEP>(a, e, nullptr) : Entry{};
            long long sum;
            const long long to = base + block_scan(x2.steps, lds, &sum);
            if (s < to && s >= to - x2.steps) w->en = x2, w->e = e, w->before = to - x2.steps;
            base += sum;
            __syncthreads();
            if (w->e < a.n_entries || e0 + (int)blockDim.x >= a.n_entries) break;
        }
    }
    __syncthreads();
    return w->e < a.n_entries;   // false not unless the lengths change meanwhile
}

// The present unit, in scalar registers.
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
struct Unit {
    Entry en;
    int h, s0, s1, slot;   // KV head; steps [s0, s1) are this workgroup's; place of its part
    bool whole, careful;
};
__device__ __forceinline__ Unit walk_unit(const Walk& w) {
    Unit u;
    const Entry& e = w.en;
    u.en = Entry{scalar(e.b), scalar(e.blk), scalar(e.r0), scalar(e.n), scalar(e.P), scalar(e.t0), scalar(e.t1), scalar(e.rows0), scalar(e.rows1), scalar(e.steps)};
    u.h = scalar(w.h);
    const long long unit0 = w.h * w.per_head + w.before;
    u.s0 = scalar((int)(w.at - unit0));
    u.s1 = scalar((int)min(w.last - unit0, (long long)e.steps));
    u.slot = 2 * scalar(w.share) + (scalar(w.first_unit) ? 0 : 1);
    u.whole = u.s0 == 0 && u.s1 == u.en.steps;
    u.careful = scalar(w.careful) != 0;
    return u;
}

// What the second launch needs of a unit, from the workgroup that has its last step: the place of its first part (bit 31: it is not that
// workgroup's first), and how many parts there are.
__device__ __forceinline__ void note_parts(const PagesAttnArgs& a, const Walk& w, const Unit& u) {
    if (threadIdx.x != 0 || u.s1 != u.en.steps) return;
    int w0 = w.share, n = 1;
    bool later = false;
    if (!u.whole) {
        const Share sh = share_of(w.per_head * a.c.n_kv_heads, w.live * a.c.n_kv_heads, gridDim.x, a.least_steps);
        const long long u0 = w.h * w.per_head + w.before;
        w0 = sh.of(u0), n = w.share - w0 + 1, later = u0 > sh.begin(w0);
    }
    a.parts[(size_t)w.e * a.c.n_kv_heads + u.h] = uint2{(uint32_t)w0 | (later ? 0x80000000u : 0u), (uint32_t)n};
}

// On to the next unit, or to a second pass over this one; false behind the last.  Called by every thread after it has read what it needs of the present one.
template <int STEP>
__device__ __forceinline__ bool walk_next(const PagesAttnArgs& a, Walk* w) {
    __syncthreads();
    if (threadIdx.x == 0 && w->odd && !w->careful) {
        w->careful = true;
    } else if (threadIdx.x == 0) {
        w->odd = w->careful = false;
        w->at = w->h * w->per_head + w->before + w->en.steps;
        w->first_unit = false;
        w->before += w->en.steps;
        while (w->at < w->last) {
            if (++w->e >= a.n_entries) {
                ++w->h, w->e = 0, w->before = 0;
                if (w->h >= a.c.n_kv_heads) {   // not unless the lengths change meanwhile
                    w->at = w->last;
                    break;
                }
            }
            w->en = entry_of<STEP>(a, w->e, nullptr);
            if (w->en.steps > 0) break;
        }
    }
    __syncthreads();
    return w->at < w->last;
}

// four dims of a finished row (token t of sequence b, query head), and its log-sum-exp: a row that sees nothing is 0
template <int D>
__device__ __forceinline__ void finish_row(const PagesAttnArgs& a, int b, int r0, int n, int t, int head, int d, float m, float l, const float* x) {
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = x[i] * by;
    if (a.o_split) {
        const size_t at = split_index(b * n + t, head * D + d, a.o_ksteps);
#pragma unroll
        for (int i = 0; i < 4; ++i) store_split(a.o_split, at + i, y[i], a.plain_o);
    } else {
        store4(a.out, r0 + t, head, d, y);
    }
    if (a.lse && d == 0) a.lse[(size_t)(r0 + t) * (a.group_heads * a.c.n_kv_heads) + head] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * 0.693147180559945309f;
}

// ---------------------------------------------------------------- attention
// A workgroup of 4 wavefronts walks its share unit by unit, with one tile of RW rows; each takes every fourth step.  A step's keys and values go straight from memory to the registers of the wavefront, in operand
// order; while a step is worked on, the next one's are under way.  Running
// maximum and sum per row in base-2 exponents; the weights are carried in two bf16 pieces (three for f32 queries, which are
// split likewise), so that P V is as exact as the f32 sums.  A unit's wavefronts meet in LDS at its end.
// Positions that a row does not see have weight 0; a value there that is not finite must not reach the row, and 0 times it
// would: in steps that some row of the tile does not see whole, values behind every row's last position count as 0, and any
// other that is not finite is left out of the product and added to the rows that see it.  In the other steps nobody looks: such a value
// leaves the sums not finite, infinite ones as NaN, since a weight's smaller pieces may be 0 or negative.  Sums that are not finite
// at the end are worked out once more (`careful`), with all values looked at as above, and infinite keys taken out of the products and
// added likewise where queries are in pieces.  So an infinite value comes out as what it is wherever it stands, and a score of -inf has
// weight 0.  Nothing is worked out twice where weights are one piece, or over 8-bit pages, which hold no infinity: NaN comes out as NaN at once.
template <int RW>
struct Tile;
template <>
struct Tile<32> {
    typedef f32x16_t Acc;
    static constexpr int REGS = 16, DIMS = 16;   // accumulators of a tile, dims of one step of the first product
    static __device__ __forceinline__ Acc mfma(uint4 a, uint4 b, Acc c) { return mfma_32x32x16(a, b, c); }
    static __device__ __forceinline__ int piece_s(int lane, int f) { return f & 1; }   // of the f-th eight weights
    static __device__ __forceinline__ int piece_hf(int lane) { return lane >> 5; }
    static __device__ __forceinline__ int out_dim(int lane, int r) { return 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3); }
    // over the lanes of a row, in every one of them
    template <typename F>
    static __device__ __forceinline__ float across(float v, F f) {
        const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    }
};
template <>
struct Tile<16> {
    typedef f32x4_t Acc;
    static constexpr int REGS = 4, DIMS = 32;
    static __device__ __forceinline__ Acc mfma(uint4 a, uint4 b, Acc c) { return mfma_16x16x32(a, b, c); }
    static __device__ __forceinline__ int piece_s(int lane, int f) { return lane >> 5; }
    static __device__ __forceinline__ int piece_hf(int lane) { return (lane >> 4) & 1; }
    static __device__ __forceinline__ int out_dim(int lane, int r) { return 4 * (lane >> 4) + r; }
    template <typename F>
    static __device__ __forceinline__ float across(float v, F f) {
        v = Tile<32>::across(v, f);
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    }
};

// A row's maximum follows its scores (in base-2 exponents) once they are 2^8 above it: until then the weights are up to 2^8, which costs
// sums in f32 and weights in bf16 nothing, and the sums so far need no new scale.
template <typename Acc, int N>
__device__ __forceinline__ void rescale(float top, float* m, float* l, Acc (&o)[N]) {
    if (!__any(top > *m + 8.0f)) return;
    const float to = fmaxf(*m, top), f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(*m - to);
    *l *= f;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] *= f;
    *m = to;
}
__device__ __forceinline__ float weight(float score, float scale_log2, float ref) { return __builtin_amdgcn_exp2f(__builtin_fmaf(score, scale_log2, -ref)); }

// Puts 0 in the place of the infinities among eight bf16 numbers; whether there were any.
__device__ __forceinline__ bool no_infinity(uint4* x) {
    uint32_t w[4] = {x->x, x->y, x->z, x->w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x7FFFu) == 0x7F80u) w[i] &= 0xFFFF0000u;
        if ((w[i] & 0x7FFF0000u) == 0x7F800000u) w[i] &= 0xFFFFu;
    }
    const bool some = ((w[0] ^ x->x) | (w[1] ^ x->y) | (w[2] ^ x->z) | (w[3] ^ x->w)) != 0u;
    *x = uint4{w[0], w[1], w[2], w[3]};
    return some;
}
template <typename Acc, int N>
__device__ __forceinline__ bool any_not_finite(const Acc (&o)[N]) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int r = 0; r < (int)(sizeof(Acc) / 4); ++r) t = __builtin_fmaf(o[i][r], 0.0f, t);   // NaN, once one is not finite
    return __any(t != t);
}

// Adds to a lane's scores x what infinite bf16 keys give them, with whole queries.
template <int D, int NQ, int N, typename F>
__device__ __forceinline__ void add_infinite_keys(const PagesAttnArgs& a, float (&x)[N], F key_of, const uint16_t* keys, int first, const Entry& en, int h, int t,
                                                    int g, bool have) {
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
        float sum = 0.0f;
        for (int d0 = 0; d0 < D; d0 += 8) {
            uint4 eight = *(const uint4*)(keys + key_at<D, false>(first + key_of(i), d0));
            if (!no_infinity(&eight) || !have) continue;
#pragma unroll 1
            for (int d = d0; d < d0 + 8; ++d) {
                const float k = bf16_to_f32(keys[key_at<D, false>(first + key_of(i), d)]);
                if (fabsf(k) != INFINITY) continue;
                float q;
                if constexpr (NQ == 2) {
                    const uint16_t* p = a.q_split + q_index(en.b * a.c.n_kv_heads + h, g * en.n + t, d, a.q_row_tiles, D);
                    q = bf16_to_f32(p[0]) + bf16_to_f32(p[SPLIT_LO]);
                } else {
                    q = ((const float*)a.q.data)[(en.r0 + t) * a.q.row_stride + (h * a.group_heads + g) * a.q.head_stride + d];
                    if (a.negate) q = -q;
                }
                sum += q * k;
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] += j == i ? sum : 0.0f;
    }
}

// A lane's queries as operands, eight dims from dim_of(step) on: a row's bf16 pieces (one, a pass's two, three of f32), 0 for a row that there is not.
template <int D, int NQ, int QS, typename F>
__device__ __forceinline__ void load_queries(const PagesAttnArgs& a, const Entry& en, int h, int t, int g, bool have, uint4 (&q)[NQ][QS], F dim_of) {
#pragma unroll
    for (int s = 0; s < QS; ++s) {
        const int d = dim_of(s);
        if constexpr (NQ == 2) {   // rows (query head, block row)
            q[0][s] = q[1][s] = uint4{0u, 0u, 0u, 0u};
            if (have) {
                const uint16_t* p = a.q_split + q_index(en.b * a.c.n_kv_heads + h, g * en.n + t, d, a.q_row_tiles, D);
                q[0][s] = *(const uint4*)p;
                q[1][s] = *(const uint4*)(p + SPLIT_LO);
            }
        } else {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
            if (have) load8(a.q, en.r0 + t, h * a.group_heads + g, d, x);
            if (a.negate)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = -x[i];
#pragma unroll
            for (int p = 0; p < NQ; ++p) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
                    x[2 * i] -= bf16_to_f32(w[i] & 0xFFFFu), x[2 * i + 1] -= __uint_as_float(w[i] & 0xFFFF0000u);
                }
                q[p][s] = uint4{w[0], w[1], w[2], w[3]};
            }
        }
    }
}

template <int D, bool E4M3, int RW>
__device__ __forceinline__ void add_not_finite(typename Tile<RW>::Acc* o, const void* values, int base, int lane, int sees, int most) {
    using Elem = typename std::conditional<E4M3, uint8_t, uint16_t>::type;
    const Elem* v = (const Elem*)values;
    for (int key = 0; key < (E4M3 ? 64 : 32); ++key) {
        const int pos = base + key;
        if (pos >= most) break;
        const int slot = pos & 63;
#pragma unroll
        for (int dt = 0; dt < D / RW; ++dt)
#pragma unroll
            for (int r = 0; r < Tile<RW>::REGS; ++r) {
                const uint32_t w = v[value_at<D, E4M3>(slot, dt * RW + Tile<RW>::out_dim(lane, r))];
                const float f = E4M3 ? ((w & 0x7Fu) == 0x7Fu ? __uint_as_float(0x7FC00000u) : 0.0f) : bf16_to_f32(w);
                if (!finite(f) && pos < sees) o[dt][r] += f;
            }
    }
}

// Few rows, up to one tile of 16 or 32 of a KV head: one pass over a share's pages with each row's running maximum and sum, the steps dealt to
// four wavefronts that meet at the unit's end through LDS.  Bound by memory: every page is read once, straight to registers, where its
// layout makes it an operand, and a wavefront asks for its next step's keys and values before it works on this one's.
// bf16 queries: two pieces of the weights, at most 2^-16 of each, since memory and not the products bounds this kernel; f32 queries: three pieces of both.
// One token of 32 sequences of up to 8192 positions, 32 query heads, e4m3 (297 MB): 59 us, 5.1 TB/s of the 6.5 that plain reads reach, and 73
// with the second launch and the gap between the two; one token over 4096 positions, bf16 (17 MB): 15 us of latency, 21.7 with the second.
template <int D, bool E4M3, int NQ, int RW>   // NQ: bf16 pieces of a query (1: bf16, 2: split, 3: f32); RW: rows of a tile
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(RW == 16 || NQ == 1 && !(E4M3 && D == 128) ? 2 : 1)))
pages_attend_kernel(PagesAttnArgs a) {
    using T = Tile<RW>;
    constexpr int STEP = E4M3 ? 64 : 32, KT = STEP / 32, NP = NQ == 3 ? 3 : 2;
    constexpr int NL = D / 16;                   // 16-byte loads per lane of a step's keys, and of its values
    constexpr int QS = D / T::DIMS;              // steps of the first product
    constexpr int SR = STEP * RW / 64;           // scores per lane
    constexpr int NF = SR / 8;                   // eights of weights: one operand each
    constexpr int DT = D / RW;
    constexpr int PITCH = D + 4;
    constexpr bool TWICE = !E4M3 && NP > 1;            // sums that are not finite are worked out once more
    constexpr bool PIECES_OF_KEYS = NQ > 1 && !E4M3;   // and infinite keys by themselves
    __shared__ __align__(16) float so[4][RW][PITCH];
    __shared__ float sml[4][RW][2];
    __shared__ long long lds[4];
    __shared__ Walk walk;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = lane % RW, part = lane / RW;
    constexpr int N_KS = 4;   // wavefronts
    const int heads = a.c.n_kv_heads, G = a.group_heads;

    if (!walk_start<STEP>(a, &walk, lds)) return;

    // places of a lane's 16 bytes in the blocks of keys and of values
    const int m32 = 8 * ((row >> 4) & 1) + (row & 7), k_lane = RW == 16 ? lane : ((row >> 3) & 1) * (D / (E4M3 ? 64 : 32)) * 64 + part * 16 + m32;
    const int v_lane = RW == 16 ? lane : (row >> 4) * 64 + part * 16 + (row & 15);
    const int key_of_row = RW == 16 ? 16 * (row >> 3) + (row & 7) : row;   // of a tile's first keys

    do {
        const Unit unit = walk_unit(walk);
        const Entry& en = unit.en;
        const int h = unit.h, s0 = unit.s0, s1 = unit.s1, slot = unit.slot;
        const bool whole = unit.whole, careful = TWICE && unit.careful;

        // this wavefront's rows
        const int myrow = en.rows0 + row;
        const bool have = myrow < en.rows1;
        const int t = have ? myrow / G : 0, g = have ? myrow % G : 0;
        const int sees = have ? sees_of(a, en.P, en.n, t) : 0;
        int least = have ? sees : 0x7FFFFFFF, most = sees;
        for (int m = RW / 2; m; m >>= 1) least = min(least, __shfl_xor(least, m)), most = max(most, __shfl_xor(most, m));
        least = __builtin_amdgcn_readfirstlane(least), most = __builtin_amdgcn_readfirstlane(most);

        typename T::Acc o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < T::REGS; ++r) o[dt][r] = 0.0f;
        float m_run = -INFINITY, l_run = 0.0f;

        // the unit's pages: lane i of the window holds the place and the id of page win + i
        const int32_t* list = a.list ? a.list + ((size_t)(en.b * a.n_blk + en.blk) * heads + h) * a.n_list : nullptr;
        int win = -1, w_page = -1, w_id = -1;
        int s = s0 + wave;
        int base = 0;          // first position of the step
        size_t head = 0;       // page and KV head
        // The next step that has keys for this wavefront, its position and page; false behind the last.
        auto next = [&]() -> bool {
            for (; s < s1; s += N_KS) {
                const int pg = s * STEP >> 6;
                if (win < 0 || pg >= win + 64) {
                    win = pg;
                    const int i = pg + lane;
                    w_page = i * (64 / STEP) < s1 ? (list ? list[i] : i) : -1;
                    w_id = w_page >= 0 && w_page < a.c.max_pages ? a.c.table[(size_t)en.b * a.c.max_pages + w_page] : -1;
                    const bool bad = w_page >= a.c.max_pages || w_page < -1 || (w_page >= 0 && (unsigned)w_id >= (unsigned)a.c.n_pages);
                    if (bad) {
                        // a page that no row sees may be one that the sequence does not have yet
                        if (w_page < -1 || w_page * 64LL < most) flag(a.status, ST_PAGE);
                        w_id = -1;
                    }
                }
                const int page = __builtin_amdgcn_readlane(w_page, pg - win), id = __builtin_amdgcn_readlane(w_id, pg - win);
                if (id < 0 || page * 64 + (s * STEP & 63) >= most) continue;
                base = page * 64 + (s * STEP & 63);
                head = (size_t)id * heads + h;
                s += N_KS;
                return true;
            }
            return false;
        };
        uint4 kf[NL], vf[NL];
        uint32_t ksc[STEP / RW], vsc[SR / 4];
        // load i: RW 16: block i.  RW 32: keys (e4m3: group of 32,) block of dims, which half of its pieces; values: dims 32 (i / 2) .., keys 16 (i % 2) ..
        auto load_k = [&](size_t hd, int bs) {
            const uint4* p = (const uint4*)((const char*)a.c.k + hd * 64 * D * (E4M3 ? 1 : 2) + (E4M3 ? 0 : (bs & 32) * D * 2)) + k_lane;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                constexpr int B = D / (E4M3 ? 64 : 32);   // blocks of a tile of 16 keys
                kf[i] = p[RW == 16 ? i * 64 : (i / (2 * B)) * 2 * B * 64 + (i % (2 * B) >> 1) * 64 + (i & 1) * 32];
            }
            if constexpr (E4M3) {
#pragma unroll
                for (int i = 0; i < STEP / RW; ++i) ksc[i] = a.c.scale[hd * 128 + (RW == 16 ? (i >> 1) * 32 + (i & 1) * 8 : i * 32) + key_of_row];
            }
        };
        auto load_v = [&](size_t hd, int bs) {
            const uint4* p = (const uint4*)((const char*)a.c.v + hd * 64 * D * (E4M3 ? 1 : 2) + (E4M3 ? 0 : (bs & 32) * D * 2)) + v_lane;
#pragma unroll
            for (int i = 0; i < NL; ++i) vf[i] = p[RW == 16 ? i * 64 : (i >> 1) * 128 + (i & 1) * 32];
            if constexpr (E4M3) {
#pragma unroll
                for (int i = 0; i < SR / 4; ++i)
                    vsc[i] = *(const uint32_t*)(a.c.scale + hd * 128 + 64 + (i / (RW / 8)) * 32 + value_key(T::piece_s(lane, i >> 1), T::piece_hf(lane), 4 * (i & 1)));
            }
        };
        // position, in the step, of a lane's score i
        auto key_of = [&](int i) { return (i / (RW / 2)) * 32 + value_key(T::piece_s(lane, i >> 3), T::piece_hf(lane), i & 7); };

        bool more = next();
        int cur_base = base;
        size_t cur_head = head;
        if (more) {
            load_k(cur_head, cur_base);
            load_v(cur_head, cur_base);
        }
        // the queries, while the first pages are under way: the keys' blocks have a lane's bytes in pieces of 8 dims (bf16) or of 16, two steps
        uint4 q[NQ][QS];
        load_queries<D, NQ>(a, en, h, t, g, have, q, [&](int s) { return E4M3 ? 2 * T::DIMS * (s >> 1) + 16 * part + 8 * (s & 1) : T::DIMS * s + 8 * part; });

        while (more) {
            float x[SR];
            bool odd_keys = false;
            if (PIECES_OF_KEYS && careful)
#pragma unroll
                for (int i = 0; i < NL; ++i) odd_keys |= no_infinity(&kf[i]);
#pragma unroll
            for (int i = 0; i < STEP / RW; ++i) {   // tiles of RW keys
                typename T::Acc sc;
#pragma unroll
                for (int r = 0; r < T::REGS; ++r) sc[r] = 0.0f;
                // the small pieces first
#pragma unroll
                for (int p = NQ - 1; p >= 0; --p)
#pragma unroll
                    for (int j = 0; j < QS; ++j) {
                        uint4 k;
                        if constexpr (E4M3) {
                            const uint4 w = kf[i * (QS / 2) + j / 2];
                            k = j & 1 ? eight_bf16(w.z, w.w, scale_of(ksc[i])) : eight_bf16(w.x, w.y, scale_of(ksc[i]));
                        } else {
                            k = kf[i * QS + j];
                        }
                        sc = T::mfma(k, q[p][j], sc);
                    }
#pragma unroll
                for (int r = 0; r < T::REGS; ++r) x[i * T::REGS + r] = sc[r];
            }
            if (PIECES_OF_KEYS && __any(odd_keys)) add_infinite_keys<D, NQ>(a, x, key_of, (const uint16_t*)a.c.k + cur_head * 64 * D, cur_base & 63, en, h, t, g, have);
            const bool masked = careful || cur_base + STEP > least;
            more = next();
            if (more) load_k(head, base);

            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < SR; ++i) {
                if (masked && cur_base + key_of(i) >= sees) x[i] = -INFINITY;
                top = fmaxf(top, x[i]);
            }
            rescale(T::across(top, [](float u, float w) { return fmaxf(u, w); }) * a.scale_log2, &m_run, &l_run, o);
            const float ref = m_run == -INFINITY ? 0.0f : m_run;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < SR; ++i) {
                float p = weight(x[i], a.scale_log2, ref);
                sum += p;
                if constexpr (E4M3) {
                    const float w = scale_of((vsc[i >> 2] >> (8 * (i & 3))) & 0xFFu);
                    p = p > 0.0f || p != p ? p * w : 0.0f;   // scales of empty places may be anything
                }
                x[i] = p;
            }
            l_run += sum;

            bool odd = false;
            if (masked) {
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    uint32_t w[4] = {vf[i].x, vf[i].y, vf[i].z, vf[i].w};
                    const int ps = RW == 16 ? T::piece_s(lane, 0) : i & 1, ph = T::piece_hf(lane);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if constexpr (E4M3) {   // four keys of the group of 32 j / 2
                            const int pos = cur_base + (j >> 1) * 32 + value_key(ps, ph, 4 * (j & 1));
#pragma unroll
                            for (int b = 0; b < 4; ++b)
                                if (pos + b >= most || ((w[j] >> (8 * b)) & 0x7Fu) == 0x7Fu) {
                                    odd |= pos + b < most;
                                    w[j] &= ~(0xFFu << (8 * b));
                                }
                        } else {
                            const int pos = cur_base + value_key(ps, ph, 2 * j);
#pragma unroll
                            for (int b = 0; b < 2; ++b)
                                if (pos + b >= most || ((w[j] >> (16 * b)) & 0x7F80u) == 0x7F80u) {
                                    odd |= pos + b < most;
                                    w[j] &= ~(0xFFFFu << (16 * b));
                                }
                        }
                    }
                    vf[i] = uint4{w[0], w[1], w[2], w[3]};
                }
            }

#pragma unroll
            for (int f = 0; f < NF; ++f) {
                uint4 pf[NP];
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    uint32_t w[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float* y = x + f * 8 + 2 * i;
                        w[i] = pack_bf16x2(y[0], y[1]);
                        y[0] -= bf16_to_f32(w[i] & 0xFFFFu), y[1] -= __uint_as_float(w[i] & 0xFFFF0000u);
                    }
                    pf[p] = uint4{w[0], w[1], w[2], w[3]};
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    uint4 v;
                    if constexpr (E4M3) {
                        const uint4 w = RW == 16 ? vf[dt] : vf[dt * 2 + (f & 1)];
                        v = (RW == 16 ? f : f >> 1) ? eight_bf16(w.z, w.w, 1.0f) : eight_bf16(w.x, w.y, 1.0f);
                    } else {
                        v = RW == 16 ? vf[dt] : vf[dt * 2 + f];
                    }
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p) o[dt] = T::mfma(v, pf[p], o[dt]);
                }
            }
            if (masked && __any(odd))
                add_not_finite<D, E4M3, RW>(o, (const char*)a.c.v + cur_head * 64 * D * (E4M3 ? 1 : 2), cur_base, lane, sees, most);
            if (more) load_v(head, base);
            cur_base = base, cur_head = head;
        }

        // the unit's wavefronts meet
#pragma unroll
        for (int m = RW; m < 64; m <<= 1) l_run += __shfl_xor(l_run, m);
        __syncthreads();
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < T::REGS / 4; ++j)
                *(float4*)&so[wave][row][dt * RW + T::out_dim(lane, 4 * j)] = float4{o[dt][4 * j], o[dt][4 * j + 1], o[dt][4 * j + 2], o[dt][4 * j + 3]};
        if (part == 0) sml[wave][row][0] = m_run, sml[wave][row][1] = l_run;
        if (TWICE && any_not_finite(o) && lane == 0) walk.odd = true;
        __syncthreads();
        for (int i = tid; i < RW * (D / 4); i += 256) {
            const int r = i / (D / 4), d = i % (D / 4) * 4, rw = en.rows0 + r;
            if (rw >= en.rows1) continue;
            float m = -INFINITY, l = 0.0f;
            for (int k = 0; k < N_KS; ++k) m = fmaxf(m, sml[k][r][0]);
            const float ref = m == -INFINITY ? 0.0f : m;
            float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int k = 0; k < N_KS; ++k) {
                const float f = __builtin_amdgcn_exp2f(sml[k][r][0] - ref);
                const float4 z = *(const float4*)&so[k][r][d];
                l += sml[k][r][1] * f;
                y[0] += z.x * f, y[1] += z.y * f, y[2] += z.z * f, y[3] += z.w * f;
            }
            if (whole) {
                finish_row<D>(a, en.b, en.r0, en.n, rw / G, h * G + rw % G, d, m, l, y);
            } else {
                const size_t at_row = (size_t)slot * a.block_rows + r;
                *(float4*)(a.part_o + at_row * D + d) = float4{y[0], y[1], y[2], y[3]};
                if (d == 0) *(float2*)(a.part_ml + at_row * 2) = float2{m, l};
            }
        }
        note_parts(a, walk, unit);
    } while (walk_next<STEP>(a, &walk));
}

// at most n of this wavefront's loads still under way (n: of a wavefront, at most 17)
__device__ __forceinline__ void wait_loads(int n) {
    switch (n) {
        case 0: stage_wait<0>(); break;
        case 1: stage_wait<1>(); break;
        case 2: stage_wait<2>(); break;
        case 3: stage_wait<3>(); break;
        case 4: stage_wait<4>(); break;
        case 5: stage_wait<5>(); break;
        case 6: stage_wait<6>(); break;
        case 7: stage_wait<7>(); break;
        case 8: stage_wait<8>(); break;
        case 10: stage_wait<10>(); break;
        case 12: stage_wait<12>(); break;
        case 14: stage_wait<14>(); break;
        case 16: stage_wait<16>(); break;
        default: stage_wait<0>(); break;   // fewer than n are as good
    }
}

// ---------------------------------------------------------------- attention of many rows
// More than one tile of 32 rows: a workgroup has `tiles` of them (up to 8), key_halves wavefronts each (two where there are up to 4
// tiles: each takes 32 of a page's 64 keys, and they meet at the unit's end).  The wavefronts share each page through LDS, double-buffered:
// bf16 pages go there straight from memory, in the order in which a wavefront's operands are read; 8-bit pages through registers, where
// they become bf16 numbers with their scales in, which is exact.  So a page is read, and converted, once for up to 256 rows.
// bf16 queries: the weights are rounded to one bf16 piece here (2^-8 of each at most, at random, next to the output's own rounding):
// a second piece is as many products again in the second product, and the subtractions and conversions that make it.  One against two:
// prompts 843 against 1065 us, draft blocks of 160 rows over 8 bits 164 against 192, selected blocks 63 against 65; error of the
// output against 64 bits 0.0022 against the 0.0017 of its own rounding.
// No unit is full: in that prompt the matrix units are busy 35% of the time and the vector units as much, wavefronts wait 37% of theirs.
// Queries of two and three pieces take 64 and 96 registers and leave none for 8-bit pages on their way: these (DEEP) go to LDS as they
// are, two stages ahead, and become bf16 a stage ahead of their use.
// 4 x up to 2048 rows over 512 to 8192 positions, 32 query heads (bf16): 850 us, 0.82 PFLOP/s of the 1.29 that a large product reaches; without
// seven eighths of the products it still takes 0.73 of that time: exponentials, sums and conversions, LDS and the pages' barriers, which
// the two wavefronts of a SIMD hide only in part.  Three or four stages under way change nothing, two pages per stage cost 2%, the next tile's products between
// the present one's exponentials in one wavefront, with three buffers, save 2% (884 against 900 us, in turn).
template <int D, bool E4M3, int NQ>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2)))
pages_attend_shared_kernel(PagesAttnArgs a) {
    using T = Tile<32>;
    constexpr int STEP = 64, QS = D / 16, DT = D / 32, NP = NQ;
    constexpr int HALF = 2 * QS * 64;               // 16-byte pieces of a stage's keys, and of its values: [32 keys][step] x 64 lanes
    constexpr bool DEEP = pages_raw(NQ, E4M3);
    constexpr bool TWICE = !E4M3 && NP > 1;            // sums that are not finite are worked out once more
    constexpr bool PIECES_OF_KEYS = NQ > 1 && !E4M3;   // and infinite keys by themselves
    constexpr int RAW = DEEP ? 3 : 0;
    constexpr int LOADS = E4M3 ? D / 4 / 2 + 1 : 4 * QS;   // 1 KiB loads of a stage (8 bits: and one of the scales)
    __shared__ __align__(16) uint4 stage[2][2][HALF];   // [buffer][keys, values]
    __shared__ __align__(16) uint4 raw[RAW ? RAW : 1][RAW ? HALF + 8 : 1];   // [buffer]: keys, values, scales in 8 bits
    __shared__ long long lds[8];
    __shared__ Walk walk;
    __shared__ int pg_base[64], pg_id[64], pg_n, pg_odd;   // pg_odd: the page that has values that are not finite
    __shared__ __align__(8) float2 lds_ml[4 * 64];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), hf = lane >> 5, row = lane & 31;
    const int waves = blockDim.x / 64, tiles = waves / a.key_halves, rt = wave % tiles, kh = wave / tiles;
    const int heads = a.c.n_kv_heads, G = a.group_heads;
    const int kt0 = a.key_halves == 2 ? kh : 0, kt1 = a.key_halves == 2 ? kh + 1 : 2;
    if (!walk_start<STEP>(a, &walk, lds)) return;

    do {
        const Unit unit = walk_unit(walk);
        const Entry& en = unit.en;
        const int h = unit.h, s0 = unit.s0, s1 = unit.s1, slot = unit.slot;
        const bool whole = unit.whole, careful = TWICE && unit.careful;

        const int r = rt * 32 + row, myrow = en.rows0 + r;
        const bool have = myrow < en.rows1;
        const int t = have ? myrow / G : 0, g = have ? myrow % G : 0;
        const int sees = have ? sees_of(a, en.P, en.n, t) : 0;
        int least = have ? sees : 0x7FFFFFFF, most = sees;
        for (int m = 16; m; m >>= 1) least = min(least, __shfl_xor(least, m)), most = max(most, __shfl_xor(most, m));
        least = __builtin_amdgcn_readfirstlane(least), most = __builtin_amdgcn_readfirstlane(most);
        const int begins = sees_of(a, en.P, en.n, en.t0), ends = sees_of(a, en.P, en.n, en.t1 - 1);   // what each row sees, and what any does

        uint4 q[NQ][QS];
        load_queries<D, NQ>(a, en, h, t, g, have, q, [&](int s) { return 16 * s + 8 * hf; });
        f32x16_t o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
        float m_run = -INFINITY, l_run = 0.0f;
        const int32_t* list = a.list ? a.list + ((size_t)(en.b * a.n_blk + en.blk) * heads + h) * a.n_list : nullptr;

        for (int win = s0; win < s1; win += 64) {
            // the window's pages, those that there are, one behind the other
            if (wave == 0) {
                int ln = lane;
                asm("" : "+v"(ln));
                const int i = win + ln, page = i < s1 ? (list ? list[i] : i) : -1;
                const int id = page >= 0 && page < a.c.max_pages ? a.c.table[(size_t)en.b * a.c.max_pages + page] : -1;
                const bool seen = page < -1 || (page >= 0 && page * 64LL < ends);
                const bool good = seen && (unsigned)id < (unsigned)a.c.n_pages;
                if (seen && !good) flag(a.status, ST_PAGE);
                const unsigned long long who = __ballot(good);
                if (good) {
                    const int at = __popcll(who & ((1ull << ln) - 1));
                    pg_base[at] = page * 64, pg_id[at] = id;
                }
                if (ln == 0) pg_n = __popcll(who), pg_odd = -1;
            }
            __syncthreads();
            const int n = __builtin_amdgcn_readfirstlane(pg_n);

            // bf16: a wavefront's loads of a stage, each one operand (64 lanes x 16 bytes) from where its lanes' pieces lie in the page
            int ln = lane;
            asm("" : "+v"(ln));
            const int m32 = 8 * ((ln >> 4) & 1) + (ln & 7), h16 = (ln >> 5) * 16;
            const uint32_t k_lane = (((ln >> 3) & 1) * (D / 32) * 64 + h16 + m32) * 16, v_lane = (((ln >> 4) & 1) * 64 + h16 + (ln & 15)) * 16;   // bytes
            auto fetch = [&](int j, int buf) {
                const size_t hd = (size_t)scalar(pg_id[j]) * heads + h;
                const char* kp = (const char*)a.c.k + hd * 64 * D * (E4M3 ? 1 : 2);
                const char* vp = (const char*)a.c.v + hd * 64 * D * (E4M3 ? 1 : 2);
                const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)(E4M3 ? &raw[RAW ? buf : 0][0] : &stage[buf][0][0]);
                for (int i = wave; i < LOADS; i += waves) {
                    const uint32_t dst = scalar(to + (uint32_t)i * 1024u);
                    if constexpr (E4M3) {
                        if (i < LOADS - 1) load_to_lds(i < LOADS / 2 ? kp + i * 1024 : vp + (i - LOADS / 2) * 1024, (uint32_t)ln * 16u, dst);
                        else if (ln < 8) load_to_lds(a.c.scale + hd * 128, (uint32_t)ln * 16u, dst);
                    } else {
                        const bool value = i >= 2 * QS;
                        const int o2 = value ? i - 2 * QS : i, kt = o2 / QS, s = o2 % QS;   // values: s = (dims of 32, step)
                        if (value) load_to_lds(vp + ((kt * (D / 16) + (s >> 1) * 2) * 64 + (s & 1) * 32) * 16, v_lane, dst);
                        else load_to_lds(kp + ((kt * 2 * (D / 32) + (s >> 1)) * 64 + (s & 1) * 32) * 16, k_lane, dst);
                    }
                }
            };
            const int mine = scalar((LOADS - wave + waves - 1) / waves);   // loads of this wavefront per stage
            // 8 bits: a thread's 16-byte pieces of a stage (at most two of the keys and two of the values: there are at least 4 wavefronts)
            constexpr int NI = D / 64;
            uint4 rk[NI], rv[NI];
            uint32_t rks[NI], rvs[4];   // of the values: the same for both pieces, which are whole blocks apart
            auto fetch8 = [&](int j) {
                const size_t hd = (size_t)__builtin_amdgcn_readfirstlane(pg_id[j]) * heads + h;
                const uint4* kp = (const uint4*)((const uint8_t*)a.c.k + hd * 64 * D);
                const uint4* vp = (const uint4*)((const uint8_t*)a.c.v + hd * 64 * D);
                const uint8_t* sc = a.c.scale + hd * 128;
#pragma unroll
                for (int u = 0; u < NI; ++u) {
                    const int i = tid + u * (int)blockDim.x;
                    if (i < 4 * D) {
                        rk[u] = kp[i];
                        const int m = i & 15, tile = i / (D / 64 * 64);
                        rks[u] = sc[(tile >> 1) * 32 + (tile & 1) * 8 + 16 * (m >> 3) + (m & 7)];
                        rv[u] = vp[i];
                    }
                }
                const int pc = (tid >> 4) & 3;
                const uint32_t* vs = (const uint32_t*)(sc + 64 + 16 * (pc >> 1) + 4 * (pc & 1));
#pragma unroll
                for (int x = 0; x < 4; ++x) rvs[x] = vs[(x >> 1) * 8 + (x & 1) * 2];
            };
            // one piece of the keys (16 dims of a key) and one of the values (8 keys of a dim, of both groups of 32) as bf16 numbers
            auto put_piece = [&](int buf, int i, const uint4& kq, uint32_t kscale, const uint4& vq, const uint32_t* vscale) {
                const int m = i & 15, pc = (i >> 4) & 3, blk = i >> 6;
                const int tile = blk / (D / 64), rho = (tile & 1) * 8 + 16 * (m >> 3) + (m & 7), s = (blk % (D / 64)) * 4 + pc, d = blk * 16 + m;
                uint4* to = &stage[buf][0][((tile >> 1) * QS + s) * 64 + rho];   // two lanes' pieces of one step
                const float f = scale_of(kscale);
                to[0] = eight_bf16(kq.x, kq.y, f);
                to[32] = eight_bf16(kq.z, kq.w, f);
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    uint32_t w[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const uint32_t b = kt ? (x < 2 ? vq.z : vq.w) : (x < 2 ? vq.x : vq.y), sb = vscale[kt * 2 + (x >> 1)] >> (16 * (x & 1));
                        const float f0 = scale_of(sb & 0xFFu), f1 = scale_of((sb >> 8) & 0xFFu);
                        const uint32_t lo = x & 1 ? pair_bf16<true>(b, f0) : pair_bf16<false>(b, f0), hi = x & 1 ? pair_bf16<true>(b, f1) : pair_bf16<false>(b, f1);
                        w[x] = (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
                    }
                    stage[buf][1][(kt * QS + (d >> 5) * 2 + (pc >> 1)) * 64 + (pc & 1) * 32 + (d & 31)] = uint4{w[0], w[1], w[2], w[3]};
                }
            };
            auto put8 = [&](int buf) {
#pragma unroll
                for (int u = 0; u < NI; ++u) {
                    const int i = tid + u * (int)blockDim.x;
                    if (i < 4 * D) put_piece(buf, i, rk[u], rks[u], rv[u], rvs);
                }
            };
            auto put_raw = [&](int from, int buf) {
                const uint8_t* sc = (const uint8_t*)&raw[RAW ? from : 0][RAW ? HALF : 0];
                int i0 = threadIdx.x;
                asm("" : "+v"(i0));
#pragma unroll 1
                for (int i = i0; i < 4 * D; i += blockDim.x) {
                    const int m = i & 15, pc = (i >> 4) & 3, tile = i / D;
                    const uint32_t* vs = (const uint32_t*)(sc + 64 + 16 * (pc >> 1) + 4 * (pc & 1));
                    const uint32_t vscale[4] = {vs[0], vs[2], vs[8], vs[10]};
                    put_piece(buf, i, raw[RAW ? from : 0][RAW ? i : 0], sc[(tile >> 1) * 32 + (tile & 1) * 8 + 16 * (m >> 3) + (m & 7)], raw[RAW ? from : 0][RAW ? HALF / 2 + i : 0], vscale);
                }
            };

            // Values of page j that some row of the block does not see, for all wavefronts: 0 behind what any row sees, and where they are not finite.
            // Whether there were any of these.
            auto clean = [&](int j, int buf) -> bool {
                const int page0 = scalar(pg_base[j]);
                if (!careful && page0 + 64 <= begins) return false;
#pragma unroll 1
                for (int i = tid; i < HALF; i += blockDim.x) {
                    const int pos = page0 + i / (QS * 64) * 32;
                    const uint4 v = stage[buf][1][i];
                    uint32_t w[4] = {v.x, v.y, v.z, v.w};
                    bool change = false;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool behind = pos + value_key((i >> 6) & 1, (i >> 5) & 1, e) >= ends, not_finite = ((w[e / 2] >> (16 * (e & 1))) & 0x7F80u) == 0x7F80u;
                        if (behind || not_finite) w[e / 2] &= ~(0xFFFFu << (16 * (e & 1))), change = true;
                        if (!behind && not_finite) pg_odd = j;
                    }
                    if (change) stage[buf][1][i] = uint4{w[0], w[1], w[2], w[3]};
                }
                __syncthreads();
                return pg_odd == j;
            };
            auto add_odd = [&](int j, int base) {
                add_not_finite<D, E4M3, 32>(o, (const char*)a.c.v + ((size_t)pg_id[j] * heads + h) * 64 * D * (E4M3 ? 1 : 2), base, lane, sees, min(most, base + 32));
            };

            if (n > 0) {
                if constexpr (DEEP) {
                    for (int i = 0; i < min(n, 3); ++i) fetch(i, i);
                    wait_loads(mine * (min(n, 3) - 1));
                    __syncthreads();
                    put_raw(0, 0);
                } else if constexpr (E4M3) {
                    fetch8(0);
                    put8(0);
                } else {
                    fetch(0, 0);
                }
            }
            for (int j = 0; j < n; ++j) {
                const int buf = j & 1;
                if constexpr (DEEP) wait_loads(mine * max(min(n - 2 - j, 1), 0));   // stage j + 2 may still be under way
                else if constexpr (!E4M3) stage_wait<0>();
                __syncthreads();   // the stage is there, and nobody reads the one before any more
                if constexpr (DEEP) {
                    if (j + 3 < n) fetch(j + 3, j % 3);
                } else if (j + 1 < n) {
                    if constexpr (E4M3) fetch8(j + 1);
                    else fetch(j + 1, buf ^ 1);
                }
                const int page0 = __builtin_amdgcn_readfirstlane(pg_base[j]);
                const bool odd = clean(j, buf);
                // A tile's keys and values are requested from LDS several at once, well before they are multiplied: one by one each product would wait
                // out the latency of its own.  Queries of one piece over bf16 pages leave registers for all of a tile's, and the next tile's keys.
                constexpr bool AHEAD = NQ == 1 && !E4M3;
                constexpr int CH = AHEAD ? QS : NQ == 3 ? 2 : 4;
                uint4 kf[CH], vf[AHEAD ? QS : DT];
                auto load_keys = [&](int kt, int s0) {
#pragma unroll
                    for (int s = 0; s < CH; ++s) kf[s] = stage[buf][0][(kt * QS + s0 + s) * 64 + lane];
                };
                if (AHEAD && page0 + kt0 * 32 < most) load_keys(kt0, 0);
#pragma unroll 1
                for (int kt = kt0; kt < kt1; ++kt) {   // 32 keys against the wavefront's rows
                    const int base = page0 + kt * 32;
                    if (base >= most) break;
                    f32x16_t x;
                    bool odd_keys = false;
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = 0.0f;
#pragma unroll
                    for (int s0 = 0; s0 < QS; s0 += CH) {
                        if (!AHEAD) load_keys(kt, s0);
                        __builtin_amdgcn_sched_barrier(0);
                        if (PIECES_OF_KEYS && careful)
#pragma unroll
                            for (int s = 0; s < CH; ++s) odd_keys |= no_infinity(&kf[s]);
#pragma unroll
                        for (int s = 0; s < CH; ++s)
#pragma unroll
                            for (int p = NQ - 1; p >= 0; --p) x = T::mfma(kf[s], q[p][s0 + s], x);
                    }
                    if (PIECES_OF_KEYS && __any(odd_keys)) {
                        float y[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = x[i];
                        add_infinite_keys<D, NQ>(a, y, [&](int i) { return value_key(i >> 3, hf, i & 7); },
                                                   (const uint16_t*)a.c.k + ((size_t)pg_id[j] * heads + h) * 64 * D, kt * 32, en, h, t, g, have);
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = y[i];
                    }
                    // values: step s of dims dt at 2 dt + s; all at once, or a step's
                    auto load_values = [&](int s) {
#pragma unroll
                        for (int i = 0; i < (AHEAD ? QS : DT); ++i) vf[i] = stage[buf][1][(kt * QS + (AHEAD ? i : 2 * i + s)) * 64 + lane];
                    };
                    load_values(0);
                    if (AHEAD && kt + 1 < kt1) load_keys(kt + 1, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if (base + 32 > least)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (base + value_key(i >> 3, hf, i & 7) >= sees) x[i] = -INFINITY;
                    float top = x[0];
#pragma unroll
                    for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
                    rescale(T::across(top, [](float u, float w) { return fmaxf(u, w); }) * a.scale_log2, &m_run, &l_run, o);
                    const float ref = m_run == -INFINITY ? 0.0f : m_run;
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        x[i] = weight(x[i], a.scale_log2, ref);
                        sum += x[i];
                    }
                    l_run += sum;
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        float y[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = x[s * 8 + i];
#pragma unroll
                        for (int p = 0; p < NP; ++p) {   // a piece of the weights at a time
                            uint32_t w[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                w[i] = pack_bf16x2(y[2 * i], y[2 * i + 1]);
                                y[2 * i] -= bf16_to_f32(w[i] & 0xFFFFu), y[2 * i + 1] -= __uint_as_float(w[i] & 0xFFFF0000u);
                            }
                            const uint4 pf{w[0], w[1], w[2], w[3]};
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt) o[dt] = T::mfma(vf[AHEAD ? dt * 2 + s : dt], pf, o[dt]);
                            if (NQ == 3) __builtin_amdgcn_sched_barrier(0);
                        }
                        if (!AHEAD && s == 0) load_values(1);
                    }
                    if (odd) add_odd(j, base);
                }
                if constexpr (E4M3)
                    if (j + 1 < n) {
                        if constexpr (DEEP) put_raw((j + 1) % 3, buf ^ 1);
                        else put8(buf ^ 1);
                    }
            }
            __syncthreads();   // the window, and the last stage, have been read
        }
        if (TWICE && any_not_finite(o) && lane == 0) walk.odd = true;

        l_run += __shfl_xor(l_run, 32);
        if (a.key_halves == 2) {   // the second half's sums go to the first's wavefront, through the stages' place
            float4* to = (float4*)&stage[0][0][0] + rt * (DT * 4) * 64 + lane;
            float2* ml = lds_ml + rt * 64 + lane;
            if (kh == 1) {
#pragma unroll
                for (int i = 0; i < DT * 4; ++i) to[i * 64] = float4{o[i >> 2][(i & 3) * 4], o[i >> 2][(i & 3) * 4 + 1], o[i >> 2][(i & 3) * 4 + 2], o[i >> 2][(i & 3) * 4 + 3]};
                *ml = float2{m_run, l_run};
            }
            __syncthreads();
            if (kh == 0) {
                const float2 z = *ml;
                const float m = fmaxf(m_run, z.x), ref = m == -INFINITY ? 0.0f : m;
                const float f0 = __builtin_amdgcn_exp2f(m_run - ref), f1 = __builtin_amdgcn_exp2f(z.x - ref);
                l_run = l_run * f0 + z.y * f1;
                m_run = m;
#pragma unroll
                for (int i = 0; i < DT * 4; ++i) {
                    const float4 y = to[i * 64];
                    const float w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i >> 2][(i & 3) * 4 + e] = o[i >> 2][(i & 3) * 4 + e] * f0 + w[e] * f1;
                }
            }
        }
        int again = threadIdx.x;
        asm("" : "+v"(again));   // worked out again: the row's place would take registers all the way
        const int r_out = rt * 32 + (again & 31);
        const int row_out = en.rows0 + r_out, t_out = row_out / G, g_out = row_out % G;
        if (kh == 0 && row_out < en.rows1) {
            const size_t at_row = (size_t)slot * a.block_rows + r_out;
#pragma unroll
            for (int i = 0; i < DT * 4; ++i) {
                const int d = (i >> 2) * 32 + T::out_dim(lane, (i & 3) * 4);
                const float y[4] = {o[i >> 2][(i & 3) * 4], o[i >> 2][(i & 3) * 4 + 1], o[i >> 2][(i & 3) * 4 + 2], o[i >> 2][(i & 3) * 4 + 3]};
                if (whole) finish_row<D>(a, en.b, en.r0, en.n, t_out, h * G + g_out, d, m_run, l_run, y);
                else *(float4*)(a.part_o + at_row * D + d) = float4{y[0], y[1], y[2], y[3]};
            }
            if (!whole && hf == 0) *(float2*)(a.part_ml + at_row * 2) = float2{m_run, l_run};
        }
        note_parts(a, walk, unit);
    } while (walk_next<STEP>(a, &walk));
}


// The parts of units that several workgroups have: a.slices workgroups per unit, each taking every a.slices-th 1024 / D of its rows.
// The first launch wrote how many parts a unit has, so no workgroup works the shares out again.  Latency: 5 us at 256 units of 4 rows, 9 at
// 256 units of 64; 22 (67 MB read) at 512 units of 256.
template <int D, int STEP>
__global__ void __launch_bounds__(256) pages_combine_kernel(PagesAttnArgs a) {
    constexpr int TPR = D / 4, ROWS = 256 / TPR;
    const int heads = a.c.n_kv_heads, G = a.group_heads;
    const int slice = blockIdx.x % a.slices, h = blockIdx.x / a.slices % heads, e = blockIdx.x / a.slices / heads;
    const Entry en = entry_of<STEP>(a, e, nullptr);
    if (en.rows0 + slice * ROWS >= en.rows1) return;
    const uint2 parts = a.parts[(size_t)e * heads + h];
    const int n = (int)parts.y, w0 = (int)(parts.x & 0x7FFFFFFFu);
    if (n <= 1 || n > a.grid || w0 > a.grid - n) return;   // past the grid: not unless lengths or rows change meanwhile, and then it may be any number
    const int d = threadIdx.x % TPR * 4, first = 2 * w0 + (int)(parts.x >> 31);
    for (int r = slice * ROWS + threadIdx.x / TPR; en.rows0 + r < en.rows1; r += a.slices * ROWS) {
        auto place = [&](int i) { return (size_t)(i == 0 ? first : 2 * (w0 + i)) * a.block_rows + r; };
        float m = -INFINITY;
        for (int i = threadIdx.x % TPR; i < n; i += TPR) m = fmaxf(m, a.part_ml[place(i) * 2]);
        for (int k = TPR / 2; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
        const float ref = m == -INFINITY ? 0.0f : m;
        float l = 0.0f, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
        for (int i = 0; i < n; ++i) {
            const size_t at = place(i);
            const float2 ml = *(const float2*)(a.part_ml + at * 2);
            const float4 y = *(const float4*)(a.part_o + at * D + d);
            const float f = __builtin_amdgcn_exp2f(ml.x - ref);
            l += ml.y * f;
            x[0] += y.x * f, x[1] += y.y * f, x[2] += y.z * f, x[3] += y.w * f;
        }
        const int rw = en.rows0 + r;
        finish_row<D>(a, en.b, en.r0, en.n, rw / G, h * G + rw % G, d, m, l, x);
    }
}

// ---------------------------------------------------------------- selection of pages
// Scores in whole numbers: a query row is rounded to 8 bits by its largest magnitude over 127, the bounds of a page are 8-bit
// too, and sum over the dims of max(qi * least, qi * largest), which no key of the page exceeds but for the rounding of q, is one matrix product of
// [min(qi, 0), max(qi, 0)] with [least, largest].  Its 32-bit result is exact below 2^24, so which pages win does not hang on any order
// of summation.
struct Group {
    int r0, n, P, t0, t1;   // tokens [t0, t1) of the sequence's
    int p0;                 // first page of its own: that of its first token's position
    int end;                // past the last page that it sees
};
__device__ __forceinline__ Group group_of(const PagesSelectArgs& a, int b, int grp, uint32_t* status) {
    Group g;
    const SeqRows sr = seq_rows(a.ch, b, status);
    g.r0 = sr.r0, g.n = sr.n;
    g.P = seq_length(a.c, b, sr.n ? status : nullptr);
    g.t0 = min(grp * a.group, g.n), g.t1 = min(g.t0 + a.group, g.n);
    g.p0 = g.end = 0;
    if (g.t1 > g.t0) {
        const int cap = a.c.max_pages, sees = a.draft && g.t1 > a.bidir_from ? g.n : g.t1;
        if (status && g.P + sees > cap * 64) flag(status, ST_CAPACITY);
        g.p0 = min((g.P + g.t0) / 64, cap);
        g.end = min((g.P + sees + 63) / 64, cap);
    }
    return g;
}


// A group's rows of one KV head as 8-bit operands: 8 dims per thread, a row's threads adjacent.  Rows up to a multiple of 32.
template <int D>
struct GroupRows {
    static constexpr int PITCH = 2 * D + 16;
    int8_t qi[PAGES_GROUP_ROWS][PITCH];   // [min(q, 0), max(q, 0)]
    float qs[PAGES_GROUP_ROWS];           // -1: a row without a part
};
template <int D>
__device__ __forceinline__ int load_group(const PagesSelectArgs& a, const Group& g, int b, int h, GroupRows<D>* out) {
    constexpr int C = D / 8;
    const int G = a.group_heads, n = (g.t1 - g.t0) * G, n32 = (n + 31) / 32 * 32;
    for (int r = threadIdx.x / C; r < n32; r += blockDim.x / C) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.0f;
        const int d = threadIdx.x % C * 8;
        if (r < n) {
            if (a.q_split) {   // a pass's split queries
                const uint16_t* p = a.q_split + q_index(b * a.c.n_kv_heads + h, r % G * g.n + g.t0 + r / G, d, a.q_row_tiles, D);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = bf16_to_f32(p[i]) + bf16_to_f32(p[SPLIT_LO + i]);
            } else {
                load8(a.q, g.r0 + g.t0 + r / G, h * G + r % G, d, x);
            }
        }
        float amax = 0.0f;
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(x[i])), odd |= !finite(x[i]);
#pragma unroll
        for (int m = 1; m < C; m <<= 1) amax = fmaxf(amax, __shfl_xor(amax, m)), odd |= __shfl_xor((int)odd, m) != 0;
        const float sc = amax / 127.0f, by = sc > 0.0f ? sc : 1.0f;
        uint32_t neg[2] = {0u, 0u}, pos[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int v = odd ? 0 : (int)fmaxf(-127.0f, fminf(127.0f, rintf(x[i] / by)));
            neg[i / 4] |= (uint32_t)(uint8_t)min(v, 0) << (8 * (i & 3));
            pos[i / 4] |= (uint32_t)max(v, 0) << (8 * (i & 3));
        }
        *(uint2*)&out->qi[r][d] = uint2{neg[0], neg[1]};
        *(uint2*)&out->qi[r][D + d] = uint2{pos[0], pos[1]};
        if (threadIdx.x % C == 0) out->qs[r] = r < n && !odd ? sc : -1.0f;
    }
    return n32;
}

// bounds of a page as an operand: lanes col and col + 32 have its halves
template <int D>
struct PageBounds {
    i32x4_t w[2 * D / 32];
    float scale;
    int id;
};
template <int D>
__device__ __forceinline__ PageBounds<D> load_bounds(const PagesSelectArgs& a, int b, int h, int page, bool there, int hf) {
    PageBounds<D> p;
    p.id = there ? page_id(a.c, b, page) : -1;
    if (there && p.id < 0) flag(a.status, ST_PAGE);
    const size_t head = (size_t)max(p.id, 0) * a.c.n_kv_heads + h;
#pragma unroll
    for (int s = 0; s < 2 * D / 32; ++s) p.w[s] = *(const i32x4_t*)(a.c.bounds + head * 2 * D + 32 * s + 16 * hf);
    p.scale = a.c.bound_scale[head];
    return p;
}
// score of a lane's page
template <int D>
__device__ __forceinline__ float page_score(const PageBounds<D>& p, const GroupRows<D>& rows, int n32, int lane) {
    const int hf = lane >> 5, col = lane & 31;
    float best = -INFINITY;
    for (int r0 = 0; r0 < n32; r0 += 32) {
        i32x16_t acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0;
#pragma unroll
        for (int s = 0; s < 2 * D / 32; ++s)
            acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(*(const i32x4_t*)&rows.qi[r0 + col][32 * s + 16 * hf], p.w[s], acc, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float f = rows.qs[r0 + 8 * (r >> 2) + 4 * hf + (r & 3)];
            if (f >= 0.0f) best = fmaxf(best, (float)acc[r] * f);
        }
    }
    best = fmaxf(best, __shfl_xor(best, 32));
    const float f = !finite(p.scale) ? INFINITY : best == -INFINITY ? -INFINITY : best * p.scale;
    return p.id < 0 ? -INFINITY : f;
}

// order of scores as unsigned numbers; -0 is 0
__device__ __forceinline__ uint32_t score_key(float v) {
    uint32_t u = __float_as_uint(v);
    if ((u & 0x7FFFFFFFu) == 0u) u = 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// The taken pages of a unit, in ascending order: the n_top-th largest of n > n_top keys (key_of(i): of page lo + i) digit by digit, with the
// counts of a digit's 256 values in LDS, then page by page.
template <int THREADS, typename F>
__device__ __forceinline__ void pick_pages(const PagesSelectArgs& a, const Group& g, int unit, int lo, int n, F key_of) {
    constexpr int W = THREADS / 64;
    __shared__ uint32_t hist[256];
    __shared__ int wsum[W][2];
    __shared__ uint32_t s_key;
    __shared__ int s_left;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t* out = a.list + (size_t)unit * a.n_list;
    uint32_t key = a.n_top > 0 ? 0u : 0xFFFFFFFFu;   // taken: above key, and `left` of those equal to it
    int left = a.n_top;
    if (n > a.n_top && a.n_top > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0u;
            __syncthreads();
            for (int i = tid; i < n; i += THREADS) {
                const uint32_t k = key_of(i);
                if (shift == 24 || (k >> (shift + 8)) == (key >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            // counts of larger digits; the digit where they reach `left`
            uint32_t up = tid < 256 ? hist[tid] : 0u;
            for (int m = 1; m < 64; m <<= 1) {
                const uint32_t o = __shfl_down(up, m);
                if (lane + m < 64) up += o;
            }
            if (lane == 0) wsum[wave][0] = (int)up;
            __syncthreads();
            if (tid < 256) {
                for (int w = wave + 1; w < 4; ++w) up += (uint32_t)wsum[w][0];
                const uint32_t above = up - hist[tid];
                if ((int)above < left && (int)up >= left) s_key = key | (uint32_t)tid << shift, s_left = left - (int)above;
            }
            __syncthreads();
            key = s_key, left = s_left;
        }
    }
    int put = 0;
    for (int i0 = 0; i0 < g.end; i0 += THREADS) {
        const int i = i0 + tid;
        bool sure = false, tie = false;
        if (i < g.end) {
            if (i < lo || i >= g.p0 || n <= a.n_top) sure = true;
            else if (a.n_top > 0) {   // 0: nobody worked out keys, and no candidate is taken
                const uint32_t k = key_of(i - lo);
                sure = k > key, tie = k == key;
            }
        }
        const unsigned long long ties = __ballot(tie), below = (1ull << lane) - 1;
        if (lane == 0) wsum[wave][0] = __popcll(ties);
        __syncthreads();
        int before = __popcll(ties & below), all = 0;
        for (int w = 0; w < W; ++w) {
            if (w < wave) before += wsum[w][0];
            all += wsum[w][0];
        }
        const bool taken = sure || (tie && before < left);
        left -= min(left, all);
        const unsigned long long takes = __ballot(taken);
        if (lane == 0) wsum[wave][1] = __popcll(takes);
        __syncthreads();
        int at = put + __popcll(takes & below);
        for (int w = 0; w < W; ++w) {
            if (w < wave) at += wsum[w][1];
            put += wsum[w][1];
        }
        if (taken && at < a.n_list) out[at] = i;
    }
    for (int i = put + tid; i < a.n_list; i += THREADS) out[i] = -1;
}

// Scores and choice of a unit in one workgroup of 8 wavefronts: the scores stay in LDS as whole numbers in the order of the floats, and the
// choice is by their bits, eight at a time.
template <int D>
__global__ void __launch_bounds__(512) pages_select_kernel(PagesSelectArgs a) {
    __shared__ __align__(16) GroupRows<D> rows;
    __shared__ uint32_t keys[SELECT_PAGES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, unit = blockIdx.x, heads = a.c.n_kv_heads;
    const int h = unit % heads, grp = unit / heads % a.n_groups, b = unit / heads / a.n_groups;
    const Group g = group_of(a, b, grp, h == 0 && threadIdx.x == 0 ? a.status : nullptr);
    const int lo = min(a.n_first, g.p0), n = g.p0 - lo;   // candidates
    if (n > a.n_top && a.n_top > 0) {
        int i = wave * 32 + (lane & 31);
        PageBounds<D> p = load_bounds<D>(a, b, h, lo + i, i < n, lane >> 5);   // under way with the queries
        const int n32 = load_group<D>(a, g, b, h, &rows);
        __syncthreads();
        for (int i0 = 0; i0 < n; i0 += 256) {
            const PageBounds<D> now = p;
            const int next = i + 256;
            if (i0 + 256 < n) p = load_bounds<D>(a, b, h, lo + next, next < n, lane >> 5);
            const float f = page_score<D>(now, rows, n32, lane);
            if (i < n && lane < 32) keys[i] = score_key(f);
            i = next;
        }
        __syncthreads();
    }
    pick_pages<512>(a, g, unit, lo, n, [&](int i) { return keys[i]; });
}

// The same in two launches, for more pages than that, or for few units: a workgroup per unit and 128 pages, then one per unit.
// 64 units of up to 1024 pages (11 MB of bounds): scores 8.5 us, choice 8.0, both latency.
template <int D>
__global__ void __launch_bounds__(256) pages_score_kernel(PagesSelectArgs a) {
    __shared__ __align__(16) GroupRows<D> rows;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int chunk = blockIdx.x % a.chunks, unit = blockIdx.x / a.chunks, heads = a.c.n_kv_heads;
    const int h = unit % heads, grp = unit / heads % a.n_groups, b = unit / heads / a.n_groups;
    const Group g = group_of(a, b, grp, nullptr);
    const int lo = max(a.n_first, chunk * SCORE_PAGES), hi = min(g.p0, chunk * SCORE_PAGES + SCORE_PAGES);
    if (lo >= hi || g.p0 - a.n_first <= a.n_top) return;   // none, or all of them are taken
    const int page = chunk * SCORE_PAGES + wave * 32 + (lane & 31);
    const bool there = page >= lo && page < hi;
    const PageBounds<D> p = load_bounds<D>(a, b, h, page, there, lane >> 5);   // under way with the queries
    const int n32 = load_group<D>(a, g, b, h, &rows);
    __syncthreads();
    const float f = page_score<D>(p, rows, n32, lane);
    if (there && lane < 32) a.scores[(size_t)unit * a.c.max_pages + page] = f;
}

__global__ void __launch_bounds__(512) pages_pick_kernel(PagesSelectArgs a) {
    __shared__ uint32_t keys[SELECT_PAGES];
    const int unit = blockIdx.x, heads = a.c.n_kv_heads;
    const Group g = group_of(a, unit / heads / a.n_groups, unit / heads % a.n_groups, unit % heads == 0 && threadIdx.x == 0 ? a.status : nullptr);
    const int lo = min(a.n_first, g.p0), n = g.p0 - lo;
    const float* score = a.scores + (size_t)unit * a.c.max_pages + lo;
    if (n > SELECT_PAGES || n <= a.n_top || a.n_top == 0) {
        pick_pages<512>(a, g, unit, lo, n, [&](int i) { return score_key(score[i]); });
        return;
    }
    for (int i = threadIdx.x; i < n; i += 512) keys[i] = score_key(score[i]);
    __syncthreads();
    pick_pages<512>(a, g, unit, lo, n, [&](int i) { return keys[i]; });
}

HeadRows with_vec(HeadRows r) {
    const uintptr_t m = r.f32 ? 3 : 7;
    r.vec = ((uintptr_t)r.data & 15) == 0 && (r.row_stride & m) == 0 && (r.head_stride & m) == 0;
    return r;
}

template <typename F>
hipError_t by_type(const PageCache& c, F f) {
    if (c.head_dim == 64) return c.e4m3 ? f(std::integral_constant<int, 64>(), std::true_type()) : f(std::integral_constant<int, 64>(), std::false_type());
    return c.e4m3 ? f(std::integral_constant<int, 128>(), std::true_type()) : f(std::integral_constant<int, 128>(), std::false_type());
}

}  // namespace

// pages that n adjacent positions touch at most
static int pages_touched(int n) { return (n + 62) / 64 + 1; }

hipError_t launch_pages_write(const PageCache& c, const HeadRows& k, const HeadRows& v, const uint16_t* blk_k, const uint16_t* blk_v,
                              const PageChunk& ch, uint32_t* status, hipStream_t s) {
    const KvSource src{with_vec(k), with_vec(v), blk_k, blk_v};
    const int touched = pages_touched(ch.max_rows);
    return by_type(c, [&](auto d, auto e) {
        launch(pages_write_kernel<decltype(d)::value, decltype(e)::value>, dim3(c.batch * touched * c.n_kv_heads), dim3(256), s, c, src, ch, touched, status);
        return hipGetLastError();
    });
}

hipError_t launch_pages_read(const PageCache& c, const HeadRows& k, const HeadRows& v, const PageChunk& ch, const int32_t* first, uint32_t* status,
                             hipStream_t s) {
    const int touched = pages_touched(ch.max_rows);
    return by_type(c, [&](auto d, auto e) {
        launch(pages_read_kernel<decltype(d)::value, decltype(e)::value>, dim3(c.batch * touched * c.n_kv_heads), dim3(256), s, c, with_vec(k), with_vec(v), ch, first,
               touched, status);
        return hipGetLastError();
    });
}

hipError_t launch_pages_attend(const PagesAttnArgs& args, hipStream_t s) {
    PagesAttnArgs a = args;
    a.q = with_vec(a.q), a.out = with_vec(a.out);
    return by_type(a.c, [&](auto d, auto e) {
        constexpr int D = decltype(d)::value;
        constexpr bool E = decltype(e)::value;
        auto run = [&](auto nq) {
            constexpr int NQ = decltype(nq)::value;
            if (a.shared_waves) launch(pages_attend_shared_kernel<D, E, NQ>, dim3(a.grid), dim3(a.shared_waves * 64), s, a);
            else if (a.block_rows == 16) launch(pages_attend_kernel<D, E, NQ, 16>, dim3(a.grid), dim3(256), s, a);
            else launch(pages_attend_kernel<D, E, NQ, 32>, dim3(a.grid), dim3(256), s, a);
        };
        if (a.q_split) run(std::integral_constant<int, 2>());
        else if (a.q.f32) run(std::integral_constant<int, 3>());
        else run(std::integral_constant<int, 1>());
        const hipError_t st = hipGetLastError();
        if (st != hipSuccess) return st;
        const int wgs = a.n_entries * a.c.n_kv_heads * a.slices;
        if (a.shared_waves || E) launch(pages_combine_kernel<D, 64>, dim3(wgs), dim3(256), s, a);
        else launch(pages_combine_kernel<D, 32>, dim3(wgs), dim3(256), s, a);
        return hipGetLastError();
    });
}

hipError_t launch_pages_select(const PagesSelectArgs& args, hipStream_t s) {
    PagesSelectArgs a = args;
    a.q = with_vec(a.q);
    a.chunks = cdiv(a.c.max_pages, SCORE_PAGES);
    const int units = a.c.batch * a.n_groups * a.c.n_kv_heads;
    if (select_in_one(a.c.max_pages, units)) {
        if (a.c.head_dim == 64) launch(pages_select_kernel<64>, dim3(units), dim3(512), s, a);
        else launch(pages_select_kernel<128>, dim3(units), dim3(512), s, a);
        return hipGetLastError();
    }
    if (a.n_top > 0) {
        if (a.c.head_dim == 64) launch(pages_score_kernel<64>, dim3(units * a.chunks), dim3(256), s, a);
        else launch(pages_score_kernel<128>, dim3(units * a.chunks), dim3(256), s, a);
        const hipError_t st = hipGetLastError();
        if (st != hipSuccess) return st;
    }
    launch(pages_pick_kernel, dim3(units), dim3(512), s, a);
    return hipGetLastError();
}

}  // namespace nld
