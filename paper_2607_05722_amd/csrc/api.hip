// C ABI of libnld: host-side validation, workspace layout and launch sequence of
// the block-decode step (declared in include/nld.h).
#include "../../include/nld.h"
#include "nld_internal.h"

#include <float.h>
#include <limits.h>
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <mutex>
#include <vector>

using namespace nld;

struct nld_model {
    nld_config cfg;
    nld_weights w;
    std::vector<nld_layer_weights> layers;
};

namespace {

thread_local char g_err[512] = "";

nld_status fail(nld_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return st;
}

#define HIP_TRY(expr)                                                                              \
    do {                                                                                           \
        hipError_t e_ = (expr);                                                                    \
        if (e_ != hipSuccess) return fail(NLD_ERR_HIP, "%s failed: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

// ---------------------------------------------------------------- tracing aid
// While tracing is on, every launch inside a TraceScope gets its own pair of events,
// recorded by the launch on its own dispatch (kernel start and end), filed under the
// scope's kernel class.
struct TraceRec {
    int cls;
    bool first;   // first launch of its scope: the scope counts once in its class
    hipEvent_t start, stop;
};
bool g_trace_on = false;
std::vector<TraceRec> g_trace;
thread_local int g_trace_cls = -1;
thread_local bool g_trace_scope_new = false;

struct TraceScope {
    int saved;
    TraceScope(int cls, hipStream_t) : saved(g_trace_cls) {
        g_trace_cls = cls;
        g_trace_scope_new = true;
    }
    ~TraceScope() { g_trace_cls = saved; }
};

int device_cus();

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Operand sites carried in plain bf16 instead of split form: NLD_PLAIN_SITES, a comma-separated list
// of norm, final, q, kv, p, o, act (precision knob; default: none, every site split).
uint32_t plain_sites() {
    const char* v = getenv("NLD_PLAIN_SITES");
    if (!v || !*v) return 0u;
    static const struct { const char* name; uint32_t bit; } names[] = {
        {"norm", SITE_NORM}, {"final", SITE_FINAL}, {"q", SITE_Q}, {"kv", SITE_KV},
        {"p", SITE_P}, {"o", SITE_O}, {"act", SITE_ACT}};
    uint32_t m = 0u;
    for (const auto& n : names) {
        const size_t len = strlen(n.name);
        for (const char* c = v; (c = strstr(c, n.name)) != nullptr; c += len) {
            const bool start = c == v || c[-1] == ',';
            const bool end = c[len] == '\0' || c[len] == ',';
            if (start && end) m |= n.bit;
        }
    }
    return m;
}

}  // namespace

bool nld::trace_launch_events(hipEvent_t* start, hipEvent_t* stop) {
    if (!g_trace_on || g_trace_cls < 0) return false;
    TraceRec r{};
    r.cls = g_trace_cls;
    r.first = g_trace_scope_new;
    g_trace_scope_new = false;
    if (hipEventCreate(&r.start) != hipSuccess) return false;
    if (hipEventCreate(&r.stop) != hipSuccess) {
        (void)hipEventDestroy(r.start);
        return false;
    }
    g_trace.push_back(r);
    *start = r.start;
    *stop = r.stop;
    return true;
}

namespace {

// ---------------------------------------------------------------- workspace layout
constexpr int CTR0 = 1;   // tile counter 0 hands out the LM head's tiles
struct Layout {
    int M, Mpad, units, n_splits, chunk, row_tiles, attn_kh, attn_waves, attn_z, n_parts, rows_pad, lm_tiles, lm_parts;
    bool attn_items;         // length-aware attention work (batches)
    int n_tile_ctr;          // tile counters in all, zeroed by the embedding kernel at the start of a pass
    int n_ctr;               // K slices: counters (one per group of tiles) from tile counter CTR0
    size_t part_floats;      // K slices: room for their partials
    size_t status, x, xg, part_ss, q, o, act, keys, lse, rope, po, pml, blk_k, blk_v, tile_ctr, part, lora_t, drafts,
        ens_logits, ens_v, total;
};

// k: block rows per sequence.  quad_k > 0: the block is a quadratic self-speculation layout
// with chain length quad_k (k = quad_k * (quad_k + 1)), which adds the ensemble verifier's buffers.
Layout make_layout(const nld_config& c, int batch, int k, int max_len, int quad_k = 0) {
    Layout L{};
    L.M = batch * k;
    // operand rows: whole row groups of the panel GEMM (128 rows for M > 64)
    L.Mpad = L.M > 64 ? cdiv(L.M, 128) * 128 : 64;
    L.units = batch * c.n_kv_heads;
    const int G = c.n_q_heads / c.n_kv_heads;
    L.row_tiles = cdiv(G * k, 16);
    L.attn_kh = L.row_tiles <= 4 ? 2 : 1;          // wavefronts per row tile (each takes half of a stage's keys)
    L.lm_tiles = cdiv(c.vocab, 16);
    L.lm_parts = L.lm_tiles;  // upper bound on argmax partials per row (one per LM-head workgroup)
    // Attention.  Partials: room for `room` rows per unit, from a first cut of max_len into key splits that
    // aims for about `target` workgroups of 8 wavefronts.
    L.attn_items = batch > 1 && !env_int("NLD_ATTN_NO_ITEMS", 0);
    const int z8 = cdiv(L.row_tiles, 8 / L.attn_kh), pairs = L.units * z8, max_splits = cdiv(max_len, 64);
    auto cut = [&](int ns) { L.chunk = cdiv(cdiv(max_len, std::max(1, std::min(std::min(ns, max_splits), 255))), 64) * 64; };
    const int finer = L.attn_items ? env_int("NLD_ATTN_ITEMS_FINER", z8 == 1 ? 2 : 1) : 1;
    const int target = env_int("NLD_ATTN_TARGET_WG", finer * device_cus() * std::min(4, std::max(1, pairs / 16)));
    cut(target / pairs - 1);
    const size_t room = (size_t)(cdiv(max_len, L.chunk) + 1) * z8 * (8 / L.attn_kh) * 16;
    // One sequence: that cut, a workgroup of 8 wavefronts (kh 2) or one per row tile; the merge handles up to
    // 256 partials per row.  A batch: workgroups as wide as the rows need, and items of about 1024 keys where
    // the capacity has at least four of those per CU, else of 384, so that the CUs share few sequences evenly
    // (an item's own start, its place in the list, queries and first stage, is about 6 us, or five stages);
    // never more than fit the room at 16 rows per row tile.  Attention and merge at 1024 / 384 keys: batch 8
    // at 16000 keys, k = 8 104 / 123 us; batch 5 at 3000 keys, k = 24 45 / 28 us; batch 2 at 4000 keys, k = 16
    // 31 / 20 us.  NLD_ATTN_ITEM_KEYS overrides.
    const int zmax = L.attn_kh == 2 ? 4 : 12;
    L.attn_z = cdiv(L.row_tiles, zmax);
    const int rz = cdiv(L.row_tiles, L.attn_z);
    L.attn_waves = L.attn_kh == 2 ? (L.attn_items ? 2 * rz : 8) : rz;
    L.rows_pad = L.row_tiles * 16;
    if (L.attn_items) {
        const int parts = (int)std::min<size_t>(room / L.rows_pad, 255);
        const bool many = (size_t)L.units * L.attn_z * cdiv(max_len, 1024) >= (size_t)4 * device_cus();
        cut(std::min(parts, cdiv(max_len, std::max(1, env_int("NLD_ATTN_ITEM_KEYS", many ? 1024 : 384)))));
    }
    L.n_splits = cdiv(max_len, L.chunk);
    L.n_parts = L.n_splits + (L.attn_items ? 0 : 1);

    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t o = off;
        off = align256(off + bytes);
        return o;
    };
    const size_t H = c.hidden, QD = (size_t)c.n_q_heads * c.head_dim;
    L.status = take(4);
    L.x = take(4 * L.Mpad * H);
    L.xg = take(4 * L.Mpad * H);   // split operand (hi and lo bf16)
    L.part_ss = take(4 * L.Mpad * (H / 16));
    // q, o and act are split operands too: 4 bytes per value
    L.q = take(4 * std::max(L.Mpad * QD, (size_t)L.units * L.row_tiles * 16 * c.head_dim));
    L.o = take(4 * L.Mpad * QD);
    L.act = take(4 * L.Mpad * (size_t)cdiv(c.ffn, 32) * 32);
    L.keys = take(8 * L.Mpad * (size_t)L.lm_parts);
    L.lse = take(8 * L.Mpad * (size_t)L.lm_parts);   // softmax statistics per argmax partial (denoising)
    L.rope = take(8 * L.Mpad * (size_t)(c.head_dim / 2));
    // K slices of a projection: counters (one per group of tiles) and room for the slices' partials.  Up to 16 rows
    // the split-K GEMM's groups hold at least two column tiles.  The panel GEMM takes slices only where groups x slices is
    // at most two per CU, so from 17 to 64 rows it needs no more than a counter per CU and the partials of two groups
    // of 12 column tiles per CU, and less for a small model.  Above, a group is 128 rows x 8 column tiles.
    const int sk_tiles = std::max((int)H / 16, (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim / 16);
    const int sk_groups = cdiv(sk_tiles, 2);
    if (L.M <= 64) {
        const int rt = L.M <= 32 ? 2 : 4;
        L.n_ctr = sk_groups;
        L.part_floats = (size_t)(2 * sk_groups + 4) * 256 * rt * SPLITK_MAX;
        if (L.M > 16) {
            const int wide = std::max(std::max(L.lm_tiles, cdiv(c.ffn, 8)), sk_tiles);
            L.n_ctr = std::min(L.n_ctr + wide, device_cus());
            L.part_floats = std::min(L.part_floats + (size_t)wide * cdiv((int)H, rt == 2 ? 2048 : 1024) * rt * 256,
                                     (size_t)2 * device_cus() * 256 * rt * 12);
        }
    } else {
        L.n_ctr = cdiv(L.M, 128) * cdiv(std::max(sk_tiles, cdiv(c.ffn, 8)), 8);
        L.part_floats = (size_t)4 * device_cus() * 16384;
    }
    L.n_tile_ctr = CTR0 + L.n_ctr;
    L.tile_ctr = take(4 * (size_t)L.n_tile_ctr);
    L.part = take(4 * L.part_floats);
    L.po = take(4 * (size_t)L.units * room * c.head_dim);
    L.pml = take(4 * 2 * (size_t)L.units * room);
    L.blk_k = take(2 * (size_t)L.units * 2 * 64 * c.head_dim);   // block K/V, split: [unit][hi, lo][64][D]
    L.blk_v = take(2 * (size_t)L.units * 2 * 64 * c.head_dim);
    L.lora_t = take(4 * (size_t)L.Mpad * c.lora_rank);   // split lora_scale * (A o), draft passes only
    L.drafts = take(4 * (size_t)batch * k);              // nld_decode_steps: one step's drafts
    // quadratic self-speculation: the verifier rows' logits [batch][2 quad_k][vocab] and the ensemble's
    // argmax keys [batch][quad_k][ENS_CHUNKS]
    L.ens_logits = take(4 * (size_t)batch * 2 * quad_k * c.vocab);
    L.ens_v = take(8 * (size_t)batch * quad_k * ENS_CHUNKS);
    L.total = off;
    return L;
}

template <typename T>
T* at(void* ws, size_t off) { return (T*)((char*)ws + off); }

nld_status check_config(const nld_config* c) {
    if (!c) return fail(NLD_ERR_INVALID_ARG, "config is NULL");
    if (c->n_layers < 1 || c->hidden < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->ffn < 1 || c->vocab < 1)
        return fail(NLD_ERR_INVALID_ARG, "config sizes must be positive");
    if (c->hidden % 32) return fail(NLD_ERR_SHAPE, "hidden (%d) must be a multiple of 32", c->hidden);
    if (c->head_dim != 64 && c->head_dim != 128) return fail(NLD_ERR_SHAPE, "head_dim must be 64 or 128");
    if (c->n_q_heads % c->n_kv_heads) return fail(NLD_ERR_SHAPE, "n_q_heads must be a multiple of n_kv_heads");
    if (c->ffn % 8) return fail(NLD_ERR_SHAPE, "ffn (%d) must be a multiple of 8", c->ffn);
    if (c->mask_token_id < 0 || c->mask_token_id >= c->vocab)
        return fail(NLD_ERR_INVALID_ARG, "mask_token_id outside [0, vocab)");
    if (!(c->rope_base > 1.0f) || !(c->rms_eps >= 0.0f)) return fail(NLD_ERR_INVALID_ARG, "bad rope_base or rms_eps");
    if (c->lora_rank < 0 || !(fabsf(c->lora_scale) < INFINITY))
        return fail(NLD_ERR_INVALID_ARG, "lora_rank must be >= 0 and lora_scale finite");
    if (c->lora_rank % 32) return fail(NLD_ERR_SHAPE, "lora_rank (%d) must be a multiple of 32", c->lora_rank);
    if (c->lora_rank > 512) return fail(NLD_ERR_SHAPE, "lora_rank (%d) must be at most 512", c->lora_rank);
    return NLD_OK;
}

// ---------------------------------------------------------------- GEMM launch plans
// Compute units of the current device (queried once per device; NLD_CUS overrides).
int device_cus() {
    const int forced = env_int("NLD_CUS", 0);
    if (forced > 0) return forced;
    static int cached[64] = {0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    if (cached[dev] == 0) {
        int n = 0;
        cached[dev] = (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n > 0)
                          ? n : 256;
    }
    return cached[dev];
}

constexpr double LOG2E = 1.44269504088896340736;

// ---------------------------------------------------------------- paged cache
constexpr int MAX_PAGE_WGS = 1 << 23;    // workgroups of 256 threads in one launch
constexpr int MAX_SEQ_PAGES = 1 << 24;   // 2^30 positions
constexpr int MAX_CHUNK_ROWS = 1 << 24;

nld_status check_pages(const nld_pages* c, int layer) {
    if (!c || !c->k || !c->v || !c->table || !c->lengths) return fail(NLD_ERR_INVALID_ARG, "pages or one of its pointers is NULL");
    if (c->dtype != NLD_BF16 && c->dtype != NLD_E4M3) return fail(NLD_ERR_INVALID_ARG, "pages: dtype must be NLD_BF16 or NLD_E4M3");
    if (c->dtype == NLD_E4M3 && !c->scale) return fail(NLD_ERR_INVALID_ARG, "pages: 8-bit pages need their scales");
    if (!c->bounds != !c->bound_scale) return fail(NLD_ERR_INVALID_ARG, "pages: bounds and bound_scale go together");
    if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1 || c->batch < 1 || c->max_pages < 1)
        return fail(NLD_ERR_INVALID_ARG, "pages: sizes must be positive");
    if (c->head_dim != 64 && c->head_dim != 128) return fail(NLD_ERR_SHAPE, "pages: head_dim must be 64 or 128");
    if (c->max_pages > MAX_SEQ_PAGES) return fail(NLD_ERR_SHAPE, "pages: max_pages (%d) exceeds %d", c->max_pages, MAX_SEQ_PAGES);
    if (layer < 0 || layer >= c->n_layers) return fail(NLD_ERR_INVALID_ARG, "layer must be in [0, %d) (got %d)", c->n_layers, layer);
    if (((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)c->scale | (uintptr_t)c->bounds) % 16 || (uintptr_t)c->bound_scale % 4)
        return fail(NLD_ERR_INVALID_ARG, "pages: arrays must be 16-byte aligned");
    return NLD_OK;
}

PageCache page_layer(const nld_pages* c, int layer) {
    const size_t heads = (size_t)layer * c->n_pages * c->n_kv_heads, page = (size_t)64 * c->head_dim * (c->dtype == NLD_BF16 ? 2 : 1);
    PageCache p{};
    p.k = (char*)c->k + heads * page;
    p.v = (char*)c->v + heads * page;
    p.scale = c->dtype == NLD_E4M3 ? (uint8_t*)c->scale + heads * 128 : nullptr;
    p.bounds = c->bounds ? (int8_t*)c->bounds + heads * 2 * c->head_dim : nullptr;
    p.bound_scale = c->bounds ? c->bound_scale + heads : nullptr;
    p.e4m3 = c->dtype == NLD_E4M3;
    p.n_pages = c->n_pages;
    p.n_kv_heads = c->n_kv_heads;
    p.head_dim = c->head_dim;
    p.table = c->table;
    p.lengths = c->lengths;
    p.batch = c->batch;
    p.max_pages = c->max_pages;
    return p;
}

nld_status check_chunk(const nld_pages* c, const nld_chunk* ch) {
    if (!ch) return fail(NLD_ERR_INVALID_ARG, "chunk is NULL");
    if (ch->rows < 1 || ch->max_rows < 1 || ch->max_rows > ch->rows)
        return fail(NLD_ERR_INVALID_ARG, "chunk: max_rows must be in [1, rows] (got %d of %d)", ch->max_rows, ch->rows);
    if (!ch->row_start && (long long)ch->max_rows * c->batch != ch->rows)
        return fail(NLD_ERR_INVALID_ARG, "chunk: without row_start, rows (%d) must be batch * max_rows (%d * %d)", ch->rows, c->batch, ch->max_rows);
    if (ch->rows > MAX_CHUNK_ROWS) return fail(NLD_ERR_SHAPE, "chunk: %d rows exceed %d", ch->rows, MAX_CHUNK_ROWS);
    return NLD_OK;
}

// out: rows and heads must be apart from each other
nld_status check_heads(const nld_heads* x, const char* what, int rows, int heads, int dim, bool out) {
    if (!x || !x->data) return fail(NLD_ERR_INVALID_ARG, "%s or its data is NULL", what);
    if (x->dtype != NLD_F32 && x->dtype != NLD_BF16) return fail(NLD_ERR_INVALID_ARG, "%s: dtype must be NLD_F32 or NLD_BF16", what);
    if (x->row_stride < 0 || x->head_stride < 0 || x->row_stride >> 38 || x->head_stride >> 38)
        return fail(NLD_ERR_INVALID_ARG, "%s: strides must be in [0, 2^38)", what);
    if ((uintptr_t)x->data % (x->dtype == NLD_BF16 ? 2 : 4)) return fail(NLD_ERR_INVALID_ARG, "%s: data is not aligned to its type", what);
    if (out) {
        const long long rs = rows > 1 ? x->row_stride : LLONG_MAX, hs = heads > 1 ? x->head_stride : LLONG_MAX;
        const long long inner = std::min(rs, hs), outer = std::max(rs, hs), n_inner = rs <= hs ? rows : heads;
        if (inner < dim || (outer != LLONG_MAX && outer < (n_inner - 1) * inner + dim))
            return fail(NLD_ERR_INVALID_ARG, "%s: its rows overlap each other", what);
    }
    return NLD_OK;
}

// Whether two arrays of rows of one type, the second without overlaps of its own, share an element.  Arrays of unlike strides: whether their
// ranges meet.
bool heads_overlap(const nld_heads* a, const nld_heads* b, int rows, int heads, int dim) {
    typedef __int128 wide;   // (rows - 1) * stride alone is up to 2^62 elements
    const int es = b->dtype == NLD_BF16 ? 2 : 4;
    auto extent = [&](const nld_heads* x) { return (wide)(rows - 1) * x->row_stride + (wide)(heads - 1) * x->head_stride + dim; };
    const wide apart = (wide)(uintptr_t)b->data - (wide)(uintptr_t)a->data;
    if (apart >= extent(a) * es || -apart >= extent(b) * es) return false;
    if ((rows > 1 && a->row_stride != b->row_stride) || (heads > 1 && a->head_stride != b->head_stride) || apart % es) return true;
    const wide d = apart / es;
    const long long rs = rows > 1 ? b->row_stride : 0, hs = heads > 1 ? b->head_stride : 0;
    // an element of both: d = i * rs + j * hs + less than dim, with i rows and j heads between the two
    for (int j = 1 - heads; j < heads; ++j) {
        const wide rest = d - (wide)j * hs, i0 = rs ? rest / rs : 0;
        for (wide i = i0 - 1; i <= i0 + 1; ++i)
            if (i > -rows && i < rows && rest - i * rs < dim && rest - i * rs > -dim) return true;
    }
    return false;
}

HeadRows head_rows(const nld_heads* x) { return HeadRows{x->data, x->dtype == NLD_F32, 0, x->row_stride, x->head_stride}; }
PageChunk page_chunk(const nld_chunk* c) { return PageChunk{c->rows, c->max_rows, c->row_start}; }

// The attention's plan and workspace: the status word, then the parts of units that workgroups share, or a selection's scores.
// Rows of a KV head (tokens x query heads of its group), or of a group of tokens with a list:
//  - up to 16: one 16-row tile per workgroup, 17 to 32: one 32-row tile; keys and values go straight to registers, four wavefronts to a
//    workgroup, two of these to a CU (a token of 32 ragged sequences over 8 bits: 79 us, 113 with 32-row tiles);
//  - more: up to eight 32-row tiles that share each page through LDS, two wavefronts per tile where there are up to four of them.  Against
//    single tiles, two or four to a workgroup: draft blocks of 160 rows over 8 bits 174 against 352 us, prompts 882 against 1383, verify
//    blocks of 64 f32 rows 164 against 222.
// Two workgroups of four wavefronts fit a CU by LDS and registers, else one.
struct PagesPlan {
    int block_rows, row_tiles, n_blk, grid, slices, shared_waves, key_halves;
    size_t part_ml, parts, total;
};

bool plan_pages(int batch, int n_kv_heads, int head_dim, int group_heads, int max_rows, int group, bool raw, PagesPlan* out) {
    PagesPlan p{};
    if ((long long)max_rows * group_heads > INT_MAX - 256) return false;   // the kernels count a sequence's rows of a KV head in int
    const long long rows = (long long)(group ? std::min(group, max_rows) : max_rows) * group_heads;
    p.row_tiles = (int)std::min<long long>(8, (rows + 31) / 32);
    p.block_rows = rows <= 16 ? 16 : 32 * p.row_tiles;
    p.key_halves = p.row_tiles <= 4 ? 2 : 1;
    p.shared_waves = p.row_tiles > 1 ? p.row_tiles * p.key_halves : 0;
    const long long blocks = group ? cdiv(max_rows, group) : (rows + p.block_rows - 1) / p.block_rows;
    if (blocks * batch * n_kv_heads > MAX_PAGE_WGS) return false;
    p.n_blk = (int)blocks;
    p.grid = p.shared_waves > 4 || (p.shared_waves && raw) ? device_cus() : 2 * device_cus();
    // the second launch: a few thousand workgroups, and one per unit where units are that many
    const int turns = cdiv((int)std::min<long long>(rows, p.block_rows), 1024 / head_dim);
    p.slices = (int)std::max(1LL, std::min<long long>(turns, 8192 / (blocks * batch * n_kv_heads)));
    const size_t part_rows = (size_t)2 * p.grid * p.block_rows;
    p.part_ml = 256 + part_rows * head_dim * 4;
    p.parts = align256(p.part_ml + part_rows * 8);
    p.total = align256(p.parts + (size_t)8 * blocks * batch * n_kv_heads);
    *out = p;
    return true;
}

long long select_units(const nld_pages* c, int max_rows, int group) { return (long long)c->batch * cdiv(max_rows, group) * c->n_kv_heads; }

// Room for the scores of two launches.  So many units that one launch takes them have scores of their own in LDS; fewer of them may take two.
size_t score_bytes(const nld_pages* c, int max_rows, int group) {
    const long long units = select_units(c, max_rows, group);
    return (size_t)(select_in_one(c->max_pages, units) ? std::min<long long>(units, SELECT_UNITS - 1) : units) * c->max_pages * 4;
}

bool select_fits(const nld_pages* c, int max_rows, int group) {
    const long long units = select_units(c, max_rows, group);
    return units * (select_in_one(c->max_pages, units) ? 1 : cdiv(c->max_pages, SCORE_PAGES)) <= MAX_PAGE_WGS;
}

nld_status check_mode(int mode, int bidir_from, int max_rows) {
    if (mode != NLD_MODE_VERIFY && mode != NLD_MODE_DRAFT) return fail(NLD_ERR_INVALID_ARG, "mode must be 0 or 1");
    if (bidir_from < 0 || bidir_from > max_rows) return fail(NLD_ERR_INVALID_ARG, "bidir_from must be in [0, max_rows]");
    return NLD_OK;
}

nld_status check_group(const nld_pages* c, int n_q_heads, int group) {
    if (group < 1) return fail(NLD_ERR_INVALID_ARG, "group must be >= 1 (got %d)", group);
    if ((long long)group * (n_q_heads / c->n_kv_heads) > PAGES_GROUP_ROWS)
        return fail(NLD_ERR_SHAPE, "group * (n_q_heads / n_kv_heads) = %lld exceeds %d", (long long)group * (n_q_heads / c->n_kv_heads), PAGES_GROUP_ROWS);
    return NLD_OK;
}

nld_status check_q_heads(const nld_pages* c, int n_q_heads) {
    if (n_q_heads < 1 || n_q_heads % c->n_kv_heads)
        return fail(NLD_ERR_SHAPE, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", n_q_heads, c->n_kv_heads);
    return NLD_OK;
}

// the launch of an attention: what does not hang on where queries come from and outputs go
PagesAttnArgs pages_args(const PageCache& c, const PageChunk& ch, int group_heads, int mode, int bidir_from, float scale, const PagesPlan& p, void* ws,
                         size_t off) {
    PagesAttnArgs a{};
    a.c = c;
    a.ch = ch;
    a.group_heads = group_heads;
    a.draft = mode == NLD_MODE_DRAFT;
    a.bidir_from = bidir_from;
    a.scale_log2 = std::max((float)(LOG2E * fabs((double)scale)), FLT_MIN);   // not 0: a position that is not seen scores -inf
    a.negate = scale < 0.0f;
    a.block_rows = p.block_rows;
    a.row_tiles = p.row_tiles;
    a.n_blk = p.n_blk;
    a.n_entries = c.batch * p.n_blk;
    a.grid = p.grid;
    a.slices = p.slices;
    a.least_steps = p.shared_waves ? 2 : 4;
    a.shared_waves = p.shared_waves;
    a.key_halves = p.key_halves;
    a.part_o = at<float>(ws, off + 256);
    a.part_ml = at<float>(ws, off + p.part_ml);
    a.parts = at<uint2>(ws, off + p.parts);
    a.status = at<uint32_t>(ws, 0);
    return a;
}

enum Source { SRC_TOKENS = 0, SRC_DRAFT = 1, SRC_VERIFY = 2, SRC_QUAD = 3 };

struct PassIO {
    int source;
    const int32_t* tokens;
    const int32_t* anchor;
    const int32_t* draft_in;
    int mode, bidir_from;
    float* logits;
    int32_t* argmax_out;
    int finish;
    int32_t* draft_out;
    int32_t* accept_len;
    int32_t* committed;
    int32_t* next_anchor;
    bool advance_lengths;
    // denoising step / refresh
    int32_t* block;
    float threshold;
    int32_t* n_committed;
    int32_t* n_masked;
    float* conf_out;
    bool kv_only;   // refresh: stop after the last layer's K/V (no attention, FFN or LM head after it)
    // quadratic self-speculation (mode NLD_MODE_QUAD_INTERNAL): chain length and the verifier's mixture
    int quad_k;
    float lambda;
    const struct PagedPass* paged;   // the cache is a paged one
};

// A pass over a paged cache: the attention's plan, the selection (n_top, n_first, group; group 0: every page is read), and where in the
// workspace, behind the pass's own part, the attention's and the lists start.
struct PagedPass {
    const nld_pages* pages;
    PagesPlan plan;
    int n_top, n_first, group, n_groups, n_list;
    size_t attn, lists, total;
};

// Attention mode of a quadratic pass (never a caller's mode value).
constexpr int NLD_MODE_QUAD_INTERNAL = 2;

nld_status validate_call(const nld_model* m, const nld_kv_cache* kv, int batch, int k, void* ws, size_t ws_bytes,
                         Layout* out, int quad_k = 0) {
    if (!m) return fail(NLD_ERR_INVALID_ARG, "model is NULL");
    if (!kv || !kv->k || !kv->v || !kv->lengths) return fail(NLD_ERR_INVALID_ARG, "kv cache or one of its pointers is NULL");
    if (!ws) return fail(NLD_ERR_INVALID_ARG, "workspace is NULL");
    if (batch < 1) return fail(NLD_ERR_INVALID_ARG, "batch must be >= 1");
    if (kv->batch != batch) return fail(NLD_ERR_INVALID_ARG, "kv->batch (%d) != batch (%d)", kv->batch, batch);
    if (k < 1 || k > 64) return fail(NLD_ERR_INVALID_ARG, "k must be in [1, 64] (got %d)", k);
    if (kv->max_len < 64 || kv->max_len % 64) return fail(NLD_ERR_INVALID_ARG, "max_len must be a positive multiple of 64");
    const nld_config& c = m->cfg;
    const int G = c.n_q_heads / c.n_kv_heads;
    if (G * k > 256) return fail(NLD_ERR_SHAPE, "(n_q_heads/n_kv_heads)*k = %d exceeds 256", G * k);
    *out = make_layout(c, batch, k, kv->max_len, quad_k);
    if (ws_bytes < out->total)
        return fail(NLD_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, out->total);
    return NLD_OK;
}

// What a pass over a paged cache needs of its arguments; kv: the lengths and sizes that the pass takes of a cache.
nld_status validate_paged(const nld_model* m, const nld_pages* pages, const nld_sparse* sparse, int k, int mode, void* ws, size_t ws_bytes, nld_kv_cache* kv,
                          Layout* out, PagedPass* pp) {
    if (!m) return fail(NLD_ERR_INVALID_ARG, "model is NULL");
    nld_status st = check_pages(pages, 0);
    if (st != NLD_OK) return st;
    const nld_config& c = m->cfg;
    if (pages->n_layers != c.n_layers || pages->n_kv_heads != c.n_kv_heads || pages->head_dim != c.head_dim)
        return fail(NLD_ERR_INVALID_ARG, "pages have %d layers, %d KV heads of %d dims, the model %d, %d of %d", pages->n_layers, pages->n_kv_heads,
                    pages->head_dim, c.n_layers, c.n_kv_heads, c.head_dim);
    *kv = nld_kv_cache{pages->k, pages->v, pages->lengths, pages->batch, 64};
    Layout L;
    st = validate_call(m, kv, pages->batch, k, ws, ~(size_t)0, &L);   // the pass's own part has none of the other attention's partials worth mention
    if (st != NLD_OK) return st;
    kv->max_len = pages->max_pages * 64;
    PagedPass p{};
    p.pages = pages;
    const int G = c.n_q_heads / c.n_kv_heads;
    if (sparse) {
        if (!pages->bounds) return fail(NLD_ERR_INVALID_ARG, "a selection needs the pages' bounds");
        st = check_group(pages, c.n_q_heads, sparse->group);
        if (st != NLD_OK) return st;
        p.n_top = sparse->n_top;
        p.n_first = sparse->n_first;
        p.group = sparse->group;
        p.n_groups = cdiv(k, p.group);
        p.n_list = nld_pages_list_len(k, p.group, p.n_top, p.n_first, mode);
        if (p.n_list < 1) return fail(NLD_ERR_INVALID_ARG, "n_top and n_first must be in [0, %d]", MAX_SEQ_PAGES);
        if (!select_fits(pages, k, p.group))
            return fail(NLD_ERR_SHAPE, "%d sequences are too many for one call", pages->batch);
    }
    if (2LL * pages->batch * pages->n_kv_heads > MAX_PAGE_WGS || !plan_pages(pages->batch, pages->n_kv_heads, pages->head_dim, G, k, p.group, pages_raw(2, pages->dtype == NLD_E4M3), &p.plan))
        return fail(NLD_ERR_SHAPE, "%d sequences are too many for one call", pages->batch);
    p.attn = align256(L.total);
    p.lists = p.attn + std::max(p.plan.total, p.group ? align256(256 + score_bytes(pages, k, p.group)) : 0);
    p.total = align256(p.lists + (size_t)4 * pages->batch * p.n_groups * pages->n_kv_heads * p.n_list);
    if (ws_bytes < p.total) return fail(NLD_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, p.total);
    *out = L;
    *pp = p;
    return NLD_OK;
}

enum ProjKind { PROJ_O = 0, PROJ_DOWN = 1, PROJ_QKV = 2, PROJ_GU = 3, PROJ_LM = 4, PROJ_LORA = 5, N_PROJ = 6 };

// Split-K plan of a residual projection with at most 16 rows: ct column tiles per workgroup and ksplit K
// slices, so that column groups x slices is at most one workgroup per CU, with every wavefront (8 per
// workgroup) getting at least two k-steps.  Default: the down projection of up to 8 rows, 2 tiles, where its groups
// are few enough for two slices.  Split-K and panel GEMM in the middle of a pass: 21.8 and 21.7 us at 1 row of the 8B
// shapes (128 groups, 2 slices), 22.0 and 21.8 at 8; whole passes of a model of hidden 256 69.8 and 70.8 us, of
// hidden 2080 232.3 and 234.2; but 39.6 and 34.9 us per launch at hidden 5120 (160 groups, one slice, 96 CUs
// idle).  (O runs streamed: 10.8 against 11.4 us at 16 rows.)  Environment overrides: NLD_SPLITK_<O|DOWN> = "ct,ksplit" ("ct,0": ksplit
// from the rule; "0": off), NLD_SPLITK / NLD_SPLITK_CT for both at once, NLD_NO_SPLITK = 1: off.
bool plan_splitk(int kind, const GemmArgs& g, const Layout& L, int* ct, int* ksplit) {
    if (g.W2 || env_int("NLD_NO_SPLITK", 0)) return false;
    int c = kind == PROJ_DOWN && g.M <= 8 && 2 * cdiv(g.n_tiles, 2) <= device_cus() ? 2 : 0, ks = 0;
    const char* v = getenv(kind == PROJ_O ? "NLD_SPLITK_O" : "NLD_SPLITK_DOWN");
    if (v && *v) {
        c = atoi(v);
        const char* comma = strchr(v, ',');
        ks = comma ? atoi(comma + 1) : 0;
    }
    c = env_int("NLD_SPLITK_CT", c);
    ks = env_int("NLD_SPLITK", ks);
    if (c < 2 || c > 4) return false;
    const int groups = cdiv(g.n_tiles, c);
    if (ks <= 0) ks = std::min(std::max(1, device_cus() / groups), std::max(1, g.ksteps / 16));
    if (groups > L.n_ctr) ks = 1;   // no counters (and no partials) for that many groups
    *ct = c;
    *ksplit = std::max(1, std::min(std::min(ks, SPLITK_MAX), g.ksteps));
    return true;
}

// Panel GEMM: workgroup shape and K slices of one projection, the cheapest by an estimate in
// microseconds from rates measured on this part: weights 6.3 TB/s from HBM with every CU reading (32 GB/s
// into one CU), operand and re-read weights 80 GB/s per CU from L2, which add up; MFMA at 80% of 1024 flops
// per cycle and SIMD, LDS 128 bytes per cycle; slices 1.5 us to meet and 0.6 us each, their partials written
// at 5 TB/s in all and read back by one CU at 60 GB/s.  Against a sweep of every shape and slice count at the
// 8B shapes (8, 16, 32, 64, 100, 512 rows) and the 14B ones (256) the picked plan is within 4% of the fastest one, for the LM
// head of a short vocabulary within 10%.
// NLD_PANEL_<O|DOWN|QKV|GU|LM|LORA> = "shape,slices" overrides a plan; NLD_TILE_KSPLIT_<O|DOWN|QKV|GU> (more
// than 64 rows) and NLD_SPLITK (up to 64) the slices alone.
struct PanelPlan {
    int shape = 0, ksplit = 1;
};

PanelPlan plan_panel(int kind, int M, int n_tiles, int K, const Layout& L) {
    static const char* names[] = {"NLD_PANEL_O", "NLD_PANEL_DOWN", "NLD_PANEL_QKV", "NLD_PANEL_GU", "NLD_PANEL_LM", "NLD_PANEL_LORA"};
    static const char* slices[] = {"NLD_TILE_KSPLIT_O", "NLD_TILE_KSPLIT_DOWN", "NLD_TILE_KSPLIT_QKV", "NLD_TILE_KSPLIT_GU", "", ""};
    const double cus = device_cus(), cyc = 2.2e3;   // cycles per microsecond
    const int rt = M <= 16 ? 1 : (M <= 32 ? 2 : (M <= 64 ? 4 : 8)), full = K / 32, R = cdiv(M, 16 * rt);
    int want = kind < PROJ_LM ? env_int(M > 64 ? slices[kind] : "NLD_SPLITK", 0) : 0, only = -1;
    if (const char* force = getenv(names[kind])) {
        only = atoi(force);
        const char* comma = strchr(force, ',');
        want = comma ? atoi(comma + 1) : 1;
    }
    PanelPlan best;
    double best_us = -1.0;
    for (int i = 0; i < gemm_panel_shapes(); ++i) {
        const PanelShape p = gemm_panel_shape(i);
        if (p.rt != rt || (kind == PROJ_LORA && !gemm_panel_narrow(p)) || (only >= 0 && i != only)) continue;
        const int wt = p.wc * p.ct, C = cdiv(n_tiles, wt), nst = full / p.kb;
        // at least two stages per slice (an override: one), two workgroups per CU, counters and partials for all
        int most = std::max(1, std::min(want > 0 ? std::min(want, nst) : nst / 2, 16));
        if (R * C > L.n_ctr) most = 1;
        while (most > 1 && ((size_t)R * C * most > 2 * cus || (size_t)R * C * most * 256 * rt * wt > L.part_floats)) --most;
        for (int ks = want > 0 ? most : 1; ks <= most; ++ks) {
            const size_t wgs = (size_t)R * C * ks;
            const double rounds = ceil(wgs / cus), steps = rounds * cdiv(std::max(nst, 1), ks) * p.kb;
            const double mfma = steps * rt * wt * 8 / 0.8 / cyc, lds = steps * (p.wc * 2 * rt + 2 * rt) * 8 / cyc;
            const double hbm = std::max((double)n_tiles * full * 1024 / 6.3e6, steps * wt * 1024 / 32e3);
            const double l2 = steps * (rt * 2048 + (R > 1 ? wt * 1024 : 0)) / 80e3;
            const double tile = 1024.0 * rt * wt;
            const double meet = ks > 1 ? 1.5 + wgs * tile / 5e6 + (ks - 1) * (0.6 + tile / 60e3) : 0.0;
            const double us = std::max(std::max(mfma, lds), hbm + l2) + meet;
            if (best_us < 0.0 || us < best_us) {
                best.shape = i;
                best.ksplit = ks;
                best_us = us;
            }
        }
    }
    return best;
}

int panel_groups(const PanelPlan& p, int n_tiles) {
    const PanelShape sh = gemm_panel_shape(p.shape);
    return cdiv(n_tiles, sh.wc * sh.ct);
}

// groups (optional): column groups, the LM head's argmax partials and a residual projection's sums of
// squares per row
hipError_t panel_gemm(int epi, const PanelPlan& p, GemmArgs& g, void* ws, const Layout& L, hipStream_t s, int* groups) {
    g.n_parts = panel_groups(p, g.n_tiles);
    if (groups) *groups = g.n_parts;
    return launch_gemm_panel(epi, p.shape, g, p.ksplit, at<float>(ws, L.part), at<unsigned>(ws, L.tile_ctr) + CTR0, s);
}

// Residual projections (O, down).  Up to 16 rows O runs streamed and, up to 8, down on the split-K kernel (both sides
// measured at the streamed kernel and at plan_splitk); the rest on the panel GEMM.  n_ss: sums of squares per row the
// projection writes for the next RMSNorm.
hipError_t resid_gemm(int kind, const PanelPlan* plans, GemmArgs& g, void* ws, const Layout& L, hipStream_t s, int* n_ss) {
    *n_ss = g.n_tiles;
    int ct = 0, ksplit = 0;
    if (g.M <= 16 && plan_splitk(kind, g, L, &ct, &ksplit))
        return launch_gemm_splitk(ct, ksplit, g, at<float>(ws, L.part), at<unsigned>(ws, L.tile_ctr) + CTR0, s);
    if (g.M <= 16 && kind == PROJ_O) return launch_gemm_stream(env_int("NLD_STREAM_NW_RESID", 16), g, s);
    return panel_gemm(EPI_RESID, plans[kind], g, ws, L, s, n_ss);
}

// The LM head of up to 16 rows on the normed multi-tile GEMM: where the reduction is a full operand slice for each of
// its 8 wavefronts, and there are at least four column tiles per CU.  At 9496 tiles, 16 rows and logits, it and the panel
// GEMM take 200 and 216 us (hidden 4096), and with fewer or shorter slices, or longer ones that do not fit the
// registers, 125 and 61 (1024), 138 and 111 (2048), 161 and 159 (3072), 305 and 262 us (5120); at 1100 tiles and
// hidden 4096 30.4 and 30.8, at 64 13.1 and 5.7 us.  NLD_NO_NORM_GEMM: never.
bool lm_normed(int M, int n_tiles, int ksteps) {
    return M <= 16 && ksteps == gemm_norm_ksteps() && n_tiles >= 4 * device_cus() && !env_int("NLD_NO_NORM_GEMM", 0);
}

// One projection whose operand is RMSNorm(x) (QKV, gate/up, LM head): the panel GEMM, or for the LM head the normed
// kernel.  Both read the split operand and the row statistics the producer of x wrote.
hipError_t normed_gemm(int kind, int epi, const PanelPlan* plans, GemmArgs g, void* ws, const Layout& L, hipStream_t s) {
    g.A = at<uint16_t>(ws, L.xg);
    g.part_ss = at<float>(ws, L.part_ss);
    if (kind == PROJ_LM && lm_normed(g.M, g.n_tiles, g.ksteps)) {
        g.n_parts = device_cus();   // tiles beyond the first one per workgroup are handed out dynamically
        return launch_gemm_norm(g.n_parts, g, s);
    }
    return panel_gemm(epi, plans[kind], g, ws, L, s, nullptr);
}

// A layer's attention over a paged cache, in place of the other one: the block's keys and values go to their pages (positions P_b + j,
// in draft passes too: they are scratch until a commit), which the block's queries then read along with the prefix.
hipError_t paged_attention(const nld_model* mdl, const PagedPass& pp, int mode, int bidir_from, int layer, int k, uint32_t plain, void* ws, const Layout& L,
                           hipStream_t s) {
    const nld_config& c = mdl->cfg;
    const PageCache cache = page_layer(pp.pages, layer);
    const PageChunk ch{L.M, k, nullptr};
    uint32_t* status = at<uint32_t>(ws, L.status);
    hipError_t e = launch_pages_write(cache, HeadRows{}, HeadRows{}, at<uint16_t>(ws, L.blk_k), at<uint16_t>(ws, L.blk_v), ch, status, s);
    if (e != hipSuccess) return e;
    PagesAttnArgs a = pages_args(cache, ch, c.n_q_heads / c.n_kv_heads, mode, bidir_from, (float)(1.0 / sqrt((double)c.head_dim)), pp.plan, ws, pp.attn);
    if (pp.group) {
        PagesSelectArgs sel{};
        sel.c = cache;
        sel.ch = ch;
        sel.q_split = at<uint16_t>(ws, L.q);
        sel.q_row_tiles = L.row_tiles;
        sel.group_heads = a.group_heads;
        sel.draft = a.draft;
        sel.bidir_from = bidir_from;
        sel.n_top = pp.n_top;
        sel.n_first = pp.n_first;
        sel.group = pp.group;
        sel.n_groups = pp.n_groups;
        sel.n_list = pp.n_list;
        sel.scores = at<float>(ws, pp.attn + 256);
        sel.list = at<int32_t>(ws, pp.lists);
        sel.status = status;
        e = launch_pages_select(sel, s);
        if (e != hipSuccess) return e;
        a.list = sel.list;
        a.n_list = pp.n_list;
        a.group = pp.group;
    }
    a.q_split = at<uint16_t>(ws, L.q);
    a.q_row_tiles = L.row_tiles;
    a.o_split = at<uint16_t>(ws, L.o);
    a.o_ksteps = cdiv(c.n_q_heads * c.head_dim, 32);
    a.plain_o = (plain & SITE_O) != 0;
    a.status = status;
    return launch_pages_attend(a, s);
}

nld_status run_pass(const nld_model* mdl, const nld_kv_cache* kv, int batch, int k, const PassIO& io, void* ws,
                    const Layout& L, hipStream_t s) {
    const nld_config& c = mdl->cfg;
    const int M = L.M;
    const int D = c.head_dim, nq = c.n_q_heads, nkv = c.n_kv_heads;
    const size_t kv_layer = (size_t)batch * nkv * kv->max_len * D;
    uint32_t* status = at<uint32_t>(ws, L.status);
    float* x = at<float>(ws, L.x);

    EmbedArgs e{};
    e.tokens = io.tokens;
    e.anchor = io.anchor;
    e.draft = io.draft_in;
    e.source = io.source;
    e.k_blk = k;
    e.M = M;
    e.mask_id = c.mask_token_id;
    e.vocab = c.vocab;
    e.hidden = c.hidden;
    e.embed = (const uint16_t*)mdl->w.embed;
    e.gain = (const uint16_t*)mdl->layers[0].attn_norm;
    e.x = x;
    e.xg = at<uint16_t>(ws, L.xg);
    e.part_ss = at<float>(ws, L.part_ss);
    e.status = status;
    e.rope = at<float2>(ws, L.rope);
    e.tile_ctr = at<unsigned>(ws, L.tile_ctr);
    e.n_tile_ctr = L.n_tile_ctr;
    e.lengths = kv->lengths;
    e.max_len = kv->max_len;
    e.head_dim = c.head_dim;
    e.quad_k = io.quad_k;
    const uint32_t plain = plain_sites();
    e.plain = plain & SITE_NORM;
    // The LM head's partials per row, and its argmax keys (the normed GEMM's are one per workgroup).  Its plan alone stands
    // before the first launch, which the others need not hold up.
    PanelPlan plans[N_PROJ];   // the same for every layer
    plans[PROJ_LM] = plan_panel(PROJ_LM, M, L.lm_tiles, c.hidden, L);
    const bool normed = lm_normed(M, L.lm_tiles, cdiv(c.hidden, 32));
    const int parts = normed ? device_cus() : panel_groups(plans[PROJ_LM], L.lm_tiles);
    const int n_keys = normed ? parts : std::min(parts, KEY_SLOTS);
    e.keys = n_keys < parts && !io.kv_only ? at<unsigned long long>(ws, L.keys) : nullptr;
    for (int i = 0; i < c.head_dim / 2; ++i) e.inv_freq[i] = pow((double)c.rope_base, -2.0 * i / (double)c.head_dim);
    {
        TraceScope ts(NLD_TRACE_EMBED, s);
        HIP_TRY(launch_embed(e, s));
    }

    int n_ss = embed_sums(c.hidden);   // sums of squares per row in part_ss, as its latest producer wrote them
    const int ks_h = cdiv(c.hidden, 32), ks_q = cdiv(nq * D, 32), ks_f = cdiv(c.ffn, 32);
    const bool lora = io.mode == NLD_MODE_DRAFT && c.lora_rank > 0;
    plans[PROJ_O] = plan_panel(PROJ_O, M, c.hidden / 16, nq * D, L);
    plans[PROJ_DOWN] = plan_panel(PROJ_DOWN, M, c.hidden / 16, c.ffn, L);
    plans[PROJ_QKV] = plan_panel(PROJ_QKV, M, (nq + 2 * nkv) * D / 16, c.hidden, L);
    plans[PROJ_GU] = plan_panel(PROJ_GU, M, cdiv(c.ffn, 8), c.hidden, L);
    if (lora) plans[PROJ_LORA] = plan_panel(PROJ_LORA, M, c.lora_rank / 16, nq * D, L);
    for (int l = 0; l < c.n_layers; ++l) {
        const nld_layer_weights& W = mdl->layers[l];
        uint16_t* kc = (uint16_t*)kv->k + (size_t)l * kv_layer;
        uint16_t* vc = (uint16_t*)kv->v + (size_t)l * kv_layer;

        GemmArgs g{};
        g.eps = c.rms_eps;
        g.n_ss = n_ss;
        g.M = M;
        g.K = c.hidden;
        g.W = (const uint4*)W.w_qkv;
        g.n_tiles = (nq + 2 * nkv) * D / 16;
        g.ksteps = ks_h;
        g.q_out = at<uint16_t>(ws, L.q);
        g.q_row_tiles = L.row_tiles;
        g.kc = kc;
        g.vc = vc;
        g.write_cache = !io.paged && (io.mode == NLD_MODE_VERIFY || io.mode == NLD_MODE_QUAD_INTERNAL);   // quad: chain rows
        g.quad_k = io.quad_k;
        g.blk_k = at<uint16_t>(ws, L.blk_k);
        g.blk_v = at<uint16_t>(ws, L.blk_v);
        g.lengths = kv->lengths;
        g.k_blk = k;
        g.n_q_heads = nq;
        g.n_kv_heads = nkv;
        g.head_dim = D;
        g.max_len = kv->max_len;
        g.rope = at<float2>(ws, L.rope);
        g.status = status;
        g.plain = plain & (SITE_Q | SITE_KV);
        {
            TraceScope ts(NLD_TRACE_QKV, s);
            HIP_TRY(normed_gemm(PROJ_QKV, EPI_QKV, plans, g, ws, L, s));
        }
        if (io.kv_only && l == c.n_layers - 1) break;   // every layer's K/V rows are written

        if (io.paged) {
            TraceScope ts(NLD_TRACE_ATTENTION, s);
            HIP_TRY(paged_attention(mdl, *io.paged, io.mode, io.bidir_from, l, k, plain, ws, L, s));
        }
        AttnArgs at_{};
        at_.q = at<uint16_t>(ws, L.q);
        at_.kc = kc;
        at_.vc = vc;
        at_.lengths = kv->lengths;
        at_.o = at<uint16_t>(ws, L.o);
        at_.blk_k = at<uint16_t>(ws, L.blk_k);
        at_.blk_v = at<uint16_t>(ws, L.blk_v);
        at_.part_o = at<float>(ws, L.po);
        at_.part_ml = at<float>(ws, L.pml);
        at_.k_blk = k;
        at_.n_q_heads = nq;
        at_.n_kv_heads = nkv;
        at_.max_len = kv->max_len;
        at_.n_splits = L.n_splits;
        at_.chunk = L.chunk;
        at_.mode = io.mode;
        at_.bidir_from = io.bidir_from;
        at_.rows_pad = L.rows_pad;
        at_.row_tiles = L.row_tiles;
        at_.quad_k = io.quad_k;
        at_.n_parts = L.n_parts;
        at_.items = L.attn_items ? 1 : 0;
        at_.n_seq = batch;
        at_.scale_log2 = (float)(1.4426950408889634 / sqrt((double)D));
        at_.plain = plain & (SITE_P | SITE_O);
        if (!io.paged) {
            TraceScope ts(NLD_TRACE_ATTENTION, s);
            HIP_TRY(launch_attention(D, L.attn_kh, L.attn_waves, L.attn_z, L.units, at_, s));
            HIP_TRY(launch_attention_combine(D, L.units, (nq / nkv) * k, at_, s));
        }

        GemmArgs go{};
        go.A = at<uint16_t>(ws, L.o);
        go.M = M;
        go.K = nq * D;
        go.W = (const uint4*)W.w_o;
        go.n_tiles = c.hidden / 16;
        go.ksteps = ks_q;
        if (lora) {
            // LoRA down-projection t = lora_scale * (A o), split; the O projection then takes
            // B as lora_rank / 32 more k-steps against t
            GemmArgs gt{};
            gt.A = at<uint16_t>(ws, L.o);
            gt.M = M;
            gt.K = nq * D;
            gt.W = (const uint4*)W.lora_a;
            gt.n_tiles = c.lora_rank / 16;
            gt.ksteps = ks_q;
            gt.xg_out = at<uint16_t>(ws, L.lora_t);
            gt.out_scale = c.lora_scale;
            {
                TraceScope ts(NLD_TRACE_O_PROJ, s);
                HIP_TRY(panel_gemm(EPI_SPLIT, plans[PROJ_LORA], gt, ws, L, s, nullptr));
            }
            go.W2 = (const uint4*)W.lora_b;
            go.A2 = at<uint16_t>(ws, L.lora_t);
            go.ksteps2 = c.lora_rank / 32;
        }
        go.x = x;
        go.xg_out = at<uint16_t>(ws, L.xg);
        go.gain_next = (const uint16_t*)W.ffn_norm;
        go.part_ss_out = at<float>(ws, L.part_ss);
        go.plain = plain & SITE_NORM;
        {
            TraceScope ts(NLD_TRACE_O_PROJ, s);
            HIP_TRY(resid_gemm(PROJ_O, plans, go, ws, L, s, &n_ss));
        }

        GemmArgs gu{};
        gu.eps = c.rms_eps;
        gu.n_ss = n_ss;
        gu.M = M;
        gu.K = c.hidden;
        gu.W = (const uint4*)W.w_gate_up;
        gu.n_tiles = cdiv(c.ffn, 8);
        gu.ksteps = ks_h;
        gu.act = at<uint16_t>(ws, L.act);
        gu.ffn = c.ffn;
        gu.plain = plain & SITE_ACT;
        {
            TraceScope ts(NLD_TRACE_GATE_UP, s);
            HIP_TRY(normed_gemm(PROJ_GU, EPI_SWIGLU, plans, gu, ws, L, s));
        }

        GemmArgs gd{};
        gd.A = at<uint16_t>(ws, L.act);
        gd.M = M;
        gd.K = c.ffn;
        gd.W = (const uint4*)W.w_down;
        gd.n_tiles = c.hidden / 16;
        gd.ksteps = ks_f;
        gd.x = x;
        gd.xg_out = at<uint16_t>(ws, L.xg);
        gd.gain_next = (const uint16_t*)(l + 1 < c.n_layers ? mdl->layers[l + 1].attn_norm : mdl->w.final_norm);
        gd.part_ss_out = at<float>(ws, L.part_ss);
        gd.plain = plain & (l + 1 < c.n_layers ? SITE_NORM : SITE_FINAL);
        {
            TraceScope ts(NLD_TRACE_DOWN, s);
            HIP_TRY(resid_gemm(PROJ_DOWN, plans, gd, ws, L, s, &n_ss));
        }
    }

    FinishArgs fa{};
    fa.k_blk = k;
    fa.batch = batch;
    fa.finish = io.finish;
    fa.status = status;
    fa.max_len = kv->max_len;
    fa.mask_id = c.mask_token_id;
    if (io.kv_only) {
        fa.block = io.block;
        fa.next_anchor = io.next_anchor;
        fa.lengths = kv->lengths;
        TraceScope ts(NLD_TRACE_ARGMAX, s);
        HIP_TRY(launch_finish(fa, s));
        return NLD_OK;
    }

    const bool denoise = io.finish == FINISH_DENOISE;
    const bool ensemble = io.finish == FINISH_QUAD && io.lambda > 0.0f && io.lambda < 1.0f;
    GemmArgs gl{};
    gl.tile_ctr = at<unsigned>(ws, L.tile_ctr);
    gl.eps = c.rms_eps;
    gl.n_ss = n_ss;
    gl.M = M;
    gl.K = c.hidden;
    gl.W = (const uint4*)mdl->w.lm_head;
    gl.n_tiles = L.lm_tiles;
    gl.ksteps = ks_h;
    gl.logits = io.logits;
    gl.part_keys = at<unsigned long long>(ws, L.keys);
    gl.n_keys = n_keys;
    gl.part_lse = (denoise || ensemble) ? at<float2>(ws, L.lse) : nullptr;
    gl.exclude_id = denoise ? c.mask_token_id : -1;
    gl.k_blk = k;
    gl.quad_k = io.quad_k;
    gl.ens_logits = ensemble ? at<float>(ws, L.ens_logits) : nullptr;
    gl.vocab = c.vocab;
    {
        TraceScope ts(NLD_TRACE_LM_HEAD, s);
        HIP_TRY(normed_gemm(PROJ_LM, EPI_LMHEAD, plans, gl, ws, L, s));
    }

    fa.part_keys = at<unsigned long long>(ws, L.keys);
    fa.part_lse = at<float2>(ws, L.lse);
    fa.n_keys = n_keys;
    fa.n_parts = parts;
    fa.vocab = c.vocab;
    fa.argmax_out = io.argmax_out;
    fa.block = io.block;
    fa.threshold = io.threshold;
    fa.n_committed = io.n_committed;
    fa.n_masked = io.n_masked;
    fa.conf_out = io.conf_out;
    fa.draft_in = io.draft_in;
    fa.draft_out = io.draft_out;
    fa.accept_len = io.accept_len;
    fa.committed = io.committed;
    fa.next_anchor = io.next_anchor;
    fa.lengths = io.advance_lengths ? kv->lengths : nullptr;
    if (io.finish == FINISH_QUAD) {
        fa.quad_k = io.quad_k;
        fa.lambda = io.lambda;
        fa.ens_logits = at<float>(ws, L.ens_logits);
        fa.ens_keys = at<unsigned long long>(ws, L.ens_v);
        fa.ens_chunks = ENS_CHUNKS;
        TraceScope ts(NLD_TRACE_ARGMAX, s);
        if (ensemble) HIP_TRY(launch_quad_ensemble(fa, s));
        HIP_TRY(launch_quad_finish(fa, s));
        return NLD_OK;
    }
    {
        TraceScope ts(NLD_TRACE_ARGMAX, s);
        HIP_TRY(launch_finish(fa, s));
    }
    return NLD_OK;
}

// ---------------------------------------------------------------- rows of logits
constexpr int MAX_LOGIT_ROWS = 1 << 20;
static_assert(TOP_MAX == NLD_TOP_MAX, "entries per row");

// The workspace of an operator on rows of logits: the status word, the partial statistics of rows that several
// workgroups share, and their largest keys (the top selection) or the entries' logits (the losses).  Few rows are
// shared by up to SHARED_WGS workgroups per CU in all, and there is room for those whatever the rows, so that a
// workspace also serves calls of fewer rows, columns and entries; very long rows are shared by as many as they need.
enum LogitsOp { OP_TOP = 0, OP_LOSS = 1, OP_LOSS_GRAD = 2 };

struct LogitsLayout {
    RowPlan plan;
    size_t part, entries, total;
};

LogitsLayout make_logits_layout(LogitsOp op, int bf16, int n_rows, int vocab, int n_top) {
    LogitsLayout L{};
    const int cus = device_cus();
    L.plan = op == OP_TOP ? plan_top(bf16, n_rows, vocab, n_top, cus) : plan_loss(bf16, n_rows, vocab, n_top, op == OP_LOSS_GRAD, cus);
    size_t shared = (size_t)SHARED_WGS * cus;
    if (L.plan.chunks > 1) shared = std::max(shared, (size_t)n_rows * L.plan.chunks);
    L.part = 256;
    L.entries = align256(L.part + sizeof(ChunkStat) * shared);
    L.total = align256(L.entries + 8 * shared * top_places(n_top));
    return L;
}

// A launch holds less than 2^32 threads: 2^21 workgroups of up to 1024, and of a long row one takes at most LOSS_MAX_COLS
// columns.
bool one_launch(int n_rows, int vocab) { return (long long)n_rows * (vocab / LOSS_MAX_COLS + 2) <= (1 << 21); }

nld_status check_logits(const nld_logits* z, const char* what) {
    if (!z || !z->data) return fail(NLD_ERR_INVALID_ARG, "%s or its data is NULL", what);
    if (z->dtype != NLD_F32 && z->dtype != NLD_BF16) return fail(NLD_ERR_INVALID_ARG, "%s: dtype must be NLD_F32 or NLD_BF16", what);
    if (z->batch < 1 || z->rows < 1 || z->vocab < 1) return fail(NLD_ERR_INVALID_ARG, "%s: sizes must be positive", what);
    if (z->seq_stride < 0 || z->row_stride < 0 || z->seq_stride >> 40 || z->row_stride >> 40)
        return fail(NLD_ERR_INVALID_ARG, "%s: strides must be in [0, 2^40)", what);
    if ((uintptr_t)z->data % (z->dtype == NLD_BF16 ? 2 : 4)) return fail(NLD_ERR_INVALID_ARG, "%s: data is not aligned to its type", what);
    if (z->vocab > NLD_LOGITS_MAX_VOCAB) return fail(NLD_ERR_SHAPE, "%s: vocab (%d) exceeds %d", what, z->vocab, NLD_LOGITS_MAX_VOCAB);
    if ((long long)z->batch * z->rows > MAX_LOGIT_ROWS)
        return fail(NLD_ERR_SHAPE, "%s: %lld rows exceed %d", what, (long long)z->batch * z->rows, MAX_LOGIT_ROWS);
    if (!one_launch(z->batch * z->rows, z->vocab))
        return fail(NLD_ERR_SHAPE, "%s: %d rows of %d columns are too many for one call", what, z->batch * z->rows, z->vocab);
    return NLD_OK;
}

nld_status validate_logits(LogitsOp op, const nld_logits* z, int n_top, float temperature, void* ws, size_t ws_bytes,
                           LogitsLayout* out) {
    nld_status st = check_logits(z, "logits");
    if (st != NLD_OK) return st;
    if (n_top < 1 || n_top > z->vocab) return fail(NLD_ERR_INVALID_ARG, "n_top must be in [1, vocab] (got %d)", n_top);
    if (n_top > NLD_TOP_MAX) return fail(NLD_ERR_SHAPE, "n_top (%d) exceeds %d", n_top, NLD_TOP_MAX);
    if (!(temperature >= 1e-3f && temperature <= 1e3f)) return fail(NLD_ERR_INVALID_ARG, "temperature must be in [1e-3, 1e3]");
    if (!ws) return fail(NLD_ERR_INVALID_ARG, "workspace is NULL");
    *out = make_logits_layout(op, z->dtype == NLD_BF16, z->batch * z->rows, z->vocab, n_top);
    if (ws_bytes < out->total) return fail(NLD_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, out->total);
    return NLD_OK;
}

LogitRows logit_rows(const nld_logits* z) {
    return LogitRows{z->data, z->dtype == NLD_BF16, z->batch, z->rows, z->vocab, z->seq_stride, z->row_stride};
}

// elements from the first one to past the last one
long long logits_extent(const nld_logits* z) {
    return (z->batch - 1) * z->seq_stride + (z->rows - 1) * z->row_stride + z->vocab;
}

// what both losses share; grad: of the logits' dtype and sizes, its rows apart from each other, and either the logits
// themselves or apart from them
nld_status loss_args(const nld_logits* z, const nld_logits* grad, float temperature, const float* weight, const int32_t* last_row,
                     float* loss, float* aux, void* ws, const LogitsLayout& L, LossArgs* out) {
    LossArgs a{};
    if (grad) {
        nld_status st = check_logits(grad, "grad");
        if (st != NLD_OK) return st;
        if (grad->dtype != z->dtype || grad->batch != z->batch || grad->rows != z->rows || grad->vocab != z->vocab)
            return fail(NLD_ERR_INVALID_ARG, "grad must have the logits' dtype and sizes");
        const long long rs = grad->rows > 1 ? grad->row_stride : LLONG_MAX, ss = grad->batch > 1 ? grad->seq_stride : LLONG_MAX;
        const long long inner = std::min(rs, ss), outer = std::max(rs, ss);
        const long long n_inner = rs <= ss ? grad->rows : grad->batch;
        if (inner < grad->vocab || (outer != LLONG_MAX && outer < (n_inner - 1) * inner + grad->vocab))
            return fail(NLD_ERR_INVALID_ARG, "rows of grad overlap each other");
        const size_t es = z->dtype == NLD_BF16 ? 2 : 4;
        const char *z0 = (const char*)z->data, *z1 = z0 + logits_extent(z) * es;
        const char *g0 = (const char*)grad->data, *g1 = g0 + logits_extent(grad) * es;
        const bool same = g0 == z0 && (grad->batch == 1 || grad->seq_stride == z->seq_stride) &&
                          (grad->rows == 1 || grad->row_stride == z->row_stride);
        if (!same && g0 < z1 && z0 < g1)
            return fail(NLD_ERR_INVALID_ARG, "grad overlaps the logits without being the same buffer with the same strides");
        a.grad = grad->data;
        a.grad_seq_stride = grad->seq_stride;
        a.grad_row_stride = grad->row_stride;
    }
    a.in = logit_rows(z);
    a.c_exact = LOG2E / (double)temperature;
    a.c = (float)a.c_exact;
    a.inv_tau = 1.0 / (double)temperature;
    a.weight = weight;
    a.last_row = last_row;
    a.loss = loss;
    a.aux = aux;
    a.status = at<uint32_t>(ws, 0);
    a.plan = L.plan;
    a.part = at<ChunkStat>(ws, L.part);
    a.saved = at<uint2>(ws, L.entries);
    *out = a;
    return NLD_OK;
}

}  // namespace

// =====================================================================================
extern "C" {

const char* nld_last_error(void) { return g_err; }

const char* nld_status_string(int32_t st) {
    switch (st) {
        case NLD_OK: return "ok";
        case NLD_ERR_INVALID_ARG: return "invalid argument";
        case NLD_ERR_SHAPE: return "unsupported shape";
        case NLD_ERR_CAPACITY: return "workspace too small";
        case NLD_ERR_HIP: return "HIP runtime error";
        case NLD_ERR_UNSUPPORTED: return "unsupported";
        case NLD_ERR_DEVICE: return "device-side error";
        default: return "unknown status";
    }
}

nld_status nld_model_create(const nld_config* cfg, const nld_weights* w, nld_model** out) {
    if (!out) return fail(NLD_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    nld_status st = check_config(cfg);
    if (st != NLD_OK) return st;
    if (!w || !w->embed || !w->final_norm || !w->lm_head || !w->layers)
        return fail(NLD_ERR_INVALID_ARG, "a model-level weight pointer is NULL");
    for (int l = 0; l < cfg->n_layers; ++l) {
        const nld_layer_weights& L = w->layers[l];
        if (!L.attn_norm || !L.w_qkv || !L.w_o || !L.ffn_norm || !L.w_gate_up || !L.w_down)
            return fail(NLD_ERR_INVALID_ARG, "a weight pointer of layer %d is NULL", l);
        if (cfg->lora_rank > 0 && (!L.lora_a || !L.lora_b))
            return fail(NLD_ERR_INVALID_ARG, "lora_rank > 0 but layer %d has no lora_a/lora_b", l);
    }
    nld_model* m = new nld_model;
    m->cfg = *cfg;
    m->w = *w;
    m->layers.assign(w->layers, w->layers + cfg->n_layers);
    m->w.layers = m->layers.data();
    *out = m;
    return NLD_OK;
}

void nld_model_destroy(nld_model* m) { delete m; }

size_t nld_packed_bytes(int32_t kind, const nld_config* cfg, int32_t out_dim, int32_t in_dim) {
    if (in_dim < 1 || out_dim < 1) return 0;
    int tiles;
    if (kind == NLD_PACK_GATE_UP) tiles = cdiv(out_dim, 8);            // out_dim = ffn
    else if (kind == NLD_PACK_QKV) {
        if (!cfg) return 0;
        tiles = (cfg->n_q_heads + 2 * cfg->n_kv_heads) * cfg->head_dim / 16;
    } else tiles = cdiv(out_dim, 16);
    return (size_t)tiles * cdiv(in_dim, 32) * 1024;
}

nld_status nld_pack_linear(const void* w, int32_t out_dim, int32_t in_dim, void* packed, void* stream) {
    if (!w || !packed) return fail(NLD_ERR_INVALID_ARG, "NULL pointer");
    if (out_dim < 1 || in_dim < 1) return fail(NLD_ERR_INVALID_ARG, "sizes must be positive");
    if (in_dim % 8) return fail(NLD_ERR_SHAPE, "in_dim (%d) must be a multiple of 8", in_dim);
    PackArgs p{};
    p.src0 = (const uint16_t*)w;
    p.kind = PACK_LINEAR;
    p.out_dim = out_dim;
    p.in_dim = in_dim;
    p.n_tiles = cdiv(out_dim, 16);
    p.ksteps = cdiv(in_dim, 32);
    p.dst = (uint4*)packed;
    HIP_TRY(launch_pack(p, (hipStream_t)stream));
    return NLD_OK;
}

nld_status nld_pack_qkv(const nld_config* cfg, const void* wq, const void* wk, const void* wv, void* packed,
                        void* stream) {
    nld_status st = check_config(cfg);
    if (st != NLD_OK) return st;
    if (!wq || !wk || !wv || !packed) return fail(NLD_ERR_INVALID_ARG, "NULL pointer");
    PackArgs p{};
    p.src0 = (const uint16_t*)wq;
    p.src1 = (const uint16_t*)wk;
    p.src2 = (const uint16_t*)wv;
    p.kind = PACK_QKV;
    p.head_dim = cfg->head_dim;
    p.rows0 = cfg->n_q_heads * cfg->head_dim;
    p.rows1 = cfg->n_kv_heads * cfg->head_dim;
    p.out_dim = p.rows0 + 2 * p.rows1;
    p.in_dim = cfg->hidden;
    p.n_tiles = p.out_dim / 16;
    p.ksteps = cdiv(cfg->hidden, 32);
    p.dst = (uint4*)packed;
    HIP_TRY(launch_pack(p, (hipStream_t)stream));
    return NLD_OK;
}

nld_status nld_pack_gate_up(const nld_config* cfg, const void* wg, const void* wu, void* packed, void* stream) {
    nld_status st = check_config(cfg);
    if (st != NLD_OK) return st;
    if (!wg || !wu || !packed) return fail(NLD_ERR_INVALID_ARG, "NULL pointer");
    PackArgs p{};
    p.src0 = (const uint16_t*)wg;
    p.src1 = (const uint16_t*)wu;
    p.kind = PACK_GATE_UP;
    p.rows0 = cfg->ffn;
    p.out_dim = 2 * cfg->ffn;
    p.in_dim = cfg->hidden;
    p.n_tiles = cdiv(cfg->ffn, 8);
    p.ksteps = cdiv(cfg->hidden, 32);
    p.dst = (uint4*)packed;
    HIP_TRY(launch_pack(p, (hipStream_t)stream));
    return NLD_OK;
}

size_t nld_workspace_bytes(const nld_model* m, int32_t batch, int32_t k, int32_t max_len) {
    if (!m || batch < 1 || k < 1 || max_len < 64) return 0;
    return make_layout(m->cfg, batch, k, max_len).total;
}

nld_status nld_workspace_init(void* workspace, size_t ws_bytes, void* stream) {
    if (!workspace) return fail(NLD_ERR_INVALID_ARG, "workspace is NULL");
    if (ws_bytes < 256) return fail(NLD_ERR_CAPACITY, "workspace too small");
    HIP_TRY(launch_fill_zero(workspace, ws_bytes & ~(size_t)3, (hipStream_t)stream));
    return NLD_OK;
}

nld_status nld_block_forward(const nld_model* m, const nld_kv_cache* kv, const int32_t* tokens, int32_t batch,
                             int32_t k, int32_t mode, int32_t bidir_from, float* logits, int32_t* argmax,
                             void* workspace, size_t ws_bytes, void* stream) {
    Layout L;
    nld_status st = validate_call(m, kv, batch, k, workspace, ws_bytes, &L);
    if (st != NLD_OK) return st;
    if (!tokens) return fail(NLD_ERR_INVALID_ARG, "tokens is NULL");
    if (mode != NLD_MODE_VERIFY && mode != NLD_MODE_DRAFT) return fail(NLD_ERR_INVALID_ARG, "mode must be 0 or 1");
    if (bidir_from < 0 || bidir_from > k) return fail(NLD_ERR_INVALID_ARG, "bidir_from must be in [0, k]");
    PassIO io{};
    io.source = SRC_TOKENS;
    io.tokens = tokens;
    io.mode = mode;
    io.bidir_from = bidir_from;
    io.logits = logits;
    io.argmax_out = argmax;
    io.finish = FINISH_NONE;
    return run_pass(m, kv, batch, k, io, workspace, L, (hipStream_t)stream);
}

nld_status nld_draft(const nld_model* m, const nld_kv_cache* kv, const int32_t* anchor, int32_t batch, int32_t k,
                     int32_t bidir_from, int32_t* draft, float* logits, void* workspace, size_t ws_bytes,
                     void* stream) {
    Layout L;
    nld_status st = validate_call(m, kv, batch, k, workspace, ws_bytes, &L);
    if (st != NLD_OK) return st;
    if (k < 2) return fail(NLD_ERR_INVALID_ARG, "a draft needs k >= 2");
    if (!anchor || !draft) return fail(NLD_ERR_INVALID_ARG, "anchor or draft is NULL");
    if (bidir_from < 0 || bidir_from > k) return fail(NLD_ERR_INVALID_ARG, "bidir_from must be in [0, k]");
    PassIO io{};
    io.source = SRC_DRAFT;
    io.anchor = anchor;
    io.mode = NLD_MODE_DRAFT;
    io.bidir_from = bidir_from;
    io.logits = logits;
    io.finish = FINISH_DRAFT;
    io.draft_out = draft;
    return run_pass(m, kv, batch, k, io, workspace, L, (hipStream_t)stream);
}

nld_status nld_verify_accept(const nld_model* m, const nld_kv_cache* kv, const int32_t* anchor,
                             const int32_t* draft, int32_t batch, int32_t k, int32_t* accept_len,
                             int32_t* committed, int32_t* next_anchor, float* logits, void* workspace,
                             size_t ws_bytes, void* stream) {
    Layout L;
    nld_status st = validate_call(m, kv, batch, k, workspace, ws_bytes, &L);
    if (st != NLD_OK) return st;
    if (!anchor || !accept_len || !committed || !next_anchor)
        return fail(NLD_ERR_INVALID_ARG, "anchor, accept_len, committed or next_anchor is NULL");
    if (k > 1 && !draft) return fail(NLD_ERR_INVALID_ARG, "draft is NULL");
    PassIO io{};
    io.source = SRC_VERIFY;
    io.anchor = anchor;
    io.draft_in = draft;
    io.mode = NLD_MODE_VERIFY;
    io.logits = logits;
    io.finish = FINISH_ACCEPT;
    io.accept_len = accept_len;
    io.committed = committed;
    io.next_anchor = next_anchor;
    io.advance_lengths = true;
    return run_pass(m, kv, batch, k, io, workspace, L, (hipStream_t)stream);
}

size_t nld_quad_workspace_bytes(const nld_model* m, int32_t batch, int32_t k, int32_t max_len) {
    if (!m || batch < 1 || k < 2 || k > NLD_QUAD_MAX_K || max_len < 1) return 0;
    return make_layout(m->cfg, batch, k * (k + 1), max_len, k).total;
}

nld_status nld_quad_step(const nld_model* m, const nld_kv_cache* kv, const int32_t* anchor, const int32_t* spec,
                         int32_t batch, int32_t k, float lambda, int32_t* accept_len, int32_t* committed,
                         int32_t* next_anchor, int32_t* next_spec, float* logits, void* workspace, size_t ws_bytes,
                         void* stream) {
    if (k < 2 || k > NLD_QUAD_MAX_K) return fail(NLD_ERR_INVALID_ARG, "quadratic k must be in [2, %d] (got %d)",
                                                 NLD_QUAD_MAX_K, k);
    if (!(lambda >= 0.0f && lambda <= 1.0f)) return fail(NLD_ERR_INVALID_ARG, "lambda must be in [0, 1]");
    Layout L;
    nld_status st = validate_call(m, kv, batch, k * (k + 1), workspace, ws_bytes, &L, k);
    if (st != NLD_OK) return st;
    if (!anchor || !spec || !accept_len || !committed || !next_anchor || !next_spec)
        return fail(NLD_ERR_INVALID_ARG, "anchor, spec, accept_len, committed, next_anchor or next_spec is NULL");
    PassIO io{};
    io.source = SRC_QUAD;
    io.anchor = anchor;
    io.draft_in = spec;
    io.mode = NLD_MODE_QUAD_INTERNAL;
    io.logits = logits;
    io.finish = FINISH_QUAD;
    io.accept_len = accept_len;
    io.committed = committed;
    io.next_anchor = next_anchor;
    io.draft_out = next_spec;
    io.advance_lengths = true;
    io.quad_k = k;
    io.lambda = lambda;
    return run_pass(m, kv, batch, k * (k + 1), io, workspace, L, (hipStream_t)stream);
}

nld_status nld_denoise_step(const nld_model* m, const nld_kv_cache* kv, int32_t* block, int32_t batch, int32_t k,
                            int32_t bidir_from, float threshold, int32_t* n_committed, int32_t* n_masked,
                            float* confidence, float* logits, void* workspace, size_t ws_bytes, void* stream) {
    Layout L;
    nld_status st = validate_call(m, kv, batch, k, workspace, ws_bytes, &L);
    if (st != NLD_OK) return st;
    if (k < 2) return fail(NLD_ERR_INVALID_ARG, "a denoising step needs k >= 2");
    if (m->cfg.vocab < 2) return fail(NLD_ERR_SHAPE, "denoising needs a vocabulary besides the mask token");
    if (!block || !n_committed || !n_masked) return fail(NLD_ERR_INVALID_ARG, "block, n_committed or n_masked is NULL");
    if (bidir_from < 0 || bidir_from > k) return fail(NLD_ERR_INVALID_ARG, "bidir_from must be in [0, k]");
    if (threshold != threshold) return fail(NLD_ERR_INVALID_ARG, "threshold is NaN");
    PassIO io{};
    io.source = SRC_TOKENS;
    io.tokens = block;
    io.mode = NLD_MODE_DRAFT;
    io.bidir_from = bidir_from;
    io.logits = logits;
    io.finish = FINISH_DENOISE;
    io.block = block;
    io.threshold = threshold;
    io.n_committed = n_committed;
    io.n_masked = n_masked;
    io.conf_out = confidence;
    return run_pass(m, kv, batch, k, io, workspace, L, (hipStream_t)stream);
}

nld_status nld_refresh_block(const nld_model* m, const nld_kv_cache* kv, const int32_t* block, int32_t batch,
                             int32_t k, int32_t* next_anchor, void* workspace, size_t ws_bytes, void* stream) {
    Layout L;
    nld_status st = validate_call(m, kv, batch, k, workspace, ws_bytes, &L);
    if (st != NLD_OK) return st;
    if (k < 2) return fail(NLD_ERR_INVALID_ARG, "a refresh needs k >= 2");
    if (!block || !next_anchor) return fail(NLD_ERR_INVALID_ARG, "block or next_anchor is NULL");
    PassIO io{};
    io.source = SRC_TOKENS;
    io.tokens = block;
    io.mode = NLD_MODE_VERIFY;
    io.finish = FINISH_REFRESH;
    io.block = (int32_t*)block;   // read only
    io.next_anchor = next_anchor;
    io.kv_only = true;
    return run_pass(m, kv, batch, k, io, workspace, L, (hipStream_t)stream);
}

nld_status nld_commit_from_logits(const float* logits, int32_t* block, int32_t batch, int32_t k, int32_t vocab,
                                  int32_t mask_token_id, float threshold, int32_t* argmax, int32_t* n_committed,
                                  int32_t* n_masked, float* confidence, void* stream) {
    if (!logits || !block || !n_committed || !n_masked) return fail(NLD_ERR_INVALID_ARG, "NULL pointer");
    if (batch < 1 || k < 2 || k > 64 || vocab < 2) return fail(NLD_ERR_INVALID_ARG, "bad batch, k or vocab");
    if (mask_token_id < 0 || mask_token_id >= vocab) return fail(NLD_ERR_INVALID_ARG, "mask_token_id outside [0, vocab)");
    if (threshold != threshold) return fail(NLD_ERR_INVALID_ARG, "threshold is NaN");
    FinishArgs fa{};
    fa.logits = logits;
    fa.vocab = vocab;
    fa.k_blk = k;
    fa.batch = batch;
    fa.argmax_out = argmax;
    fa.finish = FINISH_DENOISE;
    fa.block = block;
    fa.mask_id = mask_token_id;
    fa.threshold = threshold;
    fa.n_committed = n_committed;
    fa.n_masked = n_masked;
    fa.conf_out = confidence;
    HIP_TRY(launch_finish(fa, (hipStream_t)stream));
    return NLD_OK;
}

nld_status nld_decode_steps(const nld_model* m, const nld_kv_cache* kv, int32_t* anchor, int32_t batch, int32_t k,
                            int32_t n_steps, int32_t bidir_from, int32_t* accept_len, int32_t* committed,
                            void* workspace, size_t ws_bytes, void* stream) {
    Layout L;
    nld_status st = validate_call(m, kv, batch, k, workspace, ws_bytes, &L);
    if (st != NLD_OK) return st;
    if (n_steps < 1) return fail(NLD_ERR_INVALID_ARG, "n_steps must be >= 1");
    if (!anchor || !accept_len || !committed) return fail(NLD_ERR_INVALID_ARG, "anchor, accept_len or committed is NULL");
    if (bidir_from < 0 || bidir_from > k) return fail(NLD_ERR_INVALID_ARG, "bidir_from must be in [0, k]");
    int32_t* drafts = at<int32_t>(workspace, L.drafts);
    hipStream_t s = (hipStream_t)stream;
    for (int step = 0; step < n_steps; ++step) {
        if (k >= 2) {
            PassIO d{};
            d.source = SRC_DRAFT;
            d.anchor = anchor;
            d.mode = NLD_MODE_DRAFT;
            d.bidir_from = bidir_from;
            d.finish = FINISH_DRAFT;
            d.draft_out = drafts;
            st = run_pass(m, kv, batch, k, d, workspace, L, s);
            if (st != NLD_OK) return st;
        }
        PassIO v{};
        v.source = SRC_VERIFY;
        v.anchor = anchor;
        v.draft_in = drafts;
        v.mode = NLD_MODE_VERIFY;
        v.finish = FINISH_ACCEPT;
        v.accept_len = accept_len + (size_t)step * batch;
        v.committed = committed + (size_t)step * batch * k;
        v.next_anchor = anchor;   // written last by the finish kernel: the next step's anchor
        v.advance_lengths = true;
        st = run_pass(m, kv, batch, k, v, workspace, L, s);
        if (st != NLD_OK) return st;
    }
    return NLD_OK;
}

int32_t nld_choose_block(float ar_step_ms, float ss_step_ms, float expected_committed, int32_t k_ss) {
    if (!(ar_step_ms > 0.f) || !(ss_step_ms > 0.f) || k_ss < 2) return 1;
    // committed tokens per millisecond: 1 per AR step, expected_committed per self-speculation step
    return expected_committed / ss_step_ms > 1.0f / ar_step_ms ? k_ss : 1;
}

size_t nld_accept_workspace_bytes(int32_t batch, int32_t k) {
    if (batch < 1 || k < 1) return 0;
    return 256;
}

nld_status nld_accept_from_logits(const float* logits, const int32_t* draft, int32_t batch, int32_t k,
                                  int32_t vocab, int32_t* argmax, int32_t* accept_len, int32_t* committed,
                                  int32_t* next_anchor, void* workspace, size_t ws_bytes, void* stream) {
    if (!logits || !argmax || !accept_len || !committed || !next_anchor || !workspace)
        return fail(NLD_ERR_INVALID_ARG, "NULL pointer");
    if (batch < 1 || k < 1 || k > 64 || vocab < 1) return fail(NLD_ERR_INVALID_ARG, "bad batch, k or vocab");
    if (k > 1 && !draft) return fail(NLD_ERR_INVALID_ARG, "draft is NULL");
    if (ws_bytes < nld_accept_workspace_bytes(batch, k)) return fail(NLD_ERR_CAPACITY, "workspace too small");
    FinishArgs fa{};
    fa.part_keys = nullptr;
    fa.logits = logits;
    fa.vocab = vocab;
    fa.k_blk = k;
    fa.batch = batch;
    fa.argmax_out = argmax;
    fa.finish = FINISH_ACCEPT;
    fa.draft_in = draft;
    fa.accept_len = accept_len;
    fa.committed = committed;
    fa.next_anchor = next_anchor;
    HIP_TRY(launch_finish(fa, (hipStream_t)stream));
    return NLD_OK;
}

size_t nld_logits_workspace_bytes(int32_t batch, int32_t rows, int32_t vocab, int32_t n_top) {
    if (batch < 1 || rows < 1 || vocab < 1 || n_top < 1 || n_top > NLD_TOP_MAX || n_top > vocab ||
        vocab > NLD_LOGITS_MAX_VOCAB || (long long)batch * rows > MAX_LOGIT_ROWS || !one_launch(batch * rows, vocab))
        return 0;
    size_t total = 0;
    for (LogitsOp op : {OP_TOP, OP_LOSS, OP_LOSS_GRAD})
        for (int bf16 = 0; bf16 < 2; ++bf16) total = std::max(total, make_logits_layout(op, bf16, batch * rows, vocab, n_top).total);
    return total;
}

nld_status nld_top_logits(const nld_logits* logits, int32_t n_top, float temperature, float* values, int32_t* ids,
                          float* lse, void* workspace, size_t ws_bytes, void* stream) {
    LogitsLayout L;
    nld_status st = validate_logits(OP_TOP, logits, n_top, temperature, workspace, ws_bytes, &L);
    if (st != NLD_OK) return st;
    if (!values || !ids) return fail(NLD_ERR_INVALID_ARG, "values or ids is NULL");
    TopArgs a{};
    a.in = logit_rows(logits);
    a.n_top = n_top;
    a.c_exact = LOG2E / (double)temperature;
    a.c = (float)a.c_exact;
    a.values = values;
    a.ids = ids;
    a.lse = lse;
    a.plan = L.plan;
    a.part = at<ChunkStat>(workspace, L.part);
    a.keys = at<unsigned long long>(workspace, L.entries);
    HIP_TRY(launch_top(a, (hipStream_t)stream));
    return NLD_OK;
}

nld_status nld_distill_from_logits(const nld_logits* student, const nld_teacher* teacher, float temperature,
                                   float kl_share, float eta, const float* weight, const int32_t* last_row,
                                   float* loss, float* accept, const nld_logits* grad, void* workspace,
                                   size_t ws_bytes, void* stream) {
    if (!teacher || !teacher->values || !teacher->ids) return fail(NLD_ERR_INVALID_ARG, "teacher, its values or its ids is NULL");
    LogitsLayout L;
    nld_status st = validate_logits(grad ? OP_LOSS_GRAD : OP_LOSS, student, teacher->n_top, temperature, workspace, ws_bytes, &L);
    if (st != NLD_OK) return st;
    if (teacher->seq_rows < student->rows) return fail(NLD_ERR_INVALID_ARG, "teacher->seq_rows (%d) < rows (%d)", teacher->seq_rows, student->rows);
    if (!loss) return fail(NLD_ERR_INVALID_ARG, "loss is NULL");
    if (!(kl_share >= 0.f && kl_share <= 1.f)) return fail(NLD_ERR_INVALID_ARG, "kl_share must be in [0, 1]");
    if (!(eta >= 0.f && eta < INFINITY)) return fail(NLD_ERR_INVALID_ARG, "eta must be >= 0 and finite");
    LossArgs a{};
    st = loss_args(student, grad, temperature, weight, last_row, loss, accept, workspace, L, &a);
    if (st != NLD_OK) return st;
    a.ids = teacher->ids;
    a.values = teacher->values;
    a.lse = teacher->lse;
    a.n_top = teacher->n_top;
    a.t_seq_rows = teacher->seq_rows;
    a.kl_share = kl_share;
    a.eta = eta;
    HIP_TRY(launch_loss(LOSS_DISTILL, a, (hipStream_t)stream));
    return NLD_OK;
}

nld_status nld_policy_from_logits(const nld_logits* policy, const nld_rollout* rollout, float temperature,
                                  float clip_low, float clip_high, float kl_coef, const float* weight,
                                  const int32_t* last_row, float* loss, float* logp, const nld_logits* grad,
                                  void* workspace, size_t ws_bytes, void* stream) {
    LogitsLayout L;
    nld_status st = validate_logits(grad ? OP_LOSS_GRAD : OP_LOSS, policy, 1, temperature, workspace, ws_bytes, &L);
    if (st != NLD_OK) return st;
    if (!rollout || !rollout->actions || !rollout->advantage)
        return fail(NLD_ERR_INVALID_ARG, "rollout, its actions or its advantage is NULL");
    if (!loss) return fail(NLD_ERR_INVALID_ARG, "loss is NULL");
    if (!(clip_low >= 0.f && clip_low <= 1.f)) return fail(NLD_ERR_INVALID_ARG, "clip_low must be in [0, 1]");
    if (!(clip_high >= 0.f && clip_high < INFINITY)) return fail(NLD_ERR_INVALID_ARG, "clip_high must be >= 0 and finite");
    if (!(kl_coef >= 0.f && kl_coef < INFINITY)) return fail(NLD_ERR_INVALID_ARG, "kl_coef must be >= 0 and finite");
    LossArgs a{};
    st = loss_args(policy, grad, temperature, weight, last_row, loss, logp, workspace, L, &a);
    if (st != NLD_OK) return st;
    a.actions = rollout->actions;
    a.advantage = rollout->advantage;
    a.old_logp = rollout->old_logp;
    a.ref_logp = rollout->ref_logp;
    a.clip_low = clip_low;
    a.clip_high = clip_high;
    a.kl_coef = kl_coef;
    HIP_TRY(launch_loss(LOSS_POLICY, a, (hipStream_t)stream));
    return NLD_OK;
}

int32_t nld_pages_list_len(int32_t max_rows, int32_t group, int32_t n_top, int32_t n_first, int32_t mode) {
    if (max_rows < 1 || max_rows > MAX_CHUNK_ROWS || group < 1 || group > MAX_CHUNK_ROWS || n_top < 0 || n_first < 0 ||
        n_top > MAX_SEQ_PAGES || n_first > MAX_SEQ_PAGES || (mode != NLD_MODE_VERIFY && mode != NLD_MODE_DRAFT))
        return 0;
    // a group's own pages: those of its tokens' positions, of which there are no more than rows (a draft's: of all rows)
    return n_first + n_top + ((mode == NLD_MODE_DRAFT ? max_rows : std::min(group, max_rows)) + 62) / 64 + 1;
}

size_t nld_pages_workspace_bytes(const nld_pages* pages, int32_t n_q_heads, int32_t max_rows, int32_t group) {
    if (check_pages(pages, 0) != NLD_OK || check_q_heads(pages, n_q_heads) != NLD_OK) return 0;
    if (max_rows < 1 || max_rows > MAX_CHUNK_ROWS || group < 0) {
        fail(NLD_ERR_INVALID_ARG, "max_rows must be in [1, %d] and group >= 0 (got %d and %d)", MAX_CHUNK_ROWS, max_rows, group);
        return 0;
    }
    if (group && check_group(pages, n_q_heads, group) != NLD_OK) return 0;
    const int G = n_q_heads / pages->n_kv_heads;
    PagesPlan p;
    if (!plan_pages(pages->batch, pages->n_kv_heads, pages->head_dim, G, max_rows, group, false, &p)) {
        fail(NLD_ERR_SHAPE, "%d sequences of up to %d rows are too many for one call", pages->batch, max_rows);
        return 0;
    }
    // the most that any number of rows up to these, and any type, needs: by the tiles of a workgroup
    size_t n = 0;
    const long long rows = (long long)max_rows * G;
    for (const bool raw : {false, true})
        for (long long r = 16; r == 16 || r - 32 < std::min(rows, 256LL); r = r == 16 ? 32 : r + 32)
            if (plan_pages(1, 1, pages->head_dim, 1, (int)r, 0, raw, &p)) n = std::max(n, p.parts);
    // and a note per unit, of which groups make the most
    n = align256(n + (size_t)8 * pages->batch * pages->n_kv_heads * std::max<long long>(group ? cdiv(max_rows, group) : 0, (rows + 255) / 256));
    return group ? std::max(n, align256(256 + score_bytes(pages, max_rows, group))) : n;
}

nld_status nld_pages_write(const nld_pages* pages, int32_t layer, const nld_chunk* chunk, const nld_heads* k, const nld_heads* v, void* workspace,
                           size_t ws_bytes, void* stream) {
    nld_status st = check_pages(pages, layer);
    if (st == NLD_OK) st = check_chunk(pages, chunk);
    if (st == NLD_OK) st = check_heads(k, "k", chunk->rows, pages->n_kv_heads, pages->head_dim, false);
    if (st == NLD_OK) st = check_heads(v, "v", chunk->rows, pages->n_kv_heads, pages->head_dim, false);
    if (st != NLD_OK) return st;
    if (k->dtype != v->dtype) return fail(NLD_ERR_INVALID_ARG, "k and v must have one dtype");
    if (!workspace) return fail(NLD_ERR_INVALID_ARG, "workspace is NULL");
    if (ws_bytes < 256) return fail(NLD_ERR_CAPACITY, "workspace holds %zu bytes, this call needs 256", ws_bytes);
    if (((long long)(chunk->max_rows + 62) / 64 + 1) * pages->batch * pages->n_kv_heads > MAX_PAGE_WGS)
        return fail(NLD_ERR_SHAPE, "%d sequences of up to %d rows are too many for one call", pages->batch, chunk->max_rows);
    HIP_TRY(launch_pages_write(page_layer(pages, layer), head_rows(k), head_rows(v), nullptr, nullptr, page_chunk(chunk), at<uint32_t>(workspace, 0),
                               (hipStream_t)stream));
    return NLD_OK;
}

nld_status nld_pages_read(const nld_pages* pages, int32_t layer, const nld_chunk* chunk, const int32_t* first, const nld_heads* k, const nld_heads* v,
                          void* workspace, size_t ws_bytes, void* stream) {
    nld_status st = check_pages(pages, layer);
    if (st == NLD_OK) st = check_chunk(pages, chunk);
    if (st == NLD_OK) st = check_heads(k, "k", chunk->rows, pages->n_kv_heads, pages->head_dim, true);
    if (st == NLD_OK) st = check_heads(v, "v", chunk->rows, pages->n_kv_heads, pages->head_dim, true);
    if (st != NLD_OK) return st;
    if (k->dtype != v->dtype || k->data == v->data) return fail(NLD_ERR_INVALID_ARG, "k and v must have one dtype and be apart");
    if (!workspace) return fail(NLD_ERR_INVALID_ARG, "workspace is NULL");
    if (ws_bytes < 256) return fail(NLD_ERR_CAPACITY, "workspace holds %zu bytes, this call needs 256", ws_bytes);
    if (heads_overlap(k, v, chunk->rows, pages->n_kv_heads, pages->head_dim)) return fail(NLD_ERR_INVALID_ARG, "v overlaps k");
    if (((long long)(chunk->max_rows + 62) / 64 + 1) * pages->batch * pages->n_kv_heads > MAX_PAGE_WGS)
        return fail(NLD_ERR_SHAPE, "%d sequences of up to %d rows are too many for one call", pages->batch, chunk->max_rows);
    HIP_TRY(launch_pages_read(page_layer(pages, layer), head_rows(k), head_rows(v), page_chunk(chunk), first, at<uint32_t>(workspace, 0),
                              (hipStream_t)stream));
    return NLD_OK;
}

nld_status nld_pages_attend(const nld_pages* pages, int32_t layer, const nld_chunk* chunk, const nld_heads* q, int32_t n_q_heads, float scale,
                            int32_t mode, int32_t bidir_from, const int32_t* list, int32_t n_list, int32_t group, const nld_heads* out, float* lse,
                            void* workspace, size_t ws_bytes, void* stream) {
    nld_status st = check_pages(pages, layer);
    if (st == NLD_OK) st = check_chunk(pages, chunk);
    if (st == NLD_OK) st = check_q_heads(pages, n_q_heads);
    if (st == NLD_OK) st = check_heads(q, "q", chunk->rows, n_q_heads, pages->head_dim, false);
    if (st == NLD_OK) st = check_heads(out, "out", chunk->rows, n_q_heads, pages->head_dim, true);
    if (st == NLD_OK) st = check_mode(mode, bidir_from, chunk->max_rows);
    if (st != NLD_OK) return st;
    if (!(fabsf(scale) <= 0x1p127f)) return fail(NLD_ERR_INVALID_ARG, "scale must be in [-2^127, 2^127]");   // finite in base-2 exponents too
    if (q->dtype != out->dtype) return fail(NLD_ERR_INVALID_ARG, "q and out must have one dtype");
    if (heads_overlap(q, out, chunk->rows, n_q_heads, pages->head_dim)) return fail(NLD_ERR_INVALID_ARG, "out overlaps q");
    if (list) {
        st = check_group(pages, n_q_heads, group);
        if (st != NLD_OK) return st;
        if (n_list < 1 || n_list > MAX_SEQ_PAGES) return fail(NLD_ERR_INVALID_ARG, "n_list must be in [1, %d] (got %d)", MAX_SEQ_PAGES, n_list);
    }
    if (!workspace) return fail(NLD_ERR_INVALID_ARG, "workspace is NULL");
    PagesPlan p;
    if (!plan_pages(pages->batch, pages->n_kv_heads, pages->head_dim, n_q_heads / pages->n_kv_heads, chunk->max_rows, list ? group : 0,
                    pages_raw(q->dtype == NLD_F32 ? 3 : 1, pages->dtype == NLD_E4M3), &p))
        return fail(NLD_ERR_SHAPE, "%d sequences of up to %d rows are too many for one call", pages->batch, chunk->max_rows);
    if (ws_bytes < p.total) return fail(NLD_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, p.total);
    PagesAttnArgs a = pages_args(page_layer(pages, layer), page_chunk(chunk), n_q_heads / pages->n_kv_heads, mode, bidir_from, scale, p, workspace, 0);
    a.q = head_rows(q);
    a.out = head_rows(out);
    a.list = list;
    a.n_list = n_list;
    a.group = group;
    a.lse = lse;
    HIP_TRY(launch_pages_attend(a, (hipStream_t)stream));
    return NLD_OK;
}

nld_status nld_pages_select(const nld_pages* pages, int32_t layer, const nld_chunk* chunk, const nld_heads* q, int32_t n_q_heads, int32_t n_top,
                            int32_t n_first, int32_t group, int32_t mode, int32_t bidir_from, int32_t* list, int32_t n_list, void* workspace,
                            size_t ws_bytes, void* stream) {
    nld_status st = check_pages(pages, layer);
    if (st == NLD_OK) st = check_chunk(pages, chunk);
    if (st == NLD_OK) st = check_q_heads(pages, n_q_heads);
    if (st == NLD_OK) st = check_heads(q, "q", chunk->rows, n_q_heads, pages->head_dim, false);
    if (st == NLD_OK) st = check_mode(mode, bidir_from, chunk->max_rows);
    if (st == NLD_OK) st = check_group(pages, n_q_heads, group);
    if (st != NLD_OK) return st;
    if (!pages->bounds) return fail(NLD_ERR_INVALID_ARG, "a selection needs the pages' bounds");
    if (!list) return fail(NLD_ERR_INVALID_ARG, "list is NULL");
    if (n_top < 0 || n_first < 0) return fail(NLD_ERR_INVALID_ARG, "n_top and n_first must be >= 0");
    const int need = nld_pages_list_len(chunk->max_rows, group, n_top, n_first, mode);
    if (need < 1) return fail(NLD_ERR_SHAPE, "n_top (%d) or n_first (%d) exceeds %d", n_top, n_first, MAX_SEQ_PAGES);
    if (n_list < need) return fail(NLD_ERR_INVALID_ARG, "n_list is %d, this call needs %d", n_list, need);
    if (!select_fits(pages, chunk->max_rows, group))
        return fail(NLD_ERR_SHAPE, "%d sequences of up to %d rows are too many for one call", pages->batch, chunk->max_rows);
    if (!workspace) return fail(NLD_ERR_INVALID_ARG, "workspace is NULL");
    const size_t bytes = align256(256 + (n_top ? score_bytes(pages, chunk->max_rows, group) : 0));
    if (ws_bytes < bytes) return fail(NLD_ERR_CAPACITY, "workspace holds %zu bytes, this call needs %zu", ws_bytes, bytes);
    PagesSelectArgs a{};
    a.c = page_layer(pages, layer);
    a.ch = page_chunk(chunk);
    a.q = head_rows(q);
    a.group_heads = n_q_heads / pages->n_kv_heads;
    a.draft = mode == NLD_MODE_DRAFT;
    a.bidir_from = bidir_from;
    a.n_top = n_top;
    a.n_first = n_first;
    a.group = group;
    a.n_groups = cdiv(chunk->max_rows, group);
    a.n_list = n_list;
    a.scores = at<float>(workspace, 256);
    a.list = list;
    a.status = at<uint32_t>(workspace, 0);
    HIP_TRY(launch_pages_select(a, (hipStream_t)stream));
    return NLD_OK;
}

size_t nld_pages_pass_workspace_bytes(const nld_model* m, const nld_pages* pages, const nld_sparse* sparse, int32_t k) {
    nld_kv_cache kv;
    Layout L;
    PagedPass pp;
    // a draft pass's lists are the longer ones: its groups see all rows; any pointer stands for the workspace
    return validate_paged(m, pages, sparse, k, NLD_MODE_DRAFT, &kv, ~(size_t)0, &kv, &L, &pp) == NLD_OK ? pp.total : 0;
}

nld_status nld_pages_block_forward(const nld_model* m, const nld_pages* pages, const nld_sparse* sparse, const int32_t* tokens, int32_t k, int32_t mode,
                                   int32_t bidir_from, float* logits, int32_t* argmax, void* workspace, size_t ws_bytes, void* stream) {
    nld_kv_cache kv;
    Layout L;
    PagedPass pp;
    if (mode != NLD_MODE_VERIFY && mode != NLD_MODE_DRAFT) return fail(NLD_ERR_INVALID_ARG, "mode must be 0 or 1");
    nld_status st = validate_paged(m, pages, sparse, k, mode, workspace, ws_bytes, &kv, &L, &pp);
    if (st != NLD_OK) return st;
    if (!tokens) return fail(NLD_ERR_INVALID_ARG, "tokens is NULL");
    if (bidir_from < 0 || bidir_from > k) return fail(NLD_ERR_INVALID_ARG, "bidir_from must be in [0, k]");
    PassIO io{};
    io.source = SRC_TOKENS;
    io.tokens = tokens;
    io.mode = mode;
    io.bidir_from = bidir_from;
    io.logits = logits;
    io.argmax_out = argmax;
    io.finish = FINISH_NONE;
    io.paged = &pp;
    return run_pass(m, &kv, pages->batch, k, io, workspace, L, (hipStream_t)stream);
}

nld_status nld_pages_draft(const nld_model* m, const nld_pages* pages, const nld_sparse* sparse, const int32_t* anchor, int32_t k, int32_t bidir_from,
                           int32_t* draft, float* logits, void* workspace, size_t ws_bytes, void* stream) {
    nld_kv_cache kv;
    Layout L;
    PagedPass pp;
    nld_status st = validate_paged(m, pages, sparse, k, NLD_MODE_DRAFT, workspace, ws_bytes, &kv, &L, &pp);
    if (st != NLD_OK) return st;
    if (k < 2) return fail(NLD_ERR_INVALID_ARG, "a draft needs k >= 2");
    if (!anchor || !draft) return fail(NLD_ERR_INVALID_ARG, "anchor or draft is NULL");
    if (bidir_from < 0 || bidir_from > k) return fail(NLD_ERR_INVALID_ARG, "bidir_from must be in [0, k]");
    PassIO io{};
    io.source = SRC_DRAFT;
    io.anchor = anchor;
    io.mode = NLD_MODE_DRAFT;
    io.bidir_from = bidir_from;
    io.logits = logits;
    io.finish = FINISH_DRAFT;
    io.draft_out = draft;
    io.paged = &pp;
    return run_pass(m, &kv, pages->batch, k, io, workspace, L, (hipStream_t)stream);
}

nld_status nld_pages_verify_accept(const nld_model* m, const nld_pages* pages, const nld_sparse* sparse, const int32_t* anchor, const int32_t* draft,
                                   int32_t k, int32_t* accept_len, int32_t* committed, int32_t* next_anchor, float* logits, void* workspace,
                                   size_t ws_bytes, void* stream) {
    nld_kv_cache kv;
    Layout L;
    PagedPass pp;
    nld_status st = validate_paged(m, pages, sparse, k, NLD_MODE_VERIFY, workspace, ws_bytes, &kv, &L, &pp);
    if (st != NLD_OK) return st;
    if (!anchor || !accept_len || !committed || !next_anchor)
        return fail(NLD_ERR_INVALID_ARG, "anchor, accept_len, committed or next_anchor is NULL");
    if (k > 1 && !draft) return fail(NLD_ERR_INVALID_ARG, "draft is NULL");
    PassIO io{};
    io.source = SRC_VERIFY;
    io.anchor = anchor;
    io.draft_in = draft;
    io.mode = NLD_MODE_VERIFY;
    io.logits = logits;
    io.finish = FINISH_ACCEPT;
    io.accept_len = accept_len;
    io.committed = committed;
    io.next_anchor = next_anchor;
    io.advance_lengths = true;
    io.paged = &pp;
    return run_pass(m, &kv, pages->batch, k, io, workspace, L, (hipStream_t)stream);
}

nld_status nld_trace_enable(int32_t on) {
    g_trace_on = on != 0;
    return NLD_OK;
}

nld_status nld_trace_read(float* ms, int32_t* counts, int32_t n) {
    if (!ms || !counts || n < NLD_TRACE_CLASSES) return fail(NLD_ERR_INVALID_ARG, "need host arrays of NLD_TRACE_CLASSES");
    for (int i = 0; i < n; ++i) {
        ms[i] = 0.f;
        counts[i] = 0;
    }
    nld_status st = NLD_OK;
    for (TraceRec& r : g_trace) {
        float t = 0.f;
        if (st == NLD_OK) {
            hipError_t e = hipEventSynchronize(r.stop);
            if (e == hipSuccess) e = hipEventElapsedTime(&t, r.start, r.stop);
            if (e != hipSuccess) st = fail(NLD_ERR_HIP, "trace event: %s", hipGetErrorString(e));
        }
        ms[r.cls] += t;
        counts[r.cls] += r.first ? 1 : 0;
        (void)hipEventDestroy(r.start);
        (void)hipEventDestroy(r.stop);
    }
    g_trace.clear();
    return st;
}

nld_status nld_read_device_status(void* workspace, uint32_t* host_bits, void* stream) {
    if (!workspace || !host_bits) return fail(NLD_ERR_INVALID_ARG, "NULL pointer");
    hipStream_t s = (hipStream_t)stream;
    HIP_TRY(hipStreamSynchronize(s));
    HIP_TRY(hipMemcpy(host_bits, workspace, 4, hipMemcpyDeviceToHost));
    HIP_TRY(launch_fill_zero(workspace, 4, s));
    HIP_TRY(hipStreamSynchronize(s));
    if (*host_bits) return fail(NLD_ERR_DEVICE, "device status bits 0x%x", *host_bits);
    return NLD_OK;
}

}  // extern "C"

// ---------------------------------------------------------------- allocation-free verify
// The scratch of nld_verify_accept_noalloc: one copy per device, loaded with the code object.  In host
// code `scratch` is a stand-in symbol, not a device address; the address each device's copy has comes
// from hipGetSymbolAddress (with that device current) and is kept per device.  Only that address is
// ever passed to a kernel or a fill.
static __device__ __align__(256) unsigned char scratch[NLD_NOALLOC_SCRATCH_BYTES];

namespace {

constexpr int MAX_DEVICES = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[MAX_DEVICES] = {};

// This device's scratch address; on the device's first call the whole array is zeroed (a fill kernel on
// `s`), which is the state nld_workspace_init gives a workspace.
nld_status scratch_of_current_device(hipStream_t s, void** out) {
    int dev = -1;
    HIP_TRY(hipGetDevice(&dev));
    if (dev < 0 || dev >= MAX_DEVICES) return fail(NLD_ERR_UNSUPPORTED, "device ordinal %d outside [0, %d)", dev, MAX_DEVICES);
    std::lock_guard<std::mutex> lock(g_scratch_mu);
    if (!g_scratch_ptr[dev]) {
        void* p = nullptr;
        HIP_TRY(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)));
        if (!p) return fail(NLD_ERR_HIP, "hipGetSymbolAddress gave no address for the scratch array");
        HIP_TRY(launch_fill_zero(p, NLD_NOALLOC_SCRATCH_BYTES, s));
        g_scratch_ptr[dev] = p;
    }
    *out = g_scratch_ptr[dev];
    return NLD_OK;
}

}  // namespace

extern "C" {

nld_status nld_verify_accept_noalloc(const nld_model* m, const nld_kv_cache* kv, const int32_t* anchor,
                                     const int32_t* draft, int32_t batch, int32_t k, int32_t* accept_len,
                                     int32_t* committed, int32_t* next_anchor, float* logits,
                                     uint32_t* device_status, void* stream) {
    // host checks first, with a non-null stand-in workspace of the maximal size: the layout of this call
    // must fit the scratch array before anything touches the device
    Layout L;
    nld_status st = validate_call(m, kv, batch, k, (void*)&g_scratch_mu, NLD_NOALLOC_SCRATCH_BYTES, &L);
    if (st == NLD_ERR_CAPACITY)
        return fail(NLD_ERR_CAPACITY, "this batch (%d), k (%d) and max_len (%d) need %zu bytes of scratch; the "
                    "allocation-free entry point holds at most %u", batch, k, kv->max_len, L.total,
                    (unsigned)NLD_NOALLOC_SCRATCH_BYTES);
    if (st != NLD_OK) return st;
    if (!anchor || !accept_len || !committed || !next_anchor)
        return fail(NLD_ERR_INVALID_ARG, "anchor, accept_len, committed or next_anchor is NULL");
    if (k > 1 && !draft) return fail(NLD_ERR_INVALID_ARG, "draft is NULL");
    hipStream_t s = (hipStream_t)stream;
    void* ws = nullptr;
    st = scratch_of_current_device(s, &ws);
    if (st != NLD_OK) return st;
    uint32_t* status = at<uint32_t>(ws, L.status);
    HIP_TRY(launch_fill_zero(status, 4, s));
    PassIO io{};
    io.source = SRC_VERIFY;
    io.anchor = anchor;
    io.draft_in = draft;
    io.mode = NLD_MODE_VERIFY;
    io.logits = logits;
    io.finish = FINISH_ACCEPT;
    io.accept_len = accept_len;
    io.committed = committed;
    io.next_anchor = next_anchor;
    io.advance_lengths = true;
    st = run_pass(m, kv, batch, k, io, ws, L, s);
    if (st != NLD_OK) return st;
    if (device_status) HIP_TRY(launch_copy_u32(status, device_status, s));
    return NLD_OK;
}

}  // extern "C"
