// The token cache of libentro on the GPU: writing keys and values in 8 bits,
// reading them back, and moving pages (include/entro.h has the layouts).
//
// Eq. 1's grid map with one scale for each block of tokens and head.  A block is
// a page; new tokens may raise its scale, and then its older codes move to the
// new grid.  Everything here is bound by bytes or by launches; the page table's
// kernels work in integers only.
#include "entro_cache.h"

namespace {

using namespace entro_detail;

constexpr int kWG = 256;
constexpr int kScanWG = 1024;
constexpr int32_t kNoOwner = 0x7fffffff;      // owner[page]: no row holds it
constexpr int32_t kFullSomewhere = -1;        // owner[page]: to some row it is a full page

template <typename T> __device__ inline float load_as_f32(const T *p);
template <> __device__ inline float load_as_f32<float>(const float *p) { return *p; }
template <> __device__ inline float load_as_f32<uint16_t>(const uint16_t *p) { return bf16_to_f32(*p); }
template <typename T> __device__ inline T store_from_f32(float f);
template <> __device__ inline float store_from_f32<float>(float f) { return f; }
template <> __device__ inline uint16_t store_from_f32<uint16_t>(float f) { return f32_to_bf16(f); }

struct Rows {
    void *x[2];                  // k, v
    uint64_t token_stride[2], head_stride[2];
    const int32_t *start;
    uint32_t tokens;
};

// Eq. 1's grid map with z = 128: NaN to the zero-point, infinities to the ends.
__device__ inline uint32_t grid_code(float x, float scale) {
    if (!(scale > 0.0f)) return 128u;
    float q = rintf(x / scale);
    q = q == q ? fminf(fmaxf(q, -127.0f), 127.0f) : 0.0f;
    return static_cast<uint32_t>(static_cast<int32_t>(q) + 128);
}

// One workgroup per block that a sequence writes to, and head; k and v one after the other.
template <typename T>
__global__ __launch_bounds__(kWG) void k_append(Pool p, Rows r, uint32_t blocks_per_seq, uint32_t work) {
    __shared__ uint32_t most[kWG / 64];
    const uint32_t tid = threadIdx.x, pt = 1u << p.page_shift;
    for (uint32_t w = blockIdx.x; w < work; w += gridDim.x) {
        const uint32_t head = w % p.kv_heads, nth = w / p.kv_heads % blocks_per_seq, b = w / p.kv_heads / blocks_per_seq;
        const Span s = span_of(r.start, p.lengths, b, r.tokens);
        if (s.count == 0) continue;
        const int32_t first = max(s.pos, 0) >> p.page_shift, last = (s.length - 1) >> p.page_shift;
        for (int32_t block = first + static_cast<int32_t>(nth); block <= last; block += static_cast<int32_t>(blocks_per_seq)) {
            const int32_t page = page_of(p, b, block);
            if (page < 0) continue;
            const int32_t at = block << p.page_shift;
            const uint32_t t0 = static_cast<uint32_t>(max(s.pos - at, 0)), t1 = static_cast<uint32_t>(min(s.length - at, static_cast<int32_t>(pt)));
            for (int kv = 0; kv < 2; ++kv) {
                const uint64_t unit = uint64_t{static_cast<uint32_t>(page)} * p.kv_heads + head;
                uint8_t *codes = (kv ? p.v : p.k) + unit * pt * p.width;
                float *scale_at = (kv ? p.v_scale : p.k_scale) + unit;
                const T *x = static_cast<const T *>(r.x[kv]) + uint64_t(int64_t{s.row} + at - s.pos) * r.token_stride[kv] + head * r.head_stride[kv];
                const uint32_t n = (t1 - t0) * p.head_dim;
                uint32_t m = 0;
                for (uint32_t i = tid; i < n; i += kWG) {
                    const uint32_t t = t0 + i / p.head_dim, d = i % p.head_dim;
                    const uint32_t bits = __float_as_uint(load_as_f32(x + t * r.token_stride[kv] + d)) & 0x7fffffffu;
                    m = max(m, bits < 0x7f800000u ? bits : 0u);
                }
                for (int o = 32; o; o >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o)));
                if ((tid & 63u) == 0) most[tid >> 6] = m;
                const float old = t0 ? *scale_at : 0.0f;
                __syncthreads();
                for (int i = 0; i < kWG / 64; ++i) m = max(m, most[i]);
                const float scale = fmaxf(old, __uint_as_float(m) / 127.0f);
                if (scale > old) {
                    for (uint32_t i = tid; i < t0 * p.head_dim; i += kWG) {
                        const uint32_t t = i / p.head_dim, d = i % p.head_dim;
                        uint8_t *c = codes + (kv ? d * pt + t : t * p.width + d);
                        *c = static_cast<uint8_t>(static_cast<int32_t>(rintf(static_cast<float>(static_cast<int32_t>(*c) - 128) * old / scale)) + 128);
                    }
                }
                for (uint32_t i = tid; i < n; i += kWG) {
                    const uint32_t t = t0 + i / p.head_dim, d = i % p.head_dim;
                    codes[kv ? d * pt + t : t * p.width + d] = static_cast<uint8_t>(grid_code(load_as_f32(x + t * r.token_stride[kv] + d), scale));
                }
                if (tid == 0) *scale_at = scale;
                __syncthreads();                 // `most` is used again
            }
        }
    }
}

// A lane per row, head and dimension.
template <typename T>
__global__ __launch_bounds__(kWG) void k_read(Pool p, Rows r, uint64_t n) {
    for (uint64_t i = uint64_t{blockIdx.x} * kWG + threadIdx.x; i < n; i += uint64_t{gridDim.x} * kWG) {
        const uint32_t d = static_cast<uint32_t>(i % p.head_dim), head = static_cast<uint32_t>(i / p.head_dim % p.kv_heads);
        const int32_t row = static_cast<int32_t>(i / p.head_dim / p.kv_heads);
        uint32_t lo = 0, hi = p.seqs;            // the last sequence that starts at or before the row
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (r.start[mid] <= row) lo = mid; else hi = mid;
        }
        const Span s = span_of(r.start, p.lengths, lo, r.tokens);
        if (row < s.row || row >= s.row + s.count) continue;
        const int32_t pos = s.pos + row - s.row, page = pos < 0 ? -1 : page_of(p, lo, pos >> p.page_shift);
        const uint32_t pt = 1u << p.page_shift, t = static_cast<uint32_t>(pos) & (pt - 1);
        float k = 0.0f, v = 0.0f;
        if (page >= 0) {
            const uint64_t unit = uint64_t{static_cast<uint32_t>(page)} * p.kv_heads + head, at = unit * pt * p.width;
            k = static_cast<float>(static_cast<int32_t>(p.k[at + t * p.width + d]) - 128) * p.k_scale[unit];
            v = static_cast<float>(static_cast<int32_t>(p.v[at + d * pt + t]) - 128) * p.v_scale[unit];
        }
        static_cast<T *>(r.x[0])[static_cast<uint32_t>(row) * r.token_stride[0] + head * r.head_stride[0] + d] = store_from_f32<T>(k);
        static_cast<T *>(r.x[1])[static_cast<uint32_t>(row) * r.token_stride[1] + head * r.head_stride[1] + d] = store_from_f32<T>(v);
    }
}

// ------------------------------------------------------------------------------------------------------------- pages

struct PageWork {                // in the caller's workspace
    int32_t *owner;              // [pages]
    int32_t *free;               // [pages] free pages, lowest first
    int32_t *src, *dst;          // [max(pages, seqs)] pages to copy
    int32_t *first;              // [seqs] what a row takes of `free` begins here
    int32_t *counts;             // [0] pages to copy
};

uint64_t pages_workspace(const entro_cache *c, const entro_cache_table *next, PageWork *w, void *at) {
    const uint64_t pages = (uint64_t{c->pages} + 3) & ~3ull, seqs = (uint64_t{next->seqs} + 3) & ~3ull, most = pages > seqs ? pages : seqs;
    int32_t *p = static_cast<int32_t *>(at);
    if (w) {
        w->counts = p;
        w->owner = p + 16;
        w->free = w->owner + pages;
        w->src = w->free + pages;
        w->dst = w->src + most;
        w->first = w->dst + most;
    }
    return 4 * (16 + 2 * pages + 2 * most + seqs);
}

__global__ __launch_bounds__(kWG) void k_page_fill(int32_t *p, uint32_t n, int32_t value) {
    for (uint32_t i = blockIdx.x * kWG + threadIdx.x; i < n; i += gridDim.x * kWG) p[i] = value;
}

struct Regroup {
    entro_cache_table from, to;
    const int32_t *parent, *grow;
    uint32_t pages, page_shift, window, sinks;
};

struct Row {
    int32_t parent, kept, length;       // parent < 0: an empty row
};

__device__ inline Row regroup_row(const Regroup &g, uint32_t b) {
    Row r;
    r.parent = g.parent ? g.parent[b] : static_cast<int32_t>(b);
    if (static_cast<uint32_t>(r.parent) >= g.from.seqs) {
        r.parent = -1;
        r.kept = r.length = 0;
        return r;
    }
    const int64_t old = max(g.from.lengths[r.parent], 0), then = old + (g.grow ? g.grow[b] : 0);
    r.length = static_cast<int32_t>(min(max(then, int64_t{0}), int64_t{0x7fffff00}));
    r.kept = static_cast<int32_t>(min(old, static_cast<int64_t>(r.length)));
    return r;
}

__device__ inline int32_t slots_of(int32_t tokens, uint32_t shift) {
    return static_cast<int32_t>((static_cast<uint32_t>(tokens) + (1u << shift) - 1) >> shift);
}

// Whether slot s is partly filled after `kept` tokens: the row will write to it.
__device__ inline bool open_at(int32_t kept, uint32_t s, uint32_t shift) {
    return (static_cast<uint32_t>(kept) & ((1u << shift) - 1)) && s == static_cast<uint32_t>(kept) >> shift;
}

// What every row of the next table keeps of its parent's pages, and who owns a page: the lowest row to which it is open, or
// nobody if to some row it is full.
__global__ __launch_bounds__(kWG) void k_regroup_rows(Regroup g, int32_t *owner) {
    const uint32_t b = blockIdx.y;
    const Row r = regroup_row(g, b);
    const uint32_t pt = 1u << g.page_shift;
    const int32_t keep = slots_of(r.kept, g.page_shift);
    if (blockIdx.x == 0 && threadIdx.x == 0) g.to.lengths[b] = r.length;
    for (uint32_t s = blockIdx.x * kWG + threadIdx.x; s < g.to.stride; s += gridDim.x * kWG) {
        int32_t id = -1;
        if (static_cast<int32_t>(s) < keep && s < g.from.stride) {
            id = g.from.slots[uint64_t{static_cast<uint32_t>(r.parent)} * g.from.stride + s];
            const uint64_t at = uint64_t{s} << g.page_shift;
            if (static_cast<uint32_t>(id) >= g.pages ||
                (g.window && at + pt + g.window <= static_cast<uint64_t>(r.kept) + 1 && at >= g.sinks))
                id = -1;
        }
        g.to.slots[uint64_t{b} * g.to.stride + s] = id;
        if (id >= 0) {
            const bool open = open_at(r.kept, s, g.page_shift);
            atomicMin(owner + id, open ? static_cast<int32_t>(b) : kFullSomewhere);
        }
    }
}

// Sum of v over the workgroup's threads before this one; `total` the sum over all.
__device__ inline uint32_t scan_before(uint32_t v, uint32_t *total) {
    __shared__ uint32_t sums[kScanWG / 64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    uint32_t incl = v;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = static_cast<uint32_t>(__shfl_up(static_cast<int>(incl), o));
        if (lane >= static_cast<uint32_t>(o)) incl += up;
    }
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int i = 0; i < kScanWG / 64; ++i) {
        before += i < static_cast<int>(wave) ? sums[i] : 0u;
        all += sums[i];
    }
    __syncthreads();
    *total = all;
    return before + incl - v;
}

// One workgroup: which rows copy their open page, where every row's new pages begin among the free ones, and the free ones.
__global__ __launch_bounds__(kScanWG) void k_regroup_plan(Regroup g, PageWork w, int32_t *status) {
    uint32_t need_all = 0, copies_all = 0, total;
    bool too_long = false;
    for (uint32_t b0 = 0; b0 < g.to.seqs; b0 += kScanWG) {
        const uint32_t b = b0 + threadIdx.x;
        uint32_t copy = 0, need = 0;
        int32_t open_page = -1;
        if (b < g.to.seqs) {
            const Row r = regroup_row(g, b);
            const int32_t keep = slots_of(r.kept, g.page_shift), want = slots_of(r.length, g.page_shift);
            too_long |= want > static_cast<int32_t>(g.to.stride);
            const uint32_t s = static_cast<uint32_t>(r.kept) >> g.page_shift;
            if (s < g.to.stride && open_at(r.kept, s, g.page_shift)) open_page = g.to.slots[uint64_t{b} * g.to.stride + s];
            copy = open_page >= 0 && w.owner[open_page] != static_cast<int32_t>(b);
            need = copy + static_cast<uint32_t>(want - keep);
        }
        const uint32_t at = need_all + scan_before(need, &total);
        need_all = min(need_all + total, 0x7fffffffu);
        const uint32_t nth = copies_all + scan_before(copy, &total);
        copies_all += total;
        if (b < g.to.seqs) w.first[b] = static_cast<int32_t>(at);
        if (copy) {
            w.src[nth] = open_page;
            w.dst[nth] = static_cast<int32_t>(at);          // its place among the free pages, until those are known
        }
    }
    too_long = __syncthreads_or(too_long);
    uint32_t free_all = 0;
    for (uint32_t p0 = 0; p0 < g.pages; p0 += kScanWG) {
        const uint32_t p = p0 + threadIdx.x;
        const uint32_t is_free = p < g.pages && w.owner[p] == kNoOwner;
        const uint32_t at = free_all + scan_before(is_free, &total);
        free_all += total;
        if (is_free) w.free[at] = static_cast<int32_t>(p);
    }
    const bool fits = !too_long && need_all <= free_all;
    __threadfence_block();
    __syncthreads();
    if (fits)
        for (uint32_t i = threadIdx.x; i < copies_all; i += kScanWG) w.dst[i] = w.free[w.dst[i]];
    if (threadIdx.x == 0) {
        w.counts[0] = fits ? static_cast<int32_t>(copies_all) : 0;
        status[0] = fits ? 0 : 1;
        status[1] = static_cast<int32_t>(g.pages - free_all + (fits ? need_all : 0u));
        status[2] = static_cast<int32_t>(free_all - (fits ? need_all : 0u));
        status[3] = w.counts[0];
    }
}

// The new pages into the rows.
__global__ __launch_bounds__(kWG) void k_regroup_fill(Regroup g, PageWork w, const int32_t *status) {
    if (status[0]) return;
    const uint32_t b = blockIdx.x;
    const Row r = regroup_row(g, b);
    const int32_t keep = slots_of(r.kept, g.page_shift), want = slots_of(r.length, g.page_shift);
    int32_t *row = g.to.slots + uint64_t{b} * g.to.stride;
    const int32_t *fresh = w.free + w.first[b];
    const uint32_t s = static_cast<uint32_t>(r.kept) >> g.page_shift;
    uint32_t copy = 0;
    if (s < g.to.stride && open_at(r.kept, s, g.page_shift)) {
        const int32_t id = row[s];
        copy = id >= 0 && w.owner[id] != static_cast<int32_t>(b);
        __syncthreads();
        if (copy && threadIdx.x == 0) row[s] = fresh[0];
    }
    for (int32_t i = keep + static_cast<int32_t>(threadIdx.x); i < want; i += kWG) row[i] = fresh[copy + static_cast<uint32_t>(i - keep)];
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Copies {
    uint8_t *codes[2];
    float *scale[2];
    uint64_t page_bytes, layer_bytes;        // of codes
    uint32_t heads, layers, pages;
};

// Pages src[i] -> dst[i], i < counts[0], in all layers. A work item is a page of k or v of a layer.
__global__ __launch_bounds__(kWG) void k_copy_pages(Copies c, const int32_t *src, const int32_t *dst, const int32_t *counts) {
    const uint64_t items = uint64_t{static_cast<uint32_t>(counts[0])} * c.layers * 2;
    const uint32_t vecs = static_cast<uint32_t>(c.page_bytes / 16);
    for (uint64_t w = blockIdx.x; w < items; w += gridDim.x) {
        const uint32_t kv = static_cast<uint32_t>(w & 1), layer = static_cast<uint32_t>((w >> 1) % c.layers), i = static_cast<uint32_t>((w >> 1) / c.layers);
        const uint64_t from = static_cast<uint32_t>(src[i]), to = static_cast<uint32_t>(dst[i]);
        const u32x4 *a = reinterpret_cast<const u32x4 *>(c.codes[kv] + layer * c.layer_bytes + from * c.page_bytes);
        u32x4 *z = reinterpret_cast<u32x4 *>(c.codes[kv] + layer * c.layer_bytes + to * c.page_bytes);
        for (uint32_t j = threadIdx.x; j < vecs; j += kWG) z[j] = a[j];
        float *scale = c.scale[kv] + uint64_t{layer} * c.pages * c.heads;
        for (uint32_t j = threadIdx.x; j < c.heads; j += kWG) scale[to * c.heads + j] = scale[from * c.heads + j];
    }
}

__global__ __launch_bounds__(kWG) void k_compact_mark(entro_cache_table t, uint32_t pages, int32_t *owner) {
    const uint32_t b = blockIdx.y;
    for (uint32_t s = blockIdx.x * kWG + threadIdx.x; s < t.stride; s += gridDim.x * kWG) {
        const int32_t id = t.slots[uint64_t{b} * t.stride + s];
        if (static_cast<uint32_t>(id) < pages) owner[id] = 0;
    }
}

// One workgroup: how many pages are in use, which of them move and where to. owner[p] becomes the new number of page p.
__global__ __launch_bounds__(kScanWG) void k_compact_plan(uint32_t pages, PageWork w, int32_t *status) {
    uint32_t used = 0, total;
    for (uint32_t p0 = 0; p0 < pages; p0 += kScanWG) {
        const uint32_t p = p0 + threadIdx.x;
        scan_before(p < pages && w.owner[p] != kNoOwner, &total);
        used += total;
    }
    uint32_t holes = 0, moves = 0;
    for (uint32_t p0 = 0; p0 < pages; p0 += kScanWG) {
        const uint32_t p = p0 + threadIdx.x;
        const bool held = p < pages && w.owner[p] != kNoOwner;
        const bool hole = p < used && !held, move = p >= used && held;
        const uint32_t h = holes + scan_before(hole, &total);
        holes += total;
        const uint32_t m = moves + scan_before(move, &total);
        moves += total;
        if (hole) w.dst[h] = static_cast<int32_t>(p);
        if (move) w.src[m] = static_cast<int32_t>(p);
        if (held && !move) w.owner[p] = static_cast<int32_t>(p);
    }
    __threadfence_block();
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < moves; i += kScanWG) w.owner[w.src[i]] = w.dst[i];
    if (threadIdx.x == 0) {
        w.counts[0] = static_cast<int32_t>(moves);
        status[0] = 0;
        status[1] = static_cast<int32_t>(used);
        status[2] = static_cast<int32_t>(pages - used);
        status[3] = static_cast<int32_t>(moves);
    }
}

__global__ __launch_bounds__(kWG) void k_compact_rows(entro_cache_table t, entro_cache_table next, uint32_t pages, const int32_t *owner) {
    const uint32_t b = blockIdx.y;
    if (blockIdx.x == 0 && threadIdx.x == 0) next.lengths[b] = t.lengths[b];
    for (uint32_t s = blockIdx.x * kWG + threadIdx.x; s < t.stride; s += gridDim.x * kWG) {
        const uint64_t i = uint64_t{b} * t.stride + s;
        const int32_t id = t.slots[i];
        next.slots[i] = static_cast<uint32_t>(id) < pages ? owner[id] : -1;
    }
}

entro_status check_rows(const entro_cache *c, const entro_cache_rows *r) {
    if (!r || !r->start || (r->tokens && (!r->k || !r->v))) return ENTRO_ERR_NULL;
    if (r->type != ENTRO_F32 && r->type != ENTRO_BF16) return ENTRO_ERR_SCHEME;
    if (r->layer >= c->layers || r->tokens > 0x7fffffffu) return ENTRO_ERR_SIZE;
    if (r->k_token_stride > kMaxStride || r->k_head_stride > kMaxStride || r->v_token_stride > kMaxStride || r->v_head_stride > kMaxStride)
        return ENTRO_ERR_SIZE;
    if (!aligned16(r->k) || !aligned16(r->v) || !aligned16(r->start)) return ENTRO_ERR_ALIGN;
    return ENTRO_OK;
}

Rows rows_of(const entro_cache_rows *r) {
    return {{r->k, r->v}, {r->k_token_stride, r->v_token_stride}, {r->k_head_stride, r->v_head_stride}, r->start, r->tokens};
}

Copies copies_of(const entro_cache *c) {
    Copies x;
    x.codes[0] = static_cast<uint8_t *>(c->k);
    x.codes[1] = static_cast<uint8_t *>(c->v);
    x.scale[0] = c->k_scale;
    x.scale[1] = c->v_scale;
    x.page_bytes = uint64_t{c->kv_heads} * c->page_tokens * entro_cache_width(c->head_dim);
    x.layer_bytes = x.page_bytes * c->pages;
    x.heads = c->kv_heads;
    x.layers = c->layers;
    x.pages = c->pages;
    return x;
}

entro_status check_pages(const entro_cache *c, const entro_cache_table *t, const entro_cache_table *next, const int32_t *status,
                         const void *workspace, uint64_t workspace_bytes) {
    if (const entro_status s = check_cache(c)) return s;
    if (const entro_status s = check_table(t)) return s;
    if (const entro_status s = check_table(next)) return s;
    if (!status || !workspace) return ENTRO_ERR_NULL;
    if (!aligned16(status) || !aligned16(workspace)) return ENTRO_ERR_ALIGN;
    // in place, a row could be read after it was written
    if (next->slots == t->slots || next->lengths == t->lengths || next->seqs > 65535 || t->seqs > 65535) return ENTRO_ERR_SIZE;
    if (workspace_bytes < entro_cache_pages_workspace_bytes(c, t, next)) return ENTRO_ERR_CAPACITY;
    return ENTRO_OK;
}

dim3 rows_grid(uint32_t stride, uint32_t seqs) {
    const uint32_t x = (stride + kWG - 1) / kWG;
    return dim3(x < 64 ? x : 64, seqs);
}

unsigned copy_grid(uint64_t most, uint32_t layers) {
    const uint64_t items = most * layers * 2;
    return static_cast<unsigned>(items < 4096 ? items : 4096);
}

}  // namespace

extern "C" {

uint32_t entro_cache_width(uint32_t head_dim) {
    if (head_dim == 0 || head_dim > ENTRO_CACHE_MAX_DIM) return 0;
    for (const uint32_t w : {64u, 96u, 128u, 192u})
        if (head_dim <= w) return w;
    return 256;
}

uint64_t entro_cache_codes_bytes(const entro_cache *c) {
    if (check_sizes(c) != ENTRO_OK) return 0;
    return uint64_t{c->layers} * c->pages * c->kv_heads * c->page_tokens * entro_cache_width(c->head_dim);
}

entro_status entro_cache_append(const entro_cache *c, const entro_cache_table *t, const entro_cache_rows *r, void *hip_stream) {
    if (const entro_status s = check_cache(c)) return s;
    if (const entro_status s = check_table(t)) return s;
    if (const entro_status s = check_rows(c, r)) return s;
    if (r->tokens == 0 || r->max_new == 0) return ENTRO_OK;
    const Pool p = pool_of(c, t, r->layer);
    // as many blocks as the most rows can touch, and no more than there are slots
    const uint64_t touch = (uint64_t{r->max_new} + c->page_tokens - 2) / c->page_tokens + 1;
    const uint32_t blocks = static_cast<uint32_t>(touch < t->stride ? touch : t->stride);
    const uint64_t work = uint64_t{blocks} * c->kv_heads * t->seqs;
    if (work > 0xffffffffull) return ENTRO_ERR_SIZE;
    const unsigned grid = static_cast<unsigned>(work < 65536 ? work : 65536);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (r->type == ENTRO_F32)
        hipLaunchKernelGGL(k_append<float>, dim3(grid), dim3(kWG), 0, st, p, rows_of(r), blocks, static_cast<uint32_t>(work));
    else
        hipLaunchKernelGGL(k_append<uint16_t>, dim3(grid), dim3(kWG), 0, st, p, rows_of(r), blocks, static_cast<uint32_t>(work));
    return hip_ok(hipGetLastError(), "entro_cache_append") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

entro_status entro_cache_read(const entro_cache *c, const entro_cache_table *t, const entro_cache_rows *r, void *hip_stream) {
    if (const entro_status s = check_cache(c)) return s;
    if (const entro_status s = check_table(t)) return s;
    if (const entro_status s = check_rows(c, r)) return s;
    if (r->tokens == 0) return ENTRO_OK;
    const Pool p = pool_of(c, t, r->layer);
    const uint64_t n = uint64_t{r->tokens} * c->kv_heads * c->head_dim, wgs = (n + kWG - 1) / kWG;
    const unsigned grid = static_cast<unsigned>(wgs < 16384 ? wgs : 16384);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (r->type == ENTRO_F32)
        hipLaunchKernelGGL(k_read<float>, dim3(grid), dim3(kWG), 0, st, p, rows_of(r), n);
    else
        hipLaunchKernelGGL(k_read<uint16_t>, dim3(grid), dim3(kWG), 0, st, p, rows_of(r), n);
    return hip_ok(hipGetLastError(), "entro_cache_read") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

uint64_t entro_cache_pages_workspace_bytes(const entro_cache *c, const entro_cache_table *t, const entro_cache_table *next) {
    if (check_sizes(c) != ENTRO_OK || check_table_sizes(t) != ENTRO_OK || check_table_sizes(next) != ENTRO_OK) return 0;
    return pages_workspace(c, next, nullptr, nullptr);
}

entro_status entro_cache_regroup(const entro_cache *c, const entro_cache_table *t, const int32_t *parent, const int32_t *grow,
                                 uint32_t window, uint32_t sinks, const entro_cache_table *next, int32_t *status, void *workspace,
                                 uint64_t workspace_bytes, void *hip_stream) {
    if (const entro_status s = check_pages(c, t, next, status, workspace, workspace_bytes)) return s;
    if (!aligned16(parent) || !aligned16(grow)) return ENTRO_ERR_ALIGN;
    PageWork w;
    pages_workspace(c, next, &w, workspace);
    const Regroup g = {*t, *next, parent, grow, c->pages, static_cast<uint32_t>(__builtin_ctz(c->page_tokens)), window, sinks};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const unsigned fill = c->pages < 1024 * kWG ? (c->pages + kWG - 1) / kWG : 1024;
    hipLaunchKernelGGL(k_page_fill, dim3(fill), dim3(kWG), 0, st, w.owner, c->pages, kNoOwner);
    hipLaunchKernelGGL(k_regroup_rows, rows_grid(next->stride, next->seqs), dim3(kWG), 0, st, g, w.owner);
    hipLaunchKernelGGL(k_regroup_plan, dim3(1), dim3(kScanWG), 0, st, g, w, status);
    hipLaunchKernelGGL(k_regroup_fill, dim3(next->seqs), dim3(kWG), 0, st, g, w, static_cast<const int32_t *>(status));
    hipLaunchKernelGGL(k_copy_pages, dim3(copy_grid(next->seqs, c->layers)), dim3(kWG), 0, st, copies_of(c), static_cast<const int32_t *>(w.src),
                       static_cast<const int32_t *>(w.dst), static_cast<const int32_t *>(w.counts));
    return hip_ok(hipGetLastError(), "entro_cache_regroup") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

entro_status entro_cache_compact(const entro_cache *c, const entro_cache_table *t, const entro_cache_table *next, int32_t *status,
                                 void *workspace, uint64_t workspace_bytes, void *hip_stream) {
    if (const entro_status s = check_pages(c, t, next, status, workspace, workspace_bytes)) return s;
    if (next->seqs != t->seqs || next->stride != t->stride) return ENTRO_ERR_SIZE;
    PageWork w;
    pages_workspace(c, next, &w, workspace);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const unsigned fill = c->pages < 1024 * kWG ? (c->pages + kWG - 1) / kWG : 1024;
    hipLaunchKernelGGL(k_page_fill, dim3(fill), dim3(kWG), 0, st, w.owner, c->pages, kNoOwner);
    hipLaunchKernelGGL(k_compact_mark, rows_grid(t->stride, t->seqs), dim3(kWG), 0, st, *t, c->pages, w.owner);
    hipLaunchKernelGGL(k_compact_plan, dim3(1), dim3(kScanWG), 0, st, c->pages, w, status);
    hipLaunchKernelGGL(k_compact_rows, rows_grid(t->stride, t->seqs), dim3(kWG), 0, st, *t, *next, c->pages, static_cast<const int32_t *>(w.owner));
    hipLaunchKernelGGL(k_copy_pages, dim3(copy_grid(c->pages / 2 + 1, c->layers)), dim3(kWG), 0, st, copies_of(c),
                       static_cast<const int32_t *>(w.src), static_cast<const int32_t *>(w.dst), static_cast<const int32_t *>(w.counts));
    return hip_ok(hipGetLastError(), "entro_cache_compact") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

entro_status entro_cache_status(int32_t status_word) { return status_word ? ENTRO_ERR_CAPACITY : ENTRO_OK; }

}  // extern "C"
