// Shared by the token cache's two device sources: argument checks, rows, pages.
#ifndef ENTRO_CACHE_INTERNAL_H
#define ENTRO_CACHE_INTERNAL_H

#include "entro.h"

#include <hip/hip_runtime.h>

// defined beside entro_last_device_error
void entro_detail_note_hip_error(const char *what, int hip_error);

namespace entro_detail {

inline bool hip_ok(hipError_t e, const char *what) {
    if (e == hipSuccess) return true;
    entro_detail_note_hip_error(what, static_cast<int>(e));
    return false;
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr uint64_t kMaxStride = 1ull << 40;   // of rows, in elements: products with row numbers stay within 64 bits

// The pool's sizes alone.
inline entro_status check_sizes(const entro_cache *c) {
    if (!c) return ENTRO_ERR_NULL;
    if (entro_cache_width(c->head_dim) == 0) return ENTRO_ERR_SIZE;
    if (c->page_tokens < 16 || c->page_tokens > 256 || (c->page_tokens & (c->page_tokens - 1))) return ENTRO_ERR_SIZE;
    if (c->layers == 0 || c->layers > 65536 || c->pages == 0 || c->pages > 0x7fffffffu || c->kv_heads == 0 || c->kv_heads > 65536)
        return ENTRO_ERR_SIZE;
    // layers * pages < 2^47, kv_heads <= 2^16: an odd pool could overflow
    const double bytes = double(c->layers) * c->pages * c->kv_heads * c->page_tokens * entro_cache_width(c->head_dim);
    return bytes < 9.0e15 ? ENTRO_OK : ENTRO_ERR_SIZE;
}

inline entro_status check_cache(const entro_cache *c) {
    if (const entro_status s = check_sizes(c)) return s;
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return ENTRO_ERR_NULL;
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_scale) || !aligned16(c->v_scale)) return ENTRO_ERR_ALIGN;
    return ENTRO_OK;
}

inline entro_status check_table_sizes(const entro_cache_table *t) {
    if (!t) return ENTRO_ERR_NULL;
    if (t->seqs == 0 || t->stride == 0 || uint64_t{t->seqs} * t->stride > 0x7fffffffull) return ENTRO_ERR_SIZE;
    return ENTRO_OK;
}

inline entro_status check_table(const entro_cache_table *t) {
    if (const entro_status s = check_table_sizes(t)) return s;
    if (!t->slots || !t->lengths) return ENTRO_ERR_NULL;
    if (!aligned16(t->slots) || !aligned16(t->lengths)) return ENTRO_ERR_ALIGN;
    return ENTRO_OK;
}

// What the kernels need of pool and table, for one layer.
struct Pool {
    uint8_t *k, *v;            // of the layer
    float *k_scale, *v_scale;
    const int32_t *slots, *lengths;
    uint32_t pages, page_shift, kv_heads, head_dim, width, seqs, stride;
};

inline Pool pool_of(const entro_cache *c, const entro_cache_table *t, uint32_t layer) {
    Pool p;
    p.width = entro_cache_width(c->head_dim);
    const uint64_t codes = uint64_t{c->pages} * c->kv_heads * c->page_tokens * p.width * layer;
    const uint64_t scales = uint64_t{c->pages} * c->kv_heads * layer;
    p.k = static_cast<uint8_t *>(c->k) + codes;
    p.v = static_cast<uint8_t *>(c->v) + codes;
    p.k_scale = c->k_scale + scales;
    p.v_scale = c->v_scale + scales;
    p.slots = t->slots;
    p.lengths = t->lengths;
    p.pages = c->pages;
    p.page_shift = static_cast<uint32_t>(__builtin_ctz(c->page_tokens));
    p.kv_heads = c->kv_heads;
    p.head_dim = c->head_dim;
    p.seqs = t->seqs;
    p.stride = t->stride;
    return p;
}

// The rows of one sequence: row, row + 1, .. row + count - 1 stand at positions pos, pos + 1, ..
struct Span {
    int32_t row, count, pos, length;
};

// `start` is the caller's device memory: what it says is kept inside the row tensor.
__device__ inline Span span_of(const int32_t *start, const int32_t *lengths, uint32_t b, uint32_t tokens) {
    Span s;
    const int32_t most = static_cast<int32_t>(tokens);
    s.row = min(max(start[b], 0), most);
    s.count = min(max(start[b + 1], s.row), most) - s.row;
    s.length = max(lengths[b], 0);
    s.pos = s.length - s.count;
    return s;
}

// A position's entry in the table, asked for without waiting for it; what it is worth is looked at where it is used. (A position past the
// table's slots takes the last one's.)
__device__ inline int32_t table_entry(const Pool &p, uint32_t b, int32_t at) {
    return p.slots[uint64_t{b} * p.stride + min(static_cast<uint32_t>(at) >> p.page_shift, p.stride - 1)];
}

__device__ inline int32_t checked_page(const Pool &p, int32_t id, int32_t at) {
    const bool there = (static_cast<uint32_t>(id) < p.pages) & (static_cast<uint32_t>(at) >> p.page_shift < p.stride);
    return there ? id : -1;
}

__device__ inline float bf16_to_f32(uint16_t b) { return __uint_as_float(uint32_t{b} << 16); }

// round to nearest even; a NaN stays one
__device__ inline uint16_t f32_to_bf16(float f) {
    const uint32_t u = __float_as_uint(f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return static_cast<uint16_t>((u >> 16) | 0x40u);
    return static_cast<uint16_t>((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

}  // namespace entro_detail

#endif
