// Shared by the token cache's device sources: argument checks, rows, pages, blocks.
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

// ---------------------------------------------------------------------------------------------------- rows into blocks
template <typename T> __device__ inline T store_from_f32(float f);
template <> __device__ inline float store_from_f32<float>(float f) { return f; }
template <> __device__ inline uint16_t store_from_f32<uint16_t>(float f) { return f32_to_bf16(f); }

struct Rows {
    void *x[2];                  // k, v
    uint64_t token_stride[2], head_stride[2];
    const int32_t *start;
    uint32_t tokens;
    bool aligned;                // rows begin at multiples of 16 bytes
};

// Eq. 1's grid map with z = 128. x / scale is its correctly rounded quotient: by the reciprocal (itself correctly rounded), the remainder, which
// fma gives exactly, and one correction, where reciprocal and remainder are normal numbers, which they are for scales
// of 2^-100 and more; smaller ones and blocks with elements that are no numbers divide. Adding 1.5 * 2^23 + 128 rounds the
// quotient to the nearest even integer and leaves the code in the low byte.
struct Grid {
    float scale, inverse;
    bool divide;
};

__device__ inline Grid grid_of(float scale, bool numbers) {
    return {scale, 1.0f / scale, !numbers || scale < 7.9e-31f};
}

__device__ inline uint32_t code_by_division(float x, float scale) {
    float q = rintf(x / scale);
    q = q == q ? fminf(fmaxf(q, -127.0f), 127.0f) : 0.0f;   // NaN to the zero-point, infinities to the ends
    return scale > 0.0f ? static_cast<uint32_t>(static_cast<int32_t>(q) + 128) : 128u;
}

// The code stands in the low byte.
__device__ inline uint32_t code_by_inverse(float x, const Grid &g) {
    const float q = x * g.inverse;
    return __float_as_uint(fmaf(fmaf(-q, g.scale, x), g.inverse, q) + 12583040.0f);
}

__device__ inline uint32_t four_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}

__device__ inline uint32_t byte_of(uint32_t w, uint32_t i) { return (w >> (8 * i)) & 0xffu; }

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// A block of a sequence and a head: what LANES lanes write or read together. They take it in patches of 4 tokens x 8 dimensions,
// the smallest that is whole words of rows (16 bytes in bf16), of key codes (8 bytes of a token) and of value codes (4 bytes of a
// dimension). Neighbouring lanes have neighbouring dimensions of the keys, but neighbouring tokens of the values, as the codes lie.
struct Block {
    int64_t row;                 // of the block's token 0 (it may lie before the tensor)
    uint32_t t0, t1;             // tokens t0 .. t1 - 1 have rows
    int32_t entry, at;           // of the table, and the position it stands for: checked_page's
};

struct Patch {
    uint32_t t, d;               // its first token and dimension
};

// The `nth` of `patches` patches; kv: 0 keys, 1 values.
__device__ inline Patch patch_of(const Pool &p, uint32_t nth, int kv) {
    const uint32_t quads = 1u << (p.page_shift - 2), eights = (p.head_dim + 7) / 8;
    if (kv) return {4 * (nth & (quads - 1)), 8 * (nth >> (p.page_shift - 2))};
    return {4 * (nth / eights), 8 * (nth % eights)};
}

// The block with number w of `blocks` per sequence and kv_heads per block, then every `blocks`-th one after it; f is called with each.
template <typename F>
__device__ inline void each_block(const Pool &p, const Rows &r, uint32_t blocks, uint32_t w, F f) {
    const uint32_t head = w % p.kv_heads, nth = w / p.kv_heads % blocks, b = w / p.kv_heads / blocks;
    const Span s = span_of(r.start, p.lengths, b, r.tokens);
    if (s.count == 0) return;
    const int32_t first = max(s.pos, 0) >> p.page_shift, last = (s.length - 1) >> p.page_shift;
    for (int32_t block = first + static_cast<int32_t>(nth); block <= last; block += static_cast<int32_t>(blocks)) {
        const int32_t at = block << p.page_shift;
        Block x;
        x.entry = table_entry(p, b, at);
        x.at = at;
        x.row = int64_t{s.row} + at - s.pos;
        x.t0 = static_cast<uint32_t>(max(s.pos - at, 0));
        x.t1 = static_cast<uint32_t>(min(s.length - at, 1 << p.page_shift));
        f(x, head);
    }
}

// A patch's rows as they lie in memory: asked for all at once (rows that are not there: others in their place).
template <typename T>
struct RawPatch {
    u32x4 w[4][sizeof(T) / 2];
};

template <typename T>
__device__ inline RawPatch<T> ask_patch(const T *x, uint64_t token_stride, const Patch &a, const Block &b, uint32_t head_dim, bool aligned) {
    RawPatch<T> r;
    if (aligned && a.d + 8 <= head_dim) {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const u32x4 *row = reinterpret_cast<const u32x4 *>(x + min(max(a.t + j, b.t0), b.t1 - 1) * token_stride + a.d);
#pragma unroll
            for (uint32_t i = 0; i < sizeof(T) / 2; ++i) r.w[j][i] = row[i];
        }
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            const T *row = x + min(max(a.t + j, b.t0), b.t1 - 1) * token_stride;
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const T e = row[min(a.d + i, head_dim - 1)];
                if (sizeof(T) == 2) {
                    const uint32_t h = static_cast<uint32_t>(e) << (16 * (i & 1));
                    r.w[j][0][i / 2] = i & 1 ? r.w[j][0][i / 2] | h : h;
                } else {
                    r.w[j][(i / 4) % (sizeof(T) / 2)][i & 3] = __builtin_bit_cast(uint32_t, static_cast<float>(e));
                }
            }
        }
    }
    return r;
}

template <typename T>
__device__ inline void patch_values(const RawPatch<T> &r, const Patch &a, const Block &b, uint32_t head_dim, float (*v)[8]) {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const uint32_t w = sizeof(T) == 2 ? r.w[j][0][i / 2] : r.w[j][(i / 4) % (sizeof(T) / 2)][i & 3];
            const float x = __uint_as_float(sizeof(T) == 4 ? w : i & 1 ? w & 0xffff0000u : w << 16);
            v[j][i] = a.t + j >= b.t0 && a.t + j < b.t1 && a.d + i < head_dim ? x : 0.0f;
        }
}

// The bits of the largest |x| of a patch: of all elements, or of the finite ones.
__device__ inline uint32_t largest(const float (*v)[8], bool finite) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = __float_as_uint(v[j][i]) & 0x7fffffffu;
            m = max(m, !finite || bits < 0x7f800000u ? bits : 0u);
        }
    return m;
}

// A patch's codes: new tokens' from v, older ones moved to the new grid if the scale has grown, others left as they are.
__device__ inline void write_patch(const Pool &p, uint64_t unit, const Patch &a, const Block &b, const float (*v)[8], float old, const Grid &grid, int kv) {
    const bool moved = grid.scale > old && a.t < b.t0;
    if ((a.t + 4 <= b.t0 && !moved) || a.t >= b.t1) return;
    const uint32_t pt = 1u << p.page_shift, step = kv ? pt : p.width;
    uint8_t *at = kv ? p.v + (unit * p.width + a.d) * pt + a.t : p.k + (unit * pt + a.t) * p.width + a.d;
    if (a.t >= b.t0 && a.t + 4 <= b.t1 && a.d + 8 <= p.head_dim && !grid.divide) {
        uint32_t c[4][8];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) c[j][i] = code_by_inverse(v[j][i], grid);
        if (kv) {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) *reinterpret_cast<uint32_t *>(at + i * step) = four_codes(c[0][i], c[1][i], c[2][i], c[3][i]);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j)
                *reinterpret_cast<u32x2 *>(at + j * step) = u32x2{four_codes(c[j][0], c[j][1], c[j][2], c[j][3]), four_codes(c[j][4], c[j][5], c[j][6], c[j][7])};
        }
        return;
    }
    // code by code: nothing has to be read first but codes that move
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
        if (a.t + j >= b.t1 || (a.t + j < b.t0 && !moved)) continue;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            if (a.d + i >= p.head_dim) break;
            uint8_t *code = kv ? at + i * step + j : at + j * step + i;
            if (a.t + j >= b.t0)
                *code = static_cast<uint8_t>(grid.divide ? code_by_division(v[j][i], grid.scale) : code_by_inverse(v[j][i], grid));
            else
                *code = static_cast<uint8_t>(static_cast<int32_t>(rintf(static_cast<float>(static_cast<int32_t>(*code) - 128) * old / grid.scale)) + 128);
        }
    }
}

}  // namespace entro_detail

#endif
