// Attention over the 8-bit token cache on the GPU (include/entro.h has the layouts and the definition).
#include "entro_cache.h"

namespace {

using namespace entro_detail;

constexpr int kWG = 256;                       // four wavefronts

struct Query {
    const void *q;
    void *out;
    float *lse;
    uint64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    const int32_t *start;
    uint32_t tokens, q_heads, group, window, sinks;
    float scale;
    bool aligned;                  // rows of q begin at multiples of 16 bytes
    uint32_t splits, least;        // a group of rows takes at most `splits` workgroups, of at least `least` tiles each
    float *part_o, *part_lse;      // [row][q_heads][splits][W], [row][q_heads][splits]: joined afterwards where splits > 1
};

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr uint32_t kMostSplits = kWG;          // the join has a lane for each
constexpr uint32_t kManyRows = 128;            // of a workgroup for many rows
constexpr uint64_t kMostGroups = (1u << 24) - 1;   // workgroups of a launch: it has less than 2^32 lanes along x
constexpr int kTile = 64;                      // tokens a wavefront takes at a time
// A row's maximum may have risen by 2^kRise before its sums are brought to a new unit; that unit is 2^kRise times the last maximum, so that no
// weight is above 1 and sums stay as far from the largest number as those of the definition.
constexpr float kRise = 8.0f, kUnit = 256.0f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The upper halves of two fp32 numbers: cut off to bf16.
__device__ inline uint32_t upper_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }

// Eight codes c as bf16 numbers c - 128, exactly.
__device__ inline bf16x8 eight_values(uint32_t a, uint32_t b) {
    const uint32_t s[2] = {a ^ 0x80808080u, b ^ 0x80808080u};
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float f0 = static_cast<float>(static_cast<int8_t>(s[i])), f1 = static_cast<float>(static_cast<int8_t>(s[i] >> 8));
        const float f2 = static_cast<float>(static_cast<int8_t>(s[i] >> 16)), f3 = static_cast<float>(static_cast<int8_t>(s[i] >> 24));
        r[2 * i] = upper_halves(f0, f1);
        r[2 * i + 1] = upper_halves(f2, f3);
    }
    return __builtin_bit_cast(bf16x8, r);
}

// Eight factors of a product as sums of N bf16 numbers: 8, 16 or 24 bits of each, at any size. (A half holds 11 bits in one piece, but
// loses what is 2^-40 of the largest factor; where the larger ones meet codes of 0 that is the result.)
template <int N>
__device__ inline void split_factors(const float *x, bf16x8 *w) {
    u32x4 r[N];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
        for (int n = 0; n < N - 1; ++n) {
            r[n][i] = upper_halves(a, b);
            a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
            b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
        }
        r[N - 1][i] = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
    }
#pragma unroll
    for (int n = 0; n < N; ++n) w[n] = __builtin_bit_cast(bf16x8, r[n]);
}

// Maximum over the four lanes that hold a column (lanes c, c + 16, c + 32, c + 48).
__device__ inline float column_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

__device__ inline float column_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// The tiles of kTile tokens that rows at positions first..last see: those of the first tokens, then those of the window.
struct Tiles {
    int32_t sinks, from, count;
    __device__ int32_t at(int32_t i) const { return i < sinks ? i : from + i - sinks; }
    // how many of them lie before `tile`
    __device__ int32_t before(int32_t tile) const { return min(sinks, tile) + min(max(tile - from, 0), count - sinks); }
};

__device__ inline Tiles tiles_of(const Pool &p, const Query &a, int32_t first, int32_t last) {
    const int64_t end = min(int64_t{last} + 1, int64_t{p.stride} << p.page_shift);
    Tiles t = {0, 0, 0};
    if (end <= 0) return t;
    const int32_t until = static_cast<int32_t>((end + kTile - 1) / kTile);
    if (a.window) {
        const int64_t lo = int64_t{first} - a.window + 1;
        t.from = lo > 0 ? static_cast<int32_t>(min(lo / kTile, int64_t{until})) : 0;
        t.sinks = static_cast<int32_t>(min((int64_t{a.sinks} + kTile - 1) / kTile, int64_t{t.from}));
    }
    t.count = t.sinks + until - t.from;
    return t;
}

// How the tiles of a group of rows are shared out to at most `splits` workgroups, of at least `least` each.
__device__ inline int32_t tiles_per_split(uint32_t splits, uint32_t least, int32_t count) {
    return max((count + static_cast<int32_t>(splits) - 1) / static_cast<int32_t>(splits), static_cast<int32_t>(least));
}

__device__ inline int32_t tiles_per_split(const Query &a, int32_t count) { return tiles_per_split(a.splits, a.least, count); }

// Which of the tokens that its rows see a workgroup takes: all of a sequence's, those that a group of sequences shares, or those
// behind them.
enum { kWhole, kShared, kOwn };

// The work of a workgroup.  kWhole: s, table, head, split and the query's splits.
struct Part {
    Span s;                        // its rows; kShared: those of all sequences of a group, pos and length - 1 the least and the largest position
    uint32_t table;                // the table's row that names the pages
    uint32_t head, split;
    uint32_t splits, least;        // as a Query's, of this kind of tokens
    uint32_t parts, slot;          // parts of a row in the workspace, and the place of this kind's first one
    int32_t tiles;                 // that the group shares
    uint32_t first, last;          // sequences of the group
};

template <int MODE>
__device__ inline uint64_t part_at(const Query &a, const Part &w, uint64_t row_and_head) {
    return MODE == kWhole ? row_and_head * a.splits + w.split : row_and_head * w.parts + w.slot + w.split;
}

// The position of one of a group's rows.
__device__ inline int32_t position_of(const Pool &p, const Query &a, const Part &w, uint32_t token) {
    uint32_t lo = w.first, hi = w.last;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (a.start[mid] <= static_cast<int32_t>(token)) lo = mid;
        else hi = mid;
    }
    const Span s = span_of(a.start, p.lengths, lo, a.tokens);
    return s.pos + static_cast<int32_t>(token) - s.row;
}

template <typename T> __device__ inline float load_as_f32(const T *p);
template <> __device__ inline float load_as_f32<float>(const float *p) { return *p; }
template <> __device__ inline float load_as_f32<uint16_t>(const uint16_t *p) { return bf16_to_f32(*p); }
template <typename T> __device__ inline void store_as(T *p, float f);
template <> __device__ inline void store_as<float>(float *p, float f) { *p = f; }
template <> __device__ inline void store_as<uint16_t>(uint16_t *p, float f) { *p = f32_to_bf16(f); }

// Eight elements of a row from dimension d on, zeros from head_dim on.
template <typename T>
__device__ inline void load_eight(const T *row, uint32_t d, uint32_t head_dim, bool aligned, float *x) {
    if (aligned && d + 8 <= head_dim) {
        if (sizeof(T) == 2) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(row + d);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            const f32x4 w0 = *reinterpret_cast<const f32x4 *>(row + d), w1 = *reinterpret_cast<const f32x4 *>(row + d + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = w0[i], x[4 + i] = w1[i];
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = d + i < head_dim ? load_as_f32(row + d + i) : 0.0f;
}

// A query row's exponent e with |x| < 2^(e + 1): x * 2^-e is taken into the product, so that scores do not overflow before they are scaled.
__device__ inline int exponent_of(float most) { return max(static_cast<int>((__float_as_uint(most) >> 23) & 0xffu) - 127, -126); }

// ------------------------------------------------------------------------------------------------- few rows: token generation
//
// A wavefront multiplies 64 tokens at a time with up to 16 rows (tokens of a sequence and query heads that share a key head) on
// v_mfma_f32_16x16x32. It computes scores transposed, tokens x rows: a lane then holds 16 tokens of one row, and by the
// choice of which key goes to which matrix row these are 16 tokens side by side in memory (lane group g: tokens 16 g ..
// 16 g + 15), which is also what it loads of the values (16 bytes of one dimension) and what the second product wants of
// the probabilities. Keys, values and probabilities so go from memory through registers to the matrix units, with no
// exchange between lanes but for the maximum. Matrix unit slots that a tile of 16 rows leaves empty cost nothing.
//
// Bound by the bytes of the codes. The softmax and the turning of codes into numbers take about 750 vector instructions a
// tile, half of the time its 16 KB (128 dimensions) take to arrive; so what counts is that loads are always on their way: page numbers are
// asked for two tiles ahead, a tile's codes as soon as the last tile's have been used. Measured: 131072 tokens of 8 heads of 128
// 55 us with the join (4.9 TB/s), 32 sequences in a window of 4096 with 32 heads of 96 142 us (5.4 TB/s), 64 sequences of
// up to 8192 tokens 128 us (4.3 TB/s: sequences of different lengths, see shape_of); in fp32 the first of these 54 us, the last 127.
template <int W>
struct FewLds {
    float merge_o[4][16][W + 4], merge_m[4][16], merge_l[4][16];
};

template <int W, typename T, int MODE>
__device__ __forceinline__ void attend_few(const Pool &p, const Query &a, const Part &w, FewLds<W> &lds) {
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3;         // bf16 numbers that make an element of q in the first product
    constexpr int kWeights = sizeof(T) == 2 ? 2 : 3;       // bf16 numbers that make a weight of the second
    constexpr int kFull = W / 64, kRest = W % 64 ? 1 : 0;   // loads of 64 dimensions of 16 tokens, and of 32
    constexpr int kStep = MODE == kOwn ? 1 : 4;             // the tiles go round the four wavefronts; kOwn: a wavefront has work of its own
    constexpr int kDims = W / 16;
    auto &merge_o = lds.merge_o;
    auto &merge_m = lds.merge_m, &merge_l = lds.merge_l;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15u;
    const uint32_t b = w.table, head = w.head, split = w.split;
    const Span s = w.s;
    const uint64_t page_bytes = uint64_t{W} << p.page_shift, page_stride = page_bytes * p.kv_heads;
    const uint8_t *k_head = p.k + head * page_bytes, *v_head = p.v + head * page_bytes;
    const float *ks_head = p.k_scale + head, *vs_head = p.v_scale + head;
    const uint32_t in_page = (1u << p.page_shift) - 1;
    const int64_t rows = int64_t{s.count} * a.group;
    for (int64_t row0 = 0; row0 < rows; row0 += 16) {
        const int32_t first = MODE == kShared ? s.pos : s.pos + static_cast<int32_t>(row0 / a.group);
        const int32_t last = MODE == kShared ? s.length - 1 : s.pos + static_cast<int32_t>(min(row0 + 15, rows - 1) / a.group);
        const Tiles tiles = tiles_of(p, a, first, last);
        const int32_t cut = MODE == kWhole ? 0 : tiles.before(w.tiles), from = MODE == kOwn ? cut : 0, until = MODE == kShared ? cut : tiles.count;
        const int32_t per = MODE == kWhole ? tiles_per_split(a, tiles.count) : tiles_per_split(w.splits, w.least, until - from);
        const int32_t begin = from + static_cast<int32_t>(split) * per, end = min(begin + per, until);
        if (MODE == kWhole && begin >= end && split > 0) continue;
        if (MODE != kWhole && begin >= end) {
            const uint32_t nth = MODE == kOwn ? lane : tid;
            if (nth < 16 && row0 + nth < rows) {
                const uint32_t token = static_cast<uint32_t>(s.row) + static_cast<uint32_t>((row0 + nth) / a.group);
                const uint32_t q_head = head * a.group + static_cast<uint32_t>((row0 + nth) % a.group);
                a.part_lse[part_at<MODE>(a, w, uint64_t{token} * a.q_heads + q_head)] = -INFINITY;
            }
            continue;
        }
    // A tile's codes and scales as this lane has them: keys of the tokens 16 (c / 4) .., values of the tokens 16 g ..  As soon as a
    // tile's keys have been multiplied the next tile's are asked for, and so for the values; page numbers come a tile earlier
    // still, so that nothing waits for them.  (A second set of registers for the codes does not fit.)
    u32x4 kc[4][kFull], vc[kDims];
    u32x2 kr[4];
    float ks = 0.0f, vs = 0.0f;
    int32_t page = -1, k_page = -1, v_page = -1, k_later = -1, v_later = -1;
    const auto tile_at = [&](int32_t i) { return tiles.at(min(i, end - 1)) * kTile; };
    const auto ask_pages = [&](int32_t i) {
        k_later = table_entry(p, b, tile_at(i) + 16 * static_cast<int32_t>(c >> 2));
        v_later = table_entry(p, b, tile_at(i) + 16 * static_cast<int32_t>(g));
    };
    const auto take_pages = [&](int32_t i) {
        k_page = checked_page(p, k_later, tile_at(i) + 16 * static_cast<int32_t>(c >> 2));
        v_page = checked_page(p, v_later, tile_at(i) + 16 * static_cast<int32_t>(g));
    };
    const auto ask_keys = [&](int32_t i) {
        const uint32_t at = (static_cast<uint32_t>(tile_at(i)) + 16 * (c >> 2)) & in_page;
        const uint8_t *kp = k_head + static_cast<uint32_t>(max(k_page, 0)) * page_stride + (at + (c & 3u)) * W;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int f = 0; f < kFull; ++f) kc[t][f] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kp + 4 * t * W + 64 * f + 16 * g));
            if (kRest) kr[t] = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(kp + 4 * t * W + 64 * kFull + 8 * g));
        }
        ks = ks_head[uint64_t{static_cast<uint32_t>(max(v_page, 0))} * p.kv_heads];
    };
    const auto ask_values = [&](int32_t i) {
        const uint32_t at = (static_cast<uint32_t>(tile_at(i)) + 16 * g) & in_page;
        const uint8_t *vp = v_head + static_cast<uint32_t>(max(v_page, 0)) * page_stride + (uint64_t{c} << p.page_shift) + at;
#pragma unroll
        for (int d = 0; d < kDims; ++d) vc[d] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(vp + (uint64_t{16u * d} << p.page_shift)));
        vs = vs_head[uint64_t{static_cast<uint32_t>(max(v_page, 0))} * p.kv_heads];
    };
    const int32_t i0 = begin + (MODE == kOwn ? 0 : static_cast<int32_t>(wave));
    // the lane's row
    const int64_t my_row = row0 + c;
    const bool mine = my_row < rows;
    const uint32_t my_token = static_cast<uint32_t>(s.row) + static_cast<uint32_t>((mine ? my_row : row0) / a.group);
    const uint32_t my_head = head * a.group + static_cast<uint32_t>((mine ? my_row : row0) % a.group);
    const int32_t my_pos = MODE != kShared ? s.pos + static_cast<int32_t>(my_token) - s.row : a.window ? position_of(p, a, w, my_token) : s.pos;

    bf16x8 q[W / 32][kParts];
    float q_factor;
    {
        const T *row = static_cast<const T *>(a.q) + my_token * a.q_token_stride + my_head * a.q_head_stride;
        float x[W / 32][8], most = 0.0f;
        if (i0 < end) ask_pages(i0);
#pragma unroll
        for (int f = 0; f < W / 32; ++f)
            load_eight(row, f < 2 * kFull ? (f / 2) * 64 + g * 16 + (f & 1) * 8 : kFull * 64 + g * 8, p.head_dim, a.aligned, x[f]);
        if (i0 < end) {
            take_pages(i0);
            ask_pages(i0 + kStep);
            ask_keys(i0);
            ask_values(i0);
        }
#pragma unroll
        for (int f = 0; f < W / 32; ++f)
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[f][i]));
        const int e = exponent_of(column_max(most));
        const float sign = a.scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
        for (int f = 0; f < W / 32; ++f) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[f][i] = ldexpf(x[f][i] * sign, -e);
            split_factors<kParts>(x[f], q[f]);
        }
        q_factor = ldexpf(fabsf(a.scale) * kLog2e, e);
    }
    f32x4 o[kDims];
#pragma unroll
    for (int d = 0; d < kDims; ++d) o[d] = f32x4{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;

    for (int32_t i = i0; i < end; i += kStep) {
        const int32_t t0 = tile_at(i);
        page = v_page;
        f32x4 z[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            z[t] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int f = 0; f < kFull; ++f) {
                const bf16x8 k0 = eight_values(kc[t][f][0], kc[t][f][1]), k1 = eight_values(kc[t][f][2], kc[t][f][3]);
#pragma unroll
                for (int n = 0; n < kParts; ++n) {
                    z[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[2 * f][n], z[t], 0, 0, 0);
                    z[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[2 * f + 1][n], z[t], 0, 0, 0);
                }
            }
            if (kRest) {
                const bf16x8 k0 = eight_values(kr[t][0], kr[t][1]);
#pragma unroll
                for (int n = 0; n < kParts; ++n) z[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[2 * kFull][n], z[t], 0, 0, 0);
            }
        }
        // scores in units of log2; a page without a token that is seen may hold anything as its scale
        const float factor = fmaxf(ks * q_factor, 1e-37f);
        take_pages(i + kStep);
        ask_pages(i + 2 * kStep);
        ask_keys(i + kStep);
        if (!(t0 + kTile - 1 <= first && (!a.window || static_cast<uint32_t>(last - t0) < a.window) && __all(page >= 0))) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int32_t key = t0 + 16 * static_cast<int32_t>(g) + 4 * t + j;
                    const bool seen = (page >= 0) & (key <= my_pos) &
                                      ((a.window == 0) | (static_cast<uint32_t>(my_pos - key) < a.window) | (static_cast<uint32_t>(key) < a.sinks));
                    z[t][j] = seen ? z[t][j] : -INFINITY;
                }
        }
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, z[t][j]);
        const float scale = top > -INFINITY ? vs : 0.0f;
        top = column_max(top * factor);
        if (__any(top > m + kRise)) {
            const float now = fmaxf(m, top), by = __builtin_amdgcn_exp2f(m - (now == -INFINITY ? 0.0f : now));
            m = now;
            l *= by;
#pragma unroll
            for (int d = 0; d < kDims; ++d) o[d] *= by;
        }
        const float base = m == -INFINITY ? 0.0f : m + kRise;
        bf16x8 weights[2][kWeights];
        float tile_l = MODE == kWhole ? l : 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e = __builtin_amdgcn_exp2f(fmaf(z[2 * h + j / 4][j & 3], factor, -base));
                tile_l += e;
                x[j] = e * scale;
            }
            split_factors<kWeights>(x, weights[h]);
        }
        l = MODE == kWhole ? tile_l : l + tile_l;
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
            const bf16x8 v0 = eight_values(vc[d][0], vc[d][1]), v1 = eight_values(vc[d][2], vc[d][3]);
#pragma unroll
            for (int n = 0; n < kWeights; ++n) {
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, weights[0][n], o[d], 0, 0, 0);
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, weights[1][n], o[d], 0, 0, 0);
            }
        }
        ask_values(i + kStep);
    }
        l = column_sum(l);
        if constexpr (MODE == kOwn) {
            if (mine) {
                const float inv = l > 0.0f ? 1.0f / l : 0.0f, base = m == -INFINITY ? 0.0f : m;
                const uint64_t at = part_at<MODE>(a, w, uint64_t{my_token} * a.q_heads + my_head);
#pragma unroll
                for (int d = 0; d < kDims; ++d) *reinterpret_cast<f32x4 *>(a.part_o + at * W + 16 * d + 4 * g) = l == l ? o[d] * inv : f32x4{l, l, l, l};
                if (g == 0) a.part_lse[at] = l > 0.0f ? base + __builtin_amdgcn_logf(l * kUnit) : l == l ? -INFINITY : l;
            }
            continue;
        }
        // the four wavefronts' parts
        __syncthreads();
#pragma unroll
        for (int d = 0; d < kDims; ++d) *reinterpret_cast<f32x4 *>(&merge_o[wave][c][16 * d + 4 * g]) = o[d];
        if (g == 0) merge_m[wave][c] = m, merge_l[wave][c] = l;
        __syncthreads();
        const uint32_t r = tid >> 4, d0 = tid & 15u;           // 16 lanes to a row
        if (row0 + r < rows) {
            float most = -INFINITY, sum = 0.0f, share[4];
            for (int i = 0; i < 4; ++i) most = fmaxf(most, merge_m[i][r]);
            const float base = most == -INFINITY ? 0.0f : most;
            for (int i = 0; i < 4; ++i) {
                share[i] = __builtin_amdgcn_exp2f(merge_m[i][r] - base);
                sum += merge_l[i][r] * share[i];
            }
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
            const uint32_t token = static_cast<uint32_t>(s.row) + static_cast<uint32_t>((row0 + r) / a.group);
            const uint32_t q_head = head * a.group + static_cast<uint32_t>((row0 + r) % a.group);
            const float lse = sum > 0.0f ? base + __builtin_amdgcn_logf(sum * kUnit) : sum == sum ? -INFINITY : sum;
            const uint64_t at = uint64_t{token} * a.q_heads + q_head;
            for (uint32_t d = d0; d < p.head_dim; d += 16) {
                float x = 0.0f;
                for (int i = 0; i < 4; ++i) x += merge_o[i][r][d] * share[i];
                x = sum == sum ? x * inv : sum;
                if (MODE == kWhole && a.splits == 1)
                    store_as(static_cast<T *>(a.out) + token * a.out_token_stride + q_head * a.out_head_stride + d, x);
                else
                    a.part_o[part_at<MODE>(a, w, at) * W + d] = x;
            }
            if (d0 == 0) {
                if (MODE != kWhole || a.splits > 1) a.part_lse[part_at<MODE>(a, w, at)] = lse;
                else if (a.lse) a.lse[at] = lse * kLn2;
            }
        }
    }
}

template <int W, typename T>
__global__ __launch_bounds__(kWG, W > 128 ? 1 : 2) void k_attend_few(Pool p, Query a) {
    __shared__ FewLds<W> lds;
    // Workgroups go to the XCDs in turn. Those of one XCD take the key heads of the same sequence and split, whose codes lie side by side, and
    // the splits of a sequence go to different XCDs, so that long sequences do not meet on one.
    const uint32_t r = p.seqs < 8 ? blockIdx.x : blockIdx.x / 8, head = r % p.kv_heads, split = r / p.kv_heads % a.splits, block = r / p.kv_heads / a.splits;
    const uint32_t b = p.seqs < 8 ? block : 8 * block + ((blockIdx.x - split) & 7u);
    if (b >= p.seqs) return;
    Part w = {};
    w.s = span_of(a.start, p.lengths, b, a.tokens);
    w.table = b;
    w.head = head;
    w.split = split;
    attend_few<W, T, kWhole>(p, a, w, lds);
}

// ----------------------------------------------------------------------------------------------------- many rows: prompts
//
// A workgroup takes 32 rows a wavefront (tokens and the query heads of a key head side by side) and goes through the tokens 64 at
// a time. All its threads turn the tile's codes into the bf16 numbers of the products, once, on their way to LDS;
// rows in LDS are 16 bytes longer than their data, so that the 16 lanes that read one place of 16 rows meet 64 different banks. While a tile is multiplied, the next one is written to the other half of the LDS and the
// codes of the one after it, and the page numbers of a third, are on their way.
//
// v_mfma_f32_32x32x16, scores transposed as above: a lane holds 32 of a tile's scores of one row, tokens 8 i + 4 h + (0..3)
// of each 32, h being the lane's half. The values' tokens lie in LDS in the order 0-3, 8-11, 4-7, 12-15 of each 16, so that what a
// lane reads of them for the second product are the tokens whose weights it has.
//
// Bound by issue: of a compute unit's time, matrix instructions take 43 % and vector instructions 65 %, and together they
// run in 19 %. 4096 rows of 32 heads of 128 over 8192 tokens: 635 to 650 us, 0.63 to 0.65 PFLOP/s of the definition's operations (0.95 of the
// matrix units', as weights are two bf16 numbers). Left out one at a time, the second product takes 288 us with it, the first 202, the codes'
// way to LDS 71. fp32 rows take twice the matrix instructions, and one workgroup a compute unit (382 registers at 96 dimensions): 98 row
// groups of 4 key heads of 80 dimensions, each over about 1100 tokens, 182 us. Registers that do not fit are kept in memory: at 256 dimensions
// 170 for fp32 and 37 for bf16, at 192 36 for fp32, at 96 and 128 2 and 4 for bf16.
template <int W>
struct ManyLds {
    static constexpr int kKeyRow = 2 * W + 16, kValueRow = 2 * kTile + 16;   // bytes
    __attribute__((aligned(16))) uint8_t key[2][kTile * kKeyRow], value[2][W * kValueRow];
    f32x4 ks[2], vs[2];
    int32_t ok[2][4];
};

// ONE: a tile lies in one page (of 64 tokens and more). Its number is then a scalar, and so is all of the codes' addresses but a lane's place in the tile.
template <int W, typename T, int MODE, bool ONE = false>
__device__ __forceinline__ void attend_many(const Pool &p, const Query &a, const Part &w, uint32_t tile_from_end, uint32_t row_tiles, ManyLds<W> &lds) {
    constexpr int kThreads = kWG, kRows = kManyRows;
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kWeights = sizeof(T) == 2 ? 2 : 3;
    constexpr int kChunks = (W * 4 + kThreads - 1) / kThreads;      // pieces of 16 codes a thread turns, of keys and of values
    constexpr int kKeyRow = ManyLds<W>::kKeyRow, kValueRow = ManyLds<W>::kValueRow;
    auto &key_lds = lds.key;
    auto &value_lds = lds.value;
    auto &tile_ks = lds.ks, &tile_vs = lds.vs;
    auto &tile_ok = lds.ok;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, c = lane & 31u;
    const uint32_t b = w.table, head = w.head, split = w.split;
    const Span s = w.s;
    const uint64_t page_bytes = uint64_t{W} << p.page_shift, page_stride = page_bytes * p.kv_heads;
    const uint8_t *k_head = p.k + head * page_bytes, *v_head = p.v + head * page_bytes;
    const uint32_t in_page = (1u << p.page_shift) - 1;
    const int64_t rows = int64_t{s.count} * a.group;
    const int64_t groups = (rows + kRows - 1) / kRows;
    // the last rows see the most tokens: they come first
    for (int64_t group = groups - 1 - tile_from_end; group >= 0; group -= row_tiles) {
        const int64_t row0 = group * kRows;
        const int32_t first = MODE == kShared ? s.pos : s.pos + static_cast<int32_t>(row0 / a.group);
        const int32_t last = MODE == kShared ? s.length - 1 : s.pos + static_cast<int32_t>(min(row0 + kRows - 1, rows - 1) / a.group);
        const Tiles tiles = tiles_of(p, a, first, last);
        const int32_t cut = MODE == kWhole ? 0 : tiles.before(w.tiles), from = MODE == kOwn ? cut : 0, until = MODE == kShared ? cut : tiles.count;
        const int32_t per = MODE == kWhole ? tiles_per_split(a, tiles.count) : tiles_per_split(w.splits, w.least, until - from);
        const int32_t begin = from + static_cast<int32_t>(split) * per, end = min(begin + per, until);
        if (MODE == kWhole && begin >= end && split > 0) continue;
        const int64_t my_row = row0 + 32 * wave + c;
        const bool mine = my_row < rows;
        const uint32_t my_token = static_cast<uint32_t>(s.row) + static_cast<uint32_t>((mine ? my_row : row0) / a.group);
        const uint32_t my_head = head * a.group + static_cast<uint32_t>((mine ? my_row : row0) % a.group);
        if (MODE != kWhole && begin >= end) {
            if (mine && h == 0) a.part_lse[part_at<MODE>(a, w, uint64_t{my_token} * a.q_heads + my_head)] = -INFINITY;
            continue;
        }
        const int32_t my_pos = !mine ? -1 : MODE != kShared ? s.pos + static_cast<int32_t>(my_token) - s.row : a.window ? position_of(p, a, w, my_token) : s.pos;
        // positions of the wavefront's rows
        const int64_t wave_row = row0 + 32 * wave;
        const int32_t wave_first = MODE == kShared ? first : s.pos + static_cast<int32_t>(wave_row / a.group);
        const int32_t wave_last = wave_row >= rows ? -1 : MODE == kShared ? last : s.pos + static_cast<int32_t>(min(wave_row + 31, rows - 1) / a.group);
        bf16x8 q[W / 16][kParts];
        float q_factor;
        constexpr bool kEarly = MODE != kWhole;    // q's elements are asked for before all else and kept as they are
        u32x4 raw[W / 16][sizeof(T) / 2];
        if constexpr (kEarly) {
            const T *row = static_cast<const T *>(a.q) + my_token * a.q_token_stride + my_head * a.q_head_stride;
#pragma unroll
            for (int f = 0; f < W / 16; ++f) {
                const uint32_t d = 16 * f + 8 * h;
                if (a.aligned && d + 8 <= p.head_dim) {
#pragma unroll
                    for (uint32_t i = 0; i < sizeof(T) / 2; ++i) raw[f][i] = reinterpret_cast<const u32x4 *>(row + d)[i];
                } else {
                    float x[8];
                    load_eight(row, d, p.head_dim, false, x);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (sizeof(T) == 2) raw[f][0][i] = upper_halves(x[2 * i], x[2 * i + 1]);
                        else raw[f][0][i] = __float_as_uint(x[i]), raw[f][sizeof(T) / 2 - 1][i] = __float_as_uint(x[4 + i]);
                    }
                }
            }
        }
        const auto eight_of = [&](int f, float *x) {
            if constexpr (kEarly) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    x[i] = __uint_as_float(sizeof(T) == 4 ? raw[f][(i / 4) % (sizeof(T) / 2)][i & 3] : i & 1 ? raw[f][0][i / 2] & 0xffff0000u : raw[f][0][i / 2] << 16);
            } else {
                load_eight(static_cast<const T *>(a.q) + my_token * a.q_token_stride + my_head * a.q_head_stride, 16 * f + 8 * h, p.head_dim, a.aligned, x);
            }
        };
        const auto take_q = [&]() {
            float most = 0.0f;
#pragma unroll
            for (int f = 0; f < W / 16; ++f) {
                float x[8];
                eight_of(f, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));
            }
            const int e = exponent_of(fmaxf(most, __shfl_xor(most, 32)));
            const float sign = a.scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
            for (int f = 0; f < W / 16; ++f) {
                float x[8];
                eight_of(f, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = ldexpf(x[i] * sign, -e);
                split_factors<kParts>(x, q[f]);
            }
            q_factor = ldexpf(fabsf(a.scale) * kLog2e, e);
        };
        if (MODE == kWhole) take_q();
        constexpr int kDims = W / 32;
        f32x16 o[kDims];
#pragma unroll
        for (int d = 0; d < kDims; ++d) o[d] = f32x16{};
        float m = -INFINITY, l = 0.0f;

        int32_t k_page[kChunks], v_page[kChunks], s_page = -1;
        u32x4 kc[kChunks], vc[kChunks];
        float ks = 0.0f, vs = 0.0f;
        int32_t s_ok = 0;
        const auto ask_pages = [&](int32_t i) {
            const int32_t t0 = tiles.at(min(i, end - 1)) * kTile;
            if constexpr (ONE) {
                s_page = table_entry(p, b, t0);
                return;
            }
#pragma unroll
            for (int n = 0; n < kChunks; ++n) {
                const int32_t ch = n * kThreads + static_cast<int32_t>(tid);
                k_page[n] = table_entry(p, b, t0 + min(ch / (W / 16), kTile - 1));
                v_page[n] = table_entry(p, b, t0 + 16 * (ch & 3));
            }
            if (wave == 0) s_page = table_entry(p, b, t0 + 16 * static_cast<int32_t>(tid & 3u));
        };
        const auto ask_codes = [&](int32_t i) {
            const int32_t t0 = tiles.at(min(i, end - 1)) * kTile;
            if constexpr (ONE) {
                const int32_t id = __builtin_amdgcn_readfirstlane(checked_page(p, s_page, t0));
                const uint64_t page = static_cast<uint32_t>(max(id, 0));
                const uint32_t at = static_cast<uint32_t>(t0) & in_page;
                const uint8_t *k = k_head + page * page_stride + at * W, *v = v_head + page * page_stride + at;
#pragma unroll
                for (int n = 0; n < kChunks; ++n) {
                    const uint32_t ch = min(static_cast<uint32_t>(n * kThreads) + tid, W * 4u - 1);
                    kc[n] = *reinterpret_cast<const u32x4 *>(k + 16 * ch);
                    vc[n] = *reinterpret_cast<const u32x4 *>(v + (((ch >> 2) << p.page_shift) + 16 * (ch & 3u)));
                }
                if (wave == 0) {
                    ks = p.k_scale[page * p.kv_heads + head];
                    vs = p.v_scale[page * p.kv_heads + head];
                    s_ok = id >= 0;
                }
                return;
            }
#pragma unroll
            for (int n = 0; n < kChunks; ++n) {
                const int32_t ch = min(n * kThreads + static_cast<int32_t>(tid), W * 4 - 1);
                const int32_t k_at = t0 + ch / (W / 16), v_at = t0 + 16 * (ch & 3);
                const uint64_t k_id = static_cast<uint32_t>(max(checked_page(p, k_page[n], k_at), 0)), v_id = static_cast<uint32_t>(max(checked_page(p, v_page[n], v_at), 0));
                kc[n] = *reinterpret_cast<const u32x4 *>(k_head + k_id * page_stride + (static_cast<uint32_t>(k_at) & in_page) * W + 16 * (ch % (W / 16)));
                vc[n] = *reinterpret_cast<const u32x4 *>(v_head + v_id * page_stride + (static_cast<uint32_t>(ch >> 2) << p.page_shift) + (static_cast<uint32_t>(v_at) & in_page));
            }
            if (wave == 0) {
                const int32_t id = checked_page(p, s_page, t0 + 16 * static_cast<int32_t>(tid & 3u));
                const uint64_t at = uint64_t{static_cast<uint32_t>(max(id, 0))} * p.kv_heads + head;
                ks = p.k_scale[at];
                vs = p.v_scale[at];
                s_ok = id >= 0;
            }
        };
        const auto to_lds = [&](int half) {
#pragma unroll
            for (int n = 0; n < kChunks; ++n) {
                const int32_t ch = n * kThreads + static_cast<int32_t>(tid);
                if (kThreads * kChunks != W * 4 && ch >= W * 4) continue;
                bf16x8 *k = reinterpret_cast<bf16x8 *>(key_lds[half] + (ch / (W / 16)) * kKeyRow + 32 * (ch % (W / 16)));
                k[0] = eight_values(kc[n][0], kc[n][1]);
                k[1] = eight_values(kc[n][2], kc[n][3]);
                bf16x8 *v = reinterpret_cast<bf16x8 *>(value_lds[half] + (ch >> 2) * kValueRow + 32 * (ch & 3));
                v[0] = eight_values(vc[n][0], vc[n][2]);
                v[1] = eight_values(vc[n][1], vc[n][3]);
            }
            if (tid < 4) {
                // a page without a token that is seen may hold anything as its scale
                reinterpret_cast<float *>(&tile_ks[half])[tid] = fabsf(ks) < INFINITY ? ks : 0.0f;
                reinterpret_cast<float *>(&tile_vs[half])[tid] = fabsf(vs) < INFINITY ? vs : 0.0f;
                tile_ok[half][tid] = s_ok;
            }
        };
        __syncthreads();                           // the last group's tiles have been read
        if (begin < end) {
            ask_pages(begin);
            ask_codes(begin);
            ask_pages(begin + 1);
            if (MODE != kWhole) take_q();          // while the first codes are on their way
            to_lds(0);
            ask_codes(begin + 1);
            ask_pages(begin + 2);
        }
        __syncthreads();

        // What the matrix units take from LDS is asked for kAhead pieces before it is used.  The first product tells the compiler so in groups (matrix
        // instructions 8, LDS reads 256), as it otherwise moves each read to its use where registers are short: 1024 rows of 16 heads over 4096 tokens
        // in bf16, 192 dimensions 173 and 165 us, 256 227 and 213, in fp32 96 dimensions 136 and 132, 128 153 and 148.  (The second product's reads
        // in groups as well leave the weights' instructions behind one another: 167 and 220, 137 and 156 us.)
        constexpr int kAhead = 4;
        // the second product: weights of four times 16 tokens
        const auto add_values = [&](const bf16x8 (*weights)[kWeights], int half) {
            const uint8_t *at = value_lds[half] + c * kValueRow + 16 * h;
            const auto piece = [&](int i) { return *reinterpret_cast<const bf16x8 *>(at + 32 * (i % kDims) * kValueRow + 32 * (i / kDims)); };
            bf16x8 v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) v[i] = piece(i);
#pragma unroll
            for (int i = 0; i < 4 * kDims; ++i) {
                const bf16x8 now = v[i % kAhead];
                if (i + kAhead < 4 * kDims) v[i % kAhead] = piece(i + kAhead);
#pragma unroll
                for (int n = 0; n < kWeights; ++n) o[i % kDims] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(now, weights[i / kDims][n], o[i % kDims], 0, 0, 0);
            }
        };
        for (int32_t i = begin; i < end; ++i) {
            const int half = (i - begin) & 1;
            const int32_t t0 = tiles.at(i) * kTile;
            const bool work = t0 <= wave_last;      // a wavefront whose rows see nothing here only turns codes
            f32x16 z[2];
            if (work) {
                z[0] = z[1] = f32x16{};
                const uint8_t *at = key_lds[half] + c * kKeyRow + 16 * h;
                // two tokens' groups in turn, so that a product does not wait for the one before it
                const auto piece = [&](int j) { return *reinterpret_cast<const bf16x8 *>(at + 32 * (j & 1) * kKeyRow + 32 * (j >> 1)); };
                bf16x8 k[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j) k[j] = piece(j);
                __builtin_amdgcn_sched_group_barrier(256, kAhead, 0);
#pragma unroll
                for (int j = 0; j < W / 8; ++j) {
                    const bf16x8 now = k[j % kAhead];
                    if (j + kAhead < W / 8) k[j % kAhead] = piece(j + kAhead);
#pragma unroll
                    for (int n = 0; n < kParts; ++n) z[j & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(now, q[j >> 1][n], z[j & 1], 0, 0, 0);
                    __builtin_amdgcn_sched_group_barrier(8, kParts, 0);
                    if (j + kAhead < W / 8) __builtin_amdgcn_sched_group_barrier(256, 1, 0);
                }
            }
            if (i + 1 < end) to_lds(half ^ 1);
            ask_codes(i + 2);
            ask_pages(i + 3);
            if (work) {
                f32x4 kf = tile_ks[half] * q_factor;
                const f32x4 vf = tile_vs[half];
                const bool all = t0 + kTile - 1 <= wave_first && (!a.window || static_cast<uint32_t>(wave_last - t0) < a.window) &&
                                 (tile_ok[half][0] & tile_ok[half][1] & tile_ok[half][2] & tile_ok[half][3]);
                if (!all) {
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const int32_t key = t0 + 32 * t + 8 * (j / 4) + 4 * static_cast<int32_t>(h) + (j & 3);
                            const bool seen = (tile_ok[half][2 * t + j / 8] != 0) & (key <= my_pos) &
                                              ((a.window == 0) | (static_cast<uint32_t>(my_pos - key) < a.window) | (static_cast<uint32_t>(key) < a.sinks));
                            z[t][j] = seen ? z[t][j] : -INFINITY;
                        }
                }
                float top = -INFINITY;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    kf[g] = fmaxf(kf[g], 1e-37f);   // minus infinity stays that
                    float most = z[g / 2][8 * (g & 1)];
#pragma unroll
                    for (int j = 1; j < 8; ++j) most = fmaxf(most, z[g / 2][8 * (g & 1) + j]);
                    top = fmaxf(top, most * kf[g]);
                }
                top = fmaxf(top, __shfl_xor(top, 32));
                if (__any(top > m + kRise)) {
                    const float now = fmaxf(m, top), by = __builtin_amdgcn_exp2f(m - (now == -INFINITY ? 0.0f : now));
                    m = now;
                    l *= by;
#pragma unroll
                    for (int d = 0; d < kDims; ++d) o[d] *= by;
                }
                const float base = m == -INFINITY ? 0.0f : m + kRise;
                bf16x8 weights[4][kWeights];
                float tile_l = MODE == kWhole ? l : 0.0f;
#pragma unroll
                for (int g = 0; g < 4; ++g) {       // 16 tokens
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float e = __builtin_amdgcn_exp2f(fmaf(z[g / 2][8 * (g & 1) + j], kf[g], -base));
                        tile_l += e;
                        x[j] = e * vf[g];
                    }
                    split_factors<kWeights>(x, weights[g]);
                }
                l = MODE == kWhole ? tile_l : l + tile_l;
                add_values(weights, half);
            }
            __syncthreads();
        }
        l += __shfl_xor(l, 32);
        if (mine) {
            const float inv = l > 0.0f ? 1.0f / l : 0.0f, base = m == -INFINITY ? 0.0f : m;
            const float lse = l > 0.0f ? base + __builtin_amdgcn_logf(l * kUnit) : l == l ? -INFINITY : l;
            const uint64_t at = uint64_t{my_token} * a.q_heads + my_head;
            T *out = static_cast<T *>(a.out) + my_token * a.out_token_stride + my_head * a.out_head_stride;
            float *part = a.part_o + part_at<MODE>(a, w, at) * W;
#pragma unroll
            for (int d = 0; d < kDims; ++d)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const uint32_t dim = 32 * d + 8 * (j / 4) + 4 * h + (j & 3);
                    const float x = l == l ? o[d][j] * inv : l;
                    if (MODE != kWhole || a.splits > 1) part[dim] = x;
                    else if (dim < p.head_dim) store_as(out + dim, x);
                }
            if (h == 0) {
                if (MODE != kWhole || a.splits > 1) a.part_lse[part_at<MODE>(a, w, at)] = lse;
                else if (a.lse) a.lse[at] = lse * kLn2;
            }
        }
    }
}

template <int W, typename T>
__global__ __launch_bounds__(kWG, sizeof(T) == 2 && W <= 128 ? 2 : 1) void k_attend_many(Pool p, Query a, uint32_t row_tiles) {
    __shared__ ManyLds<W> lds;
    // workgroups of one key head follow each other at multiples of the number of heads: with 8 heads, on one XCD and its L2
    const uint32_t units = p.seqs * p.kv_heads, unit = blockIdx.x % units;
    Part w = {};
    w.head = unit % p.kv_heads;
    w.table = unit / p.kv_heads;
    w.split = blockIdx.x / units % a.splits;
    w.s = span_of(a.start, p.lengths, w.table, a.tokens);
    attend_many<W, T, kWhole>(p, a, w, blockIdx.x / units / a.splits, row_tiles, lds);
}

// Joins the parts of rows whose tiles were split. A workgroup per row and head: its lanes stand for four dimensions each, and as often as
// they cover a row they take parts in turn.
template <int W, typename T>
__global__ __launch_bounds__(kWG) void k_attend_join(Pool p, Query a) {
    constexpr int kLanes = W / 4, kSets = kWG / kLanes;
    __shared__ f32x4 sums[kSets][kLanes];
    __shared__ float wave_most[kWG / 64], wave_sum[kWG / 64], shares[kWG];
    const uint32_t tid = threadIdx.x, set = tid / kLanes, d = tid % kLanes;
    const uint32_t h = blockIdx.x % a.q_heads, b = blockIdx.x / a.q_heads;
    const Span s = span_of(a.start, p.lengths, b, a.tokens);
    for (int32_t nth = static_cast<int32_t>(blockIdx.y); nth < s.count; nth += static_cast<int32_t>(gridDim.y)) {
        const uint32_t token = static_cast<uint32_t>(s.row + nth);
        const uint64_t at = uint64_t{token} * a.q_heads + h;
        const int64_t rows = int64_t{s.count} * a.group, row = int64_t{nth} * a.group + h % a.group;
        const int64_t row0 = row / 16 * 16;
        const Tiles tiles = tiles_of(p, a, s.pos + static_cast<int32_t>(row0 / a.group),
                                     s.pos + static_cast<int32_t>(min(row0 + 15, rows - 1) / a.group));
        const int32_t per = tiles_per_split(a, tiles.count);
        const uint32_t parts = static_cast<uint32_t>(max((tiles.count + per - 1) / per, 1));
        const float *lse = a.part_lse + at * a.splits;
        const f32x4 *part = reinterpret_cast<const f32x4 *>(a.part_o + at * a.splits * W);
        // every part's share, a lane each (there are at most kMostSplits)
        const float mine = tid < parts ? lse[tid] : -INFINITY;
        float most = mine;
        for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
        if ((tid & 63u) == 0) wave_most[tid >> 6] = most;
        __syncthreads();
        for (int i = 0; i < kWG / 64; ++i) most = fmaxf(most, wave_most[i]);
        const float base = most == -INFINITY ? 0.0f : most;
        const float share = __builtin_amdgcn_exp2f(mine - base);
        shares[tid] = share;
        float sum = share;
        for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
        if ((tid & 63u) == 0) wave_sum[tid >> 6] = sum;
        __syncthreads();
        sum = 0.0f;
        for (int i = 0; i < kWG / 64; ++i) sum += wave_sum[i];
        f32x4 x = {0, 0, 0, 0};
        if (set < kSets) {
#pragma unroll 4
            for (uint32_t i = set; i < parts; i += kSets) x += part[i * kLanes + d] * shares[i];
            sums[set][d] = x;
        }
        __syncthreads();
        if (set == 0) {
#pragma unroll
            for (int i = 1; i < kSets; ++i) x += sums[i][d];
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
            T *out = static_cast<T *>(a.out) + token * a.out_token_stride + h * a.out_head_stride;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * d + j < p.head_dim) store_as(out + 4 * d + j, sum == sum ? x[j] * inv : sum);
        }
        if (tid == 0 && a.lse) a.lse[at] = sum > 0.0f ? (base + __builtin_amdgcn_logf(sum)) * kLn2 : (sum == sum ? -INFINITY : sum);
        __syncthreads();
    }
}

// The same for many rows in a few parts: a wavefront per row and head, no more than a lane a part.
template <int W, typename T>
__global__ __launch_bounds__(kWG) void k_attend_join_rows(Pool p, Query a) {
    constexpr uint32_t kLanes = W / 4, kSets = 64 / kLanes;
    const uint32_t lane = threadIdx.x & 63u, set = lane / kLanes, d = lane % kLanes;
    const uint32_t unit = blockIdx.x * (kWG / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = unit % a.q_heads, b = unit / a.q_heads;
    if (b >= p.seqs) return;
    const Span s = span_of(a.start, p.lengths, b, a.tokens);
    const int64_t rows = int64_t{s.count} * a.group;
    for (int32_t nth = static_cast<int32_t>(blockIdx.y); nth < s.count; nth += static_cast<int32_t>(gridDim.y)) {
        const uint32_t token = static_cast<uint32_t>(s.row + nth);
        const uint64_t at = uint64_t{token} * a.q_heads + h;
        const int64_t row0 = (int64_t{nth} * a.group + h % a.group) / kManyRows * kManyRows;
        const Tiles tiles = tiles_of(p, a, s.pos + static_cast<int32_t>(row0 / a.group),
                                     s.pos + static_cast<int32_t>(min(row0 + kManyRows - 1, rows - 1) / a.group));
        const int32_t per = tiles_per_split(a, tiles.count);
        const uint32_t parts = static_cast<uint32_t>(max((tiles.count + per - 1) / per, 1));
        const float mine = lane < parts ? a.part_lse[at * a.splits + lane] : -INFINITY;
        float most = mine;
        for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
        const float base = most == -INFINITY ? 0.0f : most, share = __builtin_amdgcn_exp2f(mine - base);
        float sum = share;
        for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
        const f32x4 *part = reinterpret_cast<const f32x4 *>(a.part_o + at * a.splits * W);
        f32x4 x = {0, 0, 0, 0};
        for (uint32_t i0 = 0; i0 < parts; i0 += kSets) {
            const uint32_t i = i0 + set;
            const float by = __shfl(share, static_cast<int>(min(i, 63u)));
            if (set < kSets && i < parts) x += part[i * kLanes + d] * by;
        }
#pragma unroll
        for (uint32_t i = 1; i < kSets; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float other = __shfl(x[j], static_cast<int>(d + i * kLanes));
                if (set == 0) x[j] += other;
            }
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        T *out = static_cast<T *>(a.out) + token * a.out_token_stride + h * a.out_head_stride;
        if (set == 0)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * d + j < p.head_dim) store_as(out + 4 * d + j, sum == sum ? x[j] * inv : sum);
        if (lane == 0 && a.lse) a.lse[at] = sum > 0.0f ? (base + __builtin_amdgcn_logf(sum)) * kLn2 : (sum == sum ? -INFINITY : sum);
    }
}

// ---------------------------------------------------------------------------------------- groups of sequences behind a prefix
//
// The tokens that a group's sequences share are multiplied with all its rows together (tiles of 16 rows, or 128 of many), so that their codes
// are read, turned and multiplied once and not once a sequence; every sequence's further tokens go by the same launch's other
// workgroups, and k_shared_join brings the parts of a row together.  What is shared is rounded down to whole tiles, and to
// what all of the group's rows see where there is no window; the rest of it is taken as each sequence's own.
//
// Bound by issue for many rows of long prefixes: 64 sequences of 32 / 8 heads of 128 behind 32768 shared and up to 2048 own tokens 89 to 93 us (of
// a compute unit's time vector instructions 52 %, matrix instructions 32 %; wavefronts wait for a quarter of theirs), the shared ones alone 72 (0.48 PFLOP/s; each sequence for
// itself, 64 of 32768 tokens and more, is 2.3 GB of codes).  Short ones are bound by the way to the first tile (bounds of
// the group 3 us, queries, page and codes 4 to 5) and by 2.3 us a tile: 48 answers to 4001 tokens 25 us and 5 for the join.  fp32 rows: one
// wavefront a SIMD, and three times the matrix instructions (five groups of pieces, 216 us).  A kernel holds the bodies for shared and own tokens and, with
// many rows, for both kinds of pages, which takes registers: 41 are kept in memory at 128 dimensions in bf16 (k_attend_many 4), 8 at 96, 56 at 256, in
// fp32 43 at 192, 426 at 256.
// A lane adds up a tile's weights before it adds them to its sum, which may hold a weight some 2^23 times as large: of 65536 tokens in one part, the first
// with all but 0.3 % of the weight, the lse was 1.5e-3 off with one addition a token.
struct Groups {
    const int32_t *first, *shared;
    uint32_t groups;
    uint32_t blocks;                         // workgroups for shared tokens: they come first
    uint32_t row_tiles, splits, least;       // of those
    uint32_t own_tiles, own_splits, own_least;   // of own tokens; own_tiles: 0 where wavefronts take them
};

constexpr uint32_t kMostParts = 256;         // of a row

// A number that all lanes have alike, as a scalar.
__device__ inline int32_t scalar(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// The group of sequence b, or a number that is none.  (All lanes, 64 of the ascending starts at a time.)
__device__ inline uint32_t group_of(const Groups &g, uint32_t b) {
    const uint32_t lane = threadIdx.x & 63u;
    const int32_t at = static_cast<int32_t>(b);
    uint32_t lo = 0, n = g.groups + 1;
    while (n > 64) {
        const uint32_t step = (n + 63) / 64, i = lo + min(lane * step, n - 1);
        const uint32_t below = static_cast<uint32_t>(__builtin_popcountll(__ballot(lane * step < n && g.first[i] <= at)));
        if (below == 0) return g.groups;
        lo += (below - 1) * step;
        n = min(step, n - (below - 1) * step);
    }
    const uint32_t below = static_cast<uint32_t>(__builtin_popcountll(__ballot(lane < n && g.first[lo + min(lane, n - 1)] <= at)));
    return below == 0 ? g.groups : lo + below - 1;
}

// Sequences, rows and shared tiles of group `nth`, by every wavefront for itself.
__device__ inline void take_group(const Pool &p, const Query &a, const Groups &g, uint32_t nth, Part *w) {
    const int32_t lane = static_cast<int32_t>(threadIdx.x & 63u), seqs = static_cast<int32_t>(p.seqs), rows = static_cast<int32_t>(a.tokens);
    const Span mine = span_of(a.start, p.lengths, static_cast<uint32_t>(min(lane, seqs - 1)), a.tokens);      // asked for beside the group's bounds
    const int32_t first = scalar(min(max(g.first[nth], 0), seqs)), last = scalar(min(max(g.first[nth + 1], first), seqs)), shared = g.shared[nth];
    int32_t least = 0x7fffffff, most = -1;
    const auto add = [&](const Span &s) {
        if (s.count) least = min(least, s.pos), most = max(most, s.length - 1);
    };
    if (last <= 64) {
        if (lane >= first && lane < last) add(mine);
    } else {
#pragma unroll 4
        for (int32_t b = first; b < last; b += 64) add(span_of(a.start, p.lengths, static_cast<uint32_t>(min(b + lane, last - 1)), a.tokens));
    }
    for (int o = 32; o; o >>= 1) least = min(least, __shfl_xor(least, o)), most = max(most, __shfl_xor(most, o));
    least = scalar(least);
    most = scalar(most);
    const int64_t slots = int64_t{p.stride} << p.page_shift;
    const int64_t tokens = most < 0 ? 0 : min(min(int64_t{shared}, slots), int64_t{least} + 1);
    w->tiles = tokens < kTile ? 0 : static_cast<int32_t>(tokens / kTile);
    w->first = static_cast<uint32_t>(first);
    w->last = static_cast<uint32_t>(last);
    int32_t row = 0, end = 0;
    if (first < last && last <= 64) {
        row = __builtin_amdgcn_readlane(mine.row, first);
        end = __builtin_amdgcn_readlane(mine.row + mine.count, last - 1);
    } else if (first < last) {
        row = min(max(a.start[first], 0), rows);
        end = min(max(a.start[last], row), rows);
    }
    w->s.row = row;
    w->s.count = max(end - row, 0);
    w->s.pos = least;
    w->s.length = most + 1;
}

template <int W, bool MANY> struct SharedLds {
    union {
        FewLds<W> few;
        ManyLds<W> many;
    };
};
template <int W> struct SharedLds<W, false> {
    FewLds<W> few;
};

template <int W, typename T, bool MANY>
__global__ __launch_bounds__(kWG, MANY ? (sizeof(T) == 2 && W <= 128 ? 2 : 1) : (W > 128 ? 1 : 2)) void k_attend_shared(Pool p, Query a, Groups g) {
    __shared__ SharedLds<W, MANY> lds;
    Part w = {};
    w.parts = g.splits + g.own_splits;
    if (blockIdx.x < g.blocks) {
        // the row tiles and splits of a key head follow each other at multiples of the number of units: with 8 heads, on one XCD and its L2
        const uint32_t units = g.groups * p.kv_heads, unit = blockIdx.x % units;
        w.head = unit % p.kv_heads;
        w.split = blockIdx.x / units % g.splits;
        w.splits = g.splits;
        w.least = g.least;
        take_group(p, a, g, unit / p.kv_heads, &w);
        if (w.s.count == 0) return;
        w.table = w.first;
        if constexpr (MANY) {
            const uint32_t tile = blockIdx.x / units / g.splits;
            if (p.page_shift >= 6) attend_many<W, T, kShared, true>(p, a, w, tile, g.row_tiles, lds.many);
            else attend_many<W, T, kShared, false>(p, a, w, tile, g.row_tiles, lds.many);
        } else {
            attend_few<W, T, kShared>(p, a, w, lds.few);
        }
        return;
    }
    // few rows: a wavefront for itself takes a sequence, key head and split, so that heads whose codes lie side by side are in one workgroup
    const bool by_waves = !MANY || g.own_tiles == 0;
    const uint32_t r = by_waves ? (blockIdx.x - g.blocks) * (kWG / 64) + static_cast<uint32_t>(scalar(static_cast<int32_t>(threadIdx.x >> 6))) : blockIdx.x - g.blocks;
    const uint32_t split = r / p.kv_heads % g.own_splits, rest = r / p.kv_heads / g.own_splits, b = by_waves ? rest : rest % p.seqs;
    if (b >= p.seqs) return;
    const Span s = span_of(a.start, p.lengths, b, a.tokens);
    if (s.count == 0) return;
    const uint32_t nth = group_of(g, b);
    w.head = r % p.kv_heads;
    if (nth < g.groups) {
        take_group(p, a, g, nth, &w);
    } else if (split == 0) {                       // in no group: it has no shared parts
        const uint32_t lanes = by_waves ? 64 : kWG, lane = threadIdx.x % lanes;
        const uint64_t count = uint64_t{static_cast<uint32_t>(s.count)} * a.group * g.splits;
        for (uint64_t i = lane; i < count; i += lanes) {
            const uint64_t row = i / g.splits, token = static_cast<uint32_t>(s.row) + row / a.group;
            a.part_lse[(token * a.q_heads + w.head * a.group + row % a.group) * w.parts + i % g.splits] = -INFINITY;
        }
    }
    w.s = s;
    w.table = b;
    w.split = split;
    w.splits = g.own_splits;
    w.least = g.own_least;
    w.slot = g.splits;
    if constexpr (MANY) {
        if (!by_waves) {
            attend_many<W, T, kOwn>(p, a, w, rest / p.seqs, g.own_tiles, lds.many);
            return;
        }
    }
    attend_few<W, T, kOwn>(p, a, w, lds.few);
}

// Joins the parts of every row and head, a wavefront each; a lane has the lse of every 64th part.  A part that saw nothing has minus infinity as its lse and
// left its sums unwritten: they are read, as nothing waits for what the lse says, and left out.
template <int W, typename T>
__global__ __launch_bounds__(kWG) void k_shared_join(Pool p, Query a) {
    constexpr uint32_t kLanes = W / 4, kSets = 64 / kLanes, kAhead = 4;
    const uint32_t lane = threadIdx.x & 63u, set = lane / kLanes, d = lane % kLanes, parts = min(a.splits, kMostParts);
    const int32_t first = a.start[0], last = a.start[p.seqs];
    const uint32_t all = a.tokens * a.q_heads, step = gridDim.x * (kWG / 64);
    for (uint64_t i = blockIdx.x * (kWG / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < all; i += step) {
        const uint32_t at = static_cast<uint32_t>(i), token = at / a.q_heads, h = at % a.q_heads;
        float share[kMostParts / 64];
#pragma unroll
        for (uint32_t n = 0; n < kMostParts / 64; ++n) {
            const uint32_t nth = 64 * n + lane;
            share[n] = nth < parts ? a.part_lse[uint64_t{at} * parts + nth] : -INFINITY;
        }
        if (static_cast<int32_t>(token) < first || static_cast<int32_t>(token) >= last) continue;      // a row of no sequence
        float most = fmaxf(fmaxf(share[0], share[1]), fmaxf(share[2], share[3]));
        for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
        const float base = most == -INFINITY ? 0.0f : most;
        float sum = 0.0f;
#pragma unroll
        for (uint32_t n = 0; n < kMostParts / 64; ++n) sum += share[n] = __builtin_amdgcn_exp2f(share[n] - base);
        for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
        const f32x4 *part = reinterpret_cast<const f32x4 *>(a.part_o + uint64_t{at} * parts * W);
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t m = 0; m < kMostParts / 64; ++m) {
            const uint32_t until = min(parts, 64 * m + 64);
            for (uint32_t i0 = 64 * m; i0 < until; i0 += kAhead * kSets) {
                f32x4 y[kAhead];
#pragma unroll
                for (uint32_t n = 0; n < kAhead; ++n) y[n] = part[min(i0 + n * kSets + min(set, kSets - 1), parts - 1) * kLanes + d];
#pragma unroll
                for (uint32_t n = 0; n < kAhead; ++n) {
                    const uint32_t i = i0 + n * kSets + set;
                    const float by = __shfl(share[m], static_cast<int>(i & 63u));
                    if (set < kSets && i < until && by != 0.0f) x += y[n] * by;
                }
            }
        }
#pragma unroll
        for (uint32_t i = 1; i < kSets; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float other = __shfl(x[j], static_cast<int>(d + i * kLanes));
                if (set == 0) x[j] += other;
            }
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        T *out = static_cast<T *>(a.out) + token * a.out_token_stride + h * a.out_head_stride;
        if (set == 0)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * d + j < p.head_dim) store_as(out + 4 * d + j, sum == sum ? x[j] * inv : sum);
        if (lane == 0 && a.lse) a.lse[at] = sum > 0.0f ? (base + __builtin_amdgcn_logf(sum)) * kLn2 : (sum == sum ? -INFINITY : sum);
    }
}

// Tokens in leading pages that a group's rows share.  How many slots all of its rows fill: a workgroup a group.
__device__ inline int32_t full_slots(const Pool &p, int32_t begin, int32_t end, int32_t *lds) {
    const uint32_t tid = threadIdx.x;
    int32_t full = begin < end ? static_cast<int32_t>(p.stride) : 0;
    for (int32_t b = begin + static_cast<int32_t>(tid); b < end; b += kWG) full = min(full, max(p.lengths[b], 0) >> p.page_shift);
    for (int o = 32; o; o >>= 1) full = min(full, __shfl_xor(full, o));
    __syncthreads();
    if ((tid & 63u) == 0) lds[tid >> 6] = full;
    __syncthreads();
    for (int i = 0; i < kWG / 64; ++i) full = min(full, lds[i]);
    return full;
}

// The first of 64 slots from s0 on in which the rows part, `full` if none before that: every wavefront takes a quarter of the rows.
__device__ inline int32_t first_parting(const Pool &p, int32_t begin, int32_t end, int32_t s0, int32_t full, int32_t *lds) {
    const uint32_t tid = threadIdx.x;
    const int32_t s = static_cast<int32_t>(min(static_cast<uint32_t>(s0) + (tid & 63u), p.stride - 1));
    const int32_t *column = p.slots + s;
    const int32_t id = column[uint64_t{static_cast<uint32_t>(begin)} * p.stride];
    bool parts = static_cast<uint32_t>(id) >= p.pages;
#pragma unroll 8
    for (int32_t b = begin + 1 + static_cast<int32_t>(tid >> 6); b < end; b += kWG / 64) parts |= column[uint64_t{static_cast<uint32_t>(b)} * p.stride] != id;
    int32_t at = parts ? min(s, full) : full;
    for (int o = 32; o; o >>= 1) at = min(at, __shfl_xor(at, o));
    __syncthreads();
    if ((tid & 63u) == 0) lds[tid >> 6] = at;
    __syncthreads();
    for (int i = 0; i < kWG / 64; ++i) at = min(at, lds[i]);
    return at;
}

// A workgroup a group, up to the first slot in which they part; PIECES: how far they could agree, which k_shared_pieces then lowers.
template <bool PIECES>
__global__ __launch_bounds__(kWG) void k_shared(Pool p, const int32_t *first, int32_t *shared, uint32_t groups) {
    __shared__ int32_t lds[kWG / 64];
    const int32_t seqs = static_cast<int32_t>(p.seqs);
    for (uint32_t g = blockIdx.x; g < groups; g += gridDim.x) {
        const int32_t begin = min(max(first[g], 0), seqs), end = min(max(first[g + 1], begin), seqs);
        const int32_t full = full_slots(p, begin, end, lds);
        int32_t same = full;
        if (!PIECES)
            for (int32_t s0 = 0; s0 < full && same == full; s0 += 64) same = first_parting(p, begin, end, s0, full, lds);
        if (threadIdx.x == 0) shared[g] = same << p.page_shift;
    }
}

// 64 slots of a group a workgroup: all of a long table at once (the minimum is one of integers: its order counts for nothing).
__global__ __launch_bounds__(kWG) void k_shared_pieces(Pool p, const int32_t *first, int32_t *shared, uint32_t groups, uint32_t pieces) {
    __shared__ int32_t lds[kWG / 64];
    const int32_t seqs = static_cast<int32_t>(p.seqs);
    for (uint64_t w = blockIdx.x; w < uint64_t{groups} * pieces; w += gridDim.x) {
        const uint32_t g = static_cast<uint32_t>(w / pieces);
        const int32_t begin = min(max(first[g], 0), seqs), end = min(max(first[g + 1], begin), seqs), s0 = static_cast<int32_t>(w % pieces) * 64;
        if (begin >= end) continue;
        const int32_t at = first_parting(p, begin, end, s0, 0x7fffffff >> p.page_shift, lds);
        if (threadIdx.x == 0 && at < s0 + 64) atomicMin(shared + g, at << p.page_shift);
    }
}

// defined below
using QueryCheck = entro_status(const entro_cache *, const entro_cache_query *);
QueryCheck check_query, check_query_sizes;
int compute_units();

entro_status check_groups_sizes(const entro_cache_groups *g) {
    if (!g) return ENTRO_ERR_NULL;
    return g->groups == 0 || g->groups > 0x7ffffffeu ? ENTRO_ERR_SIZE : ENTRO_OK;
}

entro_status check_groups(const entro_cache_groups *g) {
    if (const entro_status s = check_groups_sizes(g)) return s;
    if (!g->first || !g->shared) return ENTRO_ERR_NULL;
    return aligned16(g->first) && aligned16(g->shared) ? ENTRO_OK : ENTRO_ERR_ALIGN;
}

// Slots that one workgroup a group goes through; longer tables take two launches (8 groups of 8 rows, one and two: 100 slots 3.6 and 4.7 us, 200 4.4
// and 4.8, 300 5.6 and 4.8, 800 10.5 and 5.2).
constexpr uint32_t kShortTable = 256;
constexpr uint64_t kHalfGroups = kMostGroups / 2;     // workgroups for shared and for own tokens
constexpr uint32_t kMostShared = 128, kMostOwn = kMostParts - kMostShared;

struct SharedShape {
    bool many;
    Groups g;
    uint64_t bytes;
};

uint64_t tiles_in(uint64_t tokens, const entro_cache_query *q, uint64_t rows) {
    const uint64_t seen = uint64_t{q->window} + q->sinks + rows + 2 * kTile;
    return ((q->window && tokens > seen ? seen : tokens) + kTile - 1) / kTile;
}

uint32_t between(uint64_t x, uint64_t lo, uint64_t hi) { return static_cast<uint32_t>(x > hi ? hi : x < lo ? lo : x); }

// How far the tokens of either kind are split.  Hints may say anything: the kernels' own loops cover the rest.
SharedShape shared_shape_of(const entro_cache *c, const entro_cache_table *t, const entro_cache_query *q, const entro_cache_groups *groups) {
    SharedShape s = {};
    const uint32_t max_new = between(q->max_new, 1, q->tokens < 1 ? 1 : q->tokens), group = q->q_heads / c->kv_heads;
    const uint64_t seqs = between(groups->max_seqs, 1, t->seqs), own_rows = uint64_t{max_new} * group;
    const uint64_t all = seqs * max_new, rows = (all < q->tokens ? all : q->tokens) * group;
    const uint64_t shared = groups->max_shared < q->max_len ? groups->max_shared : q->max_len;
    const uint64_t alone = groups->max_own < 1 ? q->max_len - shared : groups->max_own < q->max_len ? groups->max_own : q->max_len;
    const uint64_t tiles = tiles_in(shared, q, max_new), own_tiles = tiles_in(alone + kTile, q, max_new);
    const uint64_t cus = static_cast<uint64_t>(compute_units()), units = uint64_t{groups->groups} * c->kv_heads, own_units = uint64_t{t->seqs} * c->kv_heads;
    // rows of a key head over 1024, 4096, 8192 and 32768 shared tokens of 8 of them, with 30 own ones a sequence, by tiles of 16 rows and of 128, us: 20 rows
    // 21, 22, 23, 38 and 14, 17, 21, 47; 32 rows 21, 22, 24, 39 and 15, 17, 22, 48; 40 rows 28, 29, 31, 53 and 15, 17, 22, 48; 64 rows 35, 37, 40, 69 and 16,
    // 19, 24, 50; in fp32 32 rows 24, 26, 26, 42 and 18, 28, 34, 73; 40 rows 33, 34, 35, 55 and 18, 29, 36, 74; 64 rows 42, 44, 46, 72 and 19, 30, 38, 76.
    // (The length is not looked at: up to 32 rows of prefixes below some 16384 tokens would be faster in bf16 by tiles of 128, 33 to 64 in fp32 of longer ones by those of 16.)
    s.many = rows > 32;
    s.g.groups = groups->groups;
    s.g.row_tiles = s.many ? between((rows + kManyRows - 1) / kManyRows, 1, kHalfGroups / units) : 1;
    // own tokens: up to 24 tiles in one piece; of longer ones as many pieces of 8 tiles and more as give every compute unit a workgroup (64 sequences with
    // up to 33 tiles of their own behind 32768 shared tokens: one piece 101 us at the best, two 94, four 94).  max_own says how many there may be: 32
    // sequences with 100 of their own behind 32768 beside one of 32868 in no group 969 us by max_len less max_shared, 98 by max_own
    const bool own_many = s.many && own_rows > 32;
    s.g.own_tiles = own_many ? between((own_rows + kManyRows - 1) / kManyRows, 1, kHalfGroups / own_units) : 0;
    const uint64_t own_fill = own_many ? own_units * s.g.own_tiles : (own_units + 3) / 4;
    const uint64_t own_fills = (cus + own_fill - 1) / own_fill, own_least = (own_tiles + 23) / 24, own_most = (own_tiles + 7) / 8;
    const uint64_t own_want = own_tiles <= 24 ? 1 : own_fills < own_least ? own_least : own_fills < own_most ? own_fills : own_most;
    uint64_t fit = kHalfGroups / own_fill;
    s.g.own_splits = between(own_want, 1, fit < kMostOwn ? fit : kMostOwn);
    s.g.own_least = between((own_tiles + s.g.own_splits - 1) / s.g.own_splits, 1, 0x7fffffff);
    // shared tokens: one workgroup a compute unit, those for own tokens counted unless they are short, as two on one wait for each other's loads (48
    // sequences behind 4001 tokens, 96 workgroups for own tokens: 8, 10, 12, 24 pieces of the shared ones, 16 workgroups each, 31, 29, 35, 37 us); where that
    // leaves more than 16 tiles to a workgroup, two (64 behind 32768, 256 workgroups for own tokens: 8, 12, 16, 20, 32 pieces 151, 109, 94, 112, 107 us;
    // without own tokens 147, 105, 84, 91, 72).  Short are 3 tiles and less; 3 and 7, with up to 280 tokens of their own: 16 sequences behind 8192 24 and 31 us,
    // 48 behind 4001 27 and 31, 64 behind 2048 23 and 30, behind 8192 43 and 37, in fp32 29 and 42, behind 32768 198 and 135; over 296 such calls 3 is 2 % ahead
    const uint64_t slots = cus * (entro_cache_width(c->head_dim) > 128 || (s.many && q->type == ENTRO_F32) ? 1 : 2);
    const uint64_t own_blocks = own_fill * s.g.own_splits, fill = units * s.g.row_tiles;
    const auto leaves = [&](uint64_t room) { return own_blocks < room && own_tiles > 3 ? room - own_blocks : room; };
    uint64_t want = leaves(cus) / fill;
    if (want * 16 < tiles) want = leaves(slots) / fill;
    if (want < 2) want = (tiles + 23) / 24;                    // several rounds: none of them long
    const uint64_t can = s.many ? tiles / 2 : tiles / 8;
    fit = kHalfGroups / fill;
    s.g.splits = between(want < can ? want : can, 1, fit < kMostShared ? fit : kMostShared);
    s.g.least = between((tiles + s.g.splits - 1) / s.g.splits, 1, 0x7fffffff);
    s.g.blocks = static_cast<uint32_t>(fill * s.g.splits);
    s.bytes = uint64_t{q->tokens} * q->q_heads * (s.g.splits + s.g.own_splits) * (entro_cache_width(c->head_dim) + 1) * 4;
    return s;
}

template <int W, typename T>
void launch_shared(const Pool &p, const Query &a, const SharedShape &s, hipStream_t st) {
    const uint32_t units = p.seqs * p.kv_heads * s.g.own_splits, own = s.g.own_tiles ? units * s.g.own_tiles : (units + 3) / 4;
    const dim3 grid(s.g.blocks + own);
    if (s.many)
        hipLaunchKernelGGL((k_attend_shared<W, T, true>), grid, dim3(kWG), 0, st, p, a, s.g);
    else
        hipLaunchKernelGGL((k_attend_shared<W, T, false>), grid, dim3(kWG), 0, st, p, a, s.g);
    hipLaunchKernelGGL((k_shared_join<W, T>), dim3(between((uint64_t{a.tokens} * a.q_heads + kWG / 64 - 1) / (kWG / 64), 1, kMostGroups)),
                       dim3(kWG), 0, st, p, a);
}

template <typename T>
void launch_shared_width(const Pool &p, const Query &a, const SharedShape &s, hipStream_t st) {
    switch (p.width) {
        case 64: return launch_shared<64, T>(p, a, s, st);
        case 96: return launch_shared<96, T>(p, a, s, st);
        case 128: return launch_shared<128, T>(p, a, s, st);
        case 192: return launch_shared<192, T>(p, a, s, st);
        case 256: return launch_shared<256, T>(p, a, s, st);
    }
}

bool launchable(const entro_cache *c, const entro_cache_table *t, const entro_cache_query *q, const entro_cache_groups *g) {
    return uint64_t{g->groups} * c->kv_heads <= kHalfGroups && uint64_t{t->seqs} * c->kv_heads <= kHalfGroups && uint64_t{q->tokens} * q->q_heads <= 0x7fffffffull;
}

}  // namespace

extern "C" {

entro_status entro_cache_shared(const entro_cache *c, const entro_cache_table *t, const entro_cache_groups *g, void *hip_stream) {
    if (const entro_status s = check_cache(c)) return s;
    if (const entro_status s = check_table(t)) return s;
    if (const entro_status s = check_groups(g)) return s;
    const Pool p = pool_of(c, t, 0);
    const dim3 grid(g->groups < 65536 ? g->groups : 65536);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (t->stride <= kShortTable) {
        hipLaunchKernelGGL(k_shared<false>, grid, dim3(kWG), 0, st, p, g->first, g->shared, g->groups);
    } else {
        const uint32_t pieces = (t->stride + 63) / 64;
        const uint64_t all = uint64_t{g->groups} * pieces;
        hipLaunchKernelGGL(k_shared<true>, grid, dim3(kWG), 0, st, p, g->first, g->shared, g->groups);
        hipLaunchKernelGGL(k_shared_pieces, dim3(static_cast<uint32_t>(all < 65536 ? all : 65536)), dim3(kWG), 0, st, p, g->first, g->shared, g->groups, pieces);
    }
    return hip_ok(hipGetLastError(), "entro_cache_shared") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

uint64_t entro_cache_attend_shared_workspace_bytes(const entro_cache *c, const entro_cache_table *t, const entro_cache_query *q,
                                                   const entro_cache_groups *g) {
    if (check_sizes(c) != ENTRO_OK || check_table_sizes(t) != ENTRO_OK || check_query_sizes(c, q) != ENTRO_OK || check_groups_sizes(g) != ENTRO_OK) return 0;
    return launchable(c, t, q, g) ? shared_shape_of(c, t, q, g).bytes : 0;
}

entro_status entro_cache_attend_shared(const entro_cache *c, const entro_cache_table *t, const entro_cache_query *q, const entro_cache_groups *g,
                                       void *workspace, uint64_t workspace_bytes, void *hip_stream) {
    if (const entro_status s = check_cache(c)) return s;
    if (const entro_status s = check_table(t)) return s;
    if (const entro_status s = check_query(c, q)) return s;
    if (const entro_status s = check_groups(g)) return s;
    if (q->tokens == 0) return ENTRO_OK;
    if (!launchable(c, t, q, g)) return ENTRO_ERR_SIZE;
    SharedShape shape = shared_shape_of(c, t, q, g);
    if (!workspace) return ENTRO_ERR_NULL;
    if (!aligned16(workspace)) return ENTRO_ERR_ALIGN;
    if (workspace_bytes < shape.bytes) return ENTRO_ERR_CAPACITY;
    shape.g.first = g->first;
    shape.g.shared = g->shared;
    const Pool p = pool_of(c, t, q->layer);
    const bool aligned = ((q->q_token_stride | q->q_head_stride) & 7u) == 0;
    const uint32_t parts = shape.g.splits + shape.g.own_splits;
    float *part_o = static_cast<float *>(workspace), *part_lse = part_o + uint64_t{q->tokens} * q->q_heads * parts * p.width;
    const Query a = {q->q, q->out, q->lse, q->q_token_stride, q->q_head_stride, q->out_token_stride, q->out_head_stride, q->start,
                     q->tokens, q->q_heads, q->q_heads / c->kv_heads, q->window, q->sinks, q->scale, aligned, parts, 1, part_o, part_lse};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (q->type == ENTRO_F32)
        launch_shared_width<float>(p, a, shape, st);
    else
        launch_shared_width<uint16_t>(p, a, shape, st);
    return hip_ok(hipGetLastError(), "entro_cache_attend_shared") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

}  // extern "C"

namespace {

entro_status check_query_sizes(const entro_cache *c, const entro_cache_query *q) {
    if (!q) return ENTRO_ERR_NULL;
    if (q->type != ENTRO_F32 && q->type != ENTRO_BF16) return ENTRO_ERR_SCHEME;
    if (q->layer >= c->layers || q->tokens > 0x7fffffffu || q->q_heads == 0 || q->q_heads > 65536 || q->q_heads % c->kv_heads) return ENTRO_ERR_SIZE;
    return ENTRO_OK;
}

entro_status check_query(const entro_cache *c, const entro_cache_query *q) {
    if (const entro_status s = check_query_sizes(c, q)) return s;
    if (!q->start || (q->tokens && (!q->q || !q->out))) return ENTRO_ERR_NULL;
    if (q->q_token_stride > kMaxStride || q->q_head_stride > kMaxStride || q->out_token_stride > kMaxStride || q->out_head_stride > kMaxStride)
        return ENTRO_ERR_SIZE;
    if (!(q->scale > -3.0e38f && q->scale < 3.0e38f)) return ENTRO_ERR_RANGE;
    if (!aligned16(q->q) || !aligned16(q->out) || !aligned16(q->lse) || !aligned16(q->start)) return ENTRO_ERR_ALIGN;
    return ENTRO_OK;
}

struct Shape {
    bool many;                     // the kernel for many rows
    uint32_t row_tiles, splits, least, join_rows;
    uint64_t bytes;
};

int compute_units() {
    int device = 0, cus = 0;
    if (hipGetDevice(&device) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess) return 256;
    return cus > 0 ? cus : 256;
}

// Sequences and key heads of k_attend_few's grid, which takes eight sequences at a time.
uint64_t units_of(uint32_t seqs, uint32_t kv_heads) { return (seqs < 8 ? seqs : (uint64_t{seqs} + 7) / 8 * 8) * kv_heads; }

// How far a call's tiles are split: as many workgroups as fill the chip, tiles of a workgroup not fewer than pay for the
// join, which is a launch of its own. A sequence has no more new tokens than there are rows, whatever the hint says, and the
// kernels' own loops cover what a grid of kMostGroups does not.
Shape shape_of(const entro_cache *c, const entro_cache_table *t, const entro_cache_query *q) {
    const uint32_t max_new = q->max_new < q->tokens ? q->max_new : q->tokens;
    Shape s = {false, 1, 1, 1, max_new < 1 ? 1 : max_new > 65535 ? 65535 : max_new, 0};
    const uint32_t width = entro_cache_width(c->head_dim);
    const uint64_t rows = uint64_t{max_new} * (q->q_heads / c->kv_heads);
    uint64_t len = q->max_len;
    if (q->window && len > uint64_t{q->window} + q->sinks + max_new + 2 * kTile) len = uint64_t{q->window} + q->sinks + max_new + 2 * kTile;
    const uint64_t tiles = (len + kTile - 1) / kTile, units = uint64_t{t->seqs} * c->kv_heads;
    uint64_t groups = units;
    // up to 32 rows in groups of 16, one after the other. 32 rows over 4096 tokens of 64 sequences, by the kernel for few and by that for many:
    // 89 and 115 us for 64 dimensions, 179 and 191 for 128; in fp32 98 and 269, 186 and 404. Of 8 sequences (128 dimensions): 20 rows 41 and 40, 32 rows 44 and
    // 40, 48 rows 65 and 47, 64 rows 83 and 51; in fp32 32 rows 46 and 74.
    if (rows > 32) {
        s.many = true;
        const uint64_t row_tiles = (rows + kManyRows - 1) / kManyRows, most = kMostGroups / units;
        s.row_tiles = static_cast<uint32_t>(row_tiles < most ? row_tiles : (most ? most : 1));
        groups *= s.row_tiles;
    }
    const uint64_t cus = static_cast<uint64_t>(compute_units());
    uint64_t want, can;
    if (!s.many && units * 4 > cus * 2) {
        // the heads of many sequences fill the chip; pieces of at most 96 tiles keep one long sequence from being the last
        // alone. One piece, pieces of 96 tiles, of 48: 32768 tokens beside 63 sequences of 512 tokens 272, 70, 56 us, beside 63 of 4096 307, 134, 138;
        // 64 sequences of up to 8192 tokens 130, 128, 132, all of 8192 171, 180, 185 (which one piece would suit)
        want = can = (tiles + 95) / 96;
    } else if (!s.many) {
        // two workgroups a compute unit are enough (131072 tokens, 8 heads: 64 pieces 55 us, 128 pieces 60 us); below 24 tiles the
        // join costs as much as it gives (8 heads, in one piece and in two or three: 16 tiles 14.4 and 15.6 us, 20 tiles 16.0 and 16.9, 23 tiles 18.8 and
        // 17.4, 24 tiles 19.4 and 15.9, 32 tiles 23.4 and 16.1)
        want = cus * 2 / units;
        can = tiles < 24 ? 1 : tiles / 8;
    } else {
        // two workgroups a compute unit (64 tokens of 32 heads over 8192: 46 us; 1024 over 16384 463 us)
        want = (cus * 2 + groups - 1) / groups;
        can = tiles / 8;
    }
    s.splits = static_cast<uint32_t>(want < can ? want : can);
    const uint64_t fit = uint64_t{t->seqs} * q->q_heads > kMostGroups ? 1 : kMostGroups / (units_of(t->seqs, c->kv_heads) * s.row_tiles);
    if (s.splits > (s.many ? 64 : kMostSplits)) s.splits = s.many ? 64 : kMostSplits;
    if (s.splits > fit) s.splits = static_cast<uint32_t>(fit);
    if (s.splits < 1) s.splits = 1;
    if (tiles) s.least = static_cast<uint32_t>((tiles + s.splits - 1) / s.splits);
    if (s.splits > 1) s.bytes = uint64_t{q->tokens} * q->q_heads * s.splits * (width + 1) * 4;
    return s;
}

template <int W, typename T>
void launch_width(const Pool &p, const Query &a, const Shape &s, hipStream_t st) {
    if (!s.many)
        hipLaunchKernelGGL((k_attend_few<W, T>), dim3(static_cast<uint32_t>(units_of(p.seqs, p.kv_heads)) * a.splits), dim3(kWG), 0, st, p, a);
    else
        hipLaunchKernelGGL((k_attend_many<W, T>), dim3(p.seqs * p.kv_heads * a.splits * s.row_tiles), dim3(kWG), 0, st, p, a, s.row_tiles);
    if (a.splits > 1) {
        if (s.many)
            hipLaunchKernelGGL((k_attend_join_rows<W, T>), dim3((p.seqs * a.q_heads + kWG / 64 - 1) / (kWG / 64), s.join_rows), dim3(kWG), 0, st, p, a);
        else
            hipLaunchKernelGGL((k_attend_join<W, T>), dim3(p.seqs * a.q_heads, s.join_rows), dim3(kWG), 0, st, p, a);
    }
}

template <typename T>
void launch(const Pool &p, const Query &a, const Shape &s, hipStream_t st) {
    switch (p.width) {
        case 64: return launch_width<64, T>(p, a, s, st);
        case 96: return launch_width<96, T>(p, a, s, st);
        case 128: return launch_width<128, T>(p, a, s, st);
        case 192: return launch_width<192, T>(p, a, s, st);
        case 256: return launch_width<256, T>(p, a, s, st);
    }
}

}  // namespace

extern "C" {

uint64_t entro_cache_attend_workspace_bytes(const entro_cache *c, const entro_cache_table *t, const entro_cache_query *q) {
    if (check_sizes(c) != ENTRO_OK || check_table_sizes(t) != ENTRO_OK || check_query_sizes(c, q) != ENTRO_OK) return 0;
    return shape_of(c, t, q).bytes;
}

entro_status entro_cache_attend(const entro_cache *c, const entro_cache_table *t, const entro_cache_query *q, void *workspace,
                                uint64_t workspace_bytes, void *hip_stream) {
    if (const entro_status s = check_cache(c)) return s;
    if (const entro_status s = check_table(t)) return s;
    if (const entro_status s = check_query(c, q)) return s;
    if (q->tokens == 0) return ENTRO_OK;
    if (units_of(t->seqs, c->kv_heads) > kMostGroups || uint64_t{q->tokens} * q->q_heads > 0x7fffffffull) return ENTRO_ERR_SIZE;
    const Shape shape = shape_of(c, t, q);
    if (shape.bytes) {
        if (!workspace) return ENTRO_ERR_NULL;
        if (!aligned16(workspace)) return ENTRO_ERR_ALIGN;
        if (workspace_bytes < shape.bytes) return ENTRO_ERR_CAPACITY;
    }
    const Pool p = pool_of(c, t, q->layer);
    const bool aligned = ((q->q_token_stride | q->q_head_stride) & 7u) == 0;
    float *part_o = static_cast<float *>(workspace), *part_lse = part_o + uint64_t{q->tokens} * q->q_heads * shape.splits * p.width;
    const Query a = {q->q, q->out, q->lse, q->q_token_stride, q->q_head_stride, q->out_token_stride, q->out_head_stride, q->start,
                     q->tokens, q->q_heads, q->q_heads / c->kv_heads, q->window, q->sinks, q->scale, aligned, shape.splits, shape.least,
                     part_o, part_lse};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (q->type == ENTRO_F32)
        launch<float>(p, a, shape, st);
    else
        launch<uint16_t>(p, a, shape, st);
    return hip_ok(hipGetLastError(), "entro_cache_attend") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

}  // extern "C"
