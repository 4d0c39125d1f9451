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

// How the tiles of a group of rows are shared out to at most `splits` workgroups.
__device__ inline int32_t tiles_per_split(const Query &a, int32_t count) {
    return max((count + static_cast<int32_t>(a.splits) - 1) / static_cast<int32_t>(a.splits), static_cast<int32_t>(a.least));
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
template <int W, typename T>
__global__ __launch_bounds__(kWG, W > 128 ? 1 : 2) void k_attend_few(Pool p, Query a) {
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3;         // bf16 numbers that make an element of q in the first product
    constexpr int kWeights = sizeof(T) == 2 ? 2 : 3;       // bf16 numbers that make a weight of the second
    constexpr int kFull = W / 64, kRest = W % 64 ? 1 : 0;   // loads of 64 dimensions of 16 tokens, and of 32
    constexpr int kDims = W / 16;
    __shared__ float merge_o[4][16][W + 4];
    __shared__ float merge_m[4][16], merge_l[4][16];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15u;
    // Workgroups go to the XCDs in turn. Those of one XCD take the key heads of the same sequence and split, whose codes lie side by side, and
    // the splits of a sequence go to different XCDs, so that long sequences do not meet on one.
    const uint32_t r = p.seqs < 8 ? blockIdx.x : blockIdx.x / 8, head = r % p.kv_heads, split = r / p.kv_heads % a.splits, block = r / p.kv_heads / a.splits;
    const uint32_t b = p.seqs < 8 ? block : 8 * block + ((blockIdx.x - split) & 7u);
    if (b >= p.seqs) return;
    const Span s = span_of(a.start, p.lengths, b, a.tokens);
    const uint64_t page_bytes = uint64_t{W} << p.page_shift, page_stride = page_bytes * p.kv_heads;
    const uint8_t *k_head = p.k + head * page_bytes, *v_head = p.v + head * page_bytes;
    const float *ks_head = p.k_scale + head, *vs_head = p.v_scale + head;
    const uint32_t in_page = (1u << p.page_shift) - 1;
    const int64_t rows = int64_t{s.count} * a.group;
    for (int64_t row0 = 0; row0 < rows; row0 += 16) {
        const int32_t first = s.pos + static_cast<int32_t>(row0 / a.group);
        const int32_t last = s.pos + static_cast<int32_t>(min(row0 + 15, rows - 1) / a.group);
        const Tiles tiles = tiles_of(p, a, first, last);
        const int32_t per = tiles_per_split(a, tiles.count), begin = static_cast<int32_t>(split) * per, end = min(begin + per, tiles.count);
        if (begin >= end && split > 0) continue;
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
    const int32_t i0 = begin + static_cast<int32_t>(wave);
    // the lane's row
    const int64_t my_row = row0 + c;
    const bool mine = my_row < rows;
    const uint32_t my_token = static_cast<uint32_t>(s.row) + static_cast<uint32_t>((mine ? my_row : row0) / a.group);
    const uint32_t my_head = head * a.group + static_cast<uint32_t>((mine ? my_row : row0) % a.group);
    const int32_t my_pos = s.pos + static_cast<int32_t>(my_token) - s.row;
    
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
            ask_pages(i0 + 4);
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

    for (int32_t i = i0; i < end; i += 4) {
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
        take_pages(i + 4);
        ask_pages(i + 8);
        ask_keys(i + 4);
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
        bf16x8 w[2][kWeights];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float e = __builtin_amdgcn_exp2f(fmaf(z[2 * h + j / 4][j & 3], factor, -base));
                l += e;
                x[j] = e * scale;
            }
            split_factors<kWeights>(x, w[h]);
        }
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
            const bf16x8 v0 = eight_values(vc[d][0], vc[d][1]), v1 = eight_values(vc[d][2], vc[d][3]);
#pragma unroll
            for (int n = 0; n < kWeights; ++n) {
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, w[0][n], o[d], 0, 0, 0);
                o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, w[1][n], o[d], 0, 0, 0);
            }
        }
        ask_values(i + 4);
    }
        l = column_sum(l);
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
                if (a.splits == 1)
                    store_as(static_cast<T *>(a.out) + token * a.out_token_stride + q_head * a.out_head_stride + d, x);
                else
                    a.part_o[(at * a.splits + split) * W + d] = x;
            }
            if (d0 == 0) {
                if (a.splits > 1) a.part_lse[at * a.splits + split] = lse;
                else if (a.lse) a.lse[at] = lse * kLn2;
            }
        }
    }
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
// 162 for fp32 and 30 for bf16, at 192 35 for fp32, at 96 and 128 2 and 5 for bf16.
template <int W, typename T>
__global__ __launch_bounds__(kWG, sizeof(T) == 2 && W <= 128 ? 2 : 1) void k_attend_many(Pool p, Query a, uint32_t row_tiles) {
    constexpr int kThreads = kWG, kRows = kManyRows;
    constexpr int kParts = sizeof(T) == 2 ? 1 : 3, kWeights = sizeof(T) == 2 ? 2 : 3;
    constexpr int kChunks = (W * 4 + kThreads - 1) / kThreads;      // pieces of 16 codes a thread turns, of keys and of values
    constexpr int kKeyRow = 2 * W + 16, kValueRow = 2 * kTile + 16;   // bytes
    constexpr int kKeyTile = kTile * kKeyRow, kValueTile = W * kValueRow;
    __shared__ __attribute__((aligned(16))) uint8_t key_lds[2][kKeyTile], value_lds[2][kValueTile];
    __shared__ f32x4 tile_ks[2], tile_vs[2];
    __shared__ int32_t tile_ok[2][4];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, c = lane & 31u;
    // workgroups of one key head follow each other at multiples of the number of heads: with 8 heads, on one XCD and its L2
    const uint32_t units = p.seqs * p.kv_heads, unit = blockIdx.x % units, head = unit % p.kv_heads, b = unit / p.kv_heads;
    const uint32_t split = blockIdx.x / units % a.splits, tile_from_end = blockIdx.x / units / a.splits;
    const Span s = span_of(a.start, p.lengths, b, a.tokens);
    const uint64_t page_bytes = uint64_t{W} << p.page_shift, page_stride = page_bytes * p.kv_heads;
    const uint8_t *k_head = p.k + head * page_bytes, *v_head = p.v + head * page_bytes;
    const uint32_t in_page = (1u << p.page_shift) - 1;
    const int64_t rows = int64_t{s.count} * a.group;
    const int64_t groups = (rows + kRows - 1) / kRows;
    // the last rows see the most tokens: they come first
    for (int64_t group = groups - 1 - tile_from_end; group >= 0; group -= row_tiles) {
        const int64_t row0 = group * kRows;
        const int32_t first = s.pos + static_cast<int32_t>(row0 / a.group);
        const int32_t last = s.pos + static_cast<int32_t>(min(row0 + kRows - 1, rows - 1) / a.group);
        const Tiles tiles = tiles_of(p, a, first, last);
        const int32_t per = tiles_per_split(a, tiles.count), begin = static_cast<int32_t>(split) * per, end = min(begin + per, tiles.count);
        if (begin >= end && split > 0) continue;
        const int64_t my_row = row0 + 32 * wave + c;
        const bool mine = my_row < rows;
        const uint32_t my_token = static_cast<uint32_t>(s.row) + static_cast<uint32_t>((mine ? my_row : row0) / a.group);
        const uint32_t my_head = head * a.group + static_cast<uint32_t>((mine ? my_row : row0) % a.group);
        const int32_t my_pos = mine ? s.pos + static_cast<int32_t>(my_token) - s.row : -1;
        // positions of the wavefront's rows
        const int64_t wave_row = row0 + 32 * wave;
        const int32_t wave_first = s.pos + static_cast<int32_t>(wave_row / a.group);
        const int32_t wave_last = wave_row < rows ? s.pos + static_cast<int32_t>(min(wave_row + 31, rows - 1) / a.group) : -1;
        bf16x8 q[W / 16][kParts];
        float q_factor;
        {
            const T *row = static_cast<const T *>(a.q) + my_token * a.q_token_stride + my_head * a.q_head_stride;
            float most = 0.0f;
#pragma unroll
            for (int f = 0; f < W / 16; ++f) {
                float x[8];
                load_eight(row, 16 * f + 8 * h, p.head_dim, a.aligned, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));
            }
            const int e = exponent_of(fmaxf(most, __shfl_xor(most, 32)));
            const float sign = a.scale < 0.0f ? -1.0f : 1.0f;
#pragma unroll
            for (int f = 0; f < W / 16; ++f) {
                float x[8];
                load_eight(row, 16 * f + 8 * h, p.head_dim, a.aligned, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = ldexpf(x[i] * sign, -e);
                split_factors<kParts>(x, q[f]);
            }
            q_factor = ldexpf(fabsf(a.scale) * kLog2e, e);
        }
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
            to_lds(0);
            ask_codes(begin + 1);
            ask_pages(begin + 2);
        }
        __syncthreads();

        // What the matrix units take from LDS is asked for kAhead pieces before it is used.
        constexpr int kAhead = 4;
        // the second product: weights of four times 16 tokens
        const auto add_values = [&](const bf16x8 (*w)[kWeights], int half) {
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
                for (int n = 0; n < kWeights; ++n) o[i % kDims] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(now, w[i / kDims][n], o[i % kDims], 0, 0, 0);
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
#pragma unroll
                for (int j = 0; j < W / 8; ++j) {
                    const bf16x8 now = k[j % kAhead];
                    if (j + kAhead < W / 8) k[j % kAhead] = piece(j + kAhead);
#pragma unroll
                    for (int n = 0; n < kParts; ++n) z[j & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(now, q[j >> 1][n], z[j & 1], 0, 0, 0);
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
                bf16x8 w[4][kWeights];
#pragma unroll
                for (int g = 0; g < 4; ++g) {       // 16 tokens
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float e = __builtin_amdgcn_exp2f(fmaf(z[g / 2][8 * (g & 1) + j], kf[g], -base));
                        l += e;
                        x[j] = e * vf[g];
                    }
                    split_factors<kWeights>(x, w[g]);
                }
                add_values(w, half);
            }
            __syncthreads();
        }
        l += __shfl_xor(l, 32);
        if (mine) {
            const float inv = l > 0.0f ? 1.0f / l : 0.0f, base = m == -INFINITY ? 0.0f : m;
            const float lse = l > 0.0f ? base + __builtin_amdgcn_logf(l * kUnit) : l == l ? -INFINITY : l;
            const uint64_t at = uint64_t{my_token} * a.q_heads + my_head;
            T *out = static_cast<T *>(a.out) + my_token * a.out_token_stride + my_head * a.out_head_stride;
            float *part = a.part_o + (at * a.splits + split) * W;
#pragma unroll
            for (int d = 0; d < kDims; ++d)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const uint32_t dim = 32 * d + 8 * (j / 4) + 4 * h + (j & 3);
                    const float x = l == l ? o[d][j] * inv : l;
                    if (a.splits > 1) part[dim] = x;
                    else if (dim < p.head_dim) store_as(out + dim, x);
                }
            if (h == 0) {
                if (a.splits > 1) a.part_lse[at * a.splits + split] = lse;
                else if (a.lse) a.lse[at] = lse * kLn2;
            }
        }
    }
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
