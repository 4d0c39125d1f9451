// Norms and rotations of heads on the GPU, on their own and on the way into the token cache (include/entro.h has the definitions).
#include "entro_cache.h"

#include <cmath>
#include <type_traits>

namespace {

using namespace entro_detail;

constexpr int kWG = 256;
// Heads that a lane group takes one after the other in large calls, with the angles of its position found once: 8192 rows of 40 heads of 128 in bf16,
// four heads 41 us, eight 38.  In fp32 four, and only where a quarter and more of the lanes of a head have no elements: what they ask for at a time is less
// (one head and four, memory not read before: 24 heads of 80, 5000 rows 25.2 and 22.1 us, 16 000 69.4 and 59.2, with a norm 31.7 and 29.1, 91.0 and 82.0; 28 of
// 96, 8000 rows 44.8 and 42.0; 40 of 72 58.0 and 48.1; all lanes at work: 40 of 128, 5000 rows 41.1 and 44.8, 16 000 116.6 and 123.1, with a norm 46.9 and 49.6, 137
// and 129; 28 of 112, 8000 rows 47.3 and 49.0).
template <typename T> constexpr uint32_t kHeads = sizeof(T) == 2 ? 8 : 4;
// A call is large from so many lanes on (one head a lane group and several: 40 heads of 128 in bf16 with a norm, 1600 rows 14.1 and 15.6 us, 3000 23.1 and
// 21.2, 8000 52.3 and 44.5; without 12.5 and 10.6, 20.0 and 14.9, 44.4 and 30.4; 40 heads of 96 with a norm 15.0 and 19.5, 25.1 and 25.2, 57.9 and 55.6; in fp32 24 heads of 80, 3000 rows, 64 * 4500 lanes, 16.2 and 17.3),
template <typename T> constexpr uint64_t kManyLanes = sizeof(T) == 2 ? 64 * 2560 : 64 * 6144;
// and from so many on the queries of rows for the cache have a launch of their own (32 query and 8 key heads of 128 in bf16, written and read, one launch and
// two: 3200 rows 42.5 and 45 us, 6400 76 and 78, 12 800 160 and 131; written alone in fp32, 4000 rows 39.7 and 41.1, 5600 53.0 and 52.1, 12 000 130.7 and
// 115.4, of 24 and 4 heads of 96 32.4 and 34.5, 42.6 and 40.8, 92.6 and 72.1).
template <typename T> constexpr uint64_t kApartLanes = sizeof(T) == 2 ? 64 * 8192 : 64 * 32768;
constexpr float kLeastEps = 1.2e-38f;

struct Turning {
    const uint64_t *turns;
    uint32_t half, head_dim, norm;       // half: pairs
    uint32_t shift;                      // 2^shift lanes to a head
    float eps, amplitude, inverse_dim;
};

// Rows of q or k.
struct Side {
    const void *x;
    void *y;
    uint64_t x_token_stride, x_head_stride, y_token_stride, y_head_stride;
    const float *gain;
    uint32_t gain_stride, heads;
    bool wide, gain_wide;                // rows, gains begin at multiples of four elements
};

// A lane has two runs of four elements of a head: of the turned dimensions the first and the second halves of its pairs (halves), or
// its pairs one after the other (pairs); of the others eight elements as they lie.  So rows are read and written in whole pieces,
// and both elements of a pair are in one lane.  (Runs of eight bf16 elements, half as many lanes with up to 248 registers: a row
// of each of 64 sequences into the cache 14.6 us instead of 10.9, 26 800 rows 92 instead of 85.)
constexpr uint32_t kRun = 4;

template <typename T> using Word = std::conditional_t<sizeof(T) == 2, u32x2, u32x4>;       // a run

struct Piece {
    uint32_t at[2], count[2];            // first element of a run, and how many there are
    uint32_t pair;                       // the first of its pairs
    bool turned;
};

template <bool kPairs>
__device__ inline Piece piece_of(const Turning &r, uint32_t unit) {
    constexpr uint32_t P = kRun;
    const uint32_t turned = (r.half + P - 1) / P;
    Piece c;
    c.turned = unit < turned;
    c.pair = unit * P;
    if (c.turned && !kPairs) {
        c.at[0] = c.pair;
        c.at[1] = r.half + c.pair;
        c.count[0] = c.count[1] = min(P, r.half - c.pair);
        return c;
    }
    const uint32_t begin = c.turned ? 2 * c.pair : 2 * r.half + (unit - turned) * 2 * P, end = c.turned ? 2 * r.half : r.head_dim;
    const uint32_t all = begin < end ? min(2 * P, end - begin) : 0u;
    c.at[0] = begin;
    c.at[1] = begin + P;
    c.count[0] = min(P, all);
    c.count[1] = all - c.count[0];
    return c;
}

// The two runs of a head as they lie in memory.
template <typename T>
struct Raw {
    Word<T> w[2];
};

template <typename T>
__device__ inline Raw<T> ask_head(const T *row, const Piece &c, bool wide) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        r.w[i] = Word<T>{};
        if (wide && c.count[i] == kRun && c.at[i] % kRun == 0) {
            r.w[i] = *reinterpret_cast<const Word<T> *>(row + c.at[i]);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < kRun; ++j)
                if (j < c.count[i]) {
                    const T e = row[c.at[i] + j];
                    if constexpr (sizeof(T) == 2) r.w[i][j / 2] |= static_cast<uint32_t>(e) << (16 * (j & 1));
                    else r.w[i][j] = __float_as_uint(e);
                }
        }
    }
    return r;
}

template <typename T>
__device__ inline void head_values(const Raw<T> &r, float *x) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (uint32_t j = 0; j < kRun; ++j) {
            if constexpr (sizeof(T) == 4) x[i * kRun + j] = __uint_as_float(r.w[i][j]);
            else x[i * kRun + j] = __uint_as_float(j & 1 ? r.w[i][j / 2] & 0xffff0000u : r.w[i][j / 2] << 16);
        }
}

// Two numbers rounded to nearest even, in one instruction; NaNs stay NaNs.
__device__ inline uint32_t two_bf16(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}

template <typename T>
__device__ inline void write_head(T *row, const Piece &c, bool wide, const float *x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (wide && c.count[i] == kRun && c.at[i] % kRun == 0) {
            const float *y = x + i * kRun;
            if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4 *>(row + c.at[i]) = f32x4{y[0], y[1], y[2], y[3]};
            else *reinterpret_cast<u32x2 *>(row + c.at[i]) = u32x2{two_bf16(y[0], y[1]), two_bf16(y[2], y[3])};
        } else {
#pragma unroll
            for (uint32_t j = 0; j < kRun; ++j)
                if (j < c.count[i]) row[c.at[i] + j] = store_from_f32<T>(x[i * kRun + j]);
        }
    }
}

// Cosine and sine of 2 pi * position * turns / 2^64.  The product modulo 2^64 is the angle in turns, whatever the position; its upper 32 bits
// are kept (2^-32 turns).  Within an eighth of a turn either side of a quarter their Taylor series: what is left out is below 2^-28.
__device__ inline void turn_of(int32_t position, uint64_t turns, float amplitude, float *cosine, float *sine) {
    const uint32_t p = static_cast<uint32_t>(position), lo = static_cast<uint32_t>(turns), hi = static_cast<uint32_t>(turns >> 32);
    const uint32_t phase = __umulhi(p, lo) + p * hi - (position < 0 ? lo : 0u);
    const uint32_t quarter = (phase + 0x20000000u) >> 30;
    const float x = static_cast<float>(static_cast<int32_t>(phase - (quarter << 30))) * 1.46291807926715968e-9f;      // 2 pi / 2^32
    const float xx = x * x;
    const float odd = fmaf(fmaf(fmaf(fmaf(1.0f / 362880, xx, -1.0f / 5040), xx, 1.0f / 120), xx, -1.0f / 6) * xx, x, x);
    const float even = fmaf(fmaf(fmaf(fmaf(fmaf(-1.0f / 3628800, xx, 1.0f / 40320), xx, -1.0f / 720), xx, 1.0f / 24), xx, -0.5f), xx, 1.0f);
    const float c = quarter & 1 ? odd : even, s = quarter & 1 ? even : odd;
    *cosine = amplitude * ((quarter + 1) & 2 ? -c : c);
    *sine = amplitude * (quarter & 2 ? -s : s);
}

__device__ inline void turns_of(const Turning &r, const Piece &c, int32_t position, float *cosine, float *sine) {
    constexpr uint32_t P = kRun;
    if (!c.turned) return;
    uint64_t turns[P];
    if (c.pair + P <= r.half) {
#pragma unroll
        for (uint32_t j = 0; j < P; ++j) turns[j] = r.turns[c.pair + j];
    } else {
#pragma unroll
        for (uint32_t j = 0; j < P; ++j) turns[j] = r.turns[min(c.pair + j, r.half - 1)];
    }
#pragma unroll
    for (uint32_t j = 0; j < P; ++j) turn_of(position, turns[j], r.amplitude, cosine + j, sine + j);
}

// A number of a lane that holds another part of the same head: of the one 1, 2 or 16 away, or of one in the other half of 8 or 16 lanes, whose halves
// have by then the same number in all their lanes.
template <int STEP>
__device__ inline float other_part(float v) {
    constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140;      // patterns of lane moves
    if constexpr (STEP >= 16) return __shfl_xor(v, STEP);
    else return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), STEP == 1 ? kSwap1 : STEP == 2 ? kSwap2 : STEP == 4 ? kHalfMirror : kMirror, 0xf, 0xf, true));
}

// N numbers, each brought together over the lanes of a head by f.
template <int N, typename F>
__device__ inline void over_head(float (&v)[N], uint32_t shift, F f) {
    const auto step = [&](auto far) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = f(v[i], other_part<decltype(far)::value>(v[i]));
    };
    if (shift > 0) step(std::integral_constant<int, 1>{});
    if (shift > 1) step(std::integral_constant<int, 2>{});
    if (shift > 2) step(std::integral_constant<int, 4>{});
    if (shift > 3) step(std::integral_constant<int, 8>{});
    if (shift > 4) step(std::integral_constant<int, 16>{});
    if (shift > 5) step(std::integral_constant<int, 32>{});
}

// The norm of a head, whose elements are x and, as they were read, raw.  All lanes are here.  Where the squares of some head of the wavefront leave the
// range, all is done again, for those heads on elements less the exponent of the largest one.
template <typename T>
__device__ inline void norm_head(const Turning &r, const Piece &c, const float *gain, bool gain_wide, const Raw<T> &raw, float *x) {
    constexpr uint32_t P = kRun, N = 2 * P;
    const auto here = [&](uint32_t j) { return j % P < c.count[j / P]; };
    const auto add = [](float a, float b) { return a + b; };
    const auto squares = [&]() {
        const auto less = [&](float sum) {
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) x[j] = here(j) ? fmaf(-sum, r.inverse_dim, x[j]) : 0.0f;
        };
        if (r.norm == ENTRO_NORM_CENTRED) {
            float sum[1] = {0.0f};
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) sum[0] += x[j];
            over_head(sum, r.shift, add);
            less(sum[0]);
        }
        float sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) sums[0] = fmaf(x[j], x[j], sums[0]);
        if (r.norm != ENTRO_NORM_CENTRED) {
            float sum[1] = {sums[0]};
            over_head(sum, r.shift, add);
            return sum[0];
        }
        // Sum and inverse are rounded: of a mean that is large beside the elements' spread some is left.  It goes in the same pass as the squares.
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) sums[1] += x[j];
        over_head(sums, r.shift, add);
        less(sums[1]);
        const float sum = fmaf(-sums[1] * r.inverse_dim, sums[1], sums[0]);
        return sum < 0.0f ? 0.0f : sum;
    };
    float sum = squares(), eps = r.eps;
    if (__any(!(sum < INFINITY))) {
        head_values<T>(raw, x);
        float most[1] = {0.0f};
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) most[0] = fmaxf(most[0], fabsf(x[j]));
        over_head(most, r.shift, [](float a, float b) { return fmaxf(a, b); });
        const int e = !(sum < INFINITY) && most[0] < INFINITY ? static_cast<int>(__float_as_uint(most[0]) >> 23) - 127 : 0;
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) x[j] = ldexpf(x[j], -e);
        if (e) eps = fmaxf(ldexpf(eps, -2 * e), kLeastEps);
        sum = squares();
    }
    const float by = rsqrtf(fmaf(sum, r.inverse_dim, eps));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (!gain) {
#pragma unroll
            for (uint32_t j = 0; j < P; ++j) x[i * P + j] *= by;
        } else if (gain_wide && c.count[i] == P && c.at[i] % P == 0) {
            const f32x4 w = *reinterpret_cast<const f32x4 *>(gain + c.at[i]);
#pragma unroll
            for (uint32_t j = 0; j < P; ++j) x[i * P + j] = x[i * P + j] * by * w[j];
        } else {
#pragma unroll
            for (uint32_t j = 0; j < P; ++j) x[i * P + j] = j < c.count[i] ? x[i * P + j] * by * gain[c.at[i] + j] : 0.0f;
        }
    }
}

template <bool kPairs>
__device__ inline void turn_head(const Piece &c, const float *cosine, const float *sine, float *x) {
    constexpr uint32_t P = kRun;
    if (!c.turned) return;
#pragma unroll
    for (uint32_t j = 0; j < P; ++j) {
        float &a = x[kPairs ? 2 * j : j], &b = x[kPairs ? 2 * j + 1 : P + j];
        const float u = a, w = b;
        a = fmaf(u, cosine[j], -(w * sine[j]));
        b = fmaf(w, cosine[j], u * sine[j]);
    }
}

// Heads nth, nth + per_token, .. of a row of q and k side by side, at one position. Bound by bytes in large calls (8192 rows of 40 heads of 128 in
// bf16 38 us, 4.4 TB/s; the angles and norms take about 400 vector instructions for eight heads), by latency in small ones (one row 3.4 us: position and
// elements, sums, stores). (All lanes of a wavefront come here together, `mine` or
// not: what lanes exchange is exchanged by all.)
template <typename T, bool kPairs, int HEADS>
__device__ inline void rotate_heads(const Turning &r, const Side &q, const Side &k, uint32_t row, int32_t position, uint32_t nth, uint32_t per_token, bool mine) {
    constexpr uint32_t P = kRun;
    const Piece c = piece_of<kPairs>(r, threadIdx.x & ((1u << r.shift) - 1));
    const auto side = [&](uint32_t h) -> const Side & { return h < q.heads ? q : k; };
    Raw<T> raw[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const uint32_t h = min(nth + i * per_token, q.heads + k.heads - 1);
        const Side &s = side(h);
        raw[i] = ask_head(static_cast<const T *>(s.x) + row * s.x_token_stride + (h < q.heads ? h : h - q.heads) * s.x_head_stride, c, s.wide);
    }
    float cosine[P], sine[P];
    turns_of(r, c, position, cosine, sine);
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const uint32_t h = min(nth + i * per_token, q.heads + k.heads - 1);
        const Side &s = side(h);
        const uint32_t head = h < q.heads ? h : h - q.heads;
        float x[2 * P];
        head_values<T>(raw[i], x);
        if (r.norm) norm_head<T>(r, c, s.gain ? s.gain + uint64_t{head} * s.gain_stride : nullptr, s.gain_wide, raw[i], x);
        turn_head<kPairs>(c, cosine, sine, x);
        if (mine && nth + i * per_token == h) write_head(static_cast<T *>(s.y) + row * s.y_token_stride + head * s.y_head_stride, c, s.wide, x);
    }
}

template <typename T, bool kPairs, int HEADS>
__global__ __launch_bounds__(kWG) void k_rotate(Turning r, Side q, Side k, const int32_t *positions, uint32_t items, uint32_t per_token) {
    const uint32_t each = kWG >> r.shift;
    for (uint64_t at = uint64_t{blockIdx.x} * each; at < items; at += uint64_t{gridDim.x} * each) {
        const uint64_t mine = at + (threadIdx.x >> r.shift);
        const uint32_t i = static_cast<uint32_t>(min(mine, uint64_t{items - 1})), row = i / per_token;
        rotate_heads<T, kPairs, HEADS>(r, q, k, row, positions[row], i % per_token, per_token, mine < items);
    }
}

// Query rows of a sequence that is `nth`, nth + step, .. of the grid's workgroups for it.
template <typename T, bool kPairs, int HEADS>
__device__ inline void rotate_queries(const Pool &p, const Rows &rows, const Turning &r, const Side &q, uint32_t b, uint32_t nth, uint32_t step, uint32_t per_token) {
    const Span s = span_of(rows.start, p.lengths, b, rows.tokens);
    const uint32_t items = static_cast<uint32_t>(s.count) * per_token, each = kWG >> r.shift;
    const Side none = {};
    for (uint64_t at = uint64_t{nth} * each; at < items; at += uint64_t{step} * each) {
        const uint64_t mine = at + (threadIdx.x >> r.shift);
        const uint32_t i = static_cast<uint32_t>(min(mine, uint64_t{items - 1})), row = i / per_token;
        rotate_heads<T, kPairs, HEADS>(r, q, none, static_cast<uint32_t>(s.row) + row, s.pos + static_cast<int32_t>(row), i % per_token, per_token, mine < items);
    }
}

// Query rows of sequences on their own, with many new rows: beside the cache's workgroups they would have the registers of those (26 800 rows of 32 query
// and 8 key heads of 128: 302 us in one launch, 178 in two; 1600 rows of 24 and 4 heads of 96 in fp32: 24 in one, 33 in two).  Bound by bytes: 93 us
// for those of the first, 4.7 TB/s.
template <typename T, bool kPairs, int HEADS>
__global__ __launch_bounds__(kWG) void k_rotate_queries(Pool p, Rows rows, Turning r, Side q, uint32_t each, uint32_t per_token) {
    rotate_queries<T, kPairs, HEADS>(p, rows, r, q, blockIdx.x / each, blockIdx.x % each, each, per_token);
}

// The grid of k_append_rotated: workgroups for blocks of the cache, then some for the query rows of each sequence.
struct Shares {
    uint32_t blocks, work, cache_groups;         // as entro_cache_append's; workgroups of the first kind
    uint32_t query_groups, per_token;            // workgroups for a sequence's queries; lane groups to a token of them
};

// LANES lanes to a block and head, as entro_cache_append has it, and its values' patches.  Keys go by lane groups of a head, which keep up
// to 32 elements a lane between finding the block's largest element and writing its codes; blocks of more are read, normed and
// turned twice.  A row of each of 64 sequences (8 key heads of 128, and 32 query heads beside them): 10.9 us, bound by latency (bounds, rows and table,
// sums, scale).  26 800 rows: 85 us, 1.9 TB/s, where entro_cache_append takes 44: three wavefronts a SIMD are what 168 registers leave, and every
// key head finds its angles for itself (14 us of vector instructions by their count).
template <typename T, bool kPairs, int LANES>
__global__ __launch_bounds__(kWG, 3) void k_append_rotated(Pool p, Rows rows, Turning r, Side q, Side keys, Shares g) {
    __shared__ uint32_t most[2][kWG / 64];
    constexpr uint32_t kUnits = kWG / LANES, P = kRun, kKeep = 16 / P;
    if (blockIdx.x >= g.cache_groups) {
        const uint32_t w = blockIdx.x - g.cache_groups;
        rotate_queries<T, kPairs, 1>(p, rows, r, q, w / g.query_groups, w % g.query_groups, g.query_groups, g.per_token);
        return;
    }
    const uint32_t lane = threadIdx.x % LANES, patches = ((p.head_dim + 7) / 8) << (p.page_shift - 2);
    const uint32_t lanes = 1u << r.shift, groups = LANES >> r.shift, mine = lane >> r.shift;
    const Piece c = piece_of<kPairs>(r, lane & (lanes - 1));
    for (uint32_t w = blockIdx.x * kUnits + __builtin_amdgcn_readfirstlane(threadIdx.x / LANES); w < g.work; w += g.cache_groups * kUnits) {
        each_block(p, rows, g.blocks, w, [&](const Block &b, uint32_t head) {
            const T *x = static_cast<const T *>(rows.x[0]) + static_cast<uint64_t>(b.row) * rows.token_stride[0] + head * rows.head_stride[0];
            const T *x_v = static_cast<const T *>(rows.x[1]) + static_cast<uint64_t>(b.row) * rows.token_stride[1] + head * rows.head_stride[1];
            const float *gain = keys.gain ? keys.gain + uint64_t{head} * keys.gain_stride : nullptr;
            float kept[kKeep][2 * P], v[4][8];
            uint32_t m[2] = {0, 0};
            const auto key = [&](uint32_t t, float *y) {
                const Raw<T> raw = ask_head(x + t * rows.token_stride[0], c, keys.wide);
                float cosine[P], sine[P];
                turns_of(r, c, b.at + static_cast<int32_t>(t), cosine, sine);
                head_values<T>(raw, y);
                if (r.norm) norm_head<T>(r, c, gain, keys.gain_wide, raw, y);
                turn_head<kPairs>(c, cosine, sine, y);
            };
            const auto largest_of = [&](const float *y, bool finite) {
                uint32_t all = 0;
#pragma unroll
                for (uint32_t j = 0; j < 2 * P; ++j) {
                    const uint32_t bits = __float_as_uint(y[j]) & 0x7fffffffu;
                    all = max(all, !finite || bits < 0x7f800000u ? bits : 0u);
                }
                return all;
            };
            const auto look = [&](bool finite) {
                m[0] = m[1] = 0;
                // all lanes of a wavefront go on together; those past the last token take it once more
#pragma unroll
                for (uint32_t n = 0; n < kKeep; ++n)
                    if (b.t0 + n * groups < b.t1) {
                        key(min(b.t0 + mine + n * groups, b.t1 - 1), kept[n]);
                        m[0] = max(m[0], largest_of(kept[n], finite));
                    }
                for (uint32_t t = b.t0 + kKeep * groups; t < b.t1; t += groups) {
                    float y[2 * P];
                    key(min(t + mine, b.t1 - 1), y);
                    m[0] = max(m[0], largest_of(y, finite));
                }
                for (uint32_t i = lane; i < patches; i += LANES) {
                    const Patch a = patch_of(p, i, 1);
                    patch_values<T>(ask_patch(x_v, rows.token_stride[1], a, b, p.head_dim, rows.aligned), a, b, p.head_dim, v);
                    m[1] = max(m[1], largest(v, finite));
                }
                for (int o = 32; o; o >>= 1) {
                    m[0] = max(m[0], static_cast<uint32_t>(__shfl_xor(static_cast<int>(m[0]), o)));
                    m[1] = max(m[1], static_cast<uint32_t>(__shfl_xor(static_cast<int>(m[1]), o)));
                }
                if (LANES > 64) {
                    __syncthreads();
                    if ((threadIdx.x & 63u) == 0) most[0][threadIdx.x >> 6] = m[0], most[1][threadIdx.x >> 6] = m[1];
                    __syncthreads();
                    for (int i = 0; i < kWG / 64; ++i) m[0] = max(m[0], most[0][i]), m[1] = max(m[1], most[1][i]);
                }
            };
            look(false);
            const bool numbers = max(m[0], m[1]) < 0x7f800000u;
            if (!numbers) look(true);
            const int32_t page = checked_page(p, b.entry, b.at);
            if (page < 0) return;
            const uint64_t unit = uint64_t{static_cast<uint32_t>(page)} * p.kv_heads + head;
            const uint32_t pt = 1u << p.page_shift;
            const float old[2] = {b.t0 ? p.k_scale[unit] : 0.0f, b.t0 ? p.v_scale[unit] : 0.0f};
            const Grid grid[2] = {grid_of(fmaxf(old[0], __uint_as_float(m[0]) / 127.0f), numbers), grid_of(fmaxf(old[1], __uint_as_float(m[1]) / 127.0f), numbers)};
            // keys before the new ones, where they move
            if (b.t0 && grid[0].scale > old[0]) {
                Block before = b;
                before.t1 = b.t0;
                for (uint32_t i = lane; i < patches; i += LANES) write_patch(p, unit, patch_of(p, i, 0), before, v, old[0], grid[0], 0);
            }
            const auto write_key = [&](uint32_t t, const float *y) {
                uint8_t *at = p.k + (unit * pt + t) * p.width;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t code[P];
#pragma unroll
                    for (uint32_t j = 0; j < P; ++j) code[j] = grid[0].divide ? code_by_division(y[i * P + j], grid[0].scale) : code_by_inverse(y[i * P + j], grid[0]);
                    if (c.count[i] == P && c.at[i] % P == 0) {
                        *reinterpret_cast<uint32_t *>(at + c.at[i]) = four_codes(code[0], code[1], code[2], code[3]);
                    } else {
#pragma unroll
                        for (uint32_t j = 0; j < P; ++j)
                            if (j < c.count[i]) at[c.at[i] + j] = static_cast<uint8_t>(code[j]);
                    }
                }
            };
#pragma unroll
            for (uint32_t n = 0; n < kKeep; ++n) {
                const uint32_t t = b.t0 + mine + n * groups;
                if (t < b.t1) write_key(t, kept[n]);
            }
            for (uint32_t t = b.t0 + kKeep * groups; t < b.t1; t += groups) {
                float y[2 * P];
                key(min(t + mine, b.t1 - 1), y);
                if (t + mine < b.t1) write_key(t + mine, y);
            }
            for (uint32_t i = lane; i < patches; i += LANES) {
                const Patch a = patch_of(p, i, 1);
                if (patches > LANES) patch_values<T>(ask_patch(x_v, rows.token_stride[1], a, b, p.head_dim, rows.aligned), a, b, p.head_dim, v);
                write_patch(p, unit, a, b, v, old[1], grid[1], 1);
            }
            // everybody has read the old scales
            if (LANES > 64)
                __syncthreads();
            else
                __builtin_amdgcn_wave_barrier();
            if (lane == 0) p.k_scale[unit] = grid[0].scale, p.v_scale[unit] = grid[1].scale;
        });
    }
}

// ------------------------------------------------------------------------------------------------------------------ calls
bool finite(float x) { return x > -3.0e38f && x < 3.0e38f; }

bool multiple(const void *p, uint64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

uint64_t size_of(uint32_t type) { return type == ENTRO_F32 ? 4 : 2; }

entro_status check_rotary(const entro_rotary *r, uint32_t head_dim) {
    if (!r) return ENTRO_ERR_NULL;
    if (head_dim == 0 || head_dim > ENTRO_CACHE_MAX_DIM || r->dims > head_dim || r->dims % 2) return ENTRO_ERR_SIZE;
    if (r->layout > ENTRO_ROTARY_PAIRS || r->norm > ENTRO_NORM_CENTRED) return ENTRO_ERR_SCHEME;
    if (r->dims && !r->turns) return ENTRO_ERR_NULL;
    if (!finite(r->amplitude) || (r->norm && !(r->eps >= kLeastEps && finite(r->eps)))) return ENTRO_ERR_RANGE;
    if (!multiple(r->turns, 16) || !multiple(r->q_gain, 4) || !multiple(r->k_gain, 4)) return ENTRO_ERR_ALIGN;
    return ENTRO_OK;
}

entro_status check_side(const entro_rotary_rows *s, uint32_t tokens, uint32_t type) {
    if (tokens && (!s->x || !s->y)) return ENTRO_ERR_NULL;
    if (s->heads == 0 || s->heads > 65536 || uint64_t{tokens} * s->heads > 0x7fffffffull) return ENTRO_ERR_SIZE;
    if (s->x_token_stride > kMaxStride || s->x_head_stride > kMaxStride || s->y_token_stride > kMaxStride || s->y_head_stride > kMaxStride) return ENTRO_ERR_SIZE;
    if (s->x == s->y && (s->x_token_stride != s->y_token_stride || s->x_head_stride != s->y_head_stride)) return ENTRO_ERR_SIZE;
    if (!multiple(s->x, size_of(type)) || !multiple(s->y, size_of(type))) return ENTRO_ERR_ALIGN;
    return ENTRO_OK;
}

// Lanes that have elements of a head.
uint32_t units_of(uint32_t half, uint32_t head_dim) { return (half + kRun - 1) / kRun + (head_dim - 2 * half + 2 * kRun - 1) / (2 * kRun); }

// Whether several heads a lane group pay in a large call.
template <typename T> bool heads_together(const Turning &r) { return sizeof(T) == 2 || 4 * units_of(r.half, r.head_dim) <= 3u << r.shift; }

Turning turning_of(const entro_rotary *r, uint32_t head_dim) {
    const uint32_t half = r->dims / 2, units = units_of(half, head_dim);
    uint32_t shift = 0;
    while ((1u << shift) < units) ++shift;                   // at most 33 units
    return {r->turns, half, head_dim, r->norm, shift, r->eps, r->amplitude, 1.0f / static_cast<float>(head_dim)};
}

Side side_of(const entro_rotary_rows *s, const float *gain, uint32_t gain_stride, uint32_t type) {
    if (!s) return Side{};
    const uint64_t run = kRun * size_of(type);
    const bool wide = multiple(s->x, run) && multiple(s->y, run) && (s->x_token_stride | s->x_head_stride | s->y_token_stride | s->y_head_stride) % kRun == 0;
    return {s->x, s->y, s->x_token_stride, s->x_head_stride, s->y_token_stride, s->y_head_stride, gain, gain_stride, s->heads, wide,
            multiple(gain, 16) && gain_stride % 4 == 0};
}

template <typename T, bool kPairs>
void launch_rotate(const Turning &r, const Side &q, const Side &k, const int32_t *positions, uint32_t tokens, hipStream_t st) {
    const uint32_t heads = q.heads + k.heads, few = (heads + kHeads<T> - 1) / kHeads<T>;
    const bool many = heads_together<T>(r) && ((uint64_t{tokens} * few) << r.shift) >= kManyLanes<T>;
    const uint32_t per_token = many ? few : heads, items = tokens * per_token;
    const uint64_t groups = (uint64_t{items} + (kWG >> r.shift) - 1) / (kWG >> r.shift);
    const dim3 grid(static_cast<uint32_t>(groups < (1u << 23) ? groups : 1u << 23));
    if (many)
        hipLaunchKernelGGL((k_rotate<T, kPairs, kHeads<T>>), grid, dim3(kWG), 0, st, r, q, k, positions, items, per_token);
    else
        hipLaunchKernelGGL((k_rotate<T, kPairs, 1>), grid, dim3(kWG), 0, st, r, q, k, positions, items, per_token);
}

template <typename T, bool kPairs, int LANES>
void launch_append(const Pool &p, const Rows &rows, const Turning &r, const Side &q, const Side &keys, Shares g, uint64_t most_new, hipStream_t st) {
    const uint32_t groups = (g.work + kWG / LANES - 1) / (kWG / LANES);
    g.cache_groups = groups < 65536 ? groups : 65536;
    if (q.heads) {
        const uint32_t few = (q.heads + kHeads<T> - 1) / kHeads<T>;
        const bool many = ((uint64_t{rows.tokens} * (sizeof(T) == 2 ? few : q.heads)) << r.shift) >= kApartLanes<T>, together = many && heads_together<T>(r);
        const uint32_t per_token = together ? few : q.heads;
        const uint64_t each = kWG >> r.shift, wanted = (most_new * per_token + each - 1) / each, fit = (1u << 23) / p.seqs;
        const uint32_t query_groups = wanted < 1 ? 1 : static_cast<uint32_t>(wanted < fit ? wanted : fit);
        if (together) {
            hipLaunchKernelGGL((k_rotate_queries<T, kPairs, kHeads<T>>), dim3(query_groups * p.seqs), dim3(kWG), 0, st, p, rows, r, q, query_groups, per_token);
        } else if (many) {
            if constexpr (sizeof(T) == 4)
                hipLaunchKernelGGL((k_rotate_queries<T, kPairs, 1>), dim3(query_groups * p.seqs), dim3(kWG), 0, st, p, rows, r, q, query_groups, per_token);
        } else {
            g.query_groups = query_groups;
            g.per_token = per_token;
        }
    }
    hipLaunchKernelGGL((k_append_rotated<T, kPairs, LANES>), dim3(g.cache_groups + g.query_groups * p.seqs), dim3(kWG), 0, st, p, rows, r, q, keys, g);
}

}  // namespace

extern "C" {

entro_status entro_rotary_turns(uint32_t dims, double base, uint32_t context, double factor, double trained, double low, double high,
                                uint64_t *turns) {
    if (dims && !turns) return ENTRO_ERR_NULL;
    if (dims % 2 || dims > ENTRO_CACHE_MAX_DIM) return ENTRO_ERR_SIZE;
    if (context > ENTRO_CONTEXT_BY_PARTS) return ENTRO_ERR_SCHEME;
    const double most = 1e300;
    if (!(base >= 1.0 && base < most)) return ENTRO_ERR_RANGE;
    if (context != ENTRO_CONTEXT_AS_TRAINED && !(factor >= 1.0 && factor < most)) return ENTRO_ERR_RANGE;
    if (context == ENTRO_CONTEXT_BY_PARTS && !(trained >= 1.0 && trained < most && low >= 0.0 && high > low && high < most)) return ENTRO_ERR_RANGE;
    const long double two_pi = 6.283185307179586476925286766559005768L;
    for (uint32_t i = 0; i < dims / 2; ++i) {
        long double f = std::pow(static_cast<long double>(base), -2.0L * i / dims);
        if (context == ENTRO_CONTEXT_LINEAR) f /= factor;
        if (context == ENTRO_CONTEXT_BY_PARTS) {
            long double g = (trained * f / two_pi - low) / (static_cast<long double>(high) - low);
            g = g < 0.0L ? 0.0L : g > 1.0L ? 1.0L : g;
            f *= g + (1.0L - g) / factor;
        }
        turns[i] = static_cast<uint64_t>(std::floor(f / two_pi * 18446744073709551616.0L + 0.5L));       // f is 1 at the most
    }
    return ENTRO_OK;
}

entro_status entro_rotate(const entro_rotary *r, const entro_rotary_rows *q, const entro_rotary_rows *k, const int32_t *positions,
                          uint32_t tokens, uint32_t head_dim, entro_dtype type, void *hip_stream) {
    if (const entro_status s = check_rotary(r, head_dim)) return s;
    if ((!q && !k) || (tokens && !positions)) return ENTRO_ERR_NULL;
    if (type != ENTRO_F32 && type != ENTRO_BF16) return ENTRO_ERR_SCHEME;
    for (const entro_rotary_rows *rows : {q, k})
        if (rows)
            if (const entro_status s = check_side(rows, tokens, type)) return s;
    if (uint64_t{tokens} * ((q ? q->heads : 0) + (k ? k->heads : 0)) > 0x7fffffffull) return ENTRO_ERR_SIZE;
    if (!multiple(positions, 4)) return ENTRO_ERR_ALIGN;
    if (tokens == 0) return ENTRO_OK;
    const Turning t = turning_of(r, head_dim);
    const Side a = side_of(q, r->q_gain, r->q_gain_stride, type), b = side_of(k, r->k_gain, r->k_gain_stride, type);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (type == ENTRO_F32)
        r->layout ? launch_rotate<float, true>(t, a, b, positions, tokens, st) : launch_rotate<float, false>(t, a, b, positions, tokens, st);
    else
        r->layout ? launch_rotate<uint16_t, true>(t, a, b, positions, tokens, st) : launch_rotate<uint16_t, false>(t, a, b, positions, tokens, st);
    return hip_ok(hipGetLastError(), "entro_rotate") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

entro_status entro_cache_append_rotated(const entro_cache *c, const entro_cache_table *t, const entro_cache_rows *r, const entro_rotary *rotary,
                                        const entro_rotary_rows *q, void *hip_stream) {
    if (const entro_status s = check_cache(c)) return s;
    if (const entro_status s = check_table(t)) return s;
    if (!r || !r->start || (r->tokens && (!r->k || !r->v))) return ENTRO_ERR_NULL;
    if (r->type != ENTRO_F32 && r->type != ENTRO_BF16) return ENTRO_ERR_SCHEME;
    if (r->layer >= c->layers || r->tokens > 0x7fffffffu) return ENTRO_ERR_SIZE;
    if (r->k_token_stride > kMaxStride || r->k_head_stride > kMaxStride || r->v_token_stride > kMaxStride || r->v_head_stride > kMaxStride)
        return ENTRO_ERR_SIZE;
    if (!multiple(r->k, size_of(r->type)) || !multiple(r->v, size_of(r->type)) || !aligned16(r->start)) return ENTRO_ERR_ALIGN;
    if (const entro_status s = check_rotary(rotary, c->head_dim)) return s;
    if (q)
        if (const entro_status s = check_side(q, r->tokens, r->type)) return s;
    if (r->tokens == 0) return ENTRO_OK;
    // as many blocks as the most rows can touch, and no more than there are slots; the kernel's own loops cover what 31 bits do not
    const uint64_t most_new = r->max_new < r->tokens ? r->max_new : r->tokens, units = uint64_t{c->kv_heads} * t->seqs, fit = 0x7fffffffull / units;
    if (fit == 0 || t->seqs > (1u << 23)) return ENTRO_ERR_SIZE;
    const uint64_t touch = (most_new + c->page_tokens + (most_new ? 0 : 1) - 2) / c->page_tokens + 1, wanted = touch < t->stride ? touch : t->stride;
    Shares g = {};
    g.blocks = static_cast<uint32_t>(wanted < fit ? wanted : fit);
    g.work = static_cast<uint32_t>(g.blocks * units);
    const Pool p = pool_of(c, t, r->layer);
    const bool aligned = multiple(r->v, 16) && ((r->v_token_stride | r->v_head_stride) & 7u) == 0;
    const Rows rows = {{r->k, r->v}, {r->k_token_stride, r->v_token_stride}, {r->k_head_stride, r->v_head_stride}, r->start, r->tokens, aligned};
    const Turning turning = turning_of(rotary, c->head_dim);
    const entro_rotary_rows key_rows = {r->k, r->k, r->k_token_stride, r->k_head_stride, r->k_token_stride, r->k_head_stride, c->kv_heads, 0};
    const Side a = side_of(q, rotary->q_gain, rotary->q_gain_stride, r->type), keys = side_of(&key_rows, rotary->k_gain, rotary->k_gain_stride, r->type);
    const bool few = ((c->head_dim + 7) / 8) * (c->page_tokens / 4) <= 64;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const auto launch = [&](auto element, auto pairs) {
        using T = decltype(element);
        constexpr bool kPairs = decltype(pairs)::value;
        few ? launch_append<T, kPairs, 64>(p, rows, turning, a, keys, g, most_new, st) : launch_append<T, kPairs, kWG>(p, rows, turning, a, keys, g, most_new, st);
    };
    if (r->type == ENTRO_F32)
        rotary->layout ? launch(float{}, std::true_type{}) : launch(float{}, std::false_type{});
    else
        rotary->layout ? launch(uint16_t{}, std::true_type{}) : launch(uint16_t{}, std::false_type{});
    return hip_ok(hipGetLastError(), "entro_cache_append_rotated") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

}  // extern "C"
