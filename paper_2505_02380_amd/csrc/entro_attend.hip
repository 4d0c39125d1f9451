// Attention over the 8-bit token cache on the GPU (include/entro.h has the layouts and the definition).
#include "entro_cache.h"

namespace {

using namespace entro_detail;

constexpr int kWG = 256;

struct Query {
    const void *q;
    void *out;
    float *lse;
    uint64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    const int32_t *start;
    uint32_t tokens, q_heads, group, window, sinks;
    float scale;
};

// One workgroup per row and query head: scores of 256 keys at a time, a running maximum and sum, then a lane per dimension.
template <typename T, typename S>
__global__ __launch_bounds__(kWG) void k_attend_simple(Pool p, Query a, uint64_t work) {
    __shared__ float q[ENTRO_CACHE_MAX_DIM], prob[kWG], red[kWG / 64];
    __shared__ int32_t key_page[kWG];
    const uint32_t tid = threadIdx.x, pt = 1u << p.page_shift;
    for (uint64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const uint32_t h = static_cast<uint32_t>(w % a.q_heads), head = h / a.group;
        const int32_t row = static_cast<int32_t>(w / a.q_heads);
        uint32_t lo = 0, hi = p.seqs;
        while (hi - lo > 1) {
            const uint32_t mid = (lo + hi) / 2;
            if (a.start[mid] <= row) lo = mid; else hi = mid;
        }
        const Span s = span_of(a.start, p.lengths, lo, a.tokens);
        if (row < s.row || row >= s.row + s.count) continue;
        const int32_t pos = s.pos + row - s.row;
        const T *qr = static_cast<const T *>(a.q) + static_cast<uint32_t>(row) * a.q_token_stride + h * a.q_head_stride;
        for (uint32_t d = tid; d < p.head_dim; d += kWG) q[d] = S::load(qr + d);
        float top = -INFINITY, sum = 0.0f, acc = 0.0f;
        for (int32_t j0 = 0; j0 <= pos; j0 += kWG) {
            const int32_t j = j0 + static_cast<int32_t>(tid);
            int32_t page = -1;
            if (j <= pos && (!a.window || static_cast<uint32_t>(pos - j) < a.window || static_cast<uint32_t>(j) < a.sinks)) page = page_of(p, lo, j >> p.page_shift);
            __syncthreads();
            float z = -INFINITY;
            if (page >= 0) {
                const uint64_t unit = uint64_t{static_cast<uint32_t>(page)} * p.kv_heads + head;
                const uint8_t *k = p.k + (unit * pt + (static_cast<uint32_t>(j) & (pt - 1))) * p.width;
                float dot = 0.0f;
                for (uint32_t d = 0; d < p.head_dim; ++d) dot = fmaf(q[d], static_cast<float>(static_cast<int32_t>(k[d]) - 128), dot);
                z = dot * p.k_scale[unit] * a.scale;
            }
            float m = z;
            for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
            if ((tid & 63u) == 0) red[tid >> 6] = m;
            __syncthreads();
            for (int i = 0; i < kWG / 64; ++i) m = fmaxf(m, red[i]);
            const float now = fmaxf(top, m), by = now == -INFINITY ? 0.0f : expf(top - now);
            const float e = z == -INFINITY ? 0.0f : expf(z - now);
            prob[tid] = e;
            key_page[tid] = page;
            __syncthreads();
            sum *= by;
            acc *= by;
            top = now;
            const int32_t n = min(kWG, pos - j0 + 1);
            for (int32_t i = 0; i < n; ++i) {
                if (key_page[i] < 0) continue;
                sum += prob[i];
                if (tid < p.head_dim) {
                    const uint64_t unit = uint64_t{static_cast<uint32_t>(key_page[i])} * p.kv_heads + head;
                    const uint8_t c = p.v[(unit * p.width + tid) * pt + (static_cast<uint32_t>(j0 + i) & (pt - 1))];
                    acc = fmaf(prob[i] * p.v_scale[unit], static_cast<float>(static_cast<int32_t>(c) - 128), acc);
                }
            }
        }
        if (tid < p.head_dim) {
            T *o = static_cast<T *>(a.out) + static_cast<uint32_t>(row) * a.out_token_stride + h * a.out_head_stride;
            o[tid] = S::store(sum > 0.0f ? acc / sum : 0.0f);
        }
        if (tid == 0 && a.lse) a.lse[uint64_t{static_cast<uint32_t>(row)} * a.q_heads + h] = sum > 0.0f ? top + logf(sum) : -INFINITY;
        __syncthreads();
    }
}

struct AsF32 {
    static __device__ float load(const float *p) { return *p; }
    static __device__ float store(float f) { return f; }
};
struct AsBf16 {
    static __device__ float load(const uint16_t *p) { return bf16_to_f32(*p); }
    static __device__ uint16_t store(float f) { return f32_to_bf16(f); }
};

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

}  // namespace

extern "C" {

uint64_t entro_cache_attend_workspace_bytes(const entro_cache *c, const entro_cache_table *t, const entro_cache_query *q) {
    if (check_sizes(c) != ENTRO_OK || check_table_sizes(t) != ENTRO_OK || check_query_sizes(c, q) != ENTRO_OK) return 0;
    return 0;
}

entro_status entro_cache_attend(const entro_cache *c, const entro_cache_table *t, const entro_cache_query *q, void *workspace,
                                uint64_t workspace_bytes, void *hip_stream) {
    (void)workspace, (void)workspace_bytes;
    if (const entro_status s = check_cache(c)) return s;
    if (const entro_status s = check_table(t)) return s;
    if (const entro_status s = check_query(c, q)) return s;
    if (q->tokens == 0) return ENTRO_OK;
    const Pool p = pool_of(c, t, q->layer);
    const Query a = {q->q, q->out, q->lse, q->q_token_stride, q->q_head_stride, q->out_token_stride, q->out_head_stride, q->start,
                     q->tokens, q->q_heads, q->q_heads / c->kv_heads, q->window, q->sinks, q->scale};
    const uint64_t work = uint64_t{q->tokens} * q->q_heads;
    const unsigned grid = static_cast<unsigned>(work < 65536 ? work : 65536);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (q->type == ENTRO_F32)
        hipLaunchKernelGGL((k_attend_simple<float, AsF32>), dim3(grid), dim3(kWG), 0, st, p, a, work);
    else
        hipLaunchKernelGGL((k_attend_simple<uint16_t, AsBf16>), dim3(grid), dim3(kWG), 0, st, p, a, work);
    return hip_ok(hipGetLastError(), "entro_cache_attend") ? ENTRO_OK : ENTRO_ERR_DEVICE;
}

}  // extern "C"
