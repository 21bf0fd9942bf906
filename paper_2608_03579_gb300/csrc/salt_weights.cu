// How much attention a batch's cached tokens got, added to what they gathered
// before:
//     W[j] = decay * W[j] + sum_i exp(scale * q_i k_j - lse_i)
// over the rows i (query token x query heads of the token's key/value head) that
// see token j, W[j] counted as 0 for the step's own tokens.  The rows' log-sums come from
// the attention itself, so that one pass over the keys is all there is to do, and a
// token's weight is one thread's sum in a fixed order.
#include <cmath>
#include <new>

#include <cuda_fp16.h>

#include "salt_async.cuh"
#include "salt_attn.cuh"
#include "salt_host.cuh"
#include "salt_internal.cuh"
#include "salt_pipe.cuh"
#include "salt_tcgen05.cuh"

namespace salt {
namespace {

constexpr float LOG2E = 1.4426950408889634f;

struct WeightParams {
    const int32_t *plan, *track;
    int32_t order_at, pages_at, list_at;
    KvDev kv;
    int64_t layer;
    const uint16_t *q;
    const float *lse;
    float *weights;
    int64_t q_stride;
    int32_t n_heads, max_tok;
    float scale, decay;
    uint32_t *err;
};

// A list of cached tokens and the rows that see it.
struct List {
    int pages, len, tok, ntok, old, lim, causal, tiles;
};
__device__ __forceinline__ List load_list(const WeightParams &p, int i)
{
    const int4 *w = reinterpret_cast<const int4 *>(p.track + p.list_at + i * LIST_WORDS);
    const int4 a = __ldg(w), b = __ldg(w + 1);
    return {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}
// The list that holds tile `tile` of all lists: the last one that begins at or before it.
__device__ __forceinline__ int find_list(const WeightParams &p, int n, int tile)
{
    int lo = 0;
    for (int hi = n; hi - lo > 1;) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(p.track + p.list_at + mid * LIST_WORDS + LS_TILES) <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

constexpr int ROWS_AT_ONCE = 16;

// A thread has a token's key in registers and walks the rows, which go through shared memory.
template <int D>
__global__ void __launch_bounds__(TRACK_TILE) weights_kernel(const WeightParams p)
{
    __shared__ __align__(16) float s_q[ROWS_AT_ONCE][D];
    __shared__ float s_lse[ROWS_AT_ONCE];
    const int32_t *track = p.track;
    if (track[TH_TOKENS] > p.max_tok || track[TH_SHARED]) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.err, SALT_DEVERR_BATCH);
        return;
    }
    const int KV = p.kv.heads, G = p.n_heads / KV, n_lists = track[TH_LISTS], tid = threadIdx.x;
    if (n_lists == 0) return;
    const List last = load_list(p, n_lists - 1);
    const int64_t units = (int64_t)(last.tiles + (last.len + TRACK_TILE - 1) / TRACK_TILE) * KV;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int tile = (int)(u / KV), kh = (int)(u - (int64_t)tile * KV);
        const List l = load_list(p, find_list(p, n_lists, tile));
        const int j = (tile - l.tiles) * TRACK_TILE + tid;
        const bool live = j < l.len;
        const int page = live ? __ldg(p.plan + p.pages_at + l.pages + (j >> p.kv.page_log2)) : 0;
        const int64_t at = (((p.layer * p.kv.n_pages + page) * KV + kh) << p.kv.page_log2) + (j & (p.kv.page - 1));
        float k[D];
        float kf = 0.f;
#pragma unroll
        for (int i = 0; i < D / 4; ++i) {
            const uint32_t c = live ? __ldg(reinterpret_cast<const uint32_t *>(p.kv.k + at * D) + i) : 0;
            const uint32_t lo = f16x2_of_e4m3x2((uint16_t)c), hi = f16x2_of_e4m3x2((uint16_t)(c >> 16));
            const float2 a = __half22float2(*reinterpret_cast<const __half2 *>(&lo)), b = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
            k[4 * i] = a.x, k[4 * i + 1] = a.y, k[4 * i + 2] = b.x, k[4 * i + 3] = b.y;
        }
        if (live) kf = row_scale(p.kv.k_exp[at]);
        float sum = 0.f;
        const int rows = l.ntok * G;
        for (int r0 = 0; r0 < rows; r0 += ROWS_AT_ONCE) {
            __syncthreads();
            for (int i = tid; i < ROWS_AT_ONCE * (D / 2); i += TRACK_TILE) {
                const int r = r0 + i / (D / 2), d = i % (D / 2);
                uint32_t x = 0;
                if (r < rows) {
                    const int t = __ldg(p.plan + p.order_at + l.tok + r / G);
                    x = __ldg(reinterpret_cast<const uint32_t *>(p.q + t * p.q_stride + (kh * G + r % G) * D) + d);
                    if (d == 0) s_lse[r - r0] = p.lse[(int64_t)t * p.n_heads + kh * G + r % G];
                }
                s_q[r - r0][2 * d] = __uint_as_float(x << 16);
                s_q[r - r0][2 * d + 1] = __uint_as_float(x & 0xffff0000u);
            }
            __syncthreads();
            for (int i = 0; i < min(ROWS_AT_ONCE, rows - r0); ++i) {
                float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int d = 0; d < D; d += 4) {
                    const float4 q = *reinterpret_cast<const float4 *>(&s_q[i][d]);
                    s[0] = fmaf(q.x, k[d], s[0]);
                    s[1] = fmaf(q.y, k[d + 1], s[1]);
                    s[2] = fmaf(q.z, k[d + 2], s[2]);
                    s[3] = fmaf(q.w, k[d + 3], s[3]);
                }
                const float x = fmaf((s[0] + s[1] + (s[2] + s[3])) * kf, p.scale, -s_lse[i]);
                if (j < l.lim + (l.causal ? (r0 + i) / G : 0)) sum += ex2(x * LOG2E);
            }
        }
        if (live) {
            float *w = p.weights + at;
            *w = p.decay != 0.f && j < l.old ? fmaf(p.decay, *w, sum) : sum;
        }
    }
}

}  // namespace
}  // namespace salt

using namespace salt;

extern "C" {

salt_status salt_attn_weights(salt_attn *a, int32_t layer, const void *q, int64_t q_stride, const float *lse, float scale, float decay,
                              float *weights, salt_stream_t stream_)
try {
    NvtxRange nvtx_range("salt_attn_weights");
    if (!a) return SALT_ERR_INVALID_ARG;
    salt_ctx *ctx = a->kv->ctx;
    const KvDev &kv = a->kv->dev;
    if (!std::isfinite(scale) || !std::isfinite(decay)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "scale or decay is not finite");
    if (a->built && a->T > 0) {
        if (!q || !lse || !weights) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null q, lse or weights");
        if (q_stride < (int64_t)a->cfg.n_heads * kv.dim)
            return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "rows of %lld elements %lld apart", (long long)a->cfg.n_heads * kv.dim, (long long)q_stride);
        if (q_stride % 8 || ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(weights)) & 15) || (reinterpret_cast<uintptr_t>(lse) & 3))
            return ctx_fail(ctx, SALT_ERR_ALIGN, "rows of q or weights not on 16-byte boundaries, or lse not on a 4-byte one");
    }
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    bool captured;
    const salt_status st = track_enter(a, layer, 1, stream, &captured);
    if (st != SALT_OK || (a->track.n_lists == 0 && !captured)) return st;
    WeightParams p;
    p.plan = a->plan;
    p.track = a->track.table;
    p.order_at = a->order_at;
    p.pages_at = a->pages_at;
    p.list_at = a->track.list_at;
    p.kv = kv;
    p.layer = layer;
    p.q = static_cast<const uint16_t *>(q);
    p.lse = lse;
    p.weights = weights;
    p.q_stride = q_stride;
    p.n_heads = a->cfg.n_heads;
    p.max_tok = a->T;
    p.scale = scale;
    p.decay = decay;
    p.err = ctx_error_word(ctx);
    const auto kernel = kv.dim == 128 ? weights_kernel<128> : weights_kernel<64>;
    kernel<<<a->n_sm * 3, TRACK_TILE, 0, stream>>>(p);
    SALT_CUDA_OR_FAIL(ctx, cudaGetLastError());
    return SALT_OK;
} catch (const std::bad_alloc &) {
    return ctx_fail(a->kv->ctx, SALT_ERR_OOM, "no host memory");
}

}  // extern "C"
