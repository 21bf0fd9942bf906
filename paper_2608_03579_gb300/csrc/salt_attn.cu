// Attention of a batch over the paged 8-bit cache, requests of a group
// sharing their prompt.
//
// attn_row_kernel: one warp per (query token, head).  Lanes hold D / 32
// dimensions of q and of the output; each visible token costs a dot product
// over the warp and one step of the running softmax
//     m' = max(m, s),  l' = l 2^(m - m') + 2^(s - m'),  o' = o 2^(m - m') + 2^(s - m') v.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include <cuda_fp16.h>

#include "salt_async.cuh"
#include "salt_host.cuh"
#include "salt_internal.cuh"

namespace salt {
namespace {

// The plan's device tables: int32 words at these places of one block, written
// by the host into a staging area and copied by a kernel.
constexpr int HEAD_WORDS = 8;      // [0]: query tokens
constexpr int TOK_WORDS = 4;       // per query token: first entry of its own page list, own tokens it sees, first entry
                                   // of its group's page list, the prompt's tokens

struct AttnParams {
    const int32_t *plan;           // header, token records, page lists
    KvDev kv;
    int64_t layer;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    int64_t q_stride, out_stride;
    int32_t n_heads, max_tok;
    int32_t tok_at, pages_at;      // word offsets in plan
    float scale_log2;              // scale * log2(e)
    uint32_t *err;
};

__global__ void plan_copy_kernel(const uint4 *src, uint4 *dst, int n)
{
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) dst[i] = src[i];
}

__device__ __forceinline__ float row_scale(uint32_t e) { return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23); }

template <int E>
__device__ __forceinline__ void load_codes(const uint8_t *p, float (&f)[E])
{
    uint32_t c = E == 4 ? __ldg(reinterpret_cast<const uint32_t *>(p)) : __ldg(reinterpret_cast<const uint16_t *>(p));
#pragma unroll
    for (int i = 0; i < E; i += 2) {
        uint32_t h;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(h) : "h"((uint16_t)(c >> (8 * i))));
        const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        f[i] = v.x;
        f[i + 1] = v.y;
    }
}

constexpr int ROW_WARPS = 4;

template <int D>
__global__ void __launch_bounds__(32 * ROW_WARPS) attn_row_kernel(AttnParams p)
{
    constexpr int E = D / 32;
    const int T = p.plan[0], H = p.n_heads, G = H / p.kv.heads, lane = threadIdx.x & 31;
    if (T > p.max_tok) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.err, SALT_DEVERR_BATCH);
        return;
    }
    for (int64_t row = (int64_t)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5); row < (int64_t)T * H; row += (int64_t)gridDim.x * ROW_WARPS) {
        const int t = (int)(row / H), h = (int)(row - (int64_t)t * H), kh = h / G;
        const int4 rec = *reinterpret_cast<const int4 *>(p.plan + p.tok_at + t * TOK_WORDS);
        float q[E], o[E], m = -INFINITY, l = 0.f;
        const uint16_t *qr = p.q + t * p.q_stride + h * D + lane * E;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            q[i] = bf16_to_f(qr[i]) * p.scale_log2;
            o[i] = 0.f;
        }
        bool nan = false;
        for (int part = 0; part < 2; ++part) {
            const int32_t *list = p.plan + p.pages_at + (part ? rec.x : rec.z);
            const int n = part ? rec.y : rec.w;
            for (int j = 0; j < n; ++j) {
                const int64_t at = ((p.layer * p.kv.n_pages + list[j >> p.kv.page_log2]) * p.kv.heads + kh) * p.kv.page + (j & (p.kv.page - 1));
                float k[E], v[E];
                load_codes<E>(p.kv.k + at * D + lane * E, k);
                load_codes<E>(p.kv.v + at * D + lane * E, v);
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < E; ++i) s = fmaf(q[i], k[i], s);
#pragma unroll
                for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
                s *= row_scale(p.kv.k_exp[at]);
                const float vs = row_scale(p.kv.v_exp[at]);
                nan |= !(fabsf(s) < INFINITY);
                const float m2 = fmaxf(m, s), c = exp2f(m - m2), w = exp2f(s - m2);
                l = l * c + w;
#pragma unroll
                for (int i = 0; i < E; ++i) o[i] = o[i] * c + w * vs * v[i];
                m = m2;
            }
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        uint16_t *orow = p.out + t * p.out_stride + h * D + lane * E;
#pragma unroll
        for (int i = 0; i < E; ++i) orow[i] = f_to_bf16(nan ? __uint_as_float(0x7fc00000u) : o[i] * inv);
        if (p.lse && lane == 0)
            p.lse[(int64_t)t * H + h] = nan ? __uint_as_float(0x7fc00000u) : l > 0.f ? (m + log2f(l)) * 0.69314718056f : -INFINITY;
    }
}

}  // namespace
}  // namespace salt

using namespace salt;

struct salt_attn {
    salt_kv *kv = nullptr;
    salt_attn_config cfg{};
    int32_t *plan = nullptr;                   // device tables
    int tok_at = 0, pages_at = 0;
    size_t plan_words = 0;
    int32_t *staging[2] = {nullptr, nullptr};  // page-locked host copies of the tables
    cudaEvent_t staging_ev[2] = {nullptr, nullptr};
    bool staging_used[2] = {false, false};
    int staging_next = 0;
    bool built = false;
    int T = 0;
    std::vector<cudaStream_t> use_streams;     // the build's stream and the runs' since
    cudaEvent_t tmp_ev = nullptr;
};

namespace {

// Makes `stream` wait for what the plan's other streams were given so far.
cudaError_t order_after_uses(salt_attn *a, cudaStream_t stream)
{
    for (cudaStream_t s : a->use_streams) {
        if (s == stream) continue;
        cudaError_t e = cudaEventRecord(a->tmp_ev, s);
        if (e == cudaSuccess) e = cudaStreamWaitEvent(stream, a->tmp_ev, 0);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

salt_status check_batch(const salt_attn *a, const salt_attn_batch *b, int *tokens)
{
    salt_ctx *ctx = a->kv->ctx;
    const salt_attn_config &c = a->cfg;
    const KvDev &kv = a->kv->dev;
    if (b->n_seqs < 0 || b->n_seqs > c.max_seqs)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d requests outside [0, %d]", b->n_seqs, c.max_seqs);
    if (b->n_groups < 0 || b->n_groups > c.max_groups)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d groups outside [0, %d]", b->n_groups, c.max_groups);
    if (b->n_seqs > 0 && (!b->q_len || !b->kv_len || !b->page_ptr)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null request array");
    if (b->n_groups > 0 && (!b->group_len || !b->group_page_ptr || (b->n_seqs > 0 && !b->group)))
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null group array");
    for (const void *p : {(const void *)b->q_len, (const void *)b->kv_len, (const void *)b->page_ptr, (const void *)b->pages,
                          (const void *)b->group, (const void *)b->group_len, (const void *)b->group_page_ptr,
                          (const void *)b->group_pages})
        if (p && on_device(p)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "a batch's arrays are host memory");
    auto check_lists = [&](const char *what, int n, const int32_t *len, const int32_t *ptr, const int32_t *pages, int64_t used) -> salt_status {
        if (n == 0) return SALT_OK;
        if (ptr[0] != 0) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "the %ss' page lists start at %d", what, ptr[0]);
        for (int i = 0; i < n; ++i) {
            if (len[i] < 0) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s %d has %d tokens", what, i, len[i]);
            if (ptr[i + 1] < ptr[i] || used + ptr[i + 1] > c.max_pages)
                return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s %d: page list [%d, %d) out of order or past max_pages", what, i,
                                ptr[i], ptr[i + 1]);
            const int need = (int)(((int64_t)len[i] + kv.page - 1) >> kv.page_log2);
            if (need > ptr[i + 1] - ptr[i])
                return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s %d: %d tokens need %d pages, its list has %d", what, i, len[i], need,
                                ptr[i + 1] - ptr[i]);
            if (need > 0 && !pages) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null page list");
            for (int j = ptr[i]; j < ptr[i] + need; ++j)
                if (pages[j] < 0 || pages[j] >= kv.n_pages)
                    return ctx_fail(ctx, SALT_ERR_SLOT_RANGE, "%s %d: page %d outside [0, %d)", what, i, pages[j], kv.n_pages);
        }
        return SALT_OK;
    };
    salt_status st = check_lists("request", b->n_seqs, b->kv_len, b->page_ptr, b->pages, 0);
    if (st == SALT_OK)
        st = check_lists("group", b->n_groups, b->group_len, b->group_page_ptr, b->group_pages,
                         b->n_seqs > 0 ? b->page_ptr[b->n_seqs] : 0);
    if (st != SALT_OK) return st;
    int64_t T = 0;
    for (int i = 0; i < b->n_seqs; ++i) {
        if (b->q_len[i] < 0) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "request %d has %d query tokens", i, b->q_len[i]);
        T += b->q_len[i];
        if (b->group && (b->group[i] < -1 || b->group[i] >= b->n_groups))
            return ctx_fail(ctx, SALT_ERR_DOMAIN_RANGE, "request %d: group %d outside [-1, %d)", i, b->group[i], b->n_groups);
    }
    if (T > c.max_tokens) return ctx_fail(ctx, SALT_ERR_TOO_MANY_TOKENS, "%lld query tokens, at most %d", (long long)T, c.max_tokens);
    *tokens = (int)T;
    return SALT_OK;
}

// Writes the tables of a checked batch; returns the words used.
size_t fill_plan(const salt_attn *a, const salt_attn_batch *b, int T, int32_t *w)
{
    std::memset(w, 0, HEAD_WORDS * 4);
    w[0] = T;
    const int own_pages = b->n_seqs > 0 ? b->page_ptr[b->n_seqs] : 0;
    const int grp_pages = b->n_groups > 0 ? b->group_page_ptr[b->n_groups] : 0;
    int32_t *tok = w + a->tok_at;
    for (int i = 0; i < b->n_seqs; ++i) {
        const int g = b->group && b->n_groups > 0 ? b->group[i] : -1;
        for (int j = 0; j < b->q_len[i]; ++j, tok += TOK_WORDS) {
            const int64_t see = (int64_t)b->kv_len[i] - b->q_len[i] + j + 1;
            tok[0] = b->page_ptr[i];
            tok[1] = see > 0 ? (int32_t)see : 0;
            tok[2] = g >= 0 ? own_pages + b->group_page_ptr[g] : 0;
            tok[3] = g >= 0 ? b->group_len[g] : 0;
        }
    }
    int32_t *pg = w + a->pages_at;
    if (own_pages > 0) std::memcpy(pg, b->pages, (size_t)own_pages * 4);
    if (grp_pages > 0) std::memcpy(pg + own_pages, b->group_pages, (size_t)grp_pages * 4);
    return a->pages_at + own_pages + grp_pages;
}

}  // namespace

extern "C" {

salt_status salt_attn_create(salt_kv *kv, const salt_attn_config *c, salt_attn **out)
{
    if (!out) return SALT_ERR_INVALID_ARG;
    *out = nullptr;
    if (!kv || !c) return SALT_ERR_INVALID_ARG;
    salt_ctx *ctx = kv->ctx;
    if (c->n_heads < 1 || c->n_heads % kv->dev.heads || c->n_heads / kv->dev.heads > 64)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d query heads over %d key/value heads", c->n_heads, kv->dev.heads);
    if (c->max_seqs < 1 || c->max_seqs > SALT_MAX_TOKENS || c->max_groups < 0 || c->max_groups > SALT_MAX_TOKENS)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "max_seqs %d, max_groups %d", c->max_seqs, c->max_groups);
    if (c->max_tokens < 1 || c->max_tokens > SALT_MAX_TOKENS)
        return ctx_fail(ctx, SALT_ERR_TOO_MANY_TOKENS, "max_tokens %d outside [1, %d]", c->max_tokens, SALT_MAX_TOKENS);
    if (c->max_pages < 1 || c->max_pages > (1 << 28)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "max_pages %d", c->max_pages);
    if (!ctx_select_device(ctx)) return ctx_fail(ctx, SALT_ERR_CUDA, "cannot select the device");
    salt_attn *a = new (std::nothrow) salt_attn;
    if (!a) return ctx_fail(ctx, SALT_ERR_OOM, "no host memory");
    a->kv = kv;
    a->cfg = *c;
    a->tok_at = HEAD_WORDS;
    a->pages_at = a->tok_at + c->max_tokens * TOK_WORDS;
    a->plan_words = ((size_t)a->pages_at + c->max_pages + 3) / 4 * 4;
    bool ok = cudaMalloc(&a->plan, a->plan_words * 4) == cudaSuccess;
    for (int i = 0; i < 2 && ok; ++i)
        ok = cudaHostAlloc(reinterpret_cast<void **>(&a->staging[i]), a->plan_words * 4, cudaHostAllocMapped) == cudaSuccess &&
             cudaEventCreateWithFlags(&a->staging_ev[i], cudaEventDisableTiming) == cudaSuccess;
    ok = ok && cudaEventCreateWithFlags(&a->tmp_ev, cudaEventDisableTiming) == cudaSuccess;
    if (!ok) {
        cudaGetLastError();
        salt_attn_destroy(a);
        return ctx_fail(ctx, SALT_ERR_OOM, "no memory for the plan's tables (%zu bytes)", a->plan_words * 4);
    }
    *out = a;
    return SALT_OK;
}

void salt_attn_destroy(salt_attn *a)
{
    if (!a) return;
    ctx_select_device(a->kv->ctx);
    cudaDeviceSynchronize();
    cudaFree(a->plan);
    for (int i = 0; i < 2; ++i) {
        if (a->staging[i]) cudaFreeHost(a->staging[i]);
        if (a->staging_ev[i]) cudaEventDestroy(a->staging_ev[i]);
    }
    if (a->tmp_ev) cudaEventDestroy(a->tmp_ev);
    cudaGetLastError();
    delete a;
}

salt_status salt_attn_build(salt_attn *a, const salt_attn_batch *b, salt_stream_t stream_)
{
    NvtxRange nvtx_range("salt_attn_build");
    if (!a) return SALT_ERR_INVALID_ARG;
    salt_ctx *ctx = a->kv->ctx;
    if (!b) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null batch");
    if (!ctx_select_device(ctx)) return ctx_fail(ctx, SALT_ERR_CUDA, "cannot select the device");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    cudaStreamCaptureStatus cap;
    SALT_CUDA_OR_FAIL(ctx, cudaStreamIsCapturing(stream, &cap));
    if (cap != cudaStreamCaptureStatusNone) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "a build cannot be captured");
    a->built = false;
    int T = 0;
    const salt_status st = check_batch(a, b, &T);
    if (st != SALT_OK) return st;
    const int k = a->staging_next;
    if (a->staging_used[k]) SALT_CUDA_OR_FAIL(ctx, cudaEventSynchronize(a->staging_ev[k]));
    a->staging_next ^= 1;
    const size_t words = fill_plan(a, b, T, a->staging[k]);
    SALT_CUDA_OR_FAIL(ctx, order_after_uses(a, stream));
    const int n16 = (int)((words + 3) / 4);
    plan_copy_kernel<<<std::min(64, (n16 + 255) / 256), 256, 0, stream>>>(reinterpret_cast<const uint4 *>(a->staging[k]),
                                                                          reinterpret_cast<uint4 *>(a->plan), n16);
    SALT_CUDA_OR_FAIL(ctx, cudaGetLastError());
    SALT_CUDA_OR_FAIL(ctx, cudaEventRecord(a->staging_ev[k], stream));
    a->staging_used[k] = true;
    a->T = T;
    a->built = true;
    a->use_streams.assign(1, stream);
    return SALT_OK;
}

salt_status salt_attn_run(salt_attn *a, int32_t layer, const void *q, int64_t q_stride, float scale, void *out,
                          int64_t out_stride, float *lse, salt_stream_t stream_)
{
    NvtxRange nvtx_range("salt_attn_run");
    if (!a) return SALT_ERR_INVALID_ARG;
    salt_ctx *ctx = a->kv->ctx;
    const KvDev &kv = a->kv->dev;
    if (!a->built) return ctx_fail(ctx, SALT_ERR_NOT_BUILT, "the attention plan was not built");
    if (layer < 0 || layer >= a->kv->n_layers)
        return ctx_fail(ctx, SALT_ERR_LAYER_RANGE, "layer %d outside [0, %d)", layer, a->kv->n_layers);
    if (!std::isfinite(scale)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "scale is not finite");
    if (a->T == 0) return SALT_OK;
    if (!q || !out) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null q or out");
    const int64_t row = (int64_t)a->cfg.n_heads * kv.dim;
    if (q_stride < row || out_stride < row)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "rows of %lld elements %lld and %lld apart", (long long)row,
                        (long long)q_stride, (long long)out_stride);
    if ((q_stride | out_stride) % 8 || ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) ||
        (reinterpret_cast<uintptr_t>(lse) & 3))
        return ctx_fail(ctx, SALT_ERR_ALIGN, "rows of q or out not on 16-byte boundaries, or lse not on a 4-byte one");
    if (!ctx_select_device(ctx)) return ctx_fail(ctx, SALT_ERR_CUDA, "cannot select the device");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (a->use_streams.size() != 1 || a->use_streams[0] != stream) {
        SALT_CUDA_OR_FAIL(ctx, order_after_uses(a, stream));
        if (std::find(a->use_streams.begin(), a->use_streams.end(), stream) == a->use_streams.end())
            a->use_streams.push_back(stream);
    }
    AttnParams p;
    p.plan = a->plan;
    p.kv = kv;
    p.layer = layer;
    p.q = static_cast<const uint16_t *>(q);
    p.out = static_cast<uint16_t *>(out);
    p.lse = lse;
    p.q_stride = q_stride;
    p.out_stride = out_stride;
    p.n_heads = a->cfg.n_heads;
    p.max_tok = a->T;
    p.tok_at = a->tok_at;
    p.pages_at = a->pages_at;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.err = ctx_error_word(ctx);
    const int64_t blocks = ((int64_t)a->T * a->cfg.n_heads + ROW_WARPS - 1) / ROW_WARPS;
    auto kernel = kv.dim == 128 ? attn_row_kernel<128> : attn_row_kernel<64>;
    kernel<<<(unsigned)blocks, 32 * ROW_WARPS, 0, stream>>>(p);
    SALT_CUDA_OR_FAIL(ctx, cudaGetLastError());
    return SALT_OK;
}

}  // extern "C"
