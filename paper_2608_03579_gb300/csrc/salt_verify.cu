// Drafted tokens against the target model's probabilities: accepted while
// u * q(t) < p(t), then one token drawn from what p has above q.
//
// The draw inverts the running sum of the weights max(p - q, 0).  The weights
// are taken in whole units of 2^-40 (a weight is at most 1 and a vocabulary at
// most 2^20, so 64 bits hold every sum), which makes the sums exact: any split
// of the row over threads gives the same token.
#include "salt_host.cuh"
#include "salt_internal.cuh"

namespace salt {
namespace {

constexpr int VF_THREADS = 1024;
constexpr int VF_WARPS = VF_THREADS / 32;

struct VerifyParams {
    const int32_t *ptr, *tok;
    const float *p, *q, *u, *su;
    int64_t p_stride, q_stride;
    int32_t n_drafts, n_vocab;
    int32_t *accepted, *next;
    uint32_t *err;
};

// a weight in units of 2^-40; NaN and what is not above zero count as 0
__device__ __forceinline__ int64_t units(float w) { return w > 0.f ? __float2ll_rz(fminf(w, 1.f) * 1099511627776.f) : 0ll; }

__global__ void __launch_bounds__(VF_THREADS) verify_kernel(VerifyParams a)
{
    const int b = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __shared__ int s_stop;
    __shared__ int64_t s_sum[VF_WARPS];
    const int lo = __ldg(a.ptr + b), hi = __ldg(a.ptr + b + 1);
    if (lo < 0 || hi < lo || hi > a.n_drafts) {
        if (tid == 0) {
            atomicOr(a.err, SALT_DEVERR_DRAFT);
            a.accepted[b] = 0;
            a.next[b] = -1;
        }
        return;
    }
    const int n = hi - lo, V = a.n_vocab;
    if (tid == 0) s_stop = n;
    __syncthreads();
    for (int j = tid; j < n; j += VF_THREADS) {
        const int t = __ldg(a.tok + lo + j);
        bool ok = false;
        if (t < 0 || t >= V) atomicOr(a.err, SALT_DEVERR_DRAFT);
        else ok = __fmul_rn(__ldg(a.u + lo + j), __ldg(a.q + (lo + j) * a.q_stride + t)) < __ldg(a.p + (int64_t)(lo + j + b) * a.p_stride + t);
        if (!ok) atomicMin(&s_stop, j);
    }
    __syncthreads();
    const int stop = s_stop;
    const float *p = a.p + (int64_t)(lo + b + stop) * a.p_stride;
    const float *q = stop < n ? a.q + (int64_t)(lo + stop) * a.q_stride : nullptr;
    const int chunk = (V + VF_WARPS - 1) / VF_WARPS;
    const int v0 = min(V, warp * chunk), v1 = min(V, v0 + chunk);
    auto weight = [&](int v) { return units(q ? __fsub_rn(__ldg(p + v), __ldg(q + v)) : __ldg(p + v)); };
    int64_t total = 0, before = 0;
    for (int pass = 0; pass < 2; ++pass) {
        int64_t sum = 0;
        for (int v = v0 + lane; v < v1; v += 32) sum += weight(v);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) s_sum[warp] = sum;
        __syncthreads();
        total = before = 0;
        for (int w = 0; w < VF_WARPS; ++w) {
            if (w < warp) before += s_sum[w];
            total += s_sum[w];
        }
        if (total > 0 || !q) break;
        q = nullptr;  // p is nowhere above q: p itself
        __syncthreads();
    }
    if (tid == 0) {
        a.accepted[b] = stop;
        if (total <= 0) a.next[b] = -1;
    }
    if (total <= 0) return;
    const int64_t U = __float2ll_rz(fminf(fmaxf(__ldg(a.su + b), 0.f), 0.99999994f) * 16777216.f);
    const int64_t at = U * (total >> 24) + ((U * (total & 0xffffff)) >> 24);
    if (at < before || at >= before + s_sum[warp]) return;
    // the one warp whose share of the running sum holds `at`
    for (int v = v0; v < v1; v += 32) {
        int64_t w = v + lane < v1 ? weight(v + lane) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t up = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += up;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + w > at);
        if (past) {
            if (lane == 0) a.next[b] = v + __ffs(past) - 1;
            return;
        }
        before += __shfl_sync(0xffffffffu, w, 31);
    }
}

}  // namespace
}  // namespace salt

using namespace salt;

extern "C" salt_status salt_verify_drafts(salt_ctx *ctx, int32_t n_seqs, int32_t n_drafts, int32_t n_vocab,
                                          const int32_t *draft_ptr, const int32_t *draft_tokens, const float *target_p,
                                          int64_t target_stride, const float *draft_p, int64_t draft_stride,
                                          const float *accept_u, const float *sample_u, int32_t *accepted,
                                          int32_t *next_token, salt_stream_t stream)
{
    NvtxRange nvtx_range("salt_verify_drafts");
    if (!ctx) return SALT_ERR_INVALID_ARG;
    if (n_seqs < 0 || n_drafts < 0 || n_vocab < 1 || n_vocab > SALT_MAX_VOCAB)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d requests, %d drafts, a vocabulary of %d", n_seqs, n_drafts, n_vocab);
    if (n_seqs == 0) return SALT_OK;
    if (!draft_ptr || !target_p || !sample_u || !accepted || !next_token || (n_drafts > 0 && (!draft_tokens || !draft_p || !accept_u)))
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null array");
    if (target_stride < n_vocab || (n_drafts > 0 && draft_stride < n_vocab))
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "rows of %d floats %lld and %lld apart", n_vocab, (long long)target_stride,
                        (long long)draft_stride);
    uintptr_t bits = 0;
    for (const void *p : {(const void *)draft_ptr, (const void *)draft_tokens, (const void *)target_p, (const void *)draft_p,
                          (const void *)accept_u, (const void *)sample_u, (const void *)accepted, (const void *)next_token})
        bits |= reinterpret_cast<uintptr_t>(p);
    if (bits & 3) return ctx_fail(ctx, SALT_ERR_ALIGN, "an array not on a 4-byte boundary");
    if (!ctx_select_device(ctx)) return ctx_fail(ctx, SALT_ERR_CUDA, "cannot select the device");
    const VerifyParams a{draft_ptr, draft_tokens, target_p, draft_p, accept_u, sample_u, target_stride, draft_stride,
                         n_drafts, n_vocab, accepted, next_token, ctx_error_word(ctx)};
    verify_kernel<<<n_seqs, VF_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(a);
    SALT_CUDA_OR_FAIL(ctx, cudaGetLastError());
    return SALT_OK;
}
