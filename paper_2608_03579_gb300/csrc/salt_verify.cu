// Drafted tokens against the target model's probabilities: accepted while
// u * q(t) < p(t), then one token drawn from what p has above q.
//
// The draw inverts the running sum of the weights max(p - q, 0).  The weights
// are taken in whole units of 2^-40 (a weight is at most 1 and a vocabulary at
// most 2^20, so 64 bits hold every sum), which makes the sums exact: any split
// of the row over threads gives the same token.
//
// A request's work is reading one row of p and one of q (1 MB for 131,072
// tokens), so it is spread over a cluster of CTAs: each sums its share, the
// sums meet in shared memory, and the one warp whose share holds the drawn
// place goes over that share again.
#include <cooperative_groups.h>

#include "salt_host.cuh"
#include "salt_internal.cuh"
#include "salt_pipe.cuh"

namespace salt {
namespace {

// 256 requests over 131,072 tokens, about half of which read p alone (198 MB), take 54 us (3.7 TB/s, 54% of a copy's rate)
// with 256 threads, four pieces of each row under way and five CTAs an SM.  Measured at 52 us of that kernel: with 512 threads and two CTAs 64 us, three and two pieces 60, four and two pieces 56; 256
// threads, three CTAs and eight pieces 61; 128 threads, ten CTAs 62.  What is left over the bytes (29 us) is what a CTA does before
// its rows are known, three dependent reads that its cluster's eight CTAs repeat, and the cluster's meeting at the end, in 2.7
// rounds of resident CTAs.
constexpr int VF_THREADS = 256;
constexpr int VF_WARPS = VF_THREADS / 32;
constexpr int VF_CTAS = 5;            // CTAs an SM
constexpr int VF_CLUSTER = 8;         // CTAs a request at most (with 2 for each of 256 requests a run takes 14% longer)
constexpr int VF_SHARE = 2048;        // tokens that are worth another CTA

struct VerifyParams {
    const int32_t *ptr, *tok;
    const float *p, *q, *u, *su;
    int64_t p_stride, q_stride;
    int32_t n_drafts, n_vocab;
    int32_t *accepted, *next;
    uint32_t *err;  // or none
};

// A weight in units of 2^-40; NaN and what is not above zero count as 0.  w = M 2^(E - 150) with a
// whole M below 2^24, so this is M shifted by E - 110 places (a conversion to 64-bit integers runs at a
// small part of the rate of these).
__device__ __forceinline__ int64_t units(float w)
{
    const uint32_t b = __float_as_uint(fminf(w, 1.f)), M = (b & 0x7fffffu) | 0x800000u;
    const int s = (int)(b >> 23) - 110;  // at most 17; weights below the normal range come to 0
    const uint32_t lo = s >= 0 ? M << s : M >> min(-s, 31), hi = (M >> 1) >> (31 - max(s, 0));
    return w > 0.f ? (int64_t)((uint64_t)hi << 32 | lo) : 0ll;
}

// Four weights from v on (those below end), p and q (or none) read as one
// 16-byte piece where VEC says that rows lie on such boundaries.
template <bool VEC>
__device__ __forceinline__ void weights4(const float *p, const float *q, int v, int end, float (&w)[4])
{
    float a[4] = {0.f, 0.f, 0.f, 0.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
    if (VEC && v + 4 <= end) {
        const float4 x = __ldg(reinterpret_cast<const float4 *>(p + v));
        a[0] = x.x, a[1] = x.y, a[2] = x.z, a[3] = x.w;
        if (q) {
            const float4 y = __ldg(reinterpret_cast<const float4 *>(q + v));
            b[0] = y.x, b[1] = y.y, b[2] = y.z, b[3] = y.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (v + i < end) {
                a[i] = __ldg(p + v + i);
                if (q) b[i] = __ldg(q + v + i);
            }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = q ? __fsub_rn(a[i], b[i]) : a[i];
}

template <bool VEC>
__device__ __forceinline__ int64_t sum_share(const float *p, const float *q, int v0, int v1, int lane)
{
    int64_t sum = 0;
    if (VEC) {  // whole pieces, AT_ONCE of each row under way
        constexpr int AT_ONCE = 4;
        for (; v0 + 128 * AT_ONCE <= v1; v0 += 128 * AT_ONCE) {
            float4 x[AT_ONCE], y[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                x[i] = __ldcs(reinterpret_cast<const float4 *>(p + v0 + 128 * i) + lane);
                y[i] = q ? __ldcs(reinterpret_cast<const float4 *>(q + v0 + 128 * i) + lane) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                sum += (units(__fsub_rn(x[i].x, y[i].x)) + units(__fsub_rn(x[i].y, y[i].y))) +
                       (units(__fsub_rn(x[i].z, y[i].z)) + units(__fsub_rn(x[i].w, y[i].w)));
        }
    }
    for (int v = v0 + 4 * lane; v < v1; v += 128) {
        float w[4];
        weights4<VEC>(p, q, v, v1, w);
        sum += (units(w[0]) + units(w[1])) + (units(w[2]) + units(w[3]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}

template <bool VEC>
__global__ void __launch_bounds__(VF_THREADS, VF_CTAS) verify_kernel(VerifyParams a)
{
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = blockIdx.x / C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __shared__ int s_stop;
    __shared__ int64_t s_sum[VF_WARPS], s_all[2][VF_CLUSTER];
    // A CTA writes into the others' shared memory once all of them run: they say so here, and it waits
    // when its share is summed.
    cluster_arrive();
    pdl_wait();  // (launched beside the end of what came before)
    pdl_launch_dependents();
    a.ptr = after_pdl_wait(a.ptr);
    a.su = after_pdl_wait(a.su);
    const int lo = __ldg(a.ptr + b), hi = __ldg(a.ptr + b + 1);
    if (lo < 0 || hi < lo || hi > a.n_drafts) {  // (the whole cluster)
        if (tid == 0 && rank == 0) {
            if (a.err) atomicOr(a.err, SALT_DEVERR_DRAFT);
            a.accepted[b] = 0;
            a.next[b] = -1;
        }
        cluster_wait();
        return;
    }
    const int n = hi - lo, V = a.n_vocab;
    if (tid == 0) s_stop = n;
    __syncthreads();
    for (int j = tid; j < n; j += VF_THREADS) {
        const int t = __ldg(a.tok + lo + j);
        bool ok = false;
        if (t >= 0 && t < V) ok = __fmul_rn(__ldg(a.u + lo + j), __ldg(a.q + ((int64_t)lo + j) * a.q_stride + t)) < __ldg(a.p + ((int64_t)lo + j + b) * a.p_stride + t);
        else if (a.err) atomicOr(a.err, SALT_DEVERR_DRAFT);
        if (!ok) atomicMin(&s_stop, j);
    }
    __syncthreads();
    const int stop = s_stop;
    const float *p = a.p + ((int64_t)lo + b + stop) * a.p_stride;
    const float *q = stop < n ? a.q + ((int64_t)lo + stop) * a.q_stride : nullptr;
    // this warp's share of the row
    const int share = (V + C * VF_WARPS * 4 - 1) / (C * VF_WARPS * 4) * 4;
    const int v0 = min(V, (rank * VF_WARPS + warp) * share), v1 = min(V, v0 + share);
    int64_t total = 0, before = 0, mine = 0;
    for (int pass = 0; pass < 2; ++pass) {
        mine = sum_share<VEC>(p, q, v0, v1, lane);
        if (pass == 0) cluster_wait();
        if (lane == 0) s_sum[warp] = mine;
        __syncthreads();
        if (warp == 0) {  // the CTA's sum to every CTA of the cluster
            int64_t s = lane < VF_WARPS ? s_sum[lane] : 0;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (lane < C) *cluster.map_shared_rank(&s_all[pass][rank], lane) = s;
        }
        cluster.sync();
        total = before = 0;
        for (int c = 0; c < C; ++c) {
            if (c < rank) before += s_all[pass][c];
            total += s_all[pass][c];
        }
        for (int w = 0; w < warp; ++w) before += s_sum[w];
        if (total > 0 || !q) break;
        q = nullptr;  // p is nowhere above q: p itself
        __syncthreads();
    }
    if (tid == 0 && rank == 0) {
        a.accepted[b] = stop;
        if (total <= 0) a.next[b] = -1;
    }
    if (total <= 0) return;
    const int64_t U = __float2ll_rz(fminf(fmaxf(__ldg(a.su + b), 0.f), 0.99999994f) * 16777216.f);
    const int64_t at = U * (total >> 24) + ((U * (total & 0xffffff)) >> 24);
    if (at < before || at >= before + mine) return;
    // the one warp whose share of the running sum holds `at`
    for (int v = v0; v < v1; v += 128) {
        float w[4];
        weights4<VEC>(p, q, v + 4 * lane, v1, w);
        const int64_t u0 = units(w[0]), u1 = u0 + units(w[1]), u2 = u1 + units(w[2]), u3 = u2 + units(w[3]);
        int64_t run = u3;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t up = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += up;
        }
        const uint32_t past = __ballot_sync(0xffffffffu, before + run > at);
        if (past) {
            if (lane == __ffs(past) - 1) {
                const int64_t from = before + run - u3;
                a.next[b] = v + 4 * lane + (from + u0 > at ? 0 : from + u1 > at ? 1 : from + u2 > at ? 2 : 3);
            }
            return;
        }
        before += __shfl_sync(0xffffffffu, run, 31);
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
    if (ctx && !ctx_select_device(ctx)) return ctx_fail(ctx, SALT_ERR_CUDA, "cannot select the device");
    const VerifyParams a{draft_ptr, draft_tokens, target_p, draft_p, accept_u, sample_u, target_stride, draft_stride,
                         n_drafts, n_vocab, accepted, next_token, ctx ? ctx_error_word(ctx) : nullptr};
    // One CTA for each VF_SHARE tokens, up to VF_CLUSTER (a power of two).
    int ctas = 1;
    while (ctas < VF_CLUSTER && ctas * VF_SHARE < n_vocab) ctas *= 2;
    if ((int64_t)n_seqs * ctas > 0x7fffffff) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d requests in one call", n_seqs);
    const bool vec = ((reinterpret_cast<uintptr_t>(target_p) | (n_drafts > 0 ? reinterpret_cast<uintptr_t>(draft_p) : 0)) & 15) == 0 &&
                     target_stride % 4 == 0 && (n_drafts == 0 || draft_stride % 4 == 0);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)(n_seqs * ctas), 1, 1);
    cfg.blockDim = dim3(VF_THREADS, 1, 1);
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    SALT_CUDA_OR_FAIL(ctx, cudaLaunchKernelEx(&cfg, vec ? verify_kernel<true> : verify_kernel<false>, a));
    return SALT_OK;
}
