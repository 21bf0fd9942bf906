// Requests back to their share of the cache: of each layer, request and
// key/value head the tokens that are kept, and those moved to the front of the
// request's pages in their order.
//
// Kept are the last `recent` tokens, the first `first` ones, and of the others those of
// the largest scores, ties to the earlier one.  Scores are ordered as unsigned
// words; a search by digits from the top finds the last score that is kept and how many of its ties.
//
// A kept token's new place is never behind its old one, so rows move in place: place i is written once what lies
// there was read, and that belongs to the i-th kept token or an earlier one.
#include <algorithm>
#include <new>

#include "salt_async.cuh"
#include "salt_attn.cuh"
#include "salt_host.cuh"
#include "salt_internal.cuh"
#include "salt_pipe.cuh"

namespace salt {
namespace {

constexpr int SELECT_THREADS = 1024, MOVE_THREADS = 256;

struct EvictParams {
    const int32_t *plan, *track;
    int32_t pages_at, seq_at;
    KvDev kv;
    int64_t layer;              // the first one
    const int32_t *keep;
    const float *scores;
    float *weights;             // or NULL
    int32_t *kept;              // [layers][requests][heads][kept_stride]
    int64_t kept_stride;
    int32_t n_seqs, first, recent;
    uint32_t *err;
};

// One layer's, request's and head's own tokens.
struct Line {
    const int32_t *pages;       // of the request
    int64_t page0;              // number of the layer's first page
    int head, len, keep, first, recent;
    int32_t *kept;
};

// The line's b-th in the launch; keep is 0 where there is nothing to do.
__device__ __forceinline__ Line load_line(const EvictParams &p, int b)
{
    const int KV = p.kv.heads;
    const int head = b % KV, seq = b / KV % p.n_seqs, layer = b / KV / p.n_seqs;
    const int2 s = __ldg(reinterpret_cast<const int2 *>(p.track + p.seq_at) + seq);
    Line l;
    l.pages = p.plan + p.pages_at + s.x;
    l.page0 = (p.layer + layer) * p.kv.n_pages;
    l.head = head;
    l.len = s.y;
    l.keep = __ldg(p.keep + seq);
    l.kept = p.kept + (int64_t)b * p.kept_stride;
    if (l.keep < 0 || l.keep > p.kept_stride) {
        if (head == 0 && layer == 0 && threadIdx.x == 0) atomicOr(p.err, SALT_DEVERR_KEEP);
        l.keep = 0;
    }
    if (l.keep >= l.len) l.keep = 0;
    l.recent = min(p.recent, l.keep);
    l.first = min(p.first, l.keep - l.recent);
    return l;
}
__device__ __forceinline__ int64_t row_of(const EvictParams &p, const Line &l, int j)
{
    return (((l.page0 + __ldg(l.pages + (j >> p.kv.page_log2))) * p.kv.heads + l.head) << p.kv.page_log2) + (j & (p.kv.page - 1));
}

// Larger scores are larger words; the zeros are one, a NaN is below everything.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x);
    if (!(x == x)) return 0u;
    if (x == 0.f) return 0x80000000u;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum over the block of a thread's value and of those of the threads before it.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t *s_warp, uint32_t *total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t sum = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += up;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    if (warp == 0) {
        uint32_t w = lane < (int)blockDim.x / 32 ? s_warp[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += up;
        }
        s_warp[lane] = w;
    }
    __syncthreads();
    *total = s_warp[blockDim.x / 32 - 1];
    return sum + (warp ? s_warp[warp - 1] : 0u);
}

__global__ void __launch_bounds__(SELECT_THREADS) evict_select_kernel(const EvictParams p)
{
    __shared__ uint32_t s_hist[256], s_warp[32], s_found[2];
    if (p.track[TH_SEQS] > p.n_seqs || p.track[TH_SHARED]) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(p.err, SALT_DEVERR_BATCH);
        return;
    }
    if (blockIdx.x / p.kv.heads % p.n_seqs >= p.track[TH_SEQS]) return;
    const Line l = load_line(p, blockIdx.x);
    if (l.keep == 0) return;
    const int tid = threadIdx.x, from = l.first, to = l.len - l.recent;
    uint32_t want = l.keep - l.first - l.recent, prefix = 0;
    // the smallest key that is kept, and `want` of those that are equal to it
    for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
        if (tid < 256) s_hist[tid] = 0;
        __syncthreads();
        for (int j = from + tid; j < to; j += SELECT_THREADS) {
            const uint32_t key = key_of(__ldg(p.scores + row_of(p, l, j)));
            if (shift == 24 || key >> (shift + 8) == prefix) atomicAdd(&s_hist[(key >> shift) & 255], 1);
        }
        __syncthreads();
        // from the largest digit down
        uint32_t total;
        const uint32_t n = tid < 256 ? s_hist[255 - tid] : 0u, up_to = block_scan(n, s_warp, &total);
        if (n > 0 && up_to >= want && up_to - n < want) {
            s_found[0] = 255 - tid;
            s_found[1] = want - (up_to - n);
        }
        __syncthreads();
        prefix = prefix << 8 | s_found[0];
        want = s_found[1];
        __syncthreads();
    }
    const bool any = l.keep > l.first + l.recent;
    uint32_t ties = 0, out = 0;  // so far
    for (int j0 = 0; j0 < l.len; j0 += SELECT_THREADS) {
        const int j = j0 + tid;
        bool held = j < l.len && (j < from || j >= to), tie = false;
        if (any && j >= from && j < to) {
            const uint32_t key = key_of(__ldg(p.scores + row_of(p, l, j)));
            held = key > prefix;
            tie = key == prefix;
        }
        uint32_t total;
        const uint32_t rank = block_scan(tie, s_warp, &total) - tie + ties;
        ties += total;
        held |= tie && rank < want;
        const uint32_t at = block_scan(held, s_warp, &total) - held + out;
        out += total;
        if (held) l.kept[at] = j;
    }
}

template <int D>
__global__ void __launch_bounds__(MOVE_THREADS) evict_move_kernel(const EvictParams p)
{
    constexpr int LPR = D / 16, ROWS = MOVE_THREADS / LPR;
    if (p.track[TH_SEQS] > p.n_seqs || p.track[TH_SHARED] || blockIdx.x / p.kv.heads % p.n_seqs >= p.track[TH_SEQS]) return;
    const Line l = load_line(p, blockIdx.x);
    const int part = threadIdx.x % LPR;
    for (int i0 = 0; i0 < l.keep; i0 += ROWS) {
        const int i = i0 + threadIdx.x / LPR;
        int64_t src = 0, dst = 0;
        uint4 k, v;
        uint8_t ke = 0, ve = 0;
        float w = 0.f;
        if (i < l.keep) {
            src = row_of(p, l, l.kept[i]);
            dst = row_of(p, l, i);
            k = reinterpret_cast<const uint4 *>(p.kv.k + src * D)[part];
            v = reinterpret_cast<const uint4 *>(p.kv.v + src * D)[part];
            if (part == 0) {
                ke = p.kv.k_exp[src];
                ve = p.kv.v_exp[src];
                if (p.weights) w = p.weights[src];
            }
        }
        __syncthreads();
        if (i < l.keep && src != dst) {
            reinterpret_cast<uint4 *>(p.kv.k + dst * D)[part] = k;
            reinterpret_cast<uint4 *>(p.kv.v + dst * D)[part] = v;
            if (part == 0) {
                p.kv.k_exp[dst] = ke;
                p.kv.v_exp[dst] = ve;
                if (p.weights) p.weights[dst] = w;
            }
        }
    }
}

}  // namespace
}  // namespace salt

using namespace salt;

extern "C" {

salt_status salt_attn_evict(salt_attn *a, int32_t layer, int32_t n_layers, const int32_t *keep, int32_t first, int32_t recent,
                            const float *scores, float *weights, int32_t *kept, int64_t kept_stride, salt_stream_t stream_)
try {
    NvtxRange nvtx_range("salt_attn_evict");
    if (!a) return SALT_ERR_INVALID_ARG;
    salt_ctx *ctx = a->kv->ctx;
    const KvDev &kv = a->kv->dev;
    if (first < 0 || recent < 0) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d first and %d recent tokens", first, recent);
    if (kept_stride < 0 || kept_stride >= 1ll << 31) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%lld places a line", (long long)kept_stride);
    if (a->built && a->track.n_seqs > 0 && n_layers > 0) {
        if (!keep || !scores || (!kept && kept_stride > 0)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null keep, scores or kept");
        if ((reinterpret_cast<uintptr_t>(scores) | reinterpret_cast<uintptr_t>(weights)) & 15)
            return ctx_fail(ctx, SALT_ERR_ALIGN, "scores or weights not on a 16-byte boundary");
        if ((reinterpret_cast<uintptr_t>(keep) | reinterpret_cast<uintptr_t>(kept)) & 3)
            return ctx_fail(ctx, SALT_ERR_ALIGN, "keep or kept not on a 4-byte boundary");
    }
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    bool captured;
    const salt_status st = track_enter(a, layer, n_layers, stream, &captured);
    if (st != SALT_OK || a->track.n_seqs == 0 || n_layers == 0) return st;
    EvictParams p;
    p.plan = a->plan;
    p.track = a->track.table;
    p.pages_at = a->pages_at;
    p.seq_at = a->track.seq_at;
    p.kv = kv;
    p.layer = layer;
    p.keep = keep;
    p.scores = scores;
    p.weights = weights;
    p.kept = kept;
    p.kept_stride = kept_stride;
    p.n_seqs = a->track.n_seqs;
    p.first = first;
    p.recent = recent;
    p.err = ctx_error_word(ctx);
    // (a launch's lines are numbered in 32 bits; those of a layer are 2^24 at most)
    const int64_t lines = (int64_t)p.n_seqs * kv.heads, most = std::max<int64_t>(1, (1ll << 30) / lines);
    for (int64_t l = 0; l < n_layers; l += most) {
        const unsigned n = (unsigned)(std::min<int64_t>(most, n_layers - l) * lines);
        p.layer = layer + l;
        p.kept = kept + l * lines * kept_stride;
        evict_select_kernel<<<n, SELECT_THREADS, 0, stream>>>(p);
        SALT_CUDA_OR_FAIL(ctx, cudaGetLastError());
        if (kv.dim == 128) evict_move_kernel<128><<<n, MOVE_THREADS, 0, stream>>>(p);
        else evict_move_kernel<64><<<n, MOVE_THREADS, 0, stream>>>(p);
        SALT_CUDA_OR_FAIL(ctx, cudaGetLastError());
    }
    return SALT_OK;
} catch (const std::bad_alloc &) {
    return ctx_fail(a->kv->ctx, SALT_ERR_OOM, "no host memory");
}

}  // extern "C"
