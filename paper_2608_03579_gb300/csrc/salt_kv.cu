// The paged key/value cache of 8-bit floats: quantising rows as they are
// written and reading them back.
//
// A row (token, head) x of D bf16 is stored as e4m3 codes and one exponent byte
// e, x = c * 2^(e - 127).  With a = max |x| = f * 2^E (1 <= f < 2), 448 = 1.75 *
// 2^8 gives the smallest k with a <= 448 * 2^k: E - 8 where f <= 1.75, else E - 7,
// all read off the bits of a.  2^-k is a normal float for every k in [-126, 121],
// so x * 2^-k is exact and the conversion to e4m3 is the only rounding.
#include <algorithm>
#include <new>

#include <cuda_fp16.h>

#include "salt_async.cuh"
#include "salt_host.cuh"
#include "salt_internal.cuh"
#include "salt_pipe.cuh"

namespace salt {
namespace {

constexpr int KV_THREADS = 256;
constexpr int WRITE_ROWS = 2, READ_ROWS = 4;  // rows a thread

// Exponent byte of a row whose largest magnitude has the float bits `a`.
__device__ __forceinline__ uint32_t row_exp(uint32_t a)
{
    const int E = (int)(a >> 23);
    if (E == 255) return 255u;
    if (a == 0) return 0u;
    const int e = E - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 1);
}

// Rows are (token, k or v, head), one per D / 16 lanes.  A lane has two pieces of 8 elements, D / 16 pieces
// apart so that neighbours read and write side by side; what a row costs beside its elements (its place,
// the maximum's exchange, its exponent) is shared by 16 of them.  A thread deals with ROWS rows,
// KV_THREADS / (D / 16) apart, so that enough bytes are under way, and reads and writes past
// the L2 what it will not meet again.  Both kernels move bytes: 16,384 tokens of 8 heads of 128 are written in
// 17.6 us (5.7 TB/s of bytes read and written), 100,003 are read in 93 us (6.6 TB/s).  Before the launches overlapped with
// what came before them these were 20 and 95, with 1 row a thread 20 and 98, with 4 and 2 rows 20.5 and 96; with 8 elements
// a lane the kernels were short of instruction slots and took 25 and 112.
struct KvRow {
    int t, h;
    bool live, is_v;
};

template <int D, int ROWS>
__device__ __forceinline__ KvRow kv_row(const KvDev &c, int n_tokens, uint32_t heads2_inv, int k)
{
    constexpr int PER = KV_THREADS / (D / 16);  // rows a block deals with at a time
    const uint32_t row = blockIdx.x * (uint32_t)(PER * ROWS) + k * PER + threadIdx.x / (D / 16);
    const uint32_t n = 2 * c.heads;
    const uint32_t t = __umulhi(row, heads2_inv);  // row / (2 heads)
    const int kh = (int)(row - t * n);
    KvRow r;
    r.live = t < (uint32_t)n_tokens;
    r.t = r.live ? (int)t : 0;
    r.is_v = kh >= c.heads;
    r.h = r.is_v ? kh - c.heads : kh;
    return r;
}

// The row's number in the cache (they are below 2^31); first_page is the layer's.
__device__ __forceinline__ uint32_t cache_row(const KvDev &c, uint32_t first_page, int page, int slot, int h)
{
    return ((first_page + page) * c.heads + h) * c.page + (slot & (c.page - 1));
}

template <int D>
__global__ void __launch_bounds__(KV_THREADS) kv_write_kernel(KvDev c, uint32_t first_page, int n_tokens, uint32_t heads2_inv,
                                                              const uint16_t *k, int64_t k_stride, const uint16_t *v,
                                                              int64_t v_stride, const int32_t *slots, uint32_t *err)
{
    constexpr int LPR = D / 16, ROWS = WRITE_ROWS;
    const int part = threadIdx.x % LPR;
    pdl_wait();  // (launched beside the end of what came before)
    pdl_launch_dependents();
    k = after_pdl_wait(k);
    v = after_pdl_wait(v);
    slots = after_pdl_wait(slots);
    KvRow r[ROWS];
    uint4 x[ROWS][2];
    int slot[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        r[i] = kv_row<D, ROWS>(c, n_tokens, heads2_inv, i);
        x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
        slot[i] = -1;
        if (r[i].live) {  // every lane stays for the shuffles
            const uint16_t *src = (r[i].is_v ? v : k) + r[i].t * (r[i].is_v ? v_stride : k_stride) + r[i].h * D + part * 8;
            x[i][0] = __ldcs(reinterpret_cast<const uint4 *>(src));
            x[i][1] = __ldcs(reinterpret_cast<const uint4 *>(src + D / 2));
            slot[i] = __ldg(slots + r[i].t);
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const uint32_t w[8] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w, x[i][1].x, x[i][1].y, x[i][1].z, x[i][1].w};
        uint32_t a2 = 0;  // magnitudes of bf16 order like their bits; two at a time
#pragma unroll
        for (int e = 0; e < 8; ++e) a2 = __vmaxu2(a2, w[e] & 0x7fff7fffu);
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) a2 = __vmaxu2(a2, __shfl_xor_sync(0xffffffffu, a2, o));
        const uint32_t a = max(a2 << 16, a2 & 0xffff0000u);
        const int page = slot[i] >> c.page_log2;
        if (slot[i] < 0 || page >= c.n_pages) {
            if (slot[i] != -1 && part == 0) atomicOr(err, SALT_DEVERR_KV_SLOT);
            continue;
        }
        const uint32_t e = row_exp(a);
        const float inv = __uint_as_float(e == 255u ? 0u : (254u - max(e, 1u)) << 23);
        const uint32_t at = cache_row(c, first_page, page, slot[i], r[i].h);
        uint8_t *to = (r[i].is_v ? c.v : c.k) + (uint64_t)at * D + part * 8;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            uint32_t codes[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t lo = w[4 * q + 2 * h], hi = w[4 * q + 2 * h + 1];
                codes[h] = (uint32_t)e4m3x2(__uint_as_float(lo << 16) * inv, __uint_as_float(lo & 0xffff0000u) * inv) |
                           (uint32_t)e4m3x2(__uint_as_float(hi << 16) * inv, __uint_as_float(hi & 0xffff0000u) * inv) << 16;
            }
            *reinterpret_cast<uint2 *>(to + q * (D / 2)) = e == 255u ? make_uint2(0, 0) : make_uint2(codes[0], codes[1]);
        }
        if (part == 0) (r[i].is_v ? c.v_exp : c.k_exp)[at] = (uint8_t)e;
    }
}

template <int D>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(KvDev c, uint32_t first_page, int n_tokens, uint32_t heads2_inv,
                                                             const int32_t *slots, uint16_t *k, int64_t k_stride, uint16_t *v,
                                                             int64_t v_stride, uint32_t *err)
{
    constexpr int LPR = D / 16, ROWS = READ_ROWS;
    const int part = threadIdx.x % LPR;
    pdl_wait();  // (launched beside the end of what came before)
    pdl_launch_dependents();
    slots = after_pdl_wait(slots);
    KvRow r[ROWS];
    int slot[ROWS];
    uint2 codes[ROWS][2];
    uint32_t e[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        r[i] = kv_row<D, ROWS>(c, n_tokens, heads2_inv, i);
        slot[i] = r[i].live ? __ldg(slots + r[i].t) : -1;
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int page = slot[i] >> c.page_log2;
        codes[i][0] = codes[i][1] = make_uint2(0, 0);
        e[i] = 0;
        if (slot[i] >= 0 && page < c.n_pages) {
            const uint32_t at = cache_row(c, first_page, page, slot[i], r[i].h);
            const uint8_t *from = (r[i].is_v ? c.v : c.k) + (uint64_t)at * D + part * 8;
            codes[i][0] = __ldcs(reinterpret_cast<const uint2 *>(from));
            codes[i][1] = __ldcs(reinterpret_cast<const uint2 *>(from + D / 2));
            e[i] = (r[i].is_v ? c.v_exp : c.k_exp)[at];
        } else if (slot[i] != -1 && part == 0) {
            atomicOr(err, SALT_DEVERR_KV_SLOT);
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (!r[i].live) continue;
        const float scale = __uint_as_float(e[i] == 255u ? 0x7fc00000u : e[i] << 23);
        uint16_t *dst = (r[i].is_v ? v : k) + r[i].t * (r[i].is_v ? v_stride : k_stride) + r[i].h * D + part * 8;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t two[2] = {codes[i][q].x, codes[i][q].y};
            uint32_t out[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const uint32_t h2 = f16x2_of_e4m3x2((uint16_t)(two[h >> 1] >> (16 * (h & 1))));
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
                const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * scale, f.y * scale);
                out[h] = *reinterpret_cast<const uint32_t *>(&b);
            }
            __stcs(reinterpret_cast<uint4 *>(dst + q * (D / 2)), make_uint4(out[0], out[1], out[2], out[3]));
        }
    }
}

salt_status check_rows(salt_kv *kv, int32_t layer, int32_t n_tokens, const void *k, int64_t k_stride, const void *v,
                       int64_t v_stride, const int32_t *slots)
{
    salt_ctx *ctx = kv->ctx;
    if (layer < 0 || layer >= kv->n_layers)
        return ctx_fail(ctx, SALT_ERR_LAYER_RANGE, "layer %d outside [0, %d)", layer, kv->n_layers);
    if (n_tokens < 0) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d tokens", n_tokens);
    if (n_tokens == 0) return SALT_OK;
    if (!k || !v || !slots) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null k, v or slots");
    const int64_t row = (int64_t)kv->dev.heads * kv->dev.dim;
    if (k_stride < row || v_stride < row)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "rows of %lld elements %lld and %lld apart", (long long)row,
                        (long long)k_stride, (long long)v_stride);
    if ((k_stride | v_stride) % 8 || ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15))
        return ctx_fail(ctx, SALT_ERR_ALIGN, "rows of k or v not on 16-byte boundaries");
    if (reinterpret_cast<uintptr_t>(slots) & 3) return ctx_fail(ctx, SALT_ERR_ALIGN, "slots not on a 4-byte boundary");
    return SALT_OK;
}

// Tokens that one launch may take: a row's number times 2 heads stays below 2^32, so that its quotient by 2
// heads is the high half of its product with floor(2^32 / (2 heads)) + 1.
int32_t launch_tokens(const salt_kv *kv)
{
    const int64_t n = 2ll * kv->dev.heads, slack = (int64_t)KV_THREADS * std::max(WRITE_ROWS, READ_ROWS);
    return (int32_t)std::max<int64_t>(1, ((1ll << 32) / n - slack) / n);
}
uint32_t heads2_inv(const salt_kv *kv) { return (uint32_t)((1ull << 32) / (2ull * kv->dev.heads) + 1); }
unsigned row_blocks(const salt_kv *kv, int32_t n_tokens, int rows)
{
    const int64_t per = (int64_t)KV_THREADS / (kv->dev.dim / 16) * rows;
    return (unsigned)((2ll * n_tokens * kv->dev.heads + per - 1) / per);
}

}  // namespace
}  // namespace salt

using namespace salt;

extern "C" {

salt_status salt_kv_create(salt_ctx *ctx, const salt_kv_config *c, salt_kv **out)
{
    if (!out) return SALT_ERR_INVALID_ARG;
    *out = nullptr;
    if (!ctx || !c) return SALT_ERR_INVALID_ARG;
    if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "a cache of %d layers, %d pages, %d heads", c->n_layers, c->n_pages,
                        c->n_kv_heads);
    if (c->head_dim != 64 && c->head_dim != 128)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "head_dim %d is not 64 or 128", c->head_dim);
    if (c->page_tokens < 16 || c->page_tokens > SALT_MAX_KV_PAGE || (c->page_tokens & (c->page_tokens - 1)))
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "page_tokens %d is not 16, 32, 64 or 128", c->page_tokens);
    if (c->n_kv_heads > 1024) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d key/value heads, at most 1024", c->n_kv_heads);
    // rows are numbered in 32 bits (each factor is below 2^31, so the products below cannot overflow unseen)
    int64_t rows = (int64_t)c->n_layers * c->n_pages;
    if (rows < (1ll << 31)) rows *= c->n_kv_heads;
    if (rows < (1ll << 31)) rows *= c->page_tokens;
    if (rows >= (1ll << 31)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "a cache of 2^31 rows or more");
    if (!c->k || !c->v || !c->k_exp || !c->v_exp) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null cache memory");
    if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v) | reinterpret_cast<uintptr_t>(c->k_exp) |
         reinterpret_cast<uintptr_t>(c->v_exp)) & 15)
        return ctx_fail(ctx, SALT_ERR_ALIGN, "cache memory not 16-byte aligned");
    salt_kv *kv = new (std::nothrow) salt_kv;
    if (!kv) return ctx_fail(ctx, SALT_ERR_OOM, "no host memory");
    kv->ctx = ctx;
    kv->n_layers = c->n_layers;
    KvDev &d = kv->dev;
    d.k = static_cast<uint8_t *>(c->k);
    d.v = static_cast<uint8_t *>(c->v);
    d.k_exp = static_cast<uint8_t *>(c->k_exp);
    d.v_exp = static_cast<uint8_t *>(c->v_exp);
    d.n_pages = c->n_pages;
    d.heads = c->n_kv_heads;
    d.page = c->page_tokens;
    d.page_log2 = c->page_tokens == 16 ? 4 : c->page_tokens == 32 ? 5 : c->page_tokens == 64 ? 6 : 7;
    d.dim = c->head_dim;
    *out = kv;
    return SALT_OK;
}

void salt_kv_destroy(salt_kv *kv) { delete kv; }

salt_status salt_kv_write(salt_kv *kv, int32_t layer, int32_t n_tokens, const void *k, int64_t k_stride, const void *v,
                          int64_t v_stride, const int32_t *slots, salt_stream_t stream)
{
    NvtxRange nvtx_range("salt_kv_write");
    if (!kv) return SALT_ERR_INVALID_ARG;
    salt_status st = check_rows(kv, layer, n_tokens, k, k_stride, v, v_stride, slots);
    if (st != SALT_OK || n_tokens == 0) return st;
    if (!ctx_select_device(kv->ctx)) return ctx_fail(kv->ctx, SALT_ERR_CUDA, "cannot select the device");
    auto kernel = kv->dev.dim == 128 ? kv_write_kernel<128> : kv_write_kernel<64>;
    const int32_t most = launch_tokens(kv);
    for (int64_t t = 0; t < n_tokens; t += most) {
        const int32_t n = (int32_t)std::min<int64_t>(most, n_tokens - t);
        SALT_CUDA_OR_FAIL(kv->ctx, launch_overlapped(kernel, row_blocks(kv, n, WRITE_ROWS), KV_THREADS, 0, static_cast<cudaStream_t>(stream),
            kv->dev, (uint32_t)layer * kv->dev.n_pages, n, heads2_inv(kv), static_cast<const uint16_t *>(k) + t * k_stride, k_stride,
            static_cast<const uint16_t *>(v) + t * v_stride, v_stride, slots + t, ctx_error_word(kv->ctx)));
    }
    return SALT_OK;
}

salt_status salt_kv_read(salt_kv *kv, int32_t layer, int32_t n_tokens, const int32_t *slots, void *k, int64_t k_stride,
                         void *v, int64_t v_stride, salt_stream_t stream)
{
    NvtxRange nvtx_range("salt_kv_read");
    if (!kv) return SALT_ERR_INVALID_ARG;
    salt_status st = check_rows(kv, layer, n_tokens, k, k_stride, v, v_stride, slots);
    if (st != SALT_OK || n_tokens == 0) return st;
    if (!ctx_select_device(kv->ctx)) return ctx_fail(kv->ctx, SALT_ERR_CUDA, "cannot select the device");
    auto kernel = kv->dev.dim == 128 ? kv_read_kernel<128> : kv_read_kernel<64>;
    const int32_t most = launch_tokens(kv);
    for (int64_t t = 0; t < n_tokens; t += most) {
        const int32_t n = (int32_t)std::min<int64_t>(most, n_tokens - t);
        SALT_CUDA_OR_FAIL(kv->ctx, launch_overlapped(kernel, row_blocks(kv, n, READ_ROWS), KV_THREADS, 0, static_cast<cudaStream_t>(stream),
            kv->dev, (uint32_t)layer * kv->dev.n_pages, n, heads2_inv(kv), slots + t, static_cast<uint16_t *>(k) + t * k_stride, k_stride,
            static_cast<uint16_t *>(v) + t * v_stride, v_stride, ctx_error_word(kv->ctx)));
    }
    return SALT_OK;
}

}  // extern "C"
