// The paged key/value cache of 8-bit floats: quantising rows as they are
// written and reading them back.
//
// A row (token, head) x of D bf16 is stored as e4m3 codes and one exponent byte
// e, x = c * 2^(e - 127).  With a = max |x| = f * 2^E (1 <= f < 2), 448 = 1.75 *
// 2^8 gives the smallest k with a <= 448 * 2^k: E - 8 where f <= 1.75, else E - 7,
// all read off the bits of a.  2^-k is a normal float for every k in [-126, 121],
// so x * 2^-k is exact and the conversion to e4m3 is the only rounding.
#include <new>

#include <cuda_fp16.h>

#include "salt_async.cuh"
#include "salt_host.cuh"
#include "salt_internal.cuh"

namespace salt {
namespace {

constexpr int KV_THREADS = 256;

__device__ __forceinline__ uint16_t e4m3x2(float lo, float hi)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t f16x2_of_e4m3x2(uint16_t c)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(r) : "h"(c));
    return r;
}

// Exponent byte of a row whose largest magnitude has the float bits `a`.
__device__ __forceinline__ uint32_t row_exp(uint32_t a)
{
    const int E = (int)(a >> 23);
    if (E == 255) return 255u;
    if (a == 0) return 0u;
    const int e = E - 8 + ((a & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 1);
}

// One row per D / 8 lanes, a lane 8 elements; rows are (token, k or v, head).
template <int D>
__global__ void __launch_bounds__(KV_THREADS) kv_write_kernel(KvDev c, int64_t layer, int n_tokens, const uint16_t *k,
                                                              int64_t k_stride, const uint16_t *v, int64_t v_stride,
                                                              const int32_t *slots, uint32_t *err)
{
    constexpr int LPR = D / 8;
    const int64_t rows = (int64_t)n_tokens * 2 * c.heads;
    const int64_t row = ((int64_t)blockIdx.x * KV_THREADS + threadIdx.x) / LPR;
    const int part = threadIdx.x % LPR;
    const bool live = row < rows;  // every lane stays for the shuffles
    const int t = live ? (int)(row / (2 * c.heads)) : 0;
    const int kh = live ? (int)(row - (int64_t)t * 2 * c.heads) : 0;
    const bool is_v = kh >= c.heads;
    const int h = is_v ? kh - c.heads : kh;
    uint4 x = make_uint4(0, 0, 0, 0);
    int slot = -1;
    if (live) {
        const uint16_t *src = (is_v ? v + (int64_t)t * v_stride : k + (int64_t)t * k_stride) + (int64_t)h * D + part * 8;
        x = __ldcs(reinterpret_cast<const uint4 *>(src));
        slot = __ldg(slots + t);
    }
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t a = 0;  // magnitudes of bf16 order like their bits
#pragma unroll
    for (int i = 0; i < 4; ++i) a = max(a, max((w[i] << 16) & 0x7fffffffu, w[i] & 0x7fff0000u));
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
    const int page = slot >> c.page_log2;
    if (slot < 0 || page >= c.n_pages) {
        if (live && slot != -1 && part == 0) atomicOr(err, SALT_DEVERR_KV_SLOT);
        return;
    }
    const uint32_t e = row_exp(a);
    const float inv = __uint_as_float(e == 255u ? 0u : (254u - max(e, 1u)) << 23);
    uint32_t codes[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t p = w[2 * i], q = w[2 * i + 1];
        codes[i] = (uint32_t)e4m3x2(__uint_as_float(p << 16) * inv, __uint_as_float(p & 0xffff0000u) * inv) |
                   (uint32_t)e4m3x2(__uint_as_float(q << 16) * inv, __uint_as_float(q & 0xffff0000u) * inv) << 16;
    }
    if (e == 255u) codes[0] = codes[1] = 0;
    const int64_t at = ((layer * c.n_pages + page) * c.heads + h) * c.page + (slot & (c.page - 1));
    *reinterpret_cast<uint2 *>((is_v ? c.v : c.k) + at * D + part * 8) = make_uint2(codes[0], codes[1]);
    if (part == 0) (is_v ? c.v_exp : c.k_exp)[at] = (uint8_t)e;
}

template <int D>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(KvDev c, int64_t layer, int n_tokens, const int32_t *slots,
                                                             uint16_t *k, int64_t k_stride, uint16_t *v,
                                                             int64_t v_stride, uint32_t *err)
{
    constexpr int LPR = D / 8;
    const int64_t rows = (int64_t)n_tokens * 2 * c.heads;
    const int64_t row = ((int64_t)blockIdx.x * KV_THREADS + threadIdx.x) / LPR;
    const int part = threadIdx.x % LPR;
    if (row >= rows) return;
    const int t = (int)(row / (2 * c.heads));
    const int kh = (int)(row - (int64_t)t * 2 * c.heads);
    const bool is_v = kh >= c.heads;
    const int h = is_v ? kh - c.heads : kh;
    const int slot = __ldg(slots + t);
    const int page = slot >> c.page_log2;
    uint32_t out[4] = {0, 0, 0, 0};
    if (slot >= 0 && page < c.n_pages) {
        const int64_t at = ((layer * c.n_pages + page) * c.heads + h) * c.page + (slot & (c.page - 1));
        const uint2 codes = __ldcs(reinterpret_cast<const uint2 *>((is_v ? c.v : c.k) + at * D + part * 8));
        const uint32_t e = (is_v ? c.v_exp : c.k_exp)[at];
        const float scale = __uint_as_float(e == 255u ? 0x7fc00000u : e << 23);
        const uint32_t two[2] = {codes.x, codes.y};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t h2 = f16x2_of_e4m3x2((uint16_t)(two[i >> 1] >> (16 * (i & 1))));
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h2));
            const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * scale, f.y * scale);
            out[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
    } else if (slot != -1 && part == 0) {
        atomicOr(err, SALT_DEVERR_KV_SLOT);
    }
    uint16_t *dst = (is_v ? v + (int64_t)t * v_stride : k + (int64_t)t * k_stride) + (int64_t)h * D + part * 8;
    __stcs(reinterpret_cast<uint4 *>(dst), make_uint4(out[0], out[1], out[2], out[3]));
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

int64_t row_blocks(const salt_kv *kv, int32_t n_tokens)
{
    const int64_t threads = (int64_t)n_tokens * 2 * kv->dev.heads * (kv->dev.dim / 8);
    return (threads + KV_THREADS - 1) / KV_THREADS;
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
    const int64_t blocks = row_blocks(kv, n_tokens);
    if (blocks > 0x7fffffff) return ctx_fail(kv->ctx, SALT_ERR_TOO_MANY_TOKENS, "%d tokens in one call", n_tokens);
    auto kernel = kv->dev.dim == 128 ? kv_write_kernel<128> : kv_write_kernel<64>;
    kernel<<<(unsigned)blocks, KV_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(
        kv->dev, layer, n_tokens, static_cast<const uint16_t *>(k), k_stride, static_cast<const uint16_t *>(v), v_stride, slots,
        ctx_error_word(kv->ctx));
    SALT_CUDA_OR_FAIL(kv->ctx, cudaGetLastError());
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
    const int64_t blocks = row_blocks(kv, n_tokens);
    if (blocks > 0x7fffffff) return ctx_fail(kv->ctx, SALT_ERR_TOO_MANY_TOKENS, "%d tokens in one call", n_tokens);
    auto kernel = kv->dev.dim == 128 ? kv_read_kernel<128> : kv_read_kernel<64>;
    kernel<<<(unsigned)blocks, KV_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(
        kv->dev, layer, n_tokens, slots, static_cast<uint16_t *>(k), k_stride, static_cast<uint16_t *>(v), v_stride,
        ctx_error_word(kv->ctx));
    SALT_CUDA_OR_FAIL(kv->ctx, cudaGetLastError());
    return SALT_OK;
}

}  // extern "C"
