// Norms of queries and keys, head by head, with the rotation to their
// positions, on the way into the cache or back into bf16 rows.
//
//     y = x * (mean(x^2) + eps)^(-1/2) * (w + offset)
//     (a, b) -> scale * (a cos t - b sin t, b cos t + a sin t),   t = position * inv_freq[pair]
//
// Angles are counted in turns: a pair's frequency is a fraction of a turn in 64 bits, so that the low 64 bits of
// its product with the position are the angle itself, whole turns gone, to 2^-33 of a turn at any position (a
// product in fp32 has lost 0.01 radians at position 200,000).  The sum of squares and everything after it is fp32,
// rounded once: to bf16, or to the cache's codes (keys are not rounded to bf16 between).
//
// A row (token, head) goes to D / 16 lanes, 16 elements each in two pieces of 8: where pairs are (i, i + rot / 2)
// the pieces are rot / 2 elements apart, so that a lane has both elements of its pairs.  A warp deals with rows of one token,
// whose sines and cosines it computes once, two pairs a lane, and hands round through shared memory.
//
// 16,384 tokens with 32 and 8 heads of 128, norms, the keys and values into the cache: 60 us, 6.1 TB/s (90% of a copy's rate).  Rows
// come by copies of 16 bytes a lane into shared memory, two passes ahead of those at hand (loaded into registers, 64 of them for four
// CTAs an SM: 73 us), and issue slots are the rest: weights widened once a CTA and codes' maxima for keys and values alone
// gave 6 of those us.  Warps that go on from token to token took 62, deeper copies 5 to 9 more, three passes no less.
// 64 decoding tokens: 3.2 us, a launch and a row's chain of loads and sums.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>

#include "salt_async.cuh"
#include "salt_attn.cuh"
#include "salt_host.cuh"
#include "salt_internal.cuh"
#include "salt_kvrow.cuh"
#include "salt_pipe.cuh"

struct salt_rope {
    salt_ctx *ctx;
    int dim, rot, n_sm;
    bool mixed;
    float scale, eps, offset;
    uint64_t freq[64];  // turns a position, in units of 2^-64
};

namespace salt {
namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_WARPS = ROPE_THREADS / 32;
constexpr int ROPE_ROWS = 2;  // rows a lane deals with side by side

struct RopeParams {
    const uint16_t *q, *k, *v, *q_norm, *k_norm;
    uint16_t *q_out, *k_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
    const int32_t *positions, *slots;
    int32_t n_tokens, n_heads, n_kv_heads, rot, rows, passes, splits;  // rows a token, passes of a warp over them and warps that share those
    float scale, eps, offset;
    KvDev kv;
    uint32_t first_page;
    uint32_t *err;
    uint64_t freq[64];
};

__device__ __forceinline__ void unpack8(const uint4 &x, float2 *y)
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack8(const float2 *y)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(y[i].x, y[i].y);
        w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int LANES>
__device__ __forceinline__ float sum_lanes(float x)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

template <int D, bool WRITE, bool MIXED>
__global__ void __launch_bounds__(ROPE_THREADS, 4) rope_kernel(const __grid_constant__ RopeParams p)
{
    constexpr int LPR = D / 16, RPW = 32 / LPR;  // lanes a row, rows a warp deals with at a time
    __shared__ __align__(16) float2 s_turn[ROPE_WARPS][64];
    __shared__ uint4 s_rows[2][ROPE_ROWS][2][ROPE_THREADS];  // a lane's pieces of the rows at hand and of the next ones
    __shared__ float4 s_norm[2][2][D / 8];  // weights of query and key heads, offset added: of 8 elements the first and the last 4
    // (the warp's number from a shuffle: loops by it are known to be a warp's then, and the shuffles in them are quick)
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, part = lane % LPR;
    const uint32_t task = blockIdx.x * ROPE_WARPS + warp;
    const uint32_t token = task / (uint32_t)p.splits;
    const int t = (int)token, split = (int)(task - token * p.splits);
    // the lane's pieces of a row, in units of 8 elements, and whether they are rotated
    const int n_rot = p.rot / 16;
    const bool turned0 = MIXED ? part < 2 * n_rot : part < n_rot;
    const bool turned1 = MIXED ? part + LPR < 2 * n_rot : turned0;
    const int c0 = MIXED || turned0 ? part : part + n_rot;
    const int c1 = MIXED ? part + LPR : turned0 ? part + n_rot : part + LPR;
    const uint64_t f0 = p.freq[lane], f1 = p.freq[lane + 32];
    pdl_wait();  // (launched beside the end of what came before)
    pdl_launch_dependents();
    if (p.q_norm || p.k_norm) {
        for (int i = threadIdx.x; i < 2 * D / 4; i += ROPE_THREADS) {
            const uint16_t *norm = after_pdl_wait(i < D / 4 ? p.q_norm : p.k_norm);
            if (!norm) continue;
            const int e = i % (D / 4);
            const uint2 x = __ldg(reinterpret_cast<const uint2 *>(norm) + e);
            s_norm[i / (D / 4)][e & 1][e / 2] = make_float4(__uint_as_float(x.x << 16) + p.offset, __uint_as_float(x.x & 0xffff0000u) + p.offset,
                                                            __uint_as_float(x.y << 16) + p.offset, __uint_as_float(x.y & 0xffff0000u) + p.offset);
        }
        __syncthreads();
    }
    if (token >= (uint32_t)p.n_tokens) return;
    const int32_t *positions = after_pdl_wait(p.positions), *slots = WRITE ? after_pdl_wait(p.slots) : nullptr;
    const uint16_t *q = after_pdl_wait(p.q), *k = after_pdl_wait(p.k), *v = WRITE ? after_pdl_wait(p.v) : nullptr;
    const int H = p.n_heads, KV = p.n_kv_heads;
    const int pass1 = min((p.rows + RPW - 1) / RPW, (split + 1) * p.passes);
    // Copies the lane's pieces of a pass's rows to shared memory, while the rows before them are dealt with.  (Rows past the
    // token's are zeros: every lane stays for the shuffles.)
    auto fetch = [&](int pass, int buf) {
#pragma unroll
        for (int i = 0; i < ROPE_ROWS; ++i) {
            const int r = (pass + i) * RPW + lane / LPR, row = min(r, p.rows - 1);
            const bool there = pass + i < pass1 && r < p.rows;
            const uint16_t *src = row < H ? q + t * p.q_stride + row * D
                                  : row < H + KV ? k + t * p.k_stride + (row - H) * D
                                                 : v + t * p.v_stride + (row - H - KV) * D;
            cp_async16(smem_u32(&s_rows[buf][i][0][threadIdx.x]), reinterpret_cast<const uint4 *>(src) + c0, there);
            cp_async16(smem_u32(&s_rows[buf][i][1][threadIdx.x]), reinterpret_cast<const uint4 *>(src) + c1, there);
        }
        cp_async_commit();
    };
    fetch(split * p.passes, 0);
    const int slot = WRITE ? __ldg(slots + t) : -1, page = WRITE ? slot >> p.kv.page_log2 : 0;
    const bool stored = WRITE && slot >= 0 && page < p.kv.n_pages;
    if (WRITE && split == 0 && lane == 0 && !stored && slot != -1) atomicOr(p.err, SALT_DEVERR_KV_SLOT);
    // sines and cosines of the lane's pairs, two at a time
    float2 c[4], s[4];
    {
        const int64_t at = __ldg(positions + t);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint64_t turns = (uint64_t)at * (i ? f1 : f0);
            // in half turns, [-1, 1); what fp32 leaves of them turns the pair of sine and cosine (rounded to fp32 alone an angle is
            // up to 9e-8 off, more than any of a row's other roundings)
            const float at32 = (float)(int32_t)(turns >> 32);
            const float rest = (float)(int64_t)(turns - ((uint64_t)(int64_t)at32 << 32)) * (0x1p-63f * 3.14159265f);
            float sn, cs;
            sincospif(at32 * 0x1p-31f, &sn, &cs);
            s_turn[warp][lane + 32 * i] = make_float2(fmaf(-rest, sn, cs) * p.scale, fmaf(rest, cs, sn) * p.scale);
        }
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const int pair = MIXED ? 4 * (e < 4 ? c0 : c1) + (e & 3) : part * 8 + e;
            const float4 x = *reinterpret_cast<const float4 *>(&s_turn[warp][pair & 63]);
            c[e / 2] = make_float2(x.x, x.z);
            s[e / 2] = make_float2(x.y, x.w);
        }
    }
    int buf = 0;
    for (int pass = split * p.passes; pass < pass1; pass += ROPE_ROWS, buf ^= 1) {
        asm volatile("" ::: "memory");  // (what is fetched takes the place of rows that were read)
        fetch(pass + ROPE_ROWS, buf ^ 1);
        cp_async_wait<1>();
#pragma unroll
        for (int i = 0; i < ROPE_ROWS; ++i) {
            const int r = (pass + i) * RPW + lane / LPR, row = pass + i < pass1 && r < p.rows ? r : -1;
            const bool is_q = row < H, is_v = row >= H + KV;
            float2 y[8];
            unpack8(s_rows[buf][i][0][threadIdx.x], y);
            unpack8(s_rows[buf][i][1][threadIdx.x], y + 4);
            const uint16_t *norm = is_q ? p.q_norm : p.k_norm;
            if (p.q_norm || p.k_norm) {
                float2 s2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int e = 0; e < 8; ++e) s2[e & 1] = fma2(y[e], y[e], s2[e & 1]);
                const float ss = sum_lanes<LPR>((s2[0].x + s2[0].y) + (s2[1].x + s2[1].y));
                float r = rsqrtf(ss * (1.f / D) + p.eps);
                if (__any_sync(0xffffffffu, !(ss <= FLT_MAX))) {  // squares past fp32's range: the row scaled down
                    const float down = 0x1p-70f;
                    float s1 = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) s1 = fmaf(y[e].x * down, y[e].x * down, fmaf(y[e].y * down, y[e].y * down, s1));
                    s1 = sum_lanes<LPR>(s1);
                    if (!(ss <= FLT_MAX)) r = rsqrtf(s1 * (1.f / D)) * down;
                }
                if (norm && !is_v && row >= 0) {
                    float2 w[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float4 x = s_norm[is_q ? 0 : 1][e & 1][e < 2 ? c0 : c1];
                        w[2 * e] = make_float2(x.x, x.y);
                        w[2 * e + 1] = make_float2(x.z, x.w);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = mul2(mul2(y[e], make_float2(r, r)), w[e]);
                }
            }
            if (!is_v) {  // (what is not rotated stays as it is, zeros' signs and all)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (MIXED) {
                        if (!(e < 2 ? turned0 : turned1)) continue;
                        const float2 a = y[2 * e], b = y[2 * e + 1];
                        y[2 * e] = make_float2(fmaf(a.x, c[e].x, -(a.y * s[e].x)), fmaf(a.y, c[e].x, a.x * s[e].x));
                        y[2 * e + 1] = make_float2(fmaf(b.x, c[e].y, -(b.y * s[e].y)), fmaf(b.y, c[e].y, b.x * s[e].y));
                    } else if (turned0) {
                        const float2 a = y[e], b = y[4 + e], n = make_float2(-s[e].x, -s[e].y);
                        y[e] = fma2(a, c[e], mul2(b, n));
                        y[4 + e] = fma2(b, c[e], mul2(a, s[e]));
                    }
                }
            }
            if (WRITE && (pass + i) * RPW + RPW > H) {  // (any of the warp's rows)
                uint32_t a = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) a = max(a, max(__float_as_uint(y[e].x) & 0x7fffffffu, __float_as_uint(y[e].y) & 0x7fffffffu));
#pragma unroll
                for (int o = LPR / 2; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
                if (!is_q && stored) {
                    const uint32_t e = row_exp(a > 0x7f800000u ? 0x7f800000u : a);
                    const float inv = row_inv(e);
                    const uint32_t at = cache_row(p.kv, p.first_page, page, slot, is_v ? row - H - KV : row - H);
                    uint8_t *to = (is_v ? p.kv.v : p.kv.k) + (uint64_t)at * D;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float2 *z = y + 4 * h;
                        uint2 codes;
                        codes.x = (uint32_t)e4m3x2(z[0].x * inv, z[0].y * inv) | (uint32_t)e4m3x2(z[1].x * inv, z[1].y * inv) << 16;
                        codes.y = (uint32_t)e4m3x2(z[2].x * inv, z[2].y * inv) | (uint32_t)e4m3x2(z[3].x * inv, z[3].y * inv) << 16;
                        *(reinterpret_cast<uint2 *>(to) + (h ? c1 : c0)) = e == 255u ? make_uint2(0, 0) : codes;
                    }
                    if (part == 0) (is_v ? p.kv.v_exp : p.kv.k_exp)[at] = (uint8_t)e;
                }
            }
            if (row >= 0 && (is_q || !WRITE)) {
                uint16_t *dst = is_q ? p.q_out + t * p.q_out_stride + row * D : p.k_out + t * p.k_out_stride + (row - H) * D;
                __stcs(reinterpret_cast<uint4 *>(dst) + c0, pack8(y));
                __stcs(reinterpret_cast<uint4 *>(dst) + c1, pack8(y + 4));
            }
        }
    }
    cp_async_wait<0>();
}

salt_status check_heads(salt_rope *r, const char *what, const void *x, int64_t stride, int heads)
{
    if (heads == 0) return SALT_OK;
    if (!x) return ctx_fail(r->ctx, SALT_ERR_INVALID_ARG, "null %s", what);
    if (stride < (int64_t)heads * r->dim)
        return ctx_fail(r->ctx, SALT_ERR_INVALID_ARG, "%s: rows of %d elements %lld apart", what, heads * r->dim, (long long)stride);
    if (stride % 8 || (reinterpret_cast<uintptr_t>(x) & 15))
        return ctx_fail(r->ctx, SALT_ERR_ALIGN, "rows of %s not on 16-byte boundaries", what);
    return SALT_OK;
}

salt_status check_common(salt_rope *r, int32_t n_tokens, int32_t n_heads, int32_t n_kv_heads, const void *q_norm, const void *k_norm,
                         const int32_t *positions)
{
    if (n_tokens < 0) return ctx_fail(r->ctx, SALT_ERR_INVALID_ARG, "%d tokens", n_tokens);
    if (n_heads < 0 || n_kv_heads < 0 || n_heads > 65536 || n_kv_heads > 1024 || n_heads + n_kv_heads == 0)
        return ctx_fail(r->ctx, SALT_ERR_INVALID_ARG, "%d query heads, %d key heads", n_heads, n_kv_heads);
    if ((reinterpret_cast<uintptr_t>(q_norm) | reinterpret_cast<uintptr_t>(k_norm)) & 15)
        return ctx_fail(r->ctx, SALT_ERR_ALIGN, "norm weights not on a 16-byte boundary");
    if (n_tokens > 0 && !positions) return ctx_fail(r->ctx, SALT_ERR_INVALID_ARG, "null positions");
    if (reinterpret_cast<uintptr_t>(positions) & 3) return ctx_fail(r->ctx, SALT_ERR_ALIGN, "positions not on a 4-byte boundary");
    return SALT_OK;
}

template <bool WRITE>
salt_status launch_rope(salt_rope *r, RopeParams &p, cudaStream_t stream)
{
    salt_ctx *ctx = r->ctx;
    if (!ctx_select_device(ctx)) return ctx_fail(ctx, SALT_ERR_CUDA, "cannot select the device");
    p.rot = r->rot;
    p.scale = r->scale;
    p.eps = r->eps;
    p.offset = r->offset;
    p.err = ctx_error_word(ctx);
    std::copy(r->freq, r->freq + 64, p.freq);
    const int per = 32 / (r->dim / 16), all = (p.rows + per - 1) / per;  // passes of a token
    // A warp takes all of a token's passes where there are tokens enough to fill the SMs (its sines are
    // computed once), fewer where not, two by two.
    const int64_t fill = r->n_sm * 32;
    const int64_t few = std::max<int64_t>(1, (int64_t)p.n_tokens * all / fill);
    p.passes = (int)std::min<int64_t>(all, (few + ROPE_ROWS - 1) / ROPE_ROWS * ROPE_ROWS);
    p.splits = (all + p.passes - 1) / p.passes;
    const auto kernel = r->dim == 128 ? (r->mixed ? rope_kernel<128, WRITE, true> : rope_kernel<128, WRITE, false>)
                                      : (r->mixed ? rope_kernel<64, WRITE, true> : rope_kernel<64, WRITE, false>);
    // (a token has one warp unless there are few: the warps' numbers fit 32 bits, those of the last CTA past the tokens too)
    SALT_CUDA_OR_FAIL(ctx, launch_overlapped(kernel, (unsigned)(((int64_t)p.n_tokens * p.splits + ROPE_WARPS - 1) / ROPE_WARPS), ROPE_THREADS, 0,
                                             stream, p));
    return SALT_OK;
}

}  // namespace
}  // namespace salt

using namespace salt;

extern "C" {

salt_status salt_rope_create(salt_ctx *ctx, const salt_rope_config *c, salt_rope **out)
{
    if (!out) return SALT_ERR_INVALID_ARG;
    *out = nullptr;
    if (!ctx || !c) return SALT_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "head_dim %d is not 64 or 128", c->head_dim);
    if (c->rot_dim < 0 || c->rot_dim > c->head_dim || c->rot_dim % 16)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "rot_dim %d is not a multiple of 16 up to head_dim", c->rot_dim);
    if (c->rot_dim > 0 && !c->inv_freq) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null inv_freq");
    if (!std::isfinite(c->scale) || !std::isfinite(c->norm_offset))
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "scale or norm_offset is not finite");
    if (!std::isfinite(c->eps) || c->eps < FLT_MIN) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "eps is not a positive normal number");
    for (int i = 0; i < c->rot_dim / 2; ++i)
        if (!(std::fabs(c->inv_freq[i]) <= 6.2831853071795864))
            return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "inv_freq[%d] is more than a turn a position", i);
    int n_sm = 0;
    SALT_CUDA_OR_FAIL(ctx, cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, ctx_device(ctx)));
    salt_rope *r = new (std::nothrow) salt_rope;
    if (!r) return ctx_fail(ctx, SALT_ERR_OOM, "no host memory");
    r->ctx = ctx;
    r->n_sm = n_sm;
    r->dim = c->head_dim;
    r->rot = c->rot_dim;
    r->mixed = c->interleaved != 0;
    r->scale = c->scale;
    r->eps = c->eps;
    r->offset = c->norm_offset;
    for (int i = 0; i < 64; ++i) {
        // turns = inv_freq / (2 pi) as a sum of two doubles (one alone is 2^-25 of a turn off at position 2^31)
        const double inv_2pi = 0.15915494309189535, inv_2pi_low = -9.839338337591243e-18;
        const double given = i < c->rot_dim / 2 ? c->inv_freq[i] : 0.0, f = std::fabs(given), turns = f * inv_2pi;
        const double low = std::fma(f, inv_2pi, -turns) + f * inv_2pi_low;
        const double part = (turns - std::floor(turns)) * 4294967296.0;  // [0, 2^32)
        const double hi = std::floor(part);
        const uint64_t bits = ((uint64_t)hi << 32) + (uint64_t)std::llrint((part - hi) * 4294967296.0 + low * 0x1p64);
        r->freq[i] = given < 0 ? 0 - bits : bits;
    }
    *out = r;
    return SALT_OK;
}

void salt_rope_destroy(salt_rope *r) { delete r; }

salt_status salt_rope_apply(salt_rope *r, int32_t n_tokens, const void *q, int64_t q_stride, int32_t n_heads, const void *k,
                            int64_t k_stride, int32_t n_kv_heads, const void *q_norm, const void *k_norm, const int32_t *positions,
                            void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, salt_stream_t stream)
{
    NvtxRange nvtx_range("salt_rope_apply");
    if (!r) return SALT_ERR_INVALID_ARG;
    salt_status st = check_common(r, n_tokens, n_heads, n_kv_heads, q_norm, k_norm, positions);
    if (st != SALT_OK || n_tokens == 0) return st;
    if ((st = check_heads(r, "q", q, q_stride, n_heads)) != SALT_OK) return st;
    if ((st = check_heads(r, "k", k, k_stride, n_kv_heads)) != SALT_OK) return st;
    if ((st = check_heads(r, "q_out", q_out, q_out_stride, n_heads)) != SALT_OK) return st;
    if ((st = check_heads(r, "k_out", k_out, k_out_stride, n_kv_heads)) != SALT_OK) return st;
    RopeParams p = {};
    p.q = static_cast<const uint16_t *>(q);
    p.k = static_cast<const uint16_t *>(k);
    p.q_norm = static_cast<const uint16_t *>(q_norm);
    p.k_norm = static_cast<const uint16_t *>(k_norm);
    p.q_out = static_cast<uint16_t *>(q_out);
    p.k_out = static_cast<uint16_t *>(k_out);
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.q_out_stride = q_out_stride;
    p.k_out_stride = k_out_stride;
    p.positions = positions;
    p.n_tokens = n_tokens;
    p.n_heads = n_heads;
    p.n_kv_heads = n_kv_heads;
    p.rows = n_heads + n_kv_heads;
    return launch_rope<false>(r, p, static_cast<cudaStream_t>(stream));
}

salt_status salt_rope_write(salt_rope *r, salt_kv *kv, int32_t layer, int32_t n_tokens, const void *q, int64_t q_stride, int32_t n_heads,
                            const void *k, int64_t k_stride, const void *v, int64_t v_stride, const void *q_norm, const void *k_norm,
                            const int32_t *positions, const int32_t *slots, void *q_out, int64_t q_out_stride, salt_stream_t stream)
{
    NvtxRange nvtx_range("salt_rope_write");
    if (!r || !kv) return SALT_ERR_INVALID_ARG;
    salt_ctx *ctx = r->ctx;
    if (kv->ctx != ctx) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "the cache belongs to another context");
    if (kv->dev.dim != r->dim) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "heads of %d in a cache of %d", r->dim, kv->dev.dim);
    if (layer < 0 || layer >= kv->n_layers)
        return ctx_fail(ctx, SALT_ERR_LAYER_RANGE, "layer %d outside [0, %d)", layer, kv->n_layers);
    const int KV = kv->dev.heads;
    salt_status st = check_common(r, n_tokens, n_heads, KV, q_norm, k_norm, positions);
    if (st != SALT_OK || n_tokens == 0) return st;
    if ((st = check_heads(r, "q", q, q_stride, n_heads)) != SALT_OK) return st;
    if ((st = check_heads(r, "k", k, k_stride, KV)) != SALT_OK) return st;
    if ((st = check_heads(r, "v", v, v_stride, KV)) != SALT_OK) return st;
    if ((st = check_heads(r, "q_out", q_out, q_out_stride, n_heads)) != SALT_OK) return st;
    if (!slots) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null slots");
    if (reinterpret_cast<uintptr_t>(slots) & 3) return ctx_fail(ctx, SALT_ERR_ALIGN, "slots not on a 4-byte boundary");
    RopeParams p = {};
    p.q = static_cast<const uint16_t *>(q);
    p.k = static_cast<const uint16_t *>(k);
    p.v = static_cast<const uint16_t *>(v);
    p.q_norm = static_cast<const uint16_t *>(q_norm);
    p.k_norm = static_cast<const uint16_t *>(k_norm);
    p.q_out = static_cast<uint16_t *>(q_out);
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.q_out_stride = q_out_stride;
    p.positions = positions;
    p.slots = slots;
    p.n_tokens = n_tokens;
    p.n_heads = n_heads;
    p.n_kv_heads = KV;
    p.rows = n_heads + 2 * KV;
    p.kv = kv->dev;
    p.first_page = (uint32_t)layer * kv->dev.n_pages;
    return launch_rope<true>(r, p, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
