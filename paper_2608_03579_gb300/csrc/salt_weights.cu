// How much attention a batch's cached tokens got, added to what they gathered
// before:
//     W[j] = decay * W[j] + sum_i exp(scale * q_i k_j - lse_i)
// over the rows i (query token x query heads of the token's key/value head) that
// see token j, W[j] counted as 0 for the step's own tokens.  The rows' log-sums come from
// the attention itself, so that one pass over the keys is all there is to do.  The scores are made on the
// tensor cores with the cached tokens as the 128-row operand, S[token][row] = K[token][:] . Q[row][:], so that a
// token's weight is a sum over one thread's columns of tensor memory, in a fixed order.
//
// Lists of up to 64 rows (single query tokens, a few drafts, a prompt that some requests share) are bound by reading the keys, and that by what a tile
// costs besides: their e4m3 codes go to the
// tensor cores as they are, one tile of 128 tokens after the other, and meet the query as two e4m3 terms, hi + 2^-5
// lo: 4 and 4 bits, so a bf16 whole but for elements below 2^-14 of the row's largest (off by up to 2^-22 of
// that).  The two terms have columns of their own, as lo would lose its small elements without its factor.
//
// Lists of many rows are bound by the products and exponentials: 256 tokens' keys are widened to bf16 once
// (exact) and stay, the query's rows stream past them as they are.
//
// Two requests of 200,000 tokens and more with heads of 64 take 47 us (5.4 TB/s), 64 decoding requests with four prompts of 4,096 20 us, four prompt
// chunks of 900 to 2,048 tokens behind 4,096 215 us (1,210 TFLOP/s, 63% of the products' measured rate; 1.0e9 exponentials, whose pipe
// is 54% busy as the tensor cores are).
#include <algorithm>
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
    alignas(64) CUtensorMap kmap;   // the codes of every layer as rows of D bytes, box of one page
    alignas(64) CUtensorMap qmap;   // many rows: q as [tokens][heads][D], box of 64 elements of a group's heads of a step's tokens
    alignas(64) CUtensorMap qmap1;  // the same of one token
    const int32_t *plan, *track;
    int32_t order_at, pages_at, list_at, unit_at;
    KvDev kv;
    int64_t layer;
    const uint16_t *q;
    const float *lse;
    float *weights;
    float *part;                    // partial sums of units whose rows are split
    uint32_t *arrived;              // how many of a unit's parts are there
    int32_t *failed;                // the table's TH_FAILED
    int64_t q_stride;
    int32_t n_heads, max_tok;
    int32_t behind;                 // whether the many rows' kernel is the one before
    int32_t n_sm;
    float scale, decay;
    uint32_t *err;
};

// A list of cached tokens and the rows that see it.
struct List {
    int pages, len, tok, ntok, old, lim, causal, before, cost;
};
__device__ __forceinline__ List list_of(const int4 &a, const int4 &b) { return {a.x, a.y, a.z, a.w, b.x, b.y, b.z & 1, b.w, b.z >> 1}; }
// The same word in every lane, and known to be: loops and branches by it are taken by whole warps then, and the votes in them are quick (by
// words that might differ, a vote takes hundreds of cycles).
__device__ __forceinline__ int one_word(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ int4 one_each(const int4 &x) { return make_int4(one_word(x.x), one_word(x.y), one_word(x.z), one_word(x.w)); }
// (Of the table, as all of its words by plain loads: its first ones are at places that do not hang on words read before, and loads of constants, __ldg, of those might
// be moved before the pdl_wait.)
__device__ __forceinline__ int4 four_words(const int4 *at) { return one_each(*at); }
__device__ __forceinline__ List load_list(const WeightParams &p, int i)
{
    const int4 *w = reinterpret_cast<const int4 *>(p.track + p.list_at + i * LIST_WORDS);
    return list_of(four_words(w), four_words(w + 1));
}
// Of the lists [lo, hi) the one that holds `at` of what their tiles count together: the last that begins at or before it.  The whole warp, 32 guesses at a time.
__device__ __forceinline__ int find_list(const WeightParams &p, int lo, int hi, int at)
{
    for (int n = hi - lo; n > 1;) {
        const int step = (n + 31) / 32, guess = (int)(threadIdx.x & 31) * step;
        const uint32_t on = __ballot_sync(0xffffffffu, guess < n && p.track[p.list_at + (lo + min(guess, n - 1)) * LIST_WORDS + LS_BEFORE] <= at);
        const int last = 31 - __clz(on);  // (lane 0 is)
        lo += last * step;
        n = min(step, n - last * step);
    }
    return lo;
}
__device__ __forceinline__ int64_t first_row(const WeightParams &p, int page, int kh)
{
    return ((p.layer * p.kv.n_pages + page) * p.kv.heads + kh) << p.kv.page_log2;
}

// ---------------------------------------------------------------- few rows
// Up to R rows a list.  With R = 16 three CTAs have an SM, which reading the keys needs; with 64, where one has more rows, two.
template <int D_, int R_>
struct Few {
    static constexpr int D = D_;
    static constexpr int R = R_;
    static constexpr int N = 2 * R;                         // hi and lo
    static constexpr int CTAS = R == 16 ? 3 : 2;            // an SM
    static constexpr int STAGERS = R == 16 ? 2 : 4;         // warps that stage queries
    static constexpr int THREADS = 96 + 32 * STAGERS + 128;
    static constexpr int KST = 3 * (128 / D), EST = 8;  // stages of keys, and of what goes with a tile
    static constexpr int SLOTS = 2;                         // segments' queries
    static constexpr int SB = R == 16 ? 4 : 2;              // buffers of scores
    static constexpr uint32_t TM_COLS = SB * N;
    static constexpr uint32_t SIDE = TRACK_TILE * D;
    static constexpr uint32_t K = 0;
    static constexpr uint32_t Q_BUF = N * D;
    static constexpr uint32_t Q = K + KST * SIDE;
    static constexpr uint32_t INFO_BUF = R * 12;            // factors of the scores, log-sums, tokens seen
    static constexpr uint32_t INFO = Q + SLOTS * Q_BUF;
    // a tile's old weights, exponents, first rows of its pages
    static constexpr uint32_t E_W = 0, E_EXP = TRACK_TILE * 4, E_ROW = E_EXP + TRACK_TILE, E_BUF = E_ROW + 64;
    static constexpr uint32_t E = INFO + SLOTS * INFO_BUF;
    static constexpr uint32_t K_FULL = E + EST * E_BUF;
    static constexpr uint32_t K_FREE = K_FULL + 8 * KST;
    static constexpr uint32_t E_FULL = K_FREE + 8 * KST;
    static constexpr uint32_t E_FREE = E_FULL + 8 * EST;
    static constexpr uint32_t S_FULL = E_FREE + 8 * EST;
    static constexpr uint32_t S_FREE = S_FULL + 8 * SB;
    static constexpr uint32_t Q_FULL = S_FREE + 8 * SB;
    static constexpr uint32_t Q_FREE = Q_FULL + 8 * SLOTS;  // by the products
    static constexpr uint32_t I_FREE = Q_FREE + 8 * SLOTS;  // by the sums
    static constexpr uint32_t DRAIN = I_FREE + 8 * SLOTS;
    static constexpr uint32_t MISC = DRAIN + 8;             // TMEM address, failure flag
    static constexpr uint32_t BYTES = MISC + 8 + 1024;      // slack for the 1024-byte alignment
    static_assert(BYTES + 1024 <= 228 * 1024 / CTAS, "shared memory of an SM");
    static_assert(TM_COLS * CTAS <= 512 && (TM_COLS & (TM_COLS - 1)) == 0, "tensor memory");
    static_assert(E % 16 == 0 && K_FULL % 8 == 0, "alignment");
};

// A CTA's share [g, end), one of `ctas`, of what the few rows' lists' tiles cost, in the order list, key/value head, tile.  A segment is the tiles of one list and
// head.
struct Walk {
    int64_t g, end;
    int list, n_lists, kh, j, tiles, segment;
    List l;
    int4 a, b;  // the next list's words, on their way
    __device__ __forceinline__ void ahead(const WeightParams &p)
    {
        if (list + 1 >= n_lists) return;
        const int4 *w = reinterpret_cast<const int4 *>(p.track + p.list_at + (list + 1) * LIST_WORDS);
        a = w[0];
        b = w[1];
    }
    __device__ __forceinline__ Walk(const WeightParams &p, int lists, int64_t all, int ctas) : n_lists(lists)
    {
        const int KV = p.kv.heads;
        g = all * blockIdx.x / ctas;
        end = all * (blockIdx.x + 1) / ctas;
        segment = 0;
        if ((int)blockIdx.x >= ctas) g = end;
        if (g >= end) return;
        list = find_list(p, 0, n_lists, (int)(g / KV));  // (what is before a list, for all heads, is that times the heads)
        l = load_list(p, list);
        tiles = (l.len + TRACK_TILE - 1) / TRACK_TILE;
        // the first tile that begins in the share
        const int64_t base = (int64_t)l.before * KV;
        const int at = (int)((g - base + l.cost - 1) / l.cost);
        g = base + (int64_t)at * l.cost;
        kh = at / tiles;
        j = at - kh * tiles;
        ahead(p);
        if (kh == KV) {  // it is the next list's
            --kh;
            segment = -1;
            next_segment(p);
        }
    }
    __device__ __forceinline__ bool more() const { return g < end; }
    __device__ __forceinline__ bool last_of_segment() const { return g + l.cost >= end || j + 1 == tiles; }
    __device__ __forceinline__ void next_segment(const WeightParams &p)
    {
        j = 0;
        ++segment;
        if (++kh == p.kv.heads) {
            kh = 0;
            if (g < end) {
                ++list;
                l = list_of(one_each(a), one_each(b));
                tiles = (l.len + TRACK_TILE - 1) / TRACK_TILE;
                ahead(p);
            }
        }
    }
    __device__ __forceinline__ void next(const WeightParams &p)
    {
        g += l.cost;
        if (++j == tiles) next_segment(p);
    }
    // past the segment
    __device__ __forceinline__ void skip(const WeightParams &p)
    {
        g += (int64_t)(tiles - j) * l.cost;
        next_segment(p);
    }
};

// A segment's queries, each row scaled by a power of two, and the constants of its columns: by STAGERS warps, this one the w-th.
template <class L>
__device__ __forceinline__ void stage_few(const WeightParams &p, uint32_t base, const Walk &k, int w)
{
    constexpr int LPR = L::D / 8, RPW = 32 / LPR;   // lanes a row, rows a warp deals with at a time
    constexpr int AT_ONCE = (L::R + L::STAGERS * RPW - 1) / (L::STAGERS * RPW);  // loads of a lane under way together
    const int G = p.n_heads / p.kv.heads, lane = threadIdx.x & 31, part = lane % LPR, rows = k.l.ntok * G, slot = k.segment % L::SLOTS;
    const uint32_t q_at = base + L::Q + slot * L::Q_BUF, info = base + L::INFO + slot * L::INFO_BUF;
    uint4 q[AT_ONCE];
    float lse[AT_ONCE];
    int see[AT_ONCE];
#pragma unroll
    for (int n = 0; n < AT_ONCE; ++n) {
        const int row = (L::STAGERS * n + w) * RPW + lane / LPR, i = row / G, h = k.kh * G + row - i * G;
        q[n] = make_uint4(0, 0, 0, 0);
        lse[n] = 0.f;
        see[n] = 0;
        if (row < rows) {
            const int t = k.l.causal ? k.l.tok + i : __ldg(p.plan + p.order_at + k.l.tok + i);  // (requests' own tokens are in order)
            q[n] = __ldg(reinterpret_cast<const uint4 *>(p.q + t * p.q_stride + h * L::D) + part);
            lse[n] = __ldg(p.lse + (int64_t)t * p.n_heads + h);
            see[n] = k.l.lim + (k.l.causal ? i : 0);
        }
    }
#pragma unroll
    for (int n = 0; n < AT_ONCE; ++n) {
        const int row = (L::STAGERS * n + w) * RPW + lane / LPR;
        if ((L::STAGERS * n + w) * RPW >= ((rows + 3) & ~3)) break;  // (columns go by fours; rows that fill up see nothing)
        const uint4 u = q[n];
        const uint32_t x[4] = {u.x, u.y, u.z, u.w};
        uint32_t a = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) a = max(a, max((x[e] << 16) & 0x7fffffffu, x[e] & 0x7fff0000u));
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
        const int qe = max((int)(a >> 23) - 127 - 7, -120);  // the row's largest element to [2^7, 2^8)
        const float inv = pow2(-qe);
        uint32_t hi[2] = {0, 0}, lo[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v0 = __uint_as_float(x[e] << 16) * inv, v1 = __uint_as_float(x[e] & 0xffff0000u) * inv;
            const uint16_t c = e4m3x2(v0, v1);
            const uint32_t back = f16x2_of_e4m3x2(c);
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&back));
            hi[e / 2] |= (uint32_t)c << (16 * (e & 1));
            lo[e / 2] |= (uint32_t)e4m3x2((v0 - f.x) * 32.f, (v1 - f.y) * 32.f) << (16 * (e & 1));  // (v - f at most 2^3)
        }
        if ((a >> 23) == 255) hi[0] = hi[1] = lo[0] = lo[1] = 0x7f7f7f7fu;
        if (row < L::R) {
            sts64(q_at + swz_rows<L::D>(row * L::D + part * 8), hi[0], hi[1]);
            sts64(q_at + swz_rows<L::D>((L::R + row) * L::D + part * 8), lo[0], lo[1]);
            if (part == 0) {
                stsf(info + 4 * row, pow2(qe) * p.scale);
                stsf(info + 4 * (L::R + row), -lse[n]);
                sts32(info + 4 * (2 * L::R + row), (uint32_t)see[n]);
            }
        }
    }
    fence_async_smem();
}

template <class L>
__global__ void __launch_bounds__(L::THREADS, L::CTAS) weights_few_kernel(const __grid_constant__ WeightParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(sm);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, KV = p.kv.heads;
    volatile int *dead = reinterpret_cast<volatile int *>(sm + L::MISC + 4);
    if (tid == 0) {
        for (int i = 0; i < L::KST; ++i) {
            mbar_init(base + L::K_FULL + 8 * i, 1);
            mbar_init(base + L::K_FREE + 8 * i, 1);
        }
        for (int i = 0; i < L::EST; ++i) {
            mbar_init(base + L::E_FULL + 8 * i, 1);
            mbar_init(base + L::E_FREE + 8 * i, 4);
        }
        for (int i = 0; i < L::SB; ++i) {
            mbar_init(base + L::S_FULL + 8 * i, 1);
            mbar_init(base + L::S_FREE + 8 * i, 4);
        }
        for (int i = 0; i < L::SLOTS; ++i) {
            mbar_init(base + L::Q_FULL + 8 * i, L::STAGERS);
            mbar_init(base + L::Q_FREE + 8 * i, 1);
            mbar_init(base + L::I_FREE + 8 * i, 4);
        }
        mbar_init(base + L::DRAIN, 1);
        *dead = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        tmem_alloc(base + L::MISC, L::TM_COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<uint32_t *>(sm + L::MISC);
    // (behind the many rows' kernel nothing that it writes is needed, and it lets this one begin after its own wait)
    if (!p.behind) pdl_wait();
    pdl_launch_dependents();
    const int32_t *track = after_pdl_wait(p.track);
    const bool fits = track[TH_TOKENS] <= p.max_tok && !track[TH_SHARED];
    if (!fits && blockIdx.x == 0 && tid == 0) atomicOr(p.err, SALT_DEVERR_BATCH);
    const int n_lists = one_word(fits ? track[TH_FEW] : 0);
    // The CTAs of the SMs that the lists of many rows leave: all of a direct call's; one that was captured is launched on every SM, for whatever batch it is replayed on.
    const int listed = one_word(track[TH_LISTED]), sms = listed > 0 && listed < p.n_sm ? p.n_sm - listed : p.n_sm;
    Walk k(p, n_lists, n_lists ? (int64_t)one_word(track[TH_FEW_COST]) * KV : 0, min((int)gridDim.x, sms * L::CTAS));
    bool ok = true;
    // A tile's pages, a lane each, are looked up while the one's before are waited for.  Its codes are one warp's to fetch, its exponents and old weights
    // another's (one for all took 800 cycles a tile, the longest of the roles).
    auto pages_of = [&](const Walk &x) { return min(TRACK_TILE >> p.kv.page_log2, ((x.l.len - 1) >> p.kv.page_log2) - (x.j * TRACK_TILE >> p.kv.page_log2) + 1); };
    auto look_up = [&](const Walk &x) { return lane < pages_of(x) ? __ldg(p.plan + p.pages_at + x.l.pages + (x.j * TRACK_TILE >> p.kv.page_log2) + lane) : 0; };
    if (!k.more()) {
    } else if (warp == 0) {
        // ------------------------------------------------ codes
        uint32_t ks = 0, kph = 0, n = 0;
        int page = look_up(k);
        for (; k.more(); ++n) {
            const int pages = pages_of(k);
            const int64_t row = first_row(p, page, k.kh);
            const uint32_t full = base + L::K_FULL + 8 * ks;
            k.next(p);
            if (k.more()) page = look_up(k);
            if (n >= (uint32_t)L::KST) ok = __all_sync(0xffffffffu, wait_bar(base + L::K_FREE + 8 * ks, kph ^ 1, dead));
            if (!ok) break;
            if (lane == 0) mbar_expect_tx(full, pages * p.kv.page * L::D);
            __syncwarp();
            if (lane < pages) tma_load_2d(base + L::K + ks * L::SIDE + lane * p.kv.page * L::D, &p.kmap, 0, (int)row, full);
            if (++ks == (uint32_t)L::KST) ks = 0, kph ^= 1;
        }
        if (!ok) {  // copies in flight land before the CTA ends
            if (lane == 0) {
                *dead = 1;
                atomicOr(p.err, SALT_DEVERR_TIMEOUT);
            }
            for (uint32_t i = 0; i < min(n, (uint32_t)L::KST); ++i) mbar_wait(base + L::K_FULL + 8 * ((n - 1 - i) % L::KST), ((n - 1 - i) / L::KST) & 1);
        }
    } else if (warp == 2 + L::STAGERS) {
        // ------------------------------------------------ exponents, old weights, where they lie
        uint32_t es = 0, eph = 0, n = 0;
        int page = look_up(k);
        for (; k.more(); ++n) {
            const int pages = pages_of(k);
            const int64_t row = first_row(p, page, k.kh);
            const bool old = p.decay != 0.f && k.j * TRACK_TILE < k.l.old;
            const uint32_t full = base + L::E_FULL + 8 * es, e = base + L::E + es * L::E_BUF, at = lane * p.kv.page;
            k.next(p);
            if (k.more()) page = look_up(k);
            if (n >= (uint32_t)L::EST) ok = __all_sync(0xffffffffu, wait_bar(base + L::E_FREE + 8 * es, eph ^ 1, dead));
            if (!ok) break;
            if (lane < pages) sts32(e + L::E_ROW + 4 * lane, (uint32_t)row);
            __syncwarp();
            if (lane == 0) mbar_expect_tx(full, pages * p.kv.page * (old ? 5 : 1));
            __syncwarp();
            if (lane < pages) {
                bulk_load(e + L::E_EXP + at, p.kv.k_exp + row, p.kv.page, full);
                if (old) bulk_load(e + L::E_W + 4 * at, p.weights + row, p.kv.page * 4, full);
            }
            if (++es == (uint32_t)L::EST) es = 0, eph ^= 1;
        }
        if (!ok) {  // as above
            if (lane == 0) {
                *dead = 1;
                atomicOr(p.err, SALT_DEVERR_TIMEOUT);
            }
            for (uint32_t i = 0; i < min(n, (uint32_t)L::EST); ++i) mbar_wait(base + L::E_FULL + 8 * ((n - 1 - i) % L::EST), ((n - 1 - i) / L::EST) & 1);
        }
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issue
        const bool lead = elect_one();
        const uint32_t id = idesc_e4m3_f32(128, L::N);
        uint32_t ks = 0, kph = 0, n = 0;
        bool fresh = true;
        for (; k.more(); k.next(p), ++n) {
            const int b = n % L::SB, slot = k.segment % L::SLOTS;
            if (fresh) ok = wait_bar(base + L::Q_FULL + 8 * slot, (k.segment / L::SLOTS) & 1, dead);
            fresh = k.last_of_segment();
            ok = ok && wait_bar(base + L::K_FULL + 8 * ks, kph, dead);
            if (n >= (uint32_t)L::SB) ok = ok && wait_bar(base + L::S_FREE + 8 * b, (n / L::SB - 1) & 1, dead);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const uint64_t kd = sdesc_rows(base + L::K + ks * L::SIDE, L::D, 0), qd = sdesc_rows(base + L::Q + slot * L::Q_BUF, L::D, 0);
            if (lead) {
#pragma unroll
                for (int i = 0; i < L::D / 32; ++i) umma_e4m3(tmem + b * L::N, kd + 2 * i, qd + 2 * i, id, i > 0);
                umma_commit(base + L::S_FULL + 8 * b);
                umma_commit(base + L::K_FREE + 8 * ks);
                if (fresh) umma_commit(base + L::Q_FREE + 8 * slot);
            }
            __syncwarp();
            if (++ks == (uint32_t)L::KST) ks = 0, kph ^= 1;
        }
        if (!ok) {  // the products issued so far end before the CTA does
            if (lead) {
                *dead = 1;
                atomicOr(p.err, SALT_DEVERR_TIMEOUT);
                umma_commit(base + L::DRAIN);
                mbar_wait(base + L::DRAIN, 0);
            }
            __syncwarp();
        }
    } else if (warp < 2 + L::STAGERS) {
        // ------------------------------------------------ queries, a segment ahead
        for (; k.more(); k.skip(p)) {
            const int slot = k.segment % L::SLOTS, use = k.segment / L::SLOTS;
            if (use > 0) ok = wait_bar(base + L::Q_FREE + 8 * slot, (use - 1) & 1, dead) && wait_bar(base + L::I_FREE + 8 * slot, (use - 1) & 1, dead);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            stage_few<L>(p, base, k, warp - 2);
            __syncwarp();
            if (lane == 0) mbar_arrive_release(base + L::Q_FULL + 8 * slot);
        }
        if (!ok && lane == 0) {
            *dead = 1;
            atomicOr(p.err, SALT_DEVERR_TIMEOUT);
        }
    } else {
        // ------------------------------------------------ a thread's token: its row of scores, its weight
        const int me = 32 * (warp & 3) + lane, G = p.n_heads / KV;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        uint32_t es = 0, eph = 0, n = 0;
        bool fresh = true;
        for (; k.more(); k.next(p), ++n) {
            const int b = n % L::SB, slot = k.segment % L::SLOTS, j = k.j * TRACK_TILE + me, rows = k.l.ntok * G;
            if (fresh) ok = wait_bar(base + L::Q_FULL + 8 * slot, (k.segment / L::SLOTS) & 1, dead);
            fresh = k.last_of_segment();
            ok = ok && wait_bar(base + L::E_FULL + 8 * es, eph, dead);
            const uint32_t e = base + L::E + es * L::E_BUF;
            const float kf = row_scale(lds8(e + L::E_EXP + me));
            const float was = p.decay != 0.f && j < k.l.old ? p.decay * ldsf(e + L::E_W + 4 * me) : 0.f;
            const uint32_t at = lds32(e + L::E_ROW + 4 * (me >> p.kv.page_log2)) + (me & (p.kv.page - 1));
            ok = ok && wait_bar(base + L::S_FULL + 8 * b, (n / L::SB) & 1, dead);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            if (lane == 0) mbar_arrive_release(base + L::E_FREE + 8 * es);
            tc_fence_after();
            const uint32_t info = base + L::INFO + slot * L::INFO_BUF, s_at = tmem + lanes + b * L::N;
            float sum = 0.f;
#pragma unroll 1
            for (int c0 = 0; c0 < rows; c0 += 4) {
                float hi[4], lo[4];
                tmem_ld4(s_at + c0, reinterpret_cast<uint32_t *>(hi));
                tmem_ld4(s_at + L::R + c0, reinterpret_cast<uint32_t *>(lo));
                const float4 a = lds4f(info + 4 * c0), l = lds4f(info + 4 * (L::R + c0));
                const uint4 lim = lds128(info + 4 * (2 * L::R + c0));
                tmem_ld_wait();
                const float f[4] = {a.x, a.y, a.z, a.w}, m[4] = {l.x, l.y, l.z, l.w};
                const int see[4] = {(int)lim.x, (int)lim.y, (int)lim.z, (int)lim.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = fmaf(fmaf(lo[i], 0.03125f, hi[i]), f[i] * kf, m[i]) * LOG2E;
                    if (j < see[i]) sum += ex2(x);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive_release(base + L::S_FREE + 8 * b);
                if (fresh) mbar_arrive_release(base + L::I_FREE + 8 * slot);
            }
            if (j < k.l.len) p.weights[at] = was + sum;
            if (++es == (uint32_t)L::EST) es = 0, eph ^= 1;
        }
        if (!ok && lane == 0) {
            *dead = 1;
            atomicOr(p.err, SALT_DEVERR_TIMEOUT);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, L::TM_COLS);
    pdl_wait();  // so that what follows this kernel follows the one before it too
}

// ---------------------------------------------------------------- many rows
// A unit is 256 tokens of a list and head, and a run of steps over the rows that see them, up to 128 at
// a time.  Either 128 tokens have two warpgroups, which take every other step each: what a step costs besides its sums (waiting, a vote, fetching scores; 600
// cycles of 2,100) is spent beside the others' sums.  (With one warpgroup four prompt chunks took 268 us where these took 236; with two of half a step's columns each, which
// meet at every barrier, 260.)
template <int D_>
struct Many {
    static constexpr int D = D_;
    static constexpr int THREADS = 128 + 4 * 128;           // (96 registers a thread: a score that is spilled is one that may not have come yet)
    static constexpr int QST = D == 128 ? 4 : 6, MST = 4;   // stages of queries, and of what goes with a step
    // Tensor memory: the keys of either 128 tokens as bf16, three buffers of 128 scores for both in turn.  (With the keys in shared
    // memory a step's products read 128 KB from there, as long as they take themselves, besides all else: 277 us where this took 253.)
    static constexpr int SB = 3;
    static constexpr uint32_t TM_A = 0, TM_S = 128, TM_COLS = 512;
    static constexpr uint32_t RAW_TILE = 128 * D, Q_TILE = 128 * 2 * D;
    static constexpr uint32_t RAW = 0;
    static constexpr uint32_t Q = RAW + 4 * RAW_TILE;       // (either tile's codes of this unit and the next)
    static constexpr uint32_t M_LSE = 0, M_LIM = 512, M_BUF = 1024;
    static constexpr uint32_t META = Q + QST * Q_TILE;
    static constexpr uint32_t EXPS = META + MST * M_BUF;    // 128 of either tile, of two units
    static constexpr uint32_t ROWS = EXPS + 512;            // the first rows of either tile's pages, of two units
    static constexpr uint32_t HALF = ROWS + 128;            // the second warpgroup's sums of either tile
    static constexpr uint32_t H_FULL = HALF + 1024;         // a warp's each
    static constexpr uint32_t H_FREE = H_FULL + 64;
    static constexpr uint32_t K_FULL = H_FREE + 64;
    static constexpr uint32_t K_FREE = K_FULL + 32;         // [tile][unit & 1]
    static constexpr uint32_t A_FULL = K_FREE + 32;
    static constexpr uint32_t Q_FULL = A_FULL + 16;
    static constexpr uint32_t Q_FREE = Q_FULL + 8 * QST;
    static constexpr uint32_t M_FULL = Q_FREE + 8 * QST;
    static constexpr uint32_t M_FREE = M_FULL + 8 * MST;
    // Of scores that are there two barriers for each warpgroup: of the three jobs at most that have a buffer it has two at most.  (By buffers, a
    // warpgroup would wait for the second use to come of one that had its last while it was busy.)
    static constexpr uint32_t S_FULL = M_FREE + 8 * MST;
    static constexpr uint32_t S_FREE = S_FULL + 64;
    static constexpr uint32_t DRAIN = S_FREE + 8 * SB;
    static constexpr uint32_t MISC = DRAIN + 8;
    static constexpr uint32_t BYTES = MISC + 8 + 1024;
    static_assert(BYTES + 1024 <= 228 * 1024, "shared memory of an SM");
    static_assert(TM_S + SB * 128 <= TM_COLS && D <= 128, "tensor memory");
};

struct Unit {
    List l;
    int kh, t0, r0, r1, split;  // head, first token, steps [r0, r1), where its parts meet
    bool two;                   // more than 128 tokens
};

// A CTA's units: the build's lists for CTAs blockIdx.x, blockIdx.x + gridDim.x, .. (a call has as many CTAs as there are lists, a captured one as there are
// SMs), or every gridDim-th one, whole tiles all.
struct Units {
    int at, end, cta, ctas;
    __device__ __forceinline__ void settle(const WeightParams &p)
    {
        while (ctas > 0 && at >= end && cta + (int)gridDim.x < ctas) {
            cta += gridDim.x;
            at = one_word(p.track[p.unit_at + cta]);
            end = one_word(p.track[p.unit_at + cta + 1]);
        }
    }
    __device__ __forceinline__ Units(const WeightParams &p, bool fits)
    {
        ctas = one_word(p.track[TH_FAILED] ? 0 : p.track[TH_LISTED]);
        at = blockIdx.x;
        end = ctas > 0 ? 0 : one_word(fits ? p.track[TH_MANY_TILES] * p.kv.heads : 0);
        cta = (int)blockIdx.x - (int)gridDim.x;
        if (!fits) ctas = end = 0;
        else settle(p);
    }
    __device__ __forceinline__ bool more() const { return at < end; }
    __device__ __forceinline__ void advance(const WeightParams &p)
    {
        at += ctas > 0 ? 1 : gridDim.x;
        settle(p);
    }
    __device__ __forceinline__ Unit get(const WeightParams &p, int per) const
    {
        Unit u;
        if (ctas > 0) {
            const int4 *w = reinterpret_cast<const int4 *>(p.track + p.unit_at + TRACK_CTAS) + (int64_t)at * (UNIT_WORDS / 4);
            const int4 a = four_words(w), b = four_words(w + 1), c = four_words(w + 2);
            u.l = list_of(a, b);
            u.kh = b.w;
            u.t0 = c.x;
            u.r0 = c.y;
            u.r1 = c.z;
            u.split = c.w;
        } else {
            const int tile = at / p.kv.heads;
            u.kh = at - tile * p.kv.heads;
            u.l = load_list(p, find_list(p, p.track[TH_FEW], p.track[TH_FEW] + p.track[TH_MANY], tile));
            u.t0 = (tile - u.l.before) * TRACK_MANY_TILE;
            u.r0 = first_step(u.l.causal, u.l.lim, u.t0, per);
            u.r1 = (u.l.ntok + per - 1) / per;
            u.split = -1;
        }
        u.two = u.l.len - u.t0 > 128;
        return u;
    }
};

// A CTA's steps, unit by unit, the next unit's words on their way.
struct Steps {
    Units it;
    Unit u, v;
    int r;
    bool live, next;
    __device__ __forceinline__ void ahead(const WeightParams &p, int per)
    {
        it.advance(p);
        next = it.more();
        if (next) v = it.get(p, per);
    }
    __device__ __forceinline__ Steps(const WeightParams &p, const Units &units, int per) : it(units)
    {
        live = it.more();
        if (!live) return;
        u = it.get(p, per);
        r = u.r0;
        ahead(p, per);
    }
    __device__ __forceinline__ void advance(const WeightParams &p, int per)
    {
        if (++r < u.r1) return;
        live = next;
        if (!live) return;
        u = v;
        r = u.r0;
        ahead(p, per);
    }
    // query tokens of the step; the i-th of them (a request's own follow each other in the order)
    __device__ __forceinline__ int tokens(int per) const { return min(per, u.l.ntok - r * per); }
    __device__ __forceinline__ int token(const WeightParams &p, int per, int i) const
    {
        const int at = u.l.tok + r * per + i;
        return u.l.causal ? at : __ldg(p.plan + p.order_at + at);
    }
};

// Widens a token's key: its codes to bf16, two a column of the token's lane of tensor memory.
template <class L>
__device__ __forceinline__ void widen_key(uint32_t from, uint32_t to, int me)
{
#pragma unroll
    for (int c = 0; c < L::D / 16; ++c) {
        const uint4 x = lds128(from + swz_rows<L::D>(me * L::D + c * 16));
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
        uint32_t y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t h = f16x2_of_e4m3x2((uint16_t)(w[i / 2] >> (16 * (i & 1))));
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
            const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
            y[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        tmem_st8(to + 8 * c, y);
    }
    tmem_st_wait();
}

// Adds the terms of 16 columns' scores, none of them masked.
__device__ __forceinline__ void add_columns(const float (&y)[16], uint32_t lse, float a, float2 (&sum)[2])
{
    const float2 a2 = make_float2(a, a), e2 = make_float2(LOG2E, LOG2E);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 m = lds4f(lse + 16 * i);
        const float2 u = mul2(fma2(make_float2(y[4 * i], y[4 * i + 1]), a2, make_float2(m.x, m.y)), e2);
        const float2 v = mul2(fma2(make_float2(y[4 * i + 2], y[4 * i + 3]), a2, make_float2(m.z, m.w)), e2);
        sum[0] = add2(sum[0], make_float2(ex2(u.x), ex2(u.y)));
        sum[1] = add2(sum[1], make_float2(ex2(v.x), ex2(v.y)));
    }
}

template <class L>
__global__ void __launch_bounds__(L::THREADS, 1) weights_many_kernel(const __grid_constant__ WeightParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(sm);
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, KV = p.kv.heads, G = p.n_heads / KV, per = 128 / G;
    volatile int *dead = reinterpret_cast<volatile int *>(sm + L::MISC + 4);
    if (tid == 0) {
        for (int i = 0; i < 4; ++i) {
            mbar_init(base + L::K_FULL + 8 * i, 1);
            mbar_init(base + L::K_FREE + 8 * i, 8);
        }
        for (int i = 0; i < 2; ++i) mbar_init(base + L::A_FULL + 8 * i, 4);
        for (int i = 0; i < L::QST; ++i) {
            mbar_init(base + L::Q_FULL + 8 * i, 1);
            mbar_init(base + L::Q_FREE + 8 * i, 1);
        }
        for (int i = 0; i < L::MST; ++i) {
            mbar_init(base + L::M_FULL + 8 * i, 1);
            mbar_init(base + L::M_FREE + 8 * i, 8);
        }
        for (int i = 0; i < 8; ++i) mbar_init(base + L::S_FULL + 8 * i, 1);
        for (int i = 0; i < L::SB; ++i) mbar_init(base + L::S_FREE + 8 * i, 4);
        for (int i = 0; i < 8; ++i) {
            mbar_init(base + L::H_FULL + 8 * i, 1);
            mbar_init(base + L::H_FREE + 8 * i, 1);
        }
        mbar_init(base + L::DRAIN, 1);
        *dead = 0;
        mbar_fence_init();
    }
    if (warp == 1) {
        tmem_alloc(base + L::MISC, L::TM_COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<uint32_t *>(sm + L::MISC);
    pdl_wait();
    pdl_launch_dependents();
    const int32_t *track = after_pdl_wait(p.track);
    const bool fits = track[TH_TOKENS] <= p.max_tok && !track[TH_SHARED];  // (the other kernel says so)
    Units it(p, fits);
    bool ok = true;
    if (!it.more()) {
    } else if (warp == 0) {
        // ------------------------------------------------ a step's queries, whole where their tokens follow each other, else token by
        // token
        uint32_t n = 0, st = 0, ph = 0;
        const uint32_t q_bytes = G * 128 * (L::D / 64);
        Steps s(p, it, per);
        int tok[4];
        auto look_up = [&](const Steps &x, int (&t)[4]) {
            const int m = x.tokens(per);
#pragma unroll
            for (int k = 0; k < 4; ++k) t[k] = lane + 32 * k < m ? x.token(p, per, lane + 32 * k) : -1;
        };
        look_up(s, tok);
        while (ok && s.live) {
            const int m = s.tokens(per), tok0 = __shfl_sync(0xffffffffu, tok[0], 0), kh = s.u.kh;
            bool run = true;
#pragma unroll
            for (int k = 0; k < 4; ++k) run = run && (lane + 32 * k >= m || tok[k] == tok0 + lane + 32 * k);
            run = __all_sync(0xffffffffu, run);
            if (n >= (uint32_t)L::QST) ok = wait_bar(base + L::Q_FREE + 8 * st, ph ^ 1, dead);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const uint32_t full = base + L::Q_FULL + 8 * st, to = base + L::Q + st * L::Q_TILE;
            if (lane == 0) mbar_expect_tx(full, (run ? per : m) * q_bytes);
            __syncwarp();
            if (run) {
                if (lane < L::D / 64) tma_load_3d(to + lane * (128 * 128), &p.qmap, 64 * lane, kh * G, tok0, full);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = lane + 32 * k;
                    if (i < m)
                        for (int h = 0; h < L::D / 64; ++h)
                            tma_load_3d(to + h * (128 * 128) + i * G * 128, &p.qmap1, 64 * h, kh * G, tok[k], full);
                }
            }
            __syncwarp();
            ++n;
            if (++st == (uint32_t)L::QST) st = 0, ph ^= 1;
            s.advance(p, per);
            if (s.live) look_up(s, tok);
        }
        if (!ok) {  // copies in flight land before the CTA ends
            if (lane == 0) {
                *dead = 1;
                atomicOr(p.err, SALT_DEVERR_TIMEOUT);
            }
            for (uint32_t i = 0; i < min(n, (uint32_t)L::QST); ++i) mbar_wait(base + L::Q_FULL + 8 * ((n - 1 - i) % L::QST), ((n - 1 - i) / L::QST) & 1);
        }
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issue
        const bool lead = elect_one();
        const uint32_t id = idesc_bf16_f32(128, (per * G + 15) / 16 * 16);
        uint32_t st = 0, ph = 0, units[2] = {0, 0}, job = 0, n = 0, odd = 0;  // (odd: a bit a warpgroup; a job: a step's scores of 128 tokens)
        Unit u = it.get(p, per);
        while (it.more() && ok) {
            it.advance(p);
            Unit v = u;
            if (it.more()) v = it.get(p, per);
            for (int r = u.r0; r < u.r1 && ok; ++r) {
                ok = wait_bar(base + L::Q_FULL + 8 * st, ph, dead);
                const uint64_t qd = sdesc_kmajor_sw128(base + L::Q + st * L::Q_TILE);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    if (w == 1 && !u.two) break;
                    const uint32_t b = job % L::SB;
                    if (r == u.r0) ok = ok && wait_bar(base + L::A_FULL + 8 * w, units[w] & 1, dead);
                    if (job >= (uint32_t)L::SB) ok = ok && wait_bar(base + L::S_FREE + 8 * b, (job / L::SB - 1) & 1, dead);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    if (lead) {
#pragma unroll
                        for (int k = 0; k < L::D / 16; ++k)
                            umma_bf16_ta(tmem + L::TM_S + b * 128, tmem + L::TM_A + w * 64 + 8 * k, qd + (k / 4) * (128 * 128 / 16) + 2 * (k % 4), id, k > 0);
                        umma_commit(base + L::S_FULL + 16 * (2 * w + (n & 1)) + 8 * (odd >> (2 * w + (n & 1)) & 1));
                    }
                    __syncwarp();
                    odd ^= 1u << (2 * w + (n & 1));
                    ++job;
                }
                if (!ok) break;
                if (lead) umma_commit(base + L::Q_FREE + 8 * st);
                __syncwarp();
                ++n;
                if (++st == (uint32_t)L::QST) st = 0, ph ^= 1;
            }
            ++units[0];
            units[1] += u.two;
            u = v;
        }
        if (!ok) {  // the products issued so far end before the CTA does
            if (lead) {
                *dead = 1;
                atomicOr(p.err, SALT_DEVERR_TIMEOUT);
                umma_commit(base + L::DRAIN);
                mbar_wait(base + L::DRAIN, 0);
            }
            __syncwarp();
        }
    } else if (warp == 2) {
        // ------------------------------------------------ the steps' log-sums, and how many tokens their rows see
        // (a step's log-sums are fetched while the one's before are put, its tokens one step earlier still: one behind the other they took
        // 1.3 us a step, as long as two steps' products)
        int row_token[4], row_head[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            row_token[k] = (lane + 32 * k) / G;
            row_head[k] = lane + 32 * k - row_token[k] * G;
        }
        auto look_up = [&](const Steps &x, int (&t)[4]) {
            const int m = x.tokens(per);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                t[k] = row_token[k] < m ? x.token(p, per, row_token[k]) : -1;
            }
        };
        auto fetch = [&](const Steps &x, const int (&t)[4], float (&lse)[4]) {
#pragma unroll
            for (int k = 0; k < 4; ++k) lse[k] = t[k] < 0 ? 0.f : -__ldg(p.lse + (int64_t)t[k] * p.n_heads + x.u.kh * G + row_head[k]);
        };
        Steps s(p, it, per);
        int tok[4];
        float lse[4];
        look_up(s, tok);
        fetch(s, tok, lse);
        Steps t = s;
        t.advance(p, per);
        if (t.live) look_up(t, tok);
        for (uint32_t n = 0; s.live; ++n) {
            float lse_next[4] = {0.f, 0.f, 0.f, 0.f};
            if (t.live) fetch(t, tok, lse_next);
            Steps next = t;
            if (t.live) {
                next.advance(p, per);
                if (next.live) look_up(next, tok);
            }
            const uint32_t slot = n % L::MST, to = base + L::META + slot * L::M_BUF + 4 * lane;
            if (n >= (uint32_t)L::MST) ok = wait_bar(base + L::M_FREE + 8 * slot, (n / L::MST - 1) & 1, dead);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const int m = s.tokens(per);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = row_token[k];
                stsf(to + L::M_LSE + 128 * k, lse[k]);
                sts32(to + L::M_LIM + 128 * k, i < m ? (uint32_t)(s.u.l.lim + (s.u.l.causal ? s.r * per + i : 0)) : 0u);
                lse[k] = lse_next[k];
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_release(base + L::M_FULL + 8 * slot);
            s = t;
            t = next;
        }
        if (!ok && lane == 0) {
            *dead = 1;
            atomicOr(p.err, SALT_DEVERR_TIMEOUT);
        }
    } else if (warp == 3) {
        // ------------------------------------------------ the units' codes, up to two units ahead
        uint32_t used[2] = {0, 0};
        const int page_per = 128 >> p.kv.page_log2;
        for (; it.more() && ok; it.advance(p)) {
            const Unit u = it.get(p, per);
            for (int w = 0; w < (u.two ? 2 : 1); ++w) {
                const int t = u.t0 + 128 * w, first = t >> p.kv.page_log2;
                const int pages = min(page_per, ((u.l.len - 1) >> p.kv.page_log2) - first + 1);
                int page = 0;
                if (lane < pages) page = __ldg(p.plan + p.pages_at + u.l.pages + first + lane);
                const int64_t row = first_row(p, page, u.kh);
                const uint32_t buf = 2 * w + (used[w] & 1), full = base + L::K_FULL + 8 * buf, at = lane * p.kv.page;
                if (used[w] > 1) ok = __all_sync(0xffffffffu, wait_bar(base + L::K_FREE + 8 * buf, ((used[w] >> 1) - 1) & 1, dead));
                if (!ok) break;
                if (lane < pages) sts32(base + L::ROWS + 32 * buf + 4 * lane, (uint32_t)row);
                __syncwarp();
                if (lane == 0) mbar_expect_tx(full, pages * p.kv.page * (L::D + 1));
                __syncwarp();
                if (lane < pages) {
                    tma_load_2d(base + L::RAW + buf * L::RAW_TILE + at * L::D, &p.kmap, 0, (int)row, full);
                    bulk_load(base + L::EXPS + 128 * buf + at, p.kv.k_exp + row, p.kv.page, full);
                }
                ++used[w];
            }
        }
        if (!ok) {  // copies in flight land before the CTA ends
            if (lane == 0) {
                *dead = 1;
                atomicOr(p.err, SALT_DEVERR_TIMEOUT);
            }
            for (int w = 0; w < 2; ++w)
                for (uint32_t i = 0; i < min(used[w], 2u); ++i) mbar_wait(base + L::K_FULL + 8 * (2 * w + ((used[w] - 1 - i) & 1)), ((used[w] - 1 - i) >> 1) & 1);
        }
    } else {
        // ------------------------------------------------ a thread's token: its rows of scores, its weight
        const int w = (warp - 4) >> 2 & 1, par = (warp - 4) >> 3, me = tid & 127;  // the 128 tokens, the steps
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        uint32_t n = 0, b = w, jobs = 0, units = 0, done = 0;  // (b: the buffer of the step's job)
        float a = 0.f;
        uint32_t at = 0;
        // The next unit's codes to bf16, by one of the two warpgroups; its exponent and row, by both.
        auto widen = [&]() {
            const uint32_t buf = 2 * w + (units & 1);
            ok = ok && wait_bar(base + L::K_FULL + 8 * buf, units >> 1 & 1, dead);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) return;
            widen_key<L>(base + L::RAW + buf * L::RAW_TILE, t_lane + L::TM_A + w * 64, me);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_release(base + L::A_FULL + 8 * w);
        };
        auto take_up = [&]() {
            const uint32_t buf = 2 * w + (units & 1);
            ok = ok && wait_bar(base + L::K_FULL + 8 * buf, units >> 1 & 1, dead);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) return;
            a = p.scale * row_scale(lds8(base + L::EXPS + 128 * buf + me));
            at = lds32(base + L::ROWS + 32 * buf + 4 * (me >> p.kv.page_log2)) + (me & (p.kv.page - 1));
            __syncwarp();
            if (lane == 0) mbar_arrive_release(base + L::K_FREE + 8 * buf);
            ++units;
        };
        Unit u = it.get(p, per);
        if (par == 0 && (w == 0 || u.two)) widen();
        if (w == 0 || u.two) take_up();
        while (ok && it.more()) {
            it.advance(p);
            // (all of the next unit's words are read when it begins, from the L1 then)
            const bool next = it.more(), next_two = next && it.get(p, per).two, mine = w == 0 || u.two, theirs = next && (w == 0 || next_two);
            const int j = u.t0 + 128 * w + me, end = min(u.t0 + 128 * (w + 1), u.l.len);
            const bool live = mine && j < u.l.len;
            float total = 0.f;
            // (the first one knows of both that they are done with the unit before)
            if (!mine && theirs && par == 0) widen();
            for (int r = u.r0; r < u.r1; ++r, ++n, b += u.two ? 2 : 1) {
                if (b >= (uint32_t)L::SB) b -= L::SB;
                if ((n & 1) != (uint32_t)par) continue;
                const uint32_t ms = n % L::MST, meta = base + L::META + ms * L::M_BUF;
                ok = ok && wait_bar(base + L::M_FULL + 8 * ms, (n / L::MST) & 1, dead);
                if (mine) ok = ok && wait_bar(base + L::S_FULL + 16 * (2 * w + par) + 8 * (jobs & 1), jobs >> 1 & 1, dead);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (mine) {
                    ++jobs;
                    tc_fence_after();
                    if (r + 1 == u.r1 && theirs) {  // (the unit's products are done: the next one's keys take its keys' place)
                        widen();
                        if (!ok) break;
                    }
                    const int i0 = r * per, cols = min(per, u.l.ntok - i0) * G;
                    const int full = u.l.causal && end > u.l.lim + i0 ? 0 : cols / 16;
                    const uint32_t s_at = t_lane + L::TM_S + b * 128, lse = meta + L::M_LSE;
                    auto free = [&]() {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_release(base + L::S_FREE + 8 * b);
                    };
                    float2 sums[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    if (full == 8) {  // the scores' place is free once they are in registers
                        float x[2][16];
                        auto load = [&](int c) { tmem_ld16(s_at + 16 * c, *reinterpret_cast<uint32_t(*)[16]>(x[c & 1])); };
                        load(0);
                        load(1);
#pragma unroll
                        for (int c = 0; c < 8; c += 2) {
                            tmem_ld_wait();
                            if (c == 6) free();
                            add_columns(x[0], lse + 64 * c, a, sums);
                            if (c < 6) load(c + 2);
                            add_columns(x[1], lse + 64 * c + 64, a, sums);
                            if (c < 6) load(c + 3);
                        }
                    } else {
#pragma unroll 1
                        for (int c = 0; c < full; ++c) {
                            float x[16];
                            tmem_ld16(s_at + 16 * c, *reinterpret_cast<uint32_t(*)[16]>(x));
                            tmem_ld_wait();
                            add_columns(x, lse + 64 * c, a, sums);
                        }
                    }
                    float sum = (sums[0].x + sums[0].y) + (sums[1].x + sums[1].y);
#pragma unroll 1
                    for (int c = 16 * full; c < cols; c += 4) {
                        float x[4];
                        tmem_ld4(s_at + c, reinterpret_cast<uint32_t *>(x));
                        const float4 l = lds4f(lse + 4 * c);
                        const uint4 lim = lds128(meta + L::M_LIM + 4 * c);
                        tmem_ld_wait();
                        const float m[4] = {l.x, l.y, l.z, l.w};
                        const int see[4] = {(int)lim.x, (int)lim.y, (int)lim.z, (int)lim.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float e = ex2(fmaf(x[i], a, m[i]) * LOG2E);
                            if (j < see[i]) sum += e;
                        }
                    }
                    total += sum;
                    if (full < 8) free();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_release(base + L::M_FREE + 8 * ms);
            }
            if (!ok) break;
            float was = 0.f;
            if (live && par == 0 && p.decay != 0.f && j < u.l.old) was = p.decay * p.weights[at];
            if (mine) {  // the two warpgroups' sums
                const uint32_t at_h = base + L::HALF + 512 * w + 4 * me, pair = 4 * w + (warp & 3), full = base + L::H_FULL + 8 * pair, free = base + L::H_FREE + 8 * pair;
                if (par) {
                    if (done > 0) ok = wait_bar(free, (done - 1) & 1, dead);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    stsf(at_h, total);
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release(full);
                } else {
                    ok = __all_sync(0xffffffffu, wait_bar(full, done & 1, dead));
                    if (!ok) break;
                    total += ldsf(at_h);
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release(free);
                }
                ++done;
            }
            if (!mine || par) {
            } else if (u.split < 0) {
                if (live) p.weights[at] = was + total;
            } else {
                // the warp that comes last adds up the parts, in their order
                const int parts = (u.split & 63) + 1, part = (u.split >> 6) & 63, slot = u.split >> 12;
                float *mine_at = p.part + (int64_t)slot * TRACK_MANY_TILE + w * 128 + me;
                __stcg(mine_at + part * TRACK_MANY_TILE, total);
                __syncwarp();
                uint32_t *count = p.arrived + slot * 8 + 4 * w + (warp & 3);
                uint32_t before = 0;
                if (lane == 0) asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;\n" : "=r"(before) : "l"(count) : "memory");
                before = __shfl_sync(0xffffffffu, before, 0);
                __syncwarp();  // (a shuffle orders no memory: what lane 0 acquired is the other lanes' by this)
                if ((int)before + 1 == parts) {
                    total = 0.f;
                    for (int i = 0; i < parts; ++i) total += __ldcg(mine_at + i * TRACK_MANY_TILE);
                    if (live) p.weights[at] = was + total;
                    if (lane == 0) *count = 0;
                }
            }
            if (theirs) take_up();
            if (next) u = it.get(p, per);
        }
        if (!ok && lane == 0) {
            *dead = 1;
            atomicOr(p.err, SALT_DEVERR_TIMEOUT);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, L::TM_COLS);
    if (tid == 0 && *dead) *p.failed = 1;
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q);
        return e == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiled>(f) : nullptr;
    }();
    return fn;
}

// Queries as [tokens][heads][D] bf16, a box 64 elements of a group's heads of `box_tokens` tokens.
cudaError_t encode_queries(CUtensorMap *out, const void *q, int64_t stride, int dim, int heads, int tokens, int G, int box_tokens)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)dim * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)G, (cuuint32_t)box_tokens}, es[3] = {1, 1, 1};
    const CUresult r = encode(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(q), dims, strides, box, es,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <class F>
cudaError_t launch_few(const WeightParams &p, int n_sm, int64_t tiles, cudaStream_t stream)
{
    const cudaError_t e = cudaFuncSetAttribute(weights_few_kernel<F>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::BYTES);
    if (e != cudaSuccess) return e;
    return launch_overlapped(weights_few_kernel<F>, (unsigned)std::min<int64_t>(n_sm * F::CTAS, tiles), F::THREADS, F::BYTES, stream, p);
}

// The lists of many rows on many_sms of the SMs (a CTA has one to itself), beside them those of few, of up to few_rows, on the others.
template <int D>
cudaError_t launch_weights(WeightParams &p, int n_sm, int many_sms, bool few, int few_rows, int64_t few_tiles, cudaStream_t stream)
{
    using M = Many<D>;
    if (many_sms > 0) {
        cudaError_t e = cudaFuncSetAttribute(weights_many_kernel<M>, cudaFuncAttributeMaxDynamicSharedMemorySize, M::BYTES);
        if (e == cudaSuccess) e = launch_overlapped(weights_many_kernel<M>, many_sms, M::THREADS, M::BYTES, stream, p);
        if (e != cudaSuccess) return e;
    }
    if (!few) return cudaSuccess;
    p.behind = many_sms > 0;
    const int sms = many_sms < n_sm ? n_sm - many_sms : n_sm;
    return few_rows <= 16 ? launch_few<Few<D, 16>>(p, sms, few_tiles, stream) : launch_few<Few<D, 64>>(p, sms, few_tiles, stream);
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
    const Track &tr = a->track;
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
    if (st != SALT_OK) return st;
    // a captured call may be replayed for a batch that needs the other kernel (none with more query tokens)
    const bool many = a->T > 0 && (captured || tr.many > 0), few = captured || tr.few > 0;
    if (!many && !few) return SALT_OK;
    WeightParams p;
    p.kmap = a->kmap;
    if (many) {
        const int G = a->cfg.n_heads / kv.heads;
        SALT_CUDA_OR_FAIL(ctx, encode_queries(&p.qmap, q, q_stride, kv.dim, a->cfg.n_heads, a->T, G, 128 / G));
        SALT_CUDA_OR_FAIL(ctx, encode_queries(&p.qmap1, q, q_stride, kv.dim, a->cfg.n_heads, a->T, G, 1));
    }
    p.plan = a->plan;
    p.track = tr.table;
    p.order_at = a->order_at;
    p.pages_at = a->pages_at;
    p.list_at = tr.list_at;
    p.unit_at = tr.unit_at;
    p.kv = kv;
    p.layer = layer;
    p.q = static_cast<const uint16_t *>(q);
    p.lse = lse;
    p.weights = weights;
    p.part = tr.part;
    p.arrived = tr.arrived;
    p.failed = tr.table + TH_FAILED;
    p.q_stride = q_stride;
    p.n_heads = a->cfg.n_heads;
    p.max_tok = a->T;
    p.behind = 0;
    p.n_sm = a->n_sm;
    p.scale = scale;
    p.decay = decay;
    p.err = ctx_error_word(ctx);
    const int64_t tiles = captured ? 1 << 30 : tr.few_tiles * kv.heads;
    const int rows = captured ? TRACK_FEW_ROWS : tr.few_rows, sms = !many ? 0 : captured ? a->n_sm : tr.many_sms;
    SALT_CUDA_OR_FAIL(ctx, kv.dim == 128 ? launch_weights<128>(p, a->n_sm, sms, few, rows, tiles, stream)
                                         : launch_weights<64>(p, a->n_sm, sms, few, rows, tiles, stream));
    return SALT_OK;
} catch (const std::bad_alloc &) {
    return ctx_fail(a->kv->ctx, SALT_ERR_OOM, "no host memory");
}

}  // extern "C"
