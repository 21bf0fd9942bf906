// Requests back to their share of the cache: of each layer, request and
// key/value head the tokens that are kept, and those moved to the front of the
// request's pages in their order.
//
// Kept are the last `recent` tokens, the first `first` ones, and of the others those of
// the largest scores, ties to the earlier one.  Scores are ordered as unsigned
// words; a search by digits from the top, 11, 11 and 10 bits, finds the last word that is kept and how many of its
// ties are.
//
// A kept token's new place is never behind its old one, so rows move in place: a place may be written once what lies
// there was read.  Rows move in chunks. A CTA that moves a whole line has only to take its chunks in order. Where CTAs share a line, each reads a chunk, says
// so, waits for the chunks that read what it will write over (two of those before it at most: they have as many rows as it has places) and writes.
//
// 8 layers of 32 requests of 1,200 to 2,048 tokens with 8 heads of 128: 166 us, 23 for the search (the scores lie in the L2 after the first
// digit; shuffles and shared atomics, issue slots at 59%) and 143 for the move (6.1 TB/s of rows, those of a line's first kept
// tokens that stay where they are neither read nor written).  Two requests of 200,000 tokens and more with heads of 64: 113 us, 37 and 76.
#include <algorithm>
#include <new>

#include "salt_async.cuh"
#include "salt_attn.cuh"
#include "salt_host.cuh"
#include "salt_internal.cuh"
#include "salt_pipe.cuh"

namespace salt {
namespace {

constexpr int DIGITS = 3, BINS = 2048;
constexpr int digit_shift(int d) { return d == 0 ? 21 : d == 1 ? 10 : 0; }

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
    // the plan's workspace: per request the chunks of those before it, per line and chunk how many kept tokens lie before the chunk's
    // first place and whether its rows were read, the next piece of work to move, the requests that lose tokens and how many they are
    int32_t *chunk_ptr, *bound;
    uint32_t *read, *ticket;
    int32_t *losing;            // (the number first)
    int32_t chunks;             // entries of all requests, for one layer and head
    int32_t whole;              // whether there are lines enough that CTAs of the move take some whole
    int32_t key_cap;            // keys of a CTA that its shared memory holds
    uint32_t *err;
};
constexpr int EVICT_POLLS = 1 << 20;  // of a chunk for another's rows (a fraction of a second)

// One layer's, request's and head's own tokens.
struct Line {
    const int32_t *pages;       // of the request
    int64_t page0;              // number of the layer's first page
    int head, len, keep, first, recent;
    int32_t *kept;
    int64_t chunk0;             // its first entry in the chunks' tables
};

// (Tables at places that do not hang on words read before, here and below: plain loads, as those of constants, __ldg, might be moved before the pdl_wait.)
// How many tokens of a request are kept where some go; 0 where none do, or none may stay (-1: not allowed).
__device__ __forceinline__ int kept_of(const EvictParams &p, int seq, int len)
{
    const int keep = p.keep[seq];
    return keep < 0 || keep > p.kept_stride ? -1 : keep < len ? keep : 0;
}
// lh: layer in the launch * heads + head
__device__ __forceinline__ Line load_line(const EvictParams &p, int lh, int seq)
{
    const int layer = lh / p.kv.heads;
    const int4 s = reinterpret_cast<const int4 *>(p.track + p.seq_at)[seq];
    Line l;
    l.head = lh - layer * p.kv.heads;
    l.pages = p.plan + p.pages_at + s.x;
    l.page0 = (p.layer + layer) * p.kv.n_pages;
    l.len = s.y;
    l.keep = max(kept_of(p, seq, l.len), 0);
    l.kept = p.kept + (((int64_t)layer * p.n_seqs + seq) * p.kv.heads + l.head) * p.kept_stride;
    l.recent = min(p.recent, l.keep);
    l.first = min(p.first, l.keep - l.recent);
    l.chunk0 = (int64_t)lh * p.chunks + s.z;
    return l;
}
__device__ __forceinline__ int64_t row_of(const EvictParams &p, const Line &l, int j)
{
    return (((l.page0 + __ldg(l.pages + (j >> p.kv.page_log2))) * p.kv.heads + l.head) << p.kv.page_log2) + (j & (p.kv.page - 1));
}

// Larger scores are larger words; the zeros are one, a NaN is below every number.  0 and the largest word are no scores'.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __float_as_uint(x);
    if (!(x == x)) return 1u;
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

// A word of another CTA of the cluster.
__device__ __forceinline__ uint32_t peer_word(uint32_t addr, uint32_t rank)
{
    uint32_t at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(at) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];\n" : "=r"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync(uint32_t n)
{
    if (n == 1) {
        __syncthreads();
        return;
    }
    cluster_arrive();
    cluster_wait();
}

// The places of a line's kept tokens, by a cluster, each CTA a run of the line's tokens, each warp a run of those.
template <int THREADS, int ROWS>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(const __grid_constant__ EvictParams p)
{
    constexpr int WARPS = THREADS / 32;
    constexpr bool ALONE = THREADS < 1024;              // a line has one CTA
    constexpr int HISTS = ALONE ? 1 : DIGITS;           // (other CTAs may still read the last digit's)
    extern __shared__ __align__(16) uint32_t s_keys[];
    __shared__ __align__(16) uint32_t s_hist[HISTS][BINS], s_coarse[HISTS][BINS / 32], s_total[96], s_warp[32], s_held[WARPS], s_tied[WARPS], s_all[2], s_most;
    pdl_wait();
    // (the warp's number from a shuffle, so that branches by it are known to be taken by whole warps)
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31, n_seqs = p.track[TH_SEQS];
    uint32_t C, rank;
    if (ALONE) {
        C = 1;
        rank = 0;
    } else {
        asm volatile("mov.u32 %0, %%cluster_nctarank;\n" : "=r"(C));
        asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
    }
    const bool fits = n_seqs <= p.n_seqs && !p.track[TH_SHARED];
    if (blockIdx.x == 0) {  // the chunks of every request, once for all layers and heads
        int before = 0;
        uint32_t losing = 0;
        if (tid == 0) s_most = 0;
        for (int s0 = 0; fits && s0 < n_seqs; s0 += THREADS) {
            const int s = s0 + tid, keep = s < n_seqs ? kept_of(p, s, p.track[p.seq_at + s * SEQ_WORDS + 1]) : 0;
            if (keep < 0) atomicOr(p.err, SALT_DEVERR_KEEP);
            uint32_t all;
            const uint32_t n = (max(keep, 0) + ROWS - 1) / ROWS, up_to = block_scan(n, s_warp, &all);
            if (s < n_seqs) p.chunk_ptr[s + 1] = before + (int)up_to;
            before += (int)all;
            if (!p.whole) continue;
            const uint32_t at = block_scan(n > 0, s_warp, &all);
            if (n > 0) {
                p.losing[losing + at] = s;
                atomicMax(&s_most, n);
            }
            losing += all;
        }
        if (p.whole) {  // lines of very different lengths are all shared: a CTA with a long one would be at it when the others are done
                        // (8 lines of 60,000 tokens among 240 of 1,500: 415 us whole, 122 shared)
            __syncthreads();
            if (4ll * s_most * losing > 5ll * before) losing = 0;
        }
        if (tid == 0) {
            p.chunk_ptr[0] = 0;
            p.ticket[0] = 0;
            p.losing[0] = (int)losing;
            if (!fits) atomicOr(p.err, SALT_DEVERR_BATCH);
        }
    }
    const int line = blockIdx.x / C, lh = line / p.n_seqs, seq = line - lh * p.n_seqs;
    if (!fits || seq >= n_seqs) return;  // (the cluster together)
    const Line l = load_line(p, lh, seq);
    if (l.keep == 0) return;
    // (known to be a warp's, like its number: shuffles and votes in loops and branches by them are quick then)
    auto uniform = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
    const int len = uniform(l.len), from = uniform(l.first), to = uniform(l.len - l.recent);
    const int warp_run = ((len + (int)C * WARPS - 1) / ((int)C * WARPS) + 127) & ~127, cta0 = (int)rank * WARPS * warp_run, warp0 = cta0 + warp * warp_run;
    const int warp1 = min(len, warp0 + warp_run);
    auto clear = [&]() {
        for (int i = tid; i < HISTS * BINS / 4; i += THREADS) reinterpret_cast<uint4 *>(s_hist[0])[i] = make_uint4(0, 0, 0, 0);
    };
    clear();
    for (int c = (int)rank * THREADS + tid; c * ROWS < l.keep; c += (int)C * THREADS) p.read[l.chunk0 + c] = 0;
    __syncthreads();
    // A warp goes over its run 128 tokens at a time, four of a page a lane.  The first and last tokens, kept in any case, have the largest word, places
    // past the line the least.
    auto fetch = [&](int j) {
        uint4 x = make_uint4(0, 0, 0, 0);
        if (j >= len) return x;
        const float4 f = __ldg(reinterpret_cast<const float4 *>(p.scores + row_of(p, l, j)));
        x = make_uint4(key_of(f.x), key_of(f.y), key_of(f.z), key_of(f.w));
        if (j < from || j + 4 > to) {
            uint32_t *key[4] = {&x.x, &x.y, &x.z, &x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (j + i < from || j + i >= to) *key[i] = j + i < len ? 0xffffffffu : 0u;
        }
        return x;
    };
    auto keys_at = [&](int j0) {  // (key_cap is a multiple of 128)
        return j0 - cta0 < p.key_cap ? *reinterpret_cast<const uint4 *>(s_keys + (j0 - cta0) + 4 * lane) : fetch(j0 + 4 * lane);
    };
    constexpr int AHEAD = ALONE ? 2 : 8;  // groups under way
#pragma unroll 1
    for (int j0 = warp0; j0 < warp1; j0 += 128 * AHEAD) {
        uint4 x[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) x[k] = fetch(j0 + 128 * k + 4 * lane < warp1 ? j0 + 128 * k + 4 * lane : len);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int j = j0 + 128 * k;
            if (j >= warp1) break;
            if (j - cta0 < p.key_cap) *reinterpret_cast<uint4 *>(s_keys + (j - cta0) + 4 * lane) = x[k];
            // (equal scores are common: a lane's, and a warp's, count as one)
            const uint32_t bin[4] = {x[k].x >> digit_shift(0), x[k].y >> digit_shift(0), x[k].z >> digit_shift(0), x[k].w >> digit_shift(0)};
            const bool same = bin[0] == bin[1] && bin[0] == bin[2] && bin[0] == bin[3];
            const uint32_t lead = __shfl_sync(0xffffffffu, bin[0], 0);
            if (__all_sync(0xffffffffu, same && bin[0] == lead)) {
                if (lane == 0) atomicAdd(&s_hist[0][lead], 128u);
            } else if (same) {
                atomicAdd(&s_hist[0][bin[0]], 4u);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) atomicAdd(&s_hist[0][bin[i]], 1u);
            }
            __syncwarp();
        }
    }
    // the smallest word that is kept, and `want` of those that are equal to it
    uint32_t want = (uint32_t)uniform(l.keep), prefix = 0;
#pragma unroll 1
    for (int d = 0; d < DIGITS; ++d) {
        if (d > 0) {  // of the words whose digits above are `prefix`
            const int shift = digit_shift(d), above = shift + (d == 2 ? 10 : 11);
            const uint32_t mask = d == 2 ? 1023u : 2047u;
            uint32_t *to_hist = s_hist[d % HISTS];
#pragma unroll 1
            for (int j0 = warp0; j0 < warp1; j0 += 128) {
                const uint4 x = keys_at(j0);
                const uint32_t key[4] = {x.x, x.y, x.z, x.w};
                bool in[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) in[i] = key[i] >> above == prefix;
                if (!__any_sync(0xffffffffu, in[0] || in[1] || in[2] || in[3])) continue;
                const uint32_t lead = __shfl_sync(0xffffffffu, key[0] >> shift, 0);
                const bool same = in[0] && key[0] >> shift == lead && key[1] >> shift == lead && key[2] >> shift == lead && key[3] >> shift == lead;
                if (__all_sync(0xffffffffu, same)) {
                    if (lane == 0) atomicAdd(&to_hist[lead & mask], 128u);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (in[i]) atomicAdd(&to_hist[key[i] >> shift & mask], 1u);
                }
                __syncwarp();
            }
        }
        const uint32_t *hist = s_hist[d % HISTS], *coarse = s_coarse[d % HISTS];
        __syncthreads();
#pragma unroll 2
        for (int g = warp; g < BINS / 32; g += WARPS) {
            const uint32_t sum = __reduce_add_sync(0xffffffffu, hist[g * 32 + lane]);
            if (lane == 0) s_coarse[d % HISTS][g] = sum;
        }
        cluster_sync(C);
        // from the largest digit down: the 32 bins that hold the last one kept, then which of them.  (Every warp does the same, without
        // branches: in one warp, inside a branch, the shuffles took 2 us a digit.)
        auto total = [&](const uint32_t *at) {
            uint32_t n = 0;
#pragma unroll
            for (uint32_t r = 0; r < 8; ++r)
                if (r < C) n += peer_word(smem_u32(at), r);
            return n;
        };
        if (!ALONE) {
            if (tid < BINS / 32) s_total[tid] = total(coarse + tid);
            __syncthreads();
            coarse = s_total;
        }
        auto scan = [&](uint32_t n) {
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, n, o);
                if (lane >= o) n += x;
            }
            return n;
        };
        const uint32_t a = coarse[63 - 2 * lane], ab = a + coarse[62 - 2 * lane], ab_to = scan(ab);
        const int two = __ffs(__ballot_sync(0xffffffffu, ab_to >= want)) - 1;
        uint32_t before = __shfl_sync(0xffffffffu, ab_to - ab, two);
        const uint32_t a_there = __shfl_sync(0xffffffffu, a, two);
        const bool second = before + a_there < want;
        before += second ? a_there : 0u;
        const int bin0 = (63 - 2 * two - second) * 32;
        if (!ALONE) {
            if (tid < 32) s_total[64 + tid] = total(hist + bin0 + tid);
            __syncthreads();
        }
        const uint32_t n = ALONE ? hist[bin0 + 31 - lane] : s_total[64 + 31 - lane], n_to = scan(n);
        const int at = __ffs(__ballot_sync(0xffffffffu, before + n_to >= want)) - 1;
        before += __shfl_sync(0xffffffffu, n_to - n, at);
        prefix = prefix << (d == 2 ? 10 : 11) | (uint32_t)(bin0 + 31 - at);
        want -= before;
        if (ALONE && d + 1 < DIGITS) {
            __syncthreads();
            clear();
            __syncthreads();
        }
    }
    uint32_t held = 0, tied = 0;  // words above, and equal
#pragma unroll 1
    for (int j0 = warp0; j0 < warp1; j0 += 128) {
        const uint4 x = keys_at(j0);
        held += (x.x > prefix) + (x.y > prefix) + (x.z > prefix) + (x.w > prefix);
        tied += (x.x == prefix) + (x.y == prefix) + (x.z == prefix) + (x.w == prefix);
    }
    held = __reduce_add_sync(0xffffffffu, held);
    tied = __reduce_add_sync(0xffffffffu, tied);
    if (lane == 0) {
        s_held[warp] = held;
        s_tied[warp] = tied;
    }
    __syncthreads();
    uint32_t held0 = lane < warp ? s_held[lane] : 0u, tied0 = lane < warp ? s_tied[lane] : 0u;
    held0 = __reduce_add_sync(0xffffffffu, held0);
    tied0 = __reduce_add_sync(0xffffffffu, tied0);
    if (C > 1) {
        if (warp == WARPS - 1 && lane == 0) {
            s_all[0] = held0 + held;
            s_all[1] = tied0 + tied;
        }
        cluster_sync(C);
#pragma unroll
        for (uint32_t r = 0; r < 8; ++r)
            if (r < rank) {
                held0 += peer_word(smem_u32(&s_all[0]), r);
                tied0 += peer_word(smem_u32(&s_all[1]), r);
            }
        cluster_arrive();  // (nobody leaves while its words are read)
    }
    pdl_launch_dependents();
    const uint32_t below = (1u << lane) - 1u;
    uint32_t out0 = held0 + min(tied0, want);  // kept before the warp's run
#pragma unroll 1
    for (int j0 = warp0; j0 < warp1; j0 += 128) {
        const int j = j0 + 4 * lane;
        const uint4 x = keys_at(j0);
        const uint32_t key[4] = {x.x, x.y, x.z, x.w};
        bool h[4], t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = key[i] > prefix;
            t[i] = key[i] == prefix;
        }
        // of a number below 8 a lane, the sum over the lanes before, and over all
        auto ranks = [&](uint32_t n, uint32_t &all) {
            uint32_t before = 0;
            all = 0;
#pragma unroll
            for (int b = 0; b < 3; ++b) {
                const uint32_t on = __ballot_sync(0xffffffffu, n >> b & 1);
                before += __popc(on & below) << b;
                all += __popc(on) << b;
            }
            return before;
        };
        const uint32_t ties = t[0] + t[1] + t[2] + t[3];
        if (__any_sync(0xffffffffu, ties > 0)) {  // the first `want` ties are kept
            uint32_t all, rank_t = tied0 + ranks(ties, all);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[i] = h[i] || (t[i] && rank_t < want);
                rank_t += t[i];
            }
            tied0 += all;
        }
        uint32_t all, out = out0 + ranks(h[0] + h[1] + h[2] + h[3], all);
        out0 += all;
        if (j % ROWS == 0 && j < l.keep + ROWS && j < len) p.bound[l.chunk0 + j / ROWS] = (int)out;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (h[i]) l.kept[out++] = j + i;
    }
    if (C > 1) cluster_wait();
}

// The CTAs draw whole lines first, as many as go evenly into them, and then the others' chunks one by one, in their order, so that those that a chunk waits for
// are under way.  A CTA has some chunks in slots of its shared memory, and its warps deal with them in turn: one looks up the rows' places, some read the keys
// and values, one the exponents and weights, two say in turn when all are there, one waits for the chunks that read what this one will write over, some write.
// Reading runs ahead of writing by all the slots, whatever writing waits for.  (Where a chunk was read only once the one before it was written, chunks
// waited for each other in long chains, 7 us each.)  Within a line of its own a CTA's slots order reading and writing: a chunk that was read tells that those
// before it were.  Between CTAs a chunk's flag is a release behind its reads, and the wait for it an acquire before the stores that write over them.  These cost: the
// release takes as long as the stores under way, and the acquire empties the L1.  8 layers of 32 requests take 208 us by chunks (232 with one warp that says so and
// has its slot meanwhile; 187 if nothing ordered them) and 166 by lines; 16 lines of 200,000 tokens and more 113 (121, 109).  Several chunks of a line
// a CTA are worse than either (up to 560 us: a run's first chunk waits for the last one of the run before).
constexpr int SLOTS = 5, LOAD_WARPS = 4, STORE_WARPS = 4, SAY_WARPS = 2, MOVE_THREADS = 32 * (LOAD_WARPS + STORE_WARPS + 3 + SAY_WARPS);

template <int D_, int ROWS_>
struct Move {
    static constexpr int D = D_, ROWS = ROWS_;
    static constexpr int LPR = D / 16;                                    // lanes a row
    static constexpr uint32_t K = 0, V = ROWS * D, W = 2 * ROWS * D;      // a slot: keys, values, weights,
    static constexpr uint32_t E = W + 4 * ROWS;                           // exponents of k and v,
    static constexpr uint32_t SRC = E + 2 * ROWS, DST = SRC + 4 * ROWS;   // old and new rows (new -1: stays)
    static constexpr uint32_t SLOT = DST + 4 * ROWS;
    static constexpr uint32_t BYTES = SLOTS * SLOT;
    static_assert(SLOT % 16 == 0 && 2 * (BYTES + 2048) <= 228 * 1024, "two CTAs an SM");
};

template <class M, bool WHOLE>
__global__ void __launch_bounds__(MOVE_THREADS, 2) evict_move_kernel(const __grid_constant__ EvictParams p, int layers)
{
    constexpr int D = M::D, ROWS = M::ROWS;
    extern __shared__ __align__(16) uint8_t s_slots[];
    __shared__ __align__(8) uint64_t s_full[SLOTS], s_free[SLOTS], s_read[SLOTS], s_clear[SLOTS];
    __shared__ int64_t s_chunk[SLOTS];     // the chunk's entry, -1: no more
    __shared__ int32_t s_wait[SLOTS][2];   // the first and last chunk of the line that it waits for, from here
    __shared__ int32_t s_alone[SLOTS];     // whether it is of a whole line: none waits for it
    __shared__ int s_dead;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    volatile int *dead = &s_dead;
    if (tid == 0) {
        for (int i = 0; i < SLOTS; ++i) {
            mbar_init(smem_u32(&s_full[i]), 1);
            mbar_init(smem_u32(&s_free[i]), STORE_WARPS + 1 + SAY_WARPS);
            mbar_init(smem_u32(&s_read[i]), 32 * LOAD_WARPS + 1);
            mbar_init(smem_u32(&s_clear[i]), 1);
        }
        s_dead = 0;
        mbar_fence_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    // (known to be a warp's words: what goes by them, votes and shuffles too, is quick then)
    auto uniform = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
    const int n_seqs = uniform(p.track[TH_SEQS]);
    if (n_seqs > p.n_seqs || p.track[TH_SHARED]) return;
    bool ok = true;
    auto wait = [&](uint64_t *bars, uint32_t n) {  // for the n-th use of its slot
        ok = ok && wait_bar(smem_u32(&bars[n % SLOTS]), (n / SLOTS) & 1, dead);
        ok = __all_sync(0xffffffffu, ok);
        return ok;
    };
    auto arrive = [&](uint64_t *bars, uint32_t n) {
        __syncwarp();
        if (lane == 0) mbar_arrive_release(smem_u32(&bars[n % SLOTS]));
    };
    // the chunk in a slot, -1 behind the last
    auto chunk_of = [&](uint32_t n) { return (int64_t)uniform((int)(s_chunk[n % SLOTS] >> 32)) << 32 | (uint32_t)uniform((int)s_chunk[n % SLOTS]); };
    auto slot_of = [&](uint32_t n) { return s_slots + (n % SLOTS) * M::SLOT; };
    if (warp == LOAD_WARPS + STORE_WARPS) {
        // ------------------------------------------------ places
        // (a chunk's line is found while the places of the one before are on their way: the waits for other chunks empty the L1)
        const int per_lh = uniform(p.chunk_ptr[n_seqs]), losing = WHOLE ? uniform(p.losing[0]) : 0;
        const uint32_t all = (uint32_t)per_lh * p.kv.heads * layers;  // (below 2^27, as a layer's rows are below 2^31)
        // Lines that are taken whole: full rounds of one a CTA, and all where the last round is half full.  (200 lines, two thirds of a round, take 86 us so
        // and 95 by chunks; 160 lines 50 and 51.)
        const int ctas = gridDim.x, lines = losing * p.kv.heads * layers;
        const uint32_t whole = min(lines, (lines + ctas / 2) / ctas * ctas);
        uint32_t chunk_at = 0;  // the first chunk of the other lines
        if (WHOLE && whole > 0) {
            const int lh = (int)whole / losing, at = (int)whole - lh * losing;
            chunk_at = (uint32_t)lh * per_lh + (at > 0 ? uniform(p.chunk_ptr[p.losing[1 + at]]) : 0);  // (before the first of these there are none)
        }
        struct Work {
            Line l;
            int c, end;   // chunks [c, end) of the line
            bool more, alone;
        };
        auto find = [&](uint32_t t) {
            Work r;
            r.alone = WHOLE && uniform(t < whole);
            r.c = r.end = 0;
            if (r.alone) {
                const int lh = (int)t / losing;
                r.more = true;
                r.l = load_line(p, lh, uniform(p.losing[1 + (int)t - lh * losing]));
                r.end = (uniform(r.l.keep) + ROWS - 1) / ROWS;
                return r;
            }
            t += chunk_at - whole;
            r.more = uniform(t < all);
            if (!r.more) return r;
            const int lh = t / (uint32_t)per_lh, x = t - (uint32_t)lh * per_lh;
            int lo = 0, n = n_seqs;  // the last request that begins at or before x is one of n
            while (n > 1) {
                const int step = (n + 31) / 32, at = lane * step;
                const uint32_t on = __ballot_sync(0xffffffffu, at < n && p.chunk_ptr[lo + min(at, n - 1)] <= x);
                const int last = 31 - __clz(on);  // (lane 0 is)
                lo += last * step;
                n = min(step, n - last * step);
            }
            r.c = x - uniform(p.chunk_ptr[lo]);
            r.end = r.c + 1;
            r.l = load_line(p, lh, lo);
            return r;
        };
        uint32_t ticket = 0;
        auto draw = [&]() {
            if (lane == 0) ticket = atomicAdd(p.ticket, 1u);
        };
        draw();
        // (drawn a chunk ahead, not sooner: others may wait for a chunk that is drawn)
        Work now = find(__shfl_sync(0xffffffffu, ticket, 0));
        if (!WHOLE || uniform(now.end - now.c) <= 1) draw();
        for (uint32_t n = 0;; ++n) {
            const int slot = n % SLOTS;
            if (!now.more) {
                if (n >= SLOTS && !wait(s_free, n - SLOTS)) break;
                if (lane == 0) s_chunk[slot] = -1;
                arrive(s_full, n);
                break;
            }
            const Line &l = now.l;
            const int c = now.c;
            int src[ROWS / 32], dst[ROWS / 32], from[ROWS / 32];
#pragma unroll
            for (int k = 0; k < ROWS / 32; ++k) {
                const int i = c * ROWS + 32 * k + lane;
                from[k] = i < l.keep ? l.kept[i] : i;
            }
            const int b0 = p.bound[l.chunk0 + c], b1 = (c + 1) * ROWS < l.len ? p.bound[l.chunk0 + c + 1] : l.keep;
            Work next = now;
            const int left = WHOLE ? uniform(now.end - ++next.c) : 0;
            if (left == 0) next = find(__shfl_sync(0xffffffffu, ticket, 0));
            if (!WHOLE || (left == 0 ? uniform(next.end - next.c) <= 1 : left == 1)) draw();
#pragma unroll
            for (int k = 0; k < ROWS / 32; ++k) {
                const int i = c * ROWS + 32 * k + lane;
                src[k] = 0;
                dst[k] = -1;
                if (from[k] != i) {
                    src[k] = (int)row_of(p, l, from[k]);
                    dst[k] = (int)row_of(p, l, i);
                }
            }
            if (n >= SLOTS && !wait(s_free, n - SLOTS)) break;
#pragma unroll
            for (int k = 0; k < ROWS / 32; ++k) {
                reinterpret_cast<int32_t *>(slot_of(n) + M::SRC)[32 * k + lane] = src[k];
                reinterpret_cast<int32_t *>(slot_of(n) + M::DST)[32 * k + lane] = dst[k];
            }
            if (lane == 0) {
                s_chunk[slot] = l.chunk0 + c;
                // kept tokens [b0, b1) lie where this chunk will: chunks of the line up to this one
                s_wait[slot][0] = b1 > b0 && !now.alone ? b0 / ROWS - c : 0;
                s_wait[slot][1] = b1 > b0 && !now.alone ? (b1 - 1) / ROWS - c : 0;
                if (WHOLE) s_alone[slot] = now.alone;
            }
            arrive(s_full, n);
            now = next;
        }
    } else if (warp >= LOAD_WARPS + STORE_WARPS + 3) {
        // ------------------------------------------------ chunks that were read
        for (uint32_t n = 0; wait(s_full, n); ++n) {
            const int64_t chunk = chunk_of(n);
            if (chunk < 0) break;
            const bool mine = n % SAY_WARPS == (uint32_t)(warp - (LOAD_WARPS + STORE_WARPS + 3));
            if (mine && !wait(s_read, n)) break;
            const bool alone = WHOLE && s_alone[n % SLOTS];
            arrive(s_free, n);  // (before the release, which takes as long as the stores under way)
            if (lane == 0 && mine && !alone) asm volatile("st.release.gpu.global.u32 [%0], %1;\n" ::"l"(p.read + chunk), "r"(1u) : "memory");
        }
    } else if (warp == LOAD_WARPS + STORE_WARPS + 1) {
        // ------------------------------------------------ chunks to wait for
        for (uint32_t n = 0; wait(s_full, n); ++n) {
            const int64_t chunk = chunk_of(n);
            if (chunk < 0) break;
            if (lane < 2 && s_wait[n % SLOTS][lane] < 0) {
                const uint32_t *flag = p.read + chunk + s_wait[n % SLOTS][lane];
                uint32_t x = 0;
                for (int i = 0; i < EVICT_POLLS && !x && !*dead; ++i)
                    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];\n" : "=r"(x) : "l"(flag) : "memory");
                ok = x != 0;
            }
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            arrive(s_clear, n);
            arrive(s_free, n);
        }
    } else if (warp == LOAD_WARPS + STORE_WARPS + 2) {
        // ------------------------------------------------ exponents and weights, the next chunk's on their way
        uint32_t ke[2][ROWS / 32], ve[2][ROWS / 32];
        float w[2][ROWS / 32];
        auto load = [&](int b, uint32_t n) {
            if (!wait(s_full, n) || chunk_of(n) < 0) return false;
#pragma unroll
            for (int k = 0; k < ROWS / 32; ++k) {
                const int r = 32 * k + lane;
                ke[b][k] = ve[b][k] = 0;
                w[b][k] = 0.f;
                if (reinterpret_cast<const int32_t *>(slot_of(n) + M::DST)[r] >= 0) {
                    const int64_t at = reinterpret_cast<const int32_t *>(slot_of(n) + M::SRC)[r];
                    ke[b][k] = p.kv.k_exp[at];
                    ve[b][k] = p.kv.v_exp[at];
                    if (p.weights) w[b][k] = p.weights[at];
                }
            }
            return true;
        };
        auto put = [&](int b, uint32_t n) {
#pragma unroll
            for (int k = 0; k < ROWS / 32; ++k) {
                const int r = 32 * k + lane;
                (slot_of(n) + M::E)[r] = (uint8_t)ke[b][k];
                (slot_of(n) + M::E)[ROWS + r] = (uint8_t)ve[b][k];
                reinterpret_cast<float *>(slot_of(n) + M::W)[r] = w[b][k];
            }
            arrive(s_read, n);
        };
        bool more = load(0, 0);
        for (uint32_t n = 0; more; n += 2) {
            more = load(1, n + 1);
            put(0, n);
            if (!more) break;
            more = load(0, n + 2);
            put(1, n + 1);
        }
    } else if (warp < LOAD_WARPS) {
        // ------------------------------------------------ keys and values into the slot
        const int part = tid % M::LPR;
        for (uint32_t n = 0; wait(s_full, n) && chunk_of(n) >= 0; ++n) {
            uint8_t *slot = slot_of(n);
            const int32_t *src = reinterpret_cast<const int32_t *>(slot + M::SRC), *dst = reinterpret_cast<const int32_t *>(slot + M::DST);
#pragma unroll
            for (int r = tid / M::LPR; r < ROWS; r += 32 * LOAD_WARPS / M::LPR) {
                const bool moves = dst[r] >= 0;
                const int64_t from = (int64_t)src[r] * D + part * 16;
                cp_async16(smem_u32(slot + M::K + r * D + part * 16), p.kv.k + from, moves);
                cp_async16(smem_u32(slot + M::V + r * D + part * 16), p.kv.v + from, moves);
            }
            cp_async_arrive_noinc(smem_u32(&s_read[n % SLOTS]));
        }
        cp_async_commit();
        cp_async_wait<0>();
    } else {
        // ------------------------------------------------ out of it
        const int me = tid - 32 * LOAD_WARPS, part = me % M::LPR;
        for (uint32_t n = 0; wait(s_full, n) && chunk_of(n) >= 0; ++n) {
            if (!wait(s_read, n) || !wait(s_clear, n)) break;
            const uint8_t *slot = slot_of(n);
            const int32_t *dst = reinterpret_cast<const int32_t *>(slot + M::DST);
#pragma unroll
            for (int r = me / M::LPR; r < ROWS; r += 32 * STORE_WARPS / M::LPR) {
                const int64_t to = dst[r];
                if (to < 0) continue;
                reinterpret_cast<uint4 *>(p.kv.k + to * D)[part] = *reinterpret_cast<const uint4 *>(slot + M::K + r * D + part * 16);
                reinterpret_cast<uint4 *>(p.kv.v + to * D)[part] = *reinterpret_cast<const uint4 *>(slot + M::V + r * D + part * 16);
            }
            if (me < ROWS && dst[me] >= 0) {
                const int64_t to = dst[me];
                p.kv.k_exp[to] = (slot + M::E)[me];
                p.kv.v_exp[to] = (slot + M::E)[ROWS + me];
                if (p.weights) p.weights[to] = reinterpret_cast<const float *>(slot + M::W)[me];
            }
            arrive(s_free, n);
        }
    }
    if (!ok && lane == 0) {
        s_dead = 1;
        atomicOr(p.err, SALT_DEVERR_TIMEOUT);
    }
}

template <int THREADS>
constexpr int key_cap() { return THREADS < 1024 ? 32 * THREADS : 48128; }  // (with the counts an SM's shared memory)

template <int THREADS, int ROWS>
cudaError_t launch_select(const EvictParams &params, int64_t lines, int ctas, cudaStream_t stream, int len)
{
    constexpr int CAP = key_cap<THREADS>();
    EvictParams p = params;
    const int64_t run = ((int64_t)len + ctas * (THREADS / 32) - 1) / (ctas * (THREADS / 32));
    p.key_cap = (int)std::min<int64_t>(CAP, (run + 127) / 128 * 128 * (THREADS / 32));
    cudaError_t e = cudaFuncSetAttribute(evict_select_kernel<THREADS, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize, CAP * 4);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(lines * ctas), 1, 1);
    cfg.blockDim = dim3(THREADS, 1, 1);
    cfg.dynamicSmemBytes = (size_t)p.key_cap * 4;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, evict_select_kernel<THREADS, ROWS>, p);
}

template <int D>
cudaError_t launch_evict(EvictParams &p, int n_sm, int layers, int longest, int64_t chunks, bool captured, cudaStream_t stream)
{
    constexpr int ROWS = evict_rows(D);
    const int64_t lines = (int64_t)layers * p.n_seqs * p.kv.heads;
    p.whole = lines >= n_sm;  // (the move has two CTAs an SM; 100 lines by chunks take 35 us without looking for whole ones, 37 with)
    // Long lines go to several CTAs, up to 6: clusters of 8 whose CTAs take an SM each fit 15 times into the card's
    // SMs, of 6 at least 20 times (16 lines of 262,144 tokens: 151 us with 8, one of them in a second wave, 108 with 6, all else alike but for some shorter code).
    int ctas = 1;
    while (ctas < 6 && longest > 8192 * ctas && lines * (ctas + 1) <= n_sm) ++ctas;
    // Short lines that are more than a wave of CTAs of 256 threads, 8 an SM, go by CTAs of 128.  (All of an eviction that keeps 8 tokens: 2,432 lines of 500, 1,000,
    // 2,040 and 4,000 tokens 29, 32, 39 and 51 us with 128 threads, 33, 37, 41 and 52 with 256; 1,824 lines 27, 29, 31 and 43, 27, 29, 33 and 41; 1,216 lines
    // 24, 27, 29 and 29, 21, 22, 25 and 30; 304 lines 19, 22, 24 and 24, 16, 18, 20 and 26.)
    const cudaError_t e1 = longest <= 2048 && lines > 8 * n_sm ? launch_select<128, ROWS>(p, lines, 1, stream, longest)
                           : longest <= 4096                   ? launch_select<256, ROWS>(p, lines, 1, stream, longest)
                                                               : launch_select<1024, ROWS>(p, lines, ctas, stream, longest);
    cudaError_t e = e1;
    if (e != cudaSuccess) return e;
    const int64_t most = captured ? 2 * n_sm : chunks * p.kv.heads * layers;  // (a captured call may be replayed on more)
    using M = Move<D, ROWS>;
    const auto move = p.whole ? evict_move_kernel<M, true> : evict_move_kernel<M, false>;
    e = cudaFuncSetAttribute(move, cudaFuncAttributeMaxDynamicSharedMemorySize, M::BYTES);
    if (e != cudaSuccess) return e;
    return launch_overlapped(move, (unsigned)std::max<int64_t>(1, std::min<int64_t>(most, 2 * n_sm)), MOVE_THREADS, M::BYTES, stream, p, layers);
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
    const Track &tr = a->track;
    p.chunk_ptr = tr.chunk_ptr;
    p.bound = tr.bound;
    p.read = tr.read;
    p.ticket = tr.ticket;
    p.losing = tr.losing;
    p.chunks = tr.chunks_cap;
    p.whole = p.key_cap = 0;
    // as many layers at a time as the workspace has chunks for
    for (int32_t l = 0; l < n_layers; l += tr.layers_cap) {
        const int32_t n = std::min(tr.layers_cap, n_layers - l);
        p.layer = layer + l;
        p.kept = kept + (int64_t)l * p.n_seqs * kv.heads * kept_stride;
        SALT_CUDA_OR_FAIL(ctx, kv.dim == 128 ? launch_evict<128>(p, a->n_sm, n, tr.longest, tr.chunks, captured, stream)
                                             : launch_evict<64>(p, a->n_sm, n, tr.longest, tr.chunks, captured, stream));
    }
    return SALT_OK;
} catch (const std::bad_alloc &) {
    return ctx_fail(a->kv->ctx, SALT_ERR_OOM, "no host memory");
}

}  // extern "C"
