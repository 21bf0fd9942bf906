// Attention of a batch over the paged 8-bit cache, requests of a group
// sharing their prompt.
//
// The work is cut into items: up to R rows (query token x query heads of one
// key/value head) against a range of cached tokens, either a group's prompt
// (rows of all its requests) or a request's own tokens.  An item walks its
// range in tiles of 128 tokens, on the tensor cores with the cache as the
// 128-row operand A, so that few query rows waste little:
//     S^T[token][row] = K[token][:] . Q[row][:]            (M = 128, N = R, e4m3)
//     O^T[dim][row]  += V[token][dim] P[token][row]        (M = D, K = tokens, f16)
// The e4m3 codes of K go from the cache to the MMA as they are, those of V
// are widened to f16 on the way (both exact); the exponents of a token's row
// multiply its scores (K) and its probabilities (V), exact too.  Q meets K as
// two e4m3 terms, hi + lo: the 8 bits of a bf16 are 4 and 4 (elements below 2^-9 of
// the row's largest are off by up to 2^-17 of that).  P is f16: 2^-12 relative,
// and 2^-27 of the row's largest where that is more.
//
// Softmax: thread = token, registers = rows.  The reference m of a row moves
// only when a probability passes f16's range (a vote a tile), so the usual tile
// needs no reduction over tokens: p = 2^(s - m), l += p, P = p 2^(e_v + P_UP), e_v the exponent of the token's value
// under the range's largest.  m follows the largest P; where values are small or zero p is far above it, so l
// counts p in units that leave room.  Items of one row meet in the combine kernel through their (o / l, m + log2 l).
//
// What bounds it: neither memory nor the tensor cores but the steps of a tile one behind the
// other (scores out of tensor memory, exponentials, P and V into shared memory, vote, product).  With 128
// rows of 128 elements a tile takes about 4,300 cycles, of which exponentials would take 512 at the SM's rate (32 a
// cycle, measured) and the products 512: four prompt chunks of 900 to 2,048 tokens behind 4,096 take 1.22 ms
// (515 TFLOP/s).  With four rows it is 2,100 cycles, two CTAs of an SM side by side: two requests of 200,000
// tokens and more with heads of 64 take 95.5 us (4.7 TB/s).
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include <cuda_fp16.h>

#include "salt_async.cuh"
#include "salt_host.cuh"
#include "salt_internal.cuh"
#include "salt_pipe.cuh"
#include "salt_tcgen05.cuh"

namespace salt {
namespace {

// The plan's device tables: int32 words of one block, written by the host
// into a staging area and copied by a kernel.
constexpr int HEAD_WORDS = 8;   // HD_* below
constexpr int HD_TOKENS = 0, HD_WIDE = 1, HD_NARROW = 2, HD_PARTIAL = 3;  // query tokens, records of either kind, whether rows need the combine
constexpr int TOK_WORDS = 8;    // per query token: where its partial rows are, see TK_*
constexpr int TK_OWN = 0, TK_OWN_ROWS = 1, TK_OWN_N = 2, TK_PRE = 3, TK_PRE_ROWS = 4, TK_PRE_N = 5, TK_DIRECT = 6;
constexpr int REC_WORDS = 8;    // per item, shared by the key/value heads
// flags (class, RF_*), first entry in the token order, tokens, first entry in the page lists, first and last + 1 cached
// token, tokens the first query token sees, first partial row
constexpr int RC_FLAGS = 0, RC_TOK = 1, RC_NTOK = 2, RC_PAGES = 3, RC_T0 = 4, RC_T1 = 5, RC_LIM = 6, RC_PART = 7;
constexpr int RF_DIRECT = 8, RF_CAUSAL = 16;

constexpr int TT = 128;          // cached tokens a tile
constexpr int WG = 128;          // threads of a softmax warpgroup (one per token of a tile)
// The largest P is in [2^2, 2^16), a p in units of 2^-P_UP and where the value is small up to 2^P_LOW above that: the sum of 2^26
// tokens is in fp32's range, and where a p above 2^128 makes a sum infinite what it held before was nothing
// next to it.  A row's P lose bits where one of 2^-P_LOW of its values or less (or zero) has 2^(P_LOW + 16) times their probability.
constexpr int P_UP = 40, P_LOW = 125;
constexpr float P_HOT = 120.f;   // log2 of a p that sums may not hold
constexpr float P_TOP = 2.f;     // a new reference puts the row's largest P at 2^2
constexpr float P_MOST = 15.9f;  // and is due when one passes 2^15.9 (f16 ends at 65504)
constexpr int NEVER = 0x7fffffff; // the place of a range's first value that stands for NaN where there is none
constexpr float M_NONE = -1e30f; // the reference before the first token

struct AttnParams {
    alignas(64) CUtensorMap kmap;  // the codes of every layer as rows of D bytes, box of one page
    alignas(64) CUtensorMap vmap;
    const int32_t *plan;           // header, token records, token order, items, page lists
    KvDev kv;
    int64_t layer;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    float *part_o;                 // [partial rows][D]
    float *part_l;                 // [partial rows] log2 of the sum
    int64_t q_stride, out_stride;
    int32_t n_heads, max_tok;
    int32_t behind;                // whether the wide items' kernel is the one before
    int32_t tok_at, order_at, rec_at, pages_at;  // word offsets in plan
    float scale_log2;              // scale * log2(e)
    uint32_t *err;
};

__global__ void plan_copy_kernel(const uint4 *src, uint4 *dst, int n)
{
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) dst[i] = src[i];
}

// ---------------------------------------------------------------- shared memory
// The two kernels.  WIDE: up to 128 rows an item, their columns shared by two softmax
// warpgroups, one CTA an SM.  Narrow: few rows (single query tokens and drafts), bound by the
// latency of a tile's steps and by memory: one warpgroup, two CTAs an SM.
template <int D_, bool WIDE_>
struct Shape {
    static constexpr int D = D_;
    static constexpr bool WIDE = WIDE_;
    static constexpr int NWG = WIDE ? 2 : 1;              // softmax warpgroups
    static constexpr int R_MAX = WIDE ? 128 : D == 128 ? 16 : 32;  // rows an item
    static constexpr int CW_MAX = R_MAX / NWG;            // columns of a warpgroup
    static constexpr int CH = WIDE ? 16 : 4;              // columns a softmax thread has in hand at a time
    static constexpr int THREADS = 128 + NWG * WG;
    static constexpr int CTAS = WIDE ? 1 : 2;             // an SM
    // tensor memory columns: two buffers of R_MAX scores, the output
    static constexpr uint32_t TM_S = 0, TM_O = 2 * R_MAX, TM_COLS = WIDE ? 512 : D == 128 ? 64 : 128;
    // shared memory
    static constexpr int KST = WIDE ? (D == 128 ? 3 : 6) : (D == 128 ? 2 : 4);  // stages of K and of V
    static constexpr int VST = WIDE ? (D == 128 ? 2 : 4) : (D == 128 ? 2 : 4);
    static constexpr uint32_t SIDE = TT * D;              // codes of K or V of a tile
    static constexpr uint32_t K = 0;
    static constexpr uint32_t V = K + KST * SIDE;
    static constexpr uint32_t VH = V + VST * SIDE;        // V of a tile in f16
    static constexpr uint32_t P = VH + 2 * SIDE;          // P of a tile in f16
    static constexpr uint32_t Q_BUF = 2 * R_MAX * D;
    static constexpr uint32_t Q = P + TT * 2 * R_MAX;     // two items' queries
    static constexpr uint32_t EXPS = Q + 2 * Q_BUF;       // per stage of V: 128 of K, 128 of V
    // Two items' constants of the columns, arrays of R_MAX words: the factor a of a column's scores (query
    // row's power of two, scale, log2 e), its reference -m, the tokens it sees and (query token << 8 | head in
    // the group).
    static constexpr uint32_t INFO = EXPS + VST * 2 * TT;
    static constexpr uint32_t INFO_BUF = R_MAX * 16;
    static constexpr uint32_t IN_A = 0, IN_M = R_MAX * 4, IN_LIM = R_MAX * 8, IN_ROW = R_MAX * 12;
    static constexpr uint32_t FAC = INFO + 2 * INFO_BUF;
    static constexpr uint32_t PLACE = FAC + R_MAX * 4;    // where the rows go, 64 bits each
    static constexpr uint32_t WMAX = PLACE + R_MAX * 8;   // [NWG][4][CW_MAX] floats
    // barriers: K full, K free, V full, V free (a stage each), scores full [2], P full, product done, Q full [2], Q free
    // [2], item done [2], drain
    static constexpr uint32_t K_FULL = WMAX + 4 * R_MAX * 4;
    static constexpr uint32_t K_FREE = K_FULL + 8 * KST;
    static constexpr uint32_t V_FULL = K_FREE + 8 * KST;
    static constexpr uint32_t V_FREE = V_FULL + 8 * VST;
    static constexpr uint32_t S_FULL = V_FREE + 8 * VST;
    static constexpr uint32_t P_FULL = S_FULL + 16;
    static constexpr uint32_t PV_DONE = P_FULL + 8;
    static constexpr uint32_t Q_FULL = PV_DONE + 8;
    static constexpr uint32_t O_FREE = Q_FULL + 16;
    static constexpr uint32_t Q_FREE = O_FREE + 16;
    static constexpr uint32_t DRAIN = Q_FREE + 16;
    static constexpr uint32_t MISC = DRAIN + 8;           // TMEM address, failure flag, [2][2] largest value exponents, [2][2] first NaN values
    static constexpr uint32_t BYTES = MISC + 48 + 1024;   // slack for the 1024-byte alignment
    static_assert(BYTES + 1024 <= 228 * 1024 / CTAS, "shared memory of an SM");
    static_assert(TM_O + R_MAX <= TM_COLS, "tensor memory");
};
// Rows up to which an item is narrow, and at most.  (With the wide kernel for all of them, two requests of 200,000 tokens
// took 183 us where the narrow one took 159, and a step of 256 requests 527 and 503.)
constexpr int narrow_rows(int D) { return D == 128 ? Shape<128, false>::R_MAX : Shape<64, false>::R_MAX; }
constexpr int WIDE_ROWS = Shape<128, true>::R_MAX;

__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(x));
    return r;
}
// 2^k, 0 below the normal range (k <= 127)
__device__ __forceinline__ float pow2(int k) { return __uint_as_float(k < -126 ? 0u : (uint32_t)(k + 127) << 23); }
// 2^(e - 127) of an exponent byte; 0 for a row of zeros, NaN for a row that stands for NaN
__device__ __forceinline__ float row_scale(uint32_t e) { return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23); }

__device__ __forceinline__ void sts64(uint32_t a, uint32_t x, uint32_t y)
{
    asm volatile("st.shared.v2.b32 [%0], {%1, %2};\n" ::"r"(a), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w)
{
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

__device__ __forceinline__ float4 lds4f(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];\n" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float ldsf(uint32_t a)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];\n" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];\n" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void stsf(uint32_t a, float v) { asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(a), "f"(v) : "memory"); }
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;\n" ::"r"(a), "r"(v) : "memory"); }

// two floats at a time
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("{\n .reg .b64 a, b, c;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n fma.rn.f32x2 a, a, b, c;\n mov.b64 {%0, %1}, a;\n}\n"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 r;
    asm("{\n .reg .b64 a, b;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mul.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}\n"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

struct Item {
    int flags, tok, ntok, pages, t0, t1, lim, part, kh;
    int tiles, rows, per;  // per: rows a warpgroup takes
};

// The CTA's r-th item of n: the records are in falling order of cost, handed
// out forwards and backwards in turn.
__device__ __forceinline__ int item_index(int r) { return r * (int)gridDim.x + ((r & 1) ? (int)(gridDim.x - 1 - blockIdx.x) : (int)blockIdx.x); }

template <class L>
__device__ __forceinline__ Item load_item(const AttnParams &p, int idx, int G)
{
    const int rec = idx / p.kv.heads;
    // (the wide items' records come first)
    const int4 *w = reinterpret_cast<const int4 *>(p.plan + p.rec_at + ((L::WIDE ? 0 : __ldg(p.plan + HD_WIDE)) + rec) * REC_WORDS);
    const int4 a = __ldg(w), b = __ldg(w + 1);
    Item it;
    it.flags = a.x;
    it.tok = a.y;
    it.ntok = a.z;
    it.pages = a.w;
    it.t0 = b.x;
    it.t1 = b.y;
    it.lim = b.z;
    it.kh = idx - rec * p.kv.heads;
    it.rows = it.ntok * G;
    it.part = b.w + it.kh * it.rows;
    it.per = (it.rows + L::NWG - 1) / L::NWG;
    it.tiles = (it.t1 - it.t0 + TT - 1) / TT;
    return it;
}

// A bounded wait that also gives up when another role has.
__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, const volatile int *dead)
{
    for (int i = 0; i < (1 << 20); ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 255) == 255 && *dead) return false;
    }
    return false;
}

// Reduces each of N values over the warp's lanes (N a power of two up to
// 32) by halving: a lane ends up with that of value `col`, 32 / N lanes with
// the same one.
template <int N, class Op>
__device__ __forceinline__ float reduce_columns(float *t, int lane, int &col, Op op)
{
    col = 0;
    int n = N;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        if (n > 1) {
            n >>= 1;
            const bool up = lane & o;
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                if (i < n) {
                    const float send = up ? t[i] : t[i + n];
                    t[i] = op(up ? t[i + n] : t[i], __shfl_xor_sync(0xffffffffu, send, o));
                }
            }
            if (up) col += n;
        } else {
            t[0] = op(t[0], __shfl_xor_sync(0xffffffffu, t[0], o));
        }
    }
    return t[0];
}

// What the softmax warpgroups share across their functions.
struct Soft {
    uint32_t base, tmem;
    volatile int *dead;
    int wg, tid, lane, quarter;
    uint32_t g;                    // tiles done by this CTA
    uint32_t stage, stage_phase;
    bool ok;
};

// A wait of a softmax warp: all of its lanes get the same answer.
__device__ __forceinline__ void soft_wait(Soft &s, uint32_t bar, uint32_t parity)
{
    bool r = s.ok;
    if (r) r = wait_bar(bar, parity, s.dead);
    s.ok = __all_sync(0xffffffffu, r);
}

// Addresses and constants of an item for a softmax warpgroup.
struct SoftItem {
    uint32_t info, fac, place, wmax;  // shared memory: constants of the warpgroup's columns (IN_*), scratch
    uint32_t p_row, p_mix;            // this token's row of P; a piece's place in it is XORed with p_mix (the swizzle)
    uint32_t s_at, o_at;              // tensor memory: the first buffer of the scores, the output
    int ncol, vtop, nb, j;
};

// CH columns of tensor memory, this warp's lanes
template <int CH>
__device__ __forceinline__ void load_columns(float (&x)[CH], uint32_t at)
{
    uint32_t *r = reinterpret_cast<uint32_t *>(x);
    static_assert(CH == 4 || CH == 16, "the columns a softmax thread has in hand");
    if constexpr (CH == 4) tmem_ld4(at, r);
    else tmem_ld16(at, *reinterpret_cast<uint32_t(*)[16]>(r));
}

// A token's part of a tile: factors of its scores and of its probabilities, and what
// P is to p in log2, held so that p stays in range (a value 2^100 below the
// largest may lose bits).
struct Token {
    int at;
    float kf, vf, vref;
    bool mask;                        // some row does not see the whole tile
};

// The warpgroups' share of a tile's values in f16; zeros for rows that stand
// for NaN and from row `valid` on (past the range a stage holds other tokens'
// values, or none): 0 * NaN must not arise.
template <class L>
__device__ __forceinline__ void widen_values(const Soft &s, int valid)
{
    constexpr int CPR = L::D / 16;                 // 16-byte pieces of a row's codes
    constexpr int ROWS = L::NWG * WG / CPR;        // rows a pass; a multiple of 8, so a thread's swizzle stays
    // Eight threads in a row deal with halves of rows r and r ^ 5: their pieces lie in different banks both where
    // they are read and (twice as wide, every other piece) where they are written.
    const int me = s.wg * WG + s.tid;
    const int pair = (me >> 3) & 3, up = (me >> 2) & 1, rest = me >> 5;
    const int ch = (me & 3) + 4 * (CPR == 8 ? rest & 1 : 0), row0 = 8 * (CPR == 8 ? rest >> 1 : rest) + (up ? pair ^ 5 : pair);
    const uint32_t from = s.base + L::V + s.stage * L::SIDE + swz_rows<L::D>(row0 * L::D + ch * 16);
    const uint32_t exps = s.base + L::EXPS + s.stage * 2 * TT + TT + row0;
    const uint32_t to = s.base + L::VH + (ch / 4) * (TT * 128);
    const uint32_t to0 = to + swz_rows<128>(row0 * 128 + (ch % 4) * 32), to1 = to + swz_rows<128>(row0 * 128 + (ch % 4) * 32 + 16);
    uint4 c[TT / ROWS];
    uint32_t ve[TT / ROWS];
#pragma unroll
    for (int k = 0; k < TT / ROWS; ++k) {
        c[k] = lds128(from + k * ROWS * L::D);
        ve[k] = lds8(exps + k * ROWS);
    }
#pragma unroll
    for (int k = 0; k < TT / ROWS; ++k) {
        const uint32_t x[4] = {c[k].x, c[k].y, c[k].z, c[k].w};
        const uint32_t keep = row0 + k * ROWS < valid && ve[k] != 255u ? 0xffffffffu : 0u;
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[2 * i] = f16x2_of_e4m3x2((uint16_t)(x[i] & keep));
            h[2 * i + 1] = f16x2_of_e4m3x2((uint16_t)((x[i] & keep) >> 16));
        }
        sts128(to0 + k * ROWS * 128, h[0], h[1], h[2], h[3]);
        sts128(to1 + k * ROWS * 128, h[4], h[5], h[6], h[7]);
    }
}

// P of a tile and the warpgroup's share of its widened values into shared
// memory, the probabilities times `add` to the sums l.  Returns the largest log2 P
// of the token.  Columns go by sixteens, where rows are few by fours (the last ones are filled up; fetching the next ones'
// scores ahead took 3% longer, in registers; sixteens for four rows took 10% longer).  (One copy of this code for every number of
// rows: with one for each, and one for masked tiles, the kernel had 223 KB of code and
// an item's first tile waited 6,000 cycles for instructions.)
template <class L>
__device__ __forceinline__ float soft_probs(Soft &s, const SoftItem &w, float2 (&l)[L::CW_MAX / 2], const Token &t, uint32_t s_at,
                                            float add, int valid)
{
    constexpr int CH = L::CH;
    const float2 kf2 = make_float2(t.kf, t.kf), vf2 = make_float2(t.vf, t.vf), add1 = make_float2(add, add);
    float mx = -INFINITY;
#pragma unroll
    for (int c0 = 0; c0 < L::CW_MAX; c0 += CH) {
        if (c0 >= w.ncol) break;
        float y[CH];
        load_columns<CH>(y, s_at + c0);
        tmem_ld_wait();
        const uint32_t at = w.info + 4 * c0;
#pragma unroll
        for (int i = 0; i < CH; i += 4) {
            const float4 a = lds4f(at + L::IN_A + 4 * i), m = lds4f(at + L::IN_M + 4 * i);
            const float2 u = fma2(make_float2(y[i], y[i + 1]), mul2(make_float2(a.x, a.y), kf2), make_float2(m.x, m.y));
            const float2 v = fma2(make_float2(y[i + 2], y[i + 3]), mul2(make_float2(a.z, a.w), kf2), make_float2(m.z, m.w));
            y[i] = u.x;
            y[i + 1] = u.y;
            y[i + 2] = v.x;
            y[i + 3] = v.y;
        }
        if (t.mask) {
#pragma unroll
            for (int i = 0; i < CH; i += 4) {
                const uint4 n = lds128(at + L::IN_LIM + 4 * i);
                if (t.at >= (int)n.x) y[i] = -INFINITY;
                if (t.at >= (int)n.y) y[i + 1] = -INFINITY;
                if (t.at >= (int)n.z) y[i + 2] = -INFINITY;
                if (t.at >= (int)n.w) y[i + 3] = -INFINITY;
            }
        }
        uint32_t h[CH / 2];
#pragma unroll
        for (int i = 0; i < CH; i += 2) {
            mx = fmaxf(mx, fmaxf(y[i], y[i + 1]));
            const float2 e = make_float2(ex2(y[i]), ex2(y[i + 1])), v = mul2(e, vf2);
            l[(c0 + i) / 2] = fma2(e, add1, l[(c0 + i) / 2]);
            const __half2 q = __floats2half2_rn(v.x, v.y);
            h[i / 2] = *reinterpret_cast<const uint32_t *>(&q);
        }
        // P and the values take the place of the last tile's once its product is done
        if (c0 == 0 && s.g > 0) soft_wait(s, s.base + L::PV_DONE, (s.g - 1) & 1);
        if constexpr (CH == 4) sts64(w.p_row + (w.p_mix ^ (2 * c0)), h[0], h[1]);
#pragma unroll
        for (int i = 0; i + 4 <= CH / 2; i += 4) sts128(w.p_row + (w.p_mix ^ (2 * c0 + 4 * i)), h[i], h[i + 1], h[i + 2], h[i + 3]);
    }
    if (w.ncol == 0 && s.g > 0) soft_wait(s, s.base + L::PV_DONE, (s.g - 1) & 1);
    widen_values<L>(s, valid);
    return mx + t.vref;
}

// soft_probs where every column of the warpgroup is a row and every row sees every token: no
// branches, and each sixteen columns' exponentials run beside the next ones' loads and products.
// (16 exponentials of each of an SM quarter's two warps take 128 cycles; behind one another with the
// loads, a tile of 128 rows took 2,100 cycles here.)
template <class L>
__device__ __forceinline__ float soft_probs_full(Soft &s, const SoftItem &w, float2 (&l)[L::CW_MAX / 2], const Token &t, uint32_t s_at,
                                                 float add, int valid)
{
    constexpr int CH = L::CH, N = L::CW_MAX / CH;
    const float2 kf2 = make_float2(t.kf, t.kf), vf2 = make_float2(t.vf, t.vf), add1 = make_float2(add, add);
    float mx = -INFINITY;
    float x[2][CH];
    float4 a[CH / 4], m[CH / 4];
    auto fetch = [&](int c) {
        load_columns<CH>(x[c & 1], s_at + c * CH);
#pragma unroll
        for (int i = 0; i < CH / 4; ++i) {
            a[i] = lds4f(w.info + 4 * c * CH + L::IN_A + 16 * i);
            m[i] = lds4f(w.info + 4 * c * CH + L::IN_M + 16 * i);
        }
    };
    auto args = [&](int c) {
        float (&y)[CH] = x[c & 1];
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < CH; i += 4) {
            const float2 u = fma2(make_float2(y[i], y[i + 1]), mul2(make_float2(a[i / 4].x, a[i / 4].y), kf2), make_float2(m[i / 4].x, m[i / 4].y));
            const float2 v = fma2(make_float2(y[i + 2], y[i + 3]), mul2(make_float2(a[i / 4].z, a[i / 4].w), kf2), make_float2(m[i / 4].z, m[i / 4].w));
            y[i] = u.x;
            y[i + 1] = u.y;
            y[i + 2] = v.x;
            y[i + 3] = v.y;
        }
    };
    fetch(0);
    args(0);
#pragma unroll
    for (int c = 0; c < N; ++c) {
        float (&y)[CH] = x[c & 1];
        if (c + 1 < N) fetch(c + 1);
        uint32_t h[CH / 2];
#pragma unroll
        for (int i = 0; i < CH; i += 2) {
            mx = fmaxf(mx, fmaxf(y[i], y[i + 1]));
            const float2 e = make_float2(ex2(y[i]), ex2(y[i + 1])), v = mul2(e, vf2);
            l[(c * CH + i) / 2] = fma2(e, add1, l[(c * CH + i) / 2]);
            const __half2 q = __floats2half2_rn(v.x, v.y);
            h[i / 2] = *reinterpret_cast<const uint32_t *>(&q);
        }
        if (c + 1 < N) args(c + 1);
        // P and the values take the place of the last tile's once its product is done
        if (c == 0 && s.g > 0) soft_wait(s, s.base + L::PV_DONE, (s.g - 1) & 1);
        sts128(w.p_row + (w.p_mix ^ (2 * c * CH)), h[0], h[1], h[2], h[3]);
        sts128(w.p_row + (w.p_mix ^ (2 * c * CH + 16)), h[4], h[5], h[6], h[7]);
    }
    widen_values<L>(s, valid);
    return mx + t.vref;
}

// Takes a tile's probabilities out of the sums of a thread that has very large ones.  What an infinite sum held before
// was nothing next to what made it so (a NaN stays).  The whole warp; by way of local memory, as this hardly ever runs and the
// sums' registers are better left alone.
template <class L>
__device__ __forceinline__ void take_out(const SoftItem &w, float2 (&l)[L::CW_MAX / 2], const Token &t, uint32_t s_at, bool mine)
{
    float sums[L::CW_MAX];
#pragma unroll
    for (int c = 0; c < L::CW_MAX; ++c) sums[c] = c & 1 ? l[c / 2].y : l[c / 2].x;
#pragma unroll 1
    for (int c0 = 0; c0 < w.ncol; c0 += 4) {
        float y[4];
        load_columns<4>(y, s_at + c0);
        tmem_ld_wait();
#pragma unroll 1
        for (int c = c0; c < min(c0 + 4, w.ncol); ++c) {
            const uint32_t at = w.info + 4 * c;
            const float x = fmaf(y[0], ldsf(at + L::IN_A) * t.kf, ldsf(at + L::IN_M));
            y[0] = y[1], y[1] = y[2], y[2] = y[3];
            if (mine && t.at < (int)lds32(at + L::IN_LIM)) sums[c] = sums[c] == INFINITY ? 0.f : sums[c] - ex2(x);
        }
    }
#pragma unroll
    for (int c = 0; c < L::CW_MAX; ++c) (c & 1 ? l[c / 2].y : l[c / 2].x) = sums[c];
}

// Moves the references that a score of this tile passes by too much (all of
// them where there is none yet), and with them what the output and the
// sums of earlier tiles hold.  The whole warpgroup; needs the product before this
// tile's to be done.
template <class L>
__device__ __forceinline__ void move_refs(const Soft &s, const SoftItem &w, float2 (&l)[L::CW_MAX / 2], const Token &t, uint32_t s_at)
{
    constexpr int CH = L::CH;
#pragma unroll 1
    for (int c0 = 0; c0 < w.ncol; c0 += CH) {
        float x[CH];
        load_columns<CH>(x, s_at + c0);
        tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < CH; c += 4) {
            const float4 a = lds4f(w.info + L::IN_A + 4 * (c0 + c));
            const uint4 n = lds128(w.info + L::IN_LIM + 4 * (c0 + c));
            const float k[4] = {a.x, a.y, a.z, a.w};
            const int lim[4] = {(int)n.x, (int)n.y, (int)n.z, (int)n.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[c + i] = fmaf(x[c + i], t.kf * k[i], t.vref);
                if (t.at >= lim[i] || !(x[c + i] == x[c + i])) x[c + i] = -INFINITY;
            }
        }
        int col;
        const float v = reduce_columns<CH>(x, s.lane, col, [](float p, float q) { return fmaxf(p, q); });
        stsf(w.wmax + 4 * (s.quarter * L::CW_MAX + c0 + col), v);
    }
    named_sync(w.nb, WG);
    if (s.tid < L::CW_MAX) {
        float v = ldsf(w.wmax + 4 * s.tid);
        for (int q = 1; q < 4; ++q) v = fmaxf(v, ldsf(w.wmax + 4 * (q * L::CW_MAX + s.tid)));
        bool move = false;
        float m = 0.f;
        if (s.tid < w.ncol) {
            m = -ldsf(w.info + L::IN_M + 4 * s.tid);
            move = v - m > P_MOST;
        }
        stsf(w.fac + 4 * s.tid, move ? ex2(0.5f * (m - (v - P_TOP))) : 1.f);  // (applied twice: 2^-160 is no float)
        if (move) stsf(w.info + L::IN_M + 4 * s.tid, P_TOP - v);
    }
    named_sync(w.nb, WG);
    if (w.j > 0) {
#pragma unroll 1
        for (int c0 = 0; c0 < w.ncol; c0 += 8) {
            float o[8];
            tmem_ld8(w.o_at + c0, reinterpret_cast<uint32_t *>(o));
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const float f = ldsf(w.fac + 4 * (c0 + c));
                o[c] = o[c] * f * f;
            }
            tmem_st8(w.o_at + c0, reinterpret_cast<const uint32_t *>(o));
        }
        tmem_st_wait();
#pragma unroll
        for (int c = 0; c < L::CW_MAX; c += 4) {
            const float4 f = lds4f(w.fac + 4 * c);
            l[c / 2] = mul2(mul2(l[c / 2], make_float2(f.x, f.y)), make_float2(f.x, f.y));
            l[c / 2 + 1] = mul2(mul2(l[c / 2 + 1], make_float2(f.z, f.w)), make_float2(f.z, f.w));
        }
    }
}

// A tile of an item.  False: gave up (the whole warpgroup together).
template <class L>
__device__ __forceinline__ bool soft_tile(Soft &s, const SoftItem &w, float2 (&l)[L::CW_MAX / 2], const Token &t, int valid)
{
    const uint32_t s_at = w.s_at + (s.g & 1) * L::R_MAX;
    // References are set before an item's first tile; where a later one passes
    // them by too much they are moved and the tile's P made anew.  Its probabilities are in the sums already and
    // are scaled with them, but for those of a thread whose sums may have left fp32's range.  Then P fits: scores
    // up to 2^23 are rounded by 1 at most.  (A way for larger ones took 9% more time on prompt chunks.)
    float add = 1.f;
#pragma unroll 1
    for (bool again = false;; again = true) {
        if (again && __any_sync(0xffffffffu, add != 0.f)) take_out<L>(w, l, t, s_at, add != 0.f);
        if ((again || w.j == 0) && w.ncol > 0) move_refs<L>(s, w, l, t, s_at);
        const float mx = L::WIDE && w.ncol == L::CW_MAX && !t.mask ? soft_probs_full<L>(s, w, l, t, s_at, add, valid)
                                                                   : soft_probs<L>(s, w, l, t, s_at, add, valid);
        if (named_sync_and(w.nb, WG, s.ok && !(mx > P_MOST && !again && w.j > 0))) return true;
        if (again || !named_sync_and(w.nb, WG, s.ok)) return false;
        add = mx - t.vref >= P_HOT ? 1.f : 0.f;
        tc_fence_after();
    }
}

// One item.  False: gave up (the whole warpgroup together).
template <class L>
__device__ __forceinline__ bool soft_item(const AttnParams &p, Soft &s, const Item &it, int n_item)
{
    constexpr int CH = L::CH;
    const int cw = 16 << (it.flags & 3), pitch = min(2 * L::NWG * cw, 128), at = s.wg * 2 * cw;  // columns a warpgroup; bytes of P
    const uint32_t lanes = (uint32_t)(s.quarter * 32) << 16;
    SoftItem w;
    w.info = s.base + L::INFO + (n_item & 1) * L::INFO_BUF + s.wg * cw * 4;
    w.fac = s.base + L::FAC + s.wg * L::CW_MAX * 4;
    w.place = s.base + L::PLACE + s.wg * L::CW_MAX * 8;
    w.wmax = s.base + L::WMAX + s.wg * 4 * L::CW_MAX * 4;
    w.p_row = s.base + L::P + at / 128 * (TT * 128) + s.tid * pitch;
    w.p_mix = at % 128 ^ (((uint32_t)(s.tid * pitch) >> 7 & (pitch / 16 - 1)) << 4);
    w.s_at = s.tmem + lanes + L::TM_S + s.wg * cw;
    w.o_at = s.tmem + lanes + L::TM_O + s.wg * cw;
    w.ncol = min(max(it.rows - s.wg * it.per, 0), it.per);
    w.nb = 1 + s.wg;
    // values count in units of the largest exponent of the range
    w.vtop = max((int)lds32(s.base + L::MISC + 8 + 8 * (n_item & 1)), (int)lds32(s.base + L::MISC + 12 + 8 * (n_item & 1)));
    if (w.vtop == 0) w.vtop = 127;
    float2 l[L::CW_MAX / 2];
#pragma unroll
    for (int c = 0; c < L::CW_MAX / 2; ++c) l[c] = make_float2(0.f, 0.f);
#pragma unroll 1
    for (w.j = 0; w.j < it.tiles; ++w.j) {
        const int end = it.t0 + (w.j + 1) * TT;
        soft_wait(s, s.base + L::V_FULL + 8 * s.stage, s.stage_phase);
        soft_wait(s, s.base + L::S_FULL + 8 * (s.g & 1), (s.g >> 1) & 1);
        tc_fence_after();
        const uint32_t ex = s.base + L::EXPS + s.stage * 2 * TT + s.tid;
        const uint32_t ke = lds8(ex), ve = lds8(ex + TT);
        Token t;
        t.at = end - TT + s.tid;
        t.kf = row_scale(ke);
        // (a value that stands for NaN adds nothing; the rows that see it are known at the end)
        t.vf = t.at >= it.t1 || ve == 255u ? 0.f : pow2((int)ve - w.vtop + P_UP);
        t.vref = (float)(P_UP + (ve == 255u ? -P_LOW : max((int)ve - w.vtop, -P_LOW)));
        t.mask = end > min(it.t1, it.lim);  // (the first query token sees least)
        if (!soft_tile<L>(s, w, l, t, it.t1 - (end - TT))) return false;
        tc_fence_before();
        fence_async_smem();
        __syncwarp();
        if (s.lane == 0) {
            mbar_arrive_release(s.base + L::P_FULL);
            mbar_arrive_release(s.base + L::V_FREE + 8 * s.stage);
        }
        ++s.g;
        if (++s.stage == L::VST) {
            s.stage = 0;
            s.stage_phase ^= 1;
        }
    }
    // ------------------------------------------------ the item's rows
#pragma unroll
    for (int c0 = 0; c0 < L::CW_MAX; c0 += CH) {
        if (c0 >= w.ncol) break;
        int col;
        float v[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = c & 1 ? l[(c0 + c) / 2].y : l[(c0 + c) / 2].x;
        const float t = reduce_columns<CH>(v, s.lane, col, [](float p, float q) { return p + q; });
        stsf(w.wmax + 4 * (s.quarter * L::CW_MAX + c0 + col), t);
    }
    if (!named_sync_and(w.nb, WG, s.ok)) return false;
    const int G = p.n_heads / p.kv.heads;
    const bool direct = it.flags & RF_DIRECT;
    if (s.tid < w.ncol) {
        const uint32_t at_w = w.wmax + 4 * s.tid, at_i = w.info + 4 * s.tid;
        const float t = (ldsf(at_w) + ldsf(at_w + 4 * L::CW_MAX)) + (ldsf(at_w + 8 * L::CW_MAX) + ldsf(at_w + 12 * L::CW_MAX));
        const int row = (int)lds32(at_i + L::IN_ROW);
        const float lse2 = t > 0.f ? log2f(t) - ldsf(at_i + L::IN_M) : t == t ? -INFINITY : t;
        int64_t to;  // the row's first element
        if (direct) {
            to = (row >> 8) * p.out_stride + (it.kh * G + (row & 255)) * L::D;
            if (p.lse) p.lse[(int64_t)(row >> 8) * p.n_heads + it.kh * G + (row & 255)] = lse2 * 0.693147180559945f;
        } else {
            const int part = it.part + s.wg * it.per + s.tid;
            to = (int64_t)part * L::D;
            p.part_l[part] = lse2;
        }
        // a row that sees a value that stands for NaN is NaN, but for its log-sum
        const int first_nan = min((int)lds32(s.base + L::MISC + 24 + 8 * (n_item & 1)), (int)lds32(s.base + L::MISC + 28 + 8 * (n_item & 1)));
        const bool spoiled = (int)lds32(at_i + L::IN_LIM) > first_nan;
        stsf(w.fac + 4 * s.tid, spoiled ? __uint_as_float(0x7fc00000u) : t > 0.f ? 1.f / t : t == t ? 0.f : t);
        sts64(w.place + 8 * s.tid, (uint32_t)to, (uint32_t)(to >> 32));
    }
    soft_wait(s, s.base + L::PV_DONE, (s.g - 1) & 1);
    tc_fence_after();
    if (!named_sync_and(w.nb, WG, s.ok)) return false;
    const int dim = L::D == 128 ? s.tid : s.quarter * 16 + s.lane;   // M = 64 uses 16 lanes of each quarter
    const bool live = L::D == 128 || s.lane < 16;
    // 2^(vtop - 127 - P_UP) in two factors
    const int e_unit = w.vtop - 127 - P_UP;
    const float unit = pow2(max(e_unit, -126)), rest = pow2(min(e_unit + 126, 0));
#pragma unroll 1
    for (int c0 = 0; c0 < w.ncol; c0 += CH) {
        float o[CH];
        load_columns<CH>(o, w.o_at + c0);
        tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < CH; c += 4) {
            const float4 f = lds4f(w.fac + 4 * (c0 + c));
            const uint4 p0 = lds128(w.place + 8 * (c0 + c)), p1 = lds128(w.place + 8 * (c0 + c) + 16);
            const float k[4] = {f.x, f.y, f.z, f.w};
            const uint32_t lo[4] = {p0.x, p0.z, p1.x, p1.z}, hi[4] = {p0.y, p0.w, p1.y, p1.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t to = (int64_t)((uint64_t)hi[i] << 32 | lo[i]) + dim;
                const float v = o[c + i] * k[i] * unit * rest;
                if (c0 + c + i < w.ncol && live) {
                    if (direct) p.out[to] = f_to_bf16(v);
                    else p.part_o[to] = v;
                }
            }
        }
    }
    tc_fence_before();
    __syncwarp();
    if (s.lane == 0) mbar_arrive_release(s.base + L::O_FREE + 8 * (n_item & 1));
    return true;
}

// An item's queries: rows scaled by a power of two and split in hi + lo, the
// constants of its columns, the largest exponent of its values and the first of them that stands for NaN.  W warps, this
// one the w-th.
template <class L>
__device__ __forceinline__ void stage_queries(const AttnParams &p, uint32_t base, const Item &it, int n_item, int w, int W)
{
    const int KV = p.kv.heads, G = p.n_heads / KV, lane = threadIdx.x & 31;
    const int cw = 16 << (it.flags & 3), R = L::NWG * cw;
    const int g_inv = (65535 + G) / G, per_inv = (65535 + it.per) / it.per;  // quotients by products: rows are below 129, divisors at most 64
    const int32_t *order = p.plan + p.order_at + it.tok;
    const uint32_t info = base + L::INFO + (n_item & 1) * L::INFO_BUF, q_at = base + L::Q + (n_item & 1) * L::Q_BUF;
    auto set_column = [&](int col, float a, float nm, int lim, int row) {
        stsf(info + L::IN_A + 4 * col, a);
        stsf(info + L::IN_M + 4 * col, nm);
        sts32(info + L::IN_LIM + 4 * col, (uint32_t)lim);
        sts32(info + L::IN_ROW + 4 * col, (uint32_t)row);
    };
    // exponents of 16 values a lane (their pages' numbers are on their way while the queries are)
    const int t_first = it.t0 + (w * 32 + lane) * 16, t_step = W * 32 * 16;
    const int32_t *pages = p.plan + p.pages_at + it.pages;
    int page = t_first < it.t1 ? __ldg(pages + (t_first >> p.kv.page_log2)) : 0;
    constexpr int LPR = L::D / 8;           // lanes a row, eight elements each
    constexpr int RPW = 32 / LPR;        // rows a warp deals with at a time
    constexpr int AT_ONCE = L::WIDE ? 4 : 2;  // loads of a lane under way together
    const int part = lane % LPR;
    for (int row0 = w * RPW + lane / LPR; row0 < it.rows + lane / LPR; row0 += W * RPW * AT_ONCE) {
        uint4 u[AT_ONCE];
        int id[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int row = row0 + W * RPW * k, i = row * g_inv >> 16;
            id[k] = 0;
            if (row < it.rows) id[k] = (((it.flags & RF_CAUSAL) ? it.tok + i : __ldg(order + i)) << 8) | (row - i * G);
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            u[k] = make_uint4(0, 0, 0, 0);
            if (row0 + W * RPW * k < it.rows)
                u[k] = __ldg(reinterpret_cast<const uint4 *>(p.q + (id[k] >> 8) * p.q_stride + (it.kh * G + (id[k] & 255)) * L::D + part * 8));
        }
        uint32_t a[AT_ONCE], hi[AT_ONCE][2], lo[AT_ONCE][2];
        int qe[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const uint32_t x[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
            a[k] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) a[k] = max(a[k], max((x[e] << 16) & 0x7fffffffu, x[e] & 0x7fff0000u));
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) a[k] = max(a[k], __shfl_xor_sync(0xffffffffu, a[k], o));
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            // the row's largest element to [2^7, 2^8)
            const uint32_t x[4] = {u[k].x, u[k].y, u[k].z, u[k].w};
            qe[k] = max((int)(a[k] >> 23) - 127 - 7, -120);
            const float inv = pow2(-qe[k]);
            hi[k][0] = hi[k][1] = lo[k][0] = lo[k][1] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v0 = __uint_as_float(x[e] << 16) * inv, v1 = __uint_as_float(x[e] & 0xffff0000u) * inv;
                const uint16_t h = e4m3x2(v0, v1);
                const uint32_t back = f16x2_of_e4m3x2(h);
                const float2 hf = __half22float2(*reinterpret_cast<const __half2 *>(&back));
                hi[k][e / 2] |= (uint32_t)h << (16 * (e & 1));
                lo[k][e / 2] |= (uint32_t)e4m3x2(v0 - hf.x, v1 - hf.y) << (16 * (e & 1));
            }
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int row = row0 + W * RPW * k;
            if (row < it.rows) {
                const bool bad = (a[k] >> 23) == 255;
                if (bad) hi[k][0] = hi[k][1] = lo[k][0] = lo[k][1] = 0x7f7f7f7fu;
                const int wg = row * per_inv >> 16, col = wg * cw + row - wg * it.per;
                sts64(q_at + swz_rows<L::D>(col * L::D + part * 8), hi[k][0], hi[k][1]);
                sts64(q_at + swz_rows<L::D>((R + col) * L::D + part * 8), lo[k][0], lo[k][1]);
                if (part == 0)
                    set_column(col, bad ? 1.f : pow2(qe[k]) * p.scale_log2, -M_NONE,
                               it.lim + ((it.flags & RF_CAUSAL) ? (row * g_inv >> 16) : 0), id[k]);
            }
        }
    }
    // columns that fill up a warpgroup's last CH take part, unused; they see nothing
    for (int g = w; g < L::NWG; g += W) {
        const int ncol = min(max(it.rows - g * it.per, 0), it.per);
        if (ncol + lane < ((ncol + L::CH - 1) & ~(L::CH - 1))) set_column(g * cw + ncol + lane, 0.f, -INFINITY, 0, 0);
    }
    // the largest exponent of the range's values, the first one that stands for NaN
    uint32_t top = 0;
    int first_nan = NEVER;
    for (int t = t_first; t < it.t1; t += t_step) {
        const int64_t at = (((p.layer * p.kv.n_pages + page) * KV + it.kh) << p.kv.page_log2) + (t & (p.kv.page - 1));
        const uint4 e = __ldg(reinterpret_cast<const uint4 *>(p.kv.v_exp + at));
        if (t + t_step < it.t1) page = __ldg(pages + ((t + t_step) >> p.kv.page_log2));
        const uint32_t x[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = min(max(it.t1 - t - 4 * i, 0), 4);  // bytes of tokens in the range
            const uint32_t in = n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1u;
            const uint32_t nan = __vcmpeq4(x[i], 0xffffffffu) & in;
            top = __vmaxu4(top, x[i] & in & ~nan);
            if (nan) first_nan = min(first_nan, t + 4 * i + (__ffs(nan) - 1) / 8);
        }
    }
    top = max(max(top & 255u, (top >> 8) & 255u), max((top >> 16) & 255u, top >> 24));
    top = __reduce_max_sync(0xffffffffu, top);
    first_nan = __reduce_min_sync(0xffffffffu, first_nan);
    const uint32_t slot = base + L::MISC + 8 + 8 * (n_item & 1) + 4 * (w & 1);
    if (lane == 0) {
        if (n_item == 0) {
            asm volatile("red.shared.max.u32 [%0], %1;\n" ::"r"(slot), "r"(top) : "memory");
            asm volatile("red.shared.min.s32 [%0], %1;\n" ::"r"(slot + 16), "r"(first_nan) : "memory");
        } else {  // (two warps)
            sts32(slot, top);
            sts32(slot + 16, (uint32_t)first_nan);
        }
    }
    fence_async_smem();
}

template <class L>
__global__ void __launch_bounds__(L::THREADS, L::CTAS) attn_tile_kernel(const __grid_constant__ AttnParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(sm);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int KV = p.kv.heads, G = p.n_heads / KV;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(sm + L::MISC);
    volatile int *dead = reinterpret_cast<volatile int *>(sm + L::MISC + 4);
    if (tid == 0) {
        for (int i = 0; i < L::KST; ++i) {
            mbar_init(base + L::K_FULL + 8 * i, 1);
            mbar_init(base + L::K_FREE + 8 * i, 1);
        }
        for (int i = 0; i < L::VST; ++i) {
            mbar_init(base + L::V_FULL + 8 * i, 1);
            mbar_init(base + L::V_FREE + 8 * i, L::NWG * WG / 32);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(base + L::S_FULL + 8 * i, 1);
            mbar_init(base + L::Q_FULL + 8 * i, 2);
            mbar_init(base + L::Q_FREE + 8 * i, 1);
            mbar_init(base + L::O_FREE + 8 * i, L::NWG * WG / 32);
        }
        mbar_init(base + L::P_FULL, L::NWG * WG / 32);
        mbar_init(base + L::PV_DONE, 1);
        mbar_init(base + L::DRAIN, 1);
        *dead = 0;
        sts64(base + L::MISC + 8, 0, 0);
        sts64(base + L::MISC + 24, NEVER, NEVER);
        mbar_fence_init();
    }
    if (warp == 1) {
        tmem_alloc(base + L::MISC, L::TM_COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // A run's first kernel gets this far beside the end of what came before it in the stream; the narrow
    // items' behind the wide ones' needs nothing of that one, which itself lets it begin after its own wait.
    if (!p.behind) pdl_wait();
    pdl_launch_dependents();  // (the combine waits)
    const int32_t *plan = after_pdl_wait(p.plan);
    const bool fits = plan[HD_TOKENS] <= p.max_tok;
    if (!fits && blockIdx.x == 0 && tid == 0) atomicOr(p.err, SALT_DEVERR_BATCH);
    const int n_items = fits ? plan[L::WIDE ? HD_WIDE : HD_NARROW] * KV : 0;
    if ((int)blockIdx.x >= n_items) {
        if (warp == 1) tmem_dealloc(tmem, L::TM_COLS);
        if (!L::WIDE) pdl_wait();
        return;
    }
    bool ok = true;
    if (warp > 0) {
        // ------------------------------------------------ queries: the first item's by every warp but the one that starts its
        // loads, the later ones' by warps 2 and 3 alongside the items before them
        constexpr int OTHERS = L::THREADS - 32;
        const bool stays = warp == 2 || warp == 3;
        for (int r = 0; ok; ++r) {
            const int idx = item_index(r);
            if (idx >= n_items) break;
            if (r > 1) {
                ok = wait_bar(base + L::Q_FREE + 8 * (r & 1), ((r - 2) >> 1) & 1, dead) &&
                     wait_bar(base + L::O_FREE + 8 * (r & 1), ((r - 2) >> 1) & 1, dead);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
            }
            stage_queries<L>(p, base, load_item<L>(p, idx, G), r, r == 0 ? warp - 1 : warp - 2, r == 0 ? OTHERS / 32 : 2);
            if (r == 0) {
                named_sync(1 + L::NWG, OTHERS);
                if (!stays) break;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_release(base + L::Q_FULL + 8 * (r & 1));
        }
        if (!ok && lane == 0) {
            *dead = 1;
            atomicOr(p.err, SALT_DEVERR_TIMEOUT);
        }
    }

    if (warp == 0) {
        // ------------------------------------------------ loads: a lane per page of a tile
        uint32_t ks = 0, kph = 0, vs = 0, vph = 0, k_used = 0, v_used = 0;
        for (int r = 0; ok; ++r) {
            const int idx = item_index(r);
            if (idx >= n_items) break;
            const Item it = load_item<L>(p, idx, G);
            const int32_t *list = p.plan + p.pages_at + it.pages;
            const int per = TT >> p.kv.page_log2;
            for (int j = 0; j < it.tiles && ok; ++j) {
                const int t = it.t0 + j * TT;
                const int first = t >> p.kv.page_log2;
                const int n = min(per, ((it.t1 - 1) >> p.kv.page_log2) - first + 1);
                int page = 0;
                if (lane < n) page = __ldg(list + first + lane);
                const uint32_t bytes = (uint32_t)n * p.kv.page;
                const int64_t row = ((p.layer * p.kv.n_pages + page) * KV + it.kh) << p.kv.page_log2;
                const uint32_t at = lane * p.kv.page * L::D;
                const uint32_t k_full = base + L::K_FULL + 8 * ks, v_full = base + L::V_FULL + 8 * vs;
                if (k_used >= (uint32_t)L::KST) ok = wait_bar(base + L::K_FREE + 8 * ks, kph ^ 1, dead);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) mbar_expect_tx(k_full, bytes * L::D);
                __syncwarp();
                if (lane < n) tma_load_2d(base + L::K + ks * L::SIDE + at, &p.kmap, 0, (int)row, k_full);
                ++k_used;
                if (++ks == (uint32_t)L::KST) {
                    ks = 0;
                    kph ^= 1;
                }
                if (v_used >= (uint32_t)L::VST) ok = wait_bar(base + L::V_FREE + 8 * vs, vph ^ 1, dead);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (lane == 0) mbar_expect_tx(v_full, bytes * (L::D + 2));
                __syncwarp();
                if (lane < n) {
                    const uint32_t ex = base + L::EXPS + vs * 2 * TT + lane * p.kv.page;
                    tma_load_2d(base + L::V + vs * L::SIDE + at, &p.vmap, 0, (int)row, v_full);
                    bulk_load(ex, p.kv.k_exp + row, p.kv.page, v_full);
                    bulk_load(ex + TT, p.kv.v_exp + row, p.kv.page, v_full);
                }
                ++v_used;
                if (++vs == (uint32_t)L::VST) {
                    vs = 0;
                    vph ^= 1;
                }
            }
        }
        if (!ok) {  // copies in flight land before the CTA ends
            if (lane == 0) {
                *dead = 1;
                atomicOr(p.err, SALT_DEVERR_TIMEOUT);
            }
            for (uint32_t i = 0; i < min(k_used, (uint32_t)L::KST); ++i)
                mbar_wait(base + L::K_FULL + 8 * ((k_used - 1 - i) % L::KST), ((k_used - 1 - i) / L::KST) & 1);
            for (uint32_t i = 0; i < min(v_used, (uint32_t)L::VST); ++i)
                mbar_wait(base + L::V_FULL + 8 * ((v_used - 1 - i) % L::VST), ((v_used - 1 - i) / L::VST) & 1);
        }
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issue: the whole warp goes along, one lane issues (so that the
        // descriptors stay in uniform registers).  The scores run one tile ahead of the products, into the next
        // item where its queries are there.
        const bool lead = elect_one();
        uint32_t g = 0, n = 0, st = 0, ph = 0;
        int sr = 0, sj = 0;  // the scores' next tile: item and tile in it
        bool more = true;
        Item si = load_item<L>(p, blockIdx.x, G);
        auto scores = [&](bool wait) {
            if (!ok || !more) return;
            if (sj == 0) {
                const uint32_t bar = base + L::Q_FULL + 8 * (sr & 1);
                if (!wait && !__all_sync(0xffffffffu, mbar_try_wait(bar, (sr >> 1) & 1))) return;
                ok = wait_bar(bar, (sr >> 1) & 1, dead);
            }
            ok = __all_sync(0xffffffffu, ok && wait_bar(base + L::K_FULL + 8 * st, ph, dead));
            if (!ok) return;
            tc_fence_after();
            const int R = L::NWG * (16 << (si.flags & 3));
            const uint32_t id = idesc_e4m3_f32(128, R), to = tmem + L::TM_S + (n & 1) * L::R_MAX, q_at = base + L::Q + (sr & 1) * L::Q_BUF;
            const uint64_t kd = sdesc_rows(base + L::K + st * L::SIDE, L::D, 0), qh = sdesc_rows(q_at, L::D, 0), ql = sdesc_rows(q_at + R * L::D, L::D, 0);
            const bool last = sj + 1 == si.tiles;
            if (lead) {
#pragma unroll
                for (int ks = 0; ks < L::D / 32; ++ks) umma_e4m3(to, kd + 2 * ks, qh + 2 * ks, id, ks > 0);
#pragma unroll
                for (int ks = 0; ks < L::D / 32; ++ks) umma_e4m3(to, kd + 2 * ks, ql + 2 * ks, id, 1);
                umma_commit(base + L::S_FULL + 8 * (n & 1));
                umma_commit(base + L::K_FREE + 8 * st);
                if (last) umma_commit(base + L::Q_FREE + 8 * (sr & 1));
            }
            __syncwarp();
            if (++st == (uint32_t)L::KST) {
                st = 0;
                ph ^= 1;
            }
            ++n;
            if (++sj == si.tiles) {
                sj = 0;
                ++sr;
                const int idx = item_index(sr);
                more = idx < n_items;
                if (more) si = load_item<L>(p, idx, G);
            }
        };
        for (int r = 0; ok; ++r) {
            const int idx = item_index(r);
            if (idx >= n_items) break;
            const Item it = load_item<L>(p, idx, G);
            const int R = L::NWG * (16 << (it.flags & 3)), pitch = min(2 * R, 128);
            const uint32_t id = idesc_f16_f32_mn(L::D, R);
            const uint64_t vd = sdesc_rows(base + L::VH, 128, TT * 128), pd = sdesc_rows(base + L::P, pitch, TT * 128);
            for (int j = 0; j < it.tiles && ok; ++j, ++g) {
                if (n == g) scores(true);
                if (n == g + 1) scores(false);
                ok = ok && wait_bar(base + L::P_FULL, g & 1, dead);
                if (j == 0 && r > 0) ok = ok && wait_bar(base + L::O_FREE + 8 * ((r - 1) & 1), ((r - 1) >> 1) & 1, dead);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                const int steps = min(TT, it.t1 - it.t0 - j * TT + 15) / 16;
                if (lead) {
                    for (int ks = 0; ks < steps; ++ks)
                        umma_bf16(tmem + L::TM_O, vd + ks * (16 * 128 / 16), pd + ks * (16 * pitch / 16), id, j > 0 || ks > 0);
                    umma_commit(base + L::PV_DONE);
                }
                __syncwarp();
            }
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
    } else if (warp >= 4) {
        // ------------------------------------------------ softmax and results
        Soft s;
        s.base = base;
        s.tmem = tmem;
        s.dead = dead;
        s.wg = (warp - 4) >> 2;
        s.tid = tid & (WG - 1);
        s.lane = lane;
        s.quarter = warp & 3;
        s.g = s.stage = s.stage_phase = 0;
        s.ok = true;
        for (int r = 0; ok; ++r) {
            const int idx = item_index(r);
            if (idx >= n_items) break;
            const Item it = load_item<L>(p, idx, G);
            // (the columns' constants are there before the first scores are)
            soft_wait(s, base + L::Q_FULL + 8 * (r & 1), (r >> 1) & 1);
            ok = soft_item<L>(p, s, it, r);
        }
        if (!ok && s.tid == 0) {
            *dead = 1;
            atomicOr(p.err, SALT_DEVERR_TIMEOUT);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, L::TM_COLS);
    if (!L::WIDE) pdl_wait();  // so that what follows this kernel follows the wide one too
}

// The rows that several items share (and those no item has),
//     out = sum_i 2^(l_i - L) o_i,   L = log2 sum_i 2^(l_i).
// A CTA's warps take a row each, or (SPLIT) a part of one row's items each and meet in shared memory, where
// rows are so few that the time is that of a row's loads one behind the other.  A
// warp has the logarithms of 32 items over its lanes, and four items' rows under way.
constexpr int COMBINE_WARPS = 4, COMBINE_SPLIT = 16;
// Rows an SM up to which they are split: the CTAs of COMBINE_SPLIT warps that it holds.  64 rows of 80 items each took
// 21 us with a warp a row and 7 us split; 2,048 rows of few items gain nothing (64 us a run with a warp a row, 66 split).
constexpr int COMBINE_FEW = 4;

template <int D, int SPLIT>
__global__ void __launch_bounds__(32 * (SPLIT > 1 ? SPLIT : COMBINE_WARPS)) attn_combine_kernel(const __grid_constant__ AttnParams p)
{
    constexpr int E = D / 32, AT_ONCE = 4;
    const int T = __ldg(p.plan + HD_TOKENS), H = p.n_heads, KV = p.kv.heads, G = H / KV, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int partial = __ldg(p.plan + HD_PARTIAL);
    const int row = SPLIT == 1 ? blockIdx.x * COMBINE_WARPS + warp : blockIdx.x, t = row / H, h = row - t * H, kh = h / G, g = h - kh * G;
    const bool live = T <= p.max_tok && partial && t < T;
    int4 a = make_int4(0, 0, 0, 0), b = make_int4(0, 0, 1, 0);
    if (live) {
        const int4 *rec = reinterpret_cast<const int4 *>(p.plan + p.tok_at + t * TOK_WORDS);
        a = __ldg(rec);
        b = __ldg(rec + 1);
    }
    pdl_wait();    // (the plan is older than the items' kernels)
    if (b.z) return;  // no such row, or written by its only item
    const int own_n = a.z, all = own_n + b.y;
    const int part = SPLIT == 1 ? 0 : warp, from = all * part / SPLIT, n = all * (part + 1) / SPLIT;
    auto place = [&](int i) -> int {  // the row's i-th partial
        return i < own_n ? a.x + (i * KV + kh) * a.y + g : a.w + ((i - own_n) * KV + kh) * b.x + g;
    };
    float top = -INFINITY, sum = 0.f, o[E];
    bool nan = false;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int i0 = from; i0 < n; i0 += 32) {
        const int k = min(32, n - i0), mine = place(i0 + min(lane, k - 1));
        const float l = lane < k ? __ldcg(p.part_l + mine) : -INFINITY;
        float v[AT_ONCE][E];
        auto load = [&](int i) {
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int at = __shfl_sync(0xffffffffu, mine, min(i + u, 31));
                const float *src = p.part_o + (int64_t)at * D + lane * E;
                if (i + u >= k) continue;
                if constexpr (E == 4) {
                    const float4 x = __ldcg(reinterpret_cast<const float4 *>(src));
                    v[u][0] = x.x;
                    v[u][1] = x.y;
                    v[u][2] = x.z;
                    v[u][3] = x.w;
                } else {
                    const float2 x = __ldcg(reinterpret_cast<const float2 *>(src));
                    v[u][0] = x.x;
                    v[u][1] = x.y;
                }
            }
        };
        load(0);
        nan |= !(l == l);
        float m = fmaxf(top, l);
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, w));
        if (m == -INFINITY) continue;
        const float keep = ex2(top - m), w = ex2(l - m);
        top = m;
        sum *= keep;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= keep;
        for (int i = 0; i < k; i += AT_ONCE) {
            if (i > 0) load(i);
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const float f = __shfl_sync(0xffffffffu, w, min(i + u, 31));
                if (i + u < k) {
                    sum += f;
#pragma unroll
                    for (int e = 0; e < E; ++e) o[e] = fmaf(f, v[u][e], o[e]);
                }
            }
        }
    }
    nan = __any_sync(0xffffffffu, nan);
    if constexpr (SPLIT > 1) {  // (the whole CTA has one row)
        __shared__ float s_o[SPLIT][D], s_top[SPLIT], s_sum[SPLIT];
#pragma unroll
        for (int e = 0; e < E; ++e) s_o[part][lane * E + e] = o[e];
        if (lane == 0) {
            s_top[part] = top;
            s_sum[part] = nan ? __uint_as_float(0x7fc00000u) : sum;
        }
        __syncthreads();
        if (warp > 0) return;
        top = s_top[0];
#pragma unroll
        for (int q = 1; q < SPLIT; ++q) top = fmaxf(top, s_top[q]);
        sum = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll
        for (int q = 0; q < SPLIT; ++q) {
            const float f = s_top[q] == -INFINITY ? 0.f : ex2(s_top[q] - top);
            nan |= !(s_sum[q] == s_sum[q]);
            sum = fmaf(s_sum[q], f, sum);
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(s_o[q][lane * E + e], f, o[e]);
        }
    }
    const float bad = __uint_as_float(0x7fc00000u), inv = nan ? bad : sum > 0.f ? 1.f / sum : 0.f;
    uint32_t out[E / 2];
#pragma unroll
    for (int e = 0; e < E; e += 2) {
        const __nv_bfloat162 r = __floats2bfloat162_rn(o[e] * inv, o[e + 1] * inv);
        out[e / 2] = *reinterpret_cast<const uint32_t *>(&r);
    }
    uint16_t *dst = p.out + t * p.out_stride + h * D + lane * E;
    if constexpr (E == 4) *reinterpret_cast<uint2 *>(dst) = make_uint2(out[0], out[1]);
    else *reinterpret_cast<uint32_t *>(dst) = out[0];
    if (p.lse && lane == 0) p.lse[row] = nan ? bad : sum > 0.f ? (top + log2f(sum)) * 0.693147180559945f : -INFINITY;
}

}  // namespace
}  // namespace salt

using namespace salt;

struct salt_attn {
    salt_kv *kv = nullptr;
    salt_attn_config cfg{};
    int device = 0, n_sm = 1;
    CUtensorMap kmap, vmap;
    int32_t *plan = nullptr;                   // device tables
    int tok_at = 0, order_at = 0, rec_at = 0, rec_cap = 0, pages_at = 0;
    size_t plan_words = 0;
    float *part_o = nullptr, *part_l = nullptr;
    int64_t part_cap = 0;                      // partial rows
    int32_t *staging[2] = {nullptr, nullptr};  // page-locked host copies of the tables
    cudaEvent_t staging_ev[2] = {nullptr, nullptr};
    bool staging_used[2] = {false, false};
    int staging_next = 0;
    bool built = false;
    bool wide = false, narrow = false;         // there are items of this kind
    bool partial = false;                      // some row needs the combine
    int n_items[2] = {0, 0}, most_tiles[2] = {0, 0};  // narrow and wide items of all heads, tiles of the longest
    int T = 0;
    std::vector<cudaStream_t> use_streams;     // the build's stream and the runs' since, but for captured ones
    unsigned long long capture = 0;            // the capture that the last captured run belongs to
    std::vector<cudaStream_t> capture_streams; // and its runs' streams
    cudaEvent_t tmp_ev = nullptr;
};

namespace {

// The capture that the stream takes part in, 0 for none.
cudaError_t capture_of(cudaStream_t stream, unsigned long long *id)
{
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    *id = 0;
    const cudaError_t e = cudaStreamGetCaptureInfo(stream, &status, id);
    if (e == cudaSuccess && status == cudaStreamCaptureStatusNone) *id = 0;
    return e;
}

// Makes `stream` wait for what the others were given so far.
cudaError_t order_after(salt_attn *a, const std::vector<cudaStream_t> &others, cudaStream_t stream)
{
    for (cudaStream_t s : others) {
        if (s == stream) continue;
        cudaError_t e = cudaEventRecord(a->tmp_ev, s);
        if (e == cudaSuccess) e = cudaStreamWaitEvent(stream, a->tmp_ev, 0);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// The same for a stream that is not captured and the plan's uses.  One whose stream is being captured by now cannot be waited
// for: that is refused, as a wait would draw `stream` into the capture.
salt_status order_after_uses(salt_attn *a, cudaStream_t stream)
{
    salt_ctx *ctx = a->kv->ctx;
    for (cudaStream_t s : a->use_streams) {
        unsigned long long id = 0;
        if (s != stream) SALT_CUDA_OR_FAIL(ctx, capture_of(s, &id));
        if (id) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "a stream that the plan was used on is being captured");
    }
    SALT_CUDA_OR_FAIL(ctx, order_after(a, a->use_streams, stream));
    return SALT_OK;
}

void add_stream(std::vector<cudaStream_t> &v, cudaStream_t stream)
{
    if (std::find(v.begin(), v.end(), stream) == v.end()) v.push_back(stream);
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
        // (all pointers first: only then is the last one the number of pages that may be read)
        for (int i = 0; i < n; ++i)
            if (ptr[i + 1] < ptr[i] || used + ptr[i + 1] > c.max_pages)
                return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s %d: page list [%d, %d) out of order or past max_pages", what, i,
                                ptr[i], ptr[i + 1]);
        if (ptr[n] > 0 && !pages) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null page list");
        for (int i = 0; i < n; ++i) {
            if (len[i] < 0) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s %d has %d tokens", what, i, len[i]);
            const int need = (int)(((int64_t)len[i] + kv.page - 1) >> kv.page_log2);
            if (need > ptr[i + 1] - ptr[i])
                return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s %d: %d tokens need %d pages, its list has %d", what, i, len[i], need,
                                ptr[i + 1] - ptr[i]);
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

// Rows of query tokens that go through the cache together.
struct RowTile {
    int tok, ntok;      // in the token order
    int pages;          // first entry of the page list
    int len;            // cached tokens it walks
    int lim;            // tokens the first query token sees
    bool causal, alone; // alone: no row of it has another tile
    int cls;            // columns a warpgroup: 16 << cls
    bool wide;
};

// The time of an item in units of a narrow item's tile of 128 tokens, from measurements: a
// tile of each class of wide items, and what an item takes besides.  (3, 6 and 8 for a wide item and 1.5 to 4 for
// a narrow one move the batches measured by 2% at most, 1 for a narrow one costs up to 9%.)
constexpr float NARROW_TILE = 1.f, NARROW_ITEM = 2.f;
constexpr float WIDE_TILE[3] = {1.1f, 1.4f, 2.2f};
constexpr float WIDE_ITEM = 6.f;

float tile_cost(const RowTile &x) { return x.wide ? WIDE_TILE[x.cls] : NARROW_TILE; }
int items_of(const RowTile &x, double most, int *per_item)
{
    const int n = (x.len + TT - 1) / TT;
    *per_item = (int)std::min<double>(n, std::max(1.0, std::floor(most / tile_cost(x))));
    return (n + *per_item - 1) / *per_item;
}

// Items of one cost.
struct Same {
    float cost;
    int64_t items;
};

// How long the CTAs take for items handed out in falling order of cost, forwards and backwards in turn: of
// every two rounds, the longer of a CTA's at the ends of a round and at its middle.
double run_length(std::vector<Same> &v, int ctas)
{
    std::sort(v.begin(), v.end(), [](const Same &x, const Same &y) { return x.cost > y.cost; });
    int64_t all = 0;
    for (Same &x : v) x.items = all += x.items;  // (now up to and with these)
    auto cost = [&](int64_t rank) {
        const auto it = std::upper_bound(v.begin(), v.end(), rank, [](int64_t r, const Same &x) { return r < x.items; });
        return it == v.end() ? 0.0 : (double)it->cost;
    };
    double sum = 0;
    for (int64_t r = 0; r < all; r += 2 * (int64_t)ctas)
        sum += std::max(cost(r) + cost(r + 2 * ctas - 1), cost(r + ctas - 1) + cost(r + ctas));
    return sum;
}

// How long an item of the wide (or of the narrow) tiles may get: the shortest estimated run among some lengths.
// With few tiles (long ranges, many items each) the run is what its rounds of items take, which is why
// lengths a little above a whole part of a CTA's share are among them: with the share's fourth itself some
// CTAs got a fifth item (two requests of 200,000 tokens took 116 us, now 99 us).  With many it is their items spread over
// the CTAs plus half of the longest one.  Keeps to the records and partial rows that are left, if it
// splits at all.
double split_limit(const std::vector<RowTile> &tiles, bool wide, int KV, int G, int ctas, int64_t *recs_left, int64_t *rows_left)
{
    constexpr int FEW = 64;
    double whole = 0;
    int kind = 0;
    for (const RowTile &x : tiles)
        if (x.wide == wide) {
            whole += KV * (tile_cost(x) * ((x.len + TT - 1) / TT));
            ++kind;
        }
    const double even = std::max(1.0, whole / ctas);
    double best = 1e300, limit = 1e300;
    int64_t best_recs = 0, best_rows = 0;
    std::vector<Same> same;
    auto consider = [&](double part) {  // 0: no splits
        const double most = part == 0.0 ? 1e300 : std::max(1.0, even * part);
        const float fixed = wide ? WIDE_ITEM : NARROW_ITEM;
        double sum = 0, longest = 0;
        int64_t recs = 0, rows = 0;
        same.clear();
        for (const RowTile &x : tiles) {
            if (x.wide != wide) continue;
            const float cost = tile_cost(x);
            int per_item;
            const int n = (x.len + TT - 1) / TT, items = items_of(x, most, &per_item);
            recs += items;
            rows += (int64_t)items * KV * x.ntok * G;
            sum += KV * (n * cost + items * fixed);
            longest = std::max(longest, (double)per_item * cost + fixed);
            if (kind <= FEW) {
                const int less = n / items, more = n - less * items;  // `more` items have a tile more
                if (more > 0) same.push_back({(less + 1) * cost + fixed, (int64_t)more * KV});
                same.push_back({less * cost + fixed, (int64_t)(items - more) * KV});
            }
        }
        if (part != 0.0 && (recs > *recs_left || rows > *rows_left)) return;
        const double est = kind <= FEW ? run_length(same, ctas) : std::max(longest, sum / ctas + 0.5 * longest);
        if (est < best) {
            best = est;
            limit = most;
            best_recs = recs;
            best_rows = rows;
        }
    };
    for (double part : {0.0, 2.0, 1.0, 0.66, 0.5, 0.33, 0.25, 0.125}) consider(part);
    if (kind <= FEW)
        for (int k : {1, 2, 3, 4, 6, 8})
            for (double more : {1.03, 1.06, 1.1}) consider(more / k);
    *recs_left -= best_recs;
    *rows_left -= best_rows;
    return limit;
}

// Plans a checked batch into the tables at w; returns the words used.
size_t fill_plan(salt_attn *a, const salt_attn_batch *b, int T, int32_t *w)
{
    const KvDev &kv = a->kv->dev;
    const int G = a->cfg.n_heads / kv.heads, KV = kv.heads;
    const int per = std::max(1, WIDE_ROWS / G);  // whole query tokens a tile
    std::memset(w, 0, HEAD_WORDS * 4);
    w[HD_TOKENS] = T;
    const int own_pages = b->n_seqs > 0 ? b->page_ptr[b->n_seqs] : 0;
    const int grp_pages = b->n_groups > 0 ? b->group_page_ptr[b->n_groups] : 0;
    int32_t *order = w + a->order_at, *tok = w + a->tok_at;
    std::memset(tok, 0, (size_t)T * TOK_WORDS * 4);
    for (int t = 0; t < T; ++t) order[t] = t;
    const bool grouped = b->group && b->n_groups > 0;
    auto prompt = [&](int i) { return grouped && b->group[i] >= 0 ? b->group_len[b->group[i]] : 0; };
    auto add = [&](std::vector<RowTile> &to, int tok, int ntok, int pages, int64_t len, int64_t lim, bool causal, bool alone) {
        const int rows = ntok * G;
        const bool wide = rows > narrow_rows(kv.dim);
        const int cw = wide ? (rows + 1) / 2 : rows;
        to.push_back({tok, ntok, pages, (int)len, (int)lim, causal, alone, cw <= 16 ? 0 : cw <= 32 ? 1 : 2, wide});
    };
    std::vector<RowTile> tiles;
    // own tokens: `per` query tokens of a request at a time
    int t0 = 0;
    for (int i = 0; i < b->n_seqs; t0 += b->q_len[i], ++i) {
        const int n = b->q_len[i], kvl = b->kv_len[i];
        for (int j = 0; j < n; j += per) {
            const int m = std::min(per, n - j);
            const int64_t len = (int64_t)kvl - n + j + m;  // what the last of them sees
            if (len <= 0) continue;
            add(tiles, t0 + j, m, b->page_ptr[i], len, (int64_t)kvl - n + j + 1, true, prompt(i) == 0);
        }
    }
    // prompts: the query tokens of a group's requests, in the second part of the order
    if (grouped) {
        std::vector<int> at(b->n_groups + 1, 0);
        for (int i = 0; i < b->n_seqs; ++i)
            if (b->group[i] >= 0) at[b->group[i] + 1] += b->q_len[i];
        for (int g = 0; g < b->n_groups; ++g) at[g + 1] += at[g];
        std::vector<int> next(at.begin(), at.end() - 1);
        std::vector<uint8_t> own(T, 0);
        for (const RowTile &x : tiles)
            for (int k = 0; k < x.ntok; ++k) own[x.tok + k] = 1;
        t0 = 0;
        for (int i = 0; i < b->n_seqs; t0 += b->q_len[i], ++i)
            if (b->group[i] >= 0)
                for (int j = 0; j < b->q_len[i]; ++j) order[T + next[b->group[i]]++] = t0 + j;
        for (int g = 0; g < b->n_groups; ++g) {
            if (b->group_len[g] == 0) continue;
            for (int j = at[g]; j < at[g + 1]; j += per) {
                const int m = std::min(per, at[g + 1] - j);
                bool alone = true;
                for (int k = 0; k < m; ++k) alone = alone && !own[order[T + j + k]];
                add(tiles, T + j, m, own_pages + b->group_page_ptr[g], b->group_len[g], b->group_len[g], false, alone);
            }
        }
    }
    // (without splits every list fits: its share of the records and rows is set aside first)
    int64_t recs_left = a->rec_cap, rows_left = a->part_cap;
    for (const RowTile &x : tiles)
        if (!x.wide) {
            recs_left -= 1;
            rows_left -= (int64_t)KV * x.ntok * G;
        }
    const double wide_limit = split_limit(tiles, true, KV, G, a->n_sm * Shape<128, true>::CTAS, &recs_left, &rows_left);
    for (const RowTile &x : tiles)
        if (!x.wide) {
            recs_left += 1;
            rows_left += (int64_t)KV * x.ntok * G;
        }
    const double narrow_limit = split_limit(tiles, false, KV, G, a->n_sm * Shape<128, false>::CTAS, &recs_left, &rows_left);
    struct Rec {
        float cost;
        int tile, t0, t1, part;
        bool direct, wide;
    };
    std::vector<Rec> recs;
    int n_wide = 0;
    a->most_tiles[0] = a->most_tiles[1] = 0;
    int64_t part = 0;
    bool partial = false;
    std::vector<uint8_t> seen(T, 0);
    for (size_t k = 0; k < tiles.size(); ++k) {
        const RowTile &x = tiles[k];
        const int n = (x.len + TT - 1) / TT, rows = x.ntok * G;
        int per_item;
        const int items = items_of(x, x.wide ? wide_limit : narrow_limit, &per_item);
        const bool direct = items == 1 && x.alone;
        for (int i = 0; i < items; ++i) {
            // splits of equal length but for rounding
            const int a0 = (int)((int64_t)n * i / items), a1 = (int)((int64_t)n * (i + 1) / items);
            recs.push_back({tile_cost(x) * (a1 - a0), (int)k, a0 * TT, std::min(x.len, a1 * TT),
                            direct ? 0 : (int)(part + (int64_t)i * KV * rows), direct, x.wide});
            n_wide += x.wide;
            a->most_tiles[x.wide] = std::max(a->most_tiles[x.wide], a1 - a0);
        }
        for (int i = 0; i < x.ntok; ++i) {
            const int t = order[x.tok + i];
            int32_t *r = tok + (size_t)t * TOK_WORDS;
            seen[t] = 1;
            if (direct) {
                r[TK_DIRECT] = 1;
                continue;
            }
            r[x.causal ? TK_OWN : TK_PRE] = (int)(part + i * G);
            r[x.causal ? TK_OWN_ROWS : TK_PRE_ROWS] = rows;
            r[x.causal ? TK_OWN_N : TK_PRE_N] = items;
        }
        if (!direct) {
            part += (int64_t)items * KV * rows;
            partial = true;
        }
    }
    for (int t = 0; t < T && !partial; ++t) partial = !seen[t];  // a row that sees nothing is the combine's too
    std::stable_sort(recs.begin(), recs.end(), [](const Rec &x, const Rec &y) { return x.wide != y.wide ? x.wide : x.cost > y.cost; });
    int32_t *rw = w + a->rec_at;
    for (const Rec &r : recs) {
        const RowTile &x = tiles[r.tile];
        rw[RC_FLAGS] = x.cls | (r.direct ? RF_DIRECT : 0) | (x.causal ? RF_CAUSAL : 0);
        rw[RC_TOK] = x.tok;
        rw[RC_NTOK] = x.ntok;
        rw[RC_PAGES] = x.pages;
        rw[RC_T0] = r.t0;
        rw[RC_T1] = r.t1;
        rw[RC_LIM] = x.lim;
        rw[RC_PART] = r.part;
        rw += REC_WORDS;
    }
    w[HD_WIDE] = n_wide;
    w[HD_NARROW] = (int)recs.size() - n_wide;
    a->wide = n_wide > 0;
    a->narrow = (int)recs.size() > n_wide;
    a->n_items[1] = n_wide * KV;
    a->n_items[0] = ((int)recs.size() - n_wide) * KV;
    w[HD_PARTIAL] = partial ? 1 : 0;
    a->partial = partial;
    int32_t *pg = w + a->pages_at;
    if (own_pages > 0) std::memcpy(pg, b->pages, (size_t)own_pages * 4);
    if (grp_pages > 0) std::memcpy(pg + own_pages, b->group_pages, (size_t)grp_pages * 4);
    return (size_t)a->pages_at + own_pages + grp_pages;
}

// A cache's codes as rows of D bytes, a box a page's rows of one head, swizzled over a row's width.
cudaError_t encode_codes_map(CUtensorMap *out, uint8_t *codes, int dim, int64_t rows, int page)
{
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
    if (e != cudaSuccess || q != cudaDriverEntryPointSuccess || !fn) return e != cudaSuccess ? e : cudaErrorNotSupported;
    const cuuint64_t dims[2] = {(cuuint64_t)dim, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)dim};
    const cuuint32_t box[2] = {(cuuint32_t)dim, (cuuint32_t)page}, es[2] = {1, 1};
    const CUresult r = reinterpret_cast<Encode>(fn)(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, codes, dims, strides, box, es,
                                                    CU_TENSOR_MAP_INTERLEAVE_NONE,
                                                    dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                                                    CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <class L>
cudaError_t prepare_tiles()
{
    return cudaFuncSetAttribute(attn_tile_kernel<L>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::BYTES);
}

template <class L>
cudaError_t launch_tiles(const AttnParams &params, int n_sm, bool behind, cudaStream_t stream)
{
    AttnParams p = params;
    p.behind = behind;
    return launch_overlapped(attn_tile_kernel<L>, n_sm * L::CTAS, L::THREADS, L::BYTES, stream, p);
}

// The wide items, the narrow ones (which fill the SMs as the wide ones
// end) and the rows they share.
template <int D>
cudaError_t launch_attn(const AttnParams &p, int n_sm, bool wide, bool narrow, bool combine, cudaStream_t stream)
{
    if (wide) {
        const cudaError_t e = launch_tiles<Shape<D, true>>(p, n_sm, false, stream);
        if (e != cudaSuccess) return e;
    }
    if (narrow) {
        const cudaError_t e = launch_tiles<Shape<D, false>>(p, n_sm, wide, stream);
        if (e != cudaSuccess) return e;
    }
    if (!combine) return cudaSuccess;
    // (rows in all are below 2^31: partial rows, twice as many, are)
    const int rows = p.max_tok * p.n_heads;
    const bool few = rows <= n_sm * COMBINE_FEW;
    const auto kernel = few ? attn_combine_kernel<D, COMBINE_SPLIT> : attn_combine_kernel<D, 1>;
    const unsigned blocks = few ? rows : (rows + COMBINE_WARPS - 1) / COMBINE_WARPS, threads = 32 * (few ? COMBINE_SPLIT : COMBINE_WARPS);
    // (it reads the plan before its wait: the plan is there when an items' kernel is past its own)
    if (wide || narrow) return launch_overlapped(kernel, blocks, threads, 0, stream, p);
    kernel<<<blocks, threads, 0, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

extern "C" {

salt_status salt_attn_create(salt_kv *kv, const salt_attn_config *c, salt_attn **out)
{
    if (!out) return SALT_ERR_INVALID_ARG;
    *out = nullptr;
    if (!kv || !c) return SALT_ERR_INVALID_ARG;
    salt_ctx *ctx = kv->ctx;
    const KvDev &d = kv->dev;
    if (c->n_heads < 1 || c->n_heads % d.heads || c->n_heads / d.heads > 64)
        return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d query heads over %d key/value heads", c->n_heads, d.heads);
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
    a->device = ctx_device(ctx);
    auto fail_with = [&](salt_status st, const char *what) {
        cudaGetLastError();
        salt_attn_destroy(a);
        return ctx_fail(ctx, st, "%s", what);
    };
    if (cudaDeviceGetAttribute(&a->n_sm, cudaDevAttrMultiProcessorCount, ctx_device(ctx)) != cudaSuccess ||
        prepare_tiles<Shape<64, true>>() != cudaSuccess || prepare_tiles<Shape<64, false>>() != cudaSuccess ||
        prepare_tiles<Shape<128, true>>() != cudaSuccess || prepare_tiles<Shape<128, false>>() != cudaSuccess)
        return fail_with(SALT_ERR_CUDA, "cannot prepare the attention kernel");
    const int64_t rows = (int64_t)kv->n_layers * d.n_pages * d.heads * d.page;
    if (encode_codes_map(&a->kmap, d.k, d.dim, rows, d.page) != cudaSuccess ||
        encode_codes_map(&a->vmap, d.v, d.dim, rows, d.page) != cudaSuccess)
        return fail_with(SALT_ERR_CUDA, "cannot map the cache");
    // Items: without splits at most one per request's and per group's row
    // tile; with them the plan keeps within the rest.  Partial rows: two per
    // row without splits.
    const int G = c->n_heads / d.heads, per = std::max(1, WIDE_ROWS / G);
    a->rec_cap = c->max_seqs + c->max_groups + 2 * (c->max_tokens / per + 1) + 16 * a->n_sm;
    a->part_cap = 2ll * c->max_tokens * c->n_heads + 512ll * a->n_sm;
    if (a->part_cap >= (1ll << 31)) return fail_with(SALT_ERR_INVALID_ARG, "max_tokens times n_heads is too large");
    a->tok_at = HEAD_WORDS;
    a->order_at = a->tok_at + c->max_tokens * TOK_WORDS;
    a->rec_at = (a->order_at + 2 * c->max_tokens + 3) / 4 * 4;
    a->pages_at = a->rec_at + a->rec_cap * REC_WORDS;
    a->plan_words = ((size_t)a->pages_at + c->max_pages + 3) / 4 * 4;
    bool ok = cudaMalloc(&a->plan, a->plan_words * 4) == cudaSuccess &&
              cudaMalloc(&a->part_o, (size_t)a->part_cap * d.dim * 4) == cudaSuccess &&
              cudaMalloc(&a->part_l, (size_t)a->part_cap * 4) == cudaSuccess;
    for (int i = 0; i < 2 && ok; ++i)
        ok = cudaHostAlloc(reinterpret_cast<void **>(&a->staging[i]), a->plan_words * 4, cudaHostAllocMapped) == cudaSuccess &&
             cudaEventCreateWithFlags(&a->staging_ev[i], cudaEventDisableTiming) == cudaSuccess;
    ok = ok && cudaEventCreateWithFlags(&a->tmp_ev, cudaEventDisableTiming) == cudaSuccess;
    if (!ok) return fail_with(SALT_ERR_OOM, "no memory for the plan's tables and partial results");
    *out = a;
    return SALT_OK;
}

void salt_attn_destroy(salt_attn *a)
{
    if (!a) return;
    cudaSetDevice(a->device);  // (the cache and the context may be gone already)
    cudaDeviceSynchronize();
    cudaFree(a->plan);
    cudaFree(a->part_o);
    cudaFree(a->part_l);
    for (int i = 0; i < 2; ++i) {
        if (a->staging[i]) cudaFreeHost(a->staging[i]);
        if (a->staging_ev[i]) cudaEventDestroy(a->staging_ev[i]);
    }
    if (a->tmp_ev) cudaEventDestroy(a->tmp_ev);
    cudaGetLastError();
    delete a;
}

salt_status salt_attn_build(salt_attn *a, const salt_attn_batch *b, salt_stream_t stream_)
try {
    NvtxRange nvtx_range("salt_attn_build");
    if (!a) return SALT_ERR_INVALID_ARG;
    salt_ctx *ctx = a->kv->ctx;
    if (!b) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null batch");
    if (!ctx_select_device(ctx)) return ctx_fail(ctx, SALT_ERR_CUDA, "cannot select the device");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    unsigned long long capture;
    SALT_CUDA_OR_FAIL(ctx, capture_of(stream, &capture));
    if (capture) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "a build cannot be captured");
    a->built = false;
    int T = 0;
    salt_status st = check_batch(a, b, &T);
    if (st != SALT_OK) return st;
    const int k = a->staging_next;
    if (a->staging_used[k]) SALT_CUDA_OR_FAIL(ctx, cudaEventSynchronize(a->staging_ev[k]));
    a->staging_next ^= 1;
    const size_t words = fill_plan(a, b, T, a->staging[k]);
    st = order_after_uses(a, stream);
    if (st != SALT_OK) return st;
    const int n16 = (int)((words + 3) / 4);
    plan_copy_kernel<<<std::min(64, (n16 + 255) / 256), 256, 0, stream>>>(reinterpret_cast<const uint4 *>(a->staging[k]),
                                                                          reinterpret_cast<uint4 *>(a->plan), n16);
    SALT_CUDA_OR_FAIL(ctx, cudaGetLastError());
    SALT_CUDA_OR_FAIL(ctx, cudaEventRecord(a->staging_ev[k], stream));
    a->staging_used[k] = true;
    a->T = T;
    a->use_streams.assign(1, stream);
    a->built = true;
    return SALT_OK;
} catch (const std::bad_alloc &) {
    return ctx_fail(a->kv->ctx, SALT_ERR_OOM, "no host memory");
}

salt_status salt_attn_get_shape(const salt_attn *a, salt_attn_shape *out)
{
    if (!a || !out) return SALT_ERR_INVALID_ARG;
    *out = salt_attn_shape{};
    out->workspace_bytes = (int64_t)a->plan_words * 4 + a->part_cap * (a->kv->dev.dim + 1) * 4;
    out->wide_ctas = a->n_sm * Shape<128, true>::CTAS;
    out->narrow_ctas = a->n_sm * Shape<128, false>::CTAS;
    if (!a->built) return SALT_OK;
    out->wide_items = a->n_items[1];
    out->wide_tiles = a->most_tiles[1];
    out->narrow_items = a->n_items[0];
    out->narrow_tiles = a->most_tiles[0];
    out->combined = a->partial;
    return SALT_OK;
}

salt_status salt_attn_run(salt_attn *a, int32_t layer, const void *q, int64_t q_stride, float scale, void *out,
                          int64_t out_stride, float *lse, salt_stream_t stream_)
try {
    NvtxRange nvtx_range("salt_attn_run");
    if (!a) return SALT_ERR_INVALID_ARG;
    salt_ctx *ctx = a->kv->ctx;
    const KvDev &kv = a->kv->dev;
    if (!a->built) return ctx_fail(ctx, SALT_ERR_NOT_BUILT, "the attention plan was not built");
    if (layer < 0 || layer >= a->kv->n_layers)
        return ctx_fail(ctx, SALT_ERR_LAYER_RANGE, "layer %d outside [0, %d)", layer, a->kv->n_layers);
    if (!std::isfinite(scale)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "scale is not finite");
    if (!ctx_select_device(ctx)) return ctx_fail(ctx, SALT_ERR_CUDA, "cannot select the device");
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    unsigned long long capture;
    SALT_CUDA_OR_FAIL(ctx, capture_of(stream, &capture));
    if (a->T == 0 && !capture) return SALT_OK;
    if (a->T > 0) {
        if (!q || !out) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null q or out");
        const int64_t row = (int64_t)a->cfg.n_heads * kv.dim;
        if (q_stride < row || out_stride < row)
            return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "rows of %lld elements %lld and %lld apart", (long long)row,
                            (long long)q_stride, (long long)out_stride);
        if ((q_stride | out_stride) % 8 || ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) ||
            (reinterpret_cast<uintptr_t>(lse) & 3))
            return ctx_fail(ctx, SALT_ERR_ALIGN, "rows of q or out not on 16-byte boundaries, or lse not on a 4-byte one");
    }
    if (capture) {  // in the order of its capture's other runs; what its replays come after is the caller's to say
        if (a->capture != capture) a->capture_streams.clear();
        a->capture = capture;
        SALT_CUDA_OR_FAIL(ctx, order_after(a, a->capture_streams, stream));
        add_stream(a->capture_streams, stream);
    } else if (a->use_streams.size() != 1 || a->use_streams[0] != stream) {
        const salt_status st = order_after_uses(a, stream);
        if (st != SALT_OK) return st;
        add_stream(a->use_streams, stream);
    }
    AttnParams p;
    p.kmap = a->kmap;
    p.vmap = a->vmap;
    p.plan = a->plan;
    p.kv = kv;
    p.layer = layer;
    p.q = static_cast<const uint16_t *>(q);
    p.out = static_cast<uint16_t *>(out);
    p.lse = lse;
    p.part_o = a->part_o;
    p.part_l = a->part_l;
    p.q_stride = q_stride;
    p.out_stride = out_stride;
    p.n_heads = a->cfg.n_heads;
    p.max_tok = a->T;
    p.tok_at = a->tok_at;
    p.order_at = a->order_at;
    p.rec_at = a->rec_at;
    p.pages_at = a->pages_at;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.err = ctx_error_word(ctx);
    // a captured run may be replayed for a plan that needs other launches
    const bool all = capture != 0, wide = a->wide || all, narrow = a->narrow || all, combine = (a->partial || all) && a->T > 0;
    SALT_CUDA_OR_FAIL(ctx, kv.dim == 128 ? launch_attn<128>(p, a->n_sm, wide, narrow, combine, stream)
                                         : launch_attn<64>(p, a->n_sm, wide, narrow, combine, stream));
    return SALT_OK;
} catch (const std::bad_alloc &) {
    return ctx_fail(a->kv->ctx, SALT_ERR_OOM, "no host memory");
}

}  // extern "C"
