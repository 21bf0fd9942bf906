// The attention plan as its translation units see it: the attention itself
// (salt_attn.cu), and what goes by its lists of cached tokens (salt_weights.cu,
// salt_evict.cu).
#pragma once

#include <vector>

#include "salt_internal.cuh"
#include "salt_tcgen05.cuh"

namespace salt {

// The plan's device tables: int32 words of one block, written by the host
// into a staging area and copied by a kernel.
constexpr int HEAD_WORDS = 8;   // HD_* below
constexpr int HD_TOKENS = 0, HD_WIDE = 1, HD_NARROW = 2, HD_PARTIAL = 3;  // query tokens, records of either kind, whether rows need the combine

// What a tracked plan's build writes besides: a table of its own, int32 words.
constexpr int TRACK_HEAD = 12;  // TH_* below
// query tokens, requests, lists of few rows, whether a page is listed twice, what the tiles of those lists cost, lists of many rows (behind the others),
// tiles of 256 tokens of those, the CTAs that the units of their work are listed for (0: not listed), whether a wait of a call since the build gave up (written
// by that call: the parts' counts may be anything then, and later ones go by whole tiles, which need none)
constexpr int TH_TOKENS = 0, TH_SEQS = 1, TH_FEW = 2, TH_SHARED = 3, TH_FEW_COST = 4, TH_MANY = 5, TH_MANY_TILES = 6, TH_LISTED = 7, TH_FAILED = 8;
// per request: first entry in the page lists, own cached tokens, first entry in the tables of eviction's chunks, none
constexpr int SEQ_WORDS = 4;
// per list of cached tokens that rows see, a request's own or a group's prompt: first entry in the page lists, tokens, first
// entry in the token order, query tokens, tokens that were there before the step, tokens that the first query token sees,
// whether the next ones each see one more (and twice what a tile costs), what the tiles of the lists of its kind before it cost
constexpr int LIST_WORDS = 8;
constexpr int LS_BEFORE = 7;
constexpr int TRACK_TILE = 128, TRACK_MANY_TILE = 256;
constexpr int TRACK_FEW_ROWS = 64;  // of a list whose keys stream past its rows
// units of the many rows' lists: each CTA's first one, then per unit its list's words, the last one the head instead of the cost, and first token, steps
// [from, to), (slot of its first part << 12 | part << 6 | parts - 1) or -1
constexpr int TRACK_CTAS = 512, UNIT_WORDS = 12, TRACK_UNITS = 8192;
constexpr int TRACK_SLOTS = 2048;  // of partial sums, 256 tokens each
// Rows that eviction moves at a time: 16 KB of keys and values.
constexpr int evict_rows(int dim) { return 8192 / dim; }
// What a tile of 128 tokens of a list of few rows costs, in quarters of one with a single row.  (64 lists of 8,192 tokens with 8 heads of 64, of which an SM's two CTAs take
// a tile in 0.37 us with 20 rows, 0.48 with 32, 0.61 with 48 and 0.75 with 64, where this says 5, 6, 8 and 9; three CTAs an SM, 0.26 with 1 and 8 rows, 0.28 with 16, where it
// says 4, 4 and 5.)
constexpr int few_cost(int rows) { return 4 + rows / 12; }
// The first step of `per` query tokens that sees token t0.
__host__ __device__ constexpr int first_step(bool causal, int lim, int t0, int per)
{
    return causal && t0 >= lim ? (t0 - lim + 1) / per : 0;
}

struct Track {
    int32_t *table = nullptr;                  // device
    int32_t *staging[2] = {nullptr, nullptr};  // page-locked host copies, used with the plan's own
    float *part = nullptr;                     // [TRACK_SLOTS][256]
    uint32_t *arrived = nullptr;               // [TRACK_SLOTS][8], zero between calls, but see TH_FAILED
    int seq_at = 0, list_at = 0, unit_at = 0;  // word offsets
    size_t words = 0, bytes = 0;               // of the table, of all its device memory
    bool on = false, built = false, shared = false, split = false;
    int n_seqs = 0, few = 0, many = 0, n_units = 0, few_rows = 0, many_sms = 0;  // few_rows: of the lists of few, the most that one has; SMs for the lists of many
    int64_t few_tiles = 0;
    // eviction's: the longest request, chunks of all requests in the build; room for chunks and layers; tables
    int longest = 0, chunks = 0, chunks_cap = 0, layers_cap = 0;
    int32_t *chunk_ptr = nullptr, *losing = nullptr, *bound = nullptr;
    uint32_t *read = nullptr, *ticket = nullptr;
    std::vector<uint8_t> page_seen;            // scratch of a build

    void free_device()
    {
        for (void *x : {(void *)table, (void *)part, (void *)arrived, (void *)chunk_ptr, (void *)losing, (void *)bound, (void *)read, (void *)ticket}) cudaFree(x);
        table = chunk_ptr = losing = bound = nullptr;
        part = nullptr;
        arrived = read = ticket = nullptr;
    }
};

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

__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("{\n .reg .b64 a, b;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n add.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}\n"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
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

// Checks that a call on the plan's tracked tables may go ahead on `stream` and orders it after the plan's other uses.
// *captured: whether the stream is being captured.
salt_status track_enter(salt_attn *a, int32_t layer, int32_t n_layers, cudaStream_t stream, bool *captured);

}  // namespace salt

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
    salt::Track track;                         // what salt_attn_track adds
};
