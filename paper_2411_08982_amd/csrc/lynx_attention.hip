// Attention over the paged cache (lynx_attention, lynx_attention_prefix).
//
// Rows.  The QH / KVH = G query heads that share a key head read the same keys, so the rows of a request for one key head are its
// n new tokens times G: row r is token r / G, head r % G of the group.
//
// Products.  Both are taken transposed on the matrix cores, v_mfma_f32_16x16x32_bf16:  S^T = K Q^T and O^T = V^T P^T.  A result
// fragment of S^T holds, in lane l, the scores of row l % 16 with 4 consecutive tokens; two fragments give the lane 8 tokens, and in the
// second product, whose terms may come in any order, these are what it holds of its operand.  So the weights never leave their
// lane: no LDS, no exchange; running maximum, sum and the rescaling of O^T are per lane (a row is one column of both results), and
// only the maximum is joined over the four lanes of a row.  V's operand wants those tokens of one channel: the transposed pages.
//
// Softmax in one pass: m = running maximum (of the scores times scale * log2 e), l = sum of 2^(s - m), O accumulates 2^(s - m) v; when
// m grows, l and O are multiplied by 2^(m_old - m_new).  All in fp32.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <type_traits>

#include "lynx_attention.h"

namespace lynx {

constexpr int kBlock = 64;              // tokens of a block: the unit in which a row's context is dealt out
constexpr int kRows = 16;               // rows of a tile
constexpr int kTileRows = 128;          // rows of a tile of the kernel for many rows
constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / kWave;
constexpr int kWorkgroups = 512;       // workgroups that the chip holds at once: two of four waves on each of 256 CUs
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct AttnParams {
    const uint16_t *q;
    const void *k, *v;
    const int32_t *table, *q_start, *seq_len, *prefix_table;
    uint16_t *out;
    float *lse;
    int64_t q_stride, out_stride;
    int B, T, KVH, G, num_pages, max_pages, page_size;
    unsigned page_mul;                  // division of a group of 16 tokens by the page size: page_of
    unsigned group_mul, parts_mul;      // division of rows by G (token_of) and of the line by parts (length_of)
    float scale2, v_scale;              // scale * k_scale * log2 e
    float lag;                          // 8 / scale2: by how much the maximum of a tile's row may fall behind
    int window, sinks;
    int parts;                          // parts that the contexts of all tiles together are cut into, per key head
    float *part_o, *part_ml;            // workspace: unfinished rows
    struct Cut *cuts;                   // and which tiles are to be joined from them
    int narrow;                         // requests of more rows are left to the tiles of 128 rows
    int wide_parts;                     // tiles of 128 rows: parts that all their contexts are cut into, per key head
    float *wide_o, *wide_ml;
    int prefix_blocks, prefix_splits;   // whole blocks of the shared prefix, and the parts that they are cut into
    float *prefix_o, *prefix_ml;        // the parts of all rows,
    float *own_o, *own_ml;              // and what the rows behind the prefix see of their own sequences
    unsigned prefix_groups, tile_groups; // workgroups of the prefix's tiles and of the others
    unsigned turns;                     // their order: attn_kernel
    int tiles_first;
};

// Page (index in a row of the table) of the 16 tokens from 16 * group on: group / (page_size / 16), by multiplication.
// Exact for group < 2^25 and page_size / 16 <= 64, since group * error < 2^31 / (page_size / 16).
__device__ __forceinline__ int page_of(const AttnParams &p, int group) { return (int)__umulhi(2u * (unsigned)group, p.page_mul); }
// Token of row r: r / G, by multiplication.  Exact: r < 2^24 and G <= 256, so r * error < 2^32.
__device__ __forceinline__ int token_of(const AttnParams &p, int r) { return p.G == 1 ? r : (int)__umulhi((unsigned)r, p.group_mul); }
inline unsigned reciprocal(int d) { return d > 1 ? (unsigned)(((uint64_t)1 << 32) / (unsigned)d) + 1u : 0u; }
inline unsigned page_multiplier(int page_size) { return (1u << 31) / (unsigned)(page_size / 16) + 1u; }

// The rows of request b and its length, clamped.
__device__ __forceinline__ void request_of(const AttnParams &p, int b, int &first, int &n, int &seq)
{
    first = min(max(p.q_start[b], 0), p.T);
    n = min(max(p.q_start[b + 1], first), p.T) - first;
    seq = min(max(p.seq_len[b], 0), p.max_pages * p.page_size);
}

// Whether the new tokens of a request, from position `base` on, all lie behind the whole blocks of the shared prefix: then those blocks
// are left to the prefix's tiles.
__device__ __forceinline__ bool behind_prefix(const AttnParams &p, int base) { return p.prefix_blocks > 0 && base >= p.prefix_blocks * kBlock; }

// The blocks that a span of rows at positions pmin .. pmax of a request sees: `lead` blocks of the first tokens that stay visible, then
// those from `start` on; `count` in all.
struct Blocks {
    int lead, start, count;
    __device__ __forceinline__ int at(int i) const { return i < lead ? i : start + i - lead; }
};
__device__ __forceinline__ Blocks blocks_of(const AttnParams &p, int base, int pmin, int pmax)
{
    Blocks s;
    const int end = pmax >= 0 ? pmax / kBlock + 1 : 0;
    s.start = p.window == 0 ? 0 : min(max(pmin - p.window + 1, 0) / kBlock, end);
    if (behind_prefix(p, base)) s.start = p.prefix_blocks;
    s.lead = p.window == 0 ? 0 : min((p.sinks - 1 + kBlock) / kBlock, s.start);
    s.count = s.lead + end - s.start;
    return s;
}

// Whether some row at positions pmin .. pmax sees token t.  (Not by branches: the conditions are a few comparisons.)
__device__ __forceinline__ int seen(const AttnParams &p, int t, int pmin, int pmax)
{
    return (int)(t <= pmax) & ((int)(p.window == 0) | (int)(t > pmin - p.window) | (int)(t < p.sinks));
}

// How the work is cut.  The blocks of all tiles, one tile after the other, are one long line that is cut into equal lengths, one
// for each workgroup that the chip holds at once: however ragged the contexts, all workgroups read the same amount (with whole tiles
// dealt out, 64 requests of 500 to 12000 tokens took 100 us where the equal cut took 71).  A tile that a cut goes through is
// finished by attn_join_kernel.  Request lengths are on the device only: every workgroup sums them up for itself, one round trip
// for the lengths (at most four requests a thread) and one scan.
constexpr int kMinLength = 4;               // blocks of a workgroup at least, one a wave (16 requests of 300 tokens: 15.3 us, with 8 18.9; one of 9001: 18.3 and 17.1)
constexpr int kMaxPerThread = LYNX_MAX_REQUESTS / kAttnThreads;
struct Line {
    unsigned ends[LYNX_MAX_REQUESTS];       // where each request's blocks end on the line
    unsigned long long what[LYNX_MAX_REQUESTS];   // each request's first row (17 bits), rows (17 bits) and length (30 bits)
    unsigned sum[kAttnWaves];
    float work[kAttnWaves];
};
// Blocks of each tile of a request: those that its last rows and its first see together, so no tile has more; one at least.
__device__ __forceinline__ unsigned blocks_per_tile(const AttnParams &p, int n, int seq)
{
    return (unsigned)max(blocks_of(p, seq - n, max(seq - n, 0), seq - 1).count, 1);
}
// Fills line.ends; the length of the line.  (Row ranges that overlap, which is no batch, may make it longer than 32 bits: then it is 0.)
__device__ __forceinline__ unsigned lay_out(const AttnParams &p, Line &line)
{
    const int lane = lane_id(), wv = wave_id();
    const int per = (p.B + kAttnThreads - 1) / kAttnThreads, b0 = threadIdx.x * per;
    unsigned sum[kMaxPerThread], total = 0;
    float work = 0.0f;
#pragma unroll
    for (int i = 0; i < kMaxPerThread; ++i) {
        if (i < per && b0 + i < p.B) {
            int first, n, seq;
            request_of(p, b0 + i, first, n, seq);
            const unsigned tiles = n * p.G <= p.narrow ? (unsigned)(n * p.G + kRows - 1) / kRows : 0u;
            if (tiles > 0) {
                const unsigned blocks = blocks_per_tile(p, n, seq);
                total += tiles * blocks;
                work += (float)tiles * (float)blocks;
            }
            line.what[b0 + i] = (unsigned long long)first << 47 | (unsigned long long)n << 30 | (unsigned)seq;
        }
        sum[i] = total;
    }
    unsigned before = (unsigned)wave_prefix_sum_i32((int)total);
    work = wave_sum(work);
    if (lane == kWave - 1) {
        line.sum[wv] = before;
        line.work[wv] = work;
    }
    before -= total;
    __syncthreads();
    unsigned all = 0;
    work = 0.0f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
        before += w < wv ? line.sum[w] : 0u;
        all += line.sum[w];
        work += line.work[w];
    }
    if (work > 4.0e9f) all = 0;
#pragma unroll
    for (int i = 0; i < kMaxPerThread; ++i)
        if (i < per && b0 + i < p.B) line.ends[b0 + i] = before + sum[i];
    __syncthreads();
    return (unsigned)__builtin_amdgcn_readfirstlane((int)all);
}
__device__ __forceinline__ unsigned length_of(const AttnParams &p, unsigned total) { return max((unsigned)kMinLength, (p.parts == 1 ? total : __umulhi(total, p.parts_mul)) + 1u); }

// The tile that block `at` of the line belongs to: its request, its number there, the line's blocks [begin, begin + count).
struct Place {
    int b, tile, first, n, seq;
    unsigned begin, count;
};
__device__ __forceinline__ Place place_of(const AttnParams &p, const Line &line, unsigned at)
{
    int lo = 0, hi = p.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (line.ends[mid] > at) hi = mid;
        else lo = mid + 1;
    }
    Place s;
    s.b = __builtin_amdgcn_readfirstlane(lo);
    const unsigned long long what = line.what[s.b];
    const unsigned start = (unsigned)__builtin_amdgcn_readfirstlane(s.b > 0 ? (int)line.ends[s.b - 1] : 0);
    const unsigned hi32 = (unsigned)__builtin_amdgcn_readfirstlane((int)(what >> 32)), lo32 = (unsigned)__builtin_amdgcn_readfirstlane((int)what);
    s.first = (int)(hi32 >> 15);
    s.n = (int)((hi32 & 0x7fffu) << 2 | lo32 >> 30);
    s.seq = (int)(lo32 & 0x3fffffffu);
    s.count = blocks_per_tile(p, s.n, s.seq);
    s.tile = s.n * p.G <= kRows ? 0 : (int)((at - start) / s.count);
    s.begin = start + (unsigned)s.tile * s.count;
    return s;
}

// Join over the four lanes l, l ^ 16, l ^ 32, l ^ 48 that hold parts of one row.
__device__ __forceinline__ float row_max(float v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum(float v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// 8 E4M3 codes as bf16 (exact).
__device__ __forceinline__ bf16x8 widen8(uint2 c)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, 1.0f, true),
                 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, 1.0f, false), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, 1.0f, true);
    const bf16x8 r = {a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
    return r;
}

// The softmax of 16 rows over part of the context, as a wave holds it: lane l has row l % 16; o[t] are channels 16 t + 4 (l / 16) ..
// + 3 of it.
template <int D>
struct RowState {
    float m, l;
    f32x4 o[D / 16];
};

// At most N of the loads that this wave has asked for are still on their way.
template <int N>
__device__ __forceinline__ void wait_loads()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A block of 64 tokens of the cache on its way through a wave.  Keys and values come in units of 4 KiB (2 KiB for 8 bits and D = 64), first
// those of the keys: all channels of 16 or 32 tokens, then those of the values: all tokens of 32 or 64 channels.  A unit goes from memory
// into one of the wave's four places in LDS directly, 1 KiB by each load, and every load takes cache lines whole.  (A fragment takes 64
// bytes of each of its 16 rows, of a token's key or a channel's values: loaded into registers as the products take them, that is half of
// a line at a time.  32 requests of 4096 tokens with 4 key heads: 59.9 us so, 54.5 through LDS; 64 of 6000 with 8: 266 and 249.)
// The loads carry the hint that the lines are used once (without it: 60.2 and 282 us).  As soon as a unit is read, the one four behind it
// is asked for, so a wave has 16 KiB on their way (8 KiB for 8 bits and D = 64), a CU 128.
// A row of a unit, 64 to 256 bytes, has its 16-byte pieces at their place xor a few bits of the row, for the 16 rows of a fragment to lie in
// different banks.
template <int D, bool F8>
struct Step {
    static constexpr int E = F8 ? 1 : 2;                   // bytes of an element
    static constexpr int kUnit = F8 && D == 64 ? 2048 : 4096;
    static constexpr int NU = kBlock * D * E / kUnit;      // units of keys, and of values
    static constexpr int NL = kUnit / 1024;                // loads of a unit
    static constexpr int RK = D * E, RV = kBlock * E;      // bytes of a row: a token's key, a channel's values
    static constexpr int PK = RK / 16, PV = RV / 16;       // pieces of it
    static constexpr int KL = PK / 4;                      // pieces of a key that each of its four lanes takes

    int t0, id[4];                                 // first token; page numbers of the four times 16 tokens
    unsigned there;                                // which of the four have a page
    const uint8_t *values;                         // the lane's place in the first 8 or 16 channels

    static __device__ __forceinline__ int key_swizzle(int token) { return PK == 16 ? token & 15 : PK == 8 ? token & 7 : token >> 2 & 3; }
    static __device__ __forceinline__ int value_swizzle(int channel) { return PV == 8 ? channel & 7 : channel >> 2 & 3; }

    // What the table says of the pages.  Scalar loads: they are counted apart from those into LDS, and the compiler, which waits for all of
    // these before a vector load's result, need not.
    struct Pages {
        int id[4];
    };
    static __device__ __forceinline__ Pages fetch_pages(const AttnParams &p, const int32_t *pages, int t0)
    {
        Pages s;
        const auto *table = (const __attribute__((address_space(4))) int32_t *)pages;
#pragma unroll
        for (int g = 0; g < 4; ++g) s.id[g] = table[min(page_of(p, (t0 >> 4) + g), p.max_pages - 1)];
        return s;
    }
    // Takes a block on.  (Tokens without a page are read from the first one and not seen.)
    __device__ __forceinline__ void begin(const AttnParams &p, int h, int at, const Pages &pages)
    {
        const int lane = lane_id();
        t0 = at;
        there = 0u;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int known = (int)(page_of(p, (t0 >> 4) + g) < p.max_pages) & (int)((unsigned)pages.id[g] < (unsigned)p.num_pages);
            id[g] = known ? pages.id[g] : 0;
            there |= known ? 1u << g : 0u;
        }
        const int channel = lane / PV, piece = (lane % PV) ^ value_swizzle(channel), g = F8 ? piece : piece >> 1;
        const int lo = g & 1 ? id[1] : id[0], hi = g & 1 ? id[3] : id[2];
        values = (const uint8_t *)p.v + ((((size_t)(g & 2 ? hi : lo) * p.KVH + h) * D + channel) * p.page_size + place(p, g)) * E + (F8 ? 0 : (piece & 1) * 16);
    }
    // Place in its page of 16 tokens g
    __device__ __forceinline__ int place(const AttnParams &p, int g) const
    {
        const int at = (t0 >> 4) + g;
        return at * 16 - page_of(p, at) * p.page_size;
    }

    // Asks for unit n.
    __device__ __forceinline__ void load(const AttnParams &p, int h, int n, u32x4 *to) const
    {
        const int lane = lane_id();
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const uint8_t *src;
            if (n < NU) {
                const int token = (n * NL + i) * (64 / PK), row = token % 16 + lane / PK;
                src = (const uint8_t *)p.k + ((size_t)id[token / 16] * p.KVH + h) * ((size_t)p.page_size * RK) +
                      (size_t)(place(p, token / 16) * RK) + (unsigned)(row * RK + ((lane % PK) ^ key_swizzle(row)) * 16);
            } else {
                src = values + (size_t)(((n - NU) * NL + i) * (64 / PV)) * (unsigned)(p.page_size * E);
            }
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src, (__attribute__((address_space(3))) void *)(to + i * 64), 16, 0, 2);
        }
    }

    // The fragments of a unit of keys, [16 tokens][KL pieces], and of a unit of values, [16 channels][the lane's four tokens of each 16],
    // read from LDS.  (Written out together with their wait: before a read of its own the compiler would wait for all loads
    // into LDS, since it does not follow which of them has come.)
    static constexpr int NG = 4 / NU, NT = D / 16 / NU;
    static __device__ __forceinline__ unsigned lds(const void *at) { return (unsigned)(size_t)(const __attribute__((address_space(3))) void *)at; }
    static __device__ __forceinline__ void keys(const u32x4 *unit, u32x4 (&k)[NG][KL])
    {
        const int row = lane_id() & 15, q = lane_id() >> 4;
        unsigned at[KL];
#pragma unroll
        for (int j = 0; j < KL; ++j) at[j] = lds(unit) + row * RK + ((4 * j + q) ^ key_swizzle(row)) * 16;
        if constexpr (KL == 4)
            asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(k[0][0]), "=&v"(k[0][1]), "=&v"(k[0][2]), "=&v"(k[0][3]) : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]) : "memory");
        else if constexpr (KL == 2)
            asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %4 offset:%6\n\tds_read_b128 %3, %5 offset:%6\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(k[0][0]), "=&v"(k[0][1]), "=&v"(k[1][0]), "=&v"(k[1][1]) : "v"(at[0]), "v"(at[1]), "n"(16 * RK) : "memory");
        else
            asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:%3\n\ts_waitcnt lgkmcnt(0)"
                         : "=&v"(k[0][0]), "=&v"(k[1][0]) : "v"(at[0]), "n"(16 * RK) : "memory");
    }
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    typedef typename std::conditional<F8, unsigned, u32x2>::type Four;         // four tokens of a channel
    static __device__ __forceinline__ void values_of(const u32x4 *unit, Four (&v)[NT][4])
    {
        const int row = lane_id() & 15, q = lane_id() >> 4;
        unsigned at[4];
#pragma unroll
        for (int g = 0; g < 4; ++g)
            at[g] = lds(unit) + row * RV + (F8 ? (g ^ value_swizzle(row)) * 16 + q * 4 : ((2 * g + (q >> 1)) ^ value_swizzle(row)) * 16 + (q & 1) * 8);
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
            if constexpr (F8)
                asm volatile("ds_read_b32 %0, %8 offset:%12\n\tds_read_b32 %1, %9 offset:%12\n\tds_read_b32 %2, %10 offset:%12\n\tds_read_b32 %3, %11 offset:%12\n\t"
                             "ds_read_b32 %4, %8 offset:%13\n\tds_read_b32 %5, %9 offset:%13\n\tds_read_b32 %6, %10 offset:%13\n\tds_read_b32 %7, %11 offset:%13\n\t"
                             "s_waitcnt lgkmcnt(0)"
                             : "=&v"(v[t][0]), "=&v"(v[t][1]), "=&v"(v[t][2]), "=&v"(v[t][3]), "=&v"(v[t + 1][0]), "=&v"(v[t + 1][1]), "=&v"(v[t + 1][2]), "=&v"(v[t + 1][3])
                             : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(t * 16 * RV), "n"((t + 1) * 16 * RV) : "memory");
            else
                asm volatile("ds_read_b64 %0, %8 offset:%12\n\tds_read_b64 %1, %9 offset:%12\n\tds_read_b64 %2, %10 offset:%12\n\tds_read_b64 %3, %11 offset:%12\n\t"
                             "ds_read_b64 %4, %8 offset:%13\n\tds_read_b64 %5, %9 offset:%13\n\tds_read_b64 %6, %10 offset:%13\n\tds_read_b64 %7, %11 offset:%13\n\t"
                             "s_waitcnt lgkmcnt(0)"
                             : "=&v"(v[t][0]), "=&v"(v[t][1]), "=&v"(v[t][2]), "=&v"(v[t][3]), "=&v"(v[t + 1][0]), "=&v"(v[t + 1][1]), "=&v"(v[t + 1][2]), "=&v"(v[t + 1][3])
                             : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(t * 16 * RV), "n"((t + 1) * 16 * RV) : "memory");
        }
    }
};

// One block: products, softmax, and the loads four units ahead, of `next` where they are past this block's (LAST: there is no next one).
// pos: position of the lane's row (-1: no row); pmin, pmax: least and greatest position of the tile's rows.
template <int D, bool F8, bool LAST>
__device__ __forceinline__ void row_block(const AttnParams &p, int h, const Step<D, F8> &b, Step<D, F8> &next, int next_t0, typename Step<D, F8>::Pages &pages,
                                          const int32_t *row, int t2, u32x4 *const (&place)[4],
                                          const bf16x8 (&q)[D / 32], int pos, int pmin, int pmax, RowState<D> &s)
{
    typedef Step<D, F8> S;
    constexpr int NU = S::NU, NG = S::NG, NT = S::NT;
    const int t0 = b.t0, quad = lane_id() >> 4;
    const auto ahead = [&](int n) {                // the loads behind unit n
        if (n + 4 < 2 * NU) b.load(p, h, n + 4, place[n % 4]);
        else if (!LAST) next.load(p, h, n + 4 - 2 * NU, place[n % 4]);
    };
    f32x4 z[4];
    const auto first_products = [&](auto unit) {
        constexpr int n = decltype(unit)::value;
        wait_loads<S::NL * (LAST && 2 * NU - 1 - n < 3 ? 2 * NU - 1 - n : 3)>();
        if (n == 2 * NU - 4 && !LAST) next.begin(p, h, next_t0, pages);
        u32x4 k[NG][S::KL];
        S::keys(place[n % 4], k);
        ahead(n);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            f32x4 &c = z[n * NG + g];
            c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < S::KL; ++j) {
                const u32x4 u = k[g][j];
                if (F8) {
                    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(make_uint2(u.x, u.y)), q[2 * j], c, 0, 0, 0);
                    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(make_uint2(u.z, u.w)), q[2 * j + 1], c, 0, 0, 0);
                } else {
                    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u), q[j], c, 0, 0, 0);
                }
            }
        }
    };
    first_products(std::integral_constant<int, 0>());
    first_products(std::integral_constant<int, 1>());
    if constexpr (NU == 4) {
        first_products(std::integral_constant<int, 2>());
        first_products(std::integral_constant<int, 3>());
    }

    typename S::Pages after;
    if (!LAST) after = S::fetch_pages(p, row, t2);
    // Tokens that not every row of the tile sees.  A token that none sees may hold anything, also what is no number: its
    // value is replaced by zero, since zero times it would not be.
    const bool in_window = p.window == 0 || t0 > pmax - p.window || t0 + kBlock <= p.sinks;
    const bool partly = !(t0 + kBlock - 1 <= pmin && in_window && b.there == 15u);
    float x[4][4];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[g][j] = z[g][j] * p.scale2;
    typename S::Four mask[4];
    if (partly) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int ok = b.there >> g & 1u, vt = t0 + 16 * g + 4 * quad;
            unsigned bits[2] = {0u, 0u};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[g][j] = ok & seen(p, vt + j, pos, pos) ? x[g][j] : -INFINITY;
                bits[F8 ? 0 : j / 2] |= ok & seen(p, vt + j, pmin, pmax) ? (F8 ? 0xffu << (8 * j) : 0xffffu << (16 * (j & 1))) : 0u;
            }
            if constexpr (F8) mask[g] = bits[0];
            else mask[g] = {bits[0], bits[1]};
        }
    }
    float top = x[0][0];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, x[g][j]);
    const float m = fmaxf(s.m, row_max(top));
    if (__any(m > s.m)) {
        const float a = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(s.m - m);
        s.l *= a;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) s.o[t] *= a;
        s.m = m;
    }
    const float base = s.m == -INFINITY ? 0.0f : s.m;
    // bf16 weights: half a step of 2^-8 each, of either sign, beside values that are bf16 themselves
    bf16x8 w[2];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[g][j] = __builtin_amdgcn_exp2f(x[g][j] - base);
            s.l += x[g][j];
        }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16(x[2 * i][0], x[2 * i][1]), pack_bf16(x[2 * i][2], x[2 * i][3]),
                                                     pack_bf16(x[2 * i + 1][0], x[2 * i + 1][1]), pack_bf16(x[2 * i + 1][2], x[2 * i + 1][3])));

    const auto second_products = [&](auto unit) {
        constexpr int n = decltype(unit)::value;
        wait_loads<S::NL * (LAST && 2 * NU - 1 - n < 3 ? 2 * NU - 1 - n : 3)>();
        if (n == 2 * NU - 4 && !LAST) next.begin(p, h, next_t0, pages);
        typename S::Four v[NT][4];
        S::values_of(place[n % 4], v);
        ahead(n);
        if (partly) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int g = 0; g < 4; ++g) v[t][g] &= mask[g];
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f32x4 &c = s.o[(n - NU) * NT + t];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                bf16x8 u;
                if constexpr (F8) u = widen8(make_uint2(v[t][2 * i], v[t][2 * i + 1]));
                else u = __builtin_bit_cast(bf16x8, u32x4{v[t][2 * i].x, v[t][2 * i].y, v[t][2 * i + 1].x, v[t][2 * i + 1].y});
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, w[i], c, 0, 0, 0);
            }
        }
    };
    second_products(std::integral_constant<int, NU>());
    second_products(std::integral_constant<int, NU + 1>());
    if constexpr (NU == 4) {
        second_products(std::integral_constant<int, NU + 2>());
        second_products(std::integral_constant<int, NU + 3>());
    }
    if (!LAST) pages = after;
}

// The rows' queries as operand: lane l holds row l % 16; channels in the order in which a lane's key loads bring them.
template <int D, bool F8>
__device__ __forceinline__ void load_queries(const uint16_t *row, bool real, bf16x8 (&q)[D / 32])
{
    const int g = lane_id() >> 4;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const int d = F8 ? (i >> 1) * 64 + g * 16 + (i & 1) * 8 : i * 32 + g * 8;
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (real) u = *reinterpret_cast<const uint4 *>(row + d);
        q[i] = __builtin_bit_cast(bf16x8, u);
    }
}

// Finishes a row of which this lane has N runs of four channels, c0, c0 + step, ..: divides and writes.  A row that lies behind the
// prefix is left in the workspace instead, for attn_finish_kernel.
template <int D, int N>
__device__ __forceinline__ void finish_row(const AttnParams &p, int t, int head, bool behind, int c0, int step, float m, float l, const f32x4 (&o)[N])
{
    const size_t row = (size_t)t * (p.KVH * p.G) + head;
    if (behind) {
#pragma unroll
        for (int k = 0; k < N; ++k) *reinterpret_cast<f32x4 *>(p.own_o + row * D + c0 + k * step) = o[k];
        if (c0 == 0) *reinterpret_cast<float2 *>(p.own_ml + 2 * row) = make_float2(m, l);
        return;
    }
    const float inv = l == 0.0f ? 0.0f : p.v_scale / l;
    uint16_t *dst = p.out + (size_t)t * p.out_stride + (size_t)head * D + c0;
#pragma unroll
    for (int k = 0; k < N; ++k)
        *reinterpret_cast<uint2 *>(dst + k * step) = make_uint2(pack_bf16(o[k][0] * inv, o[k][1] * inv), pack_bf16(o[k][2] * inv, o[k][3] * inv));
    if (p.lse && c0 == 0) p.lse[row] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// Where the line is cut behind a workgroup's length: the tile that goes on there, if this is the first cut through it.
struct alignas(16) Cut {
    int first, n, seq, tile;
    unsigned begin, count, length, mine;
};

// A length of the line of one key head per workgroup, a quarter of it per wave.  A wave goes through its quarter tile by tile.
// A tile that lies in it whole is finished in its registers; of the first and the last, which in general do not, it leaves its part in
// LDS, and when all waves are through, the parts of each tile are joined: to the finished rows, or to a part in the workspace if
// the tile goes on in another workgroup.  (With all four waves on one tile after the other, each with its round trips for lengths,
// queries and page numbers, 256 requests with an 8-bit cache took 137 us where this took 118.)
// Bound by HBM: 64 requests of 500 to 12000 tokens, 411 MB: 72 us, 5.7 TB/s; 256 with 657 MB of 8-bit cache: 127 us, 5.2 TB/s; a plain
// read of such pages reaches 6.0, with the hint 6.6.  One request of 9001 tokens: 12.0 us, four dependent trips to memory.  (Medians of
// a kernel trace, as all times of whole kernels here.)
constexpr int kRecords = 2 * kAttnWaves;
struct RowsShared {
    Line line;
    unsigned rec[kRecords];                         // begin of the tile that the part belongs to
    float sm[kRecords][kRows], sl[kRecords][kRows];
};
// part(k): 16 rows of D floats of LDS.
template <int D, bool F8, typename Parts>
__device__ __forceinline__ void rows_of(const AttnParams &p, unsigned x, int h, RowsShared &sh, u32x4 *const (&units)[4], const Parts &part_of)
{
    typedef Step<D, F8> S;
    constexpr unsigned kNone = 0xffffffffu;
    Line &line = sh.line;
    unsigned(&rec)[kRecords] = sh.rec;
    float(&sm)[kRecords][kRows] = sh.sm;
    float(&sl)[kRecords][kRows] = sh.sl;
    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    const unsigned total = lay_out(p, line), length = length_of(p, total);
    const unsigned from = min(x * length, total), to = min(from + length, total);
    // (four channels of a row stand at their place xor the row: the lanes that write have one place of all 16 rows)
    const auto place = [&](int k, int row, int c) -> f32x4 & { return *reinterpret_cast<f32x4 *>(part_of(k) + row * D + (c / 4 ^ row) * 4); };
    if (p.prefix_blocks == 0 && h == 0 && wv == kAttnWaves - 1) {         // (behind a prefix attn_finish_kernel finds them)
        const unsigned cut = (x + 1) * length;
        Cut c = {};
        if (cut < total) {
            const Place f = place_of(p, line, cut);
            c = {f.first, f.n, f.seq, f.tile, f.begin, f.count, length, f.begin != cut && f.begin + length >= cut ? 1u : 0u};
        }
        if (lane == 0) p.cuts[x] = c;
    }
    if (from >= to) return;
    if (lane < 2) rec[2 * wv + lane] = kNone;
    const unsigned quarter = (length + kAttnWaves - 1) / kAttnWaves;
    const unsigned wfrom = min(from + wv * quarter, to), wto = min(wfrom + quarter, to);
    RowState<D> s, left;           // left: of the first tile, where its part goes to LDS in the end (until then loads go there)
    int last = 0;                  // whether s at the end is such a part too
    for (unsigned at = wfrom; at < wto;) {
        const Place f = place_of(p, line, at);
        const unsigned i0 = at - f.begin, i1 = min(f.count, wto - f.begin);
        at = f.begin + i1;

        const int r = f.tile * kRows + (lane & 15), rows = f.n * p.G;
        const bool real = r < rows;
        const int tok = real ? token_of(p, r) : 0, head = h * p.G + (real ? r - tok * p.G : 0);
        const int pos = real ? f.seq - f.n + tok : -1;
        const int pmin = max(f.seq - f.n + token_of(p, f.tile * kRows), 0), pmax = f.seq - f.n + token_of(p, min(f.tile * kRows + kRows, rows) - 1);
        bf16x8 q[D / 32];
        load_queries<D, F8>(p.q + (size_t)(f.first + tok) * p.q_stride + (size_t)head * D, real, q);
        s.m = -INFINITY;
        s.l = 0.0f;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) s.o[t] = {0.0f, 0.0f, 0.0f, 0.0f};

        // (tiles of one request lie on the line with as many blocks each: those past a tile's own are passed over)
        const Blocks blocks = blocks_of(p, f.seq - f.n, pmin, pmax);
        const int j0 = (int)min(i0, (unsigned)blocks.count), j1 = (int)min(i1, (unsigned)blocks.count);
        const int32_t *row = p.table + (size_t)f.b * p.max_pages;
        const auto token = [&](int j) { return blocks.at(min(j, j1 - 1)) * kBlock; };
        if (j0 < j1) {
            S b, next;
            typename S::Pages pages = S::fetch_pages(p, row, token(j0));
            b.begin(p, h, token(j0), pages);
            pages = S::fetch_pages(p, row, token(j0 + 1));
            // the queries are there: waited for behind the loads into LDS, they would be waited for with all of those
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0x0f70);     // vmcnt(0)
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < 4; ++n) b.load(p, h, n, units[n]);
            for (int j = j0; j + 1 < j1; ++j) {
                row_block<D, F8, false>(p, h, b, next, token(j + 1), pages, row, token(j + 2), units, q, pos, pmin, pmax, s);
                b = next;
            }
            row_block<D, F8, true>(p, h, b, next, 0, pages, row, 0, units, q, pos, pmin, pmax, s);
        }
        s.l = row_sum(s.l);
        if (i0 == 0 && i1 == f.count) {
            if (real) finish_row<D>(p, f.first + tok, head, behind_prefix(p, f.seq - f.n), (lane >> 4) * 4, 16, s.m, s.l, s.o);
        } else {
            last = at == wto && i0 == 0;            // the wave's last tile, or its first
            if (lane == 0) rec[2 * wv + last] = f.begin;
            if (!last) left = s;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int k = 2 * wv + i;
        if (rec[k] == kNone) continue;
        const RowState<D> &part = i == 0 ? left : s;
        if (lane < kRows) {
            sm[k][lane] = part.m;
            sl[k][lane] = part.l;
        }
#pragma unroll
        for (int t = 0; t < D / 16; ++t) place(k, lane & 15, t * 16 + (lane >> 4) * 4) = part.o[t];
    }
    __syncthreads();
    // The parts in LDS, in the order of the line: those of one tile follow one another.  16 threads per row, D / 16 channels each.
    const int recs = (int)rec[lane % kRecords];
    const auto tile_of = [&](int k) { return (unsigned)__builtin_amdgcn_readlane(recs, k); };
    const int orow = threadIdx.x / kRows, c0 = threadIdx.x % kRows * (D / 16);
    for (int k = 0; k < kRecords;) {
        const unsigned begin = tile_of(k);
        int end = k + 1;
        while (end < kRecords && (tile_of(end) == begin || tile_of(end) == kNone)) ++end;
        if (begin == kNone) {
            ++k;
            continue;
        }
        const Place f = place_of(p, line, begin);
        const int ro = f.tile * kRows + orow;
        if (ro < f.n * p.G) {
            float m = -INFINITY;
            for (int w = k; w < end; ++w)
                if (tile_of(w) == begin) m = fmaxf(m, sm[w][orow]);
            float l = 0.0f;
            f32x4 o[D / 64];
#pragma unroll
            for (int i = 0; i < D / 64; ++i) o[i] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int w = k; w < end; ++w) {
                if (tile_of(w) != begin) continue;
                const float e = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm[w][orow] - m);
                l += e * sl[w][orow];
#pragma unroll
                for (int i = 0; i < D / 64; ++i) o[i] += place(w, orow, c0 + 4 * i) * e;
            }
            if (begin >= from && begin + f.count <= to) {
                const int tok = token_of(p, ro);
                finish_row<D>(p, f.first + tok, h * p.G + ro - tok * p.G, behind_prefix(p, f.seq - f.n), c0, 4, m, l, o);
            } else {
                // (a workgroup cuts two tiles at most: the one it begins inside, and the one it ends in)
                const size_t part = ((size_t)(2 * x + (begin >= from ? 1 : 0)) * p.KVH + h) * kRows + orow;
#pragma unroll
                for (int i = 0; i < D / 64; ++i) *reinterpret_cast<f32x4 *>(p.part_o + part * D + c0 + 4 * i) = o[i];
                if (c0 == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * part) = make_float2(m, l);
            }
        }
        k = end;
    }
}

// Joins the parts of the tiles that are cut (4 to 5 us: a launch, two trips to memory).  Workgroup x has the x-th cut of the line; where it is the first that goes through a
// tile, it joins the tile.  Few rows with many parts each are the case that counts (one request alone: a few rows, dozens of
// parts), so the parts of a row are spread over what the rows leave of the workgroup's D / 4-lane groups, which meet in LDS.
template <int D>
__device__ __forceinline__ void join_rows(const AttnParams &p, unsigned cut_index, int h)
{
    constexpr int L = D / 4, NG = kAttnThreads / L;         // lanes of a group (4 channels each), groups
    __shared__ float sm[NG], sl[NG];
    __shared__ __align__(16) float4 so[NG][L];
    const Cut f = p.cuts[cut_index];
    if (!f.mine) return;
    const unsigned length = f.length;
    const int here = min(f.n * p.G - f.tile * kRows, kRows);
    const int parts = (int)((f.begin + f.count - 1) / length) - (int)cut_index + 1;
    const int grp = threadIdx.x / L, lane = threadIdx.x % L;
    for (int done = 0; done < here; done += NG) {
        int width = 1;                                              // rows at a time: a power of two
        while (width < here - done && width < NG) width *= 2;
        const int orow = done + grp % width, sub = grp / width;
        const bool real = orow < here;
        float m = -INFINITY, l = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int i = sub; i < parts; i += NG / width) {
            // the first part is the last of its workgroup unless the tile begins where the workgroup does
            const unsigned x = cut_index + i;
            const size_t part = ((size_t)(2 * x + (f.begin >= x * length ? 1 : 0)) * p.KVH + h) * kRows + (real ? orow : 0);
            const float2 ml = *reinterpret_cast<const float2 *>(p.part_ml + 2 * part);
            const f32x4 u = *reinterpret_cast<const f32x4 *>(p.part_o + part * D + 4 * lane);
            const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.0f : top;
            const float a = __builtin_amdgcn_exp2f(m - base), e = __builtin_amdgcn_exp2f(ml.x - base);
            l = l * a + e * ml.y;
            o = o * a + u * e;
            m = top;
        }
        if (width < NG) {
            if (lane == 0) {
                sm[grp] = m;
                sl[grp] = l;
            }
            so[grp][lane] = make_float4(o[0], o[1], o[2], o[3]);
            __syncthreads();
            for (int w = grp + width; sub == 0 && w < NG; w += width) {
                const float4 u = so[w][lane];
                const float top = fmaxf(m, sm[w]), base = top == -INFINITY ? 0.0f : top;
                const float a = __builtin_amdgcn_exp2f(m - base), e = __builtin_amdgcn_exp2f(sm[w] - base);
                l = l * a + e * sl[w];
                o = o * a + f32x4{u.x, u.y, u.z, u.w} * e;
                m = top;
            }
            __syncthreads();
        }
        if (sub != 0 || !real) continue;
        const int ro = f.tile * kRows + orow, tok = token_of(p, ro);
        f32x4 own[1] = {o};
        finish_row<D>(p, f.first + tok, h * p.G + ro - tok * p.G, behind_prefix(p, f.seq - f.n), 4 * lane, 4, m, l, own);
    }
}

// ---- many rows ------------------------------------------------------------------------------------------------------------
// Tiles of 128 rows, 32 to a wave, on v_mfma_f32_32x32x16_bf16: a block of 64 tokens is brought into LDS once for the four waves, in
// two buffers, and every fragment that a wave reads there serves 32 rows.  The same transposed products as above: a lane has row
// l % 32, and a result fragment of S^T gives it 16 tokens of a block's half; the keys lie in LDS in such an order that they are two
// runs of 8 consecutive tokens, the operand of the second product.
// What it does: per block and wave 32 matrix instructions (1024 cycles; D = 64: 512), 32 KiB from LDS (four waves: 1024 cycles of its
// 128 bytes each) and about 900 VALU cycles for 32 weights per lane, 512 of them exponentials; two workgroups a CU, so that one's
// softmax can stand beside the other's products.  Five prompt chunks of 700 to 2048 tokens, 236 GFLOP: 294 us, 804 TFLOP/s (265 us, 890, where
// no profiler runs).  None of the three is full, matrix cores, VALU and LDS 46 % each: the two workgroups mostly take turns, and in the second
// copy of the loop's turn the compiler has most exponentials in front of the last products.  With D = 64 (40 requests, 22 GFLOP: 75 us;
// VALU 48 %, matrix cores 19 %) tiles are short, 6.5 blocks behind a start of 4 us, and are dealt out in the requests' order, so that a long one may
// begin last.
constexpr int kWaveRows = 32;
constexpr int kLdsAlign = 16384, kBuffer = kLdsAlign / 16;      // bytes and 16-byte pieces of each of the four buffers in LDS
// Blocks: what a request's first and last row see together is not cut into shorter parts (one request of 3000 tokens, 100 of them new: 33.0 us,
// with 4 34.7, with 16 39.3).  Of a long prompt with a short window a tile sees less than that, and its parts are shorter.
constexpr int kMinChunk = 8;
typedef float f32x16 __attribute__((ext_vector_type(16)));

// The contexts of all tiles are cut into parts of at most `chunk` blocks, chunk following from the work of the whole batch, so that a
// few tiles with long contexts fill the chip.  The parts of a request's last tile, the longest, come first.
struct FindShared {
    float work[kAttnWaves];
    int sum[2][kAttnWaves];
    int found[6];
};
struct Part {
    int b, tile, split, splits, item;       // item: index of the tile's first part among those of all tiles that are cut
};
// CUT: x counts the tiles that are cut, otherwise the parts of all tiles.
template <bool CUT>
__device__ __forceinline__ bool find_part(const AttnParams &p, int x, FindShared &sh, Part &f)
{
    const int lane = lane_id(), wv = wave_id();
    const int per = (p.B + kAttnThreads - 1) / kAttnThreads, b0 = threadIdx.x * per;
    int tiles[kMaxPerThread], blocks[kMaxPerThread];
    float work = 0.0f;
#pragma unroll
    for (int i = 0; i < kMaxPerThread; ++i) {
        tiles[i] = blocks[i] = 0;
        if (i < per && b0 + i < p.B) {
            int first, n, seq;
            request_of(p, b0 + i, first, n, seq);
            tiles[i] = n * p.G > p.narrow ? (n * p.G + kTileRows - 1) / kTileRows : 0;
            blocks[i] = blocks_of(p, seq - n, max(seq - n, 0), seq - 1).count;
            work += (float)tiles[i] * (float)blocks[i];
        }
    }
    work = wave_sum(work);
    if (threadIdx.x == 0) sh.found[0] = -1;
    if (lane == 0) sh.work[wv] = work;
    __syncthreads();
    work = 0.0f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) work += sh.work[w];
    // (a little more than the quotient: the sum is rounded, and there are no more than p.wide_parts + tiles workgroups)
    const int chunk = max(kMinChunk, (int)fminf(work * 1.0001f / (float)p.wide_parts, 1e9f) + 1);
    int nx = 0, nc = 0;
#pragma unroll
    for (int i = 0; i < kMaxPerThread; ++i) {
        blocks[i] = max((blocks[i] + chunk - 1) / chunk, 1);      // parts of each of its tiles
        nx += CUT ? (blocks[i] > 1 ? tiles[i] : 0) : tiles[i] * blocks[i];
        nc += blocks[i] > 1 ? tiles[i] * blocks[i] : 0;
    }
    int sx = wave_prefix_sum_i32(nx), sc = wave_prefix_sum_i32(nc);
    if (lane == kWave - 1) {
        sh.sum[0][wv] = sx;
        sh.sum[1][wv] = sc;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
        sx += w < wv ? sh.sum[0][w] : 0;
        sc += w < wv ? sh.sum[1][w] : 0;
    }
    sx -= nx;
    sc -= nc;
#pragma unroll
    for (int i = 0; i < kMaxPerThread; ++i) {
        const int items = CUT ? (blocks[i] > 1 ? tiles[i] : 0) : tiles[i] * blocks[i], at = x - sx;
        if (at >= 0 && at < items) {
            const int k = CUT ? at : at / blocks[i];
            sh.found[1] = tiles[i] - 1 - k;
            sh.found[2] = CUT ? 0 : at - k * blocks[i];
            sh.found[3] = blocks[i];
            sh.found[4] = sc + k * blocks[i];
            sh.found[0] = b0 + i;
        }
        sx += items;
        sc += blocks[i] > 1 ? tiles[i] * blocks[i] : 0;
    }
    __syncthreads();
    f.b = __builtin_amdgcn_readfirstlane(sh.found[0]);
    f.tile = __builtin_amdgcn_readfirstlane(sh.found[1]);
    f.split = __builtin_amdgcn_readfirstlane(sh.found[2]);
    f.splits = __builtin_amdgcn_readfirstlane(sh.found[3]);
    f.item = __builtin_amdgcn_readfirstlane(sh.found[4]);
    return f.b >= 0;
}

__device__ __forceinline__ float half_max(float v)
{
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float half_sum(float v)
{
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// A block of 64 tokens on its way from the pages into LDS, 16 bytes per load and lane.  Each of the block's four groups of 16 tokens lies
// in one page; what one load instruction brings is of one group, so that its address is a scalar and a constant of the lane.
//   keys [64][D]: row m holds token 16 (m / 16) + (m % 16 with bits 2 and 3 exchanged): the lane's scores are then of consecutive tokens; the 16-byte pieces of
//   a row stand at their place xor (m & 7);
//   values [4 groups][D][2 pieces]: wave w brings group w; the two pieces of a channel change places where bit 2 of it is set.
// (The lanes of a fragment read one column of pieces, which would all lie in the same banks.)
// A bf16 block goes from memory to LDS directly; an 8-bit one is widened in registers on its way.
template <int D, bool F8>
struct BlockLoad {
    static constexpr int E = F8 ? 1 : 2;
    static constexpr int KP = D * E / 16;                                // loads of a key row
    static constexpr int KI = kBlock * KP / kAttnThreads;
    static constexpr int VP = E;                                         // loads of a group of one channel
    static constexpr int VI = D * VP / kWave;
    u32x4 kw[F8 ? KI : 1], vw[F8 ? VI : 1];
    unsigned koff, voff;          // the lane's places in a group of keys and of values (bytes)
    int kput, vput;               // and, of an 8-bit block, in LDS (16-byte pieces)

    __device__ __forceinline__ BlockLoad(const AttnParams &p)
    {
        const int tid = threadIdx.x, lane = lane_id();
        const int m = tid / KP, r = m & 15, tok = (r & 3) | (r & 4) << 1 | (r & 8) >> 1, d = lane / VP, swap = d >> 2 & 1;
        koff = (unsigned)(tok * (D * E) + (F8 ? tid % KP : (tid % KP) ^ (m & 7)) * 16);
        voff = (unsigned)(d * p.page_size + (F8 ? 0 : ((lane & 1) ^ swap) * 8)) * E;
        kput = m * (D / 8) + ((2 * (tid % KP)) ^ (m & 7));
        vput = (wave_id() * D + d) * 2 + swap;
    }

    // Lane l: what the table says of the page of the block's l % 4th 16 tokens, and whether there is such a page.  (Apart, for the
    // number to be on its way until it is used.)
    static __device__ __forceinline__ int fetch_pages(const AttnParams &p, const int32_t *pages, int blk)
    {
        return pages[min(page_of(p, blk * (kBlock / 16) + (lane_id() & 3)), p.max_pages - 1)];
    }
    static __device__ __forceinline__ unsigned there(const AttnParams &p, int blk, int id)      // bit g: group g has a page
    {
        return (unsigned)__ballot(page_of(p, blk * (kBlock / 16) + (lane_id() & 3)) < p.max_pages && (unsigned)id < (unsigned)p.num_pages) & 15u;
    }

    // Where group g of the block begins in the keys or values of head h.  (Tokens without a page are read from the first one.)
    static __device__ __forceinline__ const uint8_t *group(const AttnParams &p, const void *cache, int token_bytes, int h, int blk, int ids, int g)
    {
        const int id = __builtin_amdgcn_readlane(ids, g), at = blk * (kBlock / 16) + g, place = at * 16 - page_of(p, at) * p.page_size;
        return (const uint8_t *)cache + ((size_t)((unsigned)id < (unsigned)p.num_pages ? id : 0) * p.KVH + h) * ((size_t)p.page_size * D * E) +
               (size_t)(place * token_bytes);
    }
    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t resource(const uint8_t *base)
    {
        const unsigned long long a = reinterpret_cast<unsigned long long>(base);
        const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)a), hi = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));
        return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(((unsigned long long)hi << 32) | lo), 0, 0x7fffffff, 0x00020000);
    }

    __device__ __forceinline__ void keys(const AttnParams &p, int h, int wv, int blk, int ids, u32x4 *kb)
    {
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            const uint8_t *src = group(p, p.k, D * E, h, blk, ids, (i * kAttnThreads + wv * kWave) / (16 * KP));
            if constexpr (F8) kw[i] = *reinterpret_cast<const u32x4 *>(src + koff);
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(resource(src), (__attribute__((address_space(3))) void *)(kb + i * kAttnThreads + wv * kWave), 16, koff, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void values(const AttnParams &p, int h, int wv, int blk, int ids, u32x4 *vb)
    {
        const uint8_t *src = group(p, p.v, E, h, blk, ids, wv);
        const __amdgpu_buffer_rsrc_t rs = resource(src);
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            const int next = i * (kWave / VP) * p.page_size * E;
            if constexpr (F8) vw[i] = *reinterpret_cast<const u32x4 *>(src + next + voff);
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(vb + wv * D * 2 + i * kWave), 16, voff, next, 0, 0);
        }
    }

    // The lane's values that no row of the tile sees (they may be no numbers) as a mask of zeros.
    __device__ __forceinline__ u32x4 hidden(const AttnParams &p, int wv, int blk, unsigned there, int pmin, int pmax) const
    {
        const int t0 = blk * kBlock + 16 * wv + (F8 ? 0 : (int)((lane_id() & 1) ^ (lane_id() >> 3 & 1)) * 8);
        u32x4 mask;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            mask[w] = 0u;
#pragma unroll
            for (int i = 0; i < 4 / E; ++i)
                mask[w] |= (int)(there >> wv & 1u) & seen(p, t0 + w * (4 / E) + i, pmin, pmax) ? (F8 ? 0xffu << (8 * i) : 0xffffu << (16 * i)) : 0u;
        }
        return mask;
    }

    __device__ __forceinline__ void put_keys(u32x4 *kb) const
    {
#pragma unroll
        for (int i = 0; i < KI; ++i) {
            kb[kput + i * (kAttnThreads / KP) * (D / 8)] = __builtin_bit_cast(u32x4, widen8(make_uint2(kw[i].x, kw[i].y)));
            kb[(kput ^ 1) + i * (kAttnThreads / KP) * (D / 8)] = __builtin_bit_cast(u32x4, widen8(make_uint2(kw[i].z, kw[i].w)));
        }
    }
    __device__ __forceinline__ void put_values(u32x4 *vb) const
    {
#pragma unroll
        for (int i = 0; i < VI; ++i) {
            vb[vput + i * kWave * 2] = __builtin_bit_cast(u32x4, widen8(make_uint2(vw[i].x, vw[i].y)));
            vb[(vput ^ 1) + i * kWave * 2] = __builtin_bit_cast(u32x4, widen8(make_uint2(vw[i].z, vw[i].w)));
        }
    }
};

// Everything that this wave has asked for has come, and every wave is here: what the waves brought into LDS is there for all.  (Written
// out, since a load into LDS is no write that a barrier would wait for.)
__device__ __forceinline__ void blocks_ready()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Workgroups go round the eight XCDs, each with an L2 of its own, and the key heads go round fastest: the tiles of one head, which read
// the same keys and values, meet in few L2s (five prompt chunks with 8 key heads: 378 us with the heads slowest, 299 so).
// A turn of the loop has the second product of one block and the first of the next, whose matrix instructions stand between the VALU
// instructions of the softmax.  In LDS at a turn's start: its values and the next keys; on their way during it: the next values and
// the keys after next.
// prefix: the rows are those of the whole batch, whatever request they belong to, and the context is the shared prefix's whole blocks,
// which all of them see; every row's part is left in the workspace.
template <int D, bool F8>
__device__ __forceinline__ void tile_of(const AttnParams &p, bool prefix, int x, int h, u32x4 (&kbuf0)[kBuffer], u32x4 (&vbuf0)[kBuffer],
                                        u32x4 (&kbuf1)[kBuffer], u32x4 (&vbuf1)[kBuffer])
{
    typedef BlockLoad<D, F8> B;
    constexpr int NQ = D / 16, NV = D / 32, kAhead = 4;     // fragments are read from LDS four products ahead
    static_assert(sizeof(FindShared) <= sizeof kbuf0, "LDS");
    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id());
    constexpr int kFar = 1 << 30;                   // behind every token of a prefix
    Part f;
    int first, n, seq;
    if (prefix) {
        f = {0, x / p.prefix_splits, x % p.prefix_splits, p.prefix_splits, 0};
        first = 0;
        n = p.T;
        seq = kFar + p.T;
    } else {
        if (!find_part<false>(p, x, *reinterpret_cast<FindShared *>(kbuf0), f)) return;
        request_of(p, f.b, first, n, seq);
        __syncthreads();                            // kbuf0 is free again
    }
    const int rows = n * p.G, base = seq - n, r0 = f.tile * kTileRows + wv * kWaveRows, r = r0 + (lane & 31), hf = lane >> 5;
    const bool real = r < rows;
    const int tok = real ? token_of(p, r) : 0, head = h * p.G + (real ? r - tok * p.G : 0);
    const int pos = real ? base + tok : -1;
    const int tmin = max(base + token_of(p, f.tile * kTileRows), 0), tmax = base + token_of(p, min(f.tile * kTileRows + kTileRows, rows) - 1);
    const int pmin = max(base + token_of(p, r0), 0), pmax = r0 < rows ? base + token_of(p, min(r0 + kWaveRows, rows) - 1) : -1;    // of the wave's rows
    const Blocks blocks = prefix ? Blocks{0, 0, p.prefix_blocks} : blocks_of(p, base, tmin, tmax);
    const int per = (blocks.count + f.splits - 1) / f.splits, i0 = f.split * per, i1 = min(i0 + per, blocks.count);
    const int32_t *pages = prefix ? p.prefix_table : p.table + (size_t)f.b * p.max_pages;
    const auto block = [&](int i) { return blocks.at(min(i, i1 - 1)); };

    B load(p);
    int id1 = 0, id2 = 0, id3 = 0;                  // page numbers of the next blocks
    unsigned there = 15u;                           // which groups of this turn's block have a page
    if (i0 < i1) {
        const int id0 = B::fetch_pages(p, pages, block(i0));
        id1 = B::fetch_pages(p, pages, block(i0 + 1));
        id2 = B::fetch_pages(p, pages, block(i0 + 2));
        if (F8) id3 = B::fetch_pages(p, pages, block(i0 + 3));
        there = B::there(p, block(i0), id0);
        load.keys(p, h, wv, block(i0), id0, kbuf0);
        load.values(p, h, wv, block(i0), id0, vbuf0);
    }
    bf16x8 q[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        u32x4 u = {0u, 0u, 0u, 0u};
        if (real) u = *reinterpret_cast<const u32x4 *>(p.q + (size_t)(first + tok) * p.q_stride + (size_t)head * D + i * 16 + hf * 8);
        q[i] = __builtin_bit_cast(bf16x8, u);
    }
    float m = -INFINITY, l = 0.0f;                  // (m: of the scores themselves)
    constexpr float kFarScore = 1048576.0f;
    bool far = false;                               // whether a row's maximum is beyond it
    f32x16 o[NV];
#pragma unroll
    for (int t = 0; t < NV; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;

    const int krow = (lane & 31) * (D / 8), vrow = (lane & 31) * 2 + (hf ^ (lane >> 2 & 1));
    const auto key = [&](const u32x4 *kb, int i) {      // fragment i of the 2 NQ, of 32 tokens' keys after the other
        return __builtin_bit_cast(bf16x8, kb[i / NQ * 32 * (D / 8) + krow + ((2 * (i % NQ) + hf) ^ (lane & 7))]);
    };
    const auto value = [&](const u32x4 *vb, int i) {     // fragment i of the 4 NV: 16 tokens after 16 tokens
        return __builtin_bit_cast(bf16x8, vb[(i / NV * D + i % NV * 32) * 2 + vrow]);
    };
    const auto partly = [&](int blk, unsigned t) {        // some of the block's tokens are seen by no row of the tile
        const int t0 = blk * kBlock;
        return t != 15u || t0 + kBlock - 1 > tmax || (p.window != 0 && t0 <= tmin - p.window && t0 + kBlock > p.sinks);
    };
    f32x16 za[2], zb[2];
    if (i0 < i1) {
        if constexpr (F8) {
            if (partly(block(i0), there)) {
                const u32x4 mask = load.hidden(p, wv, block(i0), there, tmin, tmax);
#pragma unroll
                for (int i = 0; i < B::VI; ++i) load.vw[i] &= mask;
            }
            load.put_keys(kbuf0);
            load.put_values(vbuf0);
            load.keys(p, h, wv, block(i0 + 1), id1, kbuf1);
            load.put_keys(kbuf1);
            load.values(p, h, wv, block(i0 + 1), id1, vbuf1);
            load.keys(p, h, wv, block(i0 + 2), id2, kbuf0);
        } else {
            load.keys(p, h, wv, block(i0 + 1), id1, kbuf1);
        }
        blocks_ready();
        bf16x8 ka[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) ka[i] = key(kbuf0, i);
#pragma unroll
        for (int i = 0; i < 16; ++i) za[0][i] = za[1][i] = 0.0f;
#pragma unroll
        for (int i = 0; i < 2 * NQ; ++i) {
            const bf16x8 a = ka[i % kAhead];
            if (i + kAhead < 2 * NQ) ka[i % kAhead] = key(kbuf0, i + kAhead);
            za[i / NQ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[i % NQ], za[i / NQ], 0, 0, 0);
        }
    }
    // kn, vn: this turn's keys, whose buffer is free, and values; kx, vx: the next ones'
    const auto turn = [&](int i, u32x4 *kn, u32x4 *vn, u32x4 *kx, u32x4 *vx, f32x16 (&z)[2], f32x16 (&zn)[2]) {
        const int blk = block(i), t0 = blk * kBlock, blk1 = block(i + 1), blk2 = block(i + 2);
        const unsigned there1 = B::there(p, blk1, id1);
        blocks_ready();
        if constexpr (F8) {
            if (partly(blk1, there1)) {
                const u32x4 mask = load.hidden(p, wv, blk1, there1, tmin, tmax);
#pragma unroll
                for (int j = 0; j < B::VI; ++j) load.vw[j] &= mask;
            }
            load.put_values(vx);
            load.put_keys(kn);
            load.values(p, h, wv, blk2, id2, vn);
            load.keys(p, h, wv, block(i + 3), id3, kx);
            id1 = id2;
            id2 = id3;
            id3 = B::fetch_pages(p, pages, block(i + 4));
        } else {
            if (partly(blk, there)) {
                const u32x4 mask = load.hidden(p, wv, blk, there, tmin, tmax);
#pragma unroll
                for (int j = 0; j < B::VI; ++j) vn[wv * D * 2 + j * kWave + lane] &= mask;
                blocks_ready();
            }
            load.values(p, h, wv, blk1, id1, vx);
            load.keys(p, h, wv, blk2, id2, kn);
            id1 = id2;
            id2 = B::fetch_pages(p, pages, block(i + 3));
        }
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 ka[kAhead], va[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) ka[j] = key(kx, j);
        // lane: tokens t0 + 32 t + 16 (j / 8) + 8 hf + j % 8
        const bool in_window = p.window == 0 || t0 > pmax - p.window || t0 + kBlock <= p.sinks;
        if (!(t0 + kBlock - 1 <= pmin && in_window && there == 15u)) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const unsigned ok = there >> (2 * t + s) & 1u;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int at = t0 + 32 * t + 16 * s + 8 * hf + j;
                        z[t][s * 8 + j] = (int)ok & seen(p, at, pos, pos) ? z[t][s * 8 + j] : -INFINITY;
                    }
                }
        }
        there = there1;
#pragma unroll
        for (int j = 0; j < 16; ++j) zn[0][j] = zn[1][j] = 0.0f;
        const auto first_product = [&](int j) {
            const bf16x8 a = ka[j % kAhead];
            if (j + kAhead < 2 * NQ) ka[j % kAhead] = key(kx, j + kAhead);
            zn[j / NQ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[j % NQ], zn[j / NQ], 0, 0, 0);
        };
        constexpr int kBefore = NQ / 2;         // products beside the maximum
        float top = z[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, z[t][j]);
#pragma unroll
        for (int j = 0; j < kBefore; ++j) first_product(j);
        top = half_max(top);
        // m follows the maximum only when it is 8 behind, times the scale: until then weights are up to 2^8, and rows are rescaled less often
        if (__any(top > m + p.lag)) {
            const float up = fmaxf(m, top), a = up == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m - up) * p.scale2);
            l *= a;
#pragma unroll
            for (int t = 0; t < NV; ++t) o[t] *= a;
            m = up;
            far = __any(m != -INFINITY && fabsf(m * p.scale2) > kFarScore);
        }
        // 2^(z scale - m scale) by one multiply-add.  The product with m is rounded, which moves all weights of a row by as much; where that could be
        // by more than 2^(1/32), and with larger scores out of range, m is taken off the scores first.
        float off = m == -INFINITY ? 0.0f : -m * p.scale2;
        if (far) {
            const float by = fabsf(off) > kFarScore ? m : 0.0f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) z[t][j] -= by;
            off = by == 0.0f ? off : 0.0f;
        }
#pragma unroll
        for (int j = kBefore; j < 2 * NQ; ++j) first_product(j);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) va[j] = value(vn, j);
        bf16x8 w[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[s / 2][s % 2 * 8 + j], p.scale2, off));
                l += e[j];
            }
            w[s] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16(e[0], e[1]), pack_bf16(e[2], e[3]), pack_bf16(e[4], e[5]), pack_bf16(e[6], e[7])));
        }
#pragma unroll
        for (int j = 0; j < 4 * NV; ++j) {
            const bf16x8 a = va[j % kAhead];
            if (j + kAhead < 4 * NV) va[j % kAhead] = value(vn, j + kAhead);
            o[j % NV] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, w[j / NV], o[j % NV], 0, 0, 0);
        }
    };
    for (int i = i0; i < i1; i += 2) {
        turn(i, kbuf0, vbuf0, kbuf1, vbuf1, za, zb);
        if (i + 1 < i1) turn(i + 1, kbuf1, vbuf1, kbuf0, vbuf0, zb, za);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // nothing on its way into LDS when the workgroup ends
    l = half_sum(l);
    m *= p.scale2;
    if (!real) return;
    // lane: channels 32 t + 8 j + 4 hf .. + 3 of its row
    f32x4 c[D / 8];
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) c[4 * t + j] = {o[t][4 * j], o[t][4 * j + 1], o[t][4 * j + 2], o[t][4 * j + 3]};
    if (!prefix && f.splits == 1) {
        finish_row<D>(p, first + tok, head, behind_prefix(p, base), hf * 4, 8, m, l, c);
    } else {
        const size_t part = ((size_t)(prefix ? f.tile * f.splits + f.split : f.item + f.split) * p.KVH + h) * kTileRows + (r - f.tile * kTileRows);
        float *dst = (prefix ? p.prefix_o : p.wide_o) + part * D + hf * 4;
#pragma unroll
        for (int k = 0; k < D / 8; ++k) *reinterpret_cast<f32x4 *>(dst + k * 8) = c[k];
        if (hf == 0) *reinterpret_cast<float2 *>((prefix ? p.prefix_ml : p.wide_ml) + 2 * part) = make_float2(m, l);
    }
}

// One launch for all of a call: the prefix's tiles, the tiles of requests of many rows, and the line of the others, whose reading of the
// cache stands beside the tiles' products (three launches one after the other: prefix of 8011, 100 requests, 8-bit cache 94 us,
// this 82; 40 mixed requests of D = 64 86 us, this 72).
// Where both kinds are large, behind a prefix or with a few prompts among many single tokens, they take turns of one to a CU as long as
// there are workgroups of both, so that a CU has one of each: 256 requests of 10 to 2000 tokens behind 30000: 193 us with all tiles in front, 182 in turns.  Where a prefix's tile has at least
// kLongPart blocks it goes first (256 requests behind 8000, 31 blocks: 70.5 us, the line first 75.1; behind 20000, 39 blocks: 134 and
// 148), else the line (128 requests behind 8000, 15 blocks: 77.1 us, tiles first 87.5; 64 behind 16000, 15 blocks: 101 and 113).
// Without a prefix the largest request tells: with kFewLarge times the average's tokens (32 single tokens behind 4000 and a chunk of 512
// behind 7500, 31 times: 139 us, with all tiles in front 172; 48 and 4 chunks of 300, D = 64, 13 times: 78 and 89; 64 and two prompts of
// 1500, 32 times: 316 and 329) the tiles go first in turns, else all in front (60 requests of 1 to 300 tokens, 6 times: 83 us, in turns
// 93; 12 of 1 to 1000, 7 times: 183 and 195; 16 single tokens and two chunks of 2000, 9 times: 207 and 215).
constexpr int kTurn = 256, kLongPart = 24, kFewLarge = 12;
template <int D, bool F8, bool TILES>
__global__ __launch_bounds__(kAttnThreads, 2) void attn_kernel(AttnParams p)
{
    // Loads into LDS reach its first 64 KiB, so these four arrays have to come first.  They are aligned to more than the rest of the LDS
    // takes: if anything stood in front of one, the kernel's LDS would be larger by a whole kLdsAlign, which the build looks for.  They are four, since which of two buffers is meant has to be known when this is compiled, for a read of one not to wait for loads
    // into the other.
    __shared__ __align__(kLdsAlign) u32x4 kbuf0[kBuffer], vbuf0[kBuffer], kbuf1[kBuffer], vbuf1[kBuffer];
    __shared__ RowsShared rows;
    static_assert(4 * sizeof kbuf0 == 65536 && 2 * kRows * D * 4 <= sizeof kbuf0 && kBlock * D * 2 <= sizeof kbuf0 && kAttnWaves * Step<D, F8>::kUnit <= sizeof kbuf0 && sizeof rows < kLdsAlign, "LDS");
    unsigned x = blockIdx.x;
    if (TILES) {
        const unsigned tiles = p.prefix_groups + p.tile_groups;
        bool tile;
        if (x < p.turns * 2 * kTurn) {
            const unsigned turn = x / (2 * kTurn), at = x % (2 * kTurn);
            tile = (at < kTurn) == (p.tiles_first != 0);
            x = turn * kTurn + at % kTurn;
        } else {
            x -= p.turns * kTurn;
            tile = x < tiles;
            if (!tile) x -= tiles - p.turns * kTurn;
        }
        if (tile) {
            const bool prefix = x < p.prefix_groups;
            if (!prefix) x -= p.prefix_groups;
            tile_of<D, F8>(p, prefix, x / p.KVH, x % p.KVH, kbuf0, vbuf0, kbuf1, vbuf1);
            return;
        }
    }
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()) * (Step<D, F8>::kUnit / 16);
    u32x4 *const units[4] = {kbuf0 + wave, vbuf0 + wave, kbuf1 + wave, vbuf1 + wave};
    rows_of<D, F8>(p, x / p.KVH, x % p.KVH, rows, units, [&](int k) {
        float *const half = reinterpret_cast<float *>(k < 4 ? (k < 2 ? kbuf0 : vbuf0) : (k < 6 ? kbuf1 : vbuf1));
        return half + (k & 1) * (kRows * D);
    });
}

// Joins the parts of the tiles of 128 rows that are cut: D / 4 lanes to a row, a tile's rows over 4 to 16 workgroups: as many as the chip
// holds at once, since most find nothing to join where the batch is large (one request of 3000 tokens, 100 of them new: 39.4 us
// with 1 workgroup a tile, 33.0 with 4, 29.5 with 16; 40 mixed requests: 72 us with 4, 80 with 16).
constexpr int kJoinGroups = 2048;
template <int D>
__device__ __forceinline__ void join_tile(const AttnParams &p, int x, int h, int slice, int slices)
{
    constexpr int L = D / 4, NG = kAttnThreads / L;
    __shared__ FindShared sh;
    Part f;
    if (!find_part<true>(p, x, sh, f)) return;
    int first, n, seq;
    request_of(p, f.b, first, n, seq);
    const int lane = threadIdx.x % L, here = min(n * p.G - f.tile * kTileRows, kTileRows);
    for (int row = slice * (kTileRows / slices) + threadIdx.x / L; row < min((slice + 1) * (kTileRows / slices), here); row += NG) {
        const size_t part = ((size_t)f.item * p.KVH + h) * kTileRows + row, step = (size_t)p.KVH * kTileRows;
        float m = -INFINITY, l = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int i = 0; i < f.splits; ++i) {
            const float2 ml = *reinterpret_cast<const float2 *>(p.wide_ml + 2 * (part + i * step));
            const f32x4 u = *reinterpret_cast<const f32x4 *>(p.wide_o + (part + i * step) * D + 4 * lane);
            const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.0f : top;
            const float a = __builtin_amdgcn_exp2f(m - base), e = __builtin_amdgcn_exp2f(ml.x - base);
            l = l * a + e * ml.y;
            o = o * a + u * e;
            m = top;
        }
        const int ro = f.tile * kTileRows + row, tok = token_of(p, ro);
        f32x4 own[1] = {o};
        finish_row<D>(p, first + tok, h * p.G + ro - tok * p.G, behind_prefix(p, seq - n), 4 * lane, 4, m, l, own);
    }
}

template <int D>
__global__ __launch_bounds__(kAttnThreads) void attn_join_kernel(AttnParams p, unsigned line_groups, int slices)
{
    unsigned x = blockIdx.x;
    if (x < line_groups) {
        join_rows<D>(p, x / p.KVH, x % p.KVH);
    } else {
        x -= line_groups;
        const int slice = x % slices;
        x /= slices;
        join_tile<D>(p, x / p.KVH, x % p.KVH, slice, slices);
    }
}

// What is left behind a call with a shared prefix: a row behind the prefix is joined from the prefix's parts and its own, and where the
// row's tile of 16 is cut, from that tile's parts, which join_rows would join first (its launch, of 5 us, is saved).  D / 4 lanes to a
// row, rows in the order of out.  256 requests, 8192 rows, 33 MB of parts: 11.7 us; 100 requests, 11000 rows: 9.8, of which the sums of all requests'
// lengths, which each workgroup takes for itself, are a good part; with few rows latency (12: 5.6).
template <int D>
__global__ __launch_bounds__(kAttnThreads) void attn_finish_kernel(AttnParams p)
{
    constexpr int L = D / 4, NG = kAttnThreads / L;
    __shared__ Line line;
    const unsigned total = lay_out(p, line), length = length_of(p, total);
    const int QH = p.KVH * p.G, row = blockIdx.x * NG + threadIdx.x / L, lane = threadIdx.x % L;
    const int t = row / QH, head = row % QH, h = head / p.G, r = t * p.G + head % p.G;
    if (t >= p.T) return;
    // the last request that begins at t or before
    int lo = 0, hi = p.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((int)(line.what[mid] >> 47) <= t) lo = mid;
        else hi = mid - 1;
    }
    const unsigned long long what = line.what[lo];
    const int first = (int)(what >> 47), n = (int)(what >> 30 & 0x1ffffu), seq = (int)(what & 0x3fffffffu);
    if (t < first || t >= first + n) return;        // (rows in front of the first request's are nobody's either)
    const bool behind = behind_prefix(p, seq - n);
    const int own_row = (t - first) * p.G + head % p.G;
    float m = -INFINITY, l = 0.0f;
    f32x4 o[1] = {{0.0f, 0.0f, 0.0f, 0.0f}};
    const auto join = [&](const float *ml, const float *values) {
        const float2 w = *reinterpret_cast<const float2 *>(ml);
        const f32x4 u = *reinterpret_cast<const f32x4 *>(values + 4 * lane);
        const float top = fmaxf(m, w.x), base = top == -INFINITY ? 0.0f : top;
        const float a = __builtin_amdgcn_exp2f(m - base), e = __builtin_amdgcn_exp2f(w.x - base);
        l = l * a + e * w.y;
        o[0] = o[0] * a + u * e;
        m = top;
    };
    unsigned x = 0, last = 0, begin = 0;           // the lengths of the line that the row's tile lies in
    if (n * p.G <= p.narrow && total > 0) {
        const unsigned count = blocks_per_tile(p, n, seq);
        begin = (lo > 0 ? line.ends[lo - 1] : 0u) + (unsigned)(own_row / kRows) * count;
        x = begin / length;
        last = (begin + count - 1) / length;
    }
    if (x < last) {
        for (; x <= last; ++x) {
            const size_t part = ((size_t)(2 * x + (begin >= x * length ? 1 : 0)) * p.KVH + h) * kRows + own_row % kRows;
            join(p.part_ml + 2 * part, p.part_o + part * D);
        }
    } else {
        if (!behind) return;
        join(p.own_ml + 2 * (size_t)row, p.own_o + (size_t)row * D);
    }
    if (behind) {
        size_t part = ((size_t)(r / kTileRows) * p.prefix_splits * p.KVH + h) * kTileRows + r % kTileRows;
#pragma unroll 8
        for (int i = 0; i < p.prefix_splits; ++i, part += (size_t)p.KVH * kTileRows) join(p.prefix_ml + 2 * part, p.prefix_o + part * D);
    }
    finish_row<D>(p, t, head, false, 4 * lane, 4, m, l, o);
}

// Requests of up to this many rows are read by tiles of 16 rows, others by tiles of 128.  Two tiles of 16 read the cache twice (32 requests
// of 4096 tokens, 8 key heads of 4 query heads: 20 rows 164 us, by one tile of 128 108 us; 64 rows 293 and 114; 64 requests with one
// key head of 32: 58 and 44).  An 8-bit block, which a wide tile has to widen on its way into LDS, is better read twice, not more
// often (100 requests of 250 to 2000: 32 rows 90 us, by a wide tile 116; 48 rows 128 and 117).
inline int narrow_rows(bool f8) { return f8 ? 2 * kRows : kRows; }
// What the workspace holds: rows of unfinished tiles with their maxima and sums.  A workgroup's length of the line leaves two tiles.
// Tiles of 128 rows: a tile that is cut has more than `chunk` blocks, so its parts are fewer than twice blocks / chunk, all such
// parts fewer than twice wide_parts, and such tiles at most wide_parts.
// The prefix's tiles leave every row's parts, and the rows behind the prefix their own.
struct AttnSpace {
    int parts, wide_parts, prefix_blocks, prefix_tiles, prefix_splits;
    size_t ml_off, cuts_off, wide_o_off, wide_ml_off, prefix_o_off, prefix_ml_off, own_o_off, own_ml_off, total;
};
// Whether a shared prefix is read apart.  Each row then leaves its own part and the prefix's, unnormalised and in fp32, in the workspace, which
// are written and read again.  A request whose rows fill a tile of 128 gains nothing by it, since the tiles read the prefix for 128 rows
// either way (8 key heads of 4 query heads, 64 requests of 128 rows and 200 tokens of their own: behind 64 tokens 37 us through the block table
// and apart 67, behind 1024 65 and 94, behind 16384 554 and 570; 16 of 96 rows behind 16384 the other way round, 151 and 134), nor does one
// whose rows are many against the prefix (64 requests of 32 rows, 4 key heads, behind 64 tokens: 21.2 and 30.1; behind 256, 8 tokens
// for a row, 25.1 and 30.4; behind 1024, 32, 41.6 and 36.0).
constexpr int kApart = 4;               // tokens of the prefix for each row of a request
inline bool reads_apart(int B, int T, int G, int prefix_len)
{
    const int64_t rows = (int64_t)T * G;            // of all requests for a key head
    return rows < (int64_t)B * kTileRows && rows * kApart <= (int64_t)B * prefix_len;
}
static AttnSpace attention_space(int B, int T, int G, int KVH, int D, int prefix_len)
{
    AttnSpace w;
    w.parts = kWorkgroups / KVH > 0 ? kWorkgroups / KVH : 1;
    const size_t rows = (size_t)2 * w.parts * KVH * kRows;
    w.ml_off = align256(rows * D * 4);
    w.cuts_off = w.ml_off + align256(rows * 8);
    w.wide_o_off = w.cuts_off + align256((size_t)w.parts * sizeof(Cut));
    w.wide_parts = w.parts;
    const size_t wide_rows = (int64_t)T * G > kRows ? (size_t)2 * w.wide_parts * KVH * kTileRows : 0;
    w.wide_ml_off = w.wide_o_off + align256(wide_rows * D * 4);
    w.prefix_o_off = w.wide_ml_off + align256(wide_rows * 8);
    // As many parts of the prefix as fill the chip, of four blocks at least; or half as many, one to a CU beside the line of what the
    // requests have of their own, where the parts would else have fewer than 32 blocks (each leaves its rows to be joined) and half the
    // chip's workgroups come out nearly full.  512 requests behind 4000, 15 blocks: 277 us, half as many parts 228; 128 behind
    // 16000, 15 blocks: 95 and 85; 64 behind 16000, 8 blocks: 121 and 101; 256 behind 16000, 31 blocks: 109 and 111, with 2000 tokens
    // of their own 213 and 208; behind 30000, 58 blocks: 173 and 186.  100 requests of 2 to 5 tokens behind 8011, whose 88 tiles
    // fill two thirds of one half: 78 and 94.
    const int blocks = T > 0 && reads_apart(B, T, G, prefix_len) ? prefix_len / kBlock : 0;
    w.prefix_blocks = blocks;
    w.prefix_tiles = (int)(((int64_t)T * G + kTileRows - 1) / kTileRows);
    const int tiles = w.prefix_tiles * KVH;
    w.prefix_splits = 0;
    if (blocks > 0) {
        int splits = std::max(1, kWorkgroups / tiles);
        const int half = kWorkgroups / 2 / tiles;
        if (blocks / splits < 32 && half * tiles * 8 >= kWorkgroups / 2 * 7) splits = half;
        w.prefix_splits = std::min(splits, (blocks + 3) / 4);
    }
    // Room for what any step of at most these sizes needs, so that a workspace for the largest one serves all: the most rows for which the
    // prefix may be read apart, and the most parts that they are cut into.
    const int64_t all_blocks = prefix_len / kBlock;
    const int64_t most = all_blocks > 0 ? std::min(std::min((int64_t)T * G, (int64_t)B * kTileRows - 1), (int64_t)B * prefix_len / kApart) : 0;
    const int64_t most_tiles = (most + kTileRows - 1) / kTileRows * KVH;
    const size_t prefix_rows = (size_t)std::max(most_tiles, std::min<int64_t>(kWorkgroups, most_tiles * ((all_blocks + 3) / 4))) * kTileRows;
    w.prefix_ml_off = w.prefix_o_off + align256(prefix_rows * D * 4);
    w.own_o_off = w.prefix_ml_off + align256(prefix_rows * 8);
    const size_t own_rows = (size_t)most * KVH;
    w.own_ml_off = w.own_o_off + align256(own_rows * D * 4);
    w.total = w.own_ml_off + align256(own_rows * 8);
    return w;
}

static int attention_impl(const char *who, const uint16_t *q, int64_t q_stride, const void *k_cache, const void *v_cache, int cache_format,
                          float k_scale, float v_scale, int num_pages, int page_size, const int32_t *block_table, int max_pages,
                          const int32_t *q_start, const int32_t *seq_len, const int32_t *prefix_table, int prefix_len, int B, int T,
                          int max_new, int QH, int KVH, int D, float scale, int window, int sinks, uint16_t *out,
                          int64_t out_stride, float *lse, void *workspace, void *stream)
{
    if (B <= 0 || T < 0 || max_pages <= 0 || max_new < 0 || window < 0 || sinks < 0 || prefix_len < 0)
        return fail(LYNX_ERR_INVALID_ARG, "%s: negative or zero size", who);
    int rc = check_cache(who, k_cache, v_cache, cache_format, k_scale, v_scale, num_pages, page_size, QH, KVH, D);
    if (rc != LYNX_OK) return rc;
    if (B > LYNX_MAX_REQUESTS || T > LYNX_MAX_STEP_TOKENS || max_pages > kMaxContext / page_size)
        return fail(LYNX_ERR_UNSUPPORTED, "%s: need B<=%d, T<=%d, max_pages*page_size<=%d", who, LYNX_MAX_REQUESTS, LYNX_MAX_STEP_TOKENS, kMaxContext);
    if (prefix_len > max_pages * page_size)
        return fail(LYNX_ERR_INVALID_ARG, "%s: the prefix is longer than a row of the block table", who);
    // (positions on the line of all tiles' blocks are 32 bits)
    const int64_t most_tiles = B + (int64_t)T * (QH / KVH) / kRows;
    if (most_tiles * (((int64_t)max_pages * page_size + kBlock - 1) / kBlock) >= (int64_t)1 << 31)
        return fail(LYNX_ERR_UNSUPPORTED, "%s: need (B + T * QH / KVH / 16) * max_pages * page_size < 2^37", who);
    if (!(scale > 0.0f) || scale > 3.0e38f) return fail(LYNX_ERR_INVALID_ARG, "%s: scale must be finite and > 0", who);
    // (a masked score is -inf, which times a factor of 0 would be no number)
    const float scale2 = scale * k_scale * kLog2e;
    if (!(scale2 >= FLT_MIN) || scale2 > FLT_MAX) return fail(LYNX_ERR_INVALID_ARG, "%s: scale * k_scale leaves the range of a float", who);
    if (T == 0) return LYNX_OK;
    if (!block_table || !q_start || !seq_len || (prefix_len > 0 && !prefix_table) || !workspace)
        return fail(LYNX_ERR_INVALID_ARG, "%s: null pointer", who);
    if ((rc = check_rows(who, "q", q, q_stride, QH, D)) != LYNX_OK || (rc = check_rows(who, "out", out, out_stride, QH, D)) != LYNX_OK) return rc;
    if (out == q) return fail(LYNX_ERR_INVALID_ARG, "%s: out must not be q", who);
    if (((uintptr_t)workspace & 255) != 0) return fail(LYNX_ERR_INVALID_ARG, "%s: the workspace must start on 256 bytes", who);
    const int G = QH / KVH;
    const AttnSpace w = attention_space(B, T, G, KVH, D, prefix_len);
    const int narrow = narrow_rows(cache_format == LYNX_CACHE_FP8);
    const bool wide = (int64_t)T * G > narrow && (int64_t)max_new * G > narrow;
    char *const ws = (char *)workspace;
    AttnParams p = {q, k_cache, v_cache, block_table, q_start, seq_len, prefix_table, out, lse, q_stride, out_stride, B, T, KVH, G,
                    num_pages, max_pages, page_size, page_multiplier(page_size), reciprocal(G), reciprocal(w.parts), scale2, v_scale,
                    std::min(8.0f / scale2, FLT_MAX),
                    window < kMaxContext ? window : 0, sinks < kMaxContext ? sinks : kMaxContext,   // (a window that long hides nothing)
                    w.parts, (float *)ws, (float *)(ws + w.ml_off), (Cut *)(ws + w.cuts_off), wide ? narrow : INT_MAX, w.wide_parts, (float *)(ws + w.wide_o_off),
                    (float *)(ws + w.wide_ml_off), w.prefix_blocks, w.prefix_splits, (float *)(ws + w.prefix_o_off), (float *)(ws + w.prefix_ml_off),
                    (float *)(ws + w.own_o_off), (float *)(ws + w.own_ml_off)};
    const bool f8 = cache_format == LYNX_CACHE_FP8;
    const dim3 threads(kAttnThreads);
    hipStream_t st = (hipStream_t)stream;
    // tiles: at most the sum of ceil(rows / 128) over requests of more than `narrow` rows
    const unsigned tiles = wide ? (unsigned)((int64_t)T * G / kTileRows + std::min<int64_t>(B, (int64_t)T * G / narrow)) : 0u;
    p.prefix_groups = p.prefix_blocks > 0 ? (unsigned)KVH * w.prefix_tiles * w.prefix_splits : 0u;
    p.tile_groups = wide ? KVH * (tiles + w.wide_parts) : 0u;
    const bool any_tiles = p.prefix_groups + p.tile_groups > 0;
    const bool few_large = any_tiles && (int64_t)max_new * B >= (int64_t)kFewLarge * T;
    p.turns = p.prefix_groups > 0 || few_large ? std::min(p.prefix_groups + p.tile_groups, (unsigned)(KVH * w.parts)) / kTurn : 0u;
    p.tiles_first = p.prefix_groups == 0 || p.prefix_blocks / w.prefix_splits >= kLongPart;
    auto kernel = D == 128 ? (f8 ? (any_tiles ? attn_kernel<128, true, true> : attn_kernel<128, true, false>)
                                 : (any_tiles ? attn_kernel<128, false, true> : attn_kernel<128, false, false>))
                           : (f8 ? (any_tiles ? attn_kernel<64, true, true> : attn_kernel<64, true, false>)
                                 : (any_tiles ? attn_kernel<64, false, true> : attn_kernel<64, false, false>));
    hipLaunchKernelGGL(kernel, dim3(p.prefix_groups + p.tile_groups + (unsigned)KVH * w.parts), threads, 0, st, p);
    const unsigned line_groups = p.prefix_blocks > 0 ? 0u : (unsigned)(w.parts - 1) * KVH, cut_tiles = std::min(tiles, (unsigned)w.wide_parts) * KVH;
    const int slices = cut_tiles * 16 <= kJoinGroups ? 16 : cut_tiles * 8 <= kJoinGroups ? 8 : 4;
    const unsigned tile_joins = cut_tiles * slices;
    if (line_groups + tile_joins > 0)
        hipLaunchKernelGGL((D == 128 ? attn_join_kernel<128> : attn_join_kernel<64>), dim3(line_groups + tile_joins), threads, 0, st, p, line_groups, slices);
    if (p.prefix_blocks > 0)
        hipLaunchKernelGGL((D == 128 ? attn_finish_kernel<128> : attn_finish_kernel<64>), dim3((unsigned)(((int64_t)T * QH * (D / 4) + kAttnThreads - 1) / kAttnThreads)),
                           threads, 0, st, p);
    return check_launch(who);
}

}  // namespace lynx

extern "C" size_t lynx_attention_workspace_bytes(int B, int T, int QH, int KVH, int D, int prefix_len)
{
    if (B <= 0 || B > LYNX_MAX_REQUESTS || T < 0 || T > LYNX_MAX_STEP_TOKENS || KVH <= 0 || QH < KVH || QH > lynx::kMaxHeads || QH % KVH != 0 ||
        QH / KVH > lynx::kMaxGroup || (D != 64 && D != 128) || prefix_len < 0)
        return 0;
    return lynx::attention_space(B, T, QH / KVH, KVH, D, prefix_len).total;
}

extern "C" int lynx_attention(const uint16_t *q, int64_t q_stride, const void *k_cache, const void *v_cache, int cache_format,
                              float k_scale, float v_scale, int num_pages, int page_size, const int32_t *block_table, int max_pages,
                              const int32_t *q_start, const int32_t *seq_len, int B, int T, int max_new, int QH, int KVH, int D,
                              float scale, int window, int sinks, uint16_t *out, int64_t out_stride, float *lse, void *workspace,
                              void *stream)
{
    return lynx::attention_impl("lynx_attention", q, q_stride, k_cache, v_cache, cache_format, k_scale, v_scale, num_pages, page_size, block_table,
                                max_pages, q_start, seq_len, nullptr, 0, B, T, max_new, QH, KVH, D, scale, window, sinks, out,
                                out_stride, lse, workspace, stream);
}

extern "C" int lynx_attention_prefix(const uint16_t *q, int64_t q_stride, const void *k_cache, const void *v_cache, int cache_format,
                                     float k_scale, float v_scale, int num_pages, int page_size, const int32_t *block_table,
                                     int max_pages, const int32_t *q_start, const int32_t *seq_len, const int32_t *prefix_table,
                                     int prefix_len, int B, int T, int max_new, int QH, int KVH, int D, float scale, uint16_t *out,
                                     int64_t out_stride, float *lse, void *workspace, void *stream)
{
    return lynx::attention_impl("lynx_attention_prefix", q, q_stride, k_cache, v_cache, cache_format, k_scale, v_scale, num_pages, page_size,
                                block_table, max_pages, q_start, seq_len, prefix_table, prefix_len, B, T, max_new, QH, KVH, D, scale, 0, 0,
                                out, out_stride, lse, workspace, stream);
}
