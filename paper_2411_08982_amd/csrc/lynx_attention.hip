// Attention over the paged cache (lynx_attention, lynx_attention_prefix).
//
// Rows.  The QH / KVH = G query heads that share a key head read the same keys, so the rows of a request for one key head are its
// n new tokens times G: row r is token r / G, head r % G of the group.
//
// Products.  Both are taken transposed on the matrix cores, v_mfma_f32_16x16x32_bf16:  S^T = K Q^T and O^T = V^T P^T.  A result
// fragment of S^T holds, in lane l, the scores of row l % 16 with 4 tokens; K's rows are handed in such an order that the fragments of
// one step give every lane 8 (bf16 cache) or 16 (8-bit cache) CONSECUTIVE tokens, and these are exactly what the lane has to hold as operand
// of the second product.  So the weights never leave their lane: no LDS, no exchange; running maximum, sum and the rescaling
// of O^T are per lane (a row is one column of both results), and only the maximum is joined over the four lanes of a row.
// V's operand wants those tokens of one channel: one 16-byte load from the transposed pages.
//
// Softmax in one pass: m = running maximum (of the scores times scale * log2 e), l = sum of 2^(s - m), O accumulates 2^(s - m) v; when
// m grows, l and O are multiplied by 2^(m_old - m_new).  All in fp32.
#include "lynx_attention.h"

namespace lynx {

constexpr int kBlock = 64;              // tokens of a block: the unit in which a row's context is dealt out
constexpr int kRows = 16;               // rows of a tile
constexpr int kAttnThreads = 256;
constexpr int kAttnWaves = kAttnThreads / kWave;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct AttnParams {
    const uint16_t *q;
    const void *k, *v;
    const int32_t *table, *q_start, *seq_len, *prefix_table;
    uint16_t *out;
    float *lse;
    int64_t q_stride, out_stride;
    int B, T, KVH, G, num_pages, max_pages, page_size, prefix_len;
    unsigned page_mul;                  // division of a group of 16 tokens by the page size: page_of
    float scale2, v_scale;              // scale * k_scale * log2 e
    int window, sinks;
    int parts;                          // parts that the contexts of all tiles together are cut into, per key head
    float *part_o, *part_ml;            // workspace: unfinished rows
};

// Page (index in a row of the table) of the 16 tokens from 16 * group on: group / (page_size / 16), by multiplication.
// Exact for group < 2^25 and page_size / 16 <= 64, since group * error < 2^31 / (page_size / 16).
__device__ __forceinline__ int page_of(const AttnParams &p, int group) { return (int)__umulhi(2u * (unsigned)group, p.page_mul); }
inline unsigned page_multiplier(int page_size) { return (1u << 31) / (unsigned)(page_size / 16) + 1u; }

// The rows of request b and its length, clamped.
__device__ __forceinline__ void request_of(const AttnParams &p, int b, int &first, int &n, int &seq)
{
    first = min(max(p.q_start[b], 0), p.T);
    n = min(max(p.q_start[b + 1], first), p.T) - first;
    seq = min(max(p.seq_len[b], 0), p.max_pages * p.page_size);
}

// The blocks that a span of rows at positions pmin .. pmax sees: `lead` blocks of the first tokens that stay visible, then those from
// `start` on; `count` in all.
struct Blocks {
    int lead, start, count;
    __device__ __forceinline__ int at(int i) const { return i < lead ? i : start + i - lead; }
};
__device__ __forceinline__ Blocks blocks_of(const AttnParams &p, int pmin, int pmax)
{
    Blocks s;
    const int end = pmax >= 0 ? pmax / kBlock + 1 : 0;
    s.start = p.window == 0 ? 0 : min(max(pmin - p.window + 1, 0) / kBlock, end);
    s.lead = p.window == 0 ? 0 : min((p.sinks - 1 + kBlock) / kBlock, s.start);
    s.count = s.lead + end - s.start;
    return s;
}

// How the work is cut.  A tile's context is cut into parts of at most `chunk` blocks, so that few rows with long contexts fill the
// chip as well: chunk follows from the work of the whole batch (all tiles' blocks over p.parts) and is the same for all, so no
// part is longer than the average workgroup's share.  Request lengths are on the device only; every workgroup works out for
// itself which part it is: one round trip for the lengths (at most four requests a thread), two sums over the workgroup.
constexpr int kMinChunk = 4;
constexpr int kWorkgroups = 512;       // workgroups that the chip holds at once: two of four waves on each of 256 CUs
constexpr int kMaxPerThread = LYNX_MAX_REQUESTS / kAttnThreads;
struct Found {
    int b, tile, split, splits, item;       // item: index of the tile's first part among those of all tiles that are cut
};
struct FindShared {
    float work[kAttnWaves];
    int sum[2][kAttnWaves];
    Found found;
};
// CUT: x counts the tiles that are cut, otherwise the parts of all tiles.
template <bool CUT>
__device__ __forceinline__ bool find_work(const AttnParams &p, int x, FindShared &sh, Found &f)
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
            tiles[i] = (n * p.G + kRows - 1) / kRows;
            blocks[i] = blocks_of(p, max(seq - n, 0), seq - 1).count;
            work += (float)tiles[i] * (float)blocks[i];
        }
    }
    work = wave_sum(work);
    if (threadIdx.x == 0) sh.found.b = -1;
    if (lane == 0) sh.work[wv] = work;
    __syncthreads();
    work = 0.0f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) work += sh.work[w];
    // (a little more than the quotient: the sum is rounded, and there are no more than p.parts + tiles workgroups)
    const int chunk = max(kMinChunk, (int)(work * 1.0001f / (float)p.parts) + 1);
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
    // the requests of this thread one by one: does x fall into one of them
#pragma unroll
    for (int i = 0; i < kMaxPerThread; ++i) {
        const int items = CUT ? (blocks[i] > 1 ? tiles[i] : 0) : tiles[i] * blocks[i], at = x - sx;
        if (at >= 0 && at < items) {
            const int tile = CUT ? at : at / blocks[i];
            sh.found.tile = tile;
            sh.found.split = CUT ? 0 : at - tile * blocks[i];
            sh.found.splits = blocks[i];
            sh.found.item = sc + tile * blocks[i];
            sh.found.b = b0 + i;
        }
        sx += items;
        sc += blocks[i] > 1 ? tiles[i] * blocks[i] : 0;
    }
    __syncthreads();
    f = sh.found;
    f.b = __builtin_amdgcn_readfirstlane(f.b);
    f.tile = __builtin_amdgcn_readfirstlane(f.tile);
    f.split = __builtin_amdgcn_readfirstlane(f.split);
    f.splits = __builtin_amdgcn_readfirstlane(f.splits);
    f.item = __builtin_amdgcn_readfirstlane(f.item);
    return f.b >= 0;
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

// One step of TN tokens from token t0 on (t0 a multiple of TN): scores, weights, second product.  pos: position of the lane's row
// (-1: no row); pmin, pmax: least and greatest position of the tile's rows.
template <int D, bool F8>
struct Step {
    static constexpr int TN = F8 ? 64 : 32;        // tokens: 16 bytes of a channel from every lane
    static constexpr int NS = TN / 16;             // fragments of S^T
    static constexpr int LT = TN / 4;              // consecutive tokens of a lane
    static constexpr int KL = D * (F8 ? 1 : 2) / 64;   // 16-byte loads of a key row by its four lanes

    static __device__ __forceinline__ void run(const AttnParams &p, const int32_t *pages, int h, int t0, const bf16x8 (&q)[D / 32], int pos,
                                               int pmin, int pmax, RowState<D> &s)
    {
        const int lane = lane_id(), g = lane >> 4, c = lane & 15;
        constexpr int E = F8 ? 1 : 2;
        const uint8_t *kc = (const uint8_t *)p.k, *vc = (const uint8_t *)p.v;
        // this lane's token for the first fragment, and its run of tokens
        const int kt = t0 + (c >> 2) * LT + (c & 3), vt = t0 + g * LT;
        const int kp = page_of(p, kt >> 4), vp = page_of(p, vt >> 4), last = p.max_pages - 1;
        const int kid = pages[min(kp, last)], vid = pages[min(vp, last)];
        const bool kok = kp <= last && (unsigned)kid < (unsigned)p.num_pages, vok = vp <= last && (unsigned)vid < (unsigned)p.num_pages;
        const size_t head_bytes = (size_t)p.page_size * D * E;
        // (tokens without a page are read from the first page's start and not seen)
        const uint8_t *ka = kc + ((size_t)(kok ? kid : 0) * p.KVH + h) * head_bytes + (kok ? kt - kp * p.page_size : 0) * (D * E) + g * 16;
        const uint8_t *va = vc + ((size_t)(vok ? vid : 0) * p.KVH + h) * head_bytes +
                            (size_t)(c * p.page_size + (vok ? vt - vp * p.page_size : 0)) * E;

        uint4 kw[NS][KL], vw[D / 16];
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int i = 0; i < KL; ++i) kw[j][i] = *reinterpret_cast<const uint4 *>(ka + j * 4 * (D * E) + i * 64);
#pragma unroll
        for (int t = 0; t < D / 16; ++t) vw[t] = *reinterpret_cast<const uint4 *>(va + (size_t)t * 16 * p.page_size * E);

        f32x4 z[NS];
#pragma unroll
        for (int j = 0; j < NS; ++j) {
            z[j] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < KL; ++i) {
                if (F8) {
                    z[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(make_uint2(kw[j][i].x, kw[j][i].y)), q[2 * i], z[j], 0, 0, 0);
                    z[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(make_uint2(kw[j][i].z, kw[j][i].w)), q[2 * i + 1], z[j], 0, 0, 0);
                } else {
                    z[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kw[j][i]), q[i], z[j], 0, 0, 0);
                }
            }
        }
        float x[LT];
#pragma unroll
        for (int i = 0; i < LT; ++i) x[i] = z[i / 4][i % 4] * p.scale2;
        // Tokens that not every row of the tile sees.  A token that none sees may hold anything, also what is no number: its
        // value is replaced by zero, since zero times it would not be.
        const bool in_window = p.window == 0 || t0 > pmax - p.window || t0 + TN <= p.sinks;
        if (!(t0 + TN - 1 <= pmin && in_window && __all(vok))) {
#pragma unroll
            for (int i = 0; i < LT; ++i) {
                const int t = vt + i;
                const bool seen = vok && t <= pos && (p.window == 0 || t > pos - p.window || t < p.sinks);
                x[i] = seen ? x[i] : -INFINITY;
            }
            uint32_t mask[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                mask[w] = 0u;
#pragma unroll
                for (int i = 0; i < 4 / E; ++i) {
                    const int t = vt + w * (4 / E) + i;
                    const bool any = vok && t <= pmax && (p.window == 0 || t > pmin - p.window || t < p.sinks);
                    mask[w] |= any ? (F8 ? 0xffu << (8 * i) : 0xffffu << (16 * i)) : 0u;
                }
            }
#pragma unroll
            for (int t = 0; t < D / 16; ++t) {
                vw[t].x &= mask[0];
                vw[t].y &= mask[1];
                vw[t].z &= mask[2];
                vw[t].w &= mask[3];
            }
        }
        float top = x[0];
#pragma unroll
        for (int i = 1; i < LT; ++i) top = fmaxf(top, x[i]);
        const float m = fmaxf(s.m, row_max(top));
        if (__any(m > s.m)) {
            const float a = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(s.m - m);
            s.l *= a;
#pragma unroll
            for (int t = 0; t < D / 16; ++t) s.o[t] *= a;
            s.m = m;
        }
        const float base = s.m == -INFINITY ? 0.0f : s.m;
#pragma unroll
        for (int i = 0; i < LT; ++i) {
            x[i] = __builtin_amdgcn_exp2f(x[i] - base);
            s.l += x[i];
        }
        // bf16 weights: half a step of 2^-8 each, of either sign, beside values that are bf16 themselves
        bf16x8 w[LT / 8];
#pragma unroll
        for (int i = 0; i < LT / 8; ++i) {
            const uint4 u = make_uint4(pack_bf16(x[8 * i], x[8 * i + 1]), pack_bf16(x[8 * i + 2], x[8 * i + 3]),
                                       pack_bf16(x[8 * i + 4], x[8 * i + 5]), pack_bf16(x[8 * i + 6], x[8 * i + 7]));
            w[i] = __builtin_bit_cast(bf16x8, u);
        }
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
            if (F8) {
                s.o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(make_uint2(vw[t].x, vw[t].y)), w[0], s.o[t], 0, 0, 0);
                s.o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(make_uint2(vw[t].z, vw[t].w)), w[LT / 8 - 1], s.o[t], 0, 0, 0);
            } else {
                s.o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vw[t]), w[0], s.o[t], 0, 0, 0);
            }
        }
    }
};

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

// A finished row piece of D / 16 channels: out = o * v_scale / l.
template <int D>
__device__ __forceinline__ void write_out(const AttnParams &p, int t, int head, int c0, float m, float l, const float (&o)[D / 16])
{
    const float inv = l == 0.0f ? 0.0f : p.v_scale / l;
    uint16_t *dst = p.out + (size_t)t * p.out_stride + (size_t)head * D + c0;
    if (D == 128) {
        *reinterpret_cast<uint4 *>(dst) = make_uint4(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv),
                                                     pack_bf16(o[D / 16 - 4] * inv, o[D / 16 - 3] * inv), pack_bf16(o[D / 16 - 2] * inv, o[D / 16 - 1] * inv));
    } else {
        *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
    }
    if (p.lse && c0 == 0) p.lse[(size_t)t * (p.KVH * p.G) + head] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// One workgroup per (part of the context of a tile of 16 rows of a request, key head); the blocks of the part go round the four
// waves, whose parts of the softmax are joined in LDS.
template <int D, bool F8>
__global__ __launch_bounds__(kAttnThreads) void attn_rows_kernel(AttnParams p)
{
    __shared__ FindShared sh;
    __shared__ float sm[kAttnWaves][kRows], sl[kAttnWaves][kRows];
    __shared__ __align__(16) float so[kAttnWaves][kRows][D + 4];
    const int lane = lane_id(), wv = __builtin_amdgcn_readfirstlane(wave_id()), h = blockIdx.y;
    Found f;
    if (!find_work<false>(p, blockIdx.x, sh, f)) return;
    int first, n, seq;
    request_of(p, f.b, first, n, seq);
    const int r = f.tile * kRows + (lane & 15), rows = n * p.G;
    const bool real = r < rows;
    const int tok = real ? r / p.G : 0;
    const int pos = real ? seq - n + tok : -1;
    const int pmin = max(seq - n + f.tile * kRows / p.G, 0), pmax = seq - n + (min(f.tile * kRows + kRows, rows) - 1) / p.G;
    bf16x8 q[D / 32];
    load_queries<D, F8>(p.q + (size_t)(first + tok) * p.q_stride + (size_t)(h * p.G + (real ? r % p.G : 0)) * D, real, q);

    RowState<D> s;
    s.m = -INFINITY;
    s.l = 0.0f;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) s.o[t] = {0.0f, 0.0f, 0.0f, 0.0f};
    const Blocks blocks = blocks_of(p, pmin, pmax);
    const int per = (blocks.count + f.splits - 1) / f.splits, i0 = f.split * per, i1 = min(i0 + per, blocks.count);
    const int32_t *row = p.table + (size_t)f.b * p.max_pages;
    for (int i = i0 + wv; i < i1; i += kAttnWaves) {
        const int blk = blocks.at(i);
        const int32_t *pages = (blk + 1) * kBlock <= p.prefix_len ? p.prefix_table : row;
        for (int t = 0; t < kBlock; t += Step<D, F8>::TN) Step<D, F8>::run(p, pages, h, blk * kBlock + t, q, pos, pmin, pmax, s);
    }
    s.l = row_sum(s.l);
    if (lane < kRows) {
        sm[wv][lane] = s.m;
        sl[wv][lane] = s.l;
    }
#pragma unroll
    for (int t = 0; t < D / 16; ++t) *reinterpret_cast<f32x4 *>(&so[wv][lane & 15][t * 16 + (lane >> 4) * 4]) = s.o[t];
    __syncthreads();
    // 16 threads per row, D / 16 channels each
    const int orow = threadIdx.x / kRows, c0 = threadIdx.x % kRows * (D / 16), ro = f.tile * kRows + orow;
    if (ro >= rows) return;
    float m = sm[0][orow];
#pragma unroll
    for (int w = 1; w < kAttnWaves; ++w) m = fmaxf(m, sm[w][orow]);
    float l = 0.0f, o[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
        const float e = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm[w][orow] - m);
        l += e * sl[w][orow];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] += e * so[w][orow][c0 + i];
    }
    if (f.splits == 1) {
        write_out<D>(p, first + ro / p.G, h * p.G + ro % p.G, c0, m, l, o);
        return;
    }
    const size_t part = ((size_t)(f.item + f.split) * p.KVH + h) * kRows + orow;
    float4 *dst = reinterpret_cast<float4 *>(p.part_o + part * D + c0);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) dst[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
    if (c0 == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * part) = make_float2(m, l);
}

// Joins the parts of a tile's rows.  Few rows with many parts each are the case that counts (one request alone: a few rows, dozens
// of parts), so a tile's rows are spread over kJoinSlices workgroups, and the parts of a row over what is left of the
// workgroup's D / 4-lane groups, which meet in LDS.
constexpr int kJoinSlices = 4;
template <int D>
__global__ __launch_bounds__(kAttnThreads) void attn_join_kernel(AttnParams p)
{
    constexpr int L = D / 4, NG = kAttnThreads / L;         // lanes of a group (4 channels each), groups
    __shared__ FindShared sh;
    __shared__ float sm[NG], sl[NG];
    __shared__ __align__(16) float4 so[NG][L];
    Found f;
    if (!find_work<true>(p, blockIdx.x, sh, f)) return;
    int first, n, seq;
    request_of(p, f.b, first, n, seq);
    const int h = blockIdx.y, slice = blockIdx.z, here = min(n * p.G - f.tile * kRows, kRows);    // the tile's rows
    const int mine = (here - slice + kJoinSlices - 1) / kJoinSlices;                               // those of this workgroup
    if (mine <= 0) return;
    const int width = mine > 2 ? 4 : mine;                                                         // (a power of two)
    const int grp = threadIdx.x / L, lane = threadIdx.x % L, k = grp % width, sub = grp / width;
    const int orow = slice + k * kJoinSlices;
    const bool real = k < mine;
    const size_t part = ((size_t)f.item * p.KVH + h) * kRows + (real ? orow : slice), step = (size_t)p.KVH * kRows;
    float m = -INFINITY, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int i = sub; i < f.splits; i += NG / width) {
        const float2 ml = *reinterpret_cast<const float2 *>(p.part_ml + 2 * (part + i * step));
        const f32x4 u = *reinterpret_cast<const f32x4 *>(p.part_o + (part + i * step) * D + 4 * lane);
        const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.0f : top;
        const float a = __builtin_amdgcn_exp2f(m - base), e = __builtin_amdgcn_exp2f(ml.x - base);
        l = l * a + e * ml.y;
        o = o * a + u * e;
        m = top;
    }
    if (lane == 0) {
        sm[grp] = m;
        sl[grp] = l;
    }
    so[grp][lane] = make_float4(o[0], o[1], o[2], o[3]);
    __syncthreads();
    if (sub != 0 || !real) return;
    for (int w = k + width; w < NG; w += width) {
        const float4 u = so[w][lane];
        const float top = fmaxf(m, sm[w]), base = top == -INFINITY ? 0.0f : top;
        const float a = __builtin_amdgcn_exp2f(m - base), e = __builtin_amdgcn_exp2f(sm[w] - base);
        l = l * a + e * sl[w];
        o = o * a + f32x4{u.x, u.y, u.z, u.w} * e;
        m = top;
    }
    const int ro = f.tile * kRows + orow, t = first + ro / p.G, head = h * p.G + ro % p.G;
    const float inv = l == 0.0f ? 0.0f : p.v_scale / l;
    *reinterpret_cast<uint2 *>(p.out + (size_t)t * p.out_stride + (size_t)head * D + 4 * lane) =
        make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
    if (p.lse && lane == 0) p.lse[(size_t)t * (p.KVH * p.G) + head] = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// What the workspace holds: rows of unfinished parts, and their maxima and sums.  A tile that is cut has more than `chunk` blocks, so its
// parts are fewer than twice blocks / chunk, and all such parts fewer than twice p.parts; there are at most p.parts such tiles.
struct AttnSpace {
    int tiles, parts;
    size_t ml_off, total;
};
static AttnSpace attention_space(int B, int T, int QH, int KVH, int D)
{
    AttnSpace w;
    w.tiles = B + (int)((int64_t)T * (QH / KVH) / kRows);     // sum of ceil(rows / 16) over requests
    w.parts = kWorkgroups / KVH > 0 ? kWorkgroups / KVH : 1;
    const size_t rows = (size_t)2 * w.parts * KVH * kRows;
    w.ml_off = align256(rows * D * 4);
    w.total = w.ml_off + align256(rows * 8);
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
    if (!(scale > 0.0f) || scale > 3.0e38f) return fail(LYNX_ERR_INVALID_ARG, "%s: scale must be finite and > 0", who);
    if (T == 0) return LYNX_OK;
    if (!block_table || !q_start || !seq_len || (prefix_len > 0 && !prefix_table) || !workspace)
        return fail(LYNX_ERR_INVALID_ARG, "%s: null pointer", who);
    if ((rc = check_rows(who, "q", q, q_stride, QH, D)) != LYNX_OK || (rc = check_rows(who, "out", out, out_stride, QH, D)) != LYNX_OK) return rc;
    if (((uintptr_t)workspace & 255) != 0) return fail(LYNX_ERR_INVALID_ARG, "%s: the workspace must start on 256 bytes", who);
    const AttnSpace w = attention_space(B, T, QH, KVH, D);
    AttnParams p = {q, k_cache, v_cache, block_table, q_start, seq_len, prefix_table, out, lse, q_stride, out_stride, B, T, KVH, QH / KVH,
                    num_pages, max_pages, page_size, prefix_len, page_multiplier(page_size), scale * k_scale * kLog2e, v_scale,
                    window < kMaxContext ? window : 0, sinks < kMaxContext ? sinks : kMaxContext,   // (a window that long hides nothing)
                    w.parts, (float *)workspace, (float *)((char *)workspace + w.ml_off)};
    const bool f8 = cache_format == LYNX_CACHE_FP8;
    auto kernel = D == 128 ? (f8 ? attn_rows_kernel<128, true> : attn_rows_kernel<128, false>)
                           : (f8 ? attn_rows_kernel<64, true> : attn_rows_kernel<64, false>);
    const bool cut = max_pages * page_size > kMinChunk * kBlock;       // else no context is long enough
    hipLaunchKernelGGL(kernel, dim3(w.tiles + (cut ? w.parts : 0), KVH), dim3(kAttnThreads), 0, (hipStream_t)stream, p);
    if (cut) hipLaunchKernelGGL((D == 128 ? attn_join_kernel<128> : attn_join_kernel<64>), dim3(w.tiles < w.parts ? w.tiles : w.parts, KVH, kJoinSlices), dim3(kAttnThreads), 0, (hipStream_t)stream, p);
    return check_launch(who);
}

}  // namespace lynx

extern "C" size_t lynx_attention_workspace_bytes(int B, int T, int QH, int KVH, int D, int prefix_len)
{
    if (B <= 0 || T < 0 || QH <= 0 || KVH <= 0 || D <= 0 || prefix_len < 0) return 0;
    return lynx::attention_space(B, T, QH, KVH, D).total;
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
