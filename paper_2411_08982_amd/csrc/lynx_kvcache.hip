// The paged cache of a decode step: lynx_kv_assign (pages and slots of the step's tokens from request lengths) and
// lynx_qk_norm_rope (norms, rotation, write into the cache).
#include "lynx_attention.h"

namespace lynx {

// ---- lynx_kv_assign ---------------------------------------------------------------------------------------------------
// Prefix sums over at most 1024 requests say where each request's rows, new pages and returned pages begin; then every new
// page, returned page and token finds its request by bisection in the sums.  Nothing here is bound by bytes: one workgroup,
// one thread per request, and what counts is the number of round trips (64 requests of one token: 4.3 us; 1000 of 1 to 60: 5.3 us and
// 4.0 for the tokens).
constexpr int kAssignThreads = LYNX_MAX_REQUESTS;
// More tokens are left to a launch of their own (64 requests: 2048 tokens 5.7 us here, 6.5 apart; 4096 7.3 and 6.7; 8192 10.6 and 6.6).
constexpr int kTokensHere = 2048;

struct AssignShared {
    int tok_end[LYNX_MAX_REQUESTS], take_end[LYNX_MAX_REQUESTS], back_end[LYNX_MAX_REQUESTS];
    int ctx[LYNX_MAX_REQUESTS], have[LYNX_MAX_REQUESTS];
    int wave[3][kAssignThreads / kWave];
    int status;
};

// First of the n ascending sums that is larger than v.
__device__ __forceinline__ int owner_of(const int *sums, int n, int v)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] > v) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Inclusive prefix sums of three values over the workgroup.
__device__ __forceinline__ void scan3(AssignShared &sh, int (&v)[3])
{
    const int lane = lane_id(), wv = wave_id();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        v[i] = wave_prefix_sum_i32(v[i]);
        if (lane == kWave - 1) sh.wave[i][wv] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const int w = wave_prefix_sum_i32(lane < kAssignThreads / kWave ? sh.wave[i][lane] : 0);
        if (wv > 0) v[i] += __builtin_amdgcn_readlane(w, __builtin_amdgcn_readfirstlane(wv) - 1);
    }
}

struct AssignParams {
    const int32_t *ctx_len, *new_len, *ring_state;
    int32_t *block_table, *free_ring, *q_start, *seq_len, *positions, *slots, *ring_state_out, *status;
    int B, T, page_size, num_pages, max_pages, shared_pages;
    bool tokens_apart;
};

__device__ __forceinline__ void place_token(const AssignParams &p, int t, int r, int pos)
{
    const int page = p.block_table[(size_t)r * p.max_pages + pos / p.page_size];
    p.positions[t] = pos;
    p.slots[t] = page >= 0 && page < p.num_pages ? page * p.page_size + pos % p.page_size : -1;
}

__global__ __launch_bounds__(kAssignThreads) void assign_kernel(AssignParams p)
{
    __shared__ AssignShared sh;
    const int b = threadIdx.x;
    const int head = (int)((unsigned)p.ring_state[0] % (unsigned)p.num_pages);
    const int count = min(max(p.ring_state[1], 0), p.num_pages);
    const int cap = p.max_pages * p.page_size;
    int n = 0, have = 0, take = 0, back = 0, ctx = 0, bits = 0;
    bool ended = false;
    if (b == 0) sh.status = 0;
    if (b < p.B) {
        const int c = p.ctx_len[b], nw = p.new_len[b];
        ended = nw < 0;
        n = max(nw, 0);
        ctx = min(max(c, 0), cap);
        if (c != ctx || n > cap - ctx) {
            bits = LYNX_KV_TOO_LONG;
            n = 0;
            ended = false;
        }
        const int held = (ctx + p.page_size - 1) / p.page_size;
        have = max(held, p.shared_pages);
        take = min(max((ctx + n + p.page_size - 1) / p.page_size - have, 0), p.num_pages + 1);
        back = ended ? min(max(held - p.shared_pages, 0), p.num_pages + 1) : 0;
    }
    int v[3] = {min(n, p.T + 1), take, back};    // (bounded, so that 1024 of them stay below 2^31)
    scan3(sh, v);
    // The sums rise, so the requests that fit are those in front of the first that does not.
    const bool fits = b < p.B && v[0] <= p.T && v[1] <= count;
    if (b < p.B && n > 0 && !fits) bits |= (v[0] > p.T ? LYNX_KV_NO_ROWS : 0) | (v[1] > count ? LYNX_KV_NO_PAGES : 0);
    sh.tok_end[b] = v[0];
    sh.take_end[b] = v[1];
    const int fitted = __syncthreads_count(fits);
    const int rows = fitted > 0 ? sh.tok_end[fitted - 1] : 0, fresh = fitted > 0 ? sh.take_end[fitted - 1] : 0;
    __syncthreads();
    if (!fits) {
        n = 0;
        sh.tok_end[b] = rows;
        sh.take_end[b] = fresh;
    }
    sh.back_end[b] = v[2];
    sh.ctx[b] = ctx;
    sh.have[b] = have;
    if (bits) atomicOr(&sh.status, bits);
    if (b < p.B) {
        p.q_start[b] = fits ? v[0] - n : rows;
        p.seq_len[b] = ended ? 0 : ctx + n;
    }
    if (b == 0) p.q_start[p.B] = rows;
    __syncthreads();
    const int returned = min(sh.back_end[p.B - 1], p.num_pages - count);
    for (int j = b; j < fresh; j += kAssignThreads) {
        const int r = owner_of(sh.take_end, p.B, j);
        const int col = sh.have[r] + j - (r > 0 ? sh.take_end[r - 1] : 0);
        p.block_table[(size_t)r * p.max_pages + col] = p.free_ring[(head + j) % p.num_pages];
    }
    // (places behind the free pages: none of those that are taken above)
    for (int j = b; j < returned; j += kAssignThreads) {
        const int r = owner_of(sh.back_end, p.B, j);
        const int col = p.shared_pages + j - (r > 0 ? sh.back_end[r - 1] : 0);
        p.free_ring[(head + count + j) % p.num_pages] = p.block_table[(size_t)r * p.max_pages + col];
    }
    if (b == 0) {
        p.ring_state_out[0] = (head + fresh) % p.num_pages;
        p.ring_state_out[1] = count - fresh + returned;
        *p.status = sh.status | (sh.back_end[p.B - 1] > returned ? LYNX_KV_LOST_PAGES : 0);
    }
    if (p.tokens_apart) return;
    __syncthreads();   // the new entries of the block table
    for (int t = b; t < p.T; t += kAssignThreads) {
        if (t < rows) {
            const int r = owner_of(sh.tok_end, p.B, t);
            place_token(p, t, r, sh.ctx[r] + t - (r > 0 ? sh.tok_end[r - 1] : 0));
        } else {
            p.positions[t] = 0;
            p.slots[t] = -1;
        }
    }
}

// Positions and slots of many tokens, from what assign_kernel has written.
constexpr int kTokenThreads = 256;
__global__ __launch_bounds__(kTokenThreads) void assign_tokens_kernel(AssignParams p)
{
    __shared__ int ends[LYNX_MAX_REQUESTS];
    for (int b = threadIdx.x; b < p.B; b += kTokenThreads) ends[b] = p.q_start[b + 1];
    __syncthreads();
    const int t = blockIdx.x * kTokenThreads + threadIdx.x;
    if (t >= p.T) return;
    if (t < ends[p.B - 1]) {
        const int r = owner_of(ends, p.B, t);
        place_token(p, t, r, p.seq_len[r] - ends[r] + t);
    } else {
        p.positions[t] = 0;
        p.slots[t] = -1;
    }
}

// ---- lynx_qk_norm_rope ------------------------------------------------------------------------------------------------
// Workgroups of two kinds in one launch.  The first T have a token each, for its queries and keys: the angles are the same for all
// heads and computed once, into LDS; a head row is held by D/8 lanes, 8 channels (16 bytes) each.  The others turn 32 tokens' values
// of one key head over in LDS, since the cache has them transposed: where the tokens' slots follow one another, as a prompt's do, a
// channel's run of 16 bytes is one store.  (Element by element 8001 tokens with 8 key heads took 70 us, with 16 of 16 heads 141.)
// Bound by HBM: 8001 tokens, 32 query and 8 key heads, 197 MB: 39.2 us, 5.0 TB/s; with an 8-bit cache 180 MB: 43.8 us, 4.1 TB/s (its conversions,
// and its runs take 16 tokens); 32 tokens: 5.4 and 5.6 us of latency.
constexpr int kRopeThreads = 256;
// More at a time lose fewer runs at their borders, fewer have more workgroups (8 key heads; prompts that begin off a page: 8000 tokens
// 35.4 us by 32, by 16 37.7, by 64 36.3; 256 tokens 5.2 by 32, 4.7 by 16, 6.4 by 64).
constexpr int kTurnTokens = 32;
constexpr int kFewTokens = 1024;        // up to so many tokens 16 at a time

struct RopeParams {
    const uint16_t *q, *k, *v, *q_weight, *k_weight;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    const int32_t *positions, *slots;
    const double *freqs;
    uint16_t *q_out;
    void *k_cache, *v_cache;
    float eps, k_scale, v_scale;
    int rot, interleaved, T, QH, KVH, num_slots, page_size;
    int turn;                   // tokens of a workgroup for values: kTurnTokens or fewer
};

__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ uint4 pack8(const float (&x)[8])
{
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}

// (by comparisons: what is no number stays none, as in a bf16 cache; fmaxf and fminf would make it -448)
__device__ __forceinline__ float in_e4m3_range(float x) { return x > 448.0f ? 448.0f : x < -448.0f ? -448.0f : x; }

__device__ __forceinline__ uint2 pack8_fp8(const float (&x)[8], float scale)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = in_e4m3_range(__fdiv_rn(x[i], scale));
    int a = 0, b = 0;
    a = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], a, false);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], a, true);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], b, false);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], b, true);
    return make_uint2((unsigned)a, (unsigned)b);
}

// The values of up to kTurnTokens tokens of one key head into the cache.
template <int D, bool F8>
__device__ __forceinline__ void write_values(const RopeParams &p, int t0, int h, uint8_t *lds, uint8_t (&list)[2][kTurnTokens])
{
    constexpr int E = F8 ? 1 : 2;
    constexpr int RUN = 16 / E;                                  // tokens of a 16-byte run
    constexpr int kStride = kTurnTokens * E + 8;                 // bytes of a channel in LDS
    const int tid = threadIdx.x, lane = lane_id();
    // every wave for itself: lane i looks at token t0 + i
    const int slot = lane < p.turn && t0 + lane < p.T ? p.slots[t0 + lane] : -1;
    const bool valid = slot >= 0 && slot < p.num_slots;
    const int next = __shfl(slot, lane + 1);
    const unsigned long long follow = __ballot(valid && lane < kWave - 1 && next == slot + 1 && next < p.num_slots);
    // runs that begin at a token: its slot begins a run of the cache, and the next RUN - 1 tokens' follow
    const unsigned long long runs = __ballot(valid && slot % RUN == 0 && lane <= kTurnTokens - RUN && (follow >> lane & ((1ull << (RUN - 1)) - 1)) == (1ull << (RUN - 1)) - 1);
    unsigned long long covered = runs;
#pragma unroll
    for (int i = 1; i < RUN; i *= 2) covered |= covered << i;
    const unsigned long long single = __ballot(valid) & ~covered;
    // the tokens that begin runs, and those in none
    const unsigned long long before = (1ull << lane) - 1;
    if (tid < kWave) {
        if (runs >> lane & 1) list[0][__popcll(runs & before)] = (uint8_t)lane;
        if (single >> lane & 1) list[1][__popcll(single & before)] = (uint8_t)lane;
    }
    for (int i = tid; i < p.turn * (D / 8); i += kRopeThreads) {
        const int tok = i / (D / 8), c = i % (D / 8) * 8;
        if (t0 + tok >= p.T) break;
        const uint4 u = *reinterpret_cast<const uint4 *>(p.v + (size_t)(t0 + tok) * p.v_stride + (size_t)h * D + c);
        if (F8) {
            float x[8];
            unpack8(u, x);
            const uint2 w = pack8_fp8(x, p.v_scale);
#pragma unroll
            for (int j = 0; j < 8; ++j) lds[(c + j) * kStride + tok] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
        } else {
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) *reinterpret_cast<uint16_t *>(lds + (c + j) * kStride + tok * 2) = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
        }
    }
    __syncthreads();
    const int n = __popcll(runs);
    uint8_t *const cache = (uint8_t *)p.v_cache;
    const auto place = [&](int s, int d) {
        const int page = s / p.page_size;
        return cache + ((((size_t)page * p.KVH + h) * D + d) * p.page_size + (s - page * p.page_size)) * E;
    };
    // a channel's runs beside one another: they lie beside one another in the page
    for (int i = tid; i < n * D; i += kRopeThreads) {
        const int d = i / n, tok = list[0][i - d * n];
        const uint2 *src = reinterpret_cast<const uint2 *>(lds + d * kStride + tok * E);
        uint4 u;
        if (tok * E % 8 == 0) {
            const uint2 lo = src[0], hi = src[1];
            u = make_uint4(lo.x, lo.y, hi.x, hi.y);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[j] = 0;
#pragma unroll
                for (int e = 0; e < 4 / E; ++e) {
                    const uint8_t *q = lds + d * kStride + tok * E + j * 4 + e * E;
                    w[j] |= F8 ? (uint32_t)*q << (8 * e) : (uint32_t) * reinterpret_cast<const uint16_t *>(q) << (16 * e);
                }
            }
            u = make_uint4(w[0], w[1], w[2], w[3]);
        }
        *reinterpret_cast<uint4 *>(place(p.slots[t0 + tok], d)) = u;
    }
    const int ns = __popcll(single);
    for (int i = tid; i < ns * D; i += kRopeThreads) {
        const int tok = list[1][i / D], d = i % D;
        uint8_t *dst = place(p.slots[t0 + tok], d);
        if (F8) *dst = lds[d * kStride + tok];
        else *reinterpret_cast<uint16_t *>(dst) = *reinterpret_cast<const uint16_t *>(lds + d * kStride + tok * 2);
    }
}

template <int D, bool F8>
__global__ __launch_bounds__(kRopeThreads) void norm_rope_kernel(RopeParams p)
{
    constexpr int L = D / 8;                    // lanes of a row
    constexpr int R = kRopeThreads / L;         // rows of a pass
    __shared__ __align__(16) uint8_t turned[D * (kTurnTokens * (F8 ? 1 : 2) + 8)];
    __shared__ uint8_t list[2][kTurnTokens];
    float *const sc = reinterpret_cast<float *>(turned), *const ss = sc + D / 2;
    const int tid = threadIdx.x;
    if ((int)blockIdx.x >= p.T) {
        const int i = blockIdx.x - p.T;
        write_values<D, F8>(p, i / p.KVH * p.turn, i % p.KVH, turned, list);
        return;
    }
    const int t = blockIdx.x;
    const int half = p.rot / 2;
    if (tid < half) {
        // turns, reduced to [-1/2, 1/2] in 64 bits
        const double turns = (double)p.positions[t] * (p.freqs[tid] * 0.15915494309189533577);
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        sc[tid] = c;
        ss[tid] = s;
    }
    __syncthreads();
    const int slot = p.slots[t];
    const bool keep = slot >= 0 && slot < p.num_slots;
    const int page = keep ? slot / p.page_size : 0, place = keep ? slot % p.page_size : 0;
    const int c0 = (tid % L) * 8;
    for (int row = tid / L; row < p.QH + p.KVH; row += R) {
        const bool is_q = row < p.QH;
        const int h = is_q ? row : row - p.QH;
        const uint16_t *src = is_q ? p.q + t * p.q_stride : p.k + t * p.k_stride;
        float x[8];
        unpack8(*reinterpret_cast<const uint4 *>(src + (size_t)h * D + c0), x);
        {
            const uint16_t *w = is_q ? p.q_weight : p.k_weight;
            if (w) {
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
#pragma unroll
                for (int m = 1; m < L; m <<= 1) sum += __shfl_xor(sum, m);
                const float r = 1.0f / sqrtf(sum / (float)D + p.eps);
                float wf[8];
                unpack8(*reinterpret_cast<const uint4 *>(w + c0), wf);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = x[i] * r * wf[i];
            }
            if (p.interleaved) {
                if (c0 < p.rot) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float c = sc[c0 / 2 + i], s = ss[c0 / 2 + i], a = x[2 * i], b = x[2 * i + 1];
                        x[2 * i] = a * c - b * s;
                        x[2 * i + 1] = b * c + a * s;
                    }
                }
            } else {
                // the other channel of each pair is rot/2 away: rot/16 lanes
                const bool first = c0 < half;
                const int partner = lane_id() + (first ? half / 8 : -(half / 8));
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = __shfl(x[i], partner);
                if (c0 < p.rot) {
                    const int f0 = first ? c0 : c0 - half;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float c = sc[f0 + i], s = ss[f0 + i];
                        x[i] = first ? x[i] * c - y[i] * s : x[i] * c + y[i] * s;
                    }
                }
            }
        }
        if (is_q) {
            *reinterpret_cast<uint4 *>(p.q_out + t * p.q_out_stride + (size_t)h * D + c0) = pack8(x);
        } else if (keep) {
            const size_t at = (((size_t)page * p.KVH + h) * p.page_size + place) * D + c0;
            if (F8) *reinterpret_cast<uint2 *>((uint8_t *)p.k_cache + at) = pack8_fp8(x, p.k_scale);
            else *reinterpret_cast<uint4 *>((uint16_t *)p.k_cache + at) = pack8(x);
        }
    }
}

// Checks of the cache that lynx_qk_norm_rope and the attention calls share.
int check_cache(const char *who, const void *k_cache, const void *v_cache, int cache_format, float k_scale, float v_scale,
                int num_pages, int page_size, int QH, int KVH, int D)
{
    if (QH <= 0 || KVH <= 0 || QH % KVH != 0) return fail(LYNX_ERR_INVALID_ARG, "%s: KVH must divide QH, both > 0", who);
    if (num_pages <= 0 || page_size <= 0) return fail(LYNX_ERR_INVALID_ARG, "%s: negative or zero size", who);
    if (cache_format != LYNX_CACHE_BF16 && cache_format != LYNX_CACHE_FP8)
        return fail(LYNX_ERR_INVALID_ARG, "%s: cache_format must be LYNX_CACHE_BF16 or LYNX_CACHE_FP8", who);
    if (!(k_scale > 0.0f) || !(v_scale > 0.0f) || k_scale > 3.0e38f || v_scale > 3.0e38f)
        return fail(LYNX_ERR_INVALID_ARG, "%s: scales must be finite and > 0", who);
    if (cache_format == LYNX_CACHE_BF16 && (k_scale != 1.0f || v_scale != 1.0f))
        return fail(LYNX_ERR_INVALID_ARG, "%s: a bf16 cache has no scales (pass 1)", who);
    if ((D != 64 && D != 128) || QH > kMaxHeads || QH / KVH > kMaxGroup || page_size % 16 != 0 ||
        page_size > LYNX_MAX_PAGE_SIZE || num_pages > LYNX_MAX_PAGES)
        return fail(LYNX_ERR_UNSUPPORTED, "%s: need D=64 or 128, QH<=%d, QH/KVH<=%d, page_size%%16==0, page_size<=%d, num_pages<=%d",
                    who, kMaxHeads, kMaxGroup, LYNX_MAX_PAGE_SIZE, LYNX_MAX_PAGES);
    if (!k_cache || !v_cache) return fail(LYNX_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned16(k_cache) || !aligned16(v_cache)) return fail(LYNX_ERR_INVALID_ARG, "%s: the cache must start on 16 bytes", who);
    return LYNX_OK;
}

// A [T][heads][D] array whose tokens lie `stride` elements apart.
int check_rows(const char *who, const char *what, const void *ptr, int64_t stride, int heads, int D)
{
    if (!ptr) return fail(LYNX_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!aligned16(ptr) || stride % 8 != 0 || stride < (int64_t)heads * D || stride > ((int64_t)1 << 40))
        return fail(LYNX_ERR_INVALID_ARG, "%s: %s must start on 16 bytes, its stride be a multiple of 8 and hold a token's heads", who, what);
    return LYNX_OK;
}

}  // namespace lynx

extern "C" int lynx_kv_assign(const int32_t *ctx_len, const int32_t *new_len, int B, int T, int page_size, int num_pages,
                              int max_pages, int shared_pages, int32_t *block_table, int32_t *free_ring,
                              const int32_t *ring_state, int32_t *q_start, int32_t *seq_len, int32_t *positions, int32_t *slots,
                              int32_t *ring_state_out, int32_t *status, void *stream)
{
    using namespace lynx;
    if (B <= 0 || T < 0 || page_size <= 0 || num_pages <= 0 || max_pages <= 0 || shared_pages < 0 || shared_pages > max_pages)
        return fail(LYNX_ERR_INVALID_ARG, "lynx_kv_assign: negative or zero size, or more shared pages than a row holds");
    if (B > LYNX_MAX_REQUESTS || T > LYNX_MAX_STEP_TOKENS || page_size % 16 != 0 || page_size > LYNX_MAX_PAGE_SIZE ||
        num_pages > LYNX_MAX_PAGES || max_pages > kMaxContext / page_size)
        return fail(LYNX_ERR_UNSUPPORTED, "lynx_kv_assign: need B<=%d, T<=%d, page_size%%16==0, page_size<=%d, num_pages<=%d, max_pages*page_size<=%d",
                    LYNX_MAX_REQUESTS, LYNX_MAX_STEP_TOKENS, LYNX_MAX_PAGE_SIZE, LYNX_MAX_PAGES, kMaxContext);
    if (!ctx_len || !new_len || !block_table || !free_ring || !ring_state || !q_start || !seq_len || !ring_state_out || !status ||
        (T > 0 && (!positions || !slots)))
        return fail(LYNX_ERR_INVALID_ARG, "lynx_kv_assign: null pointer");
    AssignParams p = {ctx_len, new_len, ring_state, block_table, free_ring, q_start, seq_len, positions, slots, ring_state_out,
                      status, B, T, page_size, num_pages, max_pages, shared_pages, T > kTokensHere};
    hipLaunchKernelGGL(assign_kernel, dim3(1), dim3(kAssignThreads), 0, (hipStream_t)stream, p);
    if (p.tokens_apart)
        hipLaunchKernelGGL(assign_tokens_kernel, dim3((T + kTokenThreads - 1) / kTokenThreads), dim3(kTokenThreads), 0, (hipStream_t)stream, p);
    return check_launch("lynx_kv_assign");
}

extern "C" int lynx_qk_norm_rope(const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride, const uint16_t *v,
                                 int64_t v_stride, const uint16_t *q_weight, const uint16_t *k_weight, float eps,
                                 const int32_t *positions, const int32_t *slots, const double *freqs, int rot, int interleaved,
                                 int T, int QH, int KVH, int D, uint16_t *q_out, int64_t q_out_stride, void *k_cache,
                                 void *v_cache, int cache_format, float k_scale, float v_scale, int num_pages, int page_size,
                                 void *stream)
{
    using namespace lynx;
    const char *who = "lynx_qk_norm_rope";
    if (T < 0) return fail(LYNX_ERR_INVALID_ARG, "%s: negative or zero size", who);
    int rc = check_cache(who, k_cache, v_cache, cache_format, k_scale, v_scale, num_pages, page_size, QH, KVH, D);
    if (rc != LYNX_OK) return rc;
    if (T > LYNX_MAX_STEP_TOKENS) return fail(LYNX_ERR_UNSUPPORTED, "%s: need T<=%d", who, LYNX_MAX_STEP_TOKENS);
    if (rot < 0 || rot > D || rot % 16 != 0) return fail(LYNX_ERR_INVALID_ARG, "%s: rot must be a multiple of 16 up to D", who);
    if (!(eps >= 0.0f) || eps > 3.0e38f) return fail(LYNX_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", who);
    if (T == 0) return LYNX_OK;
    if (!positions || !slots || (rot > 0 && !freqs)) return fail(LYNX_ERR_INVALID_ARG, "%s: null pointer", who);
    if ((q_weight && !aligned16(q_weight)) || (k_weight && !aligned16(k_weight)))
        return fail(LYNX_ERR_INVALID_ARG, "%s: the weights must start on 16 bytes", who);
    if ((rc = check_rows(who, "q", q, q_stride, QH, D)) != LYNX_OK || (rc = check_rows(who, "k", k, k_stride, KVH, D)) != LYNX_OK ||
        (rc = check_rows(who, "v", v, v_stride, KVH, D)) != LYNX_OK ||
        (rc = check_rows(who, "q_out", q_out, q_out_stride, QH, D)) != LYNX_OK)
        return rc;
    RopeParams p = {q, k, v, q_weight, k_weight, q_stride, k_stride, v_stride, q_out_stride, positions, slots, freqs, q_out, k_cache,
                    v_cache, eps, k_scale, v_scale, rot, interleaved ? 1 : 0, T, QH, KVH, num_pages * page_size, page_size,
                    T <= kFewTokens ? 16 : kTurnTokens};
    const bool f8 = cache_format == LYNX_CACHE_FP8;
    auto kernel = D == 128 ? (f8 ? norm_rope_kernel<128, true> : norm_rope_kernel<128, false>)
                           : (f8 ? norm_rope_kernel<64, true> : norm_rope_kernel<64, false>);
    hipLaunchKernelGGL(kernel, dim3(T + (T + p.turn - 1) / p.turn * KVH), dim3(kRopeThreads), 0, (hipStream_t)stream, p);
    return check_launch(who);
}
