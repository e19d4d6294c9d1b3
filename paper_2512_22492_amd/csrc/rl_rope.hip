// rl_rope.hip -- KV-cache append with the position rotation applied on the way:
// one token or several per sequence, bf16 or e4m3 pages.

#include <type_traits>

#include "rl_e4m3.h"
#include "rl_tile.h"

using namespace rl_da;

namespace {

// ------------------------------------------------- rotate and append ---
//
// A new token's head row x (128 values) goes through
//     x <- x / sqrt(mean(x^2) + eps) * w            (query and key rows, optional)
//     (a, b) <- (a c - b s, b c + a s)              (query and key rows)
// over the pairs of its first rotary_dim dims, c and s the caller's cosine and sine
// of the token's position, and is rounded once, to bf16 (queries, bf16 pages) or to
// e4m3 codes.  Everything before that rounding is fp32.
//
// 16 lanes hold a row, eight consecutive dims each (one 16-byte load): sums and
// maxima over a row are DPP operations, and the partner of a half-split pair
// sits in another lane of the row (a DPP rotation by eight lanes when the whole
// head is rotated).  There is almost no arithmetic: the rows are read once and
// written once, so HBM bounds prompts, and launch and load latency single tokens.

constexpr int kRowLanes = 16;
constexpr int kRopeThreads = 256;
constexpr int kRopeRows = kRopeThreads / kRowLanes;  // rows in flight per work-group
constexpr int kLaneDims = kHeadDim / kRowLanes;
static_assert(kRopeRows == kPageSize, "a work-group's rows are the slots of a page");
// Calls of up to so many tokens per sequence go by tokens and head rows instead of pages,
// most of whose sixteen slots they would leave idle.  512 sequences x 48 head rows, us by
// pages and so: bf16, two tokens 38 and 10.6, eight 43 and 21, twelve 45 and 37, sixteen
// 46 and 49; e4m3, whose form holds a page's tokens in registers, two 60 and 12, eight
// 65 and 25.
constexpr int kFewTokens = 8, kFewTokensBf16 = 12;
constexpr int kAhead = 6;  // head rows that a thread of rope_append_pages has in flight
constexpr int kDppRowRor8 = 0x128;

struct RopeArgs {
    const uint16_t* q;          // bf16, head rows contiguous, token strides in elements
    const uint16_t* k_new;
    const uint16_t* v_new;
    int64_t q_stride;
    int64_t k_stride;
    int64_t v_stride;
    const int32_t* q_start;     // [B+1], or null: one token per sequence
    const float* cos_sin;       // [num_positions][rotary_dim]: cosines, then sines
    const uint16_t* q_norm;     // bf16 [D], or null
    const uint16_t* k_norm;
    uint16_t* q_out;            // bf16 [T][Hq][D]
    uint8_t* k_pool;
    uint8_t* v_pool;
    float* k_scale;             // [P][Hkv], e4m3 pools only
    float* v_scale;
    const int32_t* block_table;
    const int32_t* seq_lens;    // before the append
    int32_t* dev_error;         // may be null
    int64_t num_pages;
    int64_t page_bytes;         // pool strides in bytes: per page,
    int32_t head_bytes;         //   per kv head within a page,
    int32_t row_bytes;          //   per token slot within a slab
    int32_t num_q_heads;
    int32_t num_kv_heads;
    int32_t max_pages;
    int32_t num_positions;
    int32_t rotary_dim;
    float norm_eps;
    int32_t parts;              // work-groups that share a sequence's (page's) head rows
    int32_t tiles;              // a sequence's new tokens, or the pages they may touch
};

__device__ __forceinline__ void report(const RopeArgs& a, int32_t bits)
{
    if (a.dev_error != nullptr)
        atomicOr(a.dev_error, bits);
}

// A lane's cosines and sines: dims 8j..8j+7 of the row (of no use to lanes past
// rotary_dim).  Loads without branches: a branch around a load waits for it at its end.
struct Turn {
    float c[kLaneDims], s[kLaneDims];
};

template <bool INTERLEAVED>
__device__ __forceinline__ void load_turn(const RopeArgs& a, int pos, int j, Turn& t)
{
    const int half = a.rotary_dim / 2;
    const bool low = kLaneDims * j < half;
    // dims 2i, 2i + 1 turn by angle i, or dims i, i + half
    const int dim = kLaneDims * j < a.rotary_dim ? kLaneDims * j : 0;
    const int at = INTERLEAVED ? dim / 2 : (dim >= half ? dim - half : dim);
    const float* row = a.cos_sin + (int64_t)pos * a.rotary_dim + at;
    float c[kLaneDims], s[kLaneDims];
#pragma unroll
    for (int v = 0; v < (INTERLEAVED ? 1 : 2); ++v) {
        const float4 x = *reinterpret_cast<const float4*>(row + 4 * v);
        const float4 y = *reinterpret_cast<const float4*>(row + half + 4 * v);
        c[4 * v] = x.x, c[4 * v + 1] = x.y, c[4 * v + 2] = x.z, c[4 * v + 3] = x.w;
        s[4 * v] = y.x, s[4 * v + 1] = y.y, s[4 * v + 2] = y.z, s[4 * v + 3] = y.w;
    }
#pragma unroll
    for (int i = 0; i < kLaneDims; ++i) {
        t.c[i] = c[INTERLEAVED ? i / 2 : i];
        const float sine = s[INTERLEAVED ? i / 2 : i];
        t.s[i] = (INTERLEAVED ? i % 2 == 0 : low) ? -sine : sine;
    }
}

// Norm and rotation of the row that 16 lanes hold.
template <bool INTERLEAVED>
__device__ __forceinline__ void turn_row(const RopeArgs& a, const uint16_t* norm,
                                         const float (&w)[kLaneDims], const Turn& t, int j,
                                         float (&x)[kLaneDims])
{
    if (norm != nullptr) {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < kLaneDims; ++i)
            ss = fmaf(x[i], x[i], ss);
        const float r = 1.0f / sqrtf(row16_sum(ss) * (1.0f / kHeadDim) + a.norm_eps);
#pragma unroll
        for (int i = 0; i < kLaneDims; ++i)
            x[i] = x[i] * r * w[i];
    }
    if (!INTERLEAVED && a.rotary_dim == kHeadDim) {
#pragma unroll
        for (int i = 0; i < kLaneDims; ++i) {
            const float other = __int_as_float(__builtin_amdgcn_update_dpp(
                0, __float_as_int(x[i]), kDppRowRor8, 0xf, 0xf, true));
            x[i] = fmaf(x[i], t.c[i], other * t.s[i]);
        }
        return;
    }
    float other[kLaneDims];
    const int step = a.rotary_dim / 2 / kLaneDims;
    const int from = j < step ? j + step : j - step;
#pragma unroll
    for (int i = 0; i < kLaneDims; ++i)
        other[i] = INTERLEAVED ? x[i ^ 1] : __shfl(x[i], from & (kRowLanes - 1), kRowLanes);
    // a lane past rotary_dim keeps its values, whatever its partner holds
    if (kLaneDims * j < a.rotary_dim) {
#pragma unroll
        for (int i = 0; i < kLaneDims; ++i)
            x[i] = fmaf(x[i], t.c[i], other[i] * t.s[i]);
    }
}

__device__ __forceinline__ uint4 pack8(const float (&x)[kLaneDims])
{
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                      pack_bf16x2(x[6], x[7]));
}

// A store with the non-temporal hint: the queries of a prompt are more than the caches
// hold until they are read (50k tokens: 257 us without the hints, 246 with).
__device__ __forceinline__ void store_stream16(uint16_t* p, const uint4& v)
{
    __builtin_nontemporal_store(u32x4_t{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4_t*>(p));
}

__device__ __forceinline__ float absmax8(const float (&x)[kLaneDims])
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kLaneDims; ++i)
        m = fmaxf(m, fabsf(x[i]));
    return m;
}

// Quotients by one divisor d, rounded as a / d is: with r = 1 / d rounded to nearest and
// q = a r, q + (a - q d) r is the correctly rounded quotient (P. Markstein,
// "Computation of elementary functions on the IBM RISC System/6000 processor", IBM J.
// Res. Dev. 34, 1990), three operations an element, as long as nothing leaves the
// normal range: kScaleLow <= d <= kScaleHigh keeps every a that an e4m3 code tells
// from zero, and its remainder, far inside it.  What it loses is the sign of a zero (-0 r
// + 0 is +0) and of a NaN, which the division keeps, and so does a copy of a's sign.
constexpr float kScaleLow = 0x1p-60f, kScaleHigh = 0x1p60f;

// A row at its slab's scale.  The scale is at least absmax / 448 rounded, so that an
// element exceeds 448 by a rounding at most, which e4m3's rounding removes; scales so
// small that their own rounding is coarse take the division and the clamp.
__device__ __forceinline__ uint2 encode8(const float (&x)[kLaneDims], float scale)
{
    float y[kLaneDims];
    if (scale >= kScaleLow && scale <= kScaleHigh) {
        const float r = 1.0f / scale;
#pragma unroll
        for (int i = 0; i < kLaneDims; ++i) {
            const float q = x[i] * r;
            y[i] = copysignf(fmaf(fmaf(-q, scale, x[i]), r, q), x[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kLaneDims; ++i)
            y[i] = clamp448(x[i] / scale);
    }
    return make_uint2(e4m3_pair(y[0], y[1]) | (e4m3_pair(y[2], y[3]) << 16),
                      e4m3_pair(y[4], y[5]) | (e4m3_pair(y[6], y[7]) << 16));
}

// Eight codes at a scale that has grown by 1 / ratio.
__device__ __forceinline__ uint2 shrink8(uint2 c, float ratio)
{
    auto word = [&](uint32_t w) {
        const floatx2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
        const floatx2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
        return e4m3_pair(lo.x * ratio, lo.y * ratio) |
               (e4m3_pair(hi.x * ratio, hi.y * ratio) << 16);
    };
    return make_uint2(word(c.x), word(c.y));
}

// A slab's scale once values of magnitude absmax join it; `old`: it holds
// earlier tokens, at scale was.
__device__ __forceinline__ float joined_scale(float absmax, bool old, float was)
{
    const float wanted = absmax > 0.0f ? absmax / 448.0f : 1.0f;
    return old && !(wanted > was) ? was : wanted;
}

// Which rows a head index stands for: query heads, then keys, then values.
struct HeadRow {
    bool is_q, is_v;
    int head;
};

__device__ __forceinline__ HeadRow head_row(const RopeArgs& a, int at)
{
    HeadRow r;
    r.is_q = at < a.num_q_heads;
    r.is_v = at >= a.num_q_heads + a.num_kv_heads;
    r.head = r.is_q ? at : at - a.num_q_heads - (r.is_v ? a.num_kv_heads : 0);
    return r;
}

__device__ __forceinline__ const uint16_t* row_source(const RopeArgs& a, const HeadRow& r,
                                                      int64_t token)
{
    const uint16_t* base = r.is_q ? a.q + token * a.q_stride
                                  : (r.is_v ? a.v_new + token * a.v_stride
                                            : a.k_new + token * a.k_stride);
    return base + r.head * kHeadDim;
}

// One token per sequence, or into bf16 pages, where nothing joins the tokens of a page,
// a few: 16 head rows of one token per work-group, `parts` work-groups per token and
// `tiles` tokens per sequence.
template <bool FP8, bool INTERLEAVED>
__global__ __launch_bounds__(kRopeThreads) void rope_append_token(RopeArgs a)
{
    const int step = (int)(blockIdx.x / a.parts) % a.tiles;
    const int b = (int)(blockIdx.x / a.parts) / a.tiles;
    const int at = (int)(blockIdx.x % a.parts) * kRopeRows + threadIdx.x / kRowLanes;
    const int j = threadIdx.x % kRowLanes;
    if (at >= a.num_q_heads + 2 * a.num_kv_heads)
        return;
    const int before = a.seq_lens[b];
    int64_t token = b;
    if (a.q_start != nullptr) {
        token = (int64_t)a.q_start[b] + step;
        if (a.q_start[b + 1] <= token)
            return;
    }
    // A token that has no place is left out at the end, and its reads go to position 0: the
    // row is read beside the length, and the page beside the cosines.
    const HeadRow r = head_row(a, at);
    const uint4 bits = *reinterpret_cast<const uint4*>(row_source(a, r, token) + kLaneDims * j);
    const uint16_t* norm = r.is_q ? a.q_norm : (r.is_v ? nullptr : a.k_norm);
    const uint4 weight = *reinterpret_cast<const uint4*>(
        norm != nullptr ? norm + kLaneDims * j : row_source(a, r, token) + kLaneDims * j);
    const int64_t L = before + (int64_t)step;
    const bool fits = L < a.max_pages * kPageSize && L < a.num_positions;
    const int pos = fits && before >= 0 ? (int)L : 0;
    const int32_t page = a.block_table[(int64_t)b * a.max_pages + pos / kPageSize];
    Turn t;
    load_turn<INTERLEAVED>(a, pos, j, t);
    float x[kLaneDims], w[kLaneDims];
    unpack8(bits, x);
    unpack8(weight, w);
    turn_row<INTERLEAVED>(a, norm, w, t, j, x);
    if (r.is_v)
        unpack8(bits, x);
    const bool in_pool = page >= 0 && (int64_t)page < a.num_pages;
    if (before < 0 || !fits || !in_pool) {
        if (before >= 0 && j == 0 && at == 0)
            report(a, fits ? RL_DA_DEVERR_PAGE_OUT_OF_RANGE : RL_DA_DEVERR_LENGTH_TOO_LONG);
        return;
    }
    if (r.is_q) {
        *reinterpret_cast<uint4*>(a.q_out + (token * a.num_q_heads + r.head) * kHeadDim +
                                  kLaneDims * j) = pack8(x);
        return;
    }
    const int slot = pos % kPageSize;
    uint8_t* codes = (r.is_v ? a.v_pool : a.k_pool) + page * a.page_bytes +
                     (int64_t)r.head * a.head_bytes;
    if (!FP8) {
        *reinterpret_cast<uint4*>(codes + (int64_t)slot * a.row_bytes + 16 * j) =
            r.is_v ? bits : pack8(x);
        return;
    }
    float* scale = (r.is_v ? a.v_scale : a.k_scale) + (int64_t)page * a.num_kv_heads + r.head;
    const float was = *scale;
    const float now = joined_scale(row16_max(absmax8(x)), slot != 0, was);
    if (slot != 0 && now != was) {  // the slab's earlier tokens at the grown scale
        for (int s = 0; s < slot; ++s) {
            uint2* c = reinterpret_cast<uint2*>(codes + (int64_t)s * a.row_bytes + 8 * j);
            *c = shrink8(*c, was / now);
        }
    }
    *reinterpret_cast<uint2*>(codes + (int64_t)slot * a.row_bytes + 8 * j) = encode8(x, now);
    if (j == 0)
        *scale = now;
}

// A few tokens per sequence into e4m3 pages: sixteen lanes take one head row of all the
// new tokens of one page that they touch, at most kFewTokens, and hold them until the
// slab's largest magnitude is known.  The bits are rope_append_pages'.
template <bool INTERLEAVED>
__global__ __launch_bounds__(kRopeThreads) void rope_append_few(RopeArgs a)
{
    const int part = blockIdx.x % a.parts;
    const int tile = (int)(blockIdx.x / a.parts) % a.tiles;
    const int b = (int)(blockIdx.x / a.parts) / a.tiles;
    const int at = part * kRopeRows + threadIdx.x / kRowLanes;
    const int j = threadIdx.x % kRowLanes;
    const int L = a.seq_lens[b];
    const int64_t token0 = a.q_start[b];
    const int n = (int)(a.q_start[b + 1] - token0);
    if (L < 0 || n <= 0)
        return;
    const int64_t end = (int64_t)L + n;
    const int64_t col = L / kPageSize + tile;  // page of the sequence
    if (col * kPageSize >= end)
        return;
    const bool first = threadIdx.x == 0 && part == 0;
    const int64_t cap = min((int64_t)a.max_pages * kPageSize, (int64_t)a.num_positions);
    if (first && min(end, (col + 1) * kPageSize) > cap)
        report(a, RL_DA_DEVERR_LENGTH_TOO_LONG);
    const int64_t from = max((int64_t)L, col * kPageSize);  // first position in this page
    if (from >= cap)
        return;
    const int32_t page = a.block_table[(int64_t)b * a.max_pages + col];
    if (page < 0 || (int64_t)page >= a.num_pages) {
        if (first)
            report(a, RL_DA_DEVERR_PAGE_OUT_OF_RANGE);
        return;
    }
    if (at >= a.num_q_heads + 2 * a.num_kv_heads)
        return;
    const int live = (int)(min(min(end, cap), (col + 1) * kPageSize) - from);
    const int64_t token = token0 + (from - L);
    const HeadRow r = head_row(a, at);
    const uint16_t* norm = r.is_q ? a.q_norm : (r.is_v ? nullptr : a.k_norm);
    float w[kLaneDims] = {};
    if (norm != nullptr)
        unpack8(*reinterpret_cast<const uint4*>(norm + kLaneDims * j), w);
    uint4 bits[kFewTokens];
#pragma unroll
    for (int i = 0; i < kFewTokens; ++i)  // past the last token its row again
        bits[i] = *reinterpret_cast<const uint4*>(
            row_source(a, r, token + min(i, live - 1)) + kLaneDims * j);
    float x[kFewTokens][kLaneDims], m = 0.0f;
#pragma unroll
    for (int i = 0; i < kFewTokens; ++i) {
        if (i >= live)
            break;
        unpack8(bits[i], x[i]);
        if (!r.is_v) {
            Turn t;
            load_turn<INTERLEAVED>(a, (int)from + i, j, t);
            turn_row<INTERLEAVED>(a, norm, w, t, j, x[i]);
        }
        if (r.is_q)
            *reinterpret_cast<uint4*>(a.q_out +
                                      ((token + i) * a.num_q_heads + r.head) * kHeadDim +
                                      kLaneDims * j) = pack8(x[i]);
        m = fmaxf(m, absmax8(x[i]));
    }
    if (r.is_q)
        return;
    const int held = tile == 0 ? L % kPageSize : 0;  // slots of earlier tokens
    uint8_t* codes = (r.is_v ? a.v_pool : a.k_pool) + page * a.page_bytes +
                     (int64_t)r.head * a.head_bytes + 8 * j;
    float* scale = (r.is_v ? a.v_scale : a.k_scale) + (int64_t)page * a.num_kv_heads + r.head;
    const float was = *scale;
    const float now = joined_scale(row16_max(m), held > 0, was);
    if (now != was) {  // the slab's earlier tokens at the grown scale
        for (int s = 0; s < held; ++s) {
            uint2* c = reinterpret_cast<uint2*>(codes + (int64_t)s * a.row_bytes);
            *c = shrink8(*c, was / now);
        }
    }
#pragma unroll
    for (int i = 0; i < kFewTokens; ++i)
        if (i < live)
            *reinterpret_cast<uint2*>(codes + (from % kPageSize + i) * a.row_bytes) =
                encode8(x[i], now);
    if (j == 0)
        *scale = now;
}

// Several tokens per sequence: a work-group for one page that a sequence's new
// tokens touch, its 16 rows the page's slots, and a part of the head rows, which
// it walks one after another: a row's cosines and sines are read once for all of
// them, and an e4m3 slab's new tokens meet in one work-group, so its scale
// grows once and its earlier codes are rounded once.
template <bool FP8, bool INTERLEAVED>
__global__ __launch_bounds__(kRopeThreads) void rope_append_pages(RopeArgs a)
{
    __shared__ float top[2][kAhead][kRopeThreads / kWave];
    const int part = blockIdx.x % a.parts;
    const int tile = (int)(blockIdx.x / a.parts) % a.tiles;
    const int b = (int)(blockIdx.x / a.parts) / a.tiles;
    const int slot = threadIdx.x / kRowLanes;
    const int j = threadIdx.x % kRowLanes;
    const int L = a.seq_lens[b];
    const int64_t token0 = a.q_start[b];
    const int n = (int)(a.q_start[b + 1] - token0);
    if (L < 0 || n <= 0)
        return;
    const int64_t end = (int64_t)L + n;
    const int64_t col = L / kPageSize + tile;  // page of the sequence
    if (col * kPageSize >= end)
        return;
    const bool first = threadIdx.x == 0 && part == 0;
    const int64_t cap = min((int64_t)a.max_pages * kPageSize, (int64_t)a.num_positions);
    if (first && min(end, (col + 1) * kPageSize) > cap)
        report(a, RL_DA_DEVERR_LENGTH_TOO_LONG);
    // a page without a token that counts keeps its scales as they are
    if (max((int64_t)L, col * kPageSize) >= cap)
        return;
    const int32_t page = a.block_table[(int64_t)b * a.max_pages + col];
    if (page < 0 || (int64_t)page >= a.num_pages) {
        if (first)
            report(a, RL_DA_DEVERR_PAGE_OUT_OF_RANGE);
        return;
    }
    const int pos = (int)col * kPageSize + slot;  // under cap + 16
    const bool live = pos >= L && pos < min(end, cap);
    const int64_t token = token0 + (live ? pos - L : 0);
    const int held = tile == 0 ? L % kPageSize : 0;  // slots of earlier tokens
    const int64_t row_at = page * a.page_bytes + (int64_t)slot * a.row_bytes;
    Turn t;
    load_turn<INTERLEAVED>(a, live ? pos : 0, j, t);
    float wq[kLaneDims] = {}, wk[kLaneDims] = {};
    if (a.q_norm != nullptr) {
        unpack8(*reinterpret_cast<const uint4*>(a.q_norm + kLaneDims * j), wq);
        unpack8(*reinterpret_cast<const uint4*>(a.k_norm + kLaneDims * j), wk);
    }

    // kAhead head rows are read side by side (50k prompt tokens of 48 head rows, bf16 and
    // e4m3: four 245 and 349 us, six 241 and 244, eight 246 and 282; one at a time and
    // without the parts 296 and 310), and an e4m3 round's slabs share a barrier.
    const int heads = a.num_q_heads + 2 * a.num_kv_heads;
    const int first_kv = a.num_q_heads;
    int round = 0;
    for (int at0 = part * kAhead; at0 < heads; at0 += a.parts * kAhead, ++round) {
        uint4 bits[kAhead];
        float was[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const HeadRow r = head_row(a, min(at0 + i, heads - 1));
            bits[i] = make_uint4(0, 0, 0, 0);
            if (live)
                bits[i] = load_stream16(
                    reinterpret_cast<const uint8_t*>(row_source(a, r, token) + kLaneDims * j));
            was[i] = 1.0f;
            if (FP8 && !r.is_q)
                was[i] = (r.is_v ? a.v_scale : a.k_scale)[(int64_t)page * a.num_kv_heads + r.head];
        }
        float x[kAhead][kLaneDims];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (at0 + i >= heads)
                break;
            const HeadRow r = head_row(a, at0 + i);
            unpack8(bits[i], x[i]);
            if (r.is_q)
                turn_row<INTERLEAVED>(a, a.q_norm, wq, t, j, x[i]);
            else if (!r.is_v)
                turn_row<INTERLEAVED>(a, a.k_norm, wk, t, j, x[i]);
            if (r.is_q) {
                if (live)
                    store_stream16(a.q_out + (token * a.num_q_heads + r.head) * kHeadDim +
                                       kLaneDims * j,
                                   pack8(x[i]));
            } else if (!FP8) {
                if (live)
                    *reinterpret_cast<uint4*>((r.is_v ? a.v_pool : a.k_pool) + row_at +
                                              (int64_t)r.head * a.head_bytes + 16 * j) =
                        r.is_v ? bits[i] : pack8(x[i]);
            } else {
                // the largest magnitude of the slab's new tokens (idle rows count nothing)
                const float m = max_lanes_xor32(
                    max_lanes_xor16(row16_max(live ? absmax8(x[i]) : 0.0f)));
                if (threadIdx.x % kWave == 0)
                    top[round & 1][i][threadIdx.x / kWave] = m;
            }
        }
        if (!FP8 || at0 + kAhead <= first_kv)
            continue;
        __syncthreads();  // also: the scales are read by all rows before one writes them
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (at0 + i >= heads)
                break;
            if (at0 + i < first_kv)
                continue;
            const HeadRow r = head_row(a, at0 + i);
            float m = 0.0f;
#pragma unroll
            for (int w = 0; w < kRopeThreads / kWave; ++w)
                m = fmaxf(m, top[round & 1][i][w]);
            const float now = joined_scale(m, held > 0, was[i]);
            uint8_t* row = (r.is_v ? a.v_pool : a.k_pool) + row_at +
                           (int64_t)r.head * a.head_bytes + 8 * j;
            if (live) {
                *reinterpret_cast<uint2*>(row) = encode8(x[i], now);
            } else if (slot < held && now != was[i]) {
                uint2* c = reinterpret_cast<uint2*>(row);
                *c = shrink8(*c, was[i] / now);
            }
            if (threadIdx.x == 0)
                (r.is_v ? a.v_scale
                        : a.k_scale)[(int64_t)page * a.num_kv_heads + r.head] = now;
        }
    }
}

// Work-groups that share a page's head rows: enough for a few rounds of the device (12
// replies of 5..90 tokens 30.4 -> 12.7 us), and at least kMinParts, so that the last
// round is short (50k prompt tokens: 284 us with one, 258 with four).
constexpr int64_t kPageGroups = 4096;
constexpr int64_t kMinParts = 4;

}  // namespace

extern "C" {

rl_da_status rl_rope_append(const void* q, int64_t q_stride, const void* k_new, int64_t k_stride,
                            const void* v_new, int64_t v_stride, const int32_t* q_start,
                            int32_t max_q_per_seq, const float* cos_sin, int32_t num_positions,
                            int32_t rotary_dim, int32_t interleaved, const void* q_norm,
                            const void* k_norm, float norm_eps, void* q_out, void* k_pool,
                            void* v_pool, float* k_scale, float* v_scale, int64_t num_pages,
                            const int32_t* block_table, int32_t max_pages,
                            const int32_t* seq_lens, int32_t batch, int32_t num_q_heads,
                            int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                            int32_t kv_dtype, int32_t layout, int32_t* device_error, void* stream)
{
    if (q == nullptr || k_new == nullptr || v_new == nullptr || cos_sin == nullptr ||
        q_out == nullptr || k_pool == nullptr || v_pool == nullptr || block_table == nullptr ||
        seq_lens == nullptr)
        return RL_DA_ERR_INVALID_ARG;
    if (batch < 0 || max_q_per_seq < 0 || num_q_heads <= 0 || num_kv_heads <= 0 ||
        max_pages < 1 || num_pages < 1 || num_positions < 1 || rotary_dim < 1)
        return RL_DA_ERR_INVALID_ARG;
    if (q_start == nullptr && max_q_per_seq != 1)
        return RL_DA_ERR_INVALID_ARG;
    if ((q_norm != nullptr) != (k_norm != nullptr) ||
        (q_norm != nullptr && !(isfinite(norm_eps) && norm_eps >= 0.0f)))
        return RL_DA_ERR_INVALID_ARG;
    if (kv_dtype != RL_DA_KV_BF16 && kv_dtype != RL_DA_KV_FP8_E4M3)
        return RL_DA_ERR_INVALID_ARG;
    if (head_dim != kHeadDim || page_size != kPageSize || rotary_dim > kHeadDim ||
        rotary_dim % 16 != 0)
        return RL_DA_ERR_UNSUPPORTED;
    const int64_t heads = (int64_t)num_q_heads + 2 * (int64_t)num_kv_heads;
    if (heads > INT32_MAX / kHeadDim || (int64_t)max_pages * kPageSize > INT32_MAX - kPageSize)
        return RL_DA_ERR_UNSUPPORTED;
    for (const void* p : {q, k_new, v_new, (const void*)cos_sin, q_norm, k_norm,
                          (const void*)q_out, (const void*)k_pool, (const void*)v_pool})
        if (!aligned16(p))
            return RL_DA_ERR_INVALID_ARG;
    const int64_t q_row = (int64_t)num_q_heads * kHeadDim;
    const int64_t kv_row = (int64_t)num_kv_heads * kHeadDim;
    if (q_stride < q_row || k_stride < kv_row || v_stride < kv_row || q_stride % 8 != 0 ||
        k_stride % 8 != 0 || v_stride % 8 != 0)
        return RL_DA_ERR_INVALID_ARG;
    if (q_out == q && q_stride != q_row)  // rows would overwrite each other
        return RL_DA_ERR_INVALID_ARG;
    const bool fp8 = kv_dtype == RL_DA_KV_FP8_E4M3;
    if (fp8 != (k_scale != nullptr) || fp8 != (v_scale != nullptr))
        return RL_DA_ERR_INVALID_ARG;
    if (!pools_paired(layout, k_pool, v_pool, fp8 ? 1 : 2))
        return RL_DA_ERR_INVALID_ARG;
    PoolStrides ps;
    if (!pool_strides(layout, num_kv_heads, fp8 ? 1 : 2, &ps))
        return RL_DA_ERR_INVALID_ARG;
    if (ps.page >= ((int64_t)1 << 31))  // strides inside a page are 32-bit
        return RL_DA_ERR_UNSUPPORTED;
    if (batch == 0 || max_q_per_seq == 0)
        return RL_DA_OK;
    RopeArgs a;
    a.q = (const uint16_t*)q;
    a.k_new = (const uint16_t*)k_new;
    a.v_new = (const uint16_t*)v_new;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_start = q_start;
    a.cos_sin = cos_sin;
    a.q_norm = (const uint16_t*)q_norm;
    a.k_norm = (const uint16_t*)k_norm;
    a.q_out = (uint16_t*)q_out;
    a.k_pool = (uint8_t*)k_pool;
    a.v_pool = (uint8_t*)v_pool;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.block_table = block_table;
    a.seq_lens = seq_lens;
    a.dev_error = device_error;
    a.num_pages = num_pages;
    a.page_bytes = ps.page;
    a.head_bytes = ps.head;
    a.row_bytes = ps.row;
    a.num_q_heads = num_q_heads;
    a.num_kv_heads = num_kv_heads;
    a.max_pages = max_pages;
    a.num_positions = num_positions;
    a.rotary_dim = rotary_dim;
    a.norm_eps = norm_eps;
    const bool few = max_q_per_seq <= (fp8 ? kFewTokens : kFewTokensBf16);
    const bool one = few && (!fp8 || max_q_per_seq == 1);
    // tokens of a sequence, or the pages that they touch at most from any slot on
    a.tiles = one ? max_q_per_seq : (int32_t)(((int64_t)max_q_per_seq + 14) / kPageSize + 1);
    const int64_t pages = (int64_t)batch * a.tiles;
    if (few) {
        a.parts = (int32_t)((heads + kRopeRows - 1) / kRopeRows);
    } else {
        const int64_t most = (heads + kAhead - 1) / kAhead;
        const int64_t parts = (kPageGroups + pages - 1) / pages;
        a.parts = (int32_t)(parts < kMinParts ? kMinParts : parts);
        if (a.parts > most)
            a.parts = (int32_t)most;
    }
    // a launch holds fewer than 2^32 threads (pages < 2^31 x 2^27, parts < 2^22)
    if (pages > UINT32_MAX / kRopeThreads / a.parts)
        return RL_DA_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)(pages * a.parts)), block(kRopeThreads);
    void (*kernel)(RopeArgs) = nullptr;
    auto pick = [&](auto fp8_t, auto inter_t) {
        constexpr bool F = decltype(fp8_t)::value, I = decltype(inter_t)::value;
        kernel = one ? rope_append_token<F, I> : (few ? rope_append_few<I> : rope_append_pages<F, I>);
    };
    if (fp8)
        interleaved ? pick(std::true_type{}, std::true_type{})
                    : pick(std::true_type{}, std::false_type{});
    else
        interleaved ? pick(std::false_type{}, std::true_type{})
                    : pick(std::false_type{}, std::false_type{});
    hipLaunchKernelGGL(kernel, grid, block, 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? RL_DA_OK : RL_DA_ERR_HIP;
}

}  // extern "C"
