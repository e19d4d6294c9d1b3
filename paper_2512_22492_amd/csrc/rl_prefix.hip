// rl_prefix.hip -- decode attention for sequences that share a prefix: the shared
// pages are read once for all of them.

#include <type_traits>

#include "rl_prefix_rule.h"
#include "rl_tile.h"
#include "rl_turns.h"

using namespace rl_da;

namespace {

// ----------------------------------------------- shared-prefix attention ---
//
// Softmax attention over a union of key sets is a weighted mean of the attention
// over each: with (m_s, l_s, O_s) the largest score, the sum of 2^(x - m_s) and the
// sum of 2^(x - m_s) v over set s (scores x in log2 units) and M = max m_s,
//     out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s.
// A sequence's keys are its group's shared pages and its own.  The shared ones are
// attended once for all query rows of the group (its sequences x G heads), the own
// ones for the sequence's G rows, each cut into splits; every unit of work is
// (query rows, pages), and a last kernel joins a row's partial results in a
// fixed order.
//
// Three launches: plan_prefix (one work-group) writes the list of units from the
// lengths and groups on the device, attend_prefix takes them, merge_prefix joins.
// Calls of few sequences are planned inside attend_prefix, and calls of few rows and a
// narrow table are one launch of attend_rows, which shares nothing.
//
// What bounds it: HBM while a key meets up to some 100 query rows (64 prompts x 8
// responses, 4600 MB to read: 729 us, 6.3 TB/s), the matrix and vector units above (256
// sequences x 16 heads under 8192 tokens: 104 us, 0.67 PFLOP/s over the call, 0.97 in its
// stages), launches and load latency in small calls (9 us).
//
// A sequence shorter than its group's prefix is not a member: it attends all its
// keys as its own.  So every row of a shared unit sees every key of it, and a
// finished sequence (length 0) takes part in nothing.

static_assert(kRulePage == kPageSize, "one page size");
static_assert(kMaxSplitPages == kWave * kUnitWaves, "a lane of each wavefront per page");
static_assert(kAlonePages == kUnitWaves, "a page per wavefront of a unit");
static_assert(kSmallCall == kWave, "a lane per sequence and per group");
constexpr float kNoScore = -3.0e38f;  // running max before the first key

// What the plan hands to the attention kernel.  Work-group g runs on XCD g % 8 and takes
// the work at places p = g mod 8 of the list, so each XCD has a counter in a cache line
// of its own: one counter for all of them moved between the XCDs' L2 caches at every
// turn, about 12 ns each (4096 single-page units: 60 us with it, 19 us with eight).
constexpr int kXcds = 8;
struct Queue {
    int32_t units;  // of the plan, each for num_kv_heads kv heads
    int32_t alone;  // units that a wavefront takes by itself, behind them
    int32_t pad[30];
    struct {
        int32_t next;  // places of the XCD that its work-groups have asked for
        int32_t pad[31];
    } xcd[kXcds];
};

struct PrefixArgs {
    const uint16_t* q;          // bf16 [B][Hq][D]
    const uint8_t* k_pool;
    const uint8_t* v_pool;
    const float* k_scale;       // [P][Hkv], e4m3 pools only
    const float* v_scale;
    const int32_t* block_table;
    const int32_t* seq_lens;
    const int32_t* group_start; // [num_groups + 1]
    const int32_t* prefix_pages;
    uint16_t* out;              // bf16 [B][Hq][D]
    int32_t* dev_error;         // may be null
    Queue* queue;               // workspace
    int32_t* leaders;           // workspace [num_groups]
    int2* parts;                // workspace [B]: shared and own partial results
    Unit* units;                // workspace
    float2* ml;                 // workspace [B * Hq][slots]: max (log2 units), weight sum
    float* acc;                 // workspace [B * Hq][slots][D]
    int64_t num_pages;
    int64_t page_bytes;         // pool strides in bytes: per page,
    int32_t head_bytes;         //   per kv head within a page,
    int32_t row_bytes;          //   per token slot within a slab
    int32_t batch;
    int32_t num_groups;
    int32_t num_q_heads;
    int32_t num_kv_heads;
    int32_t group_shift;        // log2 of the query heads per kv head
    int32_t max_pages;
    int32_t max_units;
    int32_t slots;
    int32_t unshared_pages;     // prefixes up to this length count as own pages
    int32_t wanted_shared;      // splits that fill the device (splits_of)
    int32_t wanted_own;
    int32_t least_shift;        // log2 of a split's least pages
    int32_t alone_pages;        // own runs up to this length are a wavefront's
    float scale_log2;           // |scale| * log2(e)
    uint32_t q_sign;            // 0x80008000 for a negative scale: Q enters negated
};

// ------------------------------------------------------------------ plan ---

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kClasses = 16;           // unit lengths, longest first
constexpr int kPlanSequences = 4096;   // batches and group tables up to these sizes are
constexpr int kPlanGroups = 2048;      // read once and kept in LDS

__device__ __forceinline__ int length_class(int pages)
{
    return kClasses - 1 - min((pages - 1) / (kMaxSplitPages / kClasses), kClasses - 1);
}

// A unit that all lanes hold alike, in scalar registers.
__device__ __forceinline__ Unit scalar_unit(const Unit& u)
{
    auto s = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return {s(u.table_row), s(u.page0), s(u.pages), s(u.limit),
            s(u.row0),      s(u.rows),  s(u.slot),  s(u.need)};
}

// Writes the units, longest first, and each sequence's number of partial results.
// Units of one class stand in any order: where a unit's results go does not depend
// on it.  One work-group, bound by the latency of what it reads: lengths and groups
// are read once, side by side, and everything after that is LDS (512 sequences in 64
// groups: 5.5 us).
template <bool CACHED>
__global__ __launch_bounds__(kPlanThreads) void plan_prefix(PrefixArgs a)
{
    __shared__ int lens_lds[CACHED ? kPlanSequences : 1];
    __shared__ int starts_lds[CACHED ? kPlanGroups + 1 : 1];
    __shared__ int pages_lds[CACHED ? kPlanGroups : 1];
    __shared__ int leader_lds[CACHED ? kPlanGroups : 1];
    __shared__ int cursor[2 * kClasses];  // units by length; those for one wavefront
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
    const int32_t* const lens = CACHED ? lens_lds : a.seq_lens;
    const int32_t* const starts = CACHED ? starts_lds : a.group_start;
    const int32_t* const pages = CACHED ? pages_lds : a.prefix_pages;
    int32_t* const leader = CACHED ? leader_lds : a.leaders;
    const int cap = a.max_pages * kPageSize;
    bool long_ones = false;
    for (int b = t; b < a.batch; b += kPlanThreads) {
        const int len = a.seq_lens[b];
        long_ones |= len > cap;
        if (CACHED)
            lens_lds[b] = len;
    }
    for (int g = t; g < a.num_groups; g += kPlanThreads) {
        leader[g] = INT32_MAX;
        if (CACHED) {
            starts_lds[g] = a.group_start[g];
            pages_lds[g] = a.prefix_pages[g];
        }
    }
    if (CACHED && t == 0 && a.num_groups > 0)
        starts_lds[a.num_groups] = a.group_start[a.num_groups];
    if (t < 2 * kClasses)
        cursor[t] = 0;
    if (long_ones && a.dev_error != nullptr)
        atomicOr(a.dev_error, RL_DA_DEVERR_LENGTH_TOO_LONG);
    __syncthreads();
    auto length_of = [&](int b) { return max(0, min(lens[b], cap)); };
    // The group that a sequence is a member of (it fills the group's prefix), or -1.
    auto group_of = [&](int b, int len) {
        int lo = -1, hi = a.num_groups;  // the last group that starts at or before b
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (starts[mid] <= b)
                lo = mid;
            else
                hi = mid;
        }
        if (lo < 0 || starts[lo + 1] <= b)
            return -1;
        const int p = prefix_of(a, pages[lo]);
        return p > 0 && len >= p * kPageSize ? lo : -1;
    };
    auto own_at = [&](int b, int g) {
        return own_of(a, length_of(b), g >= 0 ? prefix_of(a, pages[g]) : 0,
                      g >= 0 && starts[g + 1] - starts[g] > 1);
    };
    auto own_class = [&](const Own& o) {
        return o.alone(a) ? kClasses + length_class(min(o.s.pages * kUnitWaves, kMaxSplitPages))
                         : length_class(o.s.pages);
    };
    auto shared_at = [&](int g) { return shared_of(a, starts[g], starts[g + 1], pages[g]); };
    // (atomics pass the first-level cache, so must what reads their results from memory)
    auto leader_of = [&](int g) {
        return CACHED ? leader[g]
                      : __hip_atomic_load(&leader[g], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };

    // Count.  A group's first member lends its table row to the shared units; a
    // group without one has none.
    Own mine = {};  // the thread's first sequence
    for (int b = t; b < a.batch; b += kPlanThreads) {
        const int g = group_of(b, length_of(b));
        const Own o = own_at(b, g);
        if (b == t)
            mine = o;
        a.parts[b] = make_int2(o.shared, o.s.count);
        if (o.s.count > 0)
            atomicAdd(&cursor[own_class(o)], o.s.count);
        if (g >= 0)
            atomicMin(&leader[g], b);
    }
    __syncthreads();
    for (int g = t; g < a.num_groups; g += kPlanThreads) {
        if (leader_of(g) == INT32_MAX)
            continue;
        const Shared h = shared_at(g);
        if (h.units() > 0)
            atomicAdd(&cursor[length_class(h.s.pages)], h.units());
    }
    __syncthreads();
    if (t < 2 * kClasses) {
        int at = 0, units = 0, all = 0;
        for (int c = 0; c < 2 * kClasses; ++c) {
            const int n = cursor[c];
            at += c < t ? n : 0;
            units += c < kClasses ? n : 0;
            all += n;
        }
        __builtin_amdgcn_wave_barrier();
        cursor[t] = at;
        if (t == 0) {
            // group_start that runs backwards could name more than there is room for
            units = min(units, a.max_units);
            a.queue->units = units;
            a.queue->alone = min(all, a.max_units) - units;
        }
        if (t < kXcds)
            a.queue->xcd[t].next = 0;
    }
    __syncthreads();

    // Write.
    constexpr int kFirst = 4;
    auto put = [&](int at, const Unit& u) {
        if (at < a.max_units)
            a.units[at] = u;
    };
    for (int b0 = wave * kWave; b0 < a.batch; b0 += kPlanThreads) {
        const int b = b0 + lane;
        const bool has = b < a.batch;
        Own o = mine;
        if (b0 >= kPlanThreads)
            o = own_at(has ? b : b0, has ? group_of(b, length_of(b)) : -1);
        o.s.count = has ? o.s.count : 0;
        int at = 0;
        if (o.s.count > 0)
            at = atomicAdd(&cursor[own_class(o)], o.s.count);
        // a lane writes its sequence's first units, all lanes together the others
        for (int i = 0; i < min(o.s.count, kFirst); ++i)
            put(at + i, own_unit(a, b, o, i));
        for (uint64_t more = __ballot(o.s.count > kFirst); more != 0; more &= more - 1) {
            const int from = __builtin_ctzll(more);
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, from); };
            const Own w = {of(o.len), of(o.first), of(o.shared), of(o.others),
                           {of(o.s.count), of(o.s.pages), of(o.s.more)}};
            for (int i = kFirst + lane; i < w.s.count; i += kWave)
                put(of(at) + i, own_unit(a, b0 + from, w, i));
        }
    }
    // the groups likewise, from the last wavefront on, which has fewest sequences
    for (int g0 = (kPlanWaves - 1 - wave) * kWave; g0 < a.num_groups; g0 += kPlanThreads) {
        const int g = g0 + lane;
        const bool has = g < a.num_groups;
        const int first = has ? leader_of(g) : INT32_MAX;
        const Shared h = shared_at(has ? g : g0);
        const int n = first != INT32_MAX ? h.units() : 0;
        int at = 0;
        if (n > 0)
            at = atomicAdd(&cursor[length_class(h.s.pages)], n);
        for (int i = 0; i < min(n, kFirst); ++i)
            put(at + i, shared_unit(a, h, first, i));
        for (uint64_t more = __ballot(n > kFirst); more != 0; more &= more - 1) {
            const int from = __builtin_ctzll(more);
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, from); };
            const Shared w = {of(h.s0), of(h.rows), of(h.tiles), of(h.pages),
                              {of(h.s.count), of(h.s.pages), of(h.s.more)}};
            for (int i = kFirst + lane; i < of(n); i += kWave)
                put(of(at) + i, shared_unit(a, w, of(first), i));
        }
    }
}

// The plan of a small call (rl_prefix_rule.h).
struct SmallPlan {
    // running numbers of units, and what each is made from
    int shared_end[kSmallCall], own_end[kSmallCall];
    Shared shared[kSmallCall];
    int leader[kSmallCall];
    Own own[kSmallCall];
    int alone_seq[kSmallCall];  // sequences whose own run is a wavefront's alone
    int units, alone;
};

__device__ __forceinline__ int wave_inclusive_sum(int v, int lane)
{
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int below = __shfl_up(v, d);
        v += lane >= d ? below : 0;
    }
    return v;
}

// By one wavefront; `tell`: it also writes the numbers of partial results for the merge.
__device__ __forceinline__ void plan_small(const PrefixArgs& a, SmallPlan& plan, int lane,
                                           bool tell)
{
    const bool is_seq = lane < a.batch, is_group = lane < a.num_groups;
    const int cap = a.max_pages * kPageSize;
    const int raw = is_seq ? a.seq_lens[lane] : 0;
    const int start = is_group ? a.group_start[lane] : INT32_MAX;
    const int end = is_group ? a.group_start[lane + 1] : INT32_MAX;
    const int pages = is_group ? prefix_of(a, a.prefix_pages[lane]) : 0;
    const int len = max(0, min(raw, cap));
    // the last group that starts at or before the lane's sequence
    int lo = -1, hi = a.num_groups;
#pragma unroll
    for (int step = kSmallCall; step > 0; step /= 2) {  // all lanes take part in the reads
        const int mid = max((lo + hi) / 2, 0);
        const bool below = __shfl(start, mid) <= lane;
        if (hi - lo > 1) {
            lo = below ? mid : lo;
            hi = below ? hi : mid;
        }
    }
    const int group_start = __shfl(start, max(lo, 0)), group_end = __shfl(end, max(lo, 0));
    const int group_pages = __shfl(pages, max(lo, 0));
    const bool member = is_seq && lo >= 0 && group_end > lane && group_pages > 0 &&
                        len >= group_pages * kPageSize;
    const Own o = own_of(a, len, member ? group_pages : 0, group_end - group_start > 1);
    const uint64_t members = __ballot(member);
    const bool alone = o.alone(a);
    const uint64_t alone_mask = __ballot(alone);
    if (alone)
        plan.alone_seq[__popcll(alone_mask & ((1ull << lane) - 1))] = lane;
    plan.own[lane] = o;

    const Shared h = shared_of(a, is_group ? start : 0, is_group ? end : 0, pages);
    const int s1 = h.s0 + (h.rows >> a.group_shift);
    const uint64_t in_group = h.rows == 0 ? 0
                                          : (s1 < 64 ? (1ull << s1) - 1 : ~0ull) &
                                                ~((1ull << h.s0) - 1) & members;
    plan.shared[lane] = h;
    plan.leader[lane] = in_group != 0 ? (int)__builtin_ctzll(in_group) : 0;
    const int shared_end = wave_inclusive_sum(in_group != 0 ? h.units() : 0, lane);
    const int shared_all = __builtin_amdgcn_readlane(shared_end, kWave - 1);
    const int own_end = shared_all + wave_inclusive_sum(alone ? 0 : o.s.count, lane);
    plan.shared_end[lane] = shared_end;
    plan.own_end[lane] = own_end;
    if (lane == kWave - 1) {
        plan.units = own_end;
        plan.alone = __popcll(alone_mask);
    }
    if (tell) {
        if (is_seq)
            a.parts[lane] = make_int2(o.shared, o.s.count);
        if (raw > cap && a.dev_error != nullptr)
            atomicOr(a.dev_error, RL_DA_DEVERR_LENGTH_TOO_LONG);
    }
}

// Unit number i of a small call's plan.
__device__ __forceinline__ Unit small_unit(const PrefixArgs& a, const SmallPlan& plan, int lane,
                                           int i)
{
    const uint64_t shared = __ballot(plan.shared_end[lane] > i);
    if (shared != 0) {
        const int g = __builtin_ctzll(shared);
        return shared_unit(a, plan.shared[g], plan.leader[g],
                           i - (g > 0 ? plan.shared_end[g - 1] : 0));
    }
    const int b = __builtin_ctzll(__ballot(plan.own_end[lane] > i));
    return own_unit(a, b, plan.own[b],
                    i - (b > 0 ? plan.own_end[b - 1] : plan.shared_end[kSmallCall - 1]));
}

// ---------------------------------------------------------------- attend ---
//
// A unit is one work-group of four wavefronts.  Both products run transposed (S^T =
// K Q^T, O^T += V^T P^T), so that a lane keeps one query row from the scores to the
// output and P^T goes from the score registers into the second product as it lies
// there.  How a unit is shared among the wavefronts depends on its rows:
//
//   up to 16, 32 rows (attend_apart): wavefront w takes pages w, w + 4, ... for all
//     rows, each from a double buffer of its own in LDS that direct global-to-LDS
//     loads fill: no barrier until the unit's end, where the four (m, l, O) are
//     joined.  Bound by HBM: the matrix cores idle most of the time, so each weight
//     enters the value product as two bf16 terms (hi + lo, 2^-16 relative).
//   up to 64, 128 rows (attend_together): 64 keys at a time pass through a double
//     buffer of the work-group's, one barrier each; a wavefront holds 32 rows and
//     takes all 64 keys (four wavefronts for 128 rows) or half of them (two pairs for
//     64 rows, whose halves are joined at the end).  Where a byte of keys and values
//     meets 128 operations, 128 rows of bf16 and 64 of e4m3, the matrix and vector
//     units are about the bound, and a weight enters as one bf16 term (two: 256 sequences x
//     16 heads under 8192 tokens 104.4 -> 125.3 us, 64 groups of 64 rows under
//     1000..4000 e4m3 tokens 124.7 -> 132.8); 64 rows of bf16 take two terms (64 groups
//     under 2048 tokens 100.2 us with one, 101.3 with two).  bf16 pools sum the same
//     rounded weights for the normaliser, through the value product against ones, e4m3
//     pools the unrounded ones: their page's value scale is in the rounded ones.

constexpr int kAttendThreads = kWave * kUnitWaves;
constexpr int kBuffers = 2;
constexpr int kPageLds = kPageSize * kHeadDim * 2;  // a page of bf16 keys or values
constexpr int kWaveLds = kBuffers * 2 * kPageLds;
constexpr int kLdsBytes = kUnitWaves * kWaveLds;
constexpr int kStagePages = 4;                      // pages that a work-group shares
constexpr int kStageTile = kStagePages * kPageLds;
static_assert(kBuffers * 2 * kStageTile == kLdsBytes, "both ways use the same memory");

struct AttendLds {
    __attribute__((aligned(16))) char tiles[kLdsBytes];
    float2 ml[kUnitWaves][32];
    __attribute__((aligned(16))) int32_t pages[kMaxSplitPages + kStagePages];
    __attribute__((aligned(16))) float2 scales[kMaxSplitPages + kStagePages];
    NextPlace next;  // of the list, for all wavefronts
};

struct Lanes {
    int wave, lane, i16, g4;
};

template <int N>
__device__ __forceinline__ void wait_loads()  // all but the latest N of the wavefront's
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds()
{
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p)
{
    typedef __attribute__((address_space(3))) void lds_void;
    return (uint32_t)(uintptr_t)(lds_void*)p;
}

// dma16, with the non-temporal hint for bytes that no other unit reads: they would
// only push others' out of the caches (64 prompts x 8 responses of 32 query heads to 8 kv
// heads: 806 us without it, 736 with; 1024 e4m3 sequences of 512..2048 tokens, the same
// heads, 498, 452).  A prefix that each member reads with its own pages goes without it
// (32 groups of 4 sequences of 4 kv heads under 48 pages 33.7 -> 28.6 us, 32 of 8 of 2
// kv heads 35.6 -> 29.1; 64 of 8 kv heads under 16 pages 14.6 -> 15.5).
__device__ __forceinline__ void bring16(const uint8_t* gaddr, uint32_t lds, bool once)
{
    if (once)
        asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt"
                     :
                     : "v"(gaddr), "{m0}"(lds)
                     : "memory");
    else
        dma16(gaddr, lds);
}

// Eight e4m3 codes to eight bf16 (exact), in order.
__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b)
{
    auto cvt = [](uint32_t w, auto upper) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(
                                                w, 1.0f, decltype(upper)::value));
    };
    return make_uint4(cvt(a, std::false_type{}), cvt(a, std::true_type{}),
                      cvt(b, std::false_type{}), cvt(b, std::true_type{}));
}

// A table entry, checked: one outside the pool is reported, and page 0 read instead
// (what the sequence gets is not defined).
__device__ __forceinline__ int checked_page(const PrefixArgs& a, int page)
{
    if (page >= 0 && (int64_t)page < a.num_pages)
        return page;
    if (a.dev_error != nullptr)
        atomicOr(a.dev_error, RL_DA_DEVERR_PAGE_OUT_OF_RANGE);
    return 0;
}

// Query row `row` of kv head kvh as an MFMA operand: the lane's eight dims of each
// quarter, 32 ks + 8 g4 .. (e4m3 keys read sixteen codes at once: 64 (ks / 2) + 16 g4 +
// 8 (ks % 2) ..).
template <bool CODES>
__device__ __forceinline__ void load_query(const PrefixArgs& a, int kvh, int row, int g4,
                                           uint4 (&q)[4])
{
    const int G = 1 << a.group_shift;
    const uint16_t* p =
        a.q + ((int64_t)(row >> a.group_shift) * a.num_q_heads + kvh * G + (row & (G - 1))) *
                  kHeadDim;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
        q[ks] = *reinterpret_cast<const uint4*>(
            p + (CODES ? 64 * (ks / 2) + 16 * g4 + 8 * (ks % 2) : 32 * ks + 8 * g4));
        q[ks].x ^= a.q_sign;
        q[ks].y ^= a.q_sign;
        q[ks].z ^= a.q_sign;
        q[ks].w ^= a.q_sign;
    }
}

// Output row (of q and out) of a unit's row r, and whether it takes part.
__device__ __forceinline__ int64_t output_row(const PrefixArgs& a, int kvh, int row)
{
    const int G = 1 << a.group_shift;
    return (int64_t)(row >> a.group_shift) * a.num_q_heads + kvh * G + (row & (G - 1));
}

// A row's float4 chunks (dims 4c .. 4c + 3) in the joining area, moved apart so that
// sixteen rows' equal chunks fall on different banks.
__device__ __forceinline__ float4* join_chunk(char* tiles, int wave, int row, int c)
{
    return reinterpret_cast<float4*>(tiles + wave * kWaveLds + row * (kHeadDim * 4)) +
           (c ^ (row & 15));
}

// One wavefront's pages of a unit, u.page0 + first, + first + STEP, ..., for all of the
// unit's rows: m, l (the lane's own keys' share) and O^T.
template <int RB, int STEP, bool FP8>
__device__ __forceinline__ void walk_pages(const PrefixArgs& a, const Unit& u, int kvh, int first,
                                           bool once, AttendLds& lds, const Lanes& at,
                                           float (&m)[RB], float (&l)[RB], floatx4_t (&o)[RB][8])
{
    const int wave = at.wave, lane = at.lane, i16 = at.i16, g4 = at.g4;
    char* const mine = lds.tiles + wave * kWaveLds;
    const uint32_t mine_at = lds_address(mine);
    // bytes of a page's keys (or values) in a buffer, loads that bring both
    constexpr int kTile = FP8 ? kPageLds / 2 : kPageLds;
    constexpr int kLoads = 2 * kTile / 1024;
    // e4m3: a page's values widened to bf16, behind the buffers of raw pages
    char* const wide = mine + kBuffers * 2 * kTile;
    const int count = first < u.pages ? (u.pages - first + STEP - 1) / STEP : 0;
    int my_page = 0;
    float my_ks = 1.0f, my_vs = 1.0f;
    if (lane < count) {
        my_page = checked_page(a, a.block_table[(int64_t)u.table_row * a.max_pages + u.page0 +
                                                first + lane * STEP]);
        if (FP8) {
            const int64_t slab = (int64_t)my_page * a.num_kv_heads + kvh;
            my_ks = a.k_scale[slab];
            my_vs = a.v_scale[slab];
        }
    }
    uint4 q[RB][4];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
        load_query<FP8>(a, kvh, u.row0 + min(16 * rb + i16, u.rows - 1), g4, q[rb]);

    // keys of the wavefront's i-th page that count
    auto keys_of = [&](int i) {
        return u.limit - (u.page0 + first + i * STEP) * kPageSize;
    };
    auto issue = [&](int i) {
        const int64_t page = __builtin_amdgcn_readlane(my_page, i);
        const int64_t base = page * a.page_bytes + (int64_t)kvh * a.head_bytes;
        const int last = min(keys_of(i), kPageSize) - 1;
        const uint32_t to = mine_at + (i % kBuffers) * 2 * kTile;
        constexpr int kRows = FP8 ? 8 : 4;     // rows of a page in one load
        constexpr int kLanes = kWave / kRows;  // lanes, chunks of a row
#pragma unroll
        for (int r = 0; r < kPageSize / kRows; ++r) {
            const int row = r * kRows + lane / kLanes;
            const int chunk = (lane % kLanes) ^ (FP8 ? row >> 1 : chunk_swizzle(row));
            // a key past the end is read as the last one (finite, weight 0)
            const int64_t off = base + (int64_t)min(row, last) * a.row_bytes + 16 * chunk;
            bring16(a.k_pool + off, to + 1024 * r, once);
            bring16(a.v_pool + off, to + kTile + 1024 * r, once);
        }
    };

#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kNoScore;
        l[rb] = 0.0f;
#pragma unroll
        for (int db = 0; db < 8; ++db)
            o[rb][db] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    auto consume = [&](int i) {
        const char* kt = mine + (i % kBuffers) * 2 * kTile;
        const char* vt = kt + kTile;
        uint4 kv[4];
        if constexpr (FP8) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint4 c = *reinterpret_cast<const uint4*>(
                    kt + i16 * kHeadDim + 16 * ((4 * h + g4) ^ (i16 >> 1)));
                kv[2 * h] = widen8(c.x, c.y);
                kv[2 * h + 1] = widen8(c.z, c.w);
            }
            // values: lane holds rows lane / 8 and 8 + lane / 8, 16 codes of each
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = 8 * h + lane / 8, c0 = lane % 8;
                const uint4 c = *reinterpret_cast<const uint4*>(vt + row * kHeadDim +
                                                                16 * (c0 ^ (row >> 1)));
                char* w = wide + row * (2 * kHeadDim);
                const int sw = chunk_swizzle(row);
                *reinterpret_cast<uint4*>(w + 16 * ((2 * c0) ^ sw)) = widen8(c.x, c.y);
                *reinterpret_cast<uint4*>(w + 16 * ((2 * c0 + 1) ^ sw)) = widen8(c.z, c.w);
            }
            vt = wide;
        } else {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                kv[ks] = *reinterpret_cast<const uint4*>(
                    kt + i16 * (2 * kHeadDim) + 16 * ((4 * ks + g4) ^ chunk_swizzle(i16)));
        }
        floatx4_t s[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
            s[rb] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                s[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8_t, kv[ks]), __builtin_bit_cast(bf16x8_t, q[rb][ks]),
                    s[rb], 0, 0, 0);
        // lane: row i16 of each block, keys 4 g4 .. + 3
        float mult = a.scale_log2, vs = 1.0f;
        if (FP8) {
            mult *= __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), i));
            vs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), i));
        }
        const int keys = keys_of(i);
        float x[RB][4], mx[RB];
        bool grow = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[rb][j] = 4 * g4 + j < keys ? s[rb][j] * mult : -INFINITY;
            mx[rb] = fmaxf(fmaxf(x[rb][0], x[rb][1]), fmaxf(x[rb][2], x[rb][3]));
            mx[rb] = max_lanes_xor32(max_lanes_xor16(mx[rb]));
            grow |= mx[rb] > m[rb] + kMaxSlack;
        }
        if (__any(grow)) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const float m_new = mx[rb] > m[rb] + kMaxSlack ? mx[rb] : m[rb];
                const float alpha = exp2_fast(m[rb] - m_new);
                m[rb] = m_new;
                l[rb] *= alpha;
#pragma unroll
                for (int db = 0; db < 8; ++db)
                    o[rb][db] *= alpha;
            }
        }
        uint2 hi[RB], lo[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[j] = exp2_fast(x[rb][j] - m[rb]);
                l[rb] += p[j];
                p[j] *= vs;
            }
            const uint32_t h0 = pack_bf16x2(p[0], p[1]), h1 = pack_bf16x2(p[2], p[3]);
            hi[rb] = make_uint2(h0, h1);
            lo[rb] = make_uint2(pack_bf16x2(p[0] - bf16_lo(h0), p[1] - bf16_hi(h0)),
                                pack_bf16x2(p[2] - bf16_lo(h1), p[3] - bf16_hi(h1)));
        }
        if constexpr (FP8)
            wave_lds_sync();  // the widened values are in place
        const int vrow = 4 * g4 + (i16 >> 2), vsw = chunk_swizzle(vrow);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            const uint2 vv = lds_read_transposed(reinterpret_cast<const uint16_t*>(
                vt + vrow * (2 * kHeadDim) + 16 * ((2 * db + ((i16 & 3) >> 1)) ^ vsw) +
                8 * (i16 & 1)));
            const short4_t v4 = __builtin_bit_cast(short4_t, vv);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
                    v4, __builtin_bit_cast(short4_t, hi[rb]), o[rb][db], 0, 0, 0);
                o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
                    v4, __builtin_bit_cast(short4_t, lo[rb]), o[rb][db], 0, 0, 0);
            }
        }
    };

    if (count > 0)
        issue(0);
    if (count > 1)
        issue(1);
    for (int i = 0; i < count; ++i) {
        if (i + 1 < count)
            wait_loads<kLoads>();
        else
            wait_loads<0>();
        consume(i);
        wait_lds();  // the buffer has been read
        if (i + 2 < count)
            issue(i + 2);
    }
}

template <int RB, bool FP8>
__device__ __forceinline__ void attend_apart(const PrefixArgs& a, const Unit& u, int kvh,
                                             bool once, AttendLds& lds, const Lanes& at)
{
    const int wave = at.wave, i16 = at.i16, g4 = at.g4;
    float m[RB], l[RB];
    floatx4_t o[RB][8];
    walk_pages<RB, kUnitWaves, FP8>(a, u, kvh, wave, once, lds, at, m, l, o);
    __syncthreads();  // all wavefronts are done with their buffers
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        l[rb] = sum_lanes_xor32(sum_lanes_xor16(l[rb]));
#pragma unroll
        for (int db = 0; db < 8; ++db)
            *join_chunk(lds.tiles, wave, 16 * rb + i16, 4 * db + g4) =
                make_float4(o[rb][db][0], o[rb][db][1], o[rb][db][2], o[rb][db][3]);
        if (g4 == 0)
            lds.ml[wave][16 * rb + i16] = make_float2(m[rb], l[rb]);
    }
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = 16 * rb + threadIdx.x / 16;
        const int r = u.row0 + row;
        if (row >= u.rows || a.seq_lens[r >> a.group_shift] < u.need)
            continue;
        float2 ml[kUnitWaves];
        float M = kNoScore;
#pragma unroll
        for (int w = 0; w < kUnitWaves; ++w) {
            ml[w] = lds.ml[w][row];
            M = fmaxf(M, ml[w].x);
        }
        float L = 0.0f, weight[kUnitWaves];
#pragma unroll
        for (int w = 0; w < kUnitWaves; ++w) {
            weight[w] = exp2_fast(ml[w].x - M);
            L = fmaf(weight[w], ml[w].y, L);
        }
        const int64_t out_row = output_row(a, kvh, r);
        const int64_t part = out_row * a.slots + max(u.slot, 0);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = threadIdx.x % 16 + 16 * h;
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kUnitWaves; ++w) {
                const float4 x = *join_chunk(lds.tiles, w, row, c);
                v.x = fmaf(weight[w], x.x, v.x);
                v.y = fmaf(weight[w], x.y, v.y);
                v.z = fmaf(weight[w], x.z, v.z);
                v.w = fmaf(weight[w], x.w, v.w);
            }
            if (u.slot >= 0) {
                *reinterpret_cast<float4*>(a.acc + part * kHeadDim + 4 * c) = v;
            } else {
                const float inv = 1.0f / L;
                *reinterpret_cast<uint2*>(a.out + out_row * kHeadDim + 4 * c) = make_uint2(
                    pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
            }
        }
        if (u.slot >= 0 && threadIdx.x % 16 == 0)
            a.ml[part] = make_float2(M, L);
    }
}

// A whole short own run by one wavefront.
template <bool FP8>
__device__ __forceinline__ void attend_alone(const PrefixArgs& a, const Unit& u, int kvh,
                                             bool once, AttendLds& lds, const Lanes& at)
{
    float m[1], l[1];
    floatx4_t o[1][8];
    walk_pages<1, 1, FP8>(a, u, kvh, 0, once, lds, at, m, l, o);
    const float sum = sum_lanes_xor32(sum_lanes_xor16(l[0]));
    if (at.i16 >= u.rows)
        return;
    const int64_t out_row = output_row(a, kvh, u.row0 + at.i16);
    if (u.slot < 0) {
        const float inv = 1.0f / sum;
#pragma unroll
        for (int db = 0; db < 8; ++db)
            *reinterpret_cast<uint2*>(a.out + out_row * kHeadDim + 16 * db + 4 * at.g4) =
                make_uint2(pack_bf16x2(o[0][db][0] * inv, o[0][db][1] * inv),
                           pack_bf16x2(o[0][db][2] * inv, o[0][db][3] * inv));
        return;
    }
    const int64_t part = out_row * a.slots + u.slot;
#pragma unroll
    for (int db = 0; db < 8; ++db)
        *reinterpret_cast<float4*>(a.acc + part * kHeadDim + 16 * db + 4 * at.g4) =
            make_float4(o[0][db][0], o[0][db][1], o[0][db][2], o[0][db][3]);
    if (at.g4 == 0)
        a.ml[part] = make_float2(m[0], sum);
}

// KW wavefronts share 32 rows, each taking 1 / KW of a stage's keys.
template <int KW, bool FP8>
__device__ __forceinline__ void attend_together(const PrefixArgs& a, const Unit& u, int kvh,
                                                bool once, AttendLds& lds, const Lanes& at)
{
    constexpr int RB = 2;
    constexpr int KB = kStagePages / KW;  // 16-key blocks of a stage per wavefront
    constexpr int kTerms = KW == 2 && !FP8 ? 2 : 1;  // of a weight
    const int wave = at.wave, lane = at.lane, i16 = at.i16, g4 = at.g4;
    const int kw = wave % KW, row_base = wave / KW * 32;
    const int stages = (u.pages + kStagePages - 1) / kStagePages;
    auto k_tile = [&](int sel) { return lds.tiles + sel * 2 * kStageTile; };
    auto v_tile = [&](int sel) { return lds.tiles + sel * 2 * kStageTile + kStageTile; };

    // The unit's pages and their scales; a stage's pages past the unit's last are read
    // as that one (finite) and masked.
    for (int i = threadIdx.x; i < stages * kStagePages; i += kAttendThreads) {
        const int page = checked_page(
            a, a.block_table[(int64_t)u.table_row * a.max_pages + u.page0 +
                             min(i, u.pages - 1)]);
        lds.pages[i] = page;
        if (FP8) {
            const int64_t slab = (int64_t)page * a.num_kv_heads + kvh;
            lds.scales[i] = make_float2(a.k_scale[slab], a.v_scale[slab]);
        }
    }
    uint4 q[RB][4];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
        load_query<false>(a, kvh, u.row0 + min(row_base + 16 * rb + i16, u.rows - 1), g4, q[rb]);
    __syncthreads();

    // bf16: wavefront w brings rows 4w .. 4w + 3 of each page, lane l the chunk that the
    // swizzle puts at position l % 16 of row 4w + l / 16.
    const int d_row = 4 * wave + lane / 16;
    const int64_t d_off = (int64_t)kvh * a.head_bytes + (int64_t)d_row * a.row_bytes +
                          16 * ((lane % 16) ^ chunk_swizzle(d_row));
    auto bring = [&](int stage, int sel) {
        const int4 pg = *reinterpret_cast<const int4*>(&lds.pages[stage * kStagePages]);
        const int page[kStagePages] = {pg.x, pg.y, pg.z, pg.w};
        const uint32_t k_at = lds_address(k_tile(sel)), v_at = lds_address(v_tile(sel));
#pragma unroll
        for (int r = 0; r < kStagePages; ++r) {
            const int64_t off =
                (int64_t)__builtin_amdgcn_readfirstlane(page[r]) * a.page_bytes + d_off;
            bring16(a.k_pool + off, k_at + r * kPageLds + 1024 * wave, once);
            bring16(a.v_pool + off, v_at + r * kPageLds + 1024 * wave, once);
        }
    };
    // e4m3: thread t loads the codes of dims 16 (t % 8) .. + 15 of key rows 2 (t / 8)
    // and the next one, and widens them on the way into the tiles.
    const int thread = wave * kWave + lane;
    const int s_row = 2 * (thread / 8), s_chunk = 2 * (thread % 8);
    const int64_t s_off = (int64_t)kvh * a.head_bytes +
                          (int64_t)(s_row % kPageSize) * a.row_bytes + 8 * s_chunk;
    uint4 kr[2], vr[2];
    auto fetch = [&](int stage) {
        const int64_t off =
            (int64_t)lds.pages[stage * kStagePages + s_row / kPageSize] * a.page_bytes + s_off;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint8_t* k = a.k_pool + off + i * a.row_bytes;
            const uint8_t* v = a.v_pool + off + i * a.row_bytes;
            kr[i] = once ? load_stream16(k) : *reinterpret_cast<const uint4*>(k);
            vr[i] = once ? load_stream16(v) : *reinterpret_cast<const uint4*>(v);
        }
    };
    auto stash = [&](int sel) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = s_row + i, sw = chunk_swizzle(row % kPageSize);
            char* k = k_tile(sel) + row * (2 * kHeadDim);
            char* v = v_tile(sel) + row * (2 * kHeadDim);
            *reinterpret_cast<uint4*>(k + 16 * (s_chunk ^ sw)) = widen8(kr[i].x, kr[i].y);
            *reinterpret_cast<uint4*>(k + 16 * ((s_chunk + 1) ^ sw)) = widen8(kr[i].z, kr[i].w);
            *reinterpret_cast<uint4*>(v + 16 * (s_chunk ^ sw)) = widen8(vr[i].x, vr[i].y);
            *reinterpret_cast<uint4*>(v + 16 * ((s_chunk + 1) ^ sw)) = widen8(vr[i].z, vr[i].w);
        }
    };

    // Operand offsets into a tile, made once.
    int k_off[4], v_off[8];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
        k_off[ks] = i16 * (2 * kHeadDim) + 16 * ((4 * ks + g4) ^ chunk_swizzle(i16));
    const int vrow = 4 * g4 + (i16 >> 2);
#pragma unroll
    for (int db = 0; db < 8; ++db)
        v_off[db] = vrow * (2 * kHeadDim) +
                    16 * ((2 * db + ((i16 & 3) >> 1)) ^ chunk_swizzle(vrow)) + 8 * (i16 & 1);

    float m[RB], l[RB];
    floatx4_t lacc[RB], o[RB][8];
    const uint4 ones = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kNoScore;
        l[rb] = 0.0f;
        lacc[rb] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int db = 0; db < 8; ++db)
            o[rb][db] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    auto stage = [&](int j, int sel, auto last_t) __attribute__((always_inline)) {
        constexpr bool kLast = decltype(last_t)::value;
        if constexpr (FP8) {
            stash(sel);
            if (j + 1 < stages)
                fetch(j + 1);
            __syncthreads();
        } else {
            wait_loads<0>();  // this wavefront's share of the stage
            __syncthreads();
        }
        const char* kt = k_tile(sel) + kw * KB * kPageLds;
        const char* vt = v_tile(sel) + kw * KB * kPageLds;
        floatx4_t s[RB][KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
                s[rb][kb] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};
        // Scores, a quarter of the dims at a time; its keys are read ahead of the matrix
        // instructions of the quarter before.
        auto keys = [&](int ks, uint4 (&kv)[KB]) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                kv[kb] = *reinterpret_cast<const uint4*>(kt + kb * kPageLds + k_off[ks]);
        };
        __builtin_amdgcn_s_setprio(1);
        uint4 kv[2][KB];
        keys(0, kv[0]);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            if (ks + 1 < 4)
                keys(ks + 1, kv[(ks + 1) % 2]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    s[rb][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8_t, kv[ks % 2][kb]),
                        __builtin_bit_cast(bf16x8_t, q[rb][ks]), s[rb][kb], 0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        if constexpr (!FP8) {
            if (j + 1 < stages)
                bring(j + 1, 1 - sel);
        }
        // scores in log2 units are s * mult
        float mult[KB], vs[KB];
        const int page0 = j * kStagePages + kw * KB;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            mult[kb] = a.scale_log2;
            vs[kb] = 1.0f;
            if (FP8) {
                const float2 sc = lds.scales[page0 + kb];
                mult[kb] *= sc.x;
                vs[kb] = sc.y;
            }
        }
        // The row maxima: each block's multiplier times its raw maximum, if none of the
        // multipliers is negative; else the scores are multiplied out first.
        if (FP8) {
            bool folds = true;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
                folds &= mult[kb] >= 0.0f;
            if (__builtin_expect(!__builtin_amdgcn_readfirstlane(folds), 0)) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
                        s[rb][kb] *= mult[kb];
                    mult[kb] = 1.0f;
                }
            }
        }
        float mx[RB];
        bool grow = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float top[KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                if (kLast && page0 + kb >= u.pages) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        s[rb][kb][i] = -INFINITY;
                    mult[kb] = 1.0f;
                }
                const float t = __builtin_elementwise_maximum(
                    __builtin_elementwise_maximum(s[rb][kb][0], s[rb][kb][1]), s[rb][kb][2]);
                top[kb] = __builtin_elementwise_maximum(t, s[rb][kb][3]);
                if (FP8)
                    top[kb] *= mult[kb];
            }
            mx[rb] = __builtin_elementwise_maximum(top[0], top[1]);
            if (KB == 4)
                mx[rb] = __builtin_elementwise_maximum(
                    __builtin_elementwise_maximum(mx[rb], top[2]), top[KB - 1]);
            if (!FP8)
                mx[rb] *= a.scale_log2;
            mx[rb] = max_lanes_xor32(max_lanes_xor16(mx[rb]));
            grow |= mx[rb] > m[rb] + kMaxSlack;
        }
        if (__builtin_expect(__any(grow), 0)) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const float m_new = mx[rb] > m[rb] + kMaxSlack ? mx[rb] : m[rb];
                const float alpha = exp2_fast(m[rb] - m_new);
                m[rb] = m_new;
                l[rb] *= alpha;
                lacc[rb] *= alpha;
#pragma unroll
                for (int db = 0; db < 8; ++db)
                    o[rb][db] *= alpha;
            }
        }
        // Weights as operands: two 16-key blocks (a half) are one, keys 4 g4 .. + 3 of
        // each.  Piece i of half kh: row block i / 4, key block i / 2 % 2, key pair i % 2.
        uint32_t pt[kTerms][RB][KB / 2][4];
        auto make_piece = [&](int kh, int i) {
            const int rb = i / 4, kb = 2 * kh + i / 2 % 2, e = 2 * (i % 2);
            float p0 = exp2_fast(fmaf(s[rb][kb][e], mult[kb], -m[rb]));
            float p1 = exp2_fast(fmaf(s[rb][kb][e + 1], mult[kb], -m[rb]));
            if (FP8) {
                l[rb] += p0 + p1;
                p0 *= vs[kb];
                p1 *= vs[kb];
            }
            const uint32_t hi = pack_bf16x2(p0, p1);
            pt[0][rb][kh][i % 4] = hi;
            if (kTerms == 2)
                pt[kTerms - 1][rb][kh][i % 4] = pack_bf16x2(p0 - bf16_lo(hi), p1 - bf16_hi(hi));
        };
        auto operand = [&](int term, int rb, int kh) {
            const uint32_t(&w)[4] = pt[term][rb][kh];
            return __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
        };
#pragma unroll
        for (int i = 0; i < 4 * RB; ++i)
            make_piece(0, i);
        // The value product, one dim block of a half per step; the next step's values are
        // read ahead of this one's matrix instructions, and the second half's weights
        // are made a piece per step of the first.
        auto values = [&](int step) {
            const char* p = vt + 2 * (step / 8) * kPageLds + v_off[step % 8];
            const uint2 va = lds_read_transposed(reinterpret_cast<const uint16_t*>(p));
            const uint2 vb = lds_read_transposed(reinterpret_cast<const uint16_t*>(p + kPageLds));
            return __builtin_bit_cast(bf16x8_t, make_uint4(va.x, va.y, vb.x, vb.y));
        };
        __builtin_amdgcn_s_setprio(1);
        bf16x8_t next = values(0);
#pragma unroll
        for (int step = 0; step < 4 * KB; ++step) {
            const bf16x8_t v = next;
            if (step + 1 < 4 * KB)
                next = values(step + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int term = 0; term < kTerms; ++term)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    o[rb][step % 8] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        v, operand(term, rb, step / 8), o[rb][step % 8], 0, 0, 0);
            if (KB == 4 && step < 8)
                make_piece(KB / 2 - 1, step);
        }
        if (!FP8) {
#pragma unroll
            for (int kh = 0; kh < KB / 2; ++kh)
#pragma unroll
                for (int term = 0; term < kTerms; ++term)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
                        lacc[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8_t, ones), operand(term, rb, kh), lacc[rb],
                            0, 0, 0);
        }
        __builtin_amdgcn_s_setprio(0);
    };
    if constexpr (FP8)
        fetch(0);
    else
        bring(0, 0);
    int j = 0;
    for (; j < stages - 1; ++j)
        stage(j, j & 1, std::false_type{});
    stage(j, j & 1, std::true_type{});

#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
        l[rb] = FP8 ? sum_lanes_xor32(sum_lanes_xor16(l[rb])) : lacc[rb][0];
    if constexpr (KW == 2) {
        // the second wavefront of a pair hands its half to the first, lane by lane
        __syncthreads();  // the tiles have been read
        float4* area = reinterpret_cast<float4*>(lds.tiles) + (wave / 2) * (RB * 8 * kWave) + lane;
        if (kw == 1) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
                for (int db = 0; db < 8; ++db)
                    area[(8 * rb + db) * kWave] =
                        make_float4(o[rb][db][0], o[rb][db][1], o[rb][db][2], o[rb][db][3]);
                if (g4 == 0)
                    lds.ml[wave][16 * rb + i16] = make_float2(m[rb], l[rb]);
            }
        }
        __syncthreads();
        if (kw == 1)
            return;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const float2 ml = lds.ml[wave + 1][16 * rb + i16];
            const float M = fmaxf(m[rb], ml.x);
            const float w0 = exp2_fast(m[rb] - M), w1 = exp2_fast(ml.x - M);
            m[rb] = M;
            l[rb] = fmaf(w1, ml.y, w0 * l[rb]);
#pragma unroll
            for (int db = 0; db < 8; ++db) {
                const float4 x = area[(8 * rb + db) * kWave];
                o[rb][db][0] = fmaf(w1, x.x, w0 * o[rb][db][0]);
                o[rb][db][1] = fmaf(w1, x.y, w0 * o[rb][db][1]);
                o[rb][db][2] = fmaf(w1, x.z, w0 * o[rb][db][2]);
                o[rb][db][3] = fmaf(w1, x.w, w0 * o[rb][db][3]);
            }
        }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = row_base + 16 * rb + i16, r = u.row0 + row;
        if (row >= u.rows || a.seq_lens[r >> a.group_shift] < u.need)
            continue;
        const int64_t part = output_row(a, kvh, r) * a.slots + u.slot;
#pragma unroll
        for (int db = 0; db < 8; ++db)
            *reinterpret_cast<float4*>(a.acc + part * kHeadDim + 16 * db + 4 * g4) =
                make_float4(o[rb][db][0], o[rb][db][1], o[rb][db][2], o[rb][db][3]);
        if (g4 == 0)
            a.ml[part] = make_float2(m[rb], l[rb]);
    }
}

constexpr int kStealRounds = 3;

// The place in the list of the `taken`-th one that XCD xcd's work-groups asked for (the grid
// has taken whole rounds of XCDs before it); when its places have run out, one of the
// XCD's that has most left (they finish up to some percent apart: 64 prompts x 8
// responses 741 us without this, 728 with); `total` when none is left.
__device__ __forceinline__ int next_place(const PrefixArgs& a, int total, int xcd, int taken)
{
    int place = gridDim.x + taken * kXcds + xcd;
    // few rounds: the look at the others' counters, 1.5 us, would not pay
    if (total <= kStealRounds * (int)gridDim.x)
        return min(place, total);
    while (place >= total) {
        int most = 0;
#pragma unroll
        for (int x = 0; x < kXcds; ++x) {
            const int left = total - x - (int)gridDim.x -
                             kXcds * __hip_atomic_load(&a.queue->xcd[x].next, __ATOMIC_RELAXED,
                                                       __HIP_MEMORY_SCOPE_AGENT);
            if (left > most) {
                most = left;
                xcd = x;
            }
        }
        if (most <= 0)
            return total;
        // others may be faster; every turn of this loop takes a place that is gone then
        place = gridDim.x + atomicAdd(&a.queue->xcd[xcd].next, 1) * kXcds + xcd;
    }
    return place;
}

template <bool FP8, bool SMALL>
__global__ __launch_bounds__(kAttendThreads) __attribute__((amdgpu_waves_per_eu(2))) void
attend_prefix(PrefixArgs a)
{
    __shared__ AttendLds lds;
    __shared__ std::conditional_t<SMALL, SmallPlan, int> plan;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    int planned, planned_alone;
    if constexpr (SMALL) {
        if (wave == 0)
            plan_small(a, plan, threadIdx.x, blockIdx.x == 0);
        __syncthreads();
        planned = __builtin_amdgcn_readfirstlane(plan.units);
        planned_alone = __builtin_amdgcn_readfirstlane(plan.alone);
    } else {
        planned = a.queue->units;
        planned_alone = a.queue->alone;
    }
    const int units = planned * a.num_kv_heads;
    const int alone = planned_alone * a.num_kv_heads;
    const int total = units + (alone + kUnitWaves - 1) / kUnitWaves;

    // A work-group's first work is its own place in the list, the others come from its
    // XCD's counter, asked for while the one before runs (a small call, of hardly more
    // than one round, deals them out in turn).
    const int xcd = blockIdx.x % kXcds;
    int at = blockIdx.x;
    for (int turn = 0; at < total; ++turn) {
        // made anew for each unit: what a unit derives from them would otherwise be kept
        // in registers throughout, for all four ways
        Lanes lanes;
        lanes.lane = threadIdx.x % kWave;
        asm volatile("" : "+v"(lanes.lane));
        lanes.wave = wave;
        lanes.i16 = lanes.lane & 15;
        lanes.g4 = lanes.lane >> 4;
        int taken = 0;
        if (!SMALL && threadIdx.x == 0 && total > (int)gridDim.x)
            taken = atomicAdd(&a.queue->xcd[xcd].next, 1);
        if (at < units) {
            Unit u;
            if constexpr (SMALL)
                u = scalar_unit(small_unit(a, plan, lanes.lane, at / a.num_kv_heads));
            else
                u = a.units[at / a.num_kv_heads];
            const int kvh = at % a.num_kv_heads;
            const bool once = u.rows > 0;
            u.rows = once ? u.rows : -u.rows;
            if (u.rows <= 16)
                attend_apart<1, FP8>(a, u, kvh, once, lds, lanes);
            else if (u.rows <= 32)
                attend_apart<2, FP8>(a, u, kvh, once, lds, lanes);
            else if (u.rows <= 64)
                attend_together<2, FP8>(a, u, kvh, once, lds, lanes);
            else
                attend_together<1, FP8>(a, u, kvh, once, lds, lanes);
        } else {
            const int item = (at - units) * kUnitWaves + lanes.wave;
            if (item < alone) {
                const int n = item / a.num_kv_heads;
                Unit u;
                if constexpr (SMALL) {
                    const int b = __builtin_amdgcn_readfirstlane(plan.alone_seq[n]);
                    u = scalar_unit(own_unit(a, b, plan.own[b], 0));
                } else {
                    u = a.units[planned + n];
                }
                const bool once = u.rows > 0;
                u.rows = once ? u.rows : -u.rows;
                attend_alone<FP8>(a, u, item % a.num_kv_heads, once, lds, lanes);
            }
        }
        if (!SMALL && threadIdx.x == 0)
            lds.next.of(turn) = next_place(a, total, xcd, taken);
        __syncthreads();  // the next unit's loads overwrite what this one still read
        // (runs of a wavefront alone have no other barrier: what keeps thread 0's next write
        // from this read is that it goes to the other word)
        at = SMALL ? at + (int)gridDim.x : __builtin_amdgcn_readfirstlane(lds.next.of(turn));
    }
}

// A call whose table is narrow and whose work-groups are few: a work-group per sequence
// and kv head attends the whole row, shared pages included, and writes the output; no
// plan, no partial results and no merge.
template <bool FP8>
__global__ __launch_bounds__(kAttendThreads) void attend_rows(PrefixArgs a)
{
    __shared__ AttendLds lds;
    Lanes lanes;
    lanes.wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    lanes.lane = threadIdx.x % kWave;
    lanes.i16 = lanes.lane & 15;
    lanes.g4 = lanes.lane >> 4;
    const int b = blockIdx.x / a.num_kv_heads, kvh = blockIdx.x % a.num_kv_heads;
    const int cap = a.max_pages * kPageSize;
    const int raw = a.seq_lens[b];
    if (raw > cap && a.dev_error != nullptr && threadIdx.x == 0)
        atomicOr(a.dev_error, RL_DA_DEVERR_LENGTH_TOO_LONG);
    const int len = min(raw, cap), G = 1 << a.group_shift;
    if (len <= 0) {  // no keys: zeros
        uint2* out = reinterpret_cast<uint2*>(
            a.out + ((int64_t)b * a.num_q_heads + kvh * G) * kHeadDim);
        for (int i = threadIdx.x; i < G * kHeadDim / 4; i += kAttendThreads)
            out[i] = make_uint2(0, 0);
        return;
    }
    const Unit u = {b, 0, (len + kPageSize - 1) / kPageSize, len, b << a.group_shift, G, -1, 0};
    attend_apart<1, FP8>(a, u, kvh, false, lds, lanes);
}

// ----------------------------------------------------------------- merge ---
//
// 32 lanes per output row, four dims each, walk a row's partial results in order;
// with SPREAD the eight such teams of a work-group share one row, team i taking
// results i, i + 8, ..., and their sums are joined in team order.

constexpr int kMergeTeams = 8;
constexpr int kMergeThreads = kMergeTeams * 32;

struct Joined {  // partial results so far, relative to their largest score
    float m, l;
    float4 v;
};
__device__ __forceinline__ void join(Joined& j, float m, float l, const float4& v)
{
    const float M = fmaxf(j.m, m);
    const float w0 = exp2_fast(j.m - M), w1 = exp2_fast(m - M);
    j.m = M;
    j.l = fmaf(w1, l, w0 * j.l);
    j.v.x = fmaf(w1, v.x, w0 * j.v.x);
    j.v.y = fmaf(w1, v.y, w0 * j.v.y);
    j.v.z = fmaf(w1, v.z, w0 * j.v.z);
    j.v.w = fmaf(w1, v.w, w0 * j.v.w);
}

template <bool SPREAD>
__global__ __launch_bounds__(kMergeThreads) void merge_prefix(PrefixArgs a)
{
    const int team = threadIdx.x / 32, c = threadIdx.x % 32;
    const int64_t row = SPREAD ? blockIdx.x : (int64_t)blockIdx.x * kMergeTeams + team;
    if (row >= (int64_t)a.batch * a.num_q_heads)
        return;
    const int2 parts = a.parts[row / a.num_q_heads];
    const int n = parts.x + parts.y;
    if (parts.x == 0 && n == 1)
        return;  // its unit has written it
    const float2* ml = a.ml + row * a.slots;
    const float4* acc = reinterpret_cast<const float4*>(a.acc + row * a.slots * kHeadDim) + c;
    Joined j = {kNoScore, 0.0f, make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
    constexpr int kStep = SPREAD ? kMergeTeams : 1;
    constexpr int kAhead = 4;  // results read side by side
    for (int s0 = SPREAD ? team : 0; s0 < n; s0 += kAhead * kStep) {
        float2 e[kAhead];
        float4 x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int s = min(s0 + i * kStep, n - 1);
            e[i] = ml[s];
            x[i] = acc[(int64_t)s * (kHeadDim / 4)];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (s0 + i * kStep < n)
                join(j, e[i].x, e[i].y, x[i]);
    }
    if constexpr (SPREAD) {
        __shared__ float4 team_v[kMergeTeams][32];
        __shared__ float2 team_ml[kMergeTeams];
        team_v[team][c] = j.v;
        if (c == 0)
            team_ml[team] = make_float2(j.m, j.l);
        __syncthreads();
        if (team != 0)
            return;
        for (int i = 1; i < min(n, kMergeTeams); ++i)
            join(j, team_ml[i].x, team_ml[i].y, team_v[i][c]);
    }
    const float inv = n > 0 ? 1.0f / j.l : 0.0f;  // no keys: zeros
    *reinterpret_cast<uint2*>(a.out + row * kHeadDim + 4 * c) = make_uint2(
        pack_bf16x2(j.v.x * inv, j.v.y * inv), pack_bf16x2(j.v.z * inv, j.v.w * inv));
}

// ------------------------------------------------------------------ host ---

struct Workspace {
    int64_t leaders, parts, units, ml, acc, bytes;  // offsets
    PrefixRule rule;
};

// false: sizes past what the kernels index
bool lay_out(int32_t max_pages, int32_t batch, int32_t num_groups, int32_t num_q_heads,
             int32_t num_kv_heads, Workspace* w)
{
    // a launch holds fewer than 2^32 threads, and the merge takes 32 for each row
    if ((int64_t)batch * num_q_heads > UINT32_MAX / 32 - kMergeTeams ||
        (int64_t)max_pages * kPageSize > INT32_MAX - kPageSize)
        return false;
    const PrefixRule r = prefix_rule(max_pages, batch, num_groups, num_q_heads, num_kv_heads);
    if (r.max_units > INT32_MAX / 2 / num_kv_heads)
        return false;
    w->rule = r;
    auto round = [](int64_t n) { return (n + 255) / 256 * 256; };
    w->leaders = round((int64_t)sizeof(Queue));
    w->parts = w->leaders + round((int64_t)num_groups * (int64_t)sizeof(int32_t));
    w->units = w->parts + round((int64_t)batch * (int64_t)sizeof(int2));
    w->ml = w->units + round(r.max_units * (int64_t)sizeof(Unit));
    const int64_t partials = (int64_t)batch * num_q_heads * r.slots;
    w->acc = w->ml + round(partials * (int64_t)sizeof(float2));
    w->bytes = w->acc + round(partials * kHeadDim * (int64_t)sizeof(float));
    return true;
}

}  // namespace

extern "C" {

rl_da_status rl_prefix_attn_workspace_size(int32_t max_pages, int32_t batch, int32_t num_groups,
                                           int32_t num_q_heads, int32_t num_kv_heads,
                                           size_t* bytes)
{
    if (bytes == nullptr || max_pages < 1 || batch < 0 || num_groups < 0 || num_q_heads <= 0 ||
        num_kv_heads <= 0 || num_q_heads % num_kv_heads != 0)
        return RL_DA_ERR_INVALID_ARG;
    Workspace w;
    if (!lay_out(max_pages, batch, num_groups, num_q_heads, num_kv_heads, &w))
        return RL_DA_ERR_UNSUPPORTED;
    *bytes = (size_t)w.bytes;
    return RL_DA_OK;
}

rl_da_status rl_prefix_attn(const void* q, const void* k_pool, const void* v_pool,
                            const float* k_scale, const float* v_scale, int64_t num_pages,
                            const int32_t* block_table, int32_t max_pages,
                            const int32_t* seq_lens, int32_t batch, const int32_t* group_start,
                            const int32_t* prefix_pages, int32_t num_groups, int32_t num_q_heads,
                            int32_t num_kv_heads, int32_t head_dim, int32_t page_size,
                            int32_t kv_dtype, int32_t layout, float scale, void* out,
                            void* workspace, size_t workspace_bytes, int32_t* device_error,
                            void* stream)
{
    if (q == nullptr || k_pool == nullptr || v_pool == nullptr || block_table == nullptr ||
        seq_lens == nullptr || out == nullptr || workspace == nullptr)
        return RL_DA_ERR_INVALID_ARG;
    if (batch < 0 || num_groups < 0 || num_q_heads <= 0 || num_kv_heads <= 0 ||
        num_q_heads % num_kv_heads != 0 || max_pages < 1 || num_pages < 1 || !isfinite(scale))
        return RL_DA_ERR_INVALID_ARG;
    if (num_groups > 0 && (group_start == nullptr || prefix_pages == nullptr))
        return RL_DA_ERR_INVALID_ARG;
    if (kv_dtype != RL_DA_KV_BF16 && kv_dtype != RL_DA_KV_FP8_E4M3)
        return RL_DA_ERR_INVALID_ARG;
    const bool fp8 = kv_dtype == RL_DA_KV_FP8_E4M3;
    if (fp8 != (k_scale != nullptr) || fp8 != (v_scale != nullptr))
        return RL_DA_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(out) ||
        !aligned16(workspace))
        return RL_DA_ERR_INVALID_ARG;
    if (!pools_paired(layout, k_pool, v_pool, fp8 ? 1 : 2))
        return RL_DA_ERR_INVALID_ARG;
    PoolStrides ps;
    if (!pool_strides(layout, num_kv_heads, fp8 ? 1 : 2, &ps))
        return RL_DA_ERR_INVALID_ARG;
    const int G = num_q_heads / num_kv_heads;
    if (head_dim != kHeadDim || page_size != kPageSize ||
        (G != 1 && G != 2 && G != 4 && G != 8 && G != 16) ||
        ps.page >= ((int64_t)1 << 31))  // strides inside a page are 32-bit
        return RL_DA_ERR_UNSUPPORTED;
    Workspace w;
    if (!lay_out(max_pages, batch, num_groups, num_q_heads, num_kv_heads, &w))
        return RL_DA_ERR_UNSUPPORTED;
    if (workspace_bytes < (size_t)w.bytes)
        return RL_DA_ERR_INVALID_ARG;
    if (batch == 0)
        return RL_DA_OK;
    // a group's rows are read by work-groups that others' outputs do not wait for
    const uintptr_t row_bytes = (uintptr_t)batch * num_q_heads * kHeadDim * sizeof(uint16_t);
    if ((uintptr_t)q < (uintptr_t)out + row_bytes && (uintptr_t)out < (uintptr_t)q + row_bytes)
        return RL_DA_ERR_INVALID_ARG;
    PrefixArgs a;
    a.q = (const uint16_t*)q;
    a.k_pool = (const uint8_t*)k_pool;
    a.v_pool = (const uint8_t*)v_pool;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.block_table = block_table;
    a.seq_lens = seq_lens;
    a.group_start = group_start;
    a.prefix_pages = prefix_pages;
    a.out = (uint16_t*)out;
    a.dev_error = device_error;
    char* ws = (char*)workspace;
    a.queue = (Queue*)ws;
    a.leaders = (int32_t*)(ws + w.leaders);
    a.parts = (int2*)(ws + w.parts);
    a.units = (Unit*)(ws + w.units);
    a.ml = (float2*)(ws + w.ml);
    a.acc = (float*)(ws + w.acc);
    a.num_pages = num_pages;
    a.page_bytes = ps.page;
    a.head_bytes = ps.head;
    a.row_bytes = ps.row;
    a.batch = batch;
    a.num_groups = num_groups;
    a.num_q_heads = num_q_heads;
    a.num_kv_heads = num_kv_heads;
    a.group_shift = __builtin_ctz((unsigned)G);
    a.max_pages = max_pages;
    a.max_units = (int32_t)w.rule.max_units;
    a.slots = w.rule.slots;
    a.unshared_pages = w.rule.unshared_pages;
    a.wanted_shared = w.rule.wanted_shared;
    a.wanted_own = w.rule.wanted_own;
    a.least_shift = w.rule.least_shift;
    a.alone_pages = w.rule.alone_pages;
    a.scale_log2 = fabsf(scale) * kLog2e;
    a.q_sign = scale < 0.0f ? 0x80008000u : 0u;
    hipStream_t st = (hipStream_t)stream;
    if (w.rule.by_rows) {
        const dim3 grid((unsigned)(batch * num_kv_heads));
        if (fp8)
            hipLaunchKernelGGL(attend_rows<true>, grid, dim3(kAttendThreads), 0, st, a);
        else
            hipLaunchKernelGGL(attend_rows<false>, grid, dim3(kAttendThreads), 0, st, a);
        return hipGetLastError() == hipSuccess ? RL_DA_OK : RL_DA_ERR_HIP;
    }
    const bool small = w.rule.small;
    if (!small) {
        if (batch <= kPlanSequences && num_groups <= kPlanGroups)
            hipLaunchKernelGGL(plan_prefix<true>, dim3(1), dim3(kPlanThreads), 0, st, a);
        else
            hipLaunchKernelGGL(plan_prefix<false>, dim3(1), dim3(kPlanThreads), 0, st, a);
        if (hipGetLastError() != hipSuccess)
            return RL_DA_ERR_HIP;
    }
    const int64_t most = w.rule.max_units * num_kv_heads;
    const dim3 grid((unsigned)(most < kResident ? (most + kXcds - 1) / kXcds * kXcds : kResident));
    void (*attend)(PrefixArgs) = fp8 ? (small ? attend_prefix<true, true> : attend_prefix<true, false>)
                                     : (small ? attend_prefix<false, true>
                                              : attend_prefix<false, false>);
    hipLaunchKernelGGL(attend, grid, dim3(kAttendThreads), 0, st, a);
    if (hipGetLastError() != hipSuccess)
        return RL_DA_ERR_HIP;
    const int64_t rows = (int64_t)batch * num_q_heads;
    if (rows < kSpreadRows)
        hipLaunchKernelGGL(merge_prefix<true>, dim3((unsigned)rows), dim3(kMergeThreads), 0, st,
                           a);
    else
        hipLaunchKernelGGL(merge_prefix<false>,
                           dim3((unsigned)((rows + kMergeTeams - 1) / kMergeTeams)),
                           dim3(kMergeThreads), 0, st, a);
    return hipGetLastError() == hipSuccess ? RL_DA_OK : RL_DA_ERR_HIP;
}

}  // extern "C"
