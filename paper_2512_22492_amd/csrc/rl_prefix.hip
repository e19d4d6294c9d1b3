// rl_prefix.hip -- decode attention for sequences that share a prefix: the shared
// pages are read once for all of them.

#include <type_traits>

#include "rl_tile.h"

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
//
// A sequence shorter than its group's prefix is not a member: it attends all its
// keys as its own.  So every row of a shared unit sees every key of it, and a
// finished sequence (length 0) takes part in nothing.

constexpr int kMaxSplitPages = kWave * kUnitWaves;  // a lane of each wavefront per page
constexpr int kMinSplitPages = 16;
constexpr int kTargetUnits = 1024;
constexpr int kTileRows = 16;
constexpr float kNoScore = -3.0e38f;  // running max before the first key

// Splits of a run of `pages` pages: no longer than kMaxSplitPages, and for runs of
// kMinSplitPages and more as many as `wanted`, what the call's shape needs to fill
// the device.  Depends on the run's own length and the call's sizes only.
struct Splits {
    int count, pages;  // splits, pages of each but the last
};
__host__ __device__ __forceinline__ Splits splits_of(int pages, int wanted)
{
    Splits s = {0, 0};
    if (pages <= 0)
        return s;
    int n = (pages + kMaxSplitPages - 1) / kMaxSplitPages;
    const int more = min(pages / kMinSplitPages, wanted);
    n = more > n ? more : n;
    s.pages = (pages + n - 1) / n;
    s.count = (pages + s.pages - 1) / s.pages;
    return s;
}

// A unit of work for each kv head: query rows row0 .. row0 + rows - 1 (row = sequence
// * G + head of the group) against pages page0 .. of a table row.
struct Unit {
    int32_t table_row;
    int32_t page0;
    int32_t pages;
    int32_t limit;  // keys of the table row from here on are masked
    int32_t row0;
    int32_t rows;
    int32_t slot;   // partial result's place in the row's list; -1: the row's only one
    int32_t need;   // rows of sequences shorter than this are left out
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
    int32_t* num_units;         // workspace
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
    int32_t wanted_shared;      // splits that fill the device (splits_of)
    int32_t wanted_own;
    float scale_log2;           // scale * log2(e)
};

// ------------------------------------------------------------------ plan ---

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kClasses = 16;         // unit lengths, longest first
constexpr int kCachedGroups = 2048;  // group tables up to this size are searched in LDS

__device__ __forceinline__ int length_class(int pages)
{
    return kClasses - 1 - min((pages - 1) / (kMaxSplitPages / kClasses), kClasses - 1);
}

// Writes the units, longest first, and each sequence's number of partial results.
// Units of one class stand in any order: where a unit's results go does not depend
// on it.
__global__ __launch_bounds__(kPlanThreads) void plan_prefix(PrefixArgs a)
{
    __shared__ int starts[kCachedGroups + 1];
    __shared__ int cursor[kClasses];
    const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
    const bool cached = a.num_groups <= kCachedGroups;
    if (t < kClasses)
        cursor[t] = 0;
    if (cached && a.num_groups > 0)
        for (int i = t; i <= a.num_groups; i += kPlanThreads)
            starts[i] = a.group_start[i];
    __syncthreads();
    auto start_of = [&](int g) { return cached ? starts[g] : a.group_start[g]; };
    auto shared_pages = [&](int g) { return max(0, min(a.prefix_pages[g], a.max_pages)); };
    const int cap = a.max_pages * kPageSize;
    auto length_of = [&](int b) { return max(0, min(a.seq_lens[b], cap)); };

    // A sequence's shared pages (0 for one that is no member) and own splits.
    auto shared_of = [&](int b, int len) {
        // the last group that starts at or before b
        int lo = -1, hi = a.num_groups;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (start_of(mid) <= b)
                lo = mid;
            else
                hi = mid;
        }
        if (lo < 0 || start_of(lo + 1) <= b)
            return 0;  // in no group
        const int p = shared_pages(lo);
        return len >= p * kPageSize ? p : 0;
    };
    // A group's first member, whose table row the shared units read; -1: none.
    auto first_member = [&](int s0, int s1, int need) {
        for (int b0 = s0; b0 < s1; b0 += kWave) {
            const int b = b0 + lane;
            const uint64_t hit = __ballot(b < s1 && length_of(b) >= need);
            if (hit != 0)
                return b0 + (int)__builtin_ctzll(hit);
        }
        return -1;
    };

    // The two passes, counting and writing, visit the same units.
    auto pass = [&](auto sequence, auto shared) {
        for (int b = t; b < a.batch; b += kPlanThreads) {
            const int len = length_of(b);
            const int p = shared_of(b, len);
            sequence(b, len, p, splits_of((len + kPageSize - 1) / kPageSize - p, a.wanted_own));
        }
        for (int g = wave; g < a.num_groups; g += kPlanWaves) {
            const int s0 = max(0, min(start_of(g), a.batch));
            const int s1 = max(s0, min(start_of(g + 1), a.batch));
            const int p = shared_pages(g);
            if (p == 0)
                continue;
            const int leader = first_member(s0, s1, p * kPageSize);
            if (leader >= 0)
                shared(g, s0, s1, p, leader, splits_of(p, a.wanted_shared));
        }
    };
    pass(
        [&](int b, int len, int p, Splits s) {
            if (a.dev_error != nullptr && a.seq_lens[b] > cap)
                atomicOr(a.dev_error, RL_DA_DEVERR_LENGTH_TOO_LONG);
            const int ps = splits_of(p, a.wanted_shared).count;
            a.parts[b] = make_int2(ps, s.count);
            if (s.count > 0)
                atomicAdd(&cursor[length_class(s.pages)], s.count);
        },
        [&](int, int s0, int s1, int, int, Splits s) {
            const int tiles = (((s1 - s0) << a.group_shift) + kTileRows - 1) / kTileRows;
            if (lane == 0)
                atomicAdd(&cursor[length_class(s.pages)], s.count * tiles);
        });
    __syncthreads();
    if (t == 0) {
        int at = 0;
        for (int c = 0; c < kClasses; ++c) {
            const int n = cursor[c];
            cursor[c] = at;
            at += n;
        }
        // group_start that runs backwards could name more units than there is room for
        *a.num_units = min(at, a.max_units);
    }
    __syncthreads();
    auto put = [&](int at, const Unit& u) {
        if (at < a.max_units)
            a.units[at] = u;
    };
    pass(
        [&](int b, int len, int p, Splits s) {
            if (s.count == 0)
                return;
            const int at = atomicAdd(&cursor[length_class(s.pages)], s.count);
            const int total = (len + kPageSize - 1) / kPageSize;
            const int ps = splits_of(p, a.wanted_shared).count;
            for (int i = 0; i < s.count; ++i) {
                Unit u;
                u.table_row = b;
                u.page0 = p + i * s.pages;
                u.pages = min(s.pages, total - u.page0);
                u.limit = len;
                u.row0 = b << a.group_shift;
                u.rows = 1 << a.group_shift;
                u.slot = ps + s.count == 1 ? -1 : ps + i;
                u.need = 0;
                put(at + i, u);
            }
        },
        [&](int, int s0, int s1, int p, int leader, Splits s) {
            const int rows = (s1 - s0) << a.group_shift;
            const int tiles = (rows + kTileRows - 1) / kTileRows;
            int at = 0;
            if (lane == 0)
                at = atomicAdd(&cursor[length_class(s.pages)], s.count * tiles);
            at = __builtin_amdgcn_readfirstlane(at);
            // a split's tiles follow each other: they read the same pages
            for (int i = lane; i < s.count * tiles; i += kWave) {
                const int split = i / tiles, tile = i % tiles;
                Unit u;
                u.table_row = leader;
                u.page0 = split * s.pages;
                u.pages = min(s.pages, p - u.page0);
                u.limit = p * kPageSize;
                u.row0 = (s0 << a.group_shift) + tile * kTileRows;
                u.rows = min(kTileRows, rows - tile * kTileRows);
                u.slot = split;
                u.need = p * kPageSize;
                put(at + i, u);
            }
        });
}

// ---------------------------------------------------------------- attend ---
//
// A unit is one work-group of four wavefronts; wavefront w takes the unit's pages
// w, w + 4, ... for all its rows, each from a double buffer of its own in LDS that
// direct global-to-LDS loads fill: no barrier until the unit's end, where the four
// (m, l, O) are joined.  Both products run transposed (S^T = K Q^T, O^T += V^T P^T),
// so that a lane keeps one query row from the scores to the output and P^T goes from
// the score registers into the second product as it lies there.  Each weight enters
// the value product as two bf16 terms (hi + lo, 2^-16 relative).

constexpr int kAttendThreads = kWave * kUnitWaves;
constexpr int kBuffers = 2;
constexpr int kPageLds = kPageSize * kHeadDim * 2;           // a page of bf16 keys or values
constexpr int kWaveLds = kBuffers * 2 * kPageLds;
constexpr int kLdsBytes = kUnitWaves * kWaveLds;

template <int N>
__device__ __forceinline__ void wait_loads()  // all but the latest N of the wavefront's
{
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds()
{
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
}

// A row's float4 chunks (dims 4c .. 4c + 3) in the joining area, moved apart so that
// sixteen rows' equal chunks fall on different banks.
__device__ __forceinline__ float4* join_chunk(char* lds, int wave, int row, int c)
{
    return reinterpret_cast<float4*>(lds + wave * kWaveLds + row * (kHeadDim * 4)) +
           (c ^ (row & 15));
}

template <bool FP8>
__global__ __launch_bounds__(kAttendThreads) __attribute__((amdgpu_waves_per_eu(2))) void
attend_prefix(PrefixArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[kLdsBytes];
    __shared__ float2 join_ml[kUnitWaves][kTileRows];
    typedef __attribute__((address_space(3))) void lds_void;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int lane = threadIdx.x % kWave;
    const int i16 = lane & 15, g4 = lane >> 4;
    const int G = 1 << a.group_shift;
    char* const mine = lds + wave * kWaveLds;
    const uint32_t mine_at = (uint32_t)(uintptr_t)(lds_void*)mine;
    // bytes of a page's keys (or values) in a buffer, loads that bring both
    constexpr int kTile = FP8 ? kPageLds / 2 : kPageLds;
    constexpr int kLoads = 2 * kTile / 1024;
    // e4m3: a page's values widened to bf16, behind the buffers of raw pages
    char* const wide = mine + kBuffers * 2 * kTile;
    const int total = *a.num_units * a.num_kv_heads;
    const int64_t q_rows = a.num_q_heads;

    for (int at = blockIdx.x; at < total; at += gridDim.x) {
        const Unit u = a.units[at / a.num_kv_heads];
        const int kvh = at % a.num_kv_heads;
        const int count = wave < u.pages ? (u.pages - wave + kUnitWaves - 1) / kUnitWaves : 0;
        int my_page = 0;
        float my_ks = 1.0f, my_vs = 1.0f;
        if (lane < count) {
            my_page = a.block_table[(int64_t)u.table_row * a.max_pages + u.page0 + wave +
                                    lane * kUnitWaves];
            if (my_page < 0 || (int64_t)my_page >= a.num_pages) {
                // read another page instead; what the sequence gets is not defined
                if (a.dev_error != nullptr)
                    atomicOr(a.dev_error, RL_DA_DEVERR_PAGE_OUT_OF_RANGE);
                my_page = 0;
            }
            if (FP8) {
                const int64_t slab = (int64_t)my_page * a.num_kv_heads + kvh;
                my_ks = a.k_scale[slab];
                my_vs = a.v_scale[slab];
            }
        }
        // Q^T: lane holds row i16, dims 32 ks + 8 g4 .. + 7 (e4m3: the dims of the
        // codes it reads together, 64 (ks / 2) + 16 g4 + 8 (ks % 2) ..)
        const int my_row = u.row0 + min(i16, u.rows - 1);
        const uint16_t* qrow =
            a.q + ((int64_t)(my_row >> a.group_shift) * q_rows + kvh * G + (my_row & (G - 1))) *
                      kHeadDim;
        uint4 q[4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
            q[ks] = *reinterpret_cast<const uint4*>(
                qrow + (FP8 ? 64 * (ks / 2) + 16 * g4 + 8 * (ks % 2) : 32 * ks + 8 * g4));

        // keys of the wavefront's i-th page that count
        auto keys_of = [&](int i) {
            return u.limit - (u.page0 + wave + i * kUnitWaves) * kPageSize;
        };
        auto issue = [&](int i) {
            const int64_t page = __builtin_amdgcn_readlane(my_page, i);
            const int64_t base = page * a.page_bytes + (int64_t)kvh * a.head_bytes;
            const int last = min(keys_of(i), kPageSize) - 1;
            const uint32_t to = mine_at + (i % kBuffers) * 2 * kTile;
            constexpr int kRows = FP8 ? 8 : 4;       // rows of a page in one load
            constexpr int kLanes = kWave / kRows;    // lanes, chunks of a row
#pragma unroll
            for (int r = 0; r < kPageSize / kRows; ++r) {
                const int row = r * kRows + lane / kLanes;
                const int chunk = (lane % kLanes) ^ (FP8 ? row >> 1 : chunk_swizzle(row));
                // a key past the end is read as the last one (finite, weight 0)
                const int64_t off =
                    base + (int64_t)min(row, last) * a.row_bytes + 16 * chunk;
                dma16(a.k_pool + off, to + 1024 * r);
                dma16(a.v_pool + off, to + kTile + 1024 * r);
            }
        };

        float m = kNoScore, l = 0.0f;
        floatx4_t o[8];
#pragma unroll
        for (int db = 0; db < 8; ++db)
            o[db] = floatx4_t{0.0f, 0.0f, 0.0f, 0.0f};

        auto consume = [&](int i) {
            const char* kt = mine + (i % kBuffers) * 2 * kTile;
            const char* vt = kt + kTile;
            uint4 kv[4];
            if constexpr (FP8) {
                auto cvt = [](uint32_t w, auto upper) {
                    return __builtin_bit_cast(uint32_t,
                                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(
                                                  w, 1.0f, decltype(upper)::value));
                };
                using F = std::false_type;
                using T = std::true_type;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 c = *reinterpret_cast<const uint4*>(
                        kt + i16 * kHeadDim + 16 * ((4 * h + g4) ^ (i16 >> 1)));
                    kv[2 * h] = make_uint4(cvt(c.x, F{}), cvt(c.x, T{}), cvt(c.y, F{}),
                                           cvt(c.y, T{}));
                    kv[2 * h + 1] = make_uint4(cvt(c.z, F{}), cvt(c.z, T{}), cvt(c.w, F{}),
                                               cvt(c.w, T{}));
                }
                // values: lane holds rows lane / 8 and 8 + lane / 8, 16 codes of each
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int row = 8 * h + lane / 8, c0 = lane % 8;
                    const uint4 c = *reinterpret_cast<const uint4*>(
                        vt + row * kHeadDim + 16 * (c0 ^ (row >> 1)));
                    char* w = wide + row * (2 * kHeadDim);
                    const int sw = chunk_swizzle(row);
                    *reinterpret_cast<uint4*>(w + 16 * ((2 * c0) ^ sw)) =
                        make_uint4(cvt(c.x, F{}), cvt(c.x, T{}), cvt(c.y, F{}), cvt(c.y, T{}));
                    *reinterpret_cast<uint4*>(w + 16 * ((2 * c0 + 1) ^ sw)) =
                        make_uint4(cvt(c.z, F{}), cvt(c.z, T{}), cvt(c.w, F{}), cvt(c.w, T{}));
                }
                vt = wide;
            } else {
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    kv[ks] = *reinterpret_cast<const uint4*>(
                        kt + i16 * (2 * kHeadDim) + 16 * ((4 * ks + g4) ^ chunk_swizzle(i16)));
            }
            floatx4_t s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kv[ks]),
                                                            __builtin_bit_cast(bf16x8_t, q[ks]),
                                                            s, 0, 0, 0);
            // lane: row i16, keys 4 g4 .. + 3
            float mult = a.scale_log2, vs = 1.0f;
            if (FP8) {
                mult *= __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), i));
                vs = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), i));
            }
            const int keys = keys_of(i);
            float x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[j] = 4 * g4 + j < keys ? s[j] * mult : -INFINITY;
            float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
            mx = max_lanes_xor32(max_lanes_xor16(mx));
            if (__any(mx > m + kMaxSlack)) {
                const float m_new = mx > m + kMaxSlack ? mx : m;
                const float alpha = exp2_fast(m - m_new);
                m = m_new;
                l *= alpha;
#pragma unroll
                for (int db = 0; db < 8; ++db)
                    o[db] *= alpha;
            }
            float p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                p[j] = exp2_fast(x[j] - m);
                l += p[j];
                p[j] *= vs;
            }
            const uint32_t h0 = pack_bf16x2(p[0], p[1]), h1 = pack_bf16x2(p[2], p[3]);
            const uint2 hi = make_uint2(h0, h1);
            const uint2 lo = make_uint2(pack_bf16x2(p[0] - bf16_lo(h0), p[1] - bf16_hi(h0)),
                                        pack_bf16x2(p[2] - bf16_lo(h1), p[3] - bf16_hi(h1)));
            if constexpr (FP8)
                wave_lds_sync();  // the widened values are in place
            const int vrow = 4 * g4 + (i16 >> 2), vsw = chunk_swizzle(vrow);
#pragma unroll
            for (int db = 0; db < 8; ++db) {
                const uint2 vv = lds_read_transposed(reinterpret_cast<const uint16_t*>(
                    vt + vrow * (2 * kHeadDim) + 16 * ((2 * db + ((i16 & 3) >> 1)) ^ vsw) +
                    8 * (i16 & 1)));
                const short4_t v4 = __builtin_bit_cast(short4_t, vv);
                o[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
                    v4, __builtin_bit_cast(short4_t, hi), o[db], 0, 0, 0);
                o[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
                    v4, __builtin_bit_cast(short4_t, lo), o[db], 0, 0, 0);
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
        l = sum_lanes_xor32(sum_lanes_xor16(l));
        __syncthreads();  // all wavefronts are done with their buffers
#pragma unroll
        for (int db = 0; db < 8; ++db)
            *join_chunk(lds, wave, i16, 4 * db + g4) =
                make_float4(o[db][0], o[db][1], o[db][2], o[db][3]);
        if (g4 == 0)
            join_ml[wave][i16] = make_float2(m, l);
        __syncthreads();
        {
            const int row = threadIdx.x / 16;
            const int r = u.row0 + row, b = r >> a.group_shift;
            if (row < u.rows && a.seq_lens[b] >= u.need) {
                float2 ml[kUnitWaves];
                float M = kNoScore;
#pragma unroll
                for (int w = 0; w < kUnitWaves; ++w) {
                    ml[w] = join_ml[w][row];
                    M = fmaxf(M, ml[w].x);
                }
                float L = 0.0f, weight[kUnitWaves];
#pragma unroll
                for (int w = 0; w < kUnitWaves; ++w) {
                    weight[w] = exp2_fast(ml[w].x - M);
                    L = fmaf(weight[w], ml[w].y, L);
                }
                const int64_t out_row = (int64_t)b * a.num_q_heads + kvh * G + (r & (G - 1));
                const int64_t part = out_row * a.slots + max(u.slot, 0);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int c = threadIdx.x % 16 + 16 * h;
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int w = 0; w < kUnitWaves; ++w) {
                        const float4 x = *join_chunk(lds, w, row, c);
                        v.x = fmaf(weight[w], x.x, v.x);
                        v.y = fmaf(weight[w], x.y, v.y);
                        v.z = fmaf(weight[w], x.z, v.z);
                        v.w = fmaf(weight[w], x.w, v.w);
                    }
                    if (u.slot >= 0) {
                        *reinterpret_cast<float4*>(a.acc + part * kHeadDim + 4 * c) = v;
                    } else {
                        const float inv = 1.0f / L;
                        *reinterpret_cast<uint2*>(a.out + out_row * kHeadDim + 4 * c) =
                            make_uint2(pack_bf16x2(v.x * inv, v.y * inv),
                                       pack_bf16x2(v.z * inv, v.w * inv));
                    }
                }
                if (u.slot >= 0 && threadIdx.x % 16 == 0)
                    a.ml[part] = make_float2(M, L);
            }
        }
        __syncthreads();  // the next unit's loads overwrite the joining area
    }
}

// ----------------------------------------------------------------- merge ---
//
// 32 lanes per output row, four dims each; a row's partial results in order.

constexpr int kMergeRows = 8;  // of a work-group

__global__ __launch_bounds__(kMergeRows * 32) void merge_prefix(PrefixArgs a)
{
    const int64_t row = (int64_t)blockIdx.x * kMergeRows + threadIdx.x / 32;
    if (row >= (int64_t)a.batch * a.num_q_heads)
        return;
    const int c = threadIdx.x % 32;
    const int2 parts = a.parts[row / a.num_q_heads];
    const int n = parts.x + parts.y;
    if (parts.x == 0 && n == 1)
        return;  // its unit has written it
    const float2* ml = a.ml + row * a.slots;
    const float4* acc = reinterpret_cast<const float4*>(a.acc + row * a.slots * kHeadDim) + c;
    float M = kNoScore;
    for (int s = 0; s < n; ++s)
        M = fmaxf(M, ml[s].x);
    float den = 0.0f;
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int s = 0; s < n; ++s) {
        const float2 e = ml[s];
        const float4 x = acc[s * (kHeadDim / 4)];
        const float w = exp2_fast(e.x - M);
        den = fmaf(w, e.y, den);
        v.x = fmaf(w, x.x, v.x);
        v.y = fmaf(w, x.y, v.y);
        v.z = fmaf(w, x.z, v.z);
        v.w = fmaf(w, x.w, v.w);
    }
    const float inv = n > 0 ? 1.0f / den : 0.0f;  // no keys: zeros
    *reinterpret_cast<uint2*>(a.out + row * kHeadDim + 4 * c) = make_uint2(
        pack_bf16x2(v.x * inv, v.y * inv), pack_bf16x2(v.z * inv, v.w * inv));
}

// ------------------------------------------------------------------ host ---

struct Workspace {
    int64_t parts, units, ml, acc, bytes;  // offsets
    int32_t wanted_shared, wanted_own, slots;
    int64_t max_units;
};

int wanted_splits(int64_t pairs)
{
    return (int)((kTargetUnits + pairs - 1) / pairs);
}

// false: sizes past what the kernels index
bool lay_out(int32_t max_pages, int32_t batch, int32_t num_groups, int32_t num_q_heads,
             int32_t num_kv_heads, Workspace* w)
{
    const int64_t rows = (int64_t)batch * (num_q_heads / num_kv_heads);  // per kv head
    if (rows > INT32_MAX / 2 || (int64_t)batch * num_q_heads > INT32_MAX ||
        (int64_t)max_pages * kPageSize > INT32_MAX - kPageSize)
        return false;
    const int64_t tiles = (rows + kTileRows - 1) / kTileRows + num_groups;
    const int64_t pairs = (int64_t)batch * num_kv_heads;
    w->wanted_own = wanted_splits(pairs > 0 ? pairs : 1);
    // a group's rows share the splits of its prefix among 128-row tiles at least
    const int64_t shared_pairs =
        (int64_t)num_kv_heads * (num_groups > rows / 128 ? num_groups : rows / 128);
    w->wanted_shared = wanted_splits(shared_pairs > 0 ? shared_pairs : 1);
    // splits_of takes at most pages / kMaxSplitPages + 1 or `wanted`, whichever is more
    const int32_t least = max_pages / kMaxSplitPages + 1;
    const int32_t most = max_pages / kMinSplitPages + 1;
    const int32_t shared = least > (w->wanted_shared < most ? w->wanted_shared : most)
                               ? least
                               : (w->wanted_shared < most ? w->wanted_shared : most);
    const int32_t own = least > (w->wanted_own < most ? w->wanted_own : most)
                            ? least
                            : (w->wanted_own < most ? w->wanted_own : most);
    w->slots = shared + own;
    w->max_units = tiles * shared + (int64_t)batch * own;
    if (w->max_units * num_kv_heads > INT32_MAX / 2)
        return false;
    auto round = [](int64_t n) { return (n + 255) / 256 * 256; };
    w->parts = 256;
    w->units = w->parts + round((int64_t)batch * (int64_t)sizeof(int2));
    w->ml = w->units + round(w->max_units * (int64_t)sizeof(Unit));
    const int64_t partials = (int64_t)batch * num_q_heads * w->slots;
    w->acc = w->ml + round(partials * (int64_t)sizeof(float2));
    w->bytes = w->acc + round(partials * kHeadDim * (int64_t)sizeof(float));
    return true;
}

// Work-groups that the device holds at once.
constexpr int kResident = 256 * 2;

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
        (G != 1 && G != 2 && G != 4 && G != 8 && G != 16))
        return RL_DA_ERR_UNSUPPORTED;
    Workspace w;
    if (!lay_out(max_pages, batch, num_groups, num_q_heads, num_kv_heads, &w))
        return RL_DA_ERR_UNSUPPORTED;
    if (workspace_bytes < (size_t)w.bytes)
        return RL_DA_ERR_INVALID_ARG;
    if (batch == 0)
        return RL_DA_OK;
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
    a.num_units = (int32_t*)ws;
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
    a.max_units = (int32_t)w.max_units;
    a.slots = w.slots;
    a.wanted_shared = w.wanted_shared;
    a.wanted_own = w.wanted_own;
    a.scale_log2 = scale * kLog2e;
    hipStream_t st = (hipStream_t)stream;
    hipLaunchKernelGGL(plan_prefix, dim3(1), dim3(kPlanThreads), 0, st, a);
    if (hipGetLastError() != hipSuccess)
        return RL_DA_ERR_HIP;
    const int64_t most = w.max_units * num_kv_heads;
    const dim3 grid((unsigned)(most < kResident ? most : kResident));
    if (fp8)
        hipLaunchKernelGGL(attend_prefix<true>, grid, dim3(kAttendThreads), 0, st, a);
    else
        hipLaunchKernelGGL(attend_prefix<false>, grid, dim3(kAttendThreads), 0, st, a);
    if (hipGetLastError() != hipSuccess)
        return RL_DA_ERR_HIP;
    const int64_t rows = (int64_t)batch * num_q_heads;
    hipLaunchKernelGGL(merge_prefix, dim3((unsigned)((rows + kMergeRows - 1) / kMergeRows)),
                       dim3(kMergeRows * 32), 0, st, a);
    return hipGetLastError() == hipSuccess ? RL_DA_OK : RL_DA_ERR_HIP;
}

}  // extern "C"
