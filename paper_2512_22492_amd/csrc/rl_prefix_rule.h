// rl_prefix_rule.h -- which way a call of the shared-prefix attention goes, and how runs of
// pages are cut.  Plain integer functions of the call's sizes and of a run's length, for
// the host and the device.

#pragma once

#include <stdint.h>

#if defined(__HIP__)
#define RL_RULE_HD __host__ __device__
#else
#define RL_RULE_HD
#endif

namespace rl_da {

RL_RULE_HD inline int smaller(int a, int b) { return a < b ? a : b; }
RL_RULE_HD inline int larger(int a, int b) { return a > b ? a : b; }

constexpr int kRulePage = 16;         // tokens of a page
constexpr int kMaxSplitPages = 256;   // a lane of each of a unit's wavefronts per page
// Own runs of up to a page per wavefront of a unit are a wavefront's alone: it has no one
// to wait for, and a work-group takes four (512 sequences x 8 kv heads of one token
// 36 -> 19 us); where there are wavefronts' worth of them for several rounds, up to
// sixteen pages (of 1..200 tokens 61 -> 50 us, e4m3 51 -> 35; 64 sequences of 256 tokens,
// which are not, 20 -> 38).
constexpr int kAlonePages = 4, kAloneManyPages = 16;
constexpr int kTileRows = 128;        // query rows of a shared unit at most
// The plan of a small call, which every work-group of the attention kernel makes for
// itself, a lane per sequence and per group: the launch of plan_prefix and the wait for
// it cost 3 us (four responses to a short prompt 15.2 -> 12.2).
constexpr int kSmallCall = 64;        // sequences and groups at most

// Splits of a run of `pages` pages: no longer than kMaxSplitPages, and as many as
// `wanted`, what the call's shape needs to fill the device, of 2^least_shift pages at
// least.  Depends on the run's own length and the call's sizes only.
struct Splits {
    int count, pages, more;  // splits; pages of each, and one more of the first `more`
    RL_RULE_HD int first(int i) const { return i * pages + smaller(i, more); }
    RL_RULE_HD int size(int i) const { return pages + (i < more ? 1 : 0); }
};
RL_RULE_HD inline Splits splits_of(int pages, int wanted, int least_shift)
{
    Splits s;
    s.count = larger((pages + kMaxSplitPages - 1) / kMaxSplitPages,
                     smaller(pages >> least_shift, wanted));
    s.pages = pages;
    s.more = 0;
    if (s.count > 1) {
        s.pages = pages / s.count;
        s.more = pages - s.pages * s.count;
    }
    return s;
}

// Work-groups that the device holds at once.
constexpr int kResident = 256 * 2;

// How many units a call's shared and own runs are cut into, kv heads included, and the
// least pages of one.  A call whose (sequence, kv head) pairs leave the device idle is
// cut finely, into one round of units; one that fills it coarsely, since units and their
// partial results cost more there (8 responses of 1000..8000 tokens to one prompt of
// 2000, 8 kv heads: 39.5 us cut coarsely, 31.6 finely; 64 responses of 2000 to 8 prompts
// 105.5 coarsely, 114.4 finely).  Own runs of a call of a round or two are cut into
// two rounds and more, so that what is left over is short; everything else into no more
// than a round, which a few units past it would double (56 pairs of 675 shared pages: ten splits 58 us, nine
// 44.6; 120 of 499: five splits 110, four 98).
struct SplitGoal {
    int shared, own, least_shift;
    bool past_round;
};
constexpr SplitGoal kFewPairs = {512, 512, 4, false}, kManyPairs = {512, 1024, 5, true};
constexpr int kFew = kResident / 2;  // pairs

inline int wanted_splits(int64_t target, int64_t pairs, bool past)
{
    if (pairs < 1)
        pairs = 1;
    const int64_t n = (target + (past ? pairs - 1 : 0)) / pairs;
    return (int)(n > 1 ? n : 1);
}

// Fewer output rows than this are merged by a work-group each: a call of few rows cuts
// their keys into many splits, and its merge is bound by walking them.
constexpr int kSpreadRows = 2048;

// In calls whose (sequence, kv head) pairs fit the device at once a short prefix is read
// with each sequence's own pages: it comes from the caches, and a unit and a partial
// result less is worth more (16 responses of up to 80 tokens to 2 prompts of 400, 8 kv
// heads: 16.7 -> 13.5 us; 150 to 600: 19.9 -> 17.1).  At the rule's edge, 512 pairs of up to
// 160 tokens of their own under prefixes of 16, 32 and 48 pages in wide tables, bf16, us
// unshared (shared): 64 sequences of 8 kv heads under one prefix 15.5 (16.6), 19.3
// (22.0), 22.6 (27.2), under 8 prefixes 15.6 (15.7), 19.4 (19.9), 23.0 (24.1).  A kv head
// of eight stays on one XCD, whose L2 cache its group shares; of one kv head the
// members lie on different XCDs, and many short groups lose: 512 sequences under 16
// prefixes 19.7 (22.7), 23.6 (26.2), 27.4 (31.4), under 64 prefixes 25.1 (20.8), 34.3
// (24.2), 44.5 (28.4).
constexpr int kUnsharedPages = 48;
// Tables up to this width are then attended row by row altogether (the same calls with
// tables as wide as they need: 16.6 -> 9.0 us, 19.8 -> 11.8; 64 pages 23.0 -> 14.8).  At the
// edge, by rows (shared): 64 sequences of 8 kv heads under one prefix of 16, 32 and 48
// pages 11.1 (16.2), 13.9 (21.7), 16.8 (27.0); 512 of one kv head under 64 prefixes
// 17.4 (20.8), 26.3 (24.1), 35.6 (28.3).
constexpr int kRowPages = 64;

struct PrefixRule {
    bool by_rows;            // one kernel, a work-group per sequence and kv head
    bool small;              // else: planned inside the attention kernel
    int32_t unshared_pages;  // prefixes up to this length count as own pages
    int32_t alone_pages;     // own runs up to this length are a wavefront's
    int32_t wanted_shared;   // splits that fill the device (splits_of)
    int32_t wanted_own;
    int32_t least_shift;     // log2 of a split's least pages
    int32_t slots;           // partial results that a row can have
    int64_t max_units;       // that a plan can have, each for all kv heads
};

inline PrefixRule prefix_rule(int32_t max_pages, int32_t batch, int32_t num_groups,
                              int32_t num_q_heads, int32_t num_kv_heads)
{
    PrefixRule r;
    const int64_t rows = (int64_t)batch * (num_q_heads / num_kv_heads);  // per kv head
    const int64_t pairs = (int64_t)batch * num_kv_heads;
    r.by_rows = max_pages <= kRowPages && pairs <= kResident;
    r.small = batch <= kSmallCall && num_groups <= kSmallCall;
    r.unshared_pages = pairs <= kResident ? kUnsharedPages : 0;
    r.alone_pages = pairs >= 4 * kResident ? kAloneManyPages : kAlonePages;
    const SplitGoal& goal = pairs <= kFew ? kFewPairs : kManyPairs;
    r.least_shift = goal.least_shift;
    r.wanted_own = wanted_splits(goal.own, pairs, goal.past_round);
    // a group's rows share the splits of its prefix among 128-row tiles at least
    const int64_t shared_pairs =
        (int64_t)num_kv_heads * (num_groups > rows / kTileRows ? num_groups : rows / kTileRows);
    r.wanted_shared = wanted_splits(goal.shared, shared_pairs, false);
    // splits_of takes at most pages / kMaxSplitPages + 1 or `wanted`, whichever is more
    const int32_t least = max_pages / kMaxSplitPages + 1;
    const int32_t most = (max_pages >> goal.least_shift) + 1;
    auto slots = [&](int32_t wanted) { return larger(least, smaller(wanted, most)); };
    const int32_t shared = slots(r.wanted_shared), own = slots(r.wanted_own);
    r.slots = shared + own;
    const int64_t tiles = (rows + kTileRows - 1) / kTileRows + num_groups;
    r.max_units = tiles * shared + (int64_t)batch * own;
    return r;
}

// A unit of work for each kv head: query rows row0 .. row0 + rows - 1 (row = sequence
// * G + head of the group) against pages page0 .. of a table row.
struct Unit {
    int32_t table_row;
    int32_t page0;
    int32_t pages;
    int32_t limit;  // keys of the table row from here on are masked
    int32_t row0;
    int32_t rows;   // negated: other units read the same pages
    int32_t slot;   // partial result's place in the row's list; -1: the row's only one
    int32_t need;   // rows of sequences shorter than this are left out
};

// The functions below take what they need of a call from any struct `a` with the rule's
// cuts (unshared_pages, alone_pages, wanted_shared, wanted_own, least_shift), batch,
// max_pages and group_shift (log2 of the query heads per kv head).

// A group's prefix, and the pages of it that are attended once for all members.
template <class Call>
RL_RULE_HD inline int prefix_of(const Call& a, int pages)
{
    return larger(0, smaller(pages, a.max_pages));
}
template <class Call>
RL_RULE_HD inline int shared_pages(const Call& a, int pages)
{
    const int p = prefix_of(a, pages);
    return p > a.unshared_pages ? p : 0;
}

// A sequence's own run and its splits.
struct Own {
    int len, first, shared;  // tokens, first own page, partial results of the shared ones
    int others;              // pages up to here are read by other sequences too
    Splits s;
    template <class Call>
    RL_RULE_HD bool alone(const Call& a) const
    {
        return s.count == 1 && s.pages <= a.alone_pages;
    }
};
// len: the sequence's tokens, 0 .. max_pages * page; prefix: of the group it is a member
// of, 0 of none; company: the group has other sequences.
template <class Call>
RL_RULE_HD inline Own own_of(const Call& a, int len, int prefix, bool company)
{
    Own o;
    o.len = len;
    o.first = shared_pages(a, prefix);
    o.shared = splits_of(o.first, a.wanted_shared, a.least_shift).count;
    o.others = company ? prefix : 0;
    o.s = splits_of(larger((o.len + kRulePage - 1) / kRulePage - o.first, 0), a.wanted_own,
                    a.least_shift);
    return o;
}
template <class Call>
RL_RULE_HD inline Unit own_unit(const Call& a, int b, const Own& o, int i)
{
    Unit u;
    u.table_row = b;
    u.page0 = o.first + o.s.first(i);
    u.pages = o.s.size(i);
    u.limit = o.len;
    u.row0 = b << a.group_shift;
    u.rows = 1 << a.group_shift;
    if (u.page0 < o.others)
        u.rows = -u.rows;
    u.slot = o.shared + o.s.count == 1 ? -1 : o.shared + i;
    u.need = 0;
    return u;
}

// A group's shared run: its splits, each for every tile of query rows.
struct Shared {
    int s0, rows, tiles, pages;
    Splits s;
    RL_RULE_HD int units() const { return s.count * tiles; }
};
template <class Call>
RL_RULE_HD inline Shared shared_of(const Call& a, int start, int end, int pages)
{
    Shared h;
    h.s0 = larger(0, smaller(start, a.batch));
    h.rows = (larger(h.s0, smaller(end, a.batch)) - h.s0) << a.group_shift;
    h.tiles = (h.rows + kTileRows - 1) / kTileRows;
    h.pages = shared_pages(a, pages);
    h.s = splits_of(h.pages, a.wanted_shared, a.least_shift);
    return h;
}
// Unit i of a group; a split's tiles follow each other: they read the same pages, from
// the table row of `leader`, a member.
template <class Call>
RL_RULE_HD inline Unit shared_unit(const Call& a, const Shared& h, int leader, int i)
{
    const int split = i / h.tiles, tile = i % h.tiles;
    Unit u;
    u.table_row = leader;
    u.page0 = h.s.first(split);
    u.pages = h.s.size(split);
    u.limit = h.pages * kRulePage;
    u.row0 = (h.s0 << a.group_shift) + tile * kTileRows;
    u.rows = smaller(kTileRows, h.rows - tile * kTileRows);
    if (h.tiles > 1)
        u.rows = -u.rows;
    u.slot = split;
    u.need = h.pages * kRulePage;
    return u;
}

}  // namespace rl_da
