// Which tiles of keys and queries meet, and in which order blocks take them: host arithmetic of the attention operators (no HIP in here).
#pragma once
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <vector>

// Query p (a position) sees key j if j <= p + right and (j >= p - left or j < sinks); a negative left or right is no limit.
struct AttentionRules {
    int64_t left, right, sinks;
};

constexpr int ATT_STEP = 64;   // keys, or queries, that a block takes at once from the other side
constexpr int ATT_XCDS = 8;    // blocks go to them in turn, and each has its own L2

// Tiles of ATT_STEP rows, numbered from the sequence's start: 0 .. sink_tiles - 1, then first_tile and on; `tiles` together.
struct AttentionSpan {
    int32_t sink_tiles, first_tile, tiles;
};

// Key tiles that queries at positions p0 .. p1 see of a sequence of lk keys.
inline AttentionSpan att_keys_seen(const AttentionRules &r, int64_t p0, int64_t p1, int64_t lk)
{
    const int64_t hi = r.right < 0 ? lk - 1 : std::min(lk - 1, p1 + r.right);
    if (hi < 0) return {0, 0, 0};
    const int64_t lo = r.left < 0 ? 0 : std::max<int64_t>(0, p0 - r.left);
    const int64_t last = hi / ATT_STEP, first = lo > hi ? last + 1 : lo / ATT_STEP;
    const int64_t sinks = std::min((std::min(r.sinks, hi + 1) + ATT_STEP - 1) / ATT_STEP, first);
    return {(int32_t)sinks, (int32_t)first, (int32_t)(sinks + last - first + 1)};
}

// Query tiles of a sequence of lq queries, the first at position `first`, that see any of the keys j0 .. j1.
inline AttentionSpan att_queries_seen(const AttentionRules &r, int64_t j0, int64_t j1, int64_t lq, int64_t first)
{
    const int64_t from = r.right < 0 ? 0 : std::max<int64_t>(0, j0 - r.right - first);
    const int64_t to = r.left < 0 || j0 < r.sinks ? lq - 1 : std::min(lq - 1, j1 + r.left - first);
    if (to < from) return {0, 0, 0};
    return {0, (int32_t)(from / ATT_STEP), (int32_t)(to / ATT_STEP - from / ATT_STEP + 1)};
}

// A block's rows and what it goes through; 64 bytes, read by one wide scalar load.
struct AttentionTile {
    int32_t row0, rows;            // own rows: the first among all of its side, how many
    int32_t other0, others;        // the sequence's rows on the other side
    int32_t at;                    // position of the first own query; of key tiles, number of the first key
    int32_t first;                 // position of the sequence's first query
    int32_t sink_tiles, first_tile;
    int32_t begin, end;            // of the tiles on the other side, numbered as in AttentionSpan; of key tiles: those of every head that shares the key head, one head after another
    int32_t slot;                  // where a part of them leaves its sums, -1: the block has all
    int32_t per_head;              // tiles on the other side
    int32_t pad[4];
};

// Rows whose other side was split: the parts' slots.
struct AttentionJoin {
    int32_t row0, rows, slot0, slots;
};

struct AttentionItem {
    int32_t tile, head;  // tile -1: nothing to do
};

// A side's tiles of `block_rows` rows of every sequence, and the joins.  share: heads per key head.  without: sequences that are left out.  split > 0: no block has more than `split` tiles of the other side.
inline void att_make_tiles(const AttentionRules &r, int n, const int32_t *q_rows, const int32_t *k_rows, const int32_t *first, bool keys, int share, int block_rows,
                           int split, std::vector<AttentionTile> &tiles, std::vector<int32_t> &tiles_of, std::vector<AttentionJoin> &joins,
                           const std::vector<char> *without = nullptr)
{
    int64_t q0 = 0, k0 = 0;
    int32_t slots = 0;
    tiles_of.assign(n + 1, 0);
    for (int s = 0; s < n; ++s) {
        const int64_t lq = q_rows[s], lk = k_rows[s], f = first[s];
        for (int64_t i = 0; i < (keys ? lk : lq) && !(without && (*without)[s]); i += block_rows) {
            const int64_t rows = std::min<int64_t>(block_rows, (keys ? lk : lq) - i);
            const AttentionSpan span = keys ? att_queries_seen(r, i, i + rows - 1, lq, f) : att_keys_seen(r, f + i, f + i + rows - 1, lk);
            AttentionTile t = {};
            t.row0 = (int32_t)((keys ? k0 : q0) + i);
            t.rows = (int32_t)rows;
            t.other0 = (int32_t)(keys ? q0 : k0);
            t.others = (int32_t)(keys ? lq : lk);
            t.at = (int32_t)(keys ? i : f + i);
            t.first = (int32_t)f;
            t.sink_tiles = span.sink_tiles;
            t.first_tile = span.first_tile;
            t.slot = -1;
            t.per_head = span.tiles;
            const int64_t count = (int64_t)span.tiles * (keys ? share : 1);
            const int parts = split > 0 ? (int)std::max<int64_t>(1, (count + split - 1) / split) : 1;
            for (int p = 0; p < parts; ++p) {
                t.begin = (int32_t)(count * p / parts);
                t.end = (int32_t)(count * (p + 1) / parts);
                if (parts > 1) t.slot = slots + p;
                tiles.push_back(t);
            }
            if (parts > 1) {
                joins.push_back({t.row0, t.rows, slots, parts});
                slots += parts;
            }
        }
        tiles_of[s + 1] = (int32_t)tiles.size();
        q0 += lq;
        k0 += lk;
    }
}

// How many tiles a block may have so that parts of the longest ones fill the compute units: `blocks` of them per unit, `least` tiles at least; 0: nothing is long enough.
inline int att_split(const std::vector<AttentionTile> &tiles, int heads, int cus, int blocks, int least)
{
    int64_t work = 0, most = 0;
    for (const AttentionTile &t : tiles) {
        work += t.end - t.begin;
        most = std::max<int64_t>(most, t.end - t.begin);
    }
    const int64_t split = std::max<int64_t>(least, (work * heads + blocks * cus - 1) / (blocks * cus));
    return 2 * most > 3 * split ? (int)std::min<int64_t>(split, 0x7fffffff) : 0;
}

// In which order blocks take (tile, head).  A sequence's tiles that read the same rows of the other side (all of them, and the heads that share a key head) go to one
// XCD, whose L2 then has those rows; pieces of a 64th of all work, where a sequence has more, so that the XCDs' shares are alike; the dearest pieces first.
// own_heads: heads per tile, `share` of them adjacent read the same rows.
inline std::vector<AttentionItem> att_order(const std::vector<AttentionTile> &tiles, const std::vector<int32_t> &tiles_of, int own_heads, int share)
{
    struct Piece {
        int64_t cost;
        int32_t from, to;  // tiles [from, to)
    };
    auto cost = [&](int t) { return (int64_t)(tiles[t].end - tiles[t].begin) * ((tiles[t].rows + 31) / 32) + 8; };  // of a wavefront's tiles; 8: what a block takes besides
    const int groups = own_heads / share;
    int64_t total = 0;
    for (size_t t = 0; t < tiles.size(); ++t) total += cost((int)t);
    total *= groups;
    std::vector<Piece> pieces;
    pieces.reserve(tiles_of.size());
    for (size_t s = 0; s + 1 < tiles_of.size(); ++s) {
        Piece p = {0, tiles_of[s], tiles_of[s]};
        for (int t = tiles_of[s]; t < tiles_of[s + 1]; ++t) {
            p.cost += cost(t);
            p.to = t + 1;
            if (t + 1 == tiles_of[s + 1] || p.cost * (8 * ATT_XCDS) >= total) {
                pieces.push_back(p);
                p = {0, t + 1, t + 1};
            }
        }
    }
    std::stable_sort(pieces.begin(), pieces.end(), [](const Piece &a, const Piece &b) { return a.cost > b.cost; });
    // to the XCD that has the least so far; first how many items each gets, then where they lie
    std::vector<uint8_t> xcds(pieces.size() * groups);
    int64_t load[ATT_XCDS] = {};
    size_t count[ATT_XCDS] = {}, at = 0;
    for (const Piece &p : pieces)
        for (int g = 0; g < groups; ++g) {
            int x = 0;
            for (int i = 1; i < ATT_XCDS; ++i) x = load[i] < load[x] ? i : x;
            load[x] += p.cost;
            count[x] += (size_t)(p.to - p.from) * share;
            xcds[at++] = (uint8_t)x;
        }
    std::vector<AttentionItem> items(*std::max_element(count, count + ATT_XCDS) * ATT_XCDS, AttentionItem{-1, 0});
    AttentionItem *next[ATT_XCDS];
    for (int x = 0; x < ATT_XCDS; ++x) next[x] = items.data() + x;
    at = 0;
    for (const Piece &p : pieces)
        for (int g = 0; g < groups; ++g) {
            AttentionItem *&to = next[xcds[at++]];
            for (int t = p.from; t < p.to; ++t)
                for (int h = 0; h < share; ++h, to += ATT_XCDS) *to = {t, g * share + h};
        }
    return items;
}

// Bucket of each relative position (key minus query) from -distance to distance.  Of a direction's buckets the first half hold one distance each, the others ranges whose
// bounds grow by equal factors up to `distance`, which belongs to the last one with all beyond.  Both directions: half of the buckets each, keys ahead the upper half; one
// direction: keys ahead count as distance 0.  Bounds that are whole numbers (powers of one factor) are met exactly: 1e-12 is far above long double's error, and no other
// quotient of logarithms of numbers up to 1024 comes that near to a whole number.
inline void att_position_buckets(int buckets, int distance, bool both, int32_t *bucket_of)
{
    const int half = both ? buckets / 2 : buckets, single = half / 2;
    for (int d = -distance; d <= distance; ++d) {
        const int n = d < 0 ? -d : both ? d : 0;
        int b = n;
        if (n >= single) {
            const long double at = (half - single) * (std::log((long double)n / single) / std::log((long double)distance / single));
            b = std::min(half - 1, single + (int)std::floor(at + 1e-12L));
        }
        bucket_of[d + distance] = b + (both && d > 0 ? half : 0);
    }
}

// Whether any of a's rows (of a_cols elements, lda >= a_cols apart) shares a byte with any of b's.  Rows of one may lie between those of the other.
inline bool att_overlap(uint64_t a, int64_t lda, int64_t a_cols, int64_t a_rows, uint64_t b, int64_t ldb, int64_t b_cols, int64_t b_rows, int size)
{
    typedef __int128 Wide;
    if (a_rows < 1 || b_rows < 1) return false;
    const Wide a_step = (Wide)lda * size, b_step = (Wide)ldb * size, a_bytes = (Wide)a_cols * size, b_bytes = (Wide)b_cols * size, d = (Wide)b - a;
    if (d >= (a_rows - 1) * a_step + a_bytes || -d >= (b_rows - 1) * b_step + b_bytes) return false;
    if (a_step == b_step) {  // side by side in the rows of one matrix, as slices of a projection's output are
        const Wide phase = ((d % a_step) + a_step) % a_step;
        if (phase >= a_bytes && a_step - phase >= b_bytes) return false;
    }
    for (int64_t j = 0; j < b_rows; ++j) {  // b's row j against the last of a's rows that begin before its end: those before that one end earlier
        const Wide start = d + j * b_step, last = start + b_bytes - 1;
        if (last < 0) continue;
        const Wide i = last / a_step < a_rows - 1 ? last / a_step : a_rows - 1;
        if (i * a_step + a_bytes > start) return true;
    }
    return false;
}
