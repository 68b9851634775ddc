// Attention over ragged sequences with a bias by relative position, a sliding window and first tokens that stay visible: the forward pass and the plan (gfx950).
#include <math.h>
#include <string.h>

#include <new>

#include "adapter_plan.h"
#include "attention.h"
#include "wave.h"

namespace {

// ------------------------------------------------------------------ forward
// A block takes NW * 32 queries of one head through their keys, 64 at a time; a wavefront has 32 queries.  S^T = K Q^T, so that a lane owns one query: its maximum and sum
// run over its own registers, the other half of the keys is lane ^ 32's.  The bias is what the products are added to.  One pass: m the largest score so far, l = sum of
// weights 2^(scale log2 e (s - m)), O = sum of weights times v, l and O scaled when m grows.  P^T, rounded to the inputs' type (an error of half a step in each term, as the inputs themselves have), is the
// other operand of O^T = V^T P^T without leaving its registers, see Columns.
// K and V tiles go from memory to LDS without registers, one tile ahead (two ahead, with a third stage, took the same time).
// What bounds it: over few queries memory (12 heads of 64, single queries over 8 sequences of 500 to 16384 keys: 39 us, 222 MB, 5.6 TB/s).  Else a block's loads and stores, and its
// steps, overlap in part only with three wavefronts per SIMD: 256 sequences of up to 512 tokens 146 to 151 us, of which memory needs 80 and the steps some 95; vector units 56 %,
// matrix cores 25 % busy (ten vector instructions per score and lane; a sixth of them less gave 0.8 %; four wavefronts per SIMD spill registers, 200 us and more).
// Three documents of 3001 to 4096 tokens with a window of 256: 38 to 39 us, 960 blocks in two rounds; of 64 queries, with two wavefronts at each 32 and their sums joined in
// LDS, 37 to 40, and 40 sequences of 256 tokens 26 instead of 23.
template <int DP, int NW>
struct AttendCfg {
    static constexpr int STAGES = 2, TILE = ATT_STEP * DP;
    static constexpr int FIXED = STAGES * 2 * TILE * 2;  // bytes; the bias's table follows
};

template <class T, int DP, int NW, bool BIAS>
__global__ __launch_bounds__(NW * 64, NW == 4 ? (DP == 128 ? 2 : 3) : 1) void attend_kernel(const AttentionItem *__restrict__ items, const AttentionTile *__restrict__ tiles, AttentionShape a,
                                                                         const T *__restrict__ q, int64_t ldq, const T *__restrict__ k, int64_t ldk,
                                                                         const T *__restrict__ v, int64_t ldv, const float *__restrict__ bias,
                                                                         const int32_t *__restrict__ bucket_of, T *__restrict__ out, int64_t ldo,
                                                                         float *__restrict__ lse, int64_t Tq, float *__restrict__ part_o,
                                                                         float2 *__restrict__ part_ml)
{
    typedef typename Half8<T>::type V8;
    typedef TileRequests<T, DP, NW> Requests;
    constexpr int STAGES = AttendCfg<DP, NW>::STAGES, TILE = AttendCfg<DP, NW>::TILE, ND = DP / 32, NS = DP / 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    T *Ks = reinterpret_cast<T *>(smem), *Vs = Ks + STAGES * TILE;
    float *table = reinterpret_cast<float *>(smem + AttendCfg<DP, NW>::FIXED);

    const AttentionItem item = items[blockIdx.x];
    if (item.tile < 0) return;
    const AttentionTile t = tiles[item.tile];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int h = item.head, g = h / a.share;
    const T *kb = k + (int64_t)t.other0 * ldk + g * a.dim, *vb = v + (int64_t)t.other0 * ldv + g * a.dim;
    auto key_of = [&](int u) { return (u < t.sink_tiles ? u : t.first_tile + u - t.sink_tiles) * ATT_STEP; };

    Requests kr, vr;
    kr.init(ldk, a.dim, wave, lane);
    vr.init(ldv, a.dim, wave, lane);
    auto request = [&](int u, int stage) {
        const int j = key_of(u);
        kr.request(kb + j * ldk, ldk, t.others - j, a.dim, Ks + stage * TILE, wave);
        vr.request(vb + j * ldv, ldv, t.others - j, a.dim, Vs + stage * TILE, wave);
    };
    const int my_rows = min(32, t.rows - wave * 32), p0 = t.at + wave * 32;  // of this wavefront
    const int my_row = t.row0 + wave * 32 + l32;
    V8 qf[NS];
    load_rows<T, DP>(q + (int64_t)(t.row0 + wave * 32) * ldq + h * a.dim, ldq, my_rows, a.dim, lane, qf);
    if (t.begin < t.end) request(t.begin, 0);
    if (BIAS) make_bias(table, bias, bucket_of, a, h);

    f32x16 o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    float m = -INFINITY, l = 0.f;
    arrived(qf);
    take_sign(qf, a.scale);
    const float scale2 = __builtin_fabsf(a.scale) * LOG2E;
    const int p = p0 + l32;

    Columns<T, DP> columns;
    columns.init(lane);
    int stage = 0;
    for (int u = t.begin; u < t.end; ++u) {
        const int j0 = key_of(u);
        const T *Kt = Ks + stage * TILE, *Vt = Vs + stage * TILE;
        wait_for_requests<0>();
        block_barrier();  // this tile is there, and the stage of the last one has been read
        if (u + 1 < t.end) request(u + 1, stage ^ 1);
        stage ^= 1;
        const int keys = min(ATT_STEP, t.others - j0);
        const Sight see = sight(a, p0, my_rows, j0, keys);
        if (see.none) continue;

        f32x16 s[2];
        if (BIAS) {
            const int least = j0 - (p0 + 31), most = j0 + ATT_STEP - 1 - p0;  // relative positions
            const bool near = most > -a.distance && least < a.distance;
            if (near) {
                const int at = one_register(AttendCfg<DP, NW>::FIXED / 4 + j0 + 4 * half - p + a.distance + ATT_EXT);
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[kt][r] = reinterpret_cast<const float *>(smem)[at + kt * 32 + acc_row(r)];
            } else {  // one bias for all, a part of the scores as any other: it may be -inf, or all of a row's lowest
                const float c = table[most <= -a.distance ? 0 : bias_entries(a.distance) - 1];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[kt][r] = c;
            }
        } else {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
        }
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < NS; ++i) s[kt] = att_mfma(row_operand<T, DP>(Kt, kt * 32, i, lane), qf[i], s[kt]);
        V8 vf[2][ND];  // of the first 32 keys, on their way while the scores become weights
        columns.template two<0>(Vt, vf);
        // register r of tile kt is key j0 + 32 kt + 4 half + acc_row(r)
        const int j = j0 + 4 * half;
        const Edges e = edges(a, p0, my_rows, j0, keys);
        if (e.behind) {
            const int most = min(t.others - 1, p + a.right) - j;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = kt * 32 + acc_row(r) > most ? -INFINITY : s[kt][r];
        }
        if (e.before) {
            const int least = p - a.left - j, sinks = a.sinks - j;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = kt * 32 + acc_row(r);
                    s[kt][r] = ((key < least) & (key >= sinks)) ? -INFINITY : s[kt][r];
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, s[kt][r]);
        top = __builtin_fmaxf(m, both_halves_max(top));
        // m follows the largest score only where that is more than 2^8 times m's weight: sums and fp16's weights have room for it.  Lane by lane: a row's bits are its own.
        // Few queries, which memory bounds, follow it always: the largest weight then is 1, which is not rounded (380 keys: a tenth less error).
        const bool grown = (top - m) * scale2 > (NW == 1 ? 0.f : 8.f);
        if (__ballot(grown)) {
            const float alpha = grown ? __builtin_amdgcn_exp2f((m - top) * scale2) : 1.f;
            m = grown ? top : m;
            l *= alpha;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
        }
        float base = m == -INFINITY ? 0.f : -m * scale2;
        const bool large = __builtin_fabsf(base) > 0x1p24f;
        if (__ballot(large)) {  // base is off by more than a half: weights under it would leave fp16's range, then fp32's.  The maximum is taken from the scores first.
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] -= large ? m : 0.f;
            base = large ? 0.f : base;
        }
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kt][r] = __builtin_amdgcn_exp2f(fmaf(s[kt][r], scale2, base));
                l += s[kt][r];
            }
        bool taken_out = false;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            if (!see.all) {
                Finite<T> f;
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) f.look(vf[w][dt]);
                if (!f.all()) {
                    taken_out = true;
#pragma unroll
                    for (int w = 0; w < 2; ++w)
#pragma unroll
                        for (int dt = 0; dt < ND; ++dt) f.keep(vf[w][dt]);
                }
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const V8 pf = rounded<T>(s[kt], w);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) o[dt] = att_mfma(vf[w][dt], pf, o[dt]);
            }
            if (kt == 0) columns.template two<32>(Vt, vf);
        }
        if (taken_out)  // it reaches the queries that see it
            add_nonfinite<T, ND>(o, vb, ldv, j0, keys, a.dim, lane, [&](int at) { return at <= p + a.right && (at >= p - a.left || at < a.sinks); });
    }
    l = both_halves_sum(l);
    const bool valid = l32 < my_rows;
    if (t.slot >= 0) {
        const int64_t at = ((int64_t)t.slot * a.heads + h) * (NW * 32) + wave * 32 + l32;
        if (valid) {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    f32x4 x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = o[dt][4 * c + i];
                    *reinterpret_cast<f32x4 *>(part_o + at * DP + dt * 32 + 8 * c + 4 * half) = x;
                }
            if (half == 0) part_ml[at] = make_float2(m * scale2, l);
        }
        return;
    }
    if (valid && half == 0 && lse) lse[(int64_t)h * Tq + my_row] = l == 0.f ? -INFINITY : fmaf(m, scale2, __builtin_amdgcn_logf(l)) * LN2;
    store_columns<T, ND>(o, l == 0.f ? 0.f : 1.f / l, out + (int64_t)my_row * ldo + h * a.dim, valid, a.dim, lane);
}

// The parts of split rows: m the largest, l and O summed under it.  A wavefront has one row of one head; its lanes have the parts in turn for m and l, and for O the row's
// pieces of eight elements of every 8th part (of DP 32: 16th, 128: 4th), added up over the lanes at the end: the order is the same in every call.  4 us, latency of dependent loads;
// a block takes 8 rows, as 128 rows of a join in four wavefronts took 26 us more (8 sequences of 512 tokens, split).
constexpr int JOIN_ROWS = 8;  // of a block
template <class T, int DP>
__global__ __launch_bounds__(256) void join_kernel(const AttentionJoin *__restrict__ joins, int heads, int dim, int block_rows, const float *__restrict__ part_o,
                                                   const float2 *__restrict__ part_ml, T *__restrict__ out, int64_t ldo, float *__restrict__ lse, int64_t Tq)
{
    constexpr int CH = DP / 8, GROUPS = 64 / CH;
    const AttentionJoin jn = joins[blockIdx.x];
    const int h = blockIdx.y, lane = threadIdx.x & 63, c = lane % CH, group = lane / CH;
    for (int row = blockIdx.z * JOIN_ROWS + (threadIdx.x >> 6); row < min(jn.rows, (int)(blockIdx.z + 1) * JOIN_ROWS); row += 4) {
        auto at = [&](int s) { return ((int64_t)(jn.slot0 + s) * heads + h) * block_rows + row; };
        float m = -INFINITY;
        for (int s = lane; s < jn.slots; s += 64) m = __builtin_fmaxf(m, part_ml[at(s)].x);
#pragma unroll
        for (int i = 32; i; i >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, i));
        auto weight = [&](float2 ml) { return ml.x == -INFINITY && ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - (m == -INFINITY ? 0.f : m)); };
        float l = 0.f;
        for (int s = lane; s < jn.slots; s += 64) {
            const float2 ml = part_ml[at(s)];
            l = fmaf(weight(ml), ml.y, l);
        }
        l = wave_sum(l);
        f32x8 o = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int s = group; s < jn.slots; s += GROUPS) {
            const float2 ml = part_ml[at(s)];
            const f32x4 *p = reinterpret_cast<const f32x4 *>(part_o + at(s) * DP + c * 8);
            const f32x4 x = p[0], y = p[1];
            const float w = weight(ml);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[e] = fmaf(w, x[e], o[e]);
                o[4 + e] = fmaf(w, y[e], o[4 + e]);
            }
        }
#pragma unroll
        for (int i = CH; i < 64; i <<= 1)
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += __shfl_xor(o[e], i);
        if (group == 0 && c * 8 < dim) {
            Raw8<T> r;
            r.round(o * (l == 0.f ? 0.f : 1.f / l));
            r.store(out + (int64_t)(jn.row0 + row) * ldo + h * dim + c * 8, 8);
        }
        if (lane == 0 && lse) lse[(int64_t)h * Tq + jn.row0 + row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
    }
}

// ------------------------------------------------------------------ host
template <class F>
int with_type16(int dtype, F f)
{
    return dtype == LEANN_BF16 ? f((bf16_t *)nullptr) : f((f16_t *)nullptr);
}
template <class F>
int with_dim(int dim, F f)
{
    if (dim <= 32) return f(std::integral_constant<int, 32>());
    if (dim <= 64) return f(std::integral_constant<int, 64>());
    return f(std::integral_constant<int, 128>());
}

size_t att_up256(size_t v) { return (v + 255) & ~(size_t)255; }

// A forward block's table and tiles; the largest table with the largest tiles is 65 + 9 KB.
template <class T, int DP, int NW, bool BIAS>
int launch_attend(leann_ctx *ctx, const leann_attention_plan *p, const AttentionShape &a, const T *q, int64_t ldq, const T *k, int64_t ldk, const T *v, int64_t ldv,
                  const float *bias, T *out, int64_t ldo, float *lse, float *part_o, float2 *part_ml)
{
    const int smem = AttendCfg<DP, NW>::FIXED + (BIAS ? (2 * p->distance + 1 + 2 * ATT_EXT) * 4 : 0);
    hipLaunchKernelGGL((attend_kernel<T, DP, NW, BIAS>), dim3(p->n_items), dim3(NW * 64), smem, ctx->stream, p->items, p->tiles, a, q, ldq, k, ldk, v, ldv, bias,
                       p->bucket_of, out, ldo, lse, p->Tq, part_o, part_ml);
    if (p->n_joins)
        hipLaunchKernelGGL((join_kernel<T, DP>), dim3(p->n_joins, p->heads, (p->join_rows + JOIN_ROWS - 1) / JOIN_ROWS), dim3(256), 0, ctx->stream, p->joins, p->heads, p->dim, NW * 32, part_o, part_ml, out, ldo, lse,
                           p->Tq);
    return att_launched("leann_attention");
}

int make_plan(leann_ctx *ctx, const int32_t *q_rows, const int32_t *k_rows, const int32_t *first, int n, const AttentionRules &r, const int32_t *bucket_of,
              int distance, leann_attention_plan *p)
{
    std::vector<int32_t> zeros;
    if (!first) {
        zeros.assign(std::max(1, n), 0);
        first = zeros.data();
    }
    int64_t longest = 0, furthest = 1;
    for (int s = 0; s < n; ++s) {
        longest = std::max<int64_t>(longest, q_rows[s]);
        p->Tq += q_rows[s];
        p->Tk += k_rows[s];
        if (q_rows[s] && k_rows[s]) furthest = std::max<int64_t>({furthest, (int64_t)first[s] + q_rows[s] - 1, (int64_t)k_rows[s] - 1 - first[s]});
    }
    std::vector<int32_t> buckets;
    if (bucket_of) {  // no longer than the sequences
        p->distance = (int32_t)std::min<int64_t>(distance, furthest);
        buckets.assign(bucket_of + distance - p->distance, bucket_of + distance + p->distance + 1);
    }
    // 32 queries per block where no sequence has more: the other wavefronts would only load.  128 where they share the keys' tiles.
    p->query_waves = longest <= 32 ? 1 : 4;
    // Too many blocks are refused before there are tables of them: 2^30 queries of 1024 heads would have 69 GB.  The tables themselves may have a few more, see `order`.
    constexpr int64_t MOST_BLOCKS = (1 << 24) - 1;  // of 256 threads, of which a launch has fewer than 2^32
    auto refused = [&](int64_t blocks) {
        if (blocks <= MOST_BLOCKS) return LEANN_OK;
        leann_set_error("leann_attention_create: sequences of this number and length are not covered (more than 2^24 - 1 workgroups of 256 in a launch)");
        return LEANN_ESHAPE;
    };
    int64_t query_blocks = 0, key_blocks = 0;
    for (int s = 0; s < n; ++s) {
        query_blocks += ((int64_t)q_rows[s] + 127) / 128;
        key_blocks += ((int64_t)k_rows[s] + 127) / 128;
    }
    LEANN_TRY(refused(std::max(query_blocks * p->heads, key_blocks * p->kv_heads)));
    std::vector<AttentionTile> tiles;
    std::vector<int32_t> of;
    std::vector<AttentionJoin> joins;
    const int share = p->heads / p->kv_heads, cus = ctx->num_cus;
    att_make_tiles(r, n, q_rows, k_rows, first, false, share, p->query_waves * 32, 0, tiles, of, joins);
    // Keys are split where there are fewer than two blocks per compute unit.  Of few queries the parts make four blocks per unit, of four tiles at least; of 128 queries,
    // whose sums are a part's way through memory of 128 rows, one, of 16 tiles (8 sequences of 512 tokens, 12 heads: 42 us in parts of four, 19 whole; one of 2048, 8 heads of
    // 128 elements: 44 us in two parts, 51 whole).
    if ((int64_t)tiles.size() * p->heads < 2 * cus)
        if (const int split = p->query_waves == 1 ? att_split(tiles, p->heads, cus, 4, 4) : att_split(tiles, p->heads, cus, 1, 16)) {
            tiles.clear();
            att_make_tiles(r, n, q_rows, k_rows, first, false, share, p->query_waves * 32, split, tiles, of, joins);
        }
    for (const AttentionJoin &j : joins) {
        p->n_slots += j.slots;
        p->join_rows = std::max(p->join_rows, j.rows);
    }
    std::vector<char> image;
    auto put = [&](const auto &v) {
        const size_t at = att_up256(image.size()), bytes = v.size() * sizeof(v[0]);
        image.resize(at + bytes);
        if (bytes) memcpy(image.data() + at, v.data(), bytes);
        return at;
    };
    size_t most_blocks = joins.size();
    auto order = [&](const std::vector<AttentionTile> &t, const std::vector<int32_t> &t_of, int heads, int s, int threads, int32_t *count) {
        const std::vector<AttentionItem> items = att_order(t, t_of, heads, s);
        *count = (int32_t)items.size();
        most_blocks = std::max(most_blocks, items.size() * (threads / 256));
        return put(items);
    };
    const size_t tiles_at = put(tiles), items_at = order(tiles, of, p->heads, share, 256, &p->n_items), joins_at = put(joins);
    p->n_joins = (int32_t)joins.size();

    // The gradient's two sides, of all sequences or of those that are not taken whole.
    auto make_sides = [&](const std::vector<char> *taken, AttentionSides *sides, size_t (&at)[5]) {
        std::vector<AttentionTile> query_tiles, key_tiles;
        std::vector<int32_t> query_of, key_of;
        std::vector<AttentionJoin> key_joins, none;
        att_make_tiles(r, n, q_rows, k_rows, first, false, share, 128, 0, query_tiles, query_of, none, taken);
        // 64 keys per block where 128 would make fewer than two blocks per compute unit.
        att_make_tiles(r, n, q_rows, k_rows, first, true, share, 128, 0, key_tiles, key_of, key_joins, taken);
        if ((int64_t)key_tiles.size() * p->kv_heads < 2 * cus) {
            sides->key_waves = 2;
            key_tiles.clear();
            att_make_tiles(r, n, q_rows, k_rows, first, true, share, 64, 0, key_tiles, key_of, key_joins, taken);
        }
        // Keys that many queries see, as a sequence's first ones, have their queries split, so that no block has much more than half of a compute unit's share, of which it has
        // two (two documents with a window: 79 us, with parts of a unit's share 102).
        if (const int split = att_split(key_tiles, p->kv_heads, cus, 2, 8)) {
            key_tiles.clear();
            att_make_tiles(r, n, q_rows, k_rows, first, true, share, sides->key_waves * 32, split, key_tiles, key_of, key_joins, taken);
        }
        for (const AttentionJoin &j : key_joins) sides->n_slots += j.slots;
        sides->n_tiles = (int32_t)query_tiles.size();
        sides->n_joins = (int32_t)key_joins.size();
        most_blocks = std::max(most_blocks, key_joins.size());
        at[0] = put(query_tiles);
        at[1] = order(query_tiles, query_of, p->heads, share, 256, &sides->n_query_items);
        at[2] = put(key_tiles);
        at[3] = order(key_tiles, key_of, p->kv_heads, 1, 256, &sides->n_key_items);
        at[4] = put(key_joins);
    };
    size_t all_at[5], others_at[5], whole_at[2][2] = {};
    make_sides(nullptr, &p->all, all_at);
    std::vector<char> taken(n, 0);
    const bool sees_all = r.left >= (1 << 30) && r.right >= (1 << 30);
    int n_taken = 0;
    auto in_class = [&](int s) { return q_rows[s] > ATT_WHOLE / 2 || k_rows[s] > ATT_WHOLE / 2 ? 1 : 0; };
    // The tables of biases and their sums go by the distance that the plan's longest sequence has: beyond about 600 they leave a block of 8 wavefronts too little LDS.
    const bool fits[2] = {(p->dim <= 32 ? WholeCfg<32, 4>::bytes(p->distance, bucket_of, true) : WholeCfg<64, 4>::bytes(p->distance, bucket_of, true)) <= ATT_LDS,
                          (p->dim <= 32 ? WholeCfg<32, 8>::bytes(p->distance, bucket_of, true) : WholeCfg<64, 8>::bytes(p->distance, bucket_of, true)) <= ATT_LDS};
    for (int s = 0; s < n; ++s)
        n_taken += taken[s] = sees_all && share == 1 && p->dim <= 64 && q_rows[s] <= ATT_WHOLE && k_rows[s] <= ATT_WHOLE && fits[in_class(s)];
    if (n_taken) make_sides(&taken, &p->others, others_at);
    for (int c = 0; n_taken && c < 2; ++c) {
        std::vector<AttentionTile> whole;
        std::vector<int32_t> whole_of(1, 0);
        int64_t q0 = 0, k0 = 0;
        for (int s = 0; s < n; q0 += q_rows[s], k0 += k_rows[s], ++s) {
            if (!taken[s] || in_class(s) != c || (!q_rows[s] && !k_rows[s])) continue;
            AttentionTile t = {};
            t.row0 = (int32_t)k0;
            t.rows = k_rows[s];
            t.other0 = (int32_t)q0;
            t.others = q_rows[s];
            t.first = first[s];
            t.end = (q_rows[s] + 31) / 32;  // what the order goes by
            t.slot = -1;
            whole.push_back(t);
            whole_of.push_back((int32_t)whole.size());
        }
        p->whole[c].n_tiles = (int32_t)whole.size();
        whole_at[c][0] = put(whole);
        whole_at[c][1] = order(whole, whole_of, p->heads, 1, c ? 512 : 256, &p->whole[c].n_items);
    }
    LEANN_TRY(refused((int64_t)most_blocks));
    const size_t buckets_at = put(buckets);
    LEANN_TRY(ctx->reserve(p->mem, std::max<size_t>(image.size(), 1)));
    if (!image.empty()) LEANN_HIP(hipMemcpyAsync(p->mem.p, image.data(), image.size(), hipMemcpyHostToDevice, ctx->stream));
    LEANN_HIP(hipStreamSynchronize(ctx->stream));
    const char *base = (const char *)p->mem.p;
    auto set_sides = [&](AttentionSides *sides, const size_t (&at)[5]) {
        sides->query_tiles = (const AttentionTile *)(base + at[0]);
        sides->query_items = (const AttentionItem *)(base + at[1]);
        sides->key_tiles = (const AttentionTile *)(base + at[2]);
        sides->key_items = (const AttentionItem *)(base + at[3]);
        sides->joins = (const AttentionJoin *)(base + at[4]);
    };
    p->tiles = (const AttentionTile *)(base + tiles_at);
    p->items = (const AttentionItem *)(base + items_at);
    p->joins = (const AttentionJoin *)(base + joins_at);
    p->bucket_of = (const int32_t *)(base + buckets_at);
    set_sides(&p->all, all_at);
    if (n_taken) set_sides(&p->others, others_at);
    else p->others = p->all;
    for (int c = 0; c < 2; ++c) {
        p->whole[c].tiles = (const AttentionTile *)(base + whole_at[c][0]);
        p->whole[c].items = (const AttentionItem *)(base + whole_at[c][1]);
    }
    return LEANN_OK;
}

template <class T, int DP>
int allow_attend()
{
    for (const void *f : {(const void *)attend_kernel<T, DP, 1, false>, (const void *)attend_kernel<T, DP, 1, true>, (const void *)attend_kernel<T, DP, 4, false>,
                          (const void *)attend_kernel<T, DP, 4, true>})
        LEANN_HIP(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, std::max(AttendCfg<DP, 1>::FIXED, AttendCfg<DP, 4>::FIXED) + (2 * ATT_MOST_DISTANCE + 1 + 2 * ATT_EXT) * 4));
    return LEANN_OK;
}

}  // namespace

int att_launched(const char *call)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return LEANN_OK;
    leann_set_error("%s: launch failed: %s", call, hipGetErrorString(e));
    return LEANN_EDEVICE;
}

int att_check_call(const char *call, const leann_ctx *ctx, const leann_attention_plan *plan, int dtype, float scale, const float *bias_dev)
{
    if (!ctx || !plan || (dtype != LEANN_BF16 && dtype != LEANN_F16)) {
        leann_set_error("%s: null context or plan, or a type other than bf16 and f16", call);
        return LEANN_EINVAL;
    }
    if (plan->device != ctx->device) {
        leann_set_error("%s: the plan belongs to another device", call);
        return LEANN_EINVAL;
    }
    if (!(fabsf(scale) >= ATT_LEAST_SCALE && fabsf(scale) <= ATT_MOST_SCALE) || !bias_dev != !plan->buckets) {
        leann_set_error("%s: a scale whose magnitude is outside 2^-20 to 2^20, or a bias without buckets or buckets without a bias", call);
        return LEANN_EINVAL;
    }
    return LEANN_OK;
}

int att_check_rows(const char *call, const char *what, const void *p, int64_t ld, int64_t cols)
{
    if (!p || ((uintptr_t)p & 15)) {
        leann_set_error("%s: %s is null or not aligned to 16 bytes", call, what);
        return LEANN_EINVAL;
    }
    if (ld < cols || ld % 8 || ld > ATT_MOST_LD) {
        leann_set_error("%s: rows of %s are %lld elements apart, need a multiple of 8 from %lld to 2^22", call, what, (long long)ld, (long long)cols);
        return LEANN_ESHAPE;
    }
    return LEANN_OK;
}

int att_check_apart(const char *call, const AttentionMatrix &a, const AttentionMatrix &b)
{
    if (!att_overlap((uint64_t)a.p, a.ld, a.cols, a.rows, (uint64_t)b.p, b.ld, b.cols, b.rows, 2)) return LEANN_OK;
    leann_set_error("%s: %s overlaps %s", call, a.name, b.name);
    return LEANN_EINVAL;
}

AttentionShape att_shape(const leann_attention_plan *p, float scale)
{
    return AttentionShape{p->heads, p->heads / p->kv_heads, p->dim, p->left, p->right, p->sinks, p->distance, scale};
}

int attention_init_device()
{
    LEANN_TRY((allow_attend<bf16_t, 32>()));
    LEANN_TRY((allow_attend<bf16_t, 64>()));
    LEANN_TRY((allow_attend<bf16_t, 128>()));
    LEANN_TRY((allow_attend<f16_t, 32>()));
    LEANN_TRY((allow_attend<f16_t, 64>()));
    return allow_attend<f16_t, 128>();
}

extern "C" {

int leann_position_buckets(int32_t buckets, int32_t distance, int both, int32_t *bucket_of_host)
{
    static const char *call = "leann_position_buckets";
    const int half = both ? buckets / 2 : buckets;
    if (!bucket_of_host || buckets < 2 || (both && buckets % 2) || half < 2 || half > 2048 || distance > ATT_MOST_DISTANCE || distance <= half / 2) {
        leann_set_error("%s: null output, fewer than two buckets of a direction or more than 2048, an odd number for two, or a distance that is not above half of a direction's or above %d", call,
                        ATT_MOST_DISTANCE);
        return LEANN_EINVAL;
    }
    att_position_buckets(buckets, distance, both != 0, bucket_of_host);
    return LEANN_OK;
}

void leann_attention_free(leann_attention_plan *p)
{
    if (!p) return;
    (void)hipSetDevice(p->device);
    p->mem.release();
    delete p;
}

int leann_attention_create(leann_ctx *ctx, const int32_t *q_rows_host, const int32_t *k_rows_host, const int32_t *first_host, int32_t n_sequences,
                           const leann_attention_desc *desc, leann_attention_plan **out)
{
    static const char *call = "leann_attention_create";
    if (!ctx || !out || !desc || n_sequences < 0 || (n_sequences > 0 && !q_rows_host)) {
        leann_set_error("%s: null argument or negative number of sequences", call);
        return LEANN_EINVAL;
    }
    const leann_attention_desc &d = *desc;
    if (d.left < -1 || d.right < -1 || d.sinks < 0) {
        leann_set_error("%s: a window below -1 (no limit) or a negative number of first keys", call);
        return LEANN_EINVAL;
    }
    if (d.heads < 1 || d.heads > 1024 || d.kv_heads < 1 || d.heads % d.kv_heads || d.dim < 8 || d.dim > 128 || d.dim % 8) {
        leann_set_error("%s: %d heads (%d of keys) of size %d are not covered (at most 1024, a multiple of those of keys; a multiple of 8, at most 128)", call, d.heads,
                        d.kv_heads, d.dim);
        return LEANN_ESHAPE;
    }
    if (!d.bucket_of_host != !d.buckets || !d.bucket_of_host != !d.distance || d.buckets < 0 || d.distance < 0) {
        leann_set_error("%s: buckets, their distance and their table have to be given together", call);
        return LEANN_EINVAL;
    }
    if (d.buckets > 4096 || d.distance > ATT_MOST_DISTANCE) {
        leann_set_error("%s: %d buckets to a distance of %d are not covered (at most 4096 and %d)", call, d.buckets, d.distance, ATT_MOST_DISTANCE);
        return LEANN_ESHAPE;
    }
    for (int i = 0; d.bucket_of_host && i <= 2 * d.distance; ++i)
        if (d.bucket_of_host[i] < 0 || d.bucket_of_host[i] >= d.buckets) {
            leann_set_error("%s: relative position %d has bucket %d of %d", call, i - d.distance, d.bucket_of_host[i], d.buckets);
            return LEANN_EINVAL;
        }
    const int32_t *k_rows = k_rows_host ? k_rows_host : q_rows_host;
    int64_t Tq = 0, Tk = 0;
    constexpr int64_t MOST = (int64_t)1 << 30;  // positions and windows, so that their sums are 32-bit numbers
    for (int s = 0; s < n_sequences; ++s) {
        const int64_t f = first_host ? first_host[s] : 0;
        if (q_rows_host[s] < 0 || k_rows[s] < 0 || f < 0) {
            leann_set_error("%s: sequence %d has a negative number of queries or keys or a negative first position", call, s);
            return LEANN_EINVAL;
        }
        if (f + q_rows_host[s] >= MOST || k_rows[s] >= MOST) {
            leann_set_error("%s: sequence %d has positions that are not covered (below 2^30)", call, s);
            return LEANN_ESHAPE;
        }
        Tq += q_rows_host[s];
        Tk += k_rows[s];
    }
    if (Tq > 0x7fffffffll - 256 || Tk > 0x7fffffffll - 256) {
        leann_set_error("%s: %lld and %lld rows are not covered (below 2^31 - 256)", call, (long long)Tq, (long long)Tk);
        return LEANN_ESHAPE;
    }
    LEANN_HIP(hipSetDevice(ctx->device));
    leann_attention_plan *p = nullptr;
    int rc;
    try {
        p = new leann_attention_plan();
        p->device = ctx->device;
        p->heads = d.heads;
        p->kv_heads = d.kv_heads;
        p->dim = d.dim;
        p->buckets = d.buckets;
        p->left = d.left < 0 ? (int32_t)MOST : std::min<int32_t>(d.left, (int32_t)MOST);
        p->right = d.right < 0 ? (int32_t)MOST : std::min<int32_t>(d.right, (int32_t)MOST);
        p->sinks = std::min<int32_t>(d.sinks, (int32_t)MOST);
        rc = make_plan(ctx, q_rows_host, k_rows, first_host, n_sequences, AttentionRules{p->left, p->right, p->sinks}, d.bucket_of_host, d.distance, p);
    } catch (const std::exception &) {
        leann_set_error("%s: no host memory", call);
        rc = LEANN_ENOMEM;
    }
    if (rc != LEANN_OK) {
        leann_attention_free(p);
        return rc;
    }
    *out = p;
    return LEANN_OK;
}

int leann_attention(leann_ctx *ctx, const leann_attention_plan *plan, const void *q_dev, int64_t ldq, const void *k_dev, int64_t ldk, const void *v_dev, int64_t ldv,
                    int dtype, float scale, const float *bias_dev, void *out_dev, int64_t ldo, float *lse_dev)
{
    static const char *call = "leann_attention";
    LEANN_TRY(att_check_call(call, ctx, plan, dtype, scale, bias_dev));
    if (plan->Tq == 0) return LEANN_OK;
    const int64_t nq = (int64_t)plan->heads * plan->dim, nk = (int64_t)plan->kv_heads * plan->dim;
    LEANN_TRY(att_check_rows(call, "q", q_dev, ldq, nq));
    LEANN_TRY(att_check_rows(call, "out", out_dev, ldo, nq));
    if (plan->Tk > 0) {
        LEANN_TRY(att_check_rows(call, "k", k_dev, ldk, nk));
        LEANN_TRY(att_check_rows(call, "v", v_dev, ldv, nk));
    }
    const AttentionMatrix o = {"out", out_dev, ldo, nq, plan->Tq};
    LEANN_TRY(att_check_apart(call, o, AttentionMatrix{"q", q_dev, ldq, nq, plan->Tq}));
    LEANN_TRY(att_check_apart(call, o, AttentionMatrix{"k", k_dev, ldk, nk, plan->Tk}));
    LEANN_TRY(att_check_apart(call, o, AttentionMatrix{"v", v_dev, ldv, nk, plan->Tk}));
    LEANN_HIP(hipSetDevice(ctx->device));
    const AttentionShape a = att_shape(plan, scale);
    std::unique_lock<std::mutex> turn(ctx->op_work_mutex, std::defer_lock);
    return with_dim(plan->dim, [&](auto dp) {
        constexpr int DP = decltype(dp)::value;
        float *part_o = nullptr;
        float2 *part_ml = nullptr;
        if (plan->n_slots) {
            const size_t rows = (size_t)plan->n_slots * plan->heads * plan->query_waves * 32;
            turn.lock();
            LEANN_TRY(ctx->reserve(ctx->op_work, rows * (DP * sizeof(float) + sizeof(float2))));
            part_o = (float *)ctx->op_work.p;
            part_ml = (float2 *)(part_o + rows * DP);
        }
        return with_type16(dtype, [&](auto *type) {
            typedef std::remove_pointer_t<decltype(type)> T;
            auto go = [&](auto waves, auto with_bias) {
                return launch_attend<T, DP, decltype(waves)::value, decltype(with_bias)::value>(ctx, plan, a, (const T *)q_dev, ldq, (const T *)k_dev, ldk, (const T *)v_dev,
                                                                                               ldv, bias_dev, (T *)out_dev, ldo, lse_dev, part_o, part_ml);
            };
            using One = std::integral_constant<int, 1>;
            using Four = std::integral_constant<int, 4>;
            if (plan->query_waves == 1) return bias_dev ? go(One(), std::true_type()) : go(One(), std::false_type());
            return bias_dev ? go(Four(), std::true_type()) : go(Four(), std::false_type());
        });
    });
}

}  // extern "C"
