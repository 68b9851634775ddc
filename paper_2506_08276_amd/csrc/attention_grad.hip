// The gradient of attention over ragged sequences: of queries, keys, values and of the bias (gfx950).
#include <math.h>

#include "attention.h"
#include "wave.h"

namespace {

// With P_ij = exp(s_ij - lse_i), delta_i = dO_i . O_i and dS_ij = P_ij (dO_i . v_j - delta_i):
//   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij dO_i,  dbias[b][h] = sum of dS_ij over the pairs in bucket b.
// Two kernels, each with sums of its own rows in registers: one for queries (with delta and the bias), one for keys.  Scores and dO V^T are computed in both, seven products
// instead of five; in exchange nothing is added up through memory, in whichever order blocks come.  delta takes O as it was stored, rounded: an error of half a step of
// each term, no more than dO's own.
// P and dS enter products rounded to the inputs' type.  In fp16 they would leave its range at either end (P = 1 / 4096 with gradients of 1e-4 is below its normal
// numbers, gradients of 10 may be above its largest): P goes in as 2^15 P, dS likewise times a power of two that a lane lowers for its own row or key, with what it has
// summed so far, when a value would pass 2^15.
constexpr int GRAD_WAVES = 4;  // 128 own rows per block

template <class T>
constexpr float shift_of = 0.f;
template <>
constexpr float shift_of<f16_t> = 15.f;

// LDS: tiles, then what the kernels say.  Two blocks fit on a CU up to heads of 64.
template <int DP>
struct GradCfg {
    static constexpr int TILE = ATT_STEP * DP;
    static constexpr int QUERY_STAGES = DP == 128 ? 2 : 3, KEY_STAGES = DP == 128 ? 2 : 4;
    static constexpr int QUERY_TILES = QUERY_STAGES * 2 * TILE * 2, KEY_TILES = KEY_STAGES * 2 * TILE * 2;  // bytes
    static constexpr int STATS = ATT_STEP * (int)sizeof(float2);                                             // per stage
};

// fp16: lowers `factor` and scales `sums` where a value of this step would pass 2^15.
template <int ND, int NV>
__device__ inline void stay_in_range(f32x16 (&ds)[NV], f32x16 (&sums)[ND], float &factor)
{
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) most = __builtin_fmaxf(most, __builtin_fabsf(ds[i][r]));
    most = both_halves_max(most);
    if (__ballot(most * factor > 0x1p15f)) {
        const uint32_t e = __float_as_uint(most) >> 23;  // 2^(e - 127) <= most
        if (most * factor > 0x1p15f && e < 255) {
            const float lower = __uint_as_float((141 + 127 - e) << 23), by = lower / factor;  // 2^(14 - (e - 127))
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) sums[i][r] *= by;
            factor = lower;
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[i][r] *= factor;
}

// dS of a sequence's only key is 0, not what the roundings of dO V^T and delta leave of it: a factor of its sums, so that infinities and NaN stay.
__device__ inline float unless_only(int keys) { return keys == 1 ? 0.f : 1.f; }

// P is 0 for rows that see nothing, and for those whose log-sum is so large that P is its rounding's: three of 2^-24 of it, of which each makes 0.18 of the exponent at 2^21, where
// 2^15 P still is within fp16's range; under a row of biases of -1e9 P would be 2^-64 to 2^64.
__device__ inline float lse_in_log2(float lse)
{
    return __builtin_fabsf(lse) >= 0x1p21f ? INFINITY : lse * LOG2E;
}

// Sums of dS along its diagonals, by relative position, without leaving the registers: a register is one row of the tile, a lane one column of it.  Row n + 16 c (and 4 more in the
// upper half of the lanes) moves by n lanes within each 16 as it is added, so that a diagonal's elements meet in one lane: what stays within the 16 lanes is added to
// a[c], what would leave them comes in again at the other end and is added to a[c + 1], 16 diagonals further.  Two additions per register.  (Rows written to LDS and
// read along the diagonals took 110 us of the training batch's gradient, atomic additions in LDS 1100.)
template <int N>
__device__ inline void add_moved(float &stays, float &leaves, float x)
{
    if constexpr (N == 0) {
        stays += x;
    } else {
        stays += __uint_as_float(dpp_mov<0x100 + N>(__float_as_uint(x)));        // lane i has lane i + N's, or 0
        leaves += __uint_as_float(dpp_mov<0x110 + 16 - N>(__float_as_uint(x)));  // lane i has lane i + N - 16's, or 0
    }
}
template <int R, int NA, int NV>
__device__ inline void add_rows(float (&a)[NA], const f32x16 (&d)[NV])
{
    if constexpr (R < NV * 16) {
        constexpr int row = R / 16 * 32 + acc_row(R % 16);
        add_moved<row % 16>(a[row / 16], a[row / 16 + 1], d[R / 16][R % 16]);
        add_rows<R + 1>(a, d);
    }
}
// In p[0] the even 16 lanes of a pair have their own, the odd ones the even ones'; in p[1] the other way round.
__device__ inline float2 both_rows(float v)
{
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return make_float2(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// dS^T with a query per lane and 64 keys in registers; sums[0] is relative position 0 within the tile.  Lane 16 b + i (of either half) holds in a[c] position 16 (c - b) - i + 4 half.
__device__ inline void add_diagonals(const f32x16 (&d)[2], float *sums, int lane)
{
    float a[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
    add_rows<0>(a, d);
    const bool odd = lane & 16;
    const float2 one = both_rows(a[1]), three = both_rows(a[3]);
    a[0] += odd ? 0.f : one.y;
    a[2] += odd ? one.x : three.y;
    a[4] += odd ? three.x : 0.f;
    float *at = sums - (lane & 15) - (lane & 16) + 4 * (lane >> 5);
    at[0] += a[0];
    at[32] += a[2];
    at[64] += a[4];
}

// A block's sums by relative position, its wavefronts' [NW][2][room] in order; the ends have what lies beyond, `behind` and `ahead` what a lane has added to none of them.  far:
// LDS that is free behind the first barrier.
template <int NW>
__device__ inline void sums_by_position(const float *sums, int room, int distance, float behind, float ahead, float *far, float factor, float *to)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, positions = 2 * distance + 1, entries = bias_entries(distance);
    const float *mine = sums + 2 * wave * room, *other = mine + room;
    __syncthreads();
    for (int e = lane; e < ATT_EXT; e += 64) {
        behind += mine[e] + other[e];
        ahead += mine[entries - 1 - e] + other[entries - 1 - e];
    }
    behind = wave_sum(behind);
    ahead = wave_sum(ahead);
    if (lane == 0) far[wave * 2] = behind, far[wave * 2 + 1] = ahead;
    __syncthreads();
    for (int i = threadIdx.x; i < positions; i += NW * 64) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            sum += sums[2 * w * room + i + ATT_EXT] + sums[(2 * w + 1) * room + i + ATT_EXT];
            if (i == 0) sum += far[w * 2];
            if (i == positions - 1) sum += far[w * 2 + 1];
        }
        to[i] = sum * factor;
    }
}

// A block takes 128 queries of one head through their keys, as the forward pass does.  S^T and dP^T = V dO^T have a query per lane; dS^T, rounded, is the other operand of
// dQ^T = K^T dS^T.  It leaves what the other kernel needs of each query: the log-sum in units of log 2 and delta, both negative.
// The bias's gradient is summed by relative position, each wavefront into an array of its own in LDS, so that the order of the additions is the program's.  Tiles
// behind `distance` add to one place, in a register.
// Bound by the latency of its chains with two wavefronts per SIMD (200 registers): two documents of 3001 and more tokens, window 256, 12 heads of 64: 56 us, vector units 35 %,
// matrix cores 19 % busy.  64 queries per block, with two wavefronts at each 32, took 57 to 67.
template <class T, int DP, bool BIAS>
__global__ __launch_bounds__(GRAD_WAVES * 64, DP == 128 ? 1 : 2) void query_grad_kernel(
    const AttentionItem *__restrict__ items, const AttentionTile *__restrict__ tiles, AttentionShape a, const T *__restrict__ dout, int64_t ldd, const T *__restrict__ q,
    int64_t ldq, const T *__restrict__ k, int64_t ldk, const T *__restrict__ v, int64_t ldv, const T *__restrict__ o, int64_t ldo, const float *__restrict__ lse, int64_t Tq,
    const float *__restrict__ bias, const int32_t *__restrict__ bucket_of, T *__restrict__ dq, int64_t lddq, float2 *__restrict__ stats, float *__restrict__ by_position)
{
    typedef typename Half8<T>::type V8;
    typedef GradCfg<DP> Cfg;
    typedef TileRequests<T, DP, GRAD_WAVES> Requests;
    constexpr int NT = GRAD_WAVES * 64, STAGES = Cfg::QUERY_STAGES, TILE = Cfg::TILE, ND = DP / 32, NS = DP / 16;
    constexpr bool F16 = shift_of<T> != 0.f;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    T *Ks = reinterpret_cast<T *>(smem), *Vs = Ks + STAGES * TILE;
    float *table = reinterpret_cast<float *>(smem + Cfg::QUERY_TILES);
    const int entries = bias_entries(a.distance), room = (entries + 3) & ~3;
    float *sums = table + room;  // [4 wavefronts][2 halves][room]

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
    const int my_rows = min(32, t.rows - wave * 32), p0 = t.at + wave * 32;
    const int64_t my_row = t.row0 + wave * 32 + l32;
    const bool valid = l32 < my_rows;
    V8 qf[NS], gf[NS], of[NS];
    load_rows<T, DP>(q + (int64_t)(t.row0 + wave * 32) * ldq + h * a.dim, ldq, my_rows, a.dim, lane, qf);
    load_rows<T, DP>(dout + (int64_t)(t.row0 + wave * 32) * ldd + h * a.dim, ldd, my_rows, a.dim, lane, gf);
    load_rows<T, DP>(o + (int64_t)(t.row0 + wave * 32) * ldo + h * a.dim, ldo, my_rows, a.dim, lane, of);
    const float my_lse = valid ? lse_in_log2(lse[(int64_t)h * Tq + my_row]) - shift_of<T> : INFINITY;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (t.begin + i < t.end) request(t.begin + i, i);
    if (BIAS) {
        make_bias(table, bias, bucket_of, a, h);
        if (by_position)
            for (int i = tid; i < 2 * GRAD_WAVES * room; i += NT) sums[i] = 0.f;
    }
    float my_delta = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) my_delta = fmaf((float)gf[s][i], (float)of[s][i], my_delta);
    my_delta = both_halves_sum(my_delta);
    if (valid && half == 0) stats[(int64_t)h * Tq + my_row] = make_float2(-my_lse, -my_delta);

    f32x16 acc[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[dt][r] = 0.f;
    f32x16 minus_delta;  // what the products dO V^T are added to
#pragma unroll
    for (int r = 0; r < 16; ++r) minus_delta[r] = -my_delta;
    float factor = 1.f, behind = 0.f, ahead = 0.f;
    bool hurt = false;  // sees a key that is not finite
    arrived(qf);
    arrived(gf);
    take_sign(qf, a.scale);
    const float scale2 = __builtin_fabsf(a.scale) * LOG2E;
    const int p = p0 + l32;

    Columns<T, DP> columns;
    columns.init(lane);
    int stage = 0;
    for (int u = t.begin; u < t.end; ++u) {
        const int j0 = key_of(u);
        const T *Kt = Ks + stage * TILE, *Vt = Vs + stage * TILE;
        if (STAGES > 2 && u + 1 < t.end) wait_for_requests<2 * Requests::N>();
        else wait_for_requests<0>();
        block_barrier();  // this tile is there, and the stage of the last one has been read
        if (u + STAGES - 1 < t.end) request(u + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
        stage = stage == STAGES - 1 ? 0 : stage + 1;
        const int keys = min(ATT_STEP, t.others - j0);
        const Sight see = sight(a, p0, my_rows, j0, keys);
        if (see.none) continue;

        f32x16 s[2], d[2];
        const int j = j0 + 4 * half;
        const int least = j0 - (p0 + 31), most = j0 + ATT_STEP - 1 - p0;  // relative positions
        const bool near = most > -a.distance && least < a.distance;
        float c = -my_lse;
        if (BIAS && near) {
            const int at = one_register(Cfg::QUERY_TILES / 4 + j - p + a.distance + ATT_EXT);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = reinterpret_cast<const float *>(smem)[at + kt * 32 + acc_row(r)];
        } else {
            if (BIAS) c = fmaf(table[most <= -a.distance ? 0 : entries - 1], scale2, c);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = 0.f;
        }
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            d[kt] = minus_delta;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                s[kt] = att_mfma(row_operand<T, DP>(Kt, kt * 32, i, lane), qf[i], s[kt]);
                d[kt] = att_mfma(row_operand<T, DP>(Vt, kt * 32, i, lane), gf[i], d[kt]);
            }
        }
        V8 kf[2][ND];  // of the first 32 keys
        columns.template two<0>(Kt, kf);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) d[kt][r] *= __builtin_amdgcn_exp2f(fmaf(s[kt][r], scale2, c));
        // What is hidden is a choice, not a product.  So are keys behind the last one: their rows are zeros, but their weight exp(0 - lse) has no bound, is infinite from a log-sum of
        // -88 (fp16: -78) on, and would long before take fp16's range from the others.
        const Edges e = edges(a, p0, my_rows, j0, keys);
        if (e.behind) {
            const int last = min(t.others - 1, p + a.right) - j;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) d[kt][r] = kt * 32 + acc_row(r) > last ? 0.f : d[kt][r];
        }
        if (e.before) {
            const int from = p - a.left - j, sinks = a.sinks - j;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = kt * 32 + acc_row(r);
                    d[kt][r] = ((key < from) & (key >= sinks)) ? 0.f : d[kt][r];
                }
        }
        if (BIAS && by_position) {
            if (my_rows < 32) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) d[kt][r] = valid ? d[kt][r] : 0.f;
            }
            if (near) {
                add_diagonals(d, sums + (2 * wave + half) * room + (j0 - p0 + a.distance + ATT_EXT), lane);
            } else {
                float sum = 0.f;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum += d[kt][r];
                if (most <= -a.distance) behind += sum;
                else ahead += sum;
            }
        }
        if (F16) stay_in_range(d, acc, factor);
        bool taken_out = false;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            if (!see.all) {
                Finite<T> f;
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) f.look(kf[w][dt]);
                if (!f.all()) {
                    taken_out = true;
#pragma unroll
                    for (int w = 0; w < 2; ++w)
#pragma unroll
                        for (int dt = 0; dt < ND; ++dt) f.keep(kf[w][dt]);
                }
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const V8 df = rounded<T>(d[kt], w);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) acc[dt] = att_mfma(kf[w][dt], df, acc[dt]);
            }
            if (kt == 0) columns.template two<32>(Kt, kf);
        }
        if (taken_out)
            for_nonfinite_rows<T>(kb, ldk, j0, keys, a.dim, lane, [&](int at, const T *) { hurt |= at <= p + a.right && (at >= p - a.left || at < a.sinks); });
    }
    if (hurt) factor = __builtin_nanf("");
    const float some = unless_only(t.others) * (F16 ? 0x1p-15f : 1.f);
    store_columns<T, ND>(acc, a.scale / factor * some, dq + my_row * lddq + h * a.dim, valid, a.dim, lane);

    if (BIAS && by_position) {
        if (t.begin == t.end) block_barrier();  // the sums are cleared
        sums_by_position<GRAD_WAVES>(sums, room, a.distance, behind, ahead, reinterpret_cast<float *>(smem), some,
                                     by_position + ((int64_t)item.tile * a.heads + h) * (2 * a.distance + 1));
    }
}

// A block takes 32 KW keys of one key head through the queries that see them, of every head that shares it: S = Q K^T and dP = dO V^T have a key per lane; P and dS, rounded, are the
// other operands of dV^T = dO^T P and dK^T = Q^T dS.  K and V stay in registers; Q, dO and the queries' numbers come from memory to LDS, STAGES - 1 tiles ahead.
// KW = 4: a wavefront has 32 keys.  KW = 2, for few keys: two wavefronts share them, each with 32 of a step's 64 queries, and their sums meet in LDS at the end.
// Bound as the other kernel: the same documents 79 us with KW = 2, 520 blocks; 95 with KW = 4 and splits to match (25 to 31 steps in a row instead of twice as many half as dear).
template <class T, int DP, int KW, bool BIAS>
__global__ __launch_bounds__(GRAD_WAVES * 64, DP == 128 ? 1 : 2) void key_grad_kernel(
    const AttentionItem *__restrict__ items, const AttentionTile *__restrict__ tiles, AttentionShape a, const T *__restrict__ dout, int64_t ldd, const T *__restrict__ q,
    int64_t ldq, const T *__restrict__ k, int64_t ldk, const T *__restrict__ v, int64_t ldv, const float2 *__restrict__ stats, int64_t Tq, const float *__restrict__ bias,
    const int32_t *__restrict__ bucket_of, T *__restrict__ dk, int64_t lddk, T *__restrict__ dv, int64_t lddv, float *__restrict__ parts)
{
    typedef typename Half8<T>::type V8;
    typedef GradCfg<DP> Cfg;
    typedef TileRequests<T, DP, GRAD_WAVES> Requests;
    constexpr int STAGES = Cfg::KEY_STAGES, TILE = Cfg::TILE, ND = DP / 32, NS = DP / 16;
    constexpr bool F16 = shift_of<T> != 0.f;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    T *Qs = reinterpret_cast<T *>(smem), *Gs = Qs + STAGES * TILE;
    float *numbers = reinterpret_cast<float *>(smem + Cfg::KEY_TILES);  // [stage][64][2]
    float *table = reinterpret_cast<float *>(smem + Cfg::KEY_TILES + STAGES * Cfg::STATS);

    const AttentionItem item = items[blockIdx.x];
    if (item.tile < 0) return;
    const AttentionTile t = tiles[item.tile];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int g = item.head;
    const int own = wave % KW * 32, share = wave / KW;  // first of the wavefront's keys in the block, which of the sharing wavefronts it is
    const int my_rows = min(32, t.rows - own), jw = t.at + own, j = jw + l32;
    const int64_t my_row = t.row0 + own + l32;
    const bool valid = l32 < my_rows;
    V8 kf[NS], vf[NS];
    load_rows<T, DP>(k + (int64_t)(t.row0 + own) * ldk + g * a.dim, ldk, my_rows, a.dim, lane, kf);
    load_rows<T, DP>(v + (int64_t)(t.row0 + own) * ldv + g * a.dim, ldv, my_rows, a.dim, lane, vf);

    Requests qr, gr;
    qr.init(ldq, a.dim, wave, lane);
    gr.init(ldd, a.dim, wave, lane);
    // tile by tile, head by head
    struct At {
        int h, tile;
    };
    const int total = t.end - t.begin, last_tile = t.first_tile + t.per_head - 1;
    auto behind = [&](At at) { return at.tile == last_tile ? At{at.h + 1, t.first_tile} : At{at.h, at.tile + 1}; };
    auto request = [&](At at, int stage) {
        const int i0 = at.tile * ATT_STEP;
        if (wave == 0) {
            const float2 *from = stats + (int64_t)at.h * Tq + t.other0 + i0;
            // whole pieces of two queries; what is read behind the last one is masked
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float2 *>(from), 0, ((min(t.others - i0, ATT_STEP) + 1) & ~1) * 8, 0x00020000);
            if (lane < 32) lds_request(rsrc, lane * 16, numbers + stage * 128);
        }
        qr.request(q + (int64_t)(t.other0 + i0) * ldq + at.h * a.dim, ldq, t.others - i0, a.dim, Qs + stage * TILE, wave);
        gr.request(dout + (int64_t)(t.other0 + i0) * ldd + at.h * a.dim, ldd, t.others - i0, a.dim, Gs + stage * TILE, wave);
    };
    At now = {g * a.share, t.first_tile};
    if (total) now = At{now.h + t.begin / t.per_head, now.tile + t.begin % t.per_head};
    At next = now;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (i < total) {
            request(next, i);
            next = behind(next);
        }

    f32x16 dk_acc[ND], dv_acc[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk_acc[dt][r] = dv_acc[dt][r] = 0.f;
    float factor = 1.f;
    bool hurt = false;
    arrived(kf);
    arrived(vf);
    take_sign(kf, a.scale);
    const float scale2 = __builtin_fabsf(a.scale) * LOG2E;
    Columns<T, DP> columns;
    columns.init(lane);
    int stage = 0, of_table = -1;
    for (int n = 0; n < total; ++n, now = behind(now)) {
        const int h = now.h, i0 = now.tile * ATT_STEP;
        const T *Qt = Qs + stage * TILE, *Gt = Gs + stage * TILE;
        const float *nt = numbers + stage * 128;
        if (BIAS && h != of_table) {
            if (n) block_barrier();  // the last head's table has been read
            make_bias(table, bias, bucket_of, a, h);
            of_table = h;
        }
        if (STAGES > 3 && n + 2 < total) wait_for_requests<4 * Requests::N>();
        else if (STAGES > 2 && n + 1 < total) wait_for_requests<2 * Requests::N>();
        else wait_for_requests<0>();
        block_barrier();  // this tile is there, and the stage of the last one has been read
        if (n + STAGES - 1 < total) {
            request(next, stage == 0 ? STAGES - 1 : stage - 1);
            next = behind(next);
        }
        stage = stage == STAGES - 1 ? 0 : stage + 1;
        const int rows = min(ATT_STEP, t.others - i0);
        const Sight see = sight(a, t.first + i0, rows, jw, my_rows);
        if (see.none) continue;

        bool taken_out = false;
#pragma unroll
        for (int turn = 0; turn < KW / 2; ++turn) {
            const int qs = KW == 4 ? turn : share;  // which 32 of the 64 queries
            f32x16 s[1], d[1];
            // register r is query i0 + 32 qs + 4 half + acc_row(r); queries behind the last one have rows of zeros and any numbers
            const int from = i0 + qs * 32 + 4 * half, p = t.first + from;
            float ls[16];
#pragma unroll
            for (int c = 0; c < 8; ++c) {  // -lse, and -delta, to which the products dO V^T are added
                const f32x4 x = *reinterpret_cast<const f32x4 *>(nt + 2 * (qs * 32 + 4 * half + 8 * (c >> 1) + 2 * (c & 1)));
                ls[2 * c] = x[0], d[0][2 * c] = x[1], ls[2 * c + 1] = x[2], d[0][2 * c + 1] = x[3];
            }
            const int pw = t.first + i0 + qs * 32, least = jw - (pw + 31), most = jw + 31 - pw;
            const bool near = most > -a.distance && least < a.distance;
            float c = 0.f;
            if (BIAS && near) {
                const int at = one_register((Cfg::KEY_TILES + STAGES * Cfg::STATS) / 4 + j - p - 27 + a.distance + ATT_EXT);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[0][r] = reinterpret_cast<const float *>(smem)[at + 27 - acc_row(r)];
            } else {
                if (BIAS) c = table[most <= -a.distance ? 0 : bias_entries(a.distance) - 1] * scale2;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[0][r] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                s[0] = att_mfma(row_operand<T, DP>(Qt, qs * 32, i, lane), kf[i], s[0]);
                d[0] = att_mfma(row_operand<T, DP>(Gt, qs * 32, i, lane), vf[i], d[0]);
            }
            V8 qc[ND], gc[ND];  // of the first 16 queries
            const T *Gh = Gt + qs * 32 * DP, *Qh = Qt + qs * 32 * DP;
            columns.template both<0>(Gh, Qh, gc, qc);
            if (BIAS && !near) {
#pragma unroll
                for (int r = 0; r < 16; ++r) ls[r] += c;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], scale2, ls[r]));
                d[0][r] *= s[0][r];
            }
            if (!see.all) {
                const int count = t.others - from, first = j - a.right - p, last = j < a.sinks ? ATT_STEP : j + a.left - p;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int c = acc_row(r);
                    const bool hidden = (c >= count) | (c < first) | (c > last);
                    s[0][r] = hidden ? 0.f : s[0][r];
                    d[0][r] = hidden ? 0.f : d[0][r];
                }
            } else if (rows < ATT_STEP) {
                const int count = t.others - from;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[0][r] = acc_row(r) >= count ? 0.f : s[0][r];
                    d[0][r] = acc_row(r) >= count ? 0.f : d[0][r];
                }
            }
            if (F16) stay_in_range(d, dk_acc, factor);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                if (!see.all) {
                    Finite<T> f;
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) {
                        f.look(gc[dt]);
                        f.look(qc[dt]);
                    }
                    if (!f.all()) {
                        taken_out = true;
#pragma unroll
                        for (int dt = 0; dt < ND; ++dt) {
                            f.keep(gc[dt]);
                            f.keep(qc[dt]);
                        }
                    }
                }
                const V8 pf = rounded<T>(s[0], w), df = rounded<T>(d[0], w);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    dv_acc[dt] = att_mfma(gc[dt], pf, dv_acc[dt]);
                    dk_acc[dt] = att_mfma(qc[dt], df, dk_acc[dt]);
                }
                if (w == 0) columns.template both<16>(Gh, Qh, gc, qc);
            }
        }
        if (taken_out) {
            auto seen = [&](int i) { return j <= t.first + i + a.right && (j >= t.first + i - a.left || j < a.sinks); };
            for_nonfinite_rows<T>(q + (int64_t)t.other0 * ldq + h * a.dim, ldq, i0, rows, a.dim, lane, [&](int i, const T *) { hurt |= seen(i); });
            add_nonfinite<T, ND>(dv_acc, dout + (int64_t)t.other0 * ldd + h * a.dim, ldd, i0, rows, a.dim, lane, seen);
        }
    }
    if (hurt) factor = __builtin_nanf("");
    float dk_factor = a.scale * (jw == 0 ? unless_only(my_rows) : 1.f) / factor * (F16 ? 0x1p-15f : 1.f), dv_factor = F16 ? 0x1p-15f : 1.f;
    if constexpr (KW == 2) {  // the second wavefront's sums, made alike, go to the first one's
        f32x4 *meet = reinterpret_cast<f32x4 *>(smem) + (wave % KW) * (2 * ND * 4 * 64) + lane;
        __syncthreads();
        if (share) {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    f32x4 x, y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = dk_acc[dt][4 * c + e] * dk_factor, y[e] = dv_acc[dt][4 * c + e] * dv_factor;
                    meet[(dt * 4 + c) * 64] = x;
                    meet[((ND + dt) * 4 + c) * 64] = y;
                }
        }
        __syncthreads();
        if (share) return;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const f32x4 x = meet[(dt * 4 + c) * 64], y = meet[((ND + dt) * 4 + c) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    dk_acc[dt][4 * c + e] = fmaf(dk_acc[dt][4 * c + e], dk_factor, x[e]);
                    dv_acc[dt][4 * c + e] = fmaf(dv_acc[dt][4 * c + e], dv_factor, y[e]);
                }
            }
        dk_factor = dv_factor = 1.f;
    }
    if (t.slot >= 0) {  // a part of the queries: [slot][key head][dK, dV][128][DP]
        float *to = parts + ((((int64_t)t.slot * (a.heads / a.share) + g) * 2) * GRAD_WAVES * 32 + own + l32) * DP + 4 * half;
        if (valid)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    f32x4 x, y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = dk_acc[dt][4 * c + e] * dk_factor, y[e] = dv_acc[dt][4 * c + e] * dv_factor;
                    *reinterpret_cast<f32x4 *>(to + dt * 32 + 8 * c) = x;
                    *reinterpret_cast<f32x4 *>(to + GRAD_WAVES * 32 * DP + dt * 32 + 8 * c) = y;
                }
        return;
    }
    store_columns<T, ND>(dk_acc, dk_factor, dk + my_row * lddk + g * a.dim, valid, a.dim, lane);
    store_columns<T, ND>(dv_acc, dv_factor, dv + my_row * lddv + g * a.dim, valid, a.dim, lane);
}

// dK and dV of keys whose queries were split: the parts in their order.  A thread has eight elements of one key.
template <class T>
__global__ __launch_bounds__(256) void key_join_kernel(const AttentionJoin *__restrict__ joins, int kv_heads, int dim, int DP, const float *__restrict__ parts, T *__restrict__ dk,
                                                       int64_t lddk, T *__restrict__ dv, int64_t lddv)
{
    const AttentionJoin jn = joins[blockIdx.x];
    const int g = blockIdx.y, which = blockIdx.z, chunks = dim / 8;
    for (int i = threadIdx.x; i < jn.rows * chunks; i += 256) {
        const int row = i / chunks, c = i % chunks;
        const float *p = parts + ((((int64_t)jn.slot0 * kv_heads + g) * 2 + which) * GRAD_WAVES * 32 + row) * DP + c * 8;
        const int64_t step = (int64_t)kv_heads * 2 * GRAD_WAVES * 32 * DP;
        f32x8 sum = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < jn.slots; ++s) {
            f32x8 x;
            __builtin_memcpy(&x, p + s * step, sizeof(x));
            sum += x;
        }
        Raw8<T> r;
        r.round(sum);
        r.store((which ? dv + (int64_t)(jn.row0 + row) * lddv : dk + (int64_t)(jn.row0 + row) * lddk) + g * dim + c * 8, 8);
    }
}

// ------------------------------------------------------------------ whole sequences
// Sequences of up to 32 NW keys and queries, all of which see each other, one head per block: queries, keys, values, dO and O are read once and S and dO V^T computed once, where
// the two kernels above read all but O twice, which bounds them there.  A wavefront has 32 keys in registers, K in LDS as well; the queries go by, 32 at a time: S = Q K^T and
// dP = dO V^T with a key per lane, P and dS from registers into dV^T and dK^T as in key_grad_kernel; dS, rounded, through LDS into dQ^T = K^T dS^T, of which each
// wavefront has tiles of 16 x 16, all keys of them.  The stores of a step's dQ are issued behind the next step's wait, which else would be for them.
// 512 sequences of 64 to 256 tokens, 12 heads of 64, with the bias's gradient: 73 us for those up to 128 and 416 for the others, 1.03 GB (the two kernels take 622 for
// all of it where this one takes 467).  Bound by latency: wavefronts
// wait 41 % of their time, two per SIMD at 212 registers, vector units 30 %, LDS 26 % and matrix cores 14 % busy.  dQ is some 13 % of it.  One barrier per step instead of two, dQ a step
// later, took 5 % more (registers spill), four stages of Q and dO 3 % more.

// As add_diagonals, of dS with a key per lane and 32 queries in registers: lane 16 b + i holds in a[c] position 16 (b - c) + i - 4 half.
__device__ inline void add_diagonals_of_keys(const f32x16 (&d)[1], float *sums, int lane)
{
    float a[3] = {0.f, 0.f, 0.f};
    add_rows<0>(a, d);
    const bool odd = lane & 16;
    const float2 one = both_rows(a[1]);
    a[0] += odd ? 0.f : one.y;
    a[2] += odd ? one.x : 0.f;
    float *at = sums + (lane & 31) - 4 * (lane >> 5);
    at[0] += a[0];
    at[-32] += a[2];
}

// Operand A of dQ^T for four groups of 32 keys from group FROM on.
template <class T, int DP, int FROM>
__device__ inline void groups_of_keys(const uint32_t (&at)[2], typename Half8<T>::type (&x)[4])
{
    constexpr int GROUP = 32 * DP * 2;
    s16x4 o[8];
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%10\n\tds_read_b64_tr_b16 %1, %9 offset:%10\n\tds_read_b64_tr_b16 %2, %8 offset:%11\n\t"
                 "ds_read_b64_tr_b16 %3, %9 offset:%11\n\tds_read_b64_tr_b16 %4, %8 offset:%12\n\tds_read_b64_tr_b16 %5, %9 offset:%12\n\t"
                 "ds_read_b64_tr_b16 %6, %8 offset:%13\n\tds_read_b64_tr_b16 %7, %9 offset:%13\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(o[0]), "=&v"(o[1]), "=&v"(o[2]), "=&v"(o[3]), "=&v"(o[4]), "=&v"(o[5]), "=&v"(o[6]), "=&v"(o[7])
                 : "v"(at[0]), "v"(at[1]), "n"(FROM * GROUP), "n"((FROM + 1) * GROUP), "n"((FROM + 2) * GROUP), "n"((FROM + 3) * GROUP));
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = Columns<T, DP>::join(o[2 * u], o[2 * u + 1]);
}

template <class T, int DP, int NW, bool BIAS>
__global__ __launch_bounds__(NW * 64, 2) void whole_grad_kernel(const AttentionItem *__restrict__ items, const AttentionTile *__restrict__ tiles, AttentionShape a,
                                                               const T *__restrict__ dout, int64_t ldd, const T *__restrict__ q, int64_t ldq, const T *__restrict__ k, int64_t ldk,
                                                               const T *__restrict__ v, int64_t ldv, const T *__restrict__ o, int64_t ldo, const float *__restrict__ lse, int64_t Tq,
                                                               const float *__restrict__ bias, const int32_t *__restrict__ bucket_of, T *__restrict__ dq, int64_t lddq,
                                                               T *__restrict__ dk, int64_t lddk, T *__restrict__ dv, int64_t lddv, float *__restrict__ by_position)
{
    typedef typename Half8<T>::type V8;
    typedef WholeCfg<DP, NW> Cfg;
    constexpr int KEYS = Cfg::KEYS, STAGE = Cfg::STAGE, ND = DP / 32, NS = DP / 16, CPR = DP / 8, RPI = 64 / CPR;
    constexpr int TILES = DP / 16 * 2, MINE = (TILES + NW - 1) / NW;  // 16 x 16 tiles of a step's dQ^T
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    T *Ks = reinterpret_cast<T *>(smem), *Qs = Ks + KEYS * DP, *Gs = Qs + 2 * STAGE, *Ds = Gs + 2 * STAGE;  // Q and dO: [2 stages][32][DP]
    float *numbers = reinterpret_cast<float *>(smem + Cfg::K_BYTES + Cfg::STAGES_BYTES + Cfg::DS_BYTES);   // [-lse, -delta][KEYS]
    float *table = reinterpret_cast<float *>(smem + Cfg::FIXED);
    const int entries = bias_entries(a.distance), room = (entries + 3) & ~3;
    float *sums = table + room;  // [NW wavefronts][2 halves][room]

    const AttentionItem item = items[blockIdx.x];
    if (item.tile < 0) return;
    const AttentionTile t = tiles[item.tile];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int h = item.head, lq = t.others, lk = t.rows, steps = (lq + 31) / 32;
    const int my_keys = min(32, lk - wave * 32), j = wave * 32 + l32;  // keys from 0 on, queries from position t.first
    const bool valid = l32 < my_keys;
    const T *qb = q + (int64_t)t.other0 * ldq + h * a.dim, *gb = dout + (int64_t)t.other0 * ldd + h * a.dim;

    // K: the wavefront's own rows.  Q and dO: pieces of 1 KB, those of Q first, in turn.
    const auto k_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(k + (int64_t)t.row0 * ldk + h * a.dim), 0, lk > 0 ? (int)(((lk - 1) * ldk + a.dim) * 2) : 0, 0x00020000);
    const int row_in = lane / CPR;
    auto offset = [&](int row, int64_t ld) {
        const int ch = (lane % CPR) ^ att_swizzle<DP>(row);
        return ch * 8 < a.dim ? (uint32_t)(row * ld + ch * 8) * 2 : 0x80000000u;
    };
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) lds_request(k_rsrc, offset(wave * 32 + i * RPI + row_in, ldk), Ks + (wave * 32 + i * RPI) * DP);
    const auto q_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(qb), 0, lq > 0 ? (int)(((lq - 1) * ldq + a.dim) * 2) : 0, 0x00020000);
    const auto g_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(gb), 0, lq > 0 ? (int)(((lq - 1) * ldd + a.dim) * 2) : 0, 0x00020000);
    auto request = [&](int step, int stage) {
#pragma unroll
        for (int p = wave; p < 2 * 32 / RPI; p += NW) {
            const int i = p % (32 / RPI) * RPI;
            if (p < 32 / RPI) lds_request(q_rsrc, offset(step * 32 + i + row_in, ldq), Qs + stage * STAGE + i * DP);
            else lds_request(g_rsrc, offset(step * 32 + i + row_in, ldd), Gs + stage * STAGE + i * DP);
        }
    };
    request(0, 0);
    V8 vf[NS], gf[NS], of[NS];
    load_rows<T, DP>(v + (int64_t)(t.row0 + wave * 32) * ldv + h * a.dim, ldv, my_keys, a.dim, lane, vf);
    // delta and the log-sum of the queries, 32 per wavefront; behind the last query P is 0
    load_rows<T, DP>(gb + (int64_t)wave * 32 * ldd, ldd, lq - wave * 32, a.dim, lane, gf);
    load_rows<T, DP>(o + (int64_t)(t.other0 + wave * 32) * ldo + h * a.dim, ldo, lq - wave * 32, a.dim, lane, of);
    const float my_lse = j < lq ? lse_in_log2(lse[(int64_t)h * Tq + t.other0 + j]) : INFINITY;
    if (BIAS) {
        // Behind the last query P is 0 times whatever the bias makes of it, so that has to be finite: positions that no pair of this sequence has are 0.  Of those that a pair has an
        // infinity or NaN is in that query's log-sum, and so in the gradients of all its keys, which are all of the sequence's.
        make_bias(table, bias, bucket_of, a, h, 1 - t.first - lq, lk - 1 - t.first);
        if (by_position)
            for (int i = tid; i < 2 * NW * room; i += NW * 64) sums[i] = 0.f;
    }
    float my_delta = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < 8; ++i) my_delta = fmaf((float)gf[s][i], (float)of[s][i], my_delta);
    my_delta = both_halves_sum(my_delta);
    if (half == 0) numbers[j] = -my_lse;
    else numbers[KEYS + j] = -my_delta;

    f32x16 dk_acc[ND], dv_acc[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk_acc[dt][r] = dv_acc[dt][r] = 0.f;
    const float scale2 = __builtin_fabsf(a.scale) * LOG2E;
    Columns<T, DP> columns;
    columns.init(lane);
    // operand A of dQ^T's tiles: 16 columns of K, eight adjacent keys per lane
    uint32_t k_at[MINE][2];
    const int l16 = lane & 15, g16 = lane >> 4;
#pragma unroll
    for (int m = 0; m < MINE; ++m) {
        const int tile = (wave + m * NW) % TILES, d0 = tile % (DP / 16) * 16;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = 8 * g16 + 4 * i + (l16 >> 2), col = d0 + 4 * (l16 & 3);
            k_at[m][i] = Columns<T, DP>::place(Ks) + (row * DP + (((col >> 3) ^ att_swizzle<DP>(row)) << 3) + (col & 7)) * 2;
        }
    }
    const int key_groups = (lk + 31) / 32;
    // dS in LDS: rows of queries, 16-byte chunks of keys XORed with the row's last three bits.  The lane's place in rows 4 half + {0..3}; columns of no keys are zeros.
    int ds_at[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) ds_at[e] = (4 * half + e) * KEYS + (((j >> 3) ^ (4 * half + e)) << 3) + (j & 7);
    if (my_keys <= 0)
        for (int row = 0; row < 32; row += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e) Ds[ds_at[e] + row * KEYS] = (T)0.f;
    arrived(vf);
    V8 kf[NS];
    f32x4 dq_acc[MINE];
    const float some = unless_only(lk), ds_scale = a.scale * some;
    auto store_dq = [&](int step) {
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
            const int tile = wave + m * NW, d = tile % (DP / 16) * 16 + 4 * g16, row = step * 32 + tile / (DP / 16) * 16 + l16;
            if (tile < TILES && row < lq && d < a.dim) {
                typedef T V4 __attribute__((ext_vector_type(4)));
                const f32x4 x = dq_acc[m] * ds_scale;
                *reinterpret_cast<V4 *>(dq + (int64_t)(t.other0 + row) * lddq + h * a.dim + d) = __builtin_convertvector(x, V4);
            }
        }
    };
    for (int step = 0; step < steps; ++step) {
        const int stage = step & 1;
        const T *Qt = Qs + stage * STAGE, *Gt = Gs + stage * STAGE;
        wait_for_requests<0>();
        block_barrier();  // this step's rows are there; the last one's, and its dS, have been read
        if (step == 0) {
#pragma unroll
            for (int s = 0; s < NS; ++s) kf[s] = row_operand<T, DP>(Ks, wave * 32, s, lane);
            take_sign(kf, a.scale);
        } else {
            store_dq(step - 1);
        }
        if (step + 1 < steps) request(step + 1, stage ^ 1);
        if (my_keys > 0) {
            f32x16 s, d[1];
            const int i0 = step * 32, pw = t.first + i0;
            const int least = wave * 32 - (pw + 31), most = wave * 32 + 31 - pw;  // relative positions
            const bool near = most > -a.distance && least < a.distance;
            float ls[16];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(numbers + i0 + 4 * half + 8 * c), y = *reinterpret_cast<const f32x4 *>(numbers + KEYS + i0 + 4 * half + 8 * c);
#pragma unroll
                for (int e = 0; e < 4; ++e) ls[4 * c + e] = x[e], d[0][4 * c + e] = y[e];
            }
            if (BIAS && near) {
                const int at = one_register(Cfg::FIXED / 4 + j - pw - 4 * half - 27 + a.distance + ATT_EXT);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = reinterpret_cast<const float *>(smem)[at + 27 - acc_row(r)];
            } else {
                const float c = BIAS ? table[most <= -a.distance ? 0 : entries - 1] : 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = c;
            }
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                s = att_mfma(row_operand<T, DP>(Qt, 0, i, lane), kf[i], s);
                d[0] = att_mfma(row_operand<T, DP>(Gt, 0, i, lane), vf[i], d[0]);
            }
            V8 gc[ND], qc[ND];
            columns.template both<0>(Gt, Qt, gc, qc);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale2, ls[r]));
                d[0][r] *= s[r];
            }
            if (!valid)  // keys behind the last one
#pragma unroll
                for (int r = 0; r < 16; ++r) d[0][r] = 0.f;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const V8 pf = rounded<T>(s, w), df = rounded<T>(d[0], w);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    dv_acc[dt] = att_mfma(gc[dt], pf, dv_acc[dt]);
                    dk_acc[dt] = att_mfma(qc[dt], df, dk_acc[dt]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {  // dS to its rows
                    const int row = acc_row(8 * w + i);  // less 4 half
                    Ds[ds_at[row & 3] + (row & ~7) * KEYS] = df[i];
                }
                if (w == 0) columns.template both<16>(Gt, Qt, gc, qc);
            }
            if (BIAS && by_position) {  // a tile that is all behind `distance`, to either side, adds to places there
                const int first = min(max(wave * 32 - pw, -a.distance - 31), a.distance + 31);
                add_diagonals_of_keys(d, sums + (2 * wave + half) * room + first + a.distance + ATT_EXT, lane);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        block_barrier();  // dS is there
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
            const int tile = (wave + m * NW) % TILES, row = tile / (DP / 16) * 16 + l16;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int part = 0; part < NW / 4; ++part) {  // 128 keys at a time
                if (part * 4 >= key_groups) continue;
                V8 b[4], x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) b[u] = *reinterpret_cast<const V8 *>(Ds + row * KEYS + ((((part * 4 + u) * 4 + g16) ^ (row & 7)) << 3));
                if (part == 0) groups_of_keys<T, DP, 0>(k_at[m], x);
                else groups_of_keys<T, DP, 4>(k_at[m], x);
#pragma unroll
                for (int u = 0; u < 4; ++u) acc = att_mfma16(x[u], b[u], acc);
            }
            dq_acc[m] = acc;
        }
    }
    if (steps) store_dq(steps - 1);
    const int64_t my_row = t.row0 + j;
    store_columns<T, ND>(dk_acc, ds_scale, dk + my_row * lddk + h * a.dim, valid, a.dim, lane);
    store_columns<T, ND>(dv_acc, 1.f, dv + my_row * lddv + h * a.dim, valid, a.dim, lane);

    if (BIAS && by_position)
        sums_by_position<NW>(sums, room, a.distance, 0.f, 0.f, reinterpret_cast<float *>(Ds), some, by_position + ((int64_t)item.tile * a.heads + h) * (2 * a.distance + 1));
}

// Sums of the bias's gradient by relative position over `each` tiles, in their order: 16, and of more than 1024 tiles half of their number's root, so that the next kernel
// has not too many to add (100 000 sequences of 4 tokens: the gradient 13.7 instead of 13.9 ms; 512 sequences in 23 sums of 23: 7.7 instead of 4.8 us).
__global__ __launch_bounds__(256) void position_sum_kernel(const float *__restrict__ from, int n, int each, int heads, int positions, float *__restrict__ to)
{
    const int h = blockIdx.y, first = blockIdx.x * each, last = min(first + each, n);
    for (int i = threadIdx.x; i < positions; i += 256) {
        float sum = 0.f;
#pragma unroll 8
        for (int r = first; r < last; ++r) sum += from[((int64_t)r * heads + h) * positions + i];
        to[((int64_t)blockIdx.x * heads + h) * positions + i] = sum;
    }
}

// dbias[buckets][heads] of one head from n rows of sums by relative position: the rows in order, then a wavefront per bucket.
__global__ __launch_bounds__(1024) void bucket_sum_kernel(const float *__restrict__ from, int n, int heads, int positions, const int32_t *__restrict__ bucket_of, int buckets,
                                                          float *__restrict__ dbias)
{
    __shared__ float sums[2 * ATT_MOST_DISTANCE + 1];
    const int h = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < positions; i += 1024) {
        float sum = 0.f;
#pragma unroll 8
        for (int r = 0; r < n; ++r) sum += from[((int64_t)r * heads + h) * positions + i];
        sums[i] = sum;
    }
    __syncthreads();
    for (int b = wave; b < buckets; b += 16) {
        float sum = 0.f;
        for (int i = lane; i < positions; i += 64) sum += bucket_of[i] == b ? sums[i] : 0.f;
        sum = wave_sum(sum);
        if (lane == 0) dbias[(int64_t)b * heads + h] = sum;
    }
}

template <int DP>
int allow_whole()
{
    for (const void *f : {(const void *)whole_grad_kernel<bf16_t, DP, 4, false>, (const void *)whole_grad_kernel<bf16_t, DP, 4, true>,
                          (const void *)whole_grad_kernel<bf16_t, DP, 8, false>, (const void *)whole_grad_kernel<bf16_t, DP, 8, true>})
        LEANN_HIP(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, ATT_LDS));
    return LEANN_OK;
}

template <class T, int DP>
int allow_grad()
{
    for (const void *f : {(const void *)query_grad_kernel<T, DP, false>, (const void *)query_grad_kernel<T, DP, true>, (const void *)key_grad_kernel<T, DP, 4, false>,
                          (const void *)key_grad_kernel<T, DP, 4, true>, (const void *)key_grad_kernel<T, DP, 2, false>, (const void *)key_grad_kernel<T, DP, 2, true>})
        LEANN_HIP(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, ATT_LDS));
    return LEANN_OK;
}

}  // namespace

int attention_grad_init_device()
{
    LEANN_TRY((allow_whole<32>()));
    LEANN_TRY((allow_whole<64>()));
    LEANN_TRY((allow_grad<bf16_t, 32>()));
    LEANN_TRY((allow_grad<bf16_t, 64>()));
    LEANN_TRY((allow_grad<bf16_t, 128>()));
    LEANN_TRY((allow_grad<f16_t, 32>()));
    LEANN_TRY((allow_grad<f16_t, 64>()));
    return allow_grad<f16_t, 128>();
}

extern "C" int leann_attention_backward(leann_ctx *ctx, const leann_attention_plan *plan, const void *dout_dev, int64_t ldd, const void *q_dev, int64_t ldq,
                                        const void *k_dev, int64_t ldk, const void *v_dev, int64_t ldv, const void *out_dev, int64_t ldo, const float *lse_dev, int dtype,
                                        float scale, const float *bias_dev, void *dq_dev, int64_t lddq, void *dk_dev, int64_t lddk, void *dv_dev, int64_t lddv,
                                        float *dbias_dev)
{
    static const char *call = "leann_attention_backward";
    LEANN_TRY(att_check_call(call, ctx, plan, dtype, scale, bias_dev));
    if (dbias_dev && !bias_dev) {
        leann_set_error("%s: a gradient of a bias without a bias", call);
        return LEANN_EINVAL;
    }
    const int64_t nq = (int64_t)plan->heads * plan->dim, nk = (int64_t)plan->kv_heads * plan->dim;
    AttentionMatrix in[5] = {{"dout", dout_dev, ldd, nq, plan->Tq}, {"q", q_dev, ldq, nq, plan->Tq}, {"k", k_dev, ldk, nk, plan->Tk}, {"v", v_dev, ldv, nk, plan->Tk},
                             {"out", out_dev, ldo, nq, plan->Tq}};
    AttentionMatrix to[3] = {{"dq", dq_dev, lddq, nq, plan->Tq}, {"dk", dk_dev, lddk, nk, plan->Tk}, {"dv", dv_dev, lddv, nk, plan->Tk}};
    for (const AttentionMatrix &m : in)
        if (m.rows) LEANN_TRY(att_check_rows(call, m.name, m.p, m.ld, m.cols));
    for (const AttentionMatrix &m : to)
        if (m.rows) LEANN_TRY(att_check_rows(call, m.name, m.p, m.ld, m.cols));
    if (plan->Tq && !lse_dev) {
        leann_set_error("%s: lse is null", call);
        return LEANN_EINVAL;
    }
    for (int i = 0; i < 3; ++i) {
        for (const AttentionMatrix &m : in) LEANN_TRY(att_check_apart(call, to[i], m));
        for (int j = 0; j < i; ++j) LEANN_TRY(att_check_apart(call, to[i], to[j]));
    }
    LEANN_HIP(hipSetDevice(ctx->device));
    const AttentionShape a = att_shape(plan, scale);
    // bf16: short sequences go through one kernel, the others through two; what fp16 needs of a lane's own scale, one dS for two products cannot have
    const AttentionSides &sides = dtype == LEANN_BF16 ? plan->others : plan->all;
    const int n_whole = dtype == LEANN_BF16 ? plan->whole[0].n_tiles + plan->whole[1].n_tiles : 0;
    const int positions = 2 * plan->distance + 1, n = sides.n_tiles + n_whole, each = std::max(16, ((int)sqrt(0.25 * n) + 7) & ~7), groups = (n + each - 1) / each;
    const size_t stats_bytes = ((size_t)plan->heads * plan->Tq * sizeof(float2) + 8 + 255) & ~(size_t)255;  // 8: see key_grad_kernel's requests
    const size_t row_bytes = (size_t)plan->heads * positions * sizeof(float);
    std::lock_guard<std::mutex> turn(ctx->op_work_mutex);
    const int DP = plan->dim <= 32 ? 32 : plan->dim <= 64 ? 64 : 128;
    const size_t part_bytes = (size_t)sides.n_slots * plan->kv_heads * 2 * GRAD_WAVES * 32 * DP * sizeof(float);
    LEANN_TRY(ctx->reserve(ctx->op_work, stats_bytes + part_bytes + (dbias_dev ? row_bytes * (n + groups) : 0)));
    float2 *stats = (float2 *)ctx->op_work.p;
    float *parts = (float *)((char *)ctx->op_work.p + stats_bytes), *by_position = dbias_dev ? (float *)((char *)parts + part_bytes) : nullptr;
    auto go = [&](auto *type, auto dp, auto with_bias) {
        typedef std::remove_pointer_t<decltype(type)> T;
        constexpr int DP = decltype(dp)::value;
        constexpr bool BIAS = decltype(with_bias)::value;
        typedef GradCfg<DP> Cfg;
        const int table = BIAS ? ((positions + 2 * ATT_EXT + 3) & ~3) * 4 : 0;
        const int query_smem = Cfg::QUERY_TILES + table * (by_position ? 1 + 2 * GRAD_WAVES : 1);
        if (sides.n_query_items)
            hipLaunchKernelGGL((query_grad_kernel<T, DP, BIAS>), dim3(sides.n_query_items), dim3(GRAD_WAVES * 64), query_smem, ctx->stream, sides.query_items, sides.query_tiles, a,
                               (const T *)dout_dev, ldd, (const T *)q_dev, ldq, (const T *)k_dev, ldk, (const T *)v_dev, ldv, (const T *)out_dev, ldo, lse_dev, plan->Tq, bias_dev,
                               plan->bucket_of, (T *)dq_dev, lddq, stats, by_position);
        auto keys = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(sides.n_key_items), dim3(GRAD_WAVES * 64), Cfg::KEY_TILES + Cfg::KEY_STAGES * Cfg::STATS + table, ctx->stream, sides.key_items,
                               sides.key_tiles, a, (const T *)dout_dev, ldd, (const T *)q_dev, ldq, (const T *)k_dev, ldk, (const T *)v_dev, ldv, stats, plan->Tq, bias_dev,
                               plan->bucket_of, (T *)dk_dev, lddk, (T *)dv_dev, lddv, parts);
        };
        if (sides.n_key_items) sides.key_waves == 4 ? keys(key_grad_kernel<T, DP, 4, BIAS>) : keys(key_grad_kernel<T, DP, 2, BIAS>);
        if (sides.n_joins)
            hipLaunchKernelGGL(key_join_kernel<T>, dim3(sides.n_joins, plan->kv_heads, 2), dim3(256), 0, ctx->stream, sides.joins, plan->kv_heads, plan->dim, DP, parts,
                               (T *)dk_dev, lddk, (T *)dv_dev, lddv);
        if constexpr (std::is_same_v<T, bf16_t> && DP <= 64) {
            float *rows = by_position ? by_position + (size_t)sides.n_tiles * plan->heads * positions : nullptr;
            auto whole = [&](const AttentionWhole &w, auto waves) {
                constexpr int NW = decltype(waves)::value;
                typedef WholeCfg<DP, NW> Whole;
                if (!w.n_items) return;
                hipLaunchKernelGGL((whole_grad_kernel<T, DP, NW, BIAS>), dim3(w.n_items), dim3(NW * 64), Whole::bytes(plan->distance, BIAS, rows != nullptr), ctx->stream,
                                   w.items, w.tiles, a, (const T *)dout_dev, ldd, (const T *)q_dev, ldq, (const T *)k_dev, ldk, (const T *)v_dev, ldv, (const T *)out_dev, ldo, lse_dev,
                                   plan->Tq, bias_dev, plan->bucket_of, (T *)dq_dev, lddq, (T *)dk_dev, lddk, (T *)dv_dev, lddv, rows);
                if (rows) rows += (size_t)w.n_tiles * plan->heads * positions;
            };
            whole(plan->whole[0], std::integral_constant<int, 4>());
            whole(plan->whole[1], std::integral_constant<int, 8>());
        }
    };
    auto with_type = [&](auto *type) {
        auto with_bias = [&](auto dp) {
            if (bias_dev) go(type, dp, std::true_type());
            else go(type, dp, std::false_type());
        };
        if (plan->dim <= 32) with_bias(std::integral_constant<int, 32>());
        else if (plan->dim <= 64) with_bias(std::integral_constant<int, 64>());
        else with_bias(std::integral_constant<int, 128>());
    };
    if (dtype == LEANN_BF16) with_type((bf16_t *)nullptr);
    else with_type((f16_t *)nullptr);
    if (dbias_dev) {
        const float *rows = by_position;
        int left = n;
        if (groups > 1) {
            float *sums = by_position + (size_t)n * plan->heads * positions;
            hipLaunchKernelGGL(position_sum_kernel, dim3(groups, plan->heads), dim3(256), 0, ctx->stream, rows, n, each, plan->heads, positions, sums);
            rows = sums;
            left = groups;
        }
        hipLaunchKernelGGL(bucket_sum_kernel, dim3(plan->heads), dim3(1024), 0, ctx->stream, rows, left, plan->heads, positions, plan->bucket_of, plan->buckets, dbias_dev);
    }
    return att_launched(call);
}
