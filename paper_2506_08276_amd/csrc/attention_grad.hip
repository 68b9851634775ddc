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

template <int DP>
struct GradCfg {
    static constexpr int NT = GRAD_WAVES * 64, TILE = ATT_STEP * DP;
    static constexpr int TILES = 4 * TILE * 2;  // bytes
    static constexpr int FIXED = TILES + 1024 + 128;
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

__device__ inline float lse_in_log2(float lse)  // of rows that see nothing: P is 0
{
    return lse == -INFINITY ? INFINITY : lse * LOG2E;
}

// A block takes 128 queries of one head through their keys, as the forward pass does.  S^T and dP^T = V dO^T have a query per lane; dS^T, rounded, is the other operand of
// dQ^T = K^T dS^T.
// The bias's gradient is summed by relative position: each wavefront has, for either half of its lanes, an array of its own in LDS, to which 32 lanes add at 32 places that
// differ; so the order of the additions is the program's.  Tiles behind `distance` add to one place, in a register.
template <class T, int DP, bool BIAS>
__global__ __launch_bounds__(GRAD_WAVES * 64, DP == 128 ? 1 : 2) void query_grad_kernel(const AttentionItem *__restrict__ items, const AttentionTile *__restrict__ tiles, AttentionShape a,
                                                                       const T *__restrict__ dout, int64_t ldd, const T *__restrict__ q, int64_t ldq, const T *__restrict__ k,
                                                                       int64_t ldk, const T *__restrict__ v, int64_t ldv, const T *__restrict__ o, int64_t ldo,
                                                                       const float *__restrict__ lse, int64_t Tq, const float *__restrict__ bias,
                                                                       const int32_t *__restrict__ bucket_of, T *__restrict__ dq, int64_t lddq, float *__restrict__ delta,
                                                                       float *__restrict__ by_position)
{
    typedef typename Half8<T>::type V8;
    constexpr int NT = GradCfg<DP>::NT, TILE = GradCfg<DP>::TILE, ND = DP / 32, NS = DP / 16;
    constexpr bool F16 = shift_of<T> != 0.f;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    T *Ks = reinterpret_cast<T *>(smem), *Vs = Ks + 2 * TILE;
    uint32_t *bad = reinterpret_cast<uint32_t *>(smem + GradCfg<DP>::TILES);             // [3][2]
    float *far_sums = reinterpret_cast<float *>(smem + GradCfg<DP>::TILES + 64);          // [4][2]
    float *table = reinterpret_cast<float *>(smem + GradCfg<DP>::FIXED);
    const int entries = bias_entries(a.distance);
    float *sums = table + entries;  // [4 wavefronts][2 halves][entries]

    const AttentionItem item = items[blockIdx.x];
    if (item.tile < 0) return;
    const AttentionTile t = tiles[item.tile];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int h = item.head, g = h / a.share;
    const T *kb = k + (int64_t)t.other0 * ldk + g * a.dim, *vb = v + (int64_t)t.other0 * ldv + g * a.dim;
    auto tile_at = [&](int u) { return u < t.sink_tiles ? u : t.first_tile + u - t.sink_tiles; };

    TileInFlight<T, DP, NT> kin, vin;
    auto fetch = [&](int u) {
        const int row = tile_at(u) * ATT_STEP;
        kin.load(kb, ldk, row, t.others, a.dim);
        vin.load(vb, ldv, row, t.others, a.dim);
    };
    if (t.begin < t.end) fetch(t.begin);
    const int my_rows = min(32, t.rows - wave * 32), p0 = t.at + wave * 32;
    const int64_t my_row = t.row0 + wave * 32 + l32;
    const bool valid = l32 < my_rows;
    V8 qf[NS], gf[NS];
    float my_delta = 0.f;
    load_rows<T, DP>(valid ? q + my_row * ldq + h * a.dim : nullptr, a.dim, lane, qf);
    load_rows<T, DP>(valid ? dout + my_row * ldd + h * a.dim : nullptr, a.dim, lane, gf);
    {
        V8 of[NS];
        load_rows<T, DP>(valid ? o + my_row * ldo + h * a.dim : nullptr, a.dim, lane, of);
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) my_delta = fmaf((float)gf[s][i], (float)of[s][i], my_delta);
        my_delta = both_halves_sum(my_delta);
        if (valid && half == 0) delta[(int64_t)h * Tq + my_row] = my_delta;
    }
    const float my_lse = valid ? lse_in_log2(lse[(int64_t)h * Tq + my_row]) - shift_of<T> : INFINITY;
    if (BIAS) {
        make_bias(table, bias, bucket_of, a, h);
        if (by_position)
            for (int i = tid; i < GRAD_WAVES * 2 * entries; i += NT) sums[i] = 0.f;
    }
    if (tid < 6) bad[tid] = 0;
    __syncthreads();

    f32x16 acc[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[dt][r] = 0.f;
    float factor = 1.f, behind = 0.f, ahead = 0.f;
    bool hurt = false;  // sees a key that is not finite
    const float scale2 = a.scale * LOG2E;
    const int p = p0 + l32;
    float *my_sums = sums + (wave * 2 + half) * entries;

    for (int u = t.begin, n = 0; u < t.end; ++u, ++n) {
        const int j0 = tile_at(u) * ATT_STEP, buf = n & 1;
        uint32_t *bad_now = bad + 2 * (n % 3);
        const T *Kt = Ks + buf * TILE, *Vt = Vs + buf * TILE;
        const bool edge = !sight(a, t.at, t.rows, j0, t.others - j0).all;
        if (edge) kin.take_out_nonfinite(bad_now);
        kin.store(Ks + buf * TILE);
        vin.store(Vs + buf * TILE);
        __syncthreads();
        if (tid < 2) bad[2 * ((n + 2) % 3) + tid] = 0;  // read before this barrier, set again behind the next
        if (u + 1 < t.end) fetch(u + 1);
        const Sight see = sight(a, p0, my_rows, j0, t.others - j0);
        if (see.none) continue;

        f32x16 s[2], d[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = d[kt][r] = 0.f;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                s[kt] = att_mfma(row_operand<T, DP>(Kt, kt * 32, i, lane), qf[i], s[kt]);
                d[kt] = att_mfma(row_operand<T, DP>(Vt, kt * 32, i, lane), gf[i], d[kt]);
            }
        }
        const int j = j0 + 4 * half;
        const int least = j0 - (p0 + 31), most = j0 + ATT_STEP - 1 - p0;  // relative positions
        const bool near = most > -a.distance && least < a.distance;
        const int at = j - p + a.distance + ATT_EXT;
        if (BIAS && near) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = fmaf(s[kt][r], scale2, table[at + kt * 32 + acc_row(r)] - my_lse);
        } else {
            const float c = (BIAS ? table[most <= -a.distance ? 0 : entries - 1] : 0.f) - my_lse;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kt][r] = fmaf(s[kt][r], scale2, c);
        }
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) d[kt][r] = __builtin_amdgcn_exp2f(s[kt][r]) * (d[kt][r] - my_delta);
        if (!see.all) {
            const int last = min(t.others - 1, p + a.right) - j, from = p - a.left - j, sinks = a.sinks - j;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int c = kt * 32 + acc_row(r);
                    if (c > last || (c < from && c >= sinks)) d[kt][r] = 0.f;  // a choice, not a product
                }
        }
        if (BIAS && by_position) {
            if (near) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (valid) __hip_atomic_fetch_add(my_sums + at + kt * 32 + acc_row(r), d[kt][r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            } else {
                float sum = 0.f;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum += d[kt][r];
                if (!valid) sum = 0.f;
                if (most <= -a.distance) behind += sum;
                else ahead += sum;
            }
        }
        if (F16) stay_in_range(d, acc, factor);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const V8 df = rounded<T>(d[kt], w);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) acc[dt] = att_mfma(column_operand<T, DP>(Kt, kt * 32 + w * 16, dt * 32, lane), df, acc[dt]);
            }
        if (edge && (bad_now[0] | bad_now[1]))
            for (int i = 0; i < ATT_STEP; ++i)
                if (bad_now[i >> 5] >> (i & 31) & 1) hurt |= j0 + i <= p + a.right && (j0 + i >= p - a.left || j0 + i < a.sinks);
    }
    if (hurt) factor = __builtin_nanf("");
    store_columns<T, ND>(acc, a.scale / factor * (F16 ? 0x1p-15f : 1.f), dq + my_row * lddq + h * a.dim, valid, a.dim, lane);

    if (BIAS && by_position) {
        const float b = wave_sum(behind), c = wave_sum(ahead);
        if (lane == 0) far_sums[wave * 2] = b, far_sums[wave * 2 + 1] = c;
        __syncthreads();
        const int positions = 2 * a.distance + 1;
        float *to = by_position + ((int64_t)item.tile * a.heads + h) * positions;
        for (int i = tid; i < positions; i += NT) {
            float sum = 0.f;
            const int from = i == 0 ? 0 : i + ATT_EXT, last = i == positions - 1 ? entries - 1 : i + ATT_EXT;  // the ends have what lies beyond
            for (int w = 0; w < GRAD_WAVES; ++w) {
                if (i == 0) sum += far_sums[w * 2];
                if (i == positions - 1) sum += far_sums[w * 2 + 1];
                for (int e = from; e <= last; ++e) sum += sums[(2 * w) * entries + e] + sums[(2 * w + 1) * entries + e];
            }
            to[i] = sum * (F16 ? 0x1p-15f : 1.f);
        }
    }
}

// A block takes 128 keys of one key head through the queries that see them, of every head that shares it: S = Q K^T and dP = dO V^T have a key per lane; P and dS, rounded, are the
// other operands of dV^T = dO^T P and dK^T = Q^T dS.  K and V stay in registers.
template <class T, int DP, bool BIAS>
__global__ __launch_bounds__(GRAD_WAVES * 64, DP == 128 ? 1 : 2) void key_grad_kernel(const AttentionItem *__restrict__ items, const AttentionTile *__restrict__ tiles, AttentionShape a,
                                                                     const T *__restrict__ dout, int64_t ldd, const T *__restrict__ q, int64_t ldq, const T *__restrict__ k,
                                                                     int64_t ldk, const T *__restrict__ v, int64_t ldv, const float *__restrict__ lse,
                                                                     const float *__restrict__ delta, int64_t Tq, const float *__restrict__ bias,
                                                                     const int32_t *__restrict__ bucket_of, T *__restrict__ dk, int64_t lddk, T *__restrict__ dv, int64_t lddv)
{
    typedef typename Half8<T>::type V8;
    constexpr int NT = GradCfg<DP>::NT, TILE = GradCfg<DP>::TILE, ND = DP / 32, NS = DP / 16;
    constexpr bool F16 = shift_of<T> != 0.f;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    T *Qs = reinterpret_cast<T *>(smem), *Gs = Qs + 2 * TILE;
    float *stats = reinterpret_cast<float *>(smem + GradCfg<DP>::TILES);                    // [2 buffers][lse, delta][64]
    uint32_t *bad = reinterpret_cast<uint32_t *>(smem + GradCfg<DP>::TILES + 1024);          // [3][Q, dO][2]
    float *table = reinterpret_cast<float *>(smem + GradCfg<DP>::FIXED);

    const AttentionItem item = items[blockIdx.x];
    if (item.tile < 0) return;
    const AttentionTile t = tiles[item.tile];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int g = item.head;
    const int my_rows = min(32, t.rows - wave * 32), jw = t.at + wave * 32, j = jw + l32;
    const int64_t my_row = t.row0 + wave * 32 + l32;
    const bool valid = l32 < my_rows;
    V8 kf[NS], vf[NS];
    load_rows<T, DP>(valid ? k + my_row * ldk + g * a.dim : nullptr, a.dim, lane, kf);
    load_rows<T, DP>(valid ? v + my_row * ldv + g * a.dim : nullptr, a.dim, lane, vf);
    if (tid < 12) bad[tid] = 0;

    f32x16 dk_acc[ND], dv_acc[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk_acc[dt][r] = dv_acc[dt][r] = 0.f;
    float factor = 1.f;
    bool hurt = false;
    const float scale2 = a.scale * LOG2E;
    const int per_head = t.end - t.begin;
    // what keys `from` .. `from + keys - 1` get from the queries i0 .. i0 + 63
    auto look = [&](int from, int keys, int i0) {
        const int p = t.first + i0, last_p = t.first + min(i0 + ATT_STEP, t.others) - 1, last = from + keys - 1;
        const bool none = keys <= 0 || from > last_p + a.right || (last < p - a.left && from >= a.sinks);
        const bool all = i0 + ATT_STEP <= t.others && last <= p + a.right && (from >= last_p - a.left || last < a.sinks);
        return Sight{none, all};
    };

    TileInFlight<T, DP, NT> qin, gin;
    float stat = 0.f;
    auto fetch = [&](int n) {
        const int h = g * a.share + n / per_head, i0 = (t.first_tile + n % per_head) * ATT_STEP;
        qin.load(q + (int64_t)t.other0 * ldq + h * a.dim, ldq, i0, t.others, a.dim);
        gin.load(dout + (int64_t)t.other0 * ldd + h * a.dim, ldd, i0, t.others, a.dim);
        if (tid < 128) {
            const int i = i0 + (tid & 63);
            const int64_t at = (int64_t)h * Tq + t.other0 + i;
            stat = i < t.others ? (tid < 64 ? lse[at] : delta[at]) : -INFINITY;
        }
    };
    const int total = per_head * a.share;
    if (total) fetch(0);
    int of_table = -1;
    for (int n = 0; n < total; ++n) {
        const int h = g * a.share + n / per_head, i0 = (t.first_tile + n % per_head) * ATT_STEP, buf = n & 1;
        uint32_t *bad_now = bad + 4 * (n % 3);
        const T *Qt = Qs + buf * TILE, *Gt = Gs + buf * TILE;
        if (BIAS && h != of_table) {
            __syncthreads();  // the last head's table has been read
            make_bias(table, bias, bucket_of, a, h);
            of_table = h;
        }
        if (n == 0) __syncthreads();  // bad[] is cleared
        const bool edge = !look(t.at, t.rows, i0).all;
        if (edge) {
            qin.take_out_nonfinite(bad_now);
            gin.take_out_nonfinite(bad_now + 2);
        }
        qin.store(Qs + buf * TILE);
        gin.store(Gs + buf * TILE);
        if (tid < 128) stats[buf * 128 + tid] = tid < 64 ? lse_in_log2(stat) - shift_of<T> : stat;
        __syncthreads();
        if (tid < 4) bad[4 * ((n + 2) % 3) + tid] = 0;
        if (n + 1 < total) fetch(n + 1);
        const Sight see = look(jw, my_rows, i0);
        if (see.none) continue;

#pragma unroll
        for (int qs = 0; qs < 2; ++qs) {
            f32x16 s[1], d[1];
#pragma unroll
            for (int r = 0; r < 16; ++r) s[0][r] = d[0][r] = 0.f;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                s[0] = att_mfma(row_operand<T, DP>(Qt, qs * 32, i, lane), kf[i], s[0]);
                d[0] = att_mfma(row_operand<T, DP>(Gt, qs * 32, i, lane), vf[i], d[0]);
            }
            // register r is query i0 + 32 qs + 4 half + acc_row(r)
            const int from = i0 + qs * 32 + 4 * half, p = t.first + from;
            float ls[16], de[16];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(stats + buf * 128 + qs * 32 + 4 * half + 8 * c);
                const f32x4 y = *reinterpret_cast<const f32x4 *>(stats + buf * 128 + 64 + qs * 32 + 4 * half + 8 * c);
#pragma unroll
                for (int e = 0; e < 4; ++e) ls[4 * c + e] = x[e], de[4 * c + e] = y[e];
            }
            if (BIAS) {
                const int pw = t.first + i0 + qs * 32, least = jw - (pw + 31), most = jw + 31 - pw;
                if (most > -a.distance && least < a.distance) {
                    const float *at = table + (j - p + a.distance + ATT_EXT);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[0][r] = fmaf(s[0][r], scale2, at[-acc_row(r)] - ls[r]);
                } else {
                    const float c = table[most <= -a.distance ? 0 : bias_entries(a.distance) - 1];
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[0][r] = fmaf(s[0][r], scale2, c - ls[r]);
                }
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[0][r] = fmaf(s[0][r], scale2, -ls[r]);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[0][r] = __builtin_amdgcn_exp2f(s[0][r]);
                d[0][r] = s[0][r] * (d[0][r] - de[r]);
            }
            if (!see.all) {
                const int rows = t.others - from, first = j - a.right - p, last = j < a.sinks ? ATT_STEP : j + a.left - p;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int c = acc_row(r);
                    if (c >= rows || c < first || c > last) s[0][r] = d[0][r] = 0.f;
                }
            }
            if (F16) stay_in_range(d, dk_acc, factor);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const V8 pf = rounded<T>(s[0], w), df = rounded<T>(d[0], w);
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    dv_acc[dt] = att_mfma(column_operand<T, DP>(Gt, qs * 32 + w * 16, dt * 32, lane), pf, dv_acc[dt]);
                    dk_acc[dt] = att_mfma(column_operand<T, DP>(Qt, qs * 32 + w * 16, dt * 32, lane), df, dk_acc[dt]);
                }
            }
        }
        if (edge && (bad_now[0] | bad_now[1] | bad_now[2] | bad_now[3])) {
            auto seen = [&](int i) { return j <= t.first + i + a.right && (j >= t.first + i - a.left || j < a.sinks); };
            for (int i = 0; i < ATT_STEP; ++i)
                if (bad_now[i >> 5] >> (i & 31) & 1) hurt |= seen(i0 + i);
            add_nonfinite<T, ND>(dv_acc, bad_now + 2, dout + (int64_t)t.other0 * ldd + h * a.dim, ldd, i0, a.dim, half, seen);
        }
    }
    if (hurt) factor = __builtin_nanf("");
    store_columns<T, ND>(dk_acc, a.scale / factor * (F16 ? 0x1p-15f : 1.f), dk + my_row * lddk + g * a.dim, valid, a.dim, lane);
    store_columns<T, ND>(dv_acc, F16 ? 0x1p-15f : 1.f, dv + my_row * lddv + g * a.dim, valid, a.dim, lane);
}

// Sums of the bias's gradient by relative position over up to POSITION_ROWS tiles each, in their order.
constexpr int POSITION_ROWS = 32;
__global__ __launch_bounds__(256) void position_sum_kernel(const float *__restrict__ from, int n, int heads, int positions, float *__restrict__ to)
{
    const int h = blockIdx.y, first = blockIdx.x * POSITION_ROWS, last = min(first + POSITION_ROWS, n);
    for (int i = threadIdx.x; i < positions; i += 256) {
        float sum = 0.f;
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

template <class T, int DP>
int allow_grad()
{
    for (const void *f : {(const void *)query_grad_kernel<T, DP, false>, (const void *)query_grad_kernel<T, DP, true>, (const void *)key_grad_kernel<T, DP, false>,
                          (const void *)key_grad_kernel<T, DP, true>})
        LEANN_HIP(hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024));
    return LEANN_OK;
}

}  // namespace

int attention_grad_init_device()
{
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
    const int positions = 2 * plan->distance + 1, n = plan->n_grad_tiles, groups = (n + POSITION_ROWS - 1) / POSITION_ROWS;
    const size_t delta_bytes = ((size_t)plan->heads * plan->Tq * sizeof(float) + 255) & ~(size_t)255;
    const size_t row_bytes = (size_t)plan->heads * positions * sizeof(float);
    std::lock_guard<std::mutex> turn(ctx->op_work_mutex);
    LEANN_TRY(ctx->reserve(ctx->op_work, std::max<size_t>(1, delta_bytes + (dbias_dev ? row_bytes * (n + groups) : 0))));
    float *delta = (float *)ctx->op_work.p, *by_position = dbias_dev ? (float *)((char *)ctx->op_work.p + delta_bytes) : nullptr;
    auto go = [&](auto *type, auto dp, auto with_bias) {
        typedef std::remove_pointer_t<decltype(type)> T;
        constexpr int DP = decltype(dp)::value;
        constexpr bool BIAS = decltype(with_bias)::value;
        const int table = BIAS ? (positions + 2 * ATT_EXT) * 4 : 0;
        if (plan->n_grad_items)
            hipLaunchKernelGGL((query_grad_kernel<T, DP, BIAS>), dim3(plan->n_grad_items), dim3(GRAD_WAVES * 64),
                               GradCfg<DP>::FIXED + table * (by_position ? 1 + 2 * GRAD_WAVES : 1), ctx->stream, plan->grad_items, plan->grad_tiles, a, (const T *)dout_dev, ldd,
                               (const T *)q_dev, ldq, (const T *)k_dev, ldk, (const T *)v_dev, ldv, (const T *)out_dev, ldo, lse_dev, plan->Tq, bias_dev, plan->bucket_of,
                               (T *)dq_dev, lddq, delta, by_position);
        if (plan->n_key_items)
            hipLaunchKernelGGL((key_grad_kernel<T, DP, BIAS>), dim3(plan->n_key_items), dim3(GRAD_WAVES * 64), GradCfg<DP>::FIXED + table, ctx->stream, plan->key_items,
                               plan->key_tiles, a, (const T *)dout_dev, ldd, (const T *)q_dev, ldq, (const T *)k_dev, ldk, (const T *)v_dev, ldv, lse_dev, delta, plan->Tq,
                               bias_dev, plan->bucket_of, (T *)dk_dev, lddk, (T *)dv_dev, lddv);
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
            hipLaunchKernelGGL(position_sum_kernel, dim3(groups, plan->heads), dim3(256), 0, ctx->stream, rows, n, plan->heads, positions, sums);
            rows = sums;
            left = groups;
        }
        hipLaunchKernelGGL(bucket_sum_kernel, dim3(plan->heads), dim3(1024), 0, ctx->stream, rows, left, plan->heads, positions, plan->bucket_of, plan->buckets, dbias_dev);
    }
    return att_launched(call);
}
