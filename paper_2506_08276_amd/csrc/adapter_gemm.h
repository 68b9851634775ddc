// The shared projection with its adapters for many rows: 256 rows per tile, two groups of wavefronts that take turns (gfx950).
#pragma once
#include "adapter.h"

namespace {

typedef __attribute__((address_space(3))) void lds_t;
typedef const __attribute__((address_space(1))) void global_t;

__device__ u32x4 nowhere[64];  // where lanes without an output store where `out` goes on beyond 4 GB; never read

// A tile: WM x (8 / WM) wavefronts of TM x TN 32x32 MFMA tiles.  K goes by pairs of slabs of 32, 128 bytes of a row of x.
template <int WM, int TM, int TN>
struct ProjectCfg {
    static constexpr int WN = 8 / WM, BM = WM * TM * 32, BN = WN * TN * 32;
    static constexpr int A_BYTES = BM * 128, W_BYTES = BN * 64, STAGE = A_BYTES + 2 * W_BYTES;  // of a pair, of a slab, of a pair
    static constexpr int ROWS_AT = 2 * STAGE, OWN_AT = ROWS_AT + 3 * BM * 4;
    static constexpr int OWN = 2048 + 512;            // per wavefront: 16 rows of outputs on their way, the bias of its columns
    static constexpr int SMEM = OWN_AT + 8 * OWN;     // two stages, the row numbers of three tiles
    static constexpr int A_LOADS = BM / 64;           // requests of 1 KB per wavefront and pair
    static constexpr int W_LOADS = BN / 128;          // per wavefront and slab
    static constexpr int STORES = TM * ((TN + 1) / 2) * 4; // per tile
    static_assert(BN % 128 == 0 && BM % 128 == 0, "every wavefront has as many requests");
};

template <int VM>
__device__ inline void wait_memory_and_lds()  // VM requests may be on their way, no LDS access
{
    static_assert(VM < 64, "the counter has six bits");
    __builtin_amdgcn_s_waitcnt((VM & 15) | ((VM >> 4) << 14) | 0x70);
}

// Nothing is moved across, neither by the compiler's passes nor by its scheduler.
__device__ inline void fence()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
__device__ inline void barrier()
{
    fence();
    __builtin_amdgcn_s_barrier();
    fence();
}

// Memory to LDS without registers: 16 (or 4) bytes per lane, to `to` and on in the lanes' order.
__device__ inline void load_to_lds(const void *from, unsigned char *to) { __builtin_amdgcn_global_load_lds((global_t *)from, (lds_t *)to, 16, 0, 0); }
__device__ inline __amdgpu_buffer_rsrc_t buffer_of(const void *p, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, bytes, 0x00020000);
}
__device__ inline void load_to_lds(__amdgpu_buffer_rsrc_t b, int offset, int scalar_offset, unsigned char *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (lds_t *)to, 16, offset, scalar_offset, 0, 0);
}
__device__ inline void load_word_to_lds(__amdgpu_buffer_rsrc_t b, int offset, unsigned char *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (lds_t *)to, 4, offset, 0, 0, 0);
}

__device__ inline void store_past_l2(const u32x4 &v, __amdgpu_buffer_rsrc_t b, int offset) { __builtin_amdgcn_raw_buffer_store_b128(v, b, offset, 0, 2); }

// out[row][n] = sum over k of x[row][k] W[n][k] + bias[n] + the adapter's part, for many rows.  Persistent blocks of eight wavefronts, one per compute unit, a tile after the
// other; two groups of four take turns, one multiplying a slab while the other reads operands and requests, so that every SIMD has one of each.  An adapter of the
// tile is one more pair of slabs: pieces of the low-rank activations against `up`.
// 83 229 x 2304 x 768 with six adapters of rank 16: 300 us, 1.0 PFLOP/s, matrix pipes 49 % busy.  Bound by the memory phase: 48 KB of LDS reads per slab and the bytes
// of x in flight (two pairs, all that LDS holds) against the cache's latency; the write-out is 8 us per tile.  In turn: 256 x 192 tiles 421 us, two blocks
// of 128 x 192 per unit 356, three pairs of x and three slabs of W 343, at the times when this one took 372, 318 and 328 with all else of the call.
template <class T, int WM, int TM, int TN>
__global__ __launch_bounds__(512, 1) void project_large_kernel(const T *x, int64_t ldx, const T *w, const float *bias, int N, int K,
                                                               const int32_t *row_of, int rows, const int32_t *seg_ptr, const int4 *segs,
                                                               const bf16_t *pieces, int R16, const bf16_t *up, T *out, int64_t ldo, int tiles_n)
{
    typedef ProjectCfg<WM, TM, TN> Cfg;
    typedef typename Frag<T>::type F;
    constexpr int BM = Cfg::BM, BN = Cfg::BN, UP = Frag<T>::PIECES;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / Cfg::WN, wn = wave % Cfg::WN;
    const bool second = wave >= 4;  // the group that multiplies in the other's memory phases

    const int n_tiles = ((rows + BM - 1) / BM) * tiles_n;
    const int per_xcd = (n_tiles + 7) >> 3, blocks_per_xcd = gridDim.x >> 3;
    auto tile_at = [&](int step, int &tm, int &tn) -> bool {  // an XCD takes a run of tiles, all columns of a few rows
        const int in_xcd = step * blocks_per_xcd + (int)(blockIdx.x >> 3);
        const int tile = (int)(blockIdx.x & 7) * per_xcd + in_xcd;
        if (in_xcd >= per_xcd || tile >= n_tiles) return false;
        tm = tile / tiles_n;
        tn = tile % tiles_n;
        return true;
    };
    int tile_m = 0, tile_n = 0;
    if (!tile_at(0, tile_m, tile_n)) return;
    const int ksteps = project_ksteps(K), KP = (K + 63) >> 6;  // pairs: the host sees to it that there are 4
    const int whole = K >> 6, last_ct = (N - 1) >> 5;

    // The row numbers of the tile before, this one and the next, in LDS; `which`: of the three places.
    unsigned char *row_table = smem + Cfg::ROWS_AT;
    auto request_rows = [&](int tm, int which) {
        if (wave < BM / 64) load_word_to_lds(buffer_of(row_of + (size_t)tm * BM, BM * 4), (wave * 64 + lane) * 4, row_table + which * BM * 4 + wave * 256);
    };
    auto row_number = [&](int which, int at) { return (int64_t) * reinterpret_cast<const int *>(row_table + (which * BM + at) * 4); };

    // Requests.  A: 8 rows of 128 bytes each, whole lines, the lanes' pieces permuted so that piece c of row r lands at c ^ ((r >> 1) & 7): 16 rows'
    // reads of one piece reach all 64 banks.
    const int a_at = wave * Cfg::A_LOADS * 8 + (lane >> 3);
    static_assert(Cfg::A_LOADS % 2 == 0, "a wavefront's first row is a multiple of 16");
    auto a_piece = [&](int i) { return (lane & 7) ^ ((lane >> 4) + (i & 1) * 4); };  // of request i
    // Where x ends below 4 GB, offsets of 32 bits from its start (K of 768, 83 229 rows: 320 us, with addresses of 64 bits 336), else addresses; in units of 16 bytes, of
    // which the host sees to it that there are fewer than 2^32.
    const uint64_t x_bytes = ((uint64_t)(rows - 1) * ldx + K) * sizeof(T);
    const bool narrow = x_bytes < 0xffffff00u;
    const auto x_buffer = buffer_of(x, (int)(uint32_t)x_bytes);
    uint32_t p[Cfg::A_LOADS];
    auto take_rows = [&](int which) {
#pragma unroll
        for (int i = 0; i < Cfg::A_LOADS; ++i) p[i] = (uint32_t)(row_number(which, a_at + i * 8) * ldx >> 3) + a_piece(i);
    };
    auto request_a = [&](int pair, int stage) {
        unsigned char *to = smem + stage * Cfg::STAGE + wave * Cfg::A_LOADS * 1024;
        auto in = [&](int i) { return pair < whole || pair * 64 + a_piece(i) * 8 < K; };
        if (narrow) {  // beyond x: zeros
#pragma unroll
            for (int i = 0; i < Cfg::A_LOADS; ++i) load_to_lds(x_buffer, in(i) ? (int)((p[i] + pair * 8) * 16) : -256, 0, to + i * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < Cfg::A_LOADS; ++i)
                load_to_lds(in(i) ? (const void *)(reinterpret_cast<const char *>(x) + ((uint64_t)p[i] + pair * 8) * 16) : (const void *)&zero_piece, to + i * 1024);
        }
    };
    // An adapter's pair: the pieces of 32 ranks of the rows' low-rank activations (what follows them where there are fewer).
    auto request_pieces = [&](int tm, int group, int stage) {
        unsigned char *to = smem + stage * Cfg::STAGE + wave * Cfg::A_LOADS * 1024;
#pragma unroll
        for (int i = 0; i < Cfg::A_LOADS; ++i)
            load_to_lds(pieces + ((int64_t)min(tm * BM + a_at + i * 8, rows - 1) * R16 + group) * 32 + a_piece(i) * 8, to + i * 1024);
    };
    // W: 32 columns and 16 of K each, operand order in LDS too.  Offsets behind the last column: zeros.
    auto request_w = [&](__amdgpu_buffer_rsrc_t b, int column_bytes, int step_bytes, int at, int slab, int stage) {
        unsigned char *to = smem + stage * Cfg::STAGE + Cfg::A_BYTES + slab * Cfg::W_BYTES + wave * 1024;
#pragma unroll
        for (int i = 0; i < Cfg::W_LOADS; ++i)
            load_to_lds(b, lane * 16 + (wave & 1) * step_bytes + ((wave >> 1) + 4 * i) * column_bytes, at, to + i * 8192);
    };
    auto columns = [&](int tn) { return min(last_ct + 1 - tn * (BN / 32), BN / 32); };
    unsigned char *own = smem + Cfg::OWN_AT + wave * Cfg::OWN, *own_bias = own + 2048;
    const auto bias_buffer = buffer_of(bias, bias ? N * 4 : 0);
    auto request_bias = [&](int tn) {
#pragma unroll
        for (int i = 0; i < TN * 32; i += 64) load_word_to_lds(bias_buffer, (tn * BN + wn * TN * 32 + i + lane) * 4, own_bias + i * 4);
    };

    const int a_read = wm * TM * 4096 + l32 * 128 + ((half ^ ((l32 >> 1) & 7)) << 4), w_read = Cfg::A_BYTES + wn * TN * 2048 + lane * 16;
    F af[2][TM], bf[2][TN];
    f32x16 acc[TM][TN];
    auto read = [&](int a_slab, int w_slab, int stage) {
        const unsigned char *at = smem + stage * Cfg::STAGE;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const unsigned char *a = at + (a_read ^ (a_slab * 64 + ks * 32)), *w = at + w_read + w_slab * Cfg::W_BYTES + ks * 1024;
#pragma unroll
            for (int ni = 0; ni < TN; ++ni) bf[ks][ni] = *reinterpret_cast<const F *>(w + ni * 2048);
#pragma unroll
            for (int mi = 0; mi < TM; ++mi) af[ks][mi] = *reinterpret_cast<const F *>(a + mi * 4096);
        }
    };
    auto multiply = [&](int ks) {
#pragma unroll
        for (int mi = 0; mi < TM; ++mi)
#pragma unroll
            for (int ni = 0; ni < TN; ++ni) acc[mi][ni] = mfma32(bf[ks][ni], af[ks][mi], acc[mi][ni]);
    };
    auto compute_phase = [&] {
        barrier();
        __builtin_amdgcn_s_setprio(1);
        multiply(0);
        multiply(1);
        __builtin_amdgcn_s_setprio(0);
        barrier();
    };

    // Out: 16 rows of 64 columns at a time through the wavefront's own 2 KB (piece c of row r at c ^ ((r >> 1) & 7)), in whole lines of 128 bytes.  Every lane issues
    // every store, as waits count them.
    typedef typename Frag<T>::four Four;
    const uint64_t out_bytes = ((uint64_t)(rows - 1) * ldo + N) * sizeof(T);
    const bool out_narrow = out_bytes < 0xffffff00u;
    const auto out_buffer = buffer_of(out, (int)(uint32_t)out_bytes);
    auto write_out = [&](int which) {
        int l = lane;
        asm volatile("" : "+v"(l));  // what follows from it is worked out here, not held in registers over the whole tile
        const int l32 = l & 31, half = l >> 5;
#pragma unroll
        for (int mi = 0; mi < TM; ++mi)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi)
#pragma unroll
                for (int n2 = 0; n2 < TN; n2 += 2) {
                    __builtin_amdgcn_wave_barrier();  // LDS serves a wavefront's accesses in order
                    if ((l32 >> 4) == hi) {
#pragma unroll
                        for (int c2 = 0; c2 < 2 && n2 + c2 < TN; ++c2)
#pragma unroll
                            for (int g = 0; g < 4; ++g) {
                                Four v;
#pragma unroll
                                for (int i = 0; i < 4; ++i) v[i] = (T)acc[mi][n2 + c2][4 * g + i];
                                *reinterpret_cast<Four *>(own + (l32 & 15) * 128 + (((c2 * 4 + g) ^ ((l32 >> 1) & 7)) << 4) + half * 8) = v;
                            }
                    }
                    __builtin_amdgcn_wave_barrier();
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int r = j * 8 + (l >> 3), c = l & 7, at = wm * TM * 32 + mi * 32 + hi * 16 + r;
                        const int col = tile_n * BN + (wn * TN + n2) * 32 + c * 8;
                        const u32x4 v = *reinterpret_cast<const u32x4 *>(own + r * 128 + ((c ^ ((r >> 1) & 7)) << 4));
                        const int64_t row = row_number(which, at);
                        const bool has = tile_m * BM + at < rows && col < N && (n2 + 1 < TN || c < 4);
                        // Past L2, where W and x stay (83 229 x 2304 x 768: 318 us, through it 350).  Below 4 GB an offset behind the end is no access at all.
                        if (out_narrow) store_past_l2(v, out_buffer, has ? (int)(uint32_t)((row * ldo + col) * sizeof(T)) : -256);
                        else __builtin_nontemporal_store(v, has ? reinterpret_cast<u32x4 *>(out + row * ldo + col) : nowhere + l);
                    }
                }
    };

    // What comes: pairs of K of this tile, pairs of its adapters, pairs of the next tile.  Pair d is multiplied while A of pair d + 1 and W's second slab of
    // it are requested, then W's first slab of pair d + 2.  (Its first two pairs again where there is no tile after this one: in bounds, unused.)
    struct Pair {
        int tile;   // 0: this one, 1: the next
        int seg;    // of the adapters, -1: K
        int group;  // pair of K, or first group of 16 ranks
    };
    constexpr int GROUPS = 2 / UP;  // of 16 ranks in a pair: fp16's `up` takes two slabs for one
    int next_m, next_n, seg_end;
    auto after = [&](const Pair &a, int rank, int first_seg) {  // rank: of a's segment
        Pair b = a;
        if (a.seg < 0) {
            if (++b.group == KP && a.tile == 0) {
                b.group = 0;
                if (first_seg < seg_end) b.seg = first_seg;
                else b.tile = 1;
            }
        } else if ((b.group += GROUPS) >= ((rank + 15) >> 4)) {
            b.group = 0;
            if (++b.seg == seg_end) {
                b.seg = -1;
                b.tile = 1;
            }
        }
        return b;
    };
    auto ask_w = [&](const Pair &a, int number, int slab, int stage) {
        const int tn = a.tile ? next_n : tile_n;
        if (a.seg < 0) {
            request_w(buffer_of(w + (size_t)tn * (BN / 32) * ksteps * 512, columns(tn) * ksteps * 1024), ksteps * 1024, 1024, a.group * 4096 + slab * 2048,
                      slab, stage);
        } else {  // both pieces of the low-rank activations times one piece of `up`
            const int per_column = R16 * UP * 1024, step = min(a.group * UP + slab, R16 * UP - 1);
            request_w(buffer_of(up + ((size_t)number * (last_ct + 1) + tn * (BN / 32)) * R16 * UP * 512, columns(tn) * per_column), per_column, 0,
                      step * 1024, slab, stage);
        }
    };
    auto ask_a = [&](const Pair &a, int which, int stage) {
        if (a.seg >= 0) {
            request_pieces(tile_m, a.group, stage);
        } else {
            if (a.tile && a.group == 0) take_rows(which);
            request_a(a.group, stage);
        }
    };

    request_rows(tile_m, 0);
    wait_memory_and_lds<0>();
    barrier();
    next_m = tile_m;
    next_n = tile_n;
    request_bias(tile_n);
    take_rows(0);
    request_a(0, 0);
    ask_w(Pair{0, -1, 0}, 0, 0, 0);
    ask_w(Pair{0, -1, 0}, 0, 1, 0);
    ask_w(Pair{0, -1, 1}, 0, 0, 1);
    wait_memory_and_lds<Cfg::W_LOADS>();  // W's first two slabs: the first phase's wait counts on stores, which the first tile has not issued
    barrier();
    if (second) barrier();  // a phase behind
    int stage = 0;          // of the pair at hand
    for (int which = 0, step = 0;; ++step) {
        const int next_which = which == 2 ? 0 : which + 1;
        next_m = tile_m;
        next_n = tile_n;
        const bool have_next = tile_at(step + 1, next_m, next_n);
        // The first pair: the sums start at the bias.
        {
            f32x16 start[TN];
#pragma unroll
            for (int ni = 0; ni < TN; ++ni)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 b = *reinterpret_cast<const f32x4 *>(own_bias + (ni * 32 + 8 * g + 4 * half) * 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) start[ni][4 * g + i] = b[i];
                }
            read(0, 0, stage);
            request_a(1, stage ^ 1);
            ask_w(Pair{0, -1, 1}, 0, 1, stage ^ 1);
            wait_memory_and_lds<2 * Cfg::W_LOADS + Cfg::A_LOADS + Cfg::STORES>();
            barrier();
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int mi = 0; mi < TM; ++mi)
#pragma unroll
                for (int ni = 0; ni < TN; ++ni) acc[mi][ni] = mfma32(bf[0][ni], af[0][mi], start[ni]);
            multiply(1);
            __builtin_amdgcn_s_setprio(0);
            barrier();
        }
        read(1, 1, stage);
        ask_w(Pair{0, -1, 2}, 0, 0, stage);
        request_rows(next_m, next_which);  // held the rows of two tiles ago, which are out
        wait_memory_and_lds<2 * Cfg::W_LOADS>();
        compute_phase();
        stage ^= 1;
        const int first_seg = seg_ptr[tile_m];
        seg_end = seg_ptr[tile_m + 1];
        int d = 1;
        for (; d < KP - 2; ++d, stage ^= 1) {
            read(0, 0, stage);
            request_a(d + 1, stage ^ 1);
            ask_w(Pair{0, -1, d + 1}, 0, 1, stage ^ 1);
            wait_memory_and_lds<2 * Cfg::W_LOADS + Cfg::A_LOADS>();
            compute_phase();
            read(1, 1, stage);
            ask_w(Pair{0, -1, d + 2}, 0, 0, stage);
            wait_memory_and_lds<2 * Cfg::W_LOADS>();
            compute_phase();
        }
        request_bias(next_n);
        // The last two pairs of K, then the adapters'.
        Pair now = {0, -1, KP - 2}, ask1 = {0, -1, KP - 1}, ask2;
        int4 now_seg = {}, ask1_seg = {}, ask2_seg = {};
        auto first_half = [&] {
            ask2 = after(ask1, ask1_seg.z, first_seg);
            ask2_seg = ask2.seg == ask1.seg ? ask1_seg : ask2.seg >= 0 ? segs[ask2.seg] : int4{};
            ask_a(ask1, next_which, stage ^ 1);
            ask_w(ask1, ask1_seg.w, 1, stage ^ 1);
            wait_memory_and_lds<2 * Cfg::W_LOADS + Cfg::A_LOADS>();
        };
        auto second_half = [&] {
            ask_w(ask2, ask2_seg.w, 0, stage);
            wait_memory_and_lds<2 * Cfg::W_LOADS>();
        };
        auto shift = [&] {
            stage ^= 1;
            now = ask1;
            now_seg = ask1_seg;
            ask1 = ask2;
            ask1_seg = ask2_seg;
        };
        for (int i = 0; i < 2; ++i) {
            read(0, 0, stage);
            first_half();
            compute_phase();
            read(1, 1, stage);
            second_half();
            compute_phase();
            shift();
        }
        // A lane holds one slot of the output; the lanes that are not the adapter's keep what they have: another request's infinities stay with it.
        auto adapter_phase = [&](int slab) {
            barrier();
            const int first = tile_m * BM + wm * TM * 32;  // the wavefront's slots: all the adapter's, some or none
            const bool has_ranks = now.group * UP + slab < ((now_seg.z + 15) >> 4) * UP;
            if (has_ranks && now_seg.x <= first && now_seg.y >= first + TM * 32) {
#pragma unroll
                for (int ks = 1; ks >= 0; --ks)
#pragma unroll
                    for (int mi = 0; mi < TM; ++mi)
#pragma unroll
                        for (int ni = 0; ni < TN; ++ni)
                            acc[mi][ni] = mfma32(__builtin_bit_cast(bf16x8, bf[0][ni]), __builtin_bit_cast(bf16x8, af[ks][mi]), acc[mi][ni]);
            }
            if (has_ranks && now_seg.x < first + TM * 32 && now_seg.y > first && (now_seg.x > first || now_seg.y < first + TM * 32)) {
#pragma unroll
                for (int mi = 0; mi < TM; ++mi) {
                    const int slot = first + mi * 32 + l32;
                    const bool mine = slot >= now_seg.x && slot < now_seg.y;
#pragma unroll
                    for (int ni = 0; ni < TN; ++ni) {
                        const bf16x8 u = __builtin_bit_cast(bf16x8, bf[0][ni]);
                        f32x16 sum = mfma32(u, __builtin_bit_cast(bf16x8, af[1][mi]), acc[mi][ni]);
                        sum = mfma32(u, __builtin_bit_cast(bf16x8, af[0][mi]), sum);
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[mi][ni][j] = mine ? sum[j] : acc[mi][ni][j];
                    }
                }
            }
            barrier();
        };
        while (!now.tile) {
            read(0, 0, stage);
            first_half();
            adapter_phase(0);
            if (now.group * UP + 1 < ((now_seg.z + 15) >> 4) * UP) read(UP == 2 ? 0 : 1, 1, stage);
            second_half();
            adapter_phase(1);
            shift();
        }
        write_out(which);
        which = next_which;
        if (!have_next) break;
        tile_m = next_m;
        tile_n = next_n;
    }
    if (!second) barrier();
    wait_memory_and_lds<0>();  // nothing is on its way to LDS when the block's space becomes another's
}

}  // namespace
