// The shared projection with its adapters for many rows: 256 rows per tile, two groups of wavefronts that take turns (gfx950).
#pragma once
#include "adapter.h"

namespace {

typedef __attribute__((address_space(3))) void lds_t;
typedef const __attribute__((address_space(1))) void global_t;

__device__ const uint32_t zero_piece[4] = {0, 0, 0, 0};  // what rows hold beyond K

// A tile: WM x (8 / WM) wavefronts of TM x TN 32x32 MFMA tiles.
template <int WM, int TM, int TN>
struct ProjectCfg {
    static constexpr int WN = 8 / WM, BM = WM * TM * 32, BN = WN * TN * 32;
    static constexpr int A_BYTES = BM * 64, STAGE = (BM + BN) * 64;  // of a slab of 32 columns of K
    static constexpr int SMEM = 4 * STAGE + 8 * (2048 + 512);        // four stages; per wavefront 16 rows of outputs on their way, and the bias of its columns
    static constexpr int A_LOADS = BM / 128;                         // requests of 1 KB per wavefront and slab
    static constexpr int LOADS = A_LOADS + BN / 128;                 // at least
    static constexpr int STORES = TM * TN * 2;                       // per wavefront and tile
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

template <class T, int WM, int TM, int TN>
__global__ __launch_bounds__(512, 1) void project_large_kernel(const T *x, int64_t ldx, const T *w, const float *bias, int N, int K,
                                                               const int32_t *row_of, int rows, const int32_t *run_ptr, const int4 *runs, int compact,
                                                               const float *low, int R, const T *up, T *out, int64_t ldo, int tiles_n, int gcols)
{
    typedef ProjectCfg<WM, TM, TN> Cfg;
    typedef typename Frag<T>::type F;
    constexpr int BM = Cfg::BM, BN = Cfg::BN;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / Cfg::WN, wn = wave % Cfg::WN;
    const bool second = wave >= 4;  // the group that multiplies in the other's memory phases

    const int n_tiles = ((rows + BM - 1) / BM) * tiles_n, tiles_m = n_tiles / tiles_n;
    const int per_xcd = (n_tiles + 7) >> 3, blocks_per_xcd = gridDim.x >> 3;
    auto tile_at = [&](int step, int &tm, int &tn) -> bool {
        const int in_xcd = step * blocks_per_xcd + (int)(blockIdx.x >> 3);
        const int logical = (int)(blockIdx.x & 7) * per_xcd + in_xcd;
        if (in_xcd >= per_xcd || logical >= n_tiles) return false;
        const int g = logical / (tiles_m * gcols), r = logical - g * tiles_m * gcols, cg = min(gcols, tiles_n - g * gcols);
        tm = r / cg;
        tn = g * gcols + r % cg;
        return true;
    };
    int tile_m = 0, tile_n = 0;
    if (!tile_at(0, tile_m, tile_n)) return;
    const int ksteps = project_ksteps(K), KT = ksteps >> 1;  // slabs: a multiple of 4; the host sees to it that there are 8
    const int whole = K >> 5, last_ct = (N - 1) >> 5;

    // Requests.  A: 16 rows of 64 bytes each, the lanes' pieces permuted so that piece c of row r lands at c ^ ((r >> 2) & 3).
    const int a_row = lane >> 2, a_piece = (lane & 3) ^ ((lane >> 4) & 3);
    int a_next[Cfg::A_LOADS];  // rows of the lanes' pieces in the tile after this one
    const T *p[Cfg::A_LOADS];
    auto rows_at = [&](int tm) {
#pragma unroll
        for (int i = 0; i < Cfg::A_LOADS; ++i) a_next[i] = row_of[tm * BM + (wave * Cfg::A_LOADS + i) * 16 + a_row];
    };
    auto advance = [&] {
#pragma unroll
        for (int i = 0; i < Cfg::A_LOADS; ++i) p[i] = x + (int64_t)a_next[i] * ldx + a_piece * 8;
    };
    // W: 32 columns and 16 of K each, operand order in LDS too.  Offsets behind the last column: zeros.
    constexpr int W_PIECES = BN / 16, W_LOADS = (W_PIECES + 7) / 8;
    int w_off[W_LOADS];
#pragma unroll
    for (int i = 0; i < W_LOADS; ++i) w_off[i] = lane * 16 + (wave & 1) * 1024 + ((wave >> 1) + 4 * i) * ksteps * 1024;
    auto request = [&](int tn, int slab, int stage) {
        unsigned char *to = smem + stage * Cfg::STAGE;
#pragma unroll
        for (int i = 0; i < Cfg::A_LOADS; ++i) {
            const T *from = p[i] + slab * 32;
            if (slab >= whole && slab * 32 + a_piece * 8 >= K) from = reinterpret_cast<const T *>(zero_piece);
            load_to_lds(from, to + (wave * Cfg::A_LOADS + i) * 1024);
        }
        const auto wr = buffer_of(w + (size_t)tn * (BN / 32) * ksteps * 512, min(last_ct + 1 - tn * (BN / 32), BN / 32) * ksteps * 1024);
#pragma unroll
        for (int i = 0; i < W_LOADS; ++i)
            if (i * 8 + 8 <= W_PIECES || i * 8 + wave < W_PIECES)
                load_to_lds(wr, w_off[i], slab * 2048, to + Cfg::A_BYTES + (i * 8 + wave) * 1024);
    };
    unsigned char *own = smem + 4 * Cfg::STAGE + wave * (2048 + 512), *own_bias = own + 2048;
    const auto bias_buffer = buffer_of(bias, bias ? N * 4 : 0);
    auto request_bias = [&](int tn) {
#pragma unroll
        for (int i = 0; i < TN * 32; i += 64)
            load_word_to_lds(bias_buffer, (tn * BN + wn * TN * 32 + i + lane) * 4, own_bias + i * 4);
    };

    int foff[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) foff[ks] = l32 * 64 + (((ks * 2 + half) ^ ((lane >> 2) & 3)) << 4);
    F af[2][TM], bf[2][TN];
    f32x16 acc[TM][TN];
    auto read = [&](int stage) {
        const unsigned char *at = smem + stage * Cfg::STAGE;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int ni = 0; ni < TN; ++ni)
                bf[ks][ni] = *reinterpret_cast<const F *>(at + Cfg::A_BYTES + (wn * TN + ni) * 2048 + ks * 1024 + lane * 16);
#pragma unroll
            for (int mi = 0; mi < TM; ++mi) af[ks][mi] = *reinterpret_cast<const F *>(at + (wm * TM + mi) * 2048 + foff[ks]);
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

    rows_at(tile_m);
    advance();
    request_bias(tile_n);
    request(tile_n, 0, 0);
    request(tile_n, 1, 1);
    request(tile_n, 2, 2);
    wait_memory_and_lds<2 * Cfg::LOADS>();
    barrier();
    if (second) barrier();  // a phase behind
    for (int step = 0;; ++step) {
        // without a tile after this one its first slabs are requested again (in bounds, unused)
        int next_m = tile_m, next_n = tile_n;
        const bool have_next = tile_at(step + 1, next_m, next_n);
        const int s0 = tile_m * BM + wm * TM * 32, col0 = tile_n * BN + wn * TN * 32;  // the wavefront's first slot and column
        int own_row[TM];  // of slot s0 + 32 mi + l32
        {  // slab 0: the sums start at the bias
            f32x16 start[TN];
#pragma unroll
            for (int ni = 0; ni < TN; ++ni)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 b = *reinterpret_cast<const f32x4 *>(own_bias + (ni * 32 + 8 * g + 4 * half) * 4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) start[ni][4 * g + i] = b[i];
                }
            read(0);
            request(tile_n, 3, 3);
            wait_memory_and_lds<2 * Cfg::LOADS>();
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
#pragma unroll
        for (int u = 1; u < 4; ++u) {
            read(u);
            if (u == 1) {
                rows_at(next_m);
#pragma unroll
                for (int mi = 0; mi < TM; ++mi) own_row[mi] = row_of[s0 + mi * 32 + l32];
            }
            request(tile_n, u + 3, (u + 3) & 3);
            wait_memory_and_lds<2 * Cfg::LOADS>();
            compute_phase();
        }
        for (int s = 4; s < KT - 4; s += 4) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                read(u);
                request(tile_n, s + u + 3, (u + 3) & 3);
                wait_memory_and_lds<2 * Cfg::LOADS>();
                compute_phase();
            }
        }
        request_bias(next_n);
        // The wavefront's adapters: their runs, and what the first 16 ranks of the first one need, on its way during the last slabs.
        const int groups = (rows + 31) >> 5, g0 = s0 >> 5;
        int run = __builtin_amdgcn_readfirstlane(run_ptr[min(g0, groups)]);
        const int runs_end = __builtin_amdgcn_readfirstlane(run_ptr[min(g0 + TM, groups)]);
        int from = 0, to = 0, rank = 0, k = 0;
        float scale = 0.f;
        const T *u = up;
        auto next_adapter = [&] {  // the next runs of one adapter
            const int4 r = runs[run];
            from = r.y;
            rank = r.z >> 8 & 255;
            scale = __int_as_float(r.w);
            u = up + (size_t)(compact ? (uint32_t)r.z >> 16 : (uint32_t)r.x) * N * R;
            to = r.y + (r.z & 255);
            while (++run < runs_end && runs[run].x == r.x) to += runs[run].z & 255;
            k = 0;
        };
        f32x8 h[TM];
        F uf[TN];
        auto fetch = [&] {
            const bool in = k + half * 8 < rank;
#pragma unroll
            for (int mi = 0; mi < TM; ++mi) {
                h[mi] = f32x8{};
                if (in) __builtin_memcpy(&h[mi], low + (int64_t)own_row[mi] * R + k + half * 8, sizeof(h[mi]));
            }
#pragma unroll
            for (int ni = 0; ni < TN; ++ni) {
                uf[ni] = F{};
                if (in) uf[ni] = *reinterpret_cast<const F *>(u + (size_t)min(col0 + ni * 32 + l32, N - 1) * R + k + half * 8);
            }
        };
        const bool adapted = run < runs_end;
        if (adapted) {
            next_adapter();
            fetch();
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            read(v);
            if (v == 1) advance();
            if (v == 0) request(tile_n, KT - 1, 3);
            else request(next_n, v - 1, v - 1);
            wait_memory_and_lds<2 * Cfg::LOADS>();
            compute_phase();
        }
        if (adapted)
            for (;;) {
                const int left = rank - k - half * 8;
#pragma unroll
                for (int ni = 0; ni < TN; ++ni)
#pragma unroll
                    for (int j = 1; j < 8; ++j) uf[ni][j] = j < left ? uf[ni][j] : (T)0.f;  // what lies beyond the rank may be anything
#pragma unroll
                for (int mi = 0; mi < TM; ++mi) {
                    const int slot = s0 + mi * 32;
                    if (from < slot + 32 && to > slot) {
                        f32x8 v = h[mi] * scale;
                        const bf16x8 h1 = take_piece(v), h2 = take_piece(v);
                        const bool whole_group = from <= slot && to >= slot + 32, mine = slot + l32 >= from && slot + l32 < to;
#pragma unroll
                        for (int ni = 0; ni < TN; ++ni) {
                            const f32x16 sum = adapter_step(uf[ni], h1, h2, acc[mi][ni]);
                            if (whole_group) {
                                acc[mi][ni] = sum;
                            } else {
#pragma unroll
                                for (int j = 0; j < 16; ++j) acc[mi][ni][j] = mine ? sum[j] : acc[mi][ni][j];
                            }
                        }
                    }
                }
                k += 16;
                if (k >= rank) {
                    if (run >= runs_end) break;
                    next_adapter();
                }
                fetch();
            }
        // Out: 16 rows of 64 columns at a time through the wavefront's own 2 KB (piece c of row r at c ^ (r & 7)), whole lines of 128 bytes.  96 columns: 32 at a time.
#pragma unroll
        for (int mi = 0; mi < TM; ++mi)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi)
#pragma unroll
                for (int n2 = 0; n2 < TN; n2 += 2) {
                    constexpr int PAIR = 2;
                    __builtin_amdgcn_wave_barrier();  // LDS serves a wavefront's accesses in order
                    if ((l32 >> 4) == hi) {
#pragma unroll
                        for (int c2 = 0; c2 < PAIR && n2 + c2 < TN; ++c2)
#pragma unroll
                            for (int g = 0; g < 4; ++g) {
                                typename Frag<T>::four v;
#pragma unroll
                                for (int i = 0; i < 4; ++i) v[i] = (T)acc[mi][n2 + c2][4 * g + i];
                                *reinterpret_cast<typename Frag<T>::four *>(own + (l32 & 15) * 128 + (((c2 * 4 + g) ^ (l32 & 7)) << 4) + half * 8) = v;
                            }
                    }
                    __builtin_amdgcn_wave_barrier();
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int r = j * 8 + (lane >> 3), c = lane & 7, slot = s0 + mi * 32 + hi * 16 + r, col = col0 + n2 * 32 + c * 8;
                        const u32x4 v = *reinterpret_cast<const u32x4 *>(own + r * 128 + ((c ^ (r & 7)) << 4));
                        const int row = __builtin_amdgcn_ds_bpermute((hi * 16 + r) << 2, own_row[mi]);
                        if (slot < rows && col < N && (n2 + 1 < TN || c < 4)) *reinterpret_cast<u32x4 *>(out + (int64_t)row * ldo + col) = v;
                    }
                }
        if (!have_next) break;
        tile_m = next_m;
        tile_n = next_n;
    }
    if (!second) barrier();
    wait_memory_and_lds<0>();  // nothing is on its way to LDS when the block's space becomes another's
}

}  // namespace
