// MXFP4 GEMM for gfx950, dense and grouped over experts:
//
//   C[m][n] (+)= sum over groups g of 32:  2^(sa(m,g) - 127) 2^(sb(n,g) - 127) sum_{k in g} a[m][k] b[n][k]
//
// One v_mfma_scale_f32_16x16x128_f8f6f4 takes four groups: a lane feeds 32 elements (16 bytes) of one row and the scale
// byte of their group, the matrix unit applies both scales and accumulates in FP32.  Its sums are as good as an FP32
// sum's (measured, K 128 .. 65536, scales spread over 2^12 on both sides: within 9e-8 of the sum of the magnitudes).
//
// A K-step is 128 bytes of a row, 256 elements or eight groups: lane quarter g4 of a 16-row fragment reads the 16-byte
// chunks 2 * g4 and 2 * g4 + 1, the groups of the same numbers, and the two matrix instructions take one of them each.
// Both groups' scale bytes are then neighbours, one 16-bit LDS read, and the instruction's operand select picks the byte.
#include <algorithm>
#include <type_traits>

#include "ds3_internal.h"
#include "ds3_mx4_dev.h"

namespace ds3 {

constexpr int kMaxExperts = 1023;

__device__ __forceinline__ f32x4 mfma_mx4(const i32x4& a, const i32x4& b, const f32x4& c, int sa, int sb, int half) {
    const i32x8 a8 = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, b8 = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
    if (half == 0) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, 0, sa, 0, sb);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, 1, sa, 1, sb);
}

// A workgroup takes BN = 16 FN WN weight rows by BM = 16 FM activation rows, NS stages of LDS, NS - 1 of them in
// flight; WK groups of WN waves take every WK-th K-step each and their sums meet in LDS in a fixed order.  Bound by the
// weights' stream where rows are few (16x18432x7168 12.7 us, 5.6 TB/s of weights from the memory-side cache; from HBM 14.8 us, 4.8
// TB/s), by latencies where all is small.
template <int FN_, int FM_, int WN_, int WK_, int NS_>
struct TileCfg {
    static constexpr int FN = FN_, FM = FM_, WN = WN_, WK = WK_, NS = NS_;
    static constexpr int NT = 64 * WN * WK;
    static constexpr int BN = WN * FN * 16, BM = FM * 16;
    static constexpr int ROWS = BN + BM;               // rows of one K-step's codes
    static constexpr int GROUP = ROWS * 128;           // bytes of codes per K-step
    // scale words of a K-step, two a row, in loads of 64: the weight rows', then the activation rows', shared out among the
    // waves (the last ones fetch the last 64 once more, so that every wave has the same number)
    static constexpr int LW = (2 * BN + 63) / 64, LA = (2 * BM + 63) / 64, LS = (LW + LA + WN - 1) / WN;
    static constexpr int GSTAGE = GROUP + (LW + LA) * 256;      // bytes a K-step and wave group
    static constexpr int STAGE = WK * GSTAGE;
    static constexpr int NB = 2 * FN, NA = (BM / 8 + WN - 1) / WN;      // code loads per thread and stage: weights, activations
    static constexpr int LOADS = NB + NA + LS;         // vector-memory operations per wave and stage
    static constexpr int RLD = BN + 4;                 // floats per row of the reduction buffer
    static constexpr int RED = WK * BM * RLD * 4;
    static constexpr int LDS_BYTES = (NS * STAGE > RED ? NS * STAGE : RED);
    static_assert(WN % 2 == 0 || (BM / 8) % WN != 0, "load mapping");
    static_assert(NS >= 2 && (NS - 2) * LOADS < 64, "vmcnt immediate");
    static_assert(LDS_BYTES <= 160 * 1024, "LDS");
};

template <class C, bool OUT_BF16, bool GROUPED>
__global__ __launch_bounds__(C::NT) void gemm_mxfp4_tile_kernel(const MxGemmParams p) {
    constexpr int FN = C::FN, FM = C::FM, WN = C::WN, WK = C::WK, NS = C::NS, BN = C::BN, BM = C::BM;
    __shared__ __attribute__((aligned(1024))) uint8_t smem[C::LDS_BYTES];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave % WN, wk = wave / WN;
    const int l16 = lane & 15, g4 = lane >> 4;
    const int KW = p.K >> 7, KB = (KW + 1) >> 1;       // scale words a row; K-steps (the last may be half)

    // ---- which tile: one contiguous chunk of the tile list per XCD (workgroups are dealt round robin to them),
    // row tiles innermost, so that those which share weights share an L2
    int tiles_m = p.tiles_m;                           // grouped: the host's upper bound
    [[maybe_unused]] auto group_row = [&](int g) { return max(0, min(p.group_offsets[min(g, p.G)], p.M)); };
    // rows and row tiles of the expert of a lane (kept: read again once the tile's expert is known, the offsets cost a second
    // latency, 128 rows of 32 experts, N 7168, K 2048 48.5 us instead of 47.7)
    struct Expert { int first, end, tiles; };
    [[maybe_unused]] auto tiles_before = [&](int g0, Expert& mine) -> int {    // row tiles of experts g0 .. g0 + lane
        const int g = g0 + lane;
        mine.first = group_row(g);
        mine.end = group_row(g + 1);
        mine.tiles = max(0, mine.end - mine.first + BM - 1) / BM;      // (none behind the last expert)
        int sum = mine.tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
        return sum;
    };
    [[maybe_unused]] int cum = 0;                      // of the first 64 experts, kept: most calls have no more
    [[maybe_unused]] Expert mine{};
    if constexpr (GROUPED) {
        cum = tiles_before(0, mine);
        tiles_m = __builtin_amdgcn_readlane(cum, 63);
        for (int g0 = 64; g0 < p.G; g0 += 64) {
            Expert unused;
            tiles_m += __builtin_amdgcn_readlane(tiles_before(g0, unused), 63);
        }
    }
    const int ntiles = tiles_m * p.tiles_n, per_xcd = (ntiles + 7) >> 3;
    const int local = (int)(blockIdx.x >> 3), t = (int)(blockIdx.x & 7) * per_xcd + local;
    if (local >= per_xcd || t >= ntiles) return;
    int n0, m0, m_end, grp = 0;
    if constexpr (GROUPED) {
        // the expert whose tiles [before * tiles_n, (before + its row tiles) * tiles_n) hold t
        int before = 0, g0 = 0;
        for (;;) {
            const unsigned long long past = __ballot((before + cum) * p.tiles_n > t);
            if (past != 0) {
                const int l = __builtin_ctzll(past);
                const int nt_g = __builtin_amdgcn_readlane(mine.tiles, l);
                before += __builtin_amdgcn_readlane(cum, l) - nt_g;
                grp = g0 + l;
                const int r = t - before * p.tiles_n;  // its column tiles, the row tiles innermost
                n0 = r / nt_g * BN;
                m0 = __builtin_amdgcn_readlane(mine.first, l) + r % nt_g * BM;
                m_end = __builtin_amdgcn_readlane(mine.end, l);
                break;
            }
            before += __builtin_amdgcn_readlane(cum, 63);
            g0 += 64;
            if (g0 >= p.G) return;                     // (not reached: t is below the sum over all experts)
            cum = tiles_before(g0, mine);
        }
    } else {
        n0 = t / p.tiles_m * BN; m0 = t % p.tiles_m * BM; m_end = p.M;
    }
    const int m_rows = min(m_end - m0, BM);
    const int n_rows = min(p.N - n0, BN);

    // Descriptors over the tile's valid bytes: rows beyond them move no data and read as zero.
    const int kbytes = p.K >> 1;
    const __amdgpu_buffer_rsrc_t rs_a = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(p.a + (int64_t)m0 * p.lda), 0, (int)((int64_t)(m_rows - 1) * p.lda + kbytes), 0x00020000);
    const __amdgpu_buffer_rsrc_t rs_b = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(p.b + (GROUPED ? (int64_t)grp * p.b_group_stride : 0) + (int64_t)n0 * p.ldb), 0,
        (int)((int64_t)(n_rows - 1) * p.ldb + kbytes), 0x00020000);
    // (every scale offset is valid and below 2^31: the host has checked; the expert's part is in the pointer)
    const __amdgpu_buffer_rsrc_t rs_sa = __builtin_amdgcn_make_buffer_rsrc((void*)p.sa, 0, 0x7ffffffc, 0x00020000);
    const __amdgpu_buffer_rsrc_t rs_sb = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(p.sb + (GROUPED ? (int64_t)grp * p.sb_group_stride : 0)), 0, 0x7ffffffc, 0x00020000);

    // Each group of WN waves moves the rows of its own K-step, 8 * WN per load; 16-byte chunks are
    // XOR-swizzled by row so that a fragment read spreads over the banks.
    const int lrow = wn * 8 + (lane >> 3);
    const int gchunk = (lane & 7) ^ swz_key(lrow);
    const unsigned voff_b = (unsigned)(lrow * (int)p.ldb + gchunk * 16), voff_a = (unsigned)(lrow * (int)p.lda + gchunk * 16);
    const unsigned step_b = (unsigned)(8 * WN * (int)p.ldb), step_a = (unsigned)(8 * WN * (int)p.lda);
    // (an odd number of waves: every other load's rows have the other key; where the activation rows are no whole loads of
    // all waves, the waves beyond the last eight rows move those once more, the same bytes to the same place)
    constexpr bool kOdd = WN % 2 != 0, kAgain = (BM / 8) % WN != 0;
    [[maybe_unused]] const unsigned voff_b1 = (unsigned)(lrow * (int)p.ldb + (gchunk ^ 1) * 16);
    [[maybe_unused]] int dst_a[C::NA];
    [[maybe_unused]] unsigned voff_ai[C::NA];
    if constexpr (kAgain) {
#pragma unroll
        for (int i = 0; i < C::NA; ++i) {
            const int g = min(i * WN + wn, BM / 8 - 1), row = g * 8 + (lane >> 3);
            dst_a[i] = (BN / 8 + g) * 1024;
            voff_ai[i] = (unsigned)(row * (int)p.lda + ((lane & 7) ^ swz_key(row)) * 16);
        }
    }
    // a half K-step's second half: neither operand's codes are read there (zeros: E2M1 has no value whose product with
    // zero is not zero), and the scales are those of the first half once more
    // (the keys of a thread's rows differ in their lowest bit only, which leaves a chunk in its half)
    const unsigned past_half = (KW & 1) && gchunk >= 4 ? kOobOffset : 0u;
    unsigned soff[C::LS], sstep[C::LS];
    int shalf[C::LS], sdst[C::LS];
    bool sw_side[C::LS];
#pragma unroll
    for (int i = 0; i < C::LS; ++i) {
        const int l = min(wn + i * WN, C::LW + C::LA - 1);             // wave-uniform
        sw_side[i] = l < C::LW;
        const int idx = (sw_side[i] ? l : l - C::LW) * 64 + lane, width = sw_side[i] ? BN : BM;
        shalf[i] = min(idx / width, 1);
        const int row = idx - shalf[i] * width;
        soff[i] = sw_side[i] ? (unsigned)(n0 + min(row, n_rows - 1)) * (unsigned)p.sbr * 4u : (unsigned)(m0 + min(row, m_rows - 1)) * (unsigned)p.sar * 4u;
        sstep[i] = (unsigned)(sw_side[i] ? p.sbk : p.sak) * 4u;
        sdst[i] = C::GROUP + l * 256;
    }

    uint8_t* const codes = smem + wk * C::GSTAGE;                           // + stage * STAGE
    auto issue = [&](int step, int stage) {
        const int kb = step * WK + wk;
        const unsigned koff = (kb < KB ? (unsigned)kb << 7 : kOobOffset) | (kb == KB - 1 ? past_half : 0u);
        uint8_t* const base = codes + stage * C::STAGE;
#pragma unroll
        for (int i = 0; i < C::NB + C::NA; ++i) {
            const bool is_b = i < C::NB;
            unsigned voff;
            uint8_t* at = base + wn * 1024 + i * (WN * 1024);
            if (is_b) voff = (kOdd && i % 2 ? voff_b1 : voff_b) + ((unsigned)i * step_b + koff);
            else if constexpr (kAgain) {
                voff = voff_ai[i - C::NB] + koff;
                at = base + dst_a[i - C::NB];
            } else voff = voff_a + ((unsigned)(i - C::NB) * step_a + koff);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(is_b ? rs_b : rs_a, (lds_ptr_t)at, 16, (int)voff, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < C::LS; ++i) {
            const unsigned kw = (unsigned)min(2 * kb + shalf[i], KW - 1);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(sw_side[i] ? rs_sb : rs_sa, (lds_ptr_t)(base + sdst[i]), 4, (int)(soff[i] + kw * sstep[i]), 0, 0, 0);
        }
    };
    const int key = swz_key(l16);
    const int foff0 = l16 * 128 + (((2 * g4) ^ key) << 4), foff1 = l16 * 128 + (((2 * g4 + 1) ^ key) << 4);
    // this lane's two scale bytes of a row: word g4 / 2, bytes 2 * (g4 % 2) and the next
    const int so_b = C::GROUP + ((g4 >> 1) * BN + wn * FN * 16 + l16) * 4 + (g4 & 1) * 2;
    const int so_a = C::GROUP + C::LW * 256 + ((g4 >> 1) * BM + l16) * 4 + (g4 & 1) * 2;

    // what a thread writes: four columns of a row, OUTS times; what is there already is on its way during the K-loop
    // (1536x1000x2048 added to FP32: 9.8 us, read behind it 10.7)
    constexpr int OUTS = (BM * (BN / 4) + C::NT - 1) / C::NT;
    constexpr bool MAY_ADD = !OUT_BF16 && !GROUPED;
    [[maybe_unused]] f32x4 old[OUTS];
    if constexpr (MAY_ADD) {
#pragma unroll
        for (int o = 0; o < OUTS; ++o) {
            const int idx = tid + o * C::NT, row = idx / (BN / 4), col = idx % (BN / 4) * 4;
            old[o] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (p.accumulate && row < m_rows && col + 4 <= n_rows)
                old[o] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.c) + (int64_t)(m0 + row) * p.ldc + n0 + col);
        }
    }
    const int steps = (KB + WK - 1) / WK;
#pragma unroll
    for (int s = 0; s < NS - 1; ++s) issue(s, s);
    f32x4 acc[FN][FM];
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    int stage = 0;
    for (int s = 0; s < steps; ++s) {
        // This step's loads have landed (those of the NS-2 steps behind it stay in flight), in every
        // wave once the barrier is passed; and every wave is done with the stage read before it.
        asm volatile("" ::: "memory");
        constexpr int keep = (NS - 2) * C::LOADS;
        __builtin_amdgcn_s_waitcnt((keep & 15) | ((keep >> 4) << 14) | 0x70);      // vmcnt(keep) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        const uint8_t* st = codes + stage * C::STAGE;
        // (everything that is read from LDS in this step is read before the next loads are issued: the
        // compiler makes an LDS read behind LDS-bound loads wait for them)
        i32x4 w[FN][2], x[FM][2];
        int sw[FN], sx[FM];
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            const uint8_t* f = st + (wn * FN + i) * 2048;
            w[i][0] = *reinterpret_cast<const i32x4*>(f + foff0);
            w[i][1] = *reinterpret_cast<const i32x4*>(f + foff1);
            sw[i] = *reinterpret_cast<const uint16_t*>(st + so_b + i * 64);
        }
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const uint8_t* f = st + (BN + j * 16) * 128;
            x[j][0] = *reinterpret_cast<const i32x4*>(f + foff0);
            x[j][1] = *reinterpret_cast<const i32x4*>(f + foff1);
            sx[j] = *reinterpret_cast<const uint16_t*>(st + so_a + j * 64);
        }
        __builtin_amdgcn_sched_barrier(0);
        issue(s + NS - 1, stage == 0 ? NS - 1 : stage - 1);
        __builtin_amdgcn_sched_barrier(0);
        if (s * WK + wk < KB) {
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    acc[i][j] = mfma_mx4(w[i][0], x[j][0], acc[i][j], sw[i], sx[j], 0);
                    acc[i][j] = mfma_mx4(w[i][1], x[j][1], acc[i][j], sw[i], sx[j], 1);
                }
        }
        stage = stage + 1 == NS ? 0 : stage + 1;
    }

    // ---- the groups' sums meet in LDS: [wk][row][column] ----
    __builtin_amdgcn_s_waitcnt(0x70);                  // no load is on its way into the stages any more
    __syncthreads();
    float* const red = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int j = 0; j < FM; ++j)
#pragma unroll
        for (int i = 0; i < FN; ++i)
            *reinterpret_cast<f32x4*>(red + (wk * BM + j * 16 + l16) * C::RLD + (wn * FN + i) * 16 + g4 * 4) = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int out = 0; out < OUTS; ++out) {
        const int idx = tid + out * C::NT, row = idx / (BN / 4), col = idx % (BN / 4) * 4;
        if (row >= m_rows || col >= n_rows) continue;
        f32x4 v = *reinterpret_cast<const f32x4*>(red + row * C::RLD + col);
#pragma unroll
        for (int g = 1; g < WK; ++g) {
            const f32x4 o = *reinterpret_cast<const f32x4*>(red + (g * BM + row) * C::RLD + col);
            v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        }
        const int64_t at = (int64_t)(m0 + row) * p.ldc + n0 + col;
        if constexpr (OUT_BF16) {
            uint16_t* d = static_cast<uint16_t*>(p.c) + at;
            const u32x2 o = {pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)};
            if (col + 4 <= n_rows) *reinterpret_cast<u32x2*>(d) = o;
            else for (int q = 0; col + q < n_rows; ++q) d[q] = (uint16_t)((q & 2 ? o.y : o.x) >> (16 * (q & 1)));
        } else {
            float* d = static_cast<float*>(p.c) + at;
            if (col + 4 <= n_rows) {
                if (MAY_ADD && p.accumulate) { v.x += old[out].x; v.y += old[out].y; v.z += old[out].z; v.w += old[out].w; }
                *reinterpret_cast<f32x4*>(d) = v;
            } else {
                const float o[4] = {v.x, v.y, v.z, v.w};
                for (int q = 0; col + q < n_rows; ++q) d[q] = p.accumulate ? d[q] + o[q] : o[q];
            }
        }
    }
}

// ---- the kernel for many tiles ------------------------------------------------------
// BN x BM output tiles, WN x WM waves, NS stages of LDS with loads NS - 1 K-steps ahead of the matrix instructions.
// 4096x18432x7168: 227 us back to back, 4.8 PFLOP/s (248 with casts between).  Two things bound it.  Waits: of 435 thousand
// cycles the matrix units are busy for 258 (59%; in a loop on registers 94%), waves wait for data and barriers for 31% of their
// cycles, to issue for 35%.  Power: random codes run at 1.89 GHz; codes of one value at 2.38, 180 us, in as many cycles.
// Grouped 256x128 tiles, 8192 rows of 32 experts, N 4096, K 7168: 167 us, 365 thousand cycles at 2.18 GHz, busy for 129 (35%).
template <int BN_, int BM_, int WN_, int WM_, int NS_>
struct MainCfg {
    static constexpr int BN = BN_, BM = BM_, WN = WN_, WM = WM_, NS = NS_;
    static constexpr int NT = 64 * WN * WM;
    static constexpr int TN = BN / WN, TM = BM / WM;   // wave tile
    static constexpr int FN = TN / 16, FM = TM / 16, NSUB = FN * FM;
    static constexpr int ROWS = BN + BM;
    static constexpr int STAGE = ROWS * 128;           // bytes of codes per K-step
    static constexpr int RPI = NT / 8;                 // tile rows one load instruction of the workgroup covers
    static constexpr int LPT = ROWS / RPI;             // 16-byte loads per thread per K-step
    static constexpr int TAILN = LPT < FN ? LPT : FN;  // of them issued right behind the barrier that frees their stage
    static constexpr int HEADN = LPT - TAILN;          // and at the head of the next K-step
    static constexpr int SROW = ROWS + 16;             // words between the two words of a row's scales (other banks)
    static constexpr int SSTAGE = 2 * SROW * 4;        // bytes of scales per K-step
    static constexpr int LDS_BYTES = NS * (STAGE + SSTAGE) + (kMaxExperts + 1) * 4;
    static constexpr int WG_PER_CU = NT > 256 || LDS_BYTES > 80 * 1024 ? 1 : 2;
    static_assert(BN % RPI == 0 && BM % RPI == 0 && RPI % 16 == 0, "load mapping");
    static_assert(BN % 64 == 0 && BM % 64 == 0 && ROWS <= NT, "a thread fetches one row's scales, a wave those of one side");
    static_assert(FM % 2 == 0 && HEADN <= NSUB - FN && LPT <= 2 * FN, "loads are interleaved with the matrix instructions");
    static_assert((NT / 64) * 16 * (TN * 4 + 16) <= STAGE, "epilogue strips take the last stage");
    static_assert(LDS_BYTES <= 160 * 1024, "LDS");
};

struct MxTile {
    int m0, n0, m_rows, n_rows;
    __amdgpu_buffer_rsrc_t rs_a, rs_b, rs_s;
    unsigned s_off;            // byte offset of the row of scales this thread fetches from
};

// Persistent workgroups; XCD x (workgroups are dealt to the eight of them in turn) walks its eighth of the tile list.  The
// K-step's order of instructions is pinned: the matrix instructions of all sub-tiles but the last activation fragment's,
// ONE barrier (the next stage is complete, this one is read), then behind it the loads that refill this stage and the
// next K-step's first fragments, under the last fragment's matrix instructions.
template <class C, bool OUT_BF16, bool GROUPED>
__global__ __launch_bounds__(C::NT) void gemm_mxfp4_kernel(const MxGemmParams p) {
    constexpr int BN = C::BN, BM = C::BM, NT = C::NT, NS = C::NS, FN = C::FN, FM = C::FM, STAGE = C::STAGE;
    // The way out: PASSES times 64 lanes x 16 bytes are 16 rows x TN columns, through an LDS strip a wave in the last stage.
    constexpr int ESZ = OUT_BF16 ? 2 : 4, SEG = C::TN * ESZ, ROWB = SEG + 16, CPR = SEG / 16, PASSES = 16 * CPR / 64, STORES = FM * PASSES;
    static_assert(16 * CPR % 64 == 0, "epilogue mapping");
    __shared__ __attribute__((aligned(1024))) uint8_t smem[C::LDS_BYTES];
    uint8_t* const scales = smem + NS * STAGE;
    int* const before = reinterpret_cast<int*>(scales + NS * C::SSTAGE);       // [G + 1] row tiles before expert g

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave % C::WN, wm = wave / C::WN;
    const int l16 = lane & 15, g4 = lane >> 4;
    const int KW = p.K >> 7, KB = (KW + 1) >> 1;       // scale words a row; K-steps (the last may be half)

    // ---- tile walk -------------------------------------------------------------------
    int tiles_m = p.tiles_m;
    if constexpr (GROUPED) {
        auto row_of = [&](int g) { return max(0, min(p.group_offsets[g], p.M)); };
        if (wave == 0) {
            int cum = 0;
            for (int g0 = 0; g0 < p.G; g0 += 64) {
                const int g = g0 + lane;
                int sum = g < p.G ? max(0, row_of(g + 1) - row_of(g) + BM - 1) / BM : 0;
                const int mine = sum;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int o = __shfl_up(sum, d);
                    if (lane >= d) sum += o;
                }
                if (g < p.G) before[g] = cum + sum - mine;
                cum += __builtin_amdgcn_readlane(sum, 63);
            }
            if (lane == 0) before[p.G] = cum;
        }
        __syncthreads();
        tiles_m = before[p.G];
    }
    const int ntiles = tiles_m * p.tiles_n;
    const int per_xcd = (ntiles + 7) >> 3;
    const int xcd = (int)(blockIdx.x & 7), slot = (int)(blockIdx.x >> 3), nslots = (int)(gridDim.x >> 3);
    const int mine = max(0, min(per_xcd, ntiles - xcd * per_xcd));     // tiles of this XCD
    const int rounds = mine / nslots, tail = mine - rounds * nslots;
    // What is left after the last full round: at most half as many tiles as workgroups are cut into halves of BM / 2
    // rows, whose other half's waves issue no matrix instruction (a half takes .55 of a tile's time).
    const bool halves = !GROUPED && C::WM == 2 && rounds > 0 && tail > 0 && 2 * tail <= nslots && p.M % BM == 0;
    const int units = rounds + (halves ? (slot < 2 * tail ? 1 : 0) : (slot < tail ? 1 : 0));

    const int kbytes = p.K >> 1;
    auto setup = [&](int u, MxTile& c) -> bool {
        if (u >= units) return false;
        int local = u * nslots + slot, half = -1;
        if (halves && u == rounds) { half = slot & 1; local = rounds * nslots + (slot >> 1); }
        const int t = xcd * per_xcd + local;
        int m0, m_end, n0, grp = 0;
        if constexpr (!GROUPED) {
            constexpr int PM = 4;                      // row tiles of a panel: the tiles side by side share operands
            const int panel = PM * p.tiles_n;
            const int pi = t / panel, r = t - pi * panel;
            const int pm = min(PM, tiles_m - pi * PM);
            m0 = (pi * PM + r % pm) * BM;
            n0 = (r / pm) * BN;
            m_end = p.M;
            if (half >= 0) { m0 += half * (BM / 2); m_end = min(m_end, m0 + BM / 2); }
        } else {
            // expert by expert, then by column tile, the expert's row tiles innermost: side by side they share weights
            int lo = 0, hi = p.G;                      // largest g with before[g] * tiles_n <= t
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (before[mid] * p.tiles_n <= t) lo = mid; else hi = mid;
            }
            grp = lo;
            const int nt_g = before[grp + 1] - before[grp];
            const int r = t - before[grp] * p.tiles_n;
            n0 = (r / nt_g) * BN;
            m0 = max(0, min(p.group_offsets[grp], p.M)) + (r % nt_g) * BM;
            m_end = max(0, min(p.group_offsets[grp + 1], p.M));
            // uniform, but read through vector registers: said so here, the descriptors live in scalar registers
            grp = __builtin_amdgcn_readfirstlane(grp);
            n0 = __builtin_amdgcn_readfirstlane(n0);
            m0 = __builtin_amdgcn_readfirstlane(m0);
            m_end = __builtin_amdgcn_readfirstlane(m_end);
        }
        c.m0 = m0; c.n0 = n0;
        c.m_rows = min(m_end - m0, BM);
        c.n_rows = min(p.N - n0, BN);
        // Descriptors over the tile's valid bytes: rows beyond them read as zero and touch no memory.
        c.rs_a = __builtin_amdgcn_make_buffer_rsrc((void*)(p.a + (int64_t)m0 * p.lda), 0, (int)((int64_t)(c.m_rows - 1) * p.lda + kbytes), 0x00020000);
        c.rs_b = __builtin_amdgcn_make_buffer_rsrc((void*)(p.b + (int64_t)grp * p.b_group_stride + (int64_t)n0 * p.ldb), 0,
                                                   (int)((int64_t)(c.n_rows - 1) * p.ldb + kbytes), 0x00020000);
        // Thread t fetches the scales of tile row t, weight rows first (rows past the valid ones repeat the last; all
        // offsets are valid, the range check is not relied on).
        const bool w_side = wave * 64 < BN;
        c.rs_s = __builtin_amdgcn_make_buffer_rsrc((void*)(w_side ? p.sb + (int64_t)grp * p.sb_group_stride : p.sa), 0, 0x7ffffffc, 0x00020000);
        c.s_off = w_side ? (unsigned)(n0 + min(tid, c.n_rows - 1)) * (unsigned)p.sbr * 4u
                         : (unsigned)(m0 + min(max(tid - BN, 0), c.m_rows - 1)) * (unsigned)p.sar * 4u;
        return true;
    };

    // this thread moves chunk position (tid & 7) of tile row i * RPI + (tid >> 3); 16-byte chunks are XOR-swizzled by row
    const int lrow = tid >> 3;
    const int gchunk = (tid & 7) ^ swz_key(lrow);
    const unsigned voff_b = (unsigned)(lrow * (int)p.ldb + gchunk * 16), voff_a = (unsigned)(lrow * (int)p.lda + gchunk * 16);
    const unsigned step_b = (unsigned)(C::RPI * (int)p.ldb), step_a = (unsigned)(C::RPI * (int)p.lda);
    // a half K-step's second half: neither operand's codes are read there (zeros), the scales are the first half's again
    const unsigned past_half = (KW & 1) && gchunk >= 4 ? kOobOffset : 0u;
    const int key = swz_key(l16);
    const int foff0 = l16 * 128 + (((2 * g4) ^ key) << 4), foff1 = l16 * 128 + (((2 * g4 + 1) ^ key) << 4);
    const int p_base = wn * C::TN * 128, q_base = (BN + wm * C::TM) * 128;
    // this lane's two scale bytes: word g4 / 2 of its row, bytes 2 * (g4 % 2) and the next
    const int so = (g4 >> 1) * (C::SROW * 4) + (g4 & 1) * 2 + l16 * 4;
    const int ps_base = so + wn * C::TN * 4, qs_base = so + (BN + wm * C::TM) * 4;
    const bool scale_role = wave * 64 < C::ROWS;
    // (in a vector register: as a scalar it would be re-read from the kernel arguments inside the K-loop)
    unsigned sc_kstride = (unsigned)(wave * 64 < BN ? (int)p.sbk : (int)p.sak) * 4u;
    asm volatile("" : "+v"(sc_kstride));

    // byte offset of K-step kb for this thread's loads (out of range beyond the last)
    auto koff_of = [&](int kb) -> unsigned {
        const unsigned o = kb < KB ? (unsigned)kb << 7 : kOobOffset;
        return kb == KB - 1 ? o | past_half : o;
    };
    auto issue_load = [&](const MxTile& c, int i, int stage, unsigned koff) {
        const bool is_b = i * C::RPI < BN;
        const int ii = is_b ? i : i - BN / C::RPI;
        unsigned uoff = (unsigned)ii * (is_b ? step_b : step_a);
        asm volatile("" : "+s"(uoff));                 // (summed in a scalar register, added last)
        const unsigned voff = (is_b ? voff_b : voff_a) + uoff + koff;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(is_b ? c.rs_b : c.rs_a, (lds_ptr_t)(smem + stage * STAGE + (i * NT + wave * 64) * 16), 16,
                                                 (int)voff, 0, 0, 0);
    };
    auto issue_scales = [&](const MxTile& c, int kb, int stage) {
        if (!scale_role) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned kw = (unsigned)min(2 * kb + h, KW - 1);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(c.rs_s, (lds_ptr_t)(scales + stage * C::SSTAGE + (h * C::SROW + wave * 64) * 4), 4,
                                                     (int)(c.s_off + kw * sc_kstride), 0, 0, 0);
        }
    };
    struct Frag { i32x4 h0, h1; };
    auto load_frag = [&](const uint8_t* base) -> Frag {
        return Frag{*reinterpret_cast<const i32x4*>(base + foff0), *reinterpret_cast<const i32x4*>(base + foff1)};
    };
    auto read_scale = [&](int stage, int at) -> int { return *reinterpret_cast<const uint16_t*>(scales + stage * C::SSTAGE + at); };
    // Barrier that lets the newest `keep` vector-memory operations of this wave stay in flight.
    auto barrier_keep = [&](auto keep_tag) {
        constexpr int keep = decltype(keep_tag)::value;
        static_assert(keep >= 0 && keep < 64, "vmcnt immediate");
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((keep & 15) | ((keep >> 4) << 14) | 0x70);      // vmcnt(keep) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto kstep_barrier = [&]() {
        if constexpr (NS == 2) barrier_keep(std::integral_constant<int, 0>{});
        else if (scale_role) barrier_keep(std::integral_constant<int, C::LPT + 2>{});
        else barrier_keep(std::integral_constant<int, C::LPT>{});
    };
    auto issue_first_steps = [&](const MxTile& c) {
#pragma unroll
        for (int ks = 0; ks < NS - 1; ++ks) {
            const unsigned koff = koff_of(ks);
#pragma unroll
            for (int i = 0; i < C::LPT; ++i) issue_load(c, i, ks, koff);
            issue_scales(c, ks, ks);
        }
    };

    // Barrier that lets the newest `steps` K-steps' loads stay in flight, and the previous tile's stores with them: those are
    // waited for only where data asked for behind them is needed (vector-memory operations end in order).  us without / with
    // it: 4096x18432x7168 256 / 251, FP32 4096x16384x7168 254 / 243, added to what was there 308 / 314, 7168x7168x4096 added
    // 174 / 166.  Strips outside the stages, so that two K-steps run before the stores have to be done, need an own form of
    // the first K-step, whose registers spill: 264.
    bool flying = false;                               // whether this wave has issued STORES stores behind the first loads
    auto barrier_flying = [&](auto steps_tag) {
        constexpr int steps = decltype(steps_tag)::value, few = steps * C::LPT, many = steps * (C::LPT + 2);
        if (scale_role) {
            if (flying) barrier_keep(std::integral_constant<int, many + STORES>{});
            else barrier_keep(std::integral_constant<int, many>{});
        } else {
            if (flying) barrier_keep(std::integral_constant<int, few + STORES>{});
            else barrier_keep(std::integral_constant<int, few>{});
        }
    };

    MxTile cur;
    int unit = 0;
    if (!setup(unit, cur)) return;
    issue_first_steps(cur);
    for (;;) {
        // ---- K-steps 0 .. NS-2 of `cur` are in flight into stages 0 .. NS-2, and behind them the stores ----
        barrier_flying(std::integral_constant<int, NS - 2>{});
        {
            const unsigned koff = koff_of(NS - 1);
#pragma unroll
            for (int i = 0; i < C::TAILN; ++i) issue_load(cur, i, NS - 1, koff);
            issue_scales(cur, NS - 1, NS - 1);
        }
        Frag pf[FN], qf[2];
        int ps[FN], qs[2];
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            pf[i] = load_frag(smem + p_base + i * 2048);
            ps[i] = read_scale(0, ps_base + i * 64);
        }
        qf[0] = load_frag(smem + q_base);
        qs[0] = read_scale(0, qs_base);
        f32x4 acc[FN][FM];
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

        auto kstep = [&](int kb, auto stage_tag, auto first_tag) {
            constexpr bool FIRST = decltype(first_tag)::value;         // the stores may be in flight behind what its barrier waits for
            constexpr int S = decltype(stage_tag)::value, SN = (S + 1) % NS, SL = (S + NS - 1) % NS;
            const uint8_t* st = smem + S * STAGE;
            const uint8_t* nst = smem + SN * STAGE;
            const unsigned koff1 = koff_of(kb + NS - 1), koff2 = koff_of(kb + NS);
            __builtin_amdgcn_sched_barrier(0);
            // activation fragment j, weight fragment i, half h (four of the eight groups).  An accumulator's two matrix
            // instructions follow each other: FN apart, so that neither would wait for the other, 4096x18432x7168 takes
            // 263 us instead of 255.
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                if (j == FM - 1) {
                    if constexpr (FIRST) barrier_flying(std::integral_constant<int, NS - 2>{});
                    else kstep_barrier();
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int i = 0; i < FN; ++i) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int s = (j * 2 + h) * FN + i;
                        if (s < C::HEADN) issue_load(cur, C::TAILN + s, SL, koff1);
                        if (h == 0 && i == 0 && j + 1 < FM) {
                            qf[(j + 1) & 1] = load_frag(st + q_base + (j + 1) * 2048);
                            qs[(j + 1) & 1] = read_scale(S, qs_base + (j + 1) * 64);
                        }
                        acc[i][j] = mfma_mx4(h ? pf[i].h1 : pf[i].h0, h ? qf[j & 1].h1 : qf[j & 1].h0, acc[i][j], ps[i], qs[j & 1], h);
                        // (ties it to this point of the K-step)
                        asm volatile("" : "+v"(acc[i][j]));
                        if (j == FM - 1 && h == 1) {
                            pf[i] = load_frag(nst + p_base + i * 2048);
                            ps[i] = read_scale(SN, ps_base + i * 64);
#pragma unroll
                            for (int l = i; l < C::TAILN; l += FN) issue_load(cur, l, S, koff2);
                            if (i == 0) issue_scales(cur, kb + NS, S);
                            if (i == FN - 1) {
                                qf[0] = load_frag(nst + q_base);
                                qs[0] = read_scale(SN, qs_base);
                            }
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        };
        // The same for a wave whose rows all lie beyond the tile's: it moves its share of the data, in the same order.
        auto kstep_idle = [&](int kb, auto stage_tag, auto first_tag) {
            constexpr bool FIRST = decltype(first_tag)::value;
            constexpr int S = decltype(stage_tag)::value, SL = (S + NS - 1) % NS;
            const unsigned koff1 = koff_of(kb + NS - 1), koff2 = koff_of(kb + NS);
#pragma unroll
            for (int i = 0; i < C::HEADN; ++i) issue_load(cur, C::TAILN + i, SL, koff1);
            if constexpr (FIRST) barrier_flying(std::integral_constant<int, NS - 2>{});
            else kstep_barrier();
            issue_load(cur, 0, S, koff2);
            issue_scales(cur, kb + NS, S);
#pragma unroll
            for (int i = 1; i < C::TAILN; ++i) issue_load(cur, i, S, koff2);
        };
        using st0 = std::integral_constant<int, 0>;
        using st1 = std::integral_constant<int, 1>;
        using st2 = std::integral_constant<int, 2>;
        const bool active = wm * C::TM < cur.m_rows;    // wave-uniform
        auto kloop = [&](auto step) {
            std::false_type other;
            int kb = 0;
            if constexpr (NS == 2) {
                for (; kb + 1 < KB; kb += 2) {
                    step(kb, st0{}, other);
                    step(kb + 1, st1{}, other);
                }
                if (kb < KB) step(kb, st0{}, other);
            } else {
                step(kb++, st0{}, std::true_type{});
                for (; kb + 2 < KB; kb += 3) {
                    step(kb, st1{}, other);
                    step(kb + 1, st2{}, other);
                    step(kb + 2, st0{}, other);
                }
                if (kb < KB) step(kb, st1{}, other);
                if (kb + 1 < KB) step(kb + 1, st2{}, other);
            }
        };
        if (active) kloop(kstep);
        else kloop(kstep_idle);
        __builtin_amdgcn_s_waitcnt(0x70);              // nothing is on its way into the stages any more
        __syncthreads();                               // every wave is done with all of them

        // ---- the next tile's first K-steps fly into their stages during this one's way out ----
        MxTile nxt;
        ++unit;
        const bool more = setup(unit, nxt);
        if (more) issue_first_steps(nxt);
        asm volatile("" ::: "memory");                 // (the stores are counted on to be behind these loads)
        __builtin_amdgcn_sched_barrier(0);
        // A lane owns one activation row and, per weight fragment, four consecutive columns: each wave turns 16 rows x
        // TN columns at a time through its LDS strip, so that stores are 16 bytes a lane and whole 128- or 256-byte row
        // segments (64-byte ones straight from the registers: 257 -> 271 us with non-temporal stores, 264 with plain ones).
        // (every address here derives from this copy of the thread index, which the compiler cannot see through: none is
        // computed before the K-loop and kept in a register across it)
        int tid_e = threadIdx.x;
        asm volatile("" : "+v"(tid_e));
        const int lane = tid_e & 63, l16 = tid_e & 15, g4 = (tid_e >> 4) & 3;
        uint8_t* strip = smem + (NS - 1) * STAGE + wave * (16 * ROWB);
        uint64_t c_bits = reinterpret_cast<uint64_t>(p.c);
        int64_t ldc = p.ldc;
        asm volatile("" : "+s"(c_bits), "+s"(ldc));    // (registers of their own: not re-read in front of every store)
        uint8_t* c_base = (uint8_t*)(__attribute__((address_space(1))) uint8_t*)c_bits;
        // FULL: all of the wave's rows and columns are the tile's, so it issues exactly STORES stores.  (ADD, what was there
        // is added to, is settled outside: behind a branch inside, every store would wait for loads.)
        auto way_out = [&](auto full_tag, auto add_tag) {
            constexpr bool FULL = decltype(full_tag)::value, ADD = decltype(add_tag)::value;
            // of how many 16 rows the old values are fetched at once: of all (2048x2048x4096 22.0 -> 20.1 us), or, beside the sums of a
            // 128x64 wave tile, of one (of two the registers spill: 332 -> 355)
            constexpr int OLD = C::NSUB <= 16 ? FM : 1;
            [[maybe_unused]] f32x4 old[OLD][PASSES];
            [[maybe_unused]] auto fetch_old = [&](int j, f32x4* into) {
#pragma unroll
                for (int ps_ = 0; ps_ < PASSES; ++ps_) {
                    const int idx = ps_ * 64 + lane, ml = wm * C::TM + j * 16 + idx / CPR, nl = wn * C::TN + (idx % CPR) * 4;
                    into[ps_] = f32x4{0.f, 0.f, 0.f, 0.f};
                    if (FULL || (ml < cur.m_rows && nl + 4 <= cur.n_rows))
                        into[ps_] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(c_base + ((int64_t)(cur.m0 + ml) * ldc + cur.n0 + nl) * 4));
                }
            };
            if constexpr (ADD && OLD > 1) {
#pragma unroll
                for (int j = 0; j < FM; ++j) fetch_old(j, old[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                if constexpr (ADD && OLD == 1) fetch_old(j, old[0]);
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    const f32x4 v = acc[i][j];
                    uint8_t* dst = strip + l16 * ROWB + (i * 16 + g4 * 4) * ESZ;
                    if constexpr (OUT_BF16) *reinterpret_cast<u32x2*>(dst) = u32x2{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)};
                    else *reinterpret_cast<f32x4*>(dst) = v;
                }
                __builtin_amdgcn_wave_barrier();       // same-wave LDS accesses complete in order
                u32x4 wv[PASSES];
#pragma unroll
                for (int ps_ = 0; ps_ < PASSES; ++ps_) {
                    const int idx = ps_ * 64 + lane;
                    wv[ps_] = *reinterpret_cast<const u32x4*>(strip + (idx / CPR) * ROWB + (idx % CPR) * 16);
                }
#pragma unroll
                for (int ps_ = 0; ps_ < PASSES; ++ps_) {
                    const int idx = ps_ * 64 + lane;
                    const int ml = wm * C::TM + j * 16 + idx / CPR, nl = wn * C::TN + (idx % CPR) * (16 / ESZ);
                    if (!FULL && (ml >= cur.m_rows || nl >= cur.n_rows)) continue;
                    uint8_t* gp = c_base + ((int64_t)(cur.m0 + ml) * ldc + cur.n0 + nl) * ESZ;
                    const u32x4 w = wv[ps_];
                    if (FULL || nl + 16 / ESZ <= cur.n_rows) {
                        if constexpr (OUT_BF16) {
                            __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(gp));
                        } else {
                            f32x4 o = f32x4{as_f32(w.x), as_f32(w.y), as_f32(w.z), as_f32(w.w)};
                            if constexpr (ADD) { const f32x4 v = old[j % OLD][ps_]; o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w; }
                            __builtin_nontemporal_store(o, reinterpret_cast<f32x4*>(gp));
                        }
                    } else {
                        const unsigned int wd[4] = {w.x, w.y, w.z, w.w};
                        for (int q = 0; q < 16 / ESZ && nl + q < cur.n_rows; ++q) {
                            if constexpr (OUT_BF16) {
                                reinterpret_cast<uint16_t*>(gp)[q] = (uint16_t)(wd[q >> 1] >> (16 * (q & 1)));
                            } else {
                                float* d = reinterpret_cast<float*>(gp) + q;
                                *d = ADD ? *d + as_f32(wd[q]) : as_f32(wd[q]);
                            }
                        }
                    }
                }
                __builtin_amdgcn_wave_barrier();       // the strip is read before the next rows replace it
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        flying = (wm + 1) * C::TM <= cur.m_rows && (wn + 1) * C::TN <= cur.n_rows;
        auto leave = [&](auto full_tag) {
            if constexpr (!OUT_BF16 && !GROUPED) {
                if (p.accumulate) return way_out(full_tag, std::true_type{});
            }
            way_out(full_tag, std::false_type{});
        };
        if (flying) {
            leave(std::true_type{});
        } else {
            if (active) leave(std::false_type{});
            __builtin_amdgcn_s_waitcnt(0xf70);         // (unknown how many: none flies on.  vmcnt(0))
        }
        if (!more) break;
        cur = nxt;
    }
}

// ---- host side -------------------------------------------------------------------
// Row tiles of a grouped call, an upper bound (a row tile has a row).
static int64_t most_row_tiles(int G, int M, int bm) { return std::min<int64_t>(((int64_t)M + bm - 1) / bm + G, M); }

template <class C, bool GROUPED>
static ds3_status launch_tile(MxGemmParams p, ds3_dtype ct, hipStream_t st) {
    p.tiles_m = (p.M + C::BM - 1) / C::BM;
    // (workgroups beyond the true count leave at once)
    if (GROUPED) p.tiles_m = (int)most_row_tiles(p.G, p.M, C::BM);
    p.tiles_n = (p.N + C::BN - 1) / C::BN;
    const int64_t n = ((int64_t)p.tiles_m * p.tiles_n + 7) / 8 * 8;
    if (n * C::NT >= (1ll << 32)) return DS3_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)n), block(C::NT);
    (void)hipGetLastError();                            // a stale error of earlier, unrelated work is not this launch's
    if (ct == DS3_BF16) gemm_mxfp4_tile_kernel<C, true, GROUPED><<<grid, block, 0, st>>>(p);
    else gemm_mxfp4_tile_kernel<C, false, GROUPED><<<grid, block, 0, st>>>(p);
    return hipGetLastError() == hipSuccess ? DS3_OK : DS3_ERR_LAUNCH;
}

// Compute units of the current device, a multiple of 8.
static int compute_units_x8() {
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 8) return 256;
    return n / 8 * 8;
}

template <class C, bool GROUPED>
static ds3_status launch_main(MxGemmParams p, ds3_dtype ct, int cus, hipStream_t st) {
    p.tiles_m = (p.M + C::BM - 1) / C::BM;
    if (GROUPED) p.tiles_m = (int)most_row_tiles(p.G, p.M, C::BM);
    p.tiles_n = (p.N + C::BN - 1) / C::BN;
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n, want = (tiles + 7) / 8 * 8, slots = (int64_t)cus * C::WG_PER_CU;
    if (tiles > (1ll << 31) - 16) return DS3_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)std::min(want, slots)), block(C::NT);
    (void)hipGetLastError();                            // a stale error of earlier, unrelated work is not this launch's
    if (ct == DS3_BF16) gemm_mxfp4_kernel<C, true, GROUPED><<<grid, block, 0, st>>>(p);
    else gemm_mxfp4_kernel<C, false, GROUPED><<<grid, block, 0, st>>>(p);
    return hipGetLastError() == hipSuccess ? DS3_OK : DS3_ERR_LAUNCH;
}

// The configurations and what a call takes with each: `fixed` + one round of tiles after another, a round being K-steps
// (of 256) / `wk` steps of `full` us when every workgroup slot has a tile and `alone` us when few have, plus the sums' way
// out.  Fitted to 9000 shapes with BF16 output (M 1 .. 4096, N 64 .. 24576, K 128 .. 18432, weights from HBM), before a tile's
// stores flew on under the next one.  With the kernels as they are the one it picks takes, on 12600 other shapes, 1.015 of the
// best of these eight's time on average with BF16 output, 1.016 with FP32 (one call in twenty more than 1.1), and 1.030 where the
// sums are added to what is there, which costs more than `out` says: 1.07 above 20 us, there one call in four more than 1.1.
struct MxChoice { int bn, bm, wk, per_cu; float fixed, full, alone, out; };
enum { kMx32x32, kMx64x32, kMx80x32, kMx96x32, kMx64x64two, kMx64x64, kMx128x128, kMx256x256, kMxCfgs };
constexpr MxChoice kMx[kMxCfgs] = {
    {32, 32, 4, 1, 2.80f, 0.496f, 0.259f, 1.04f},   {64, 32, 2, 2, 2.69f, 0.660f, 0.244f, 1.38f},
    {80, 32, 2, 1, 2.50f, 0.487f, 0.321f, 1.59f},   {96, 32, 2, 1, 2.49f, 0.520f, 0.340f, 1.55f},
    {64, 64, 2, 1, 2.35f, 0.580f, 0.410f, 1.62f},   {64, 64, 1, 2, 2.23f, 0.488f, 0.246f, 1.84f},
    {128, 128, 1, 2, 1.87f, 1.210f, 0.417f, 2.62f}, {256, 256, 1, 1, 0.00f, 2.017f, 0.798f, 5.64f},
};
static double mx_time(const MxChoice& c, int64_t tiles_m, int N, int K, int cus) {
    const int64_t tiles = tiles_m * ((N + c.bn - 1) / c.bn), slots = (int64_t)cus * c.per_cu, rest = tiles % slots;
    const double steps = ((K + 255) / 256 + c.wk - 1) / c.wk, part = (double)rest / (double)slots;
    double us = c.fixed + (double)(tiles / slots) * (steps * c.full + c.out);
    if (rest) us += steps * (c.alone + (c.full - c.alone) * part) + c.out;
    return us;
}
static int mx_dense_choice(int M, int N, int K, int cus) {
    int best = kMx256x256;
    double best_us = 0.;
    for (int i = kMxCfgs - 1; i >= 0; --i) {
        const MxChoice& c = kMx[i];
        if (c.wk > (K + 255) / 256) continue;          // (groups of waves without a K-step)
        const int64_t tiles_m = (M + c.bm - 1) / c.bm;
        // (a grid of a workgroup a tile: far beyond where these are the fastest)
        if (i < kMx128x128 && tiles_m * ((N + c.bn - 1) / c.bn) > (1 << 20)) continue;
        const double us = mx_time(c, tiles_m, N, K, cus);
        if (i == kMx256x256 || us < best_us) { best = i; best_us = us; }
    }
    return best;
}

// Grouped: by the rows that there is room for, an expert's mean (the host knows no more, the offsets are on the device).  Room
// for all the rows / eight times as many, us: 32 experts, N 7168, K 2048, 128 rows 46.8 / 47.7, 512 rows 49.9 / 63.7; N 4096,
// K 7168, 8192 rows 177 / 171.  Weights from HBM, us with 64x32 / 128x64 / 128x128 /
// 256x128 / 256x256 tiles: 32 experts of 4 rows, N 7168, K 2048 46 / 49 / - / - / -; of 32, N 4096, K 7168 113 / 93 / - / - /
// -; of 64 - / 122 / 97 / 94 / 106; of 128 - / 158 / 148 / 137 / 119; of 256 - / 236 / 194 / 174 / 172; 8 experts of 512 - /
// 111 / 101 / 92 / 98; N 7168, K 2048, 32 experts of 64 - / 68 / 59 / 61 / 68, of 256 - / 158 / 124 / 114 / 111.
// Few tiles (8 experts of 128 rows, N 2048, K 1024): 64x64 9.2, 128x128 7.6, 256x256 11.4.
enum { kMxG64x32, kMxG128x64, kMxG64x64, kMxG128x128, kMxG256x128, kMxG256x256 };
static int mx_grouped_choice(int G, int M, int N, int K, int cus) {
    const int64_t mean = ((int64_t)M + G - 1) / G;
    // (few rows take a workgroup of 256 threads a tile; so many columns that a grid does not hold those go on to larger
    // tiles, in the end to the workgroups that walk)
    auto fits = [&](int bn, int bm) { return most_row_tiles(G, M, bm) * (((int64_t)N + bn - 1) / bn) <= (1 << 24) - 8; };
    if (mean <= 24 && fits(64, 32)) return kMxG64x32;
    if (mean <= 48 && fits(128, 64)) return kMxG128x64;
    const int most = mean > 96 && mean <= 256 ? kMxG256x256 : kMxG256x128;
    auto tiles_m = [&](int bm) { return (int64_t)M / bm + (G + 1) / 2; };      // (half a tile an expert is lost on average)
    if (tiles_m(most == kMxG256x256 ? 256 : 128) * ((N + 255) / 256) * 4 >= 3 * (int64_t)cus) return most;
    const double t64 = mx_time(kMx[kMx64x64], tiles_m(64), N, K, cus), t128 = mx_time(kMx[kMx128x128], tiles_m(128), N, K, cus);
    return t64 < t128 ? kMxG64x64 : kMxG128x128;
}

int gemm_mxfp4_config(int G, int M, int N, int K, int cus) {
    return G > 0 ? kMxCfgs + mx_grouped_choice(G, M, N, K, cus) : mx_dense_choice(M, N, K, cus);
}

ds3_status launch_gemm_mxfp4(const MxGemmParams& p, ds3_dtype ct, hipStream_t st) {
    // 32-bit offsets inside a tile of up to 256 rows
    if ((int64_t)257 * p.ldb + p.K / 2 >= (1ll << 31) || (int64_t)257 * p.lda + p.K / 2 >= (1ll << 31)) return DS3_ERR_UNSUPPORTED;
    const int cus = compute_units_x8();
    if (p.G > 0) {
        switch (mx_grouped_choice(p.G, p.M, p.N, p.K, cus)) {
            case kMxG64x32: return launch_tile<TileCfg<1, 2, 4, 1, 3>, true>(p, ct, st);
            case kMxG128x64: return launch_tile<TileCfg<2, 4, 4, 1, 3>, true>(p, ct, st);
            case kMxG64x64: return launch_tile<TileCfg<1, 4, 4, 1, 4>, true>(p, ct, st);
            case kMxG128x128: return launch_main<MainCfg<128, 128, 2, 2, 2>, true>(p, ct, cus, st);
            case kMxG256x128: return launch_main<MainCfg<256, 128, 4, 2, 3>, true>(p, ct, cus, st);
            default: return launch_main<MainCfg<256, 256, 4, 2, 2>, true>(p, ct, cus, st);
        }
    }
    switch (mx_dense_choice(p.M, p.N, p.K, cus)) {
        case kMx32x32: return launch_tile<TileCfg<1, 2, 2, 4, 3>, false>(p, ct, st);
        case kMx64x32: return launch_tile<TileCfg<1, 2, 4, 2, 3>, false>(p, ct, st);
        case kMx80x32: return launch_tile<TileCfg<1, 2, 5, 2, 4>, false>(p, ct, st);
        case kMx96x32: return launch_tile<TileCfg<1, 2, 6, 2, 3>, false>(p, ct, st);
        case kMx64x64two: return launch_tile<TileCfg<1, 4, 4, 2, 3>, false>(p, ct, st);
        case kMx64x64: return launch_tile<TileCfg<1, 4, 4, 1, 4>, false>(p, ct, st);
        case kMx128x128: return launch_main<MainCfg<128, 128, 2, 2, 2>, false>(p, ct, cus, st);
        default: return launch_main<MainCfg<256, 256, 4, 2, 2>, false>(p, ct, cus, st);
    }
}

}  // namespace ds3
