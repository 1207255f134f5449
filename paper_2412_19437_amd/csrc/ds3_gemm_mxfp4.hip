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

#include "ds3_internal.h"
#include "ds3_mx4_dev.h"

namespace ds3 {

__device__ __forceinline__ f32x4 mfma_mx4(const i32x4& a, const i32x4& b, const f32x4& c, int sa, int sb, int half) {
    const i32x8 a8 = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, b8 = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
    if (half == 0) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, 0, sa, 0, sb);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, 1, sa, 1, sb);
}

// A workgroup takes BN = 16 FN WN weight rows by BM = 16 FM activation rows, NS stages of LDS, NS - 1 of them in
// flight; WK groups of WN waves take every WK-th K-step each and their sums meet in LDS in a fixed order.
template <int FN_, int FM_, int WN_, int WK_, int NS_>
struct TileCfg {
    static constexpr int FN = FN_, FM = FM_, WN = WN_, WK = WK_, NS = NS_;
    static constexpr int NT = 64 * WN * WK;
    static constexpr int BN = WN * FN * 16, BM = FM * 16;
    static constexpr int ROWS = BN + BM;               // rows of one K-step's codes
    static constexpr int GROUP = ROWS * 128;           // bytes of codes per K-step
    static constexpr int NSA = (BM + 63) / 64;         // 64-row pieces of the activation scales
    static constexpr int SCALES = (NSA + 1) * 512;     // per wave and stage: two words an activation row, two a weight row
    static constexpr int STAGE = WK * GROUP + WN * WK * SCALES;
    static constexpr int NB = 2 * FN, NA = BM / 8 / WN;         // code loads per thread and stage: weights, activations
    static constexpr int LOADS = NB + NA + 2 * (NSA + 1);       // vector-memory operations per wave and stage
    static constexpr int RLD = BN + 4;                 // floats per row of the reduction buffer
    static constexpr int RED = WK * BM * RLD * 4;
    static constexpr int LDS_BYTES = (NS * STAGE > RED ? NS * STAGE : RED);
    static_assert(FN * 16 <= 64, "one weight row a lane");
    static_assert(WN % 2 == 0 && (BM / 8) % WN == 0, "load mapping");
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
    [[maybe_unused]] auto tiles_before = [&](int g0, int& mine) -> int {   // row tiles of experts g0 .. g0 + lane; `mine`: of the last of them
        const int g = g0 + lane;
        mine = g < p.G ? max(0, group_row(g + 1) - group_row(g) + BM - 1) / BM : 0;
        int sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
        return sum;
    };
    [[maybe_unused]] int cum = 0, mine = 0;            // of the first 64 experts, kept: most calls have no more
    if constexpr (GROUPED) {
        cum = tiles_before(0, mine);
        tiles_m = __builtin_amdgcn_readlane(cum, 63);
        for (int g0 = 64; g0 < p.G; g0 += 64) {
            int unused;
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
                const int nt_g = __builtin_amdgcn_readlane(mine, l);
                before += __builtin_amdgcn_readlane(cum, l) - nt_g;
                grp = g0 + l;
                const int r = t - before * p.tiles_n;  // its column tiles, the row tiles innermost
                n0 = r / nt_g * BN;
                m0 = __builtin_amdgcn_readfirstlane(group_row(grp)) + r % nt_g * BM;
                m_end = __builtin_amdgcn_readfirstlane(group_row(grp + 1));
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
    // a half K-step's second half: neither operand's codes are read there (zeros: E2M1 has no value whose product with
    // zero is not zero), and the scales are those of the first half once more
    const unsigned past_half = (KW & 1) && gchunk >= 4 ? kOobOffset : 0u;
    unsigned soff_a[C::NSA];
#pragma unroll
    for (int h = 0; h < C::NSA; ++h) soff_a[h] = (unsigned)(m0 + min(h * 64 + lane, m_rows - 1)) * (unsigned)p.sar * 4u;
    const unsigned soff_b = (unsigned)(n0 + min(wn * FN * 16 + lane, n_rows - 1)) * (unsigned)p.sbr * 4u;
    const unsigned sa_step = (unsigned)p.sak * 4u, sb_step = (unsigned)p.sbk * 4u;

    uint8_t* const codes = smem + wk * C::GROUP;                            // + stage * STAGE
    uint8_t* const scales = smem + WK * C::GROUP + wave * C::SCALES;        // + stage * STAGE
    auto issue = [&](int step, int stage) {
        const int kb = step * WK + wk;
        const unsigned koff = (kb < KB ? (unsigned)kb << 7 : kOobOffset);
        const unsigned more = kb == KB - 1 ? past_half : 0u;
        uint8_t* dst = codes + stage * C::STAGE + wn * 1024;
#pragma unroll
        for (int i = 0; i < C::NB + C::NA; ++i) {
            const bool is_b = i < C::NB;
            const unsigned voff = ((is_b ? voff_b + (unsigned)i * step_b : voff_a + (unsigned)(i - C::NB) * step_a) + koff) | more;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(is_b ? rs_b : rs_a, (lds_ptr_t)(dst + i * (WN * 1024)), 16, (int)voff, 0, 0, 0);
        }
        uint8_t* sd = scales + stage * C::STAGE;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const unsigned kw = (unsigned)min(2 * kb + w, KW - 1);
#pragma unroll
            for (int h = 0; h < C::NSA; ++h)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_sa, (lds_ptr_t)(sd + (w * C::NSA + h) * 256), 4, (int)(soff_a[h] + kw * sa_step), 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_sb, (lds_ptr_t)(sd + (2 * C::NSA + w) * 256), 4, (int)(soff_b + kw * sb_step), 0, 0, 0);
        }
    };
    const int key = swz_key(l16);
    const int foff0 = l16 * 128 + (((2 * g4) ^ key) << 4), foff1 = l16 * 128 + (((2 * g4 + 1) ^ key) << 4);
    // this lane's two scale bytes of row r: word g4 / 2, bytes 2 * (g4 % 2) and the next
    const int so_a = (g4 >> 1) * (C::NSA * 256) + (g4 & 1) * 2 + l16 * 4;
    const int so_b = C::NSA * 512 + (g4 >> 1) * 256 + (g4 & 1) * 2 + l16 * 4;

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
        const uint8_t* sc = scales + stage * C::STAGE;
        // (everything that is read from LDS in this step is read before the next loads are issued: the
        // compiler makes an LDS read behind LDS-bound loads wait for them)
        i32x4 w[FN][2], x[FM][2];
        int sw[FN], sx[FM];
#pragma unroll
        for (int i = 0; i < FN; ++i) {
            const uint8_t* f = st + (wn * FN + i) * 2048;
            w[i][0] = *reinterpret_cast<const i32x4*>(f + foff0);
            w[i][1] = *reinterpret_cast<const i32x4*>(f + foff1);
            sw[i] = *reinterpret_cast<const uint16_t*>(sc + so_b + i * 64);
        }
#pragma unroll
        for (int j = 0; j < FM; ++j) {
            const uint8_t* f = st + (BN + j * 16) * 128;
            x[j][0] = *reinterpret_cast<const i32x4*>(f + foff0);
            x[j][1] = *reinterpret_cast<const i32x4*>(f + foff1);
            sx[j] = *reinterpret_cast<const uint16_t*>(sc + so_a + j * 64);
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
    for (int idx = tid; idx < m_rows * (BN / 4); idx += C::NT) {
        const int row = idx / (BN / 4), col = idx % (BN / 4) * 4;
        if (col >= n_rows) continue;
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
                if (p.accumulate) {
                    const f32x4 old = *reinterpret_cast<const f32x4*>(d);
                    v.x += old.x; v.y += old.y; v.z += old.z; v.w += old.w;
                }
                *reinterpret_cast<f32x4*>(d) = v;
            } else {
                const float o[4] = {v.x, v.y, v.z, v.w};
                for (int q = 0; col + q < n_rows; ++q) d[q] = p.accumulate ? d[q] + o[q] : o[q];
            }
        }
    }
}

// ---- host side -------------------------------------------------------------------
template <class C>
static ds3_status launch_tile(MxGemmParams p, ds3_dtype ct, hipStream_t st) {
    p.tiles_m = (p.M + C::BM - 1) / C::BM;
    if (p.G > 0) {
        // an upper bound (a row tile has a row); workgroups beyond the true count leave at once
        p.tiles_m = (int)std::min<int64_t>((int64_t)p.tiles_m + p.G, p.M);
    }
    p.tiles_n = (p.N + C::BN - 1) / C::BN;
    const int64_t n = ((int64_t)p.tiles_m * p.tiles_n + 7) / 8 * 8;
    if (n * C::NT >= (1ll << 32)) return DS3_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)n), block(C::NT);
    (void)hipGetLastError();                            // a stale error of earlier, unrelated work is not this launch's
    if (p.G > 0) {
        if (ct == DS3_BF16) gemm_mxfp4_tile_kernel<C, true, true><<<grid, block, 0, st>>>(p);
        else gemm_mxfp4_tile_kernel<C, false, true><<<grid, block, 0, st>>>(p);
    } else {
        if (ct == DS3_BF16) gemm_mxfp4_tile_kernel<C, true, false><<<grid, block, 0, st>>>(p);
        else gemm_mxfp4_tile_kernel<C, false, false><<<grid, block, 0, st>>>(p);
    }
    return hipGetLastError() == hipSuccess ? DS3_OK : DS3_ERR_LAUNCH;
}

ds3_status launch_gemm_mxfp4(const MxGemmParams& p, ds3_dtype ct, hipStream_t st) {
    // 32-bit offsets inside a tile of up to 256 rows
    if ((int64_t)257 * p.ldb + p.K / 2 >= (1ll << 31) || (int64_t)257 * p.lda + p.K / 2 >= (1ll << 31)) return DS3_ERR_UNSUPPORTED;
    const int64_t rows = p.G > 0 ? (p.M + p.G - 1) / p.G : p.M;
    if (rows <= 32) return launch_tile<TileCfg<2, 2, 4, 1, 3>>(p, ct, st);
    return launch_tile<TileCfg<2, 8, 4, 1, 3>>(p, ct, st);
}

}  // namespace ds3
