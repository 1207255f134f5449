// MXFP4 quantizers for gfx950: groups of 32 along a row, groups of 32 along the
// rows with the result transposed (the operand of the product that contracts
// over them), and the way back to BF16.  All are single-pass HBM scans.
#include "ds3_internal.h"
#include "ds3_mx4_dev.h"

namespace ds3 {

// =============================================================================
// Along a row: 16 lanes a 128-element block, eight elements a lane, so a group is
// four neighbouring lanes and the block's scale bytes meet in one word by two lane
// exchanges.  A workgroup is 16 rows by TPG consecutive blocks (each lane has TPG
// loads in flight, and the 16 words of a block column are 64 contiguous bytes of a
// block-major scale array); the grid walks along the rows first.  Bound by memory:
// 18432 x 7168 BF16 55 us, 6.0 TB/s.
// =============================================================================
template <typename T, int TPG>
__global__ __launch_bounds__(256) void quant_mxfp4_kernel(const uint8_t* __restrict__ x, int64_t rows, int64_t cols, int64_t ldx_bytes,
                                                          uint8_t* __restrict__ q, int64_t ldq, uint32_t* __restrict__ s,
                                                          int64_t ssr, int64_t ssk, int ngroups) {
    constexpr int ESZ = 16 / T::EPL;
    const int lane16 = threadIdx.x & 15;
    const int64_t row = (int64_t)(blockIdx.x / (unsigned)ngroups) * 16 + (threadIdx.x >> 4);
    if (row >= rows) return;                      // a whole DPP row leaves together
    const int64_t kb0 = (int64_t)(blockIdx.x % (unsigned)ngroups) * TPG;
    const int64_t nkb = (cols + 127) >> 7;
    const uint8_t* xr = x + row * ldx_bytes;
    Granule8<T> g[TPG];
#pragma unroll
    for (int t = 0; t < TPG; ++t) {
        const int64_t col = (kb0 + t) * 128 + lane16 * 8;
        g[t].load(xr + col * ESZ, cols - col);
    }
#pragma unroll
    for (int t = 0; t < TPG; ++t) {
        if (kb0 + t >= nkb) break;
        const int64_t col = (kb0 + t) * 128 + lane16 * 8;
        const MxScale ms = mx_scale(quad_max_bits(g[t].amax_bits()));
        const unsigned int word = row16_scale_word(ms.e, lane16);
        float v[8];
        g[t].values(v);
        const unsigned int w = cvt8_e2m1(v, ms.r);
        uint8_t* dst = q + row * ldq + (col >> 1);
        if (col + 8 <= cols) st_stream(dst, w);
        else if (col < cols) st_stream(dst, (uint16_t)w);      // (FP32 rows may end after four)
        if (lane16 == 0) s[row * ssr + (kb0 + t) * ssk] = word;
    }
}

// =============================================================================
// Along the rows (tokens): a workgroup takes 256 tokens x 64 channels.  A thread
// loads TPT consecutive tokens of one 16-byte channel granule, so it holds TPT
// consecutive codes of each of its channels; a group's other tokens are in lanes
// of the same wave.  Codes and scale bytes go through LDS laid out by channel and
// leave as 16-byte stores, 128 bytes a channel.  Bound by memory: 7168 x 4096 BF16
// 15.3 us, 4.9 TB/s.
// =============================================================================
template <typename T>
__global__ __launch_bounds__(256) void quant_mxfp4_t_kernel(const uint8_t* __restrict__ x, int64_t rows, int64_t cols, int64_t ldx_bytes,
                                                            uint8_t* __restrict__ qt, int64_t ldq, uint32_t* __restrict__ st,
                                                            int64_t ssc, int64_t sst) {
    constexpr int EPL = T::EPL, ESZ = 16 / EPL;
    constexpr int LPR = 64 / EPL;                 // lanes across the 64 channels (8 BF16, 16 FP32)
    constexpr int TPT = 256 * LPR / 256;          // consecutive tokens per thread (8, 16)
    constexpr int KS = EPL == 8 ? 3 : 2;          // swizzle key: the lane index across the channels
    __shared__ __attribute__((aligned(16))) uint8_t tile[64 * 144];   // [channel][128 bytes of codes, 16 spare]
    __shared__ __attribute__((aligned(8))) uint8_t se[64][8];         // scale bytes of each channel's eight groups
    const int64_t c0 = (int64_t)blockIdx.x * 64, t0 = (int64_t)blockIdx.y * 256;
    const int lc = threadIdx.x % LPR, sl = threadIdx.x / LPR;
    const int64_t col = c0 + lc * EPL;
    u32x4 g[TPT];
#pragma unroll
    for (int p = 0; p < TPT; ++p) {
        const int64_t tok = t0 + sl * TPT + p;
        g[p] = u32x4{0u, 0u, 0u, 0u};
        if (col < cols && tok < rows) g[p] = ld_stream(x + tok * ldx_bytes + col * ESZ);
    }
    float v[TPT][EPL];
#pragma unroll
    for (int p = 0; p < TPT; ++p) widen<T>(g[p], v[p]);
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
        unsigned int m = 0;
#pragma unroll
        for (int p = 0; p < TPT; ++p) m = umax(m, as_u32(v[p][e]) & 0x7fffffffu);
        // the group's other tokens: lanes 8 and 16 further on (BF16: four lanes of eight tokens), 16 (FP32: two of 16)
        if constexpr (EPL == 8) m = umax(m, dpp_u32<0x128>(m));              // row_ror:8
        m = umax(m, (unsigned int)__shfl_xor((int)m, 16));
        if constexpr (EPL == 8) static_assert(LPR == 8 && TPT == 8, "a group is lanes that differ in bits 3 and 4");
        else static_assert(LPR == 16 && TPT == 16, "a group is lanes that differ in bit 4");
        const MxScale ms = mx_scale(m);
        const int ch = lc * EPL + e;
        if (sl % (32 / TPT) == 0) se[ch][sl / (32 / TPT)] = (uint8_t)ms.e;
        float u[8];
#pragma unroll
        for (int h = 0; h < TPT / 8; ++h) {
#pragma unroll
            for (int p = 0; p < 8; ++p) u[p] = v[h * 8 + p][e];
            *reinterpret_cast<unsigned int*>(tile + tile_off<KS>(ch, sl * (TPT / 2) + h * 4)) = cvt8_e2m1(u, ms.r);
        }
    }
    __syncthreads();
    const int64_t nbytes = (rows + 1) >> 1;
#pragma unroll
    for (int it = 0; it < 2; ++it) {
        const int ch = it * 32 + (threadIdx.x >> 3), chunk = threadIdx.x & 7;
        const int64_t c = c0 + ch, b = (t0 >> 1) + chunk * 16;
        if (c >= cols || b >= nbytes) continue;
        const u32x4 w = *reinterpret_cast<const u32x4*>(tile + tile_off<KS>(ch, chunk * 16));
        uint8_t* dst = qt + c * ldq + b;
        if (b + 16 <= nbytes) {
            st_stream(dst, w);
        } else {
            const unsigned int wd[4] = {w.x, w.y, w.z, w.w};
            for (int i = 0; i < 16 && b + i < nbytes; ++i) dst[i] = (uint8_t)(wd[i >> 2] >> (8 * (i & 3)));
        }
    }
    if (threadIdx.x < 128) {
        const int ch = threadIdx.x & 63, h = threadIdx.x >> 6;
        const int64_t c = c0 + ch, tb = (t0 >> 7) + h;
        if (c < cols && tb * 128 < rows) st[c * ssc + tb * sst] = *reinterpret_cast<const uint32_t*>(&se[ch][h * 4]);
    }
}

// =============================================================================
// Codes and scales back to BF16 (exact unless a value exceeds BF16's range): eight
// elements a lane, 16 bytes out.  Bound by memory: 7168 x 4096 13.2 us, 5.6 TB/s.
// =============================================================================
template <bool NT>
__global__ __launch_bounds__(256) void dequant_mxfp4_kernel(const uint8_t* __restrict__ q, int64_t rows, int64_t cols, int64_t ldq,
                                                            const uint32_t* __restrict__ s, int64_t ssr, int64_t ssk,
                                                            uint8_t* __restrict__ y, int64_t ldy, int ngroups) {
    const int lane16 = threadIdx.x & 15;
    const int64_t row = (int64_t)(blockIdx.x / (unsigned)ngroups) * 16 + (threadIdx.x >> 4);
    if (row >= rows) return;
    const int64_t kb0 = (int64_t)(blockIdx.x % (unsigned)ngroups) * 2;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int64_t col = (kb0 + t) * 128 + lane16 * 8;
        if (col >= cols) return;
        const unsigned int sw = s[row * ssr + (kb0 + t) * ssk];
        const float sc = e8m0((sw >> (8 * (lane16 >> 2))) & 255u);
        const uint8_t* src = q + row * ldq + (col >> 1);
        unsigned int w = 0;
        const int64_t left = cols - col;
        if (left >= 8) w = *reinterpret_cast<const uint32_t*>(src);
        else for (int i = 0; 2 * i < left; ++i) w |= (unsigned int)src[i] << (8 * i);
        unsigned int o[4];
        auto two = [&](auto v) { return pack_bf16x2(v[0] * sc, v[1] * sc); };
        o[0] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0));
        o[1] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1));
        o[2] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2));
        o[3] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3));
        uint8_t* dst = y + (row * ldy + col) * 2;
        if (left >= 8) {
            if constexpr (NT) st_nt(dst, u32x4{o[0], o[1], o[2], o[3]});
            else st_stream(dst, u32x4{o[0], o[1], o[2], o[3]});
        }
        else for (int i = 0; i < left; ++i) reinterpret_cast<uint16_t*>(dst)[i] = (uint16_t)(o[i >> 1] >> (16 * (i & 1)));
    }
}

// ---- host side -------------------------------------------------------------------
static ds3_status launch_status() { return hipGetLastError() == hipSuccess ? DS3_OK : DS3_ERR_LAUNCH; }

// A grid may have 2^32 threads: 2^24 workgroups of 256.
constexpr int64_t kMaxGrid = (1ll << 24) - 1;

// Blocks a lane: with four instead of two 18432 x 7168 BF16 takes 54.9 us instead of 55.5 (6.0 TB/s), FP32 rows 29.2
// instead of 28.6.
constexpr int kBlocksPerLane = 2;

ds3_status launch_quant_mxfp4(const void* x, ds3_dtype xt, int64_t rows, int64_t cols, int64_t ldx, uint8_t* q, int64_t ldq,
                              uint32_t* s, int64_t ssr, int64_t ssk, hipStream_t st) {
    constexpr int TPG = kBlocksPerLane;
    const int64_t ng = ((cols + 127) / 128 + TPG - 1) / TPG, n = (rows + 15) / 16 * ng;
    if (n > kMaxGrid) return DS3_ERR_UNSUPPORTED;
    (void)hipGetLastError();                            // a stale error of earlier, unrelated work is not this launch's
    if (xt == DS3_BF16)
        quant_mxfp4_kernel<Bf16, TPG><<<dim3((unsigned)n), 256, 0, st>>>((const uint8_t*)x, rows, cols, ldx * 2, q, ldq, s, ssr, ssk, (int)ng);
    else
        quant_mxfp4_kernel<F32, TPG><<<dim3((unsigned)n), 256, 0, st>>>((const uint8_t*)x, rows, cols, ldx * 4, q, ldq, s, ssr, ssk, (int)ng);
    return launch_status();
}

ds3_status launch_quant_mxfp4_t(const void* x, ds3_dtype xt, int64_t rows, int64_t cols, int64_t ldx, uint8_t* qt, int64_t ldq,
                                uint32_t* s_t, int64_t ssc, int64_t sst, hipStream_t st) {
    const int64_t gx = (cols + 63) / 64, gy = (rows + 255) / 256;
    if (gx > kMaxGrid || gy > 65535) return DS3_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    const dim3 grid((unsigned)gx, (unsigned)gy);
    if (xt == DS3_BF16)
        quant_mxfp4_t_kernel<Bf16><<<grid, 256, 0, st>>>((const uint8_t*)x, rows, cols, ldx * 2, qt, ldq, s_t, ssc, sst);
    else
        quant_mxfp4_t_kernel<F32><<<grid, 256, 0, st>>>((const uint8_t*)x, rows, cols, ldx * 4, qt, ldq, s_t, ssc, sst);
    return launch_status();
}

ds3_status launch_dequant_mxfp4(const uint8_t* q, int64_t rows, int64_t cols, int64_t ldq, const uint32_t* s, int64_t ssr,
                                int64_t ssk, void* y, int64_t ldy, hipStream_t st) {
    const int64_t ng = ((cols + 127) / 128 + 1) / 2, n = (rows + 15) / 16 * ng;
    if (n > kMaxGrid) return DS3_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    // (non-temporal stores where little of the values would stay in the caches: 264 MB 77 -> 49 us, 59 MB 12.8 -> 11.7)
    if (rows * cols * 2 >= (48ll << 20)) dequant_mxfp4_kernel<true><<<dim3((unsigned)n), 256, 0, st>>>(q, rows, cols, ldq, s, ssr, ssk, (uint8_t*)y, ldy, (int)ng);
    else dequant_mxfp4_kernel<false><<<dim3((unsigned)n), 256, 0, st>>>(q, rows, cols, ldq, s, ssr, ssk, (uint8_t*)y, ldy, (int)ng);
    return launch_status();
}

}  // namespace ds3
