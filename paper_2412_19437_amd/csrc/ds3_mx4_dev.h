// Device-side helpers of the MXFP4 format: groups of 32 elements share a power
// of two (an E8M0 byte, bias 127), elements are E2M1 nibbles, two in a byte, the
// element with the lower index in the low half.  The bytes of the four groups of a
// 128-element block are one 32-bit word, the first group's in the low byte.
#pragma once
#include "ds3_dev.h"

namespace ds3 {

// Scale of a group from the bit pattern of its largest magnitude: the exponent byte e of the smallest power of two
// 2^(e - 127) with 6 * 2^(e - 127) >= amax, and the exact reciprocal r = 2^(127 - e).  6 = 1.5 * 2^2: amax = 1.f * 2^E
// needs E - 2, one more where 1.f > 1.5.  Magnitudes below 6 * 2^-127 (FP32's subnormals among them) take e = 0, zeros
// 2^0.  A group that holds an infinity or a NaN takes e = 255, E8M0's NaN, and codes of zero (r = 0).
struct MxScale { unsigned int e; float r; };
__device__ __forceinline__ MxScale mx_scale(unsigned int amax_bits) {
    const int up = (int)(amax_bits >> 23) - 2 + ((amax_bits & 0x7fffffu) > 0x400000u ? 1 : 0);
    unsigned int e = (unsigned int)(up > 0 ? up : 0);
    e = amax_bits == 0 ? 127u : e;
    const bool bad = amax_bits >= 0x7f800000u;
    return MxScale{bad ? 255u : e, bad ? 0.f : as_f32((254u - e) << 23)};
}

// Eight FP32 values -> eight E2M1 codes in one word: the hardware conversion rounds to nearest even and saturates.
// Zeros where r is 0, in a group whose scale is NaN.
__device__ __forceinline__ unsigned int cvt8_e2m1(const float* v, float r) {
    unsigned int w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * r, v[1] * r, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * r, v[3] * r, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * r, v[5] * r, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * r, v[7] * r, 1.0f, 3);
    return r == 0.f ? 0u : w;
}

// Over the 16 lanes of a DPP row, eight consecutive elements each (one 128-element block): the group's largest magnitude
// in each of its four lanes, and the block's word of scale bytes, in every lane, from each group's.
__device__ __forceinline__ unsigned int quad_max_bits(unsigned int v) {
    v = umax(v, dpp_u32<0xB1>(v));   // quad_perm [1,0,3,2]
    return umax(v, dpp_u32<0x4E>(v));   // quad_perm [2,3,0,1]
}
__device__ __forceinline__ unsigned int row16_scale_word(unsigned int e, int lane16) {
    unsigned int w = e << (8 * (lane16 >> 2));
    w |= dpp_u32<0x141>(w);          // row_half_mirror: quads 0<->1, 2<->3
    return w | dpp_u32<0x140>(w);    // row_mirror: halves
}

// 2^(e - 127) as FP32 (2^-127 is subnormal, 255 is NaN).
__device__ __forceinline__ float e8m0(unsigned int e) {
    return e == 0 ? as_f32(0x00400000u) : e == 255 ? as_f32(0x7fc00000u) : as_f32(e << 23);
}

// One granule of eight consecutive elements: BF16 is one 16-byte load, FP32 two.  Elements from `left` on (a
// multiple of a 16-byte load's) are zeros.
template <typename T> struct Granule8 {
    static constexpr int N = 8 / T::EPL;
    u32x4 g[N];
    __device__ __forceinline__ void load(const uint8_t* p, int64_t left) {
#pragma unroll
        for (int h = 0; h < N; ++h) {
            g[h] = u32x4{0u, 0u, 0u, 0u};
            if (h * T::EPL < left) g[h] = ld_stream(p + h * 16);
        }
    }
    // ... of what other waves read too
    __device__ __forceinline__ void load_kept(const uint8_t* p, int64_t left) {
#pragma unroll
        for (int h = 0; h < N; ++h) {
            g[h] = u32x4{0u, 0u, 0u, 0u};
            if (h * T::EPL < left) g[h] = *reinterpret_cast<const u32x4*>(p + h * 16);
        }
    }
    __device__ __forceinline__ unsigned int amax_bits() const {
        unsigned int m = granule_amax_bits<T>(g[0]);
        if constexpr (N == 2) m = umax(m, granule_amax_bits<T>(g[1]));
        return m;
    }
    __device__ __forceinline__ void values(float* v) const {
        widen<T>(g[0], v);
        if constexpr (N == 2) widen<T>(g[1], v + 4);
    }
};

}  // namespace ds3
