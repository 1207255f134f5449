// Rows of a mixture-of-experts layer taken into expert order and back, for gfx950.
//
// The sort is a counting sort whose rows are in the order (expert, token, choice), so nothing depends on timing.
// Dispatch and combine go token by token: dispatch reads (and quantizes) a token's row once and writes it to the row of
// each of its choices, combine reads those rows and sums them in FP32 in the order of the choices.  No atomics on
// results.  All of them are bound by memory.
#include <algorithm>

#include "ds3_internal.h"
#include "ds3_mx4_dev.h"

namespace ds3 {

// =============================================================================
// Sort
// =============================================================================
constexpr int kSortThreads = 1024;
constexpr int kSortChunk = 4096;                       // choices a workgroup of the long form places
constexpr int kSortMaxGroups = 1023;

struct SortParams {
    const int32_t* ids;
    int64_t ld;
    int n, top_k, first, G;                            // n = tokens * top_k
    int32_t* offsets;
    int32_t* rows;
};

// expert of choice p among those held here, or -1
__device__ __forceinline__ int sort_expert(const SortParams& p, int i) {
    const int64_t at = p.ld == p.top_k ? (int64_t)i : (int64_t)(i / p.top_k) * p.ld + i % p.top_k;
    const unsigned int e = (unsigned int)p.ids[at] - (unsigned int)p.first;
    return e < (unsigned int)p.G ? (int)e : -1;
}

// Exclusive prefix sum of one value a thread over the workgroup.
__device__ __forceinline__ int block_exclusive(int v, int* part) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int sum = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(sum, d);
        if (lane >= d) sum += o;
    }
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += part[w];
    return before + sum - v;
}

// Places choices [i0, i1) (at most kSortChunk) in order: base[g] is the next free row of expert g.  Within a wave the
// lanes of the same expert find each other by a ballot per bit of its number; the waves take turns.
__device__ __forceinline__ void place(const SortParams& p, int i0, int i1, int* base) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int bits = 32 - __clz(p.G);
    for (int at = i0; at < i1; at += kSortThreads) {
        const int i = at + (int)threadIdx.x;
        const int e = i < i1 ? sort_expert(p, i) : -1;
        unsigned long long same = __ballot(e >= 0);
        for (int b = 0; b < bits; ++b) {
            const unsigned long long set = __ballot((e >> b) & 1);
            same &= ((e >> b) & 1) ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        int row = -1;
        const int waves = min(kSortThreads, i1 - at + 63) >> 6;
        for (int w = 0; w < waves; ++w) {
            if (wave == w && e >= 0) {
                row = base[e] + rank;
                if (rank == 0) base[e] = row + __popcll(same);
            }
            __syncthreads();
        }
        if (i < i1) p.rows[i] = row;
    }
}

// One launch: every workgroup counts all choices, those before its own 1024 apart, so none waits for another.
__global__ __launch_bounds__(kSortThreads) void moe_sort_kernel(const SortParams p) {
    __shared__ int before[kSortMaxGroups + 1], total[kSortMaxGroups + 1], part[kSortThreads / 64];
    const int tid = threadIdx.x, start = (int)blockIdx.x * kSortThreads;
    before[tid] = 0;
    total[tid] = 0;
    __syncthreads();
    for (int i = tid; i < p.n; i += kSortThreads) {
        const int e = sort_expert(p, i);
        if (e >= 0) atomicAdd(i < start ? &before[e] : &total[e], 1);
    }
    __syncthreads();
    const int all = tid < p.G ? before[tid] + total[tid] : 0;
    const int off = block_exclusive(all, part);
    if (tid < p.G) before[tid] += off;
    if (blockIdx.x == 0 && tid <= p.G) p.offsets[tid] = off;     // (thread G holds no expert: the sum of all)
    __syncthreads();
    place(p, start, min(start + kSortThreads, p.n), before);
}

// The long form, for more choices than each workgroup should count: chunks are counted, the counts summed up over the
// chunks, and the chunks placed.  A chunk's counts, then its first free rows, lie where its rows will be (a chunk has at
// least as many choices as there are experts); the last chunk, which may be shorter, is counted where it is needed.
__device__ __forceinline__ void count_chunk(const SortParams& p, int chunk, int* cnt) {
    cnt[threadIdx.x] = 0;
    __syncthreads();
    const int end = min((chunk + 1) * kSortChunk, p.n);
    for (int i = chunk * kSortChunk + (int)threadIdx.x; i < end; i += kSortThreads) {
        const int e = sort_expert(p, i);
        if (e >= 0) atomicAdd(&cnt[e], 1);
    }
    __syncthreads();
}
__global__ __launch_bounds__(kSortThreads) void moe_sort_count_kernel(const SortParams p) {
    __shared__ int cnt[kSortMaxGroups + 1];
    count_chunk(p, blockIdx.x, cnt);
    if ((int)threadIdx.x < p.G) p.rows[(int64_t)blockIdx.x * kSortChunk + threadIdx.x] = cnt[threadIdx.x];
}
__global__ __launch_bounds__(kSortThreads) void moe_sort_scan_kernel(const SortParams p, int chunks) {
    __shared__ int cnt[kSortMaxGroups + 1], part[kSortThreads / 64];
    const int tid = threadIdx.x;
    count_chunk(p, chunks - 1, cnt);
    int sum = 0;
    if (tid < p.G) {
        constexpr int AHEAD = 16;                      // counts in flight: one after another each would wait out a latency
        for (int c0 = 0; c0 < chunks - 1; c0 += AHEAD) {
            int v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) v[k] = c0 + k < chunks - 1 ? p.rows[(int64_t)(c0 + k) * kSortChunk + tid] : 0;
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (c0 + k < chunks - 1) p.rows[(int64_t)(c0 + k) * kSortChunk + tid] = sum;
                sum += v[k];
            }
        }
        sum += cnt[tid];
    }
    const int off = block_exclusive(sum, part);
    if (tid <= p.G) p.offsets[tid] = off;
}
__global__ __launch_bounds__(kSortThreads) void moe_sort_place_kernel(const SortParams p, int chunks) {
    __shared__ int base[kSortMaxGroups + 1];
    const int tid = threadIdx.x, chunk = blockIdx.x;
    if (chunk == chunks - 1) {
        count_chunk(p, chunk, base);
        if (tid < p.G) base[tid] = p.offsets[tid + 1] - base[tid];
    } else if (tid < p.G) {
        base[tid] = p.offsets[tid] + p.rows[(int64_t)chunk * kSortChunk + tid];
    }
    __syncthreads();                                   // (the counts are read before the first rows are written over them)
    place(p, chunk * kSortChunk, min((chunk + 1) * kSortChunk, p.n), base);
}

// =============================================================================
// The rows of a token's choices, one a lane (top_k <= 64): the lanes whose choice has a row here, and its row.
// =============================================================================
__device__ __forceinline__ unsigned long long token_rows(const int32_t* rows, int64_t token, int top_k, int64_t total_rows, int lane, int& row) {
    row = lane < top_k ? rows[token * top_k + lane] : -1;
    return __ballot(row >= 0 && row < total_rows);
}

// Eight columns of a row.
template <typename T> __device__ __forceinline__ void store8(uint8_t* p, const float* v, int64_t left);
template <> __device__ __forceinline__ void store8<Bf16>(uint8_t* p, const float* v, int64_t left) {
    if (left > 0)
        *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
template <> __device__ __forceinline__ void store8<F32>(uint8_t* p, const float* v, int64_t left) {
    if (left > 0) *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    if (left > 4) *reinterpret_cast<f32x4*>(p + 16) = f32x4{v[4], v[5], v[6], v[7]};
}
template <typename T> __device__ __forceinline__ int64_t bytes_of(int64_t n) { return n * (16 / T::EPL); }

// =============================================================================
// Dispatch: a workgroup takes 2048 columns of one token, a lane eight of them (one 1x128 tile or 128-element block is 16
// lanes); what it leaves is written to every row of the token's choices.
// =============================================================================
template <typename T, DispatchTo TO>
__global__ __launch_bounds__(256) void moe_dispatch_kernel(const DispatchParams p, int segs) {
    const int lane = threadIdx.x & 63, lane16 = threadIdx.x & 15;
    const int64_t token = blockIdx.x / (unsigned)segs;
    const int64_t col = (int64_t)(blockIdx.x % (unsigned)segs) * 2048 + threadIdx.x * 8;
    int row;
    unsigned long long todo = token_rows(p.row_of_slot, token, p.top_k, p.total_rows, lane, row);
    if (todo == 0) return;
    Granule8<T> g;
    g.load(p.x + token * p.ldx_bytes + bytes_of<T>(col), p.cols - col);
    const int64_t left = p.cols - col;
    if constexpr (TO == kDispatchRows) {
        for (; todo; todo &= todo - 1) {
            const int64_t r = __builtin_amdgcn_readlane(row, __builtin_ctzll(todo));
            uint8_t* dst = p.y + r * p.ldy_bytes + bytes_of<T>(col);
#pragma unroll
            for (int h = 0; h < Granule8<T>::N; ++h)
                if (h * T::EPL < left) st_stream(dst + h * 16, g.g[h]);
        }
    } else {
        float v[8];
        g.values(v);
        unsigned int w0, w1 = 0, sw;
        if constexpr (TO == kDispatchFp8) {
            const GroupScale gs = group_scale(as_f32(row16_max_bits(g.amax_bits())), p.pow2);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = v[i] * gs.r;
            w0 = cvt4_e4m3(v[0], v[1], v[2], v[3]);
            w1 = cvt4_e4m3(v[4], v[5], v[6], v[7]);
            sw = as_u32(gs.s);
        } else {
            const MxScale ms = mx_scale(quad_max_bits(g.amax_bits()));
            w0 = cvt8_e2m1(v, ms.r);
            sw = row16_scale_word(ms.e, lane16);
        }
        const int64_t kb = col >> 7;
        for (; todo; todo &= todo - 1) {
            const int64_t r = __builtin_amdgcn_readlane(row, __builtin_ctzll(todo));
            if constexpr (TO == kDispatchFp8) {
                uint8_t* dst = p.y + r * p.ldy_bytes + col;
                if (left >= 8) st_stream(dst, u32x2{w0, w1});
                else if (left > 0) st_stream(dst, w0);
            } else {
                uint8_t* dst = p.y + r * p.ldy_bytes + (col >> 1);
                if (left >= 8) st_stream(dst, w0);
                else if (left > 0) st_stream(dst, (uint16_t)w0);
            }
            if (lane16 == 0 && left > 0) static_cast<uint32_t*>(p.s)[r * p.ssr + kb * p.ssk] = sw;
        }
    }
}

// =============================================================================
// Combine: the same split; up to four of the rows are in flight at a time.
// =============================================================================
template <typename TY, typename TO>
__global__ __launch_bounds__(256) void moe_combine_kernel(const CombineParams p, int segs) {
    const int lane = threadIdx.x & 63;
    const int64_t token = blockIdx.x / (unsigned)segs;
    const int64_t col = (int64_t)(blockIdx.x % (unsigned)segs) * 2048 + threadIdx.x * 8;
    int row;
    unsigned long long todo = token_rows(p.row_of_slot, token, p.top_k, p.total_rows, lane, row);
    float weight = 1.f;
    if (p.w != nullptr && lane < p.top_k) weight = p.w[token * p.top_k + lane];
    const int64_t left = p.cols - col;
    const uint8_t* y = p.y + bytes_of<TY>(col);
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    while (todo) {
        Granule8<TY> g[4];
        float w[4];
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (todo) {
                const int s = __builtin_ctzll(todo);
                todo &= todo - 1;
                w[i] = as_f32((unsigned int)__builtin_amdgcn_readlane((int)as_u32(weight), s));
                g[i].load(y + (int64_t)__builtin_amdgcn_readlane(row, s) * p.ldy_bytes, left);
                n = i + 1;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < n) {
                float v[8];
                g[i].values(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = __builtin_fmaf(w[i], v[e], acc[e]);
            }
        }
    }
    store8<TO>(p.out + token * p.ldo_bytes + bytes_of<TO>(col), acc, left);
}

// =============================================================================
// Combine's gradients: a workgroup takes a token.  dy of each row is the weight times the token's gradient, dw the
// product of the two rows: lane by lane over the columns, then over the lanes and waves, always in the same order.
// =============================================================================
template <typename TY, typename TO>
__global__ __launch_bounds__(256) void moe_combine_bwd_kernel(const CombineParams p) {
    constexpr int NC = 4;                              // 8-column pieces a thread keeps of the gradient
    __shared__ float dots[64][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = blockIdx.x;
    int row;
    const unsigned long long here = token_rows(p.row_of_slot, token, p.top_k, p.total_rows, lane, row);
    float weight = 1.f;
    if (p.w != nullptr && lane < p.top_k) weight = p.w[token * p.top_k + lane];
    if (here != 0) {
        for (int64_t c0 = 0; c0 < p.cols; c0 += 2048 * NC) {
            Granule8<TO> d[NC];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int64_t col = c0 + c * 2048 + threadIdx.x * 8;
                d[c].load(p.out + token * p.ldo_bytes + bytes_of<TO>(col), p.cols - col);
            }
            for (unsigned long long todo = here; todo; todo &= todo - 1) {
                const int s = __builtin_ctzll(todo);
                const int64_t r = __builtin_amdgcn_readlane(row, s);
                const float w = as_f32((unsigned int)__builtin_amdgcn_readlane((int)as_u32(weight), s));
                Granule8<TY> g[NC];
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const int64_t col = c0 + c * 2048 + threadIdx.x * 8;
                    g[c].load(p.y + r * p.ldy_bytes + bytes_of<TY>(col), p.cols - col);
                }
                float dot = 0.f;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const int64_t col = c0 + c * 2048 + threadIdx.x * 8;
                    float dv[8], yv[8];
                    d[c].values(dv);
                    g[c].values(yv);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        dot = __builtin_fmaf(dv[e], yv[e], dot);
                        dv[e] *= w;
                    }
                    store8<TY>(p.dy + r * p.lddy_bytes + bytes_of<TY>(col), dv, p.cols - col);
                }
#pragma unroll
                for (int m = 1; m < 64; m <<= 1) dot += __shfl_xor(dot, m);
                if (lane == 0) dots[s][wave] = c0 == 0 ? dot : dots[s][wave] + dot;
            }
        }
    }
    __syncthreads();
    if ((int)threadIdx.x < p.top_k) {
        const int s = threadIdx.x;
        float v = 0.f;
        if ((here >> s) & 1) v = ((dots[s][0] + dots[s][1]) + dots[s][2]) + dots[s][3];
        p.dw[token * p.top_k + s] = v;
    }
}

// ---- host side -------------------------------------------------------------------
static ds3_status launch_status() { return hipGetLastError() == hipSuccess ? DS3_OK : DS3_ERR_LAUNCH; }
constexpr int64_t kMaxGrid = (1ll << 24) - 1;          // a grid may have 2^32 threads

// Up to here every workgroup counts all choices itself.
constexpr int kSortOneLaunch = 65536;

ds3_status launch_moe_sort(const int32_t* ids, int64_t tokens, int top_k, int64_t ld, int first, int G, int32_t* offsets,
                           int32_t* row_of_slot, hipStream_t st) {
    const SortParams p{ids, ld, (int)(tokens * top_k), top_k, first, G, offsets, row_of_slot};
    (void)hipGetLastError();                            // a stale error of earlier, unrelated work is not this launch's
    if (p.n <= kSortOneLaunch) {
        const int blocks = std::max(1, (p.n + kSortThreads - 1) / kSortThreads);
        moe_sort_kernel<<<dim3(blocks), kSortThreads, 0, st>>>(p);
        return launch_status();
    }
    const int chunks = (p.n + kSortChunk - 1) / kSortChunk;
    moe_sort_count_kernel<<<dim3(chunks - 1), kSortThreads, 0, st>>>(p);
    moe_sort_scan_kernel<<<dim3(1), kSortThreads, 0, st>>>(p, chunks);
    moe_sort_place_kernel<<<dim3(chunks), kSortThreads, 0, st>>>(p, chunks);
    return launch_status();
}

ds3_status launch_moe_dispatch(const DispatchParams& p, ds3_dtype xt, DispatchTo to, hipStream_t st) {
    const int64_t segs = (p.cols + 2047) / 2048, n = p.tokens * segs;
    if (n > kMaxGrid) return DS3_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    const dim3 grid((unsigned)n);
    const bool b = xt == DS3_BF16;
    switch (to) {
        case kDispatchRows:
            if (b) moe_dispatch_kernel<Bf16, kDispatchRows><<<grid, 256, 0, st>>>(p, (int)segs);
            else moe_dispatch_kernel<F32, kDispatchRows><<<grid, 256, 0, st>>>(p, (int)segs);
            break;
        case kDispatchFp8:
            if (b) moe_dispatch_kernel<Bf16, kDispatchFp8><<<grid, 256, 0, st>>>(p, (int)segs);
            else moe_dispatch_kernel<F32, kDispatchFp8><<<grid, 256, 0, st>>>(p, (int)segs);
            break;
        case kDispatchMx4:
            if (b) moe_dispatch_kernel<Bf16, kDispatchMx4><<<grid, 256, 0, st>>>(p, (int)segs);
            else moe_dispatch_kernel<F32, kDispatchMx4><<<grid, 256, 0, st>>>(p, (int)segs);
            break;
    }
    return launch_status();
}

ds3_status launch_moe_combine(const CombineParams& p, ds3_dtype yt, ds3_dtype ot, hipStream_t st) {
    const int64_t segs = (p.cols + 2047) / 2048, n = p.tokens * segs;
    if (n > kMaxGrid) return DS3_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    const dim3 grid((unsigned)n);
    if (yt == DS3_BF16) {
        if (ot == DS3_BF16) moe_combine_kernel<Bf16, Bf16><<<grid, 256, 0, st>>>(p, (int)segs);
        else moe_combine_kernel<Bf16, F32><<<grid, 256, 0, st>>>(p, (int)segs);
    } else {
        if (ot == DS3_BF16) moe_combine_kernel<F32, Bf16><<<grid, 256, 0, st>>>(p, (int)segs);
        else moe_combine_kernel<F32, F32><<<grid, 256, 0, st>>>(p, (int)segs);
    }
    return launch_status();
}

ds3_status launch_moe_combine_bwd(const CombineParams& p, ds3_dtype yt, ds3_dtype ot, hipStream_t st) {
    if (p.tokens > kMaxGrid) return DS3_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    const dim3 grid((unsigned)p.tokens);
    if (yt == DS3_BF16) {
        if (ot == DS3_BF16) moe_combine_bwd_kernel<Bf16, Bf16><<<grid, 256, 0, st>>>(p);
        else moe_combine_bwd_kernel<Bf16, F32><<<grid, 256, 0, st>>>(p);
    } else {
        if (ot == DS3_BF16) moe_combine_bwd_kernel<F32, Bf16><<<grid, 256, 0, st>>>(p);
        else moe_combine_bwd_kernel<F32, F32><<<grid, 256, 0, st>>>(p);
    }
    return launch_status();
}

}  // namespace ds3
