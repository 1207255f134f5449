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

// Expert of choice i among those held here, or -1.  PACKED: rows of ids without gaps on a 16-byte border.
template <bool PACKED>
__device__ __forceinline__ int sort_expert(const SortParams& p, int i) {
    const int64_t at = PACKED || p.ld == p.top_k ? (int64_t)i : (int64_t)(i / p.top_k) * p.ld + i % p.top_k;
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
#pragma unroll
    for (int w = 0; w < kSortThreads / 64; ++w) before += w < wave ? part[w] : 0;
    return before + sum - v;
}

// Places choices [i0, i1) in order: base[g] is the next free row of expert g, e the expert of choice i0 + tid.  Within a
// wave the lanes of the same expert find each other by a ballot per bit of its number; the waves leave their counts, a byte
// each, in the expert's row of `waves` (zeros before and after), where each sums up those of the waves before it.
struct SortShared {
    int base[kSortMaxGroups + 1];
    u32x4 waves[kSortMaxGroups + 1];
    int part[kSortThreads / 64];
};
__device__ __forceinline__ int byte_sum(unsigned int v, int acc) { return (int)__builtin_amdgcn_sad_u8(v, 0u, (unsigned int)acc); }
template <bool PACKED>
__device__ __forceinline__ void place(const SortParams& p, int i0, int i1, int e, SortShared& s) {
    static_assert(kSortThreads == 64 * 16, "a byte a wave");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int bits = 32 - __clz(p.G);
    for (int at = i0; at < i1; at += kSortThreads) {
        const int i = at + tid;
        if (at != i0) e = i < i1 ? sort_expert<PACKED>(p, i) : -1;
        unsigned long long same = __ballot(e >= 0);
        for (int b = 0; b < bits; ++b) {
            const unsigned long long set = __ballot((e >> b) & 1);
            same &= ((e >> b) & 1) ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (e >= 0 && rank == 0) reinterpret_cast<uint8_t*>(&s.waves[e])[wave] = (uint8_t)__popcll(same);
        __syncthreads();
        int row = -1;
        if (e >= 0) {
            const u32x4 w = s.waves[e];
            int n = s.base[e] + rank;
            // the bytes of waves 0 .. wave - 1
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int k = wave - 4 * q;
                n = byte_sum(k >= 4 ? w[q] : k > 0 ? w[q] & ((1u << (8 * k)) - 1) : 0u, n);
            }
            row = n;
        }
        if (i < i1) p.rows[i] = row;
        if (at + kSortThreads < i1) {
            __syncthreads();
            const u32x4 w = s.waves[tid];
            s.base[tid] += byte_sum(w.x, byte_sum(w.y, byte_sum(w.z, byte_sum(w.w, 0))));
            s.waves[tid] = u32x4{0u, 0u, 0u, 0u};
            __syncthreads();
        }
    }
}

// One launch: every workgroup counts all choices, those before its own 1024 apart, so none waits for another.
template <bool PACKED>
__global__ __launch_bounds__(kSortThreads) void moe_sort_kernel(const SortParams p) {
    __shared__ SortShared s;
    __shared__ int total[kSortMaxGroups + 1];
    int* const before = s.base;
    const int tid = threadIdx.x, start = (int)blockIdx.x * kSortThreads;
    const int own = start + tid < p.n ? sort_expert<PACKED>(p, start + tid) : -1;      // (fetched while the others are counted)
    s.waves[tid] = u32x4{0u, 0u, 0u, 0u};
    before[tid] = 0;
    total[tid] = 0;
    // few experts: several copies of each count, a lane's own, or the lanes of a wave wait for each other (65536 choices
    // of 8 experts 17 us)
    const int shift = min(4, __clz(p.G | 1) - 22), copy = tid & ((1 << shift) - 1);       // 2^shift copies of at most 1023 counts
    __syncthreads();
    if constexpr (PACKED) {
        // four choices a load, eight loads in flight
        constexpr int AHEAD = 8, BATCH = 4 * AHEAD * kSortThreads;
        for (int b = 0; b < p.n; b += BATCH) {
            i32x4 v[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int i = b + (k * kSortThreads + tid) * 4;
                v[k] = i32x4{-1, -1, -1, -1} + p.first;                   // (no expert held here)
                if (i + 4 <= p.n) v[k] = *reinterpret_cast<const i32x4*>(p.ids + i);
                else for (int q = 0; i + q < p.n; ++q) v[k][q] = p.ids[i + q];
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                int* const cnt = (b + (k * kSortThreads + tid) * 4 < start ? before : total) + copy;    // (`start` is a multiple of four)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const unsigned int e = (unsigned int)v[k][q] - (unsigned int)p.first;
                    if (e < (unsigned int)p.G) atomicAdd(&cnt[e << shift], 1);
                }
            }
        }
    } else {
        constexpr int AHEAD = 8;
        for (int b = 0; b < p.n; b += AHEAD * kSortThreads) {
            int e[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int i = b + k * kSortThreads + tid;
                e[k] = i < p.n ? sort_expert<PACKED>(p, i) : -1;
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (e[k] >= 0) atomicAdd((b + k * kSortThreads < start ? before : total) + ((e[k] << shift) + copy), 1);
        }
    }
    __syncthreads();
    int all = 0, mine = 0;
    if (tid < p.G) {
        for (int c = 0; c < 1 << shift; ++c) {
            mine += before[(tid << shift) + c];
            all += total[(tid << shift) + c];
        }
        all += mine;
    }
    const int off = block_exclusive(all, s.part);      // (its barrier: the copies are summed before the sums replace them)
    if (tid < p.G) before[tid] = mine + off;
    if (blockIdx.x == 0 && tid <= p.G) p.offsets[tid] = off;     // (thread G holds no expert: the sum of all)
    __syncthreads();
    place<PACKED>(p, start, min(start + kSortThreads, p.n), own, s);
}

// The long form, for more choices than each workgroup should count: chunks are counted, the counts summed up over the
// chunks, and the chunks placed.  A chunk's counts, then its first free rows, lie where its rows will be (a chunk has at
// least as many choices as there are experts); the last chunk, which may be shorter, is counted where it is needed.
template <bool PACKED>
__device__ __forceinline__ void count_chunk(const SortParams& p, int chunk, int* cnt) {
    cnt[threadIdx.x] = 0;
    __syncthreads();
    const int end = min((chunk + 1) * kSortChunk, p.n);
    for (int i = chunk * kSortChunk + (int)threadIdx.x; i < end; i += kSortThreads) {
        const int e = sort_expert<PACKED>(p, i);
        if (e >= 0) atomicAdd(&cnt[e], 1);
    }
    __syncthreads();
}
template <bool PACKED>
__global__ __launch_bounds__(kSortThreads) void moe_sort_count_kernel(const SortParams p) {
    __shared__ int cnt[kSortMaxGroups + 1];
    count_chunk<PACKED>(p, blockIdx.x, cnt);
    if ((int)threadIdx.x < p.G) p.rows[(int64_t)blockIdx.x * kSortChunk + threadIdx.x] = cnt[threadIdx.x];
}
template <bool PACKED>
__global__ __launch_bounds__(kSortThreads) void moe_sort_scan_kernel(const SortParams p, int chunks) {
    __shared__ int cnt[kSortMaxGroups + 1], part[kSortThreads / 64];
    const int tid = threadIdx.x;
    count_chunk<PACKED>(p, chunks - 1, cnt);
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
template <bool PACKED>
__global__ __launch_bounds__(kSortThreads) void moe_sort_place_kernel(const SortParams p, int chunks) {
    __shared__ SortShared s;
    int* const base = s.base;
    const int tid = threadIdx.x, chunk = blockIdx.x, start = chunk * kSortChunk;
    const int own = start + tid < p.n ? sort_expert<PACKED>(p, start + tid) : -1;
    s.waves[tid] = u32x4{0u, 0u, 0u, 0u};
    if (chunk == chunks - 1) {
        count_chunk<PACKED>(p, chunk, base);
        if (tid < p.G) base[tid] = p.offsets[tid + 1] - base[tid];
    } else if (tid < p.G) {
        base[tid] = p.offsets[tid] + p.rows[(int64_t)chunk * kSortChunk + tid];
    }
    __syncthreads();                                   // (the counts are read before the first rows are written over them)
    place<PACKED>(p, start, min(start + kSortChunk, p.n), own, s);
}

// =============================================================================
// The rows of a token's choices, one a lane (top_k <= 64): the lanes whose choice has a row here, and its row.
// =============================================================================
__device__ __forceinline__ unsigned long long token_rows(const int32_t* rows, int64_t token, int top_k, int64_t total_rows, int lane, int& row) {
    row = lane < top_k ? rows[token * top_k + lane] : -1;
    return __ballot(row >= 0 && row < total_rows);
}

// Eight columns of a row.  NT: with the non-temporal hint (a template parameter: of the two stores behind a branch the
// compiler makes one, without the hint).
template <bool NT, typename V> __device__ __forceinline__ void store16(uint8_t* p, V v) {
    if constexpr (NT) st_nt(p, v);
    else st_stream(p, v);
}
template <typename T, bool NT> __device__ __forceinline__ void store8(uint8_t* p, const float* v, int64_t left) {
    if constexpr (T::EPL == 8) {
        if (left > 0)
            store16<NT>(p, u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])});
    } else {
        if (left > 0) store16<NT>(p, f32x4{v[0], v[1], v[2], v[3]});
        if (left > 4) store16<NT>(p + 16, f32x4{v[4], v[5], v[6], v[7]});
    }
}
template <typename T> __device__ __forceinline__ int64_t bytes_of(int64_t n) { return n * (16 / T::EPL); }

// =============================================================================
// Dispatch: a wave takes NG * 512 columns of one token, a lane eight of each 512 (one 1x128 tile or 128-element block is
// 16 lanes); what it leaves is written to every row of the token's choices.  Bound by memory: 8192 tokens of 7168 columns to
// FP8, one row each on average, 30 us, 4.6 TB/s.
// =============================================================================
template <typename T, DispatchTo TO, int NG>
__global__ __launch_bounds__(256) void moe_dispatch_kernel(const DispatchParams p, int segs) {
    const int lane = threadIdx.x & 63, lane16 = threadIdx.x & 15;
    const unsigned int task = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int64_t token = task / (unsigned)segs;
    if (token >= p.tokens) return;
    const int64_t col0 = (int64_t)(task % (unsigned)segs) * (NG * 512) + lane * 8;
    int row;
    const unsigned long long here = token_rows(p.row_of_slot, token, p.top_k, p.total_rows, lane, row);
    if (here == 0) return;
    Granule8<T> g[NG];
#pragma unroll
    for (int c = 0; c < NG; ++c) g[c].load(p.x + token * p.ldx_bytes + bytes_of<T>(col0 + c * 512), p.cols - col0 - c * 512);
    if constexpr (TO == kDispatchRows) {
        for (unsigned long long todo = here; todo; todo &= todo - 1) {
            const int64_t r = __builtin_amdgcn_readlane(row, __builtin_ctzll(todo));
#pragma unroll
            for (int c = 0; c < NG; ++c) {
                const int64_t col = col0 + c * 512;
                uint8_t* dst = p.y + r * p.ldy_bytes + bytes_of<T>(col);
#pragma unroll
                for (int h = 0; h < Granule8<T>::N; ++h)
                    if (col + h * T::EPL < p.cols) st_stream(dst + h * 16, g[c].g[h]);
            }
        }
    } else {
        unsigned int w0[NG], w1[NG], sw[NG];
#pragma unroll
        for (int c = 0; c < NG; ++c) {
            float v[8];
            g[c].values(v);
            if constexpr (TO == kDispatchFp8) {
                const GroupScale gs = group_scale(as_f32(row16_max_bits(g[c].amax_bits())), p.pow2);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = v[i] * gs.r;
                w0[c] = cvt4_e4m3(v[0], v[1], v[2], v[3]);
                w1[c] = cvt4_e4m3(v[4], v[5], v[6], v[7]);
                sw[c] = as_u32(gs.s);
            } else {
                const MxScale ms = mx_scale(quad_max_bits(g[c].amax_bits()));
                w0[c] = cvt8_e2m1(v, ms.r);
                sw[c] = row16_scale_word(ms.e, lane16);
            }
        }
        for (unsigned long long todo = here; todo; todo &= todo - 1) {
            const int64_t r = __builtin_amdgcn_readlane(row, __builtin_ctzll(todo));
#pragma unroll
            for (int c = 0; c < NG; ++c) {
                const int64_t col = col0 + c * 512, left = p.cols - col;
                if (left <= 0) break;
                if constexpr (TO == kDispatchFp8) {
                    uint8_t* dst = p.y + r * p.ldy_bytes + col;
                    if (left >= 8) st_stream(dst, u32x2{w0[c], w1[c]});
                    else st_stream(dst, w0[c]);
                } else {
                    uint8_t* dst = p.y + r * p.ldy_bytes + (col >> 1);
                    if (left >= 8) st_stream(dst, w0[c]);
                    else st_stream(dst, (uint16_t)w0[c]);
                }
                if (lane16 == 0) static_cast<uint32_t*>(p.s)[r * p.ssr + (col >> 7) * p.ssk] = sw[c];
            }
        }
    }
}

// =============================================================================
// Combine: the same split; NR rows are in flight at a time.  Bound by memory: of 8192 rows back to 8192 tokens 42 us, 5.6 TB/s.
// =============================================================================
template <typename TY, typename TO, int NG, bool NT>
__global__ __launch_bounds__(256) void moe_combine_kernel(const CombineParams p, int segs) {
    constexpr int NR = 4;
    const int lane = threadIdx.x & 63;
    const unsigned int task = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int64_t token = task / (unsigned)segs;
    if (token >= p.tokens) return;
    const int64_t col0 = (int64_t)(task % (unsigned)segs) * (NG * 512) + lane * 8;
    int row;
    unsigned long long todo = token_rows(p.row_of_slot, token, p.top_k, p.total_rows, lane, row);
    float weight = 1.f;
    if (p.w != nullptr && lane < p.top_k) weight = p.w[token * p.top_k + lane];
    float acc[NG][8];
#pragma unroll
    for (int c = 0; c < NG; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[c][e] = 0.f;
    while (todo) {
        Granule8<TY> g[NR][NG];
        float w[NR];
        int n = 0;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            if (todo) {
                const int s = __builtin_ctzll(todo);
                todo &= todo - 1;
                w[i] = as_f32((unsigned int)__builtin_amdgcn_readlane((int)as_u32(weight), s));
                const uint8_t* y = p.y + (int64_t)__builtin_amdgcn_readlane(row, s) * p.ldy_bytes;
#pragma unroll
                for (int c = 0; c < NG; ++c) g[i][c].load(y + bytes_of<TY>(col0 + c * 512), p.cols - col0 - c * 512);
                n = i + 1;
            }
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            if (i < n) {
#pragma unroll
                for (int c = 0; c < NG; ++c) {
                    float v[8];
                    g[i][c].values(v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[c][e] = __builtin_fmaf(w[i], v[e], acc[c][e]);
                }
            }
        }
    }
#pragma unroll
    for (int c = 0; c < NG; ++c)
        store8<TO, NT>(p.out + token * p.ldo_bytes + bytes_of<TO>(col0 + c * 512), acc[c], p.cols - col0 - c * 512);
}

// =============================================================================
// Combine's gradients: a wave takes a choice, the choices of a token side by side, so that the token's gradient comes
// from memory once.  dy is the weight times that gradient; dw is summed lane by lane over the columns, then over the
// lanes, always in the same order.  Bound by memory: the same rows 54.5 us, 5.7 TB/s.
// =============================================================================
template <typename TY, typename TO, bool NT>
__global__ __launch_bounds__(256) void moe_combine_bwd_kernel(const CombineParams p) {
    constexpr int NG = 4;
    const int lane = threadIdx.x & 63;
    const int64_t choice = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (choice >= p.tokens * p.top_k) return;
    const int64_t token = (unsigned int)choice / (unsigned int)p.top_k;
    const int64_t r = p.row_of_slot[choice];
    float dot = 0.f;
    if (r >= 0 && r < p.total_rows) {
        const float w = p.w != nullptr ? p.w[choice] : 1.f;
        const uint8_t* const d = p.out + token * p.ldo_bytes;
        const uint8_t* const y = p.y + r * p.ldy_bytes;
        uint8_t* const dy = p.dy + r * p.lddy_bytes;
        for (int64_t c0 = lane * 8; c0 < p.cols; c0 += NG * 512) {
            Granule8<TO> dg[NG];
            Granule8<TY> yg[NG];
#pragma unroll
            for (int c = 0; c < NG; ++c) dg[c].load_kept(d + bytes_of<TO>(c0 + c * 512), p.cols - c0 - c * 512);
#pragma unroll
            for (int c = 0; c < NG; ++c) yg[c].load(y + bytes_of<TY>(c0 + c * 512), p.cols - c0 - c * 512);
#pragma unroll
            for (int c = 0; c < NG; ++c) {
                float dv[8], yv[8];
                dg[c].values(dv);
                yg[c].values(yv);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    dot = __builtin_fmaf(dv[e], yv[e], dot);
                    dv[e] *= w;
                }
                store8<TY, NT>(dy + bytes_of<TY>(c0 + c * 512), dv, p.cols - c0 - c * 512);
            }
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) dot += __shfl_xor(dot, m);
    }
    if (lane == 0) p.dw[choice] = dot;
}

// ---- host side -------------------------------------------------------------------
static ds3_status launch_status() { return hipGetLastError() == hipSuccess ? DS3_OK : DS3_ERR_LAUNCH; }
constexpr int64_t kMaxGrid = (1ll << 24) - 1;          // a grid may have 2^32 threads

// Up to here every workgroup counts all choices itself (65536 of 256 experts 10 us, of which 32 are here 8; the long form
// takes three launches, of 4, 4 and 13 us at 65536).  In all, 131072 of 256 experts in one launch 13 us, 131080 in three 14,
// 262144 17, a million 30.  Below the second line four choices a load do not pay for the longer kernel (32 choices: 3.4 / 4.6
// us, 16384: 8.0 / 7.2, 65536: 17 / 10).
constexpr int kSortOneLaunch = 131072, kSortPacked = 8192;

template <bool PACKED>
static ds3_status sort_as(const SortParams& p, hipStream_t st) {
    (void)hipGetLastError();                            // a stale error of earlier, unrelated work is not this launch's
    if (p.n <= kSortOneLaunch) {
        const int blocks = std::max(1, (p.n + kSortThreads - 1) / kSortThreads);
        moe_sort_kernel<PACKED><<<dim3(blocks), kSortThreads, 0, st>>>(p);
        return launch_status();
    }
    const int chunks = (p.n + kSortChunk - 1) / kSortChunk;
    moe_sort_count_kernel<PACKED><<<dim3(chunks - 1), kSortThreads, 0, st>>>(p);
    moe_sort_scan_kernel<PACKED><<<dim3(1), kSortThreads, 0, st>>>(p, chunks);
    moe_sort_place_kernel<PACKED><<<dim3(chunks), kSortThreads, 0, st>>>(p, chunks);
    return launch_status();
}

ds3_status launch_moe_sort(const int32_t* ids, int64_t tokens, int top_k, int64_t ld, int first, int G, int32_t* offsets,
                           int32_t* row_of_slot, hipStream_t st) {
    const SortParams p{ids, ld, (int)(tokens * top_k), top_k, first, G, offsets, row_of_slot};
    const bool packed = ld == top_k && (reinterpret_cast<uintptr_t>(ids) & 15u) == 0 && p.n > kSortPacked;
    return packed ? sort_as<true>(p, st) : sort_as<false>(p, st);
}

template <typename T, int NG>
static void dispatch_as(const DispatchParams& p, DispatchTo to, unsigned grid, int segs, hipStream_t st) {
    if (to == kDispatchRows) moe_dispatch_kernel<T, kDispatchRows, NG><<<dim3(grid), 256, 0, st>>>(p, segs);
    else if (to == kDispatchFp8) moe_dispatch_kernel<T, kDispatchFp8, NG><<<dim3(grid), 256, 0, st>>>(p, segs);
    else moe_dispatch_kernel<T, kDispatchMx4, NG><<<dim3(grid), 256, 0, st>>>(p, segs);
}

// Columns a wave takes, in units of 512: the more, the more is in flight and the fewer waves look up a token's rows; few
// tokens want more waves.  us with 1 / 2 / 4 units, 7168 columns: FP8, 8192 tokens with one row each on average 35 / 29 / 30,
// MXFP4 33 / 26 / 24, eight rows each 93 / 95 / 96; 64 tokens 4.0 / 4.3 / 5.3; 2048 columns of FP8 17.4 / 17.1 / 14.7.
static int columns_per_wave(int64_t tokens, int64_t cols) {
    const int64_t units = (cols + 511) / 512;
    return tokens * units < 4096 ? 1 : units >= 3 ? 4 : units >= 2 ? 2 : 1;
}
// Workgroups of four waves for every token's columns; 0: more than a grid holds.
static unsigned wave_grid(int64_t tokens, int64_t cols, int ng, int* segs) {
    const int64_t s = (cols + ng * 512 - 1) / (ng * 512);
    if (s > kMaxGrid || tokens > kMaxGrid * 4 / s) return 0;
    *segs = (int)s;
    return (unsigned)((tokens * s + 3) / 4);
}

ds3_status launch_moe_dispatch(const DispatchParams& p, ds3_dtype xt, DispatchTo to, hipStream_t st) {
    int ng = columns_per_wave(p.tokens, p.cols);
    // (rows as they are, about one a token: 8192 x 7168 BF16 37 / 38 / 40 us with 1 / 2 / 4 units; eight a token 211 / 212 / 208)
    if (to == kDispatchRows && p.total_rows < 2 * p.tokens) ng = std::min(ng, 2);
    int segs;
    const unsigned grid = wave_grid(p.tokens, p.cols, ng, &segs);
    if (grid == 0) return DS3_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    if (xt == DS3_BF16) {
        if (ng == 4) dispatch_as<Bf16, 4>(p, to, grid, segs, st);
        else if (ng == 2) dispatch_as<Bf16, 2>(p, to, grid, segs, st);
        else dispatch_as<Bf16, 1>(p, to, grid, segs, st);
    } else {
        if (ng == 4) dispatch_as<F32, 4>(p, to, grid, segs, st);
        else if (ng == 2) dispatch_as<F32, 2>(p, to, grid, segs, st);
        else dispatch_as<F32, 1>(p, to, grid, segs, st);
    }
    return launch_status();
}

// Whether what combine and its gradients write carries the non-temporal hint: where it is so much that little of it would be
// left in the caches for the next reader.  us without / with it: gradients of 8192 tokens of 7168 columns, one row each on
// average (117 MB), 68 / 56, eight (940 MB) 405 / 394, of 512 tokens with eight (59 MB) 23.4 / 25.2; the sums of 8192 tokens
// with eight 192 / 184.
static bool streams_past(int64_t rows, int64_t row_bytes) { return rows * row_bytes >= (64ll << 20); }

template <typename TY, typename TO, bool NT>
static void combine_as(const CombineParams& p, int ng, unsigned grid, int segs, hipStream_t st) {
    if (ng == 1) moe_combine_kernel<TY, TO, 1, NT><<<dim3(grid), 256, 0, st>>>(p, segs);
    else moe_combine_kernel<TY, TO, 2, NT><<<dim3(grid), 256, 0, st>>>(p, segs);
}
template <typename TY, typename TO>
static ds3_status combine(const CombineParams& p, hipStream_t st) {
    // (8192 tokens of 7168 columns with one row each on average, 1 / 2 units: 47 / 43 us; 64 tokens with eight 4.3 / 5.3)
    const int ng = std::min(2, columns_per_wave(p.tokens, p.cols));
    int segs;
    const unsigned grid = wave_grid(p.tokens, p.cols, ng, &segs);
    if (grid == 0) return DS3_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    if (streams_past(p.tokens, p.cols * (16 / TO::EPL))) combine_as<TY, TO, true>(p, ng, grid, segs, st);
    else combine_as<TY, TO, false>(p, ng, grid, segs, st);
    return launch_status();
}
template <typename TY, typename TO>
static ds3_status combine_bwd(const CombineParams& p, hipStream_t st) {
    const int64_t n = (p.tokens * p.top_k + 3) / 4;
    if (n > kMaxGrid) return DS3_ERR_UNSUPPORTED;
    (void)hipGetLastError();
    const dim3 grid((unsigned)n);
    if (streams_past(std::min(p.total_rows, p.tokens * p.top_k), p.cols * (16 / TY::EPL))) moe_combine_bwd_kernel<TY, TO, true><<<grid, 256, 0, st>>>(p);
    else moe_combine_bwd_kernel<TY, TO, false><<<grid, 256, 0, st>>>(p);
    return launch_status();
}

ds3_status launch_moe_combine(const CombineParams& p, ds3_dtype yt, ds3_dtype ot, hipStream_t st) {
    if (yt == DS3_BF16) return ot == DS3_BF16 ? combine<Bf16, Bf16>(p, st) : combine<Bf16, F32>(p, st);
    return ot == DS3_BF16 ? combine<F32, Bf16>(p, st) : combine<F32, F32>(p, st);
}

ds3_status launch_moe_combine_bwd(const CombineParams& p, ds3_dtype yt, ds3_dtype ot, hipStream_t st) {
    if (yt == DS3_BF16) return ot == DS3_BF16 ? combine_bwd<Bf16, Bf16>(p, st) : combine_bwd<Bf16, F32>(p, st);
    return ot == DS3_BF16 ? combine_bwd<F32, Bf16>(p, st) : combine_bwd<F32, F32>(p, st);
}

}  // namespace ds3
