// The paged cache of keys and values, sm_100a: rows of new tokens encoded as they are written, and rows read back.
//
//     cell(page, head, slot) = (page * heads + head) * page_size + slot,   row i -> (sequence s, position t = starts[s] + i - offsets[s])
//                                                                        -> page table[s][t / page_size], slot t % page_size
// A cell holds C = 32 ceil(d / 32) channels: 16-bit values, E4M3 codes or packed E2M1 codes; its scale row one E8M0 byte per 32 channels.
// Pages keep a head's positions together ([pages][heads][page_size]): the attention reads one head at a time and finds whole
// lines.  Encoder per 32 channels, as in the quantizer:  S = max(floor(log2 amax) - e + 127, 0),  code = rn(y 2^(127 - S)), saturating.
//
// Both directions are bound by memory (2 bytes of 16-bit values and 0.53, 1.03 or 2 bytes of cache per element) or, for a few rows,
// by latency.  A thread keeps a place within a row, 16 channels of one head, and walks the rows of its CTA, so that what it computes
// per 16 channels is two addresses and the code; the two threads of a block of 32 channels exchange its largest magnitude by one
// shuffle.  The cell of a row (a search of offsets and one table entry) is found once per CTA and row.
// Measured: 2823 new rows into and 32823 rows out of an MXFP4 cache of 8 heads x 128 39.8 us, of which the read takes 30: 134 MB of writes at
// 4.4 TB/s, the rate at which this device is filled.  The write waits for offsets, starts, table and a barrier one after another before it asks for
// its first row: 9 us from memory (2.2 of bytes), 5.5 with rows in L2 (MXFP8 5.6, 16 bits 8.4).
#pragma once
#include "kq_mma16.cuh"
#include "kq_rotary.cuh"

namespace kq {

enum { kCache16 = 0, kCacheFp8 = 1, kCacheFp4 = 2 };

struct CacheRef {
    int format;
    int64_t pages;
    int page_size, heads, head_dim;
    int blocks;                          // ceil(head_dim / 32)
    int scale_row;                       // bytes of a scale row
    uint8_t *k, *v, *k_scales, *v_scales;
    FastDiv by_page;                     // page_size
    __host__ __device__ int row_bytes() const { return format == kCache16 ? 64 * blocks : format == kCacheFp8 ? 32 * blocks : 16 * blocks; }
};

// Cell of head 0 at a position (the heads' cells are page_size apart), -1 without a place.
__device__ __forceinline__ int64_t cache_cell(const CacheRef& c, const int32_t* table_row, int table_width, int64_t position) {
    if (position < 0 || position >= (int64_t)table_width * c.page_size) return -1;
    const uint32_t entry = position < 0x7FFFFFFF ? c.by_page.div((uint32_t)position) : (uint32_t)(position / c.page_size);
    const int page = table_row[entry];
    if (page < 0 || page >= c.pages) return -1;
    return (int64_t)page * c.heads * c.page_size + (position - (int64_t)entry * c.page_size);
}

struct CacheRows {
    int64_t rows;
    int sequences;
    const int32_t* table;
    int64_t table_stride;
    int table_width;
    const int32_t *offsets, *starts;
    void *k, *v;
    int64_t k_row, k_head, v_row, v_head;
    int rows_per_cta;
    int units;                           // of a row: heads * groups of 16 channels
    FastDiv by_groups;
};

// cells[i]: of row row0 + i for head 0; -1: no place, -2: a row of no sequence.  All threads of the CTA, one per row.
__device__ __forceinline__ void find_cells(const CacheRef& c, const CacheRows& p, int64_t row0, int rows, int64_t* cells, int thread, int threads) {
    for (int i = thread; i < rows; i += threads) {
        const int64_t row = row0 + i;
        int s = (int)row;
        int64_t first = row;
        bool exists = true;
        if (p.offsets) {
            int lo = 0, hi = p.sequences;                                // the last sequence whose offset is <= row (offsets out of order: some sequence)
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (p.offsets[mid] <= row) lo = mid; else hi = mid;
            }
            s = lo;
            first = p.offsets[s];
            exists = row >= first && row < p.offsets[s + 1];
        }
        const int64_t position = (p.starts ? (int64_t)p.starts[s] : 0) + (row - first);
        cells[i] = exists ? cache_cell(c, p.table + (int64_t)s * p.table_stride, p.table_width, position) : -2;
    }
    __syncthreads();
}

// ---- codes -----------------------------------------------------------------------------------------
// eight values to eight E4M3 codes, channel order kept
__device__ __forceinline__ uint2 e4m3x8(const float (&v)[8]) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint16_t two;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        h[i] = two;
    }
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}
__device__ __forceinline__ float2 scale_pair(float2 f, float scale) {
    unsigned long long v, s;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(f.x), "f"(f.y));
    asm("mov.b64 %0, {%1, %1};" : "=l"(s) : "f"(scale));
    asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(v) : "l"(s));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
    return f;
}
__device__ __forceinline__ void store_32_bytes(void* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g, uint32_t h) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"l"(p), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f), "r"(g), "r"(h) : "memory");
}

constexpr int kCacheThreads = 256;       // at most
constexpr int kCacheRowsMax = 256;       // rows of a CTA

// blockDim: x = units of a row (or 256 of them), y = rows at a time.  blockIdx.y: keys, values.  T: type of the rows.  VEC: rows allow
// 16-byte accesses and head_dim is a multiple of 8.
template <typename T, int FORMAT, bool VEC>
__global__ void __launch_bounds__(kCacheThreads) cache_write_kernel(const __grid_constant__ CacheRef c, const __grid_constant__ CacheRows p) {
    __shared__ int64_t cells[kCacheRowsMax];
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_cta;
    const int rows = (int)(p.rows - row0 < p.rows_per_cta ? p.rows - row0 : p.rows_per_cta);
    const int thread = threadIdx.y * blockDim.x + threadIdx.x;
    find_cells(c, p, row0, rows, cells, thread, blockDim.x * blockDim.y);
    const bool values = blockIdx.y != 0;
    const int64_t row_stride = values ? p.v_row : p.k_row, head_stride = values ? p.v_head : p.k_head;
    const T* src = static_cast<const T*>(values ? p.v : p.k) + row0 * row_stride;
    const int groups = 2 * c.blocks;
    const uint32_t row_bytes = (uint32_t)c.row_bytes();
    // (the units of a block of 32 channels are two neighbouring lanes, which pass or fail every test but the channel's together)
    const uint32_t pair = 3u << (thread & 30);
    for (int u = threadIdx.x; u < p.units; u += blockDim.x) {
        const int head = (int)p.by_groups.div((uint32_t)u), g = u - head * groups, left = c.head_dim - 16 * g;
        const T* from = src + head * head_stride + 16 * g;
        const uint64_t head_cells = (uint64_t)head * c.page_size;
        uint8_t* codes = (values ? c.v : c.k) + head_cells * row_bytes + g * (FORMAT == kCache16 ? 32 : FORMAT == kCacheFp8 ? 16 : 8);
        uint8_t* scales = (values ? c.v_scales : c.k_scales) + head_cells * c.scale_row + (g >> 1);
#pragma unroll 2
        for (int r = threadIdx.y; r < rows; r += blockDim.y) {
            const int64_t cell = cells[r];
            if (cell < 0) continue;
            const T* at = from + r * row_stride;
            uint32_t w[8];                                               // sixteen 16-bit values
            if (VEC) {
                const uint4 zero = make_uint4(0, 0, 0, 0);
                const uint4 a = left > 0 ? ld_stream_16(at) : zero, b = left > 8 ? ld_stream_16(at + 8) : zero;
                w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
            } else {
                const uint16_t* q = reinterpret_cast<const uint16_t*>(at);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w[i] = (2 * i < left ? (uint32_t)q[2 * i] : 0u) | (2 * i + 1 < left ? (uint32_t)q[2 * i + 1] << 16 : 0u);
            }
            uint8_t* to = codes + (uint64_t)(uint32_t)cell * row_bytes;
            if constexpr (FORMAT == kCache16) {
                reinterpret_cast<uint4*>(to)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                reinterpret_cast<uint4*>(to)[1] = make_uint4(w[4], w[5], w[6], w[7]);
            } else {
                float v[8], x[8];
                widen8_any<__is_same(T, __half)>(make_uint4(w[0], w[1], w[2], w[3]), v);
                widen8_any<__is_same(T, __half)>(make_uint4(w[4], w[5], w[6], w[7]), x);
                float amax = fmaxf(absmax8(v), absmax8(x));
                amax = fmaxf(amax, __shfl_xor_sync(pair, amax, 1));
                const int e = (int)((__float_as_uint(amax) >> 23) & 0xFFu) - (FORMAT == kCacheFp8 ? 8 : 2);
                const uint32_t S = (uint32_t)(e < 0 ? 0 : e);
                const float inv = inv_scale_from_e8m0(S);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[i] *= inv;
                    x[i] *= inv;
                }
                if constexpr (FORMAT == kCacheFp8) {
                    const uint2 a = e4m3x8(v), b = e4m3x8(x);
                    *reinterpret_cast<uint4*>(to) = make_uint4(a.x, a.y, b.x, b.y);
                } else {
                    *reinterpret_cast<uint2*>(to) = make_uint2(e2m1x8(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]),
                                                               e2m1x8(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]));
                }
                if ((g & 1) == 0) {
                    uint8_t* s = scales + (uint64_t)(uint32_t)cell * c.scale_row;
                    s[0] = (uint8_t)S;
                    if ((g >> 1) == c.blocks - 1)
                        for (int b = c.blocks; b < c.scale_row; ++b) s[b - c.blocks + 1] = 0;
                }
            }
        }
    }
}

// sixteen values to a row of T: `width` 32 or 16 bytes at a time (all of them, or the first eight), or the first `left` one by one
template <typename T>
__device__ __forceinline__ void cache_store16(T* at, int left, int width, const float (&v)[16]) {
    if (width) {
        constexpr int kWords = sizeof(T) == 4 ? 16 : 8;
        uint32_t w[kWords];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (sizeof(T) == 4) {
                w[2 * i] = __float_as_uint(v[2 * i]);
                w[2 * i + 1] = __float_as_uint(v[2 * i + 1]);
            } else if constexpr (__is_same(T, __half)) {
                w[i] = pack_f16(v[2 * i], v[2 * i + 1]);
            } else {
                w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
            }
        }
        uint32_t* to = reinterpret_cast<uint32_t*>(at);
        if (width == 32) {
#pragma unroll
            for (int i = 0; i < kWords; i += 8) store_32_bytes(to + i, w[i], w[i + 1], w[i + 2], w[i + 3], w[i + 4], w[i + 5], w[i + 6], w[i + 7]);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4)
                if (i < kWords / 2 || left > 8) st_stream_16(to + i, make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < left) at[i] = rotary_round<T>(v[i]);
    }
}

// CF16: a 16-bit cache holds fp16 (else bf16).  T: type of the rows.  width: bytes of a store to them (32, 16 or, for any alignment, 0).
// blockDim and blockIdx as above.
template <typename T, int FORMAT, bool CF16>
__global__ void __launch_bounds__(kCacheThreads) cache_read_kernel(const __grid_constant__ CacheRef c, const __grid_constant__ CacheRows p, const int width) {
    constexpr int kAhead = FORMAT == kCache16 ? 2 : 4;                   // rows of a thread in flight
    constexpr int kWords = FORMAT == kCache16 ? 8 : (FORMAT == kCacheFp8 ? 4 : 2);
    __shared__ int64_t cells[kCacheRowsMax];
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_cta;
    const int rows = (int)(p.rows - row0 < p.rows_per_cta ? p.rows - row0 : p.rows_per_cta);
    find_cells(c, p, row0, rows, cells, threadIdx.y * blockDim.x + threadIdx.x, blockDim.x * blockDim.y);
    const bool values = blockIdx.y != 0;
    const int64_t row_stride = values ? p.v_row : p.k_row, head_stride = values ? p.v_head : p.k_head;
    T* dst = static_cast<T*>(values ? p.v : p.k) + row0 * row_stride;
    const int groups = (c.head_dim + 15) / 16, step = blockDim.y;
    const uint32_t row_bytes = (uint32_t)c.row_bytes();
    for (int u = threadIdx.x; u < p.units; u += blockDim.x) {
        const int head = (int)p.by_groups.div((uint32_t)u), g = u - head * groups, left = c.head_dim - 16 * g;
        T* to = dst + head * head_stride + 16 * g;
        const uint64_t head_cells = (uint64_t)head * c.page_size;
        const uint8_t* codes = (values ? c.v : c.k) + head_cells * row_bytes + g * 4 * kWords;
        const uint8_t* scales = (values ? c.v_scales : c.k_scales) + head_cells * c.scale_row + (g >> 1);
        for (int r0 = threadIdx.y; r0 < rows; r0 += kAhead * step) {
            uint32_t w[kAhead][kWords], S[kAhead];
            int64_t cell[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                cell[k] = r0 + k * step < rows ? cells[r0 + k * step] : -2;
                S[k] = 0;
#pragma unroll
                for (int i = 0; i < kWords; ++i) w[k][i] = 0;
                if (cell[k] < 0) continue;
                const uint8_t* at = codes + (uint64_t)(uint32_t)cell[k] * row_bytes;
                if constexpr (FORMAT == kCacheFp4) {
                    const uint2 q = *reinterpret_cast<const uint2*>(at);
                    w[k][0] = q.x; w[k][1] = q.y;
                } else {
#pragma unroll
                    for (int i = 0; i < kWords / 4; ++i) {
                        const uint4 q = reinterpret_cast<const uint4*>(at)[i];
                        w[k][4 * i] = q.x; w[k][4 * i + 1] = q.y; w[k][4 * i + 2] = q.z; w[k][4 * i + 3] = q.w;
                    }
                }
                if constexpr (FORMAT != kCache16) S[k] = scales[(uint64_t)(uint32_t)cell[k] * c.scale_row];
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (cell[k] == -2) continue;
                T* at = to + (r0 + k * step) * row_stride;
                float v[16];
                if constexpr (FORMAT == kCache16) {
                    float a[8], b[8];
                    widen8_any<CF16>(make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]), a);
                    widen8_any<CF16>(make_uint4(w[k][4], w[k][5], w[k][6], w[k][7]), b);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        v[i] = a[i];
                        v[8 + i] = b[i];
                    }
                } else {
                    const float scale = scale_from_e8m0(S[k]);
#pragma unroll
                    for (int i = 0; i < kWords; ++i) {
                        uint32_t h[4];
                        if constexpr (FORMAT == kCacheFp8) e4m3x4_to_f16(w[k][i], h[0], h[1]);
                        else e2m1x8_to_f16(w[k][i], h);
                        constexpr int kPairs = FORMAT == kCacheFp8 ? 2 : 4;
#pragma unroll
                        for (int q = 0; q < kPairs; ++q) {
                            const float2 f = scale_pair(__half22float2(*reinterpret_cast<const __half2*>(&h[q])), scale);
                            v[2 * (kPairs * i + q)] = f.x;
                            v[2 * (kPairs * i + q) + 1] = f.y;
                        }
                    }
                }
                cache_store16<T>(at, left, width, v);
            }
        }
    }
}

}  // namespace kq
