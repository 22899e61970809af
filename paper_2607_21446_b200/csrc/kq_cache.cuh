// The paged cache of keys and values, sm_100a: rows of new tokens encoded as they are written, and rows read back.
//
//     cell(page, head, slot) = (page * heads + head) * page_size + slot,   row i -> (sequence s, position t = starts[s] + i - offsets[s])
//                                                                        -> page table[s][t / page_size], slot t % page_size
// A cell holds C = 32 ceil(d / 32) channels: 16-bit values, E4M3 codes or packed E2M1 codes; its scale row one E8M0 byte per 32 channels.
// Pages keep a head's positions together ([pages][heads][page_size]): the attention reads one head at a time and finds whole
// lines.  Encoder per 32 channels, as in the quantizer:  S = max(floor(log2 amax) - e + 127, 0),  code = rn(y 2^(127 - S)), saturating.
//
// Both directions are bound by memory (2 bytes of 16-bit values and 0.53, 1.03 or 2 bytes of cache per element) or, for a few rows,
// by latency.  A thread takes 8 channels of a row at a time, 16 bytes of it; the four threads of a block of 32 channels exchange
// its largest magnitude by two shuffles.  The place of a row (a search of offsets by one warp, 32 entries at a time, and one table
// entry) is found once per CTA and row.
#pragma once
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

struct CachePlace { int page, slot; };   // page -1: no place, -2: a row of no sequence
__device__ __forceinline__ CachePlace cache_place(const CacheRef& c, const int32_t* table_row, int table_width, int64_t position) {
    if (position < 0 || position >= (int64_t)table_width * c.page_size) return {-1, 0};
    const uint32_t entry = position < 0x7FFFFFFF ? c.by_page.div((uint32_t)position) : (uint32_t)(position / c.page_size);
    const int page = __ldg(table_row + entry);
    if (page < 0 || page >= c.pages) return {-1, 0};
    return {page, (int)(position - (int64_t)entry * c.page_size)};
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
    int units;                           // of a row: heads * groups
    FastDiv by_units, by_groups;         // units of a row, groups of 8 channels of a head
};

// The last sequence whose offset is <= row, by one warp: 32 entries at a time.
__device__ __forceinline__ int find_sequence(const int32_t* offsets, int sequences, int64_t row, int lane) {
    int lo = 0, count = sequences;                                       // offsets[lo] <= row < offsets[lo + count] where row has one
    while (count > 1) {
        const int step = (count + 31) / 32;
        const int at = lane * step;
        const bool below = at < count && (lane == 0 || __ldg(offsets + lo + at) <= row);
        const uint32_t mask = __ballot_sync(0xFFFFFFFFu, below);
        const int last = 31 - __clz(mask);                                // (with offsets out of order: some entry, in range all the same)
        lo += last * step;
        count = count - last * step < step ? count - last * step : step;
    }
    return lo;
}
// places[i]: of row row0 + i.  All warps of the CTA.
__device__ __forceinline__ void find_places(const CacheRef& c, const CacheRows& p, int64_t row0, int rows, CachePlace* places) {
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x >> 5; i < rows; i += blockDim.x >> 5) {
        const int64_t row = row0 + i;
        int s = (int)row;
        int64_t first = row;
        bool exists = true;
        if (p.offsets) {
            s = find_sequence(p.offsets, p.sequences, row, lane);
            first = __ldg(p.offsets + s);
            exists = row >= first && row < __ldg(p.offsets + s + 1);
        }
        if (lane == 0) {
            const int64_t position = (p.starts ? (int64_t)__ldg(p.starts + s) : 0) + (row - first);
            places[i] = exists ? cache_place(c, p.table + (int64_t)s * p.table_stride, p.table_width, position) : CachePlace{-2, 0};
        }
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
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t two) {
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((uint16_t)two));
    return __half22float2(*reinterpret_cast<const __half2*>(&h2));
}

constexpr int kCacheThreads = 256;
constexpr int kCacheRowsMax = 64;        // rows of a CTA

// blockIdx.y: keys, values.  T: type of the rows.  VEC: rows allow 16-byte accesses and head_dim is a multiple of 8.
template <typename T, int FORMAT, bool VEC>
__global__ void __launch_bounds__(kCacheThreads) cache_write_kernel(const __grid_constant__ CacheRef c, const __grid_constant__ CacheRows p) {
    __shared__ CachePlace places[kCacheRowsMax];
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_cta;
    const int rows = (int)(p.rows - row0 < p.rows_per_cta ? p.rows - row0 : p.rows_per_cta);
    find_places(c, p, row0, rows, places);
    const bool values = blockIdx.y != 0;
    const T* src = static_cast<const T*>(values ? p.v : p.k);
    const int64_t row_stride = values ? p.v_row : p.k_row, head_stride = values ? p.v_head : p.k_head;
    uint8_t* codes = values ? c.v : c.k;
    uint8_t* scales = values ? c.v_scales : c.k_scales;
    const int groups = 4 * c.blocks, total = rows * p.units, row_bytes = c.row_bytes();
    // (units of a block of 32 channels are four neighbours: whole quads of lanes pass or fail every test below but the channel's)
    for (int u = threadIdx.x; u < total; u += kCacheThreads) {
        const int r = (int)p.by_units.div((uint32_t)u), rest = u - r * p.units;
        const int head = (int)p.by_groups.div((uint32_t)rest), g = rest - head * groups;
        const CachePlace place = places[r];
        if (place.page < 0) continue;
        const int64_t cell = ((int64_t)place.page * c.heads + head) * c.page_size + place.slot;
        const T* at = src + (row0 + r) * row_stride + head * head_stride + 8 * g;
        const int left = c.head_dim - 8 * g;
        uint32_t w[4] = {0, 0, 0, 0};                                    // eight 16-bit values
        if (VEC) {
            if (left > 0) {
                const uint4 q = ld_stream_16(at);
                w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
            }
        } else {
            const uint16_t* q = reinterpret_cast<const uint16_t*>(at);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left) w[i / 2] |= (uint32_t)q[i] << (16 * (i & 1));
        }
        if constexpr (FORMAT == kCache16) {
            *reinterpret_cast<uint4*>(codes + cell * row_bytes + 16 * g) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            float v[8];
            widen8_any<__is_same(T, __half)>(make_uint4(w[0], w[1], w[2], w[3]), v);
            float amax = absmax8(v);
            const uint32_t quad = 0xFu << (threadIdx.x & 28);
            amax = fmaxf(amax, __shfl_xor_sync(quad, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(quad, amax, 2));
            const int e = (int)((__float_as_uint(amax) >> 23) & 0xFFu) - (FORMAT == kCacheFp8 ? 8 : 2);
            const uint32_t S = (uint32_t)(e < 0 ? 0 : e);
            const float inv = inv_scale_from_e8m0(S);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= inv;
            if constexpr (FORMAT == kCacheFp8)
                *reinterpret_cast<uint2*>(codes + cell * row_bytes + 8 * g) = e4m3x8(v);
            else
                *reinterpret_cast<uint32_t*>(codes + cell * row_bytes + 4 * g) = e2m1x8(v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]);
            if ((g & 3) == 0) {
                uint8_t* s = scales + cell * c.scale_row;
                s[g >> 2] = (uint8_t)S;
                if ((g >> 2) == c.blocks - 1)
                    for (int b = c.blocks; b < c.scale_row; ++b) s[b] = 0;
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ void cache_store8(T* at, int left, bool vec, const float (&v)[8]) {
    if (vec) {
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4*>(at)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(at)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (__is_same(T, __half)) {
                    const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t*>(&h);
                } else {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t*>(&h);
                }
            }
            st_stream_16(at, make_uint4(w[0], w[1], w[2], w[3]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) at[i] = rotary_round<T>(v[i]);
    }
}

constexpr int kReadAhead = 4;            // units of a thread in flight

// CF16: a 16-bit cache holds fp16 (else bf16).  T: type of the rows.
template <typename T, int FORMAT, bool CF16>
__global__ void __launch_bounds__(kCacheThreads) cache_read_kernel(const __grid_constant__ CacheRef c, const __grid_constant__ CacheRows p, const int vec) {
    __shared__ CachePlace places[kCacheRowsMax];
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_cta;
    const int rows = (int)(p.rows - row0 < p.rows_per_cta ? p.rows - row0 : p.rows_per_cta);
    find_places(c, p, row0, rows, places);
    const bool values = blockIdx.y != 0;
    T* dst = static_cast<T*>(values ? p.v : p.k);
    const int64_t row_stride = values ? p.v_row : p.k_row, head_stride = values ? p.v_head : p.k_head;
    const uint8_t* codes = values ? c.v : c.k;
    const uint8_t* scales = values ? c.v_scales : c.k_scales;
    const int groups = (c.head_dim + 7) / 8, total = rows * p.units, row_bytes = c.row_bytes();
    for (int u0 = threadIdx.x; u0 < total; u0 += kReadAhead * kCacheThreads) {
        uint4 w[kReadAhead];
        uint32_t S[kReadAhead];
        int left[kReadAhead];                                            // channels to write; 0: no unit
        T* at[kReadAhead];
#pragma unroll
        for (int k = 0; k < kReadAhead; ++k) {
            const int u = u0 + k * kCacheThreads;
            left[k] = 0;
            w[k] = make_uint4(0, 0, 0, 0);
            S[k] = 0;
            if (u >= total) continue;
            const int r = (int)p.by_units.div((uint32_t)u), rest = u - r * p.units;
            const int head = (int)p.by_groups.div((uint32_t)rest), g = rest - head * groups;
            const CachePlace place = places[r];
            if (place.page == -2) continue;
            left[k] = c.head_dim - 8 * g;
            at[k] = dst + (row0 + r) * row_stride + head * head_stride + 8 * g;
            if (place.page < 0) continue;
            const int64_t cell = ((int64_t)place.page * c.heads + head) * c.page_size + place.slot;
            if constexpr (FORMAT == kCache16) {
                w[k] = ld_stream_16(codes + cell * row_bytes + 16 * g);
            } else {
                if constexpr (FORMAT == kCacheFp8) {
                    const uint2 q = __ldg(reinterpret_cast<const uint2*>(codes + cell * row_bytes + 8 * g));
                    w[k].x = q.x;
                    w[k].y = q.y;
                } else {
                    w[k].x = __ldg(reinterpret_cast<const uint32_t*>(codes + cell * row_bytes + 4 * g));
                }
                S[k] = __ldg(scales + cell * c.scale_row + (g >> 2));
            }
        }
#pragma unroll
        for (int k = 0; k < kReadAhead; ++k) {
            if (left[k] <= 0) continue;
            float v[8];
            if constexpr (FORMAT == kCache16) {
                widen8_any<CF16>(w[k], v);
            } else {
                const float scale = scale_from_e8m0(S[k]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float2 f;
                    if constexpr (FORMAT == kCacheFp8) f = e4m3x2_to_float2((i < 2 ? w[k].x : w[k].y) >> (16 * (i & 1)));
                    else f = e2m1x2_to_float2((w[k].x >> (8 * i)) & 0xFFu);
                    v[2 * i] = f.x * scale;
                    v[2 * i + 1] = f.y * scale;
                }
            }
            cache_store8<T>(at[k], left[k], vec != 0, v);
        }
    }
}

}  // namespace kq
