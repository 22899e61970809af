// Norms before and after a transformer block, fused with the block's gate and residual scale, and their backward pass.
//
// Forward, one row t of d channels, b = t / rows_per_batch:
//     r = post(y) post_weight          post, norm in {none, rms, layer}:  v -> (v - mean) / sqrt(mean((v - mean)^2) + eps)
//     h = alpha x + gate_b r                                              (rms: mean taken as 0)
//     n = norm(h) weight (1 + scale_b) + shift_b
// One read and one write of a row; h enters the norm unrounded (32 bits), so n does not carry the rounding of h to the stream's
// type.  All statistics are 32-bit sums, and squares are taken about a mean, because E[v^2] - E[v]^2 loses what a large mean, or a few
// large channels, leave: the small kernels take two passes over the row, the staged ones (many rows; wide rows in the backward pass)
// let every warp take squares about the mean of its own channels and join them by Chan's update.
//
// Backward, with m = weight (1 + scale_b), xhat = norm(h), yhat = post(y), g = dn m:
//     H  = dh + (g - [mean g] - xhat mean(g xhat)) / dev(h)          [..]: layer only
//     dx = alpha H,   a = gate_b H post_weight,   dy = (a - [mean a] - yhat mean(a yhat)) / dev(y)   (dy = gate_b H without post)
//     P_b = sum_t dn xhat,  S_b = sum_t dn,  Q_b = sum_t H yhat      column sums over the rows of a batch
//     dweight = sum_b (1 + scale_b) P_b,  dscale_b = weight P_b,  dshift_b = S_b,
//     dgate_b = post_weight Q_b,  dpost_weight = sum_b gate_b Q_b
// so three column sums carry every vector gradient.  Statistics are recomputed from h and y, which are read anyway.
// Column sums: a worker (a warp or a CTA) walks a contiguous run of rows and keeps the sums of its columns itself; at
// the end of a batch it writes them to slot (worker + batch), unique because both only grow along the rows, and a second
// kernel adds the slots in a fixed order: no atomics, the same bits every time.
//
// 2 reads and 2 writes (forward), 4 reads and 2 writes (backward) per element.  Memory bounds the wide rows with a 32-bit stream; the
// others wait for instructions and their latency next to it (figures at the kernels).
#pragma once
#include "kq_common.cuh"
#include "kq_umma.cuh"

namespace kq {

enum { kNormNone = 0, kNormRms = 1, kNormLayer = 2 };
enum { kTypeF32 = 0, kTypeBf16 = 1, kTypeF16 = 2 };
constexpr int kNormMaxD = 16384;
enum { KQ_DEV_TIMEOUT_NORM = 15 };

// a [d] or [batches][d] vector of any of the three types; ptr null = absent; stride 0 = the same for every batch
struct NormVec {
    const void* ptr;
    int64_t stride;
    int type;
};

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int kRegs = 8;
    __device__ static float to_f32(float v) { return v; }
    __device__ static float from_f32(float v) { return v; }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int kRegs = 4;
    __device__ static float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
    __device__ static __nv_bfloat16 from_f32(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<__half> {
    static constexpr int kRegs = 4;
    __device__ static float to_f32(__half v) { return __half2float(v); }
    __device__ static __half from_f32(float v) { return __float2half_rn(v); }
};

// Eight elements as loaded (4 or 8 registers) and their widening.
template <typename T> struct Pack8 { uint32_t w[Elem<T>::kRegs]; };

template <typename T>
__device__ __forceinline__ void pack_widen(const Pack8<T>& p, float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(p.w[i]);
    } else if constexpr (sizeof(T) == 2 && Elem<T>::kRegs == 4) {
        const uint4 u = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
        if constexpr (__is_same(T, __half)) widen8_f16(u, v); else widen8(u, v);
    }
}
// a row's elements are read once, and an output may take their place: no read-only path, no L1 line
__device__ __forceinline__ uint4 ld_row_16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// Eight elements of a row from p on.  Vector path: they are contiguous.  Otherwise (rows at any alignment, any d) a thread's
// eight are `step` apart, neighbouring threads hold neighbouring elements and every access is one coalesced element;
// `count` of them exist, the others read as 0.
template <typename T>
__device__ __forceinline__ void load_pack(const T* p, int count, bool vec, int step, Pack8<T>& out) {
    if (vec) {
        if constexpr (sizeof(T) == 4) {
            const uint4 a = ld_row_16(p), b = ld_row_16(p + 4);
            out.w[0] = a.x; out.w[1] = a.y; out.w[2] = a.z; out.w[3] = a.w;
            out.w[4] = b.x; out.w[5] = b.y; out.w[6] = b.z; out.w[7] = b.w;
        } else {
            const uint4 a = ld_row_16(p);
            out.w[0] = a.x; out.w[1] = a.y; out.w[2] = a.z; out.w[3] = a.w;
        }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out.w[i] = i < count ? reinterpret_cast<const uint32_t*>(p)[i * step] : 0u;
    } else {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = 2 * i < count ? q[2 * i * step] : 0u, hi = 2 * i + 1 < count ? q[(2 * i + 1) * step] : 0u;
            out.w[i] = lo | (hi << 16);
        }
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int count, bool vec, int step, const float (&v)[8]) {
    if (vec) {
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
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
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i * step] = Elem<T>::from_f32(v[i]);
    }
}
__device__ __forceinline__ float vec_entry(const NormVec& p, int64_t which, int at, float none) {
    if (!p.ptr) return none;
    const int64_t i = which * p.stride + at;
    if (p.type == kTypeF32) return static_cast<const float*>(p.ptr)[i];
    if (p.type == kTypeF16) return __half2float(static_cast<const __half*>(p.ptr)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p.ptr)[i]);
}
// how many of the elements c, c + step, ..., c + 7 step of a row of d exist
__device__ __forceinline__ int owned(int d, int c, int step) {
    const int left = c < d ? (d - c + step - 1) / step : 0;
    return left < 8 ? left : 8;
}
// eight entries of a parameter vector at channel c (absent: `none`)
__device__ __forceinline__ void load_param(const NormVec& p, int64_t batch, int c, int count, bool vec, int step, float none, float (&v)[8]) {
    if (!p.ptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = none;
        return;
    }
    const int64_t at = batch * p.stride + c;
    if (p.type == kTypeF32) {
        const float* q = static_cast<const float*>(behind_wait(p.ptr)) + at;
        if (vec) {
            const uint4 a = ld_vector_16(q), b = ld_vector_16(q + 4);
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < count ? ld_vector_4(q + i * step) : 0.f;
        }
    } else {
        const uint16_t* q = static_cast<const uint16_t*>(behind_wait(p.ptr)) + at;
        uint4 u;
        if (vec) {
            u = ld_vector_16(q);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = 2 * i < count ? ld_vector_2(q + 2 * i * step) : 0u, hi = 2 * i + 1 < count ? ld_vector_2(q + (2 * i + 1) * step) : 0u;
                w[i] = lo | (hi << 16);
            }
            u = make_uint4(w[0], w[1], w[2], w[3]);
        }
        if (p.type == kTypeF16) widen8_f16(u, v); else widen8(u, v);
    }
}

// Sums of N values over the threads of a row: warp shuffles, then one exchange through shared memory when the row
// has more than one warp.  `red` holds two sets of 32 N floats used in turn, so one barrier per sum is enough.
template <int N>
__device__ __forceinline__ void row_sum(float (&v)[N], float* red, int& phase) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
    if (blockDim.x == 32) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    float* at = red + phase * 128;
    phase ^= 1;
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) at[i * 32 + warp] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = lane < warps ? at[i * 32 + lane] : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
    }
}

// Sums of four values over a warp, every lane gets all four: ten shuffles instead of twenty.  The first steps trade values
// for lanes (a lane keeps the half of the values that its lane bit names), the last three reduce what is left.
__device__ __forceinline__ void warp_sum4(float (&v)[4], int lane) {
    const bool b4 = lane & 16, b3 = lane & 8;
    float k0 = b4 ? v[2] : v[0], k1 = b4 ? v[3] : v[1];
    k0 += __shfl_xor_sync(0xFFFFFFFFu, b4 ? v[0] : v[2], 16);
    k1 += __shfl_xor_sync(0xFFFFFFFFu, b4 ? v[1] : v[3], 16);
    float k = b3 ? k1 : k0;
    k += __shfl_xor_sync(0xFFFFFFFFu, b3 ? k0 : k1, 8);
    k += __shfl_xor_sync(0xFFFFFFFFu, k, 4);
    k += __shfl_xor_sync(0xFFFFFFFFu, k, 2);
    k += __shfl_xor_sync(0xFFFFFFFFu, k, 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __shfl_sync(0xFFFFFFFFu, k, 8 * i);
}

// the same with two values: seven shuffles instead of ten
__device__ __forceinline__ void warp_sum2(float (&v)[2], int lane) {
    const bool b4 = lane & 16;
    float k = b4 ? v[1] : v[0];
    k += __shfl_xor_sync(0xFFFFFFFFu, b4 ? v[0] : v[1], 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) k += __shfl_xor_sync(0xFFFFFFFFu, k, o);
    v[0] = __shfl_sync(0xFFFFFFFFu, k, 0);
    v[1] = __shfl_sync(0xFFFFFFFFu, k, 16);
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Four floats to the same place in the shared memory of CTA `rank` of the cluster, counted as 16 bytes on the mbarrier at the
// same place there.  (A cluster barrier would order the exchange too, but its release waits for the global stores in
// flight: 1.7 us per row.)
__device__ __forceinline__ void st_async_v4(uint32_t addr, uint32_t bar, uint32_t rank, const float4& v) {
    asm volatile("{\n\t.reg .u32 a, b;\n\tmapa.shared::cluster.u32 a, %0, %2;\n\tmapa.shared::cluster.u32 b, %1, %2;\n\t"
                 "st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [a], {%3, %4, %5, %6}, [b];\n\t}"
                 ::"r"(addr), "r"(bar), "r"(rank), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

struct NormForward {
    int64_t rows;
    int d;
    int64_t rows_per_batch;
    const void* x; int64_t ld_x;
    const void* y; int64_t ld_y;      // null: no branch
    void* h; int64_t ld_h;            // null: not wanted
    void* n; int64_t ld_n;            // null with norm == none
    NormVec gate, post_weight, weight, scale, shift;
    float alpha, eps;
    int norm, post;
    int vec;                          // every pointer, pitch and d allow 16-byte accesses
    // staged kernel: rows of a worker, stages, bytes of a stage, offset of y, which parameter vectors are kept in shared memory
    int64_t rows_per_worker;
    int stages, stage_bytes, off_y, cache;
};

// blockDim = (threads of a row, rows of a CTA): one warp per row and several rows for narrow d, else one row per CTA.
// Thread i owns the 8-channel groups i, i + blockDim.x, ...: VPT of them.
// Measured: one row of 4096 3.2 us (a launch); layer, gate and modulation 16384 x 256 11 us, 16384 x 1024 41 us (a warp reloads its
// vectors for every row); rms 16384 x 2241 (no vector accesses) 129 us.
template <typename S, typename Y, int VPT>
__global__ void __launch_bounds__(VPT == 2 ? 1024 : 256) norm_residual_forward(const __grid_constant__ NormForward p) {
    __shared__ float red[2 * 128];
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    pdl_wait_prior_grid();
    if (row >= p.rows) return;        // whole warps: a CTA with more than one row has one warp per row
    const int64_t batch = row / p.rows_per_batch;
    const bool vec = p.vec != 0;
    const float inv_d = 1.0f / (float)p.d;
    int phase = 0;
    Pack8<S> xs[VPT];
    Pack8<Y> ys[VPT];
    int count[VPT];
    const int step = vec ? 1 : (int)blockDim.x;
    auto column = [&](int k) { return vec ? ((int)threadIdx.x + k * (int)blockDim.x) * 8 : (int)threadIdx.x + k * 8 * (int)blockDim.x; };
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int c = column(k);
        count[k] = owned(p.d, c, step);
        if (count[k] > 0) {
            load_pack(static_cast<const S*>(p.x) + row * p.ld_x + c, count[k], vec, step, xs[k]);
            if (p.y) load_pack(static_cast<const Y*>(p.y) + row * p.ld_y + c, count[k], vec, step, ys[k]);
        }
    }
    float h[VPT][8];
    float mean_y = 0.f, inv_y = 1.f;
    if (p.y && p.post != kNormNone) {
        if (p.post == kNormLayer) {
            float s[1] = {0.f};
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) {
                    float v[8];
                    pack_widen(ys[k], v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[0] += v[i];
                }
            row_sum<1>(s, red, phase);
            mean_y = s[0] * inv_d;
        }
        float s[1] = {0.f};
#pragma unroll
        for (int k = 0; k < VPT; ++k)
            if (count[k] > 0) {
                float v[8];
                pack_widen(ys[k], v);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < count[k]) s[0] = fmaf(v[i] - mean_y, v[i] - mean_y, s[0]);
            }
        row_sum<1>(s, red, phase);
        inv_y = rsqrtf(s[0] * inv_d + p.eps);
    }
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        if (count[k] > 0) {
            const int c = column(k);
            pack_widen(xs[k], h[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[k][i] *= p.alpha;
            if (p.y) {
                float v[8], g[8];
                pack_widen(ys[k], v);
                if (p.post != kNormNone) {
                    load_param(p.post_weight, 0, c, count[k], vec, step, 1.f, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = (v[i] - mean_y) * inv_y * g[i];
                }
                load_param(p.gate, batch, c, count[k], vec, step, 1.f, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[k][i] = i < count[k] ? fmaf(g[i], v[i], h[k][i]) : 0.f;
            }
            if (p.h) store8(static_cast<S*>(p.h) + row * p.ld_h + c, count[k], vec, step, h[k]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) h[k][i] = 0.f;
        }
    }
    if (p.norm == kNormNone) return;
    float mean = 0.f;
    if (p.norm == kNormLayer) {
        float s[1] = {0.f};
#pragma unroll
        for (int k = 0; k < VPT; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += h[k][i];
        row_sum<1>(s, red, phase);
        mean = s[0] * inv_d;
    }
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < VPT; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count[k]) s[0] = fmaf(h[k][i] - mean, h[k][i] - mean, s[0]);
    row_sum<1>(s, red, phase);
    const float inv = rsqrtf(s[0] * inv_d + p.eps);
#pragma unroll
    for (int k = 0; k < VPT; ++k)
        if (count[k] > 0) {
            const int c = column(k);
            float a[8], w[8];
            load_param(p.weight, 0, c, count[k], vec, step, 1.f, w);
            load_param(p.scale, batch, c, count[k], vec, step, 0.f, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = fmaf(w[i], a[i], w[i]);
            load_param(p.shift, batch, c, count[k], vec, step, 0.f, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = fmaf((h[k][i] - mean) * inv, w[i], a[i]);
            store8(static_cast<Y*>(p.n) + row * p.ld_n + c, count[k], vec, step, a);
        }
}

struct NormBackward {
    int64_t rows;
    int d;
    int64_t rows_per_batch, rows_per_worker;
    const void* dn; int64_t ld_dn;    // null with norm == none
    const void* dh; int64_t ld_dh;    // null: no gradient comes along the stream
    const void* h; int64_t ld_h;
    const void* y; int64_t ld_y;      // null: no branch
    void* dx; int64_t ld_dx;
    void* dy; int64_t ld_dy;
    NormVec gate, post_weight, weight, scale;
    float alpha, eps;
    int norm, post;
    int vec;
    float* partial;                   // [slots][3][d]: P, S, Q of a worker's rows of one batch; null: no vector gradient wanted
    // staged kernel: CTAs of a worker and columns of each, stages, bytes of a stage, offsets of its rows, which parameter
    // vectors are kept in shared memory
    int cluster, columns, stages, stage_bytes, off_dh, off_dn, off_y, cache_m, cache_gate, cache_post;
};

// ---- backward, narrow rows: one warp per row --------------------------------------------------------
// A CTA of eight warps is a worker and takes the rows [blockIdx.x rows_per_worker, ...), its warps every eighth of them; d <= 256
// VPT, rows in registers.  At the end of a batch the warps' column sums meet in shared memory and are added in warp order.
constexpr int kNormWarps = 8;

template <typename S, typename Y, int VPT>
__global__ void __launch_bounds__(32 * kNormWarps) norm_residual_backward_warp(const __grid_constant__ NormBackward p) {
    extern __shared__ float warp_sums[];                              // [warps][3][d]
    const int64_t first = (int64_t)blockIdx.x * p.rows_per_worker;
    const int64_t last = first + p.rows_per_worker < p.rows ? first + p.rows_per_worker : p.rows;
    pdl_wait_prior_grid();
    const int warp = (int)threadIdx.y;
    const int lane = (int)threadIdx.x;
    const bool vec = p.vec != 0;
    const float inv_d = 1.0f / (float)p.d;
    const bool layer_h = p.norm == kNormLayer, layer_y = p.post == kNormLayer, post = p.y && p.post != kNormNone;
    const int step = vec ? 1 : 32;
    auto column = [&](int k) { return vec ? (lane + k * 32) * 8 : lane + k * 256; };
    int count[VPT];
#pragma unroll
    for (int k = 0; k < VPT; ++k) count[k] = owned(p.d, column(k), step);
    float sum[3][VPT][8];
    auto clear = [&]() {
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int k = 0; k < VPT; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[q][k][i] = 0.f;
    };
    auto flush = [&](int64_t slot) {
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int k = 0; k < VPT; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < count[k]) warp_sums[(warp * 3 + q) * p.d + column(k) + i * step] = sum[q][k][i];
        __syncthreads();
        for (int x = (int)(threadIdx.y * 32 + threadIdx.x); x < 3 * p.d; x += 32 * kNormWarps) {
            float a = 0.f;
#pragma unroll
            for (int w = 0; w < kNormWarps; ++w) a += warp_sums[w * 3 * p.d + x];
            p.partial[slot * 3 * p.d + x] = a;
        }
        __syncthreads();
        clear();
    };
    clear();
    for (int64_t begin = first; begin < last;) {
    const int64_t batch = begin / p.rows_per_batch;
    const int64_t end = (batch + 1) * p.rows_per_batch < last ? (batch + 1) * p.rows_per_batch : last;
    for (int64_t row = begin + warp; row < end; row += kNormWarps) {
        float h[VPT][8], g[VPT][8], H[VPT][8], y[VPT][8];
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int c = column(k);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[k][i] = g[k][i] = H[k][i] = y[k][i] = 0.f;
            if (count[k] > 0) {
                Pack8<S> s, s2;
                Pack8<Y> b, b2;
                load_pack(static_cast<const S*>(p.h) + row * p.ld_h + c, count[k], vec, step, s);
                if (p.dh) load_pack(static_cast<const S*>(p.dh) + row * p.ld_dh + c, count[k], vec, step, s2);
                if (p.dn) load_pack(static_cast<const Y*>(p.dn) + row * p.ld_dn + c, count[k], vec, step, b);
                if (p.y) load_pack(static_cast<const Y*>(p.y) + row * p.ld_y + c, count[k], vec, step, b2);
                pack_widen(s, h[k]);
                if (p.dh) pack_widen(s2, H[k]);
                if (p.dn) pack_widen(b, g[k]);
                if (p.y) pack_widen(b2, y[k]);
            }
        }
        auto multiplier = [&](int k, float (&m)[8]) {          // weight (1 + scale)
            float a[8];
            load_param(p.weight, 0, column(k), count[k], vec, step, 1.f, m);
            load_param(p.scale, batch, column(k), count[k], vec, step, 0.f, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) m[i] = fmaf(m[i], a[i], m[i]);
        };
        float mu[4] = {0.f, 0.f, 0.f, 0.f};                     // means of h, g, y (layer)
        if (layer_h || layer_y) {
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) {
                    float m[8];
                    multiplier(k, m);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        mu[0] += h[k][i];
                        mu[1] = fmaf(g[k][i], i < count[k] ? m[i] : 0.f, mu[1]);
                        mu[2] += y[k][i];
                    }
                }
            warp_sum4(mu, lane);
            mu[0] = layer_h ? mu[0] * inv_d : 0.f;
            mu[1] = layer_h ? mu[1] * inv_d : 0.f;
            mu[2] = layer_y ? mu[2] * inv_d : 0.f;
        }
        float sq[4] = {0.f, 0.f, 0.f, 0.f};                     // squares about the means, g . (h - mean)
#pragma unroll
        for (int k = 0; k < VPT; ++k)
            if (count[k] > 0) {
                float m[8];
                multiplier(k, m);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < count[k]) {
                        const float u = h[k][i] - mu[0], v = y[k][i] - mu[2];
                        sq[0] = fmaf(u, u, sq[0]);
                        sq[1] = fmaf(g[k][i] * m[i], u, sq[1]);
                        sq[2] = fmaf(v, v, sq[2]);
                    }
            }
        warp_sum4(sq, lane);
        const float inv_h = rsqrtf(sq[0] * inv_d + p.eps);
        const float along_h = sq[1] * inv_d * inv_h;
        const float inv_y = post ? rsqrtf(sq[2] * inv_d + p.eps) : 1.f;
        float back[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < VPT; ++k)
            if (count[k] > 0) {
                float m[8], v[8];
                multiplier(k, m);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float xhat = (h[k][i] - mu[0]) * inv_h;
                    sum[0][k][i] = fmaf(g[k][i], xhat, sum[0][k][i]);
                    sum[1][k][i] += g[k][i];
                    if (p.norm != kNormNone) H[k][i] = fmaf(inv_h, g[k][i] * m[i] - mu[1] - xhat * along_h, H[k][i]);
                    v[i] = p.alpha * H[k][i];
                }
                store8(static_cast<S*>(p.dx) + row * p.ld_dx + column(k), count[k], vec, step, v);
                if (p.y) {
                    load_param(p.gate, batch, column(k), count[k], vec, step, 1.f, m);
                    if (post) load_param(p.post_weight, 0, column(k), count[k], vec, step, 1.f, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float yhat = (y[k][i] - mu[2]) * inv_y;
                        sum[2][k][i] = fmaf(H[k][i], yhat, sum[2][k][i]);
                        H[k][i] *= post ? m[i] * v[i] : m[i];
                        if (i < count[k]) {
                            back[0] += H[k][i];
                            back[1] = fmaf(H[k][i], yhat, back[1]);
                        }
                    }
                    if (!post) store8(static_cast<Y*>(p.dy) + row * p.ld_dy + column(k), count[k], vec, step, H[k]);
                }
            }
        if (post) {
            warp_sum4(back, lane);
            const float mean_a = layer_y ? back[0] * inv_d : 0.f, along_y = back[1] * inv_d;
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) {
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = (H[k][i] - mean_a - (y[k][i] - mu[2]) * inv_y * along_y) * inv_y;
                    store8(static_cast<Y*>(p.dy) + row * p.ld_dy + column(k), count[k], vec, step, v);
                }
        }
    }
    if (p.partial) flush(blockIdx.x + batch);
    begin = end;
    }
}

// ---- backward, wide rows: a CTA, or a cluster of two or four, per row; rows staged in shared memory ----------------
// A worker is one CTA up to d = 4608 and a cluster of two or four above, each CTA with its part of the columns: one group of 8
// channels per thread, so that the column sums (24 registers) and two rows with their parameters (shared memory) always
// fit.  The four rows of an iteration arrive in shared memory by bulk copies issued `stages` rows ahead: nothing waits for a
// load, and a row needs no registers.  A thread reads its group twice (statistics, gradients) or, with a post norm, y and
// one more value a third time.  What a thread writes to shared memory (parameters, the value between the phases) only it reads.
// The statistics take one pass and one barrier.  A warp sums about a pivot p, s1 = sum (v - p), s2 = sum (v - p)^2, g1 = sum g (h - p),
// and moves them to its mean, M2 = s2 - s1^2 / n; Chan's update then joins the warps.  The pivot is the mean of the warp's first 256
// channels of at most 512: the mean of n1 of n values lies within sqrt(n / n1 - 1) deviations of theirs, here one, so that at
// most half of s2 cancels, wherever the outliers of a row are.  (A pivot from 32 sampled channels of the row, joined in one step,
// was off by a factor d / 32 for rows with their outliers in those; it was faster only on narrow rows, 16384 x 1024 75 us against 80.)
// With 18 warps on an SM the instructions bound the kernel next to memory, so the arithmetic is done on pairs (f32x2).
// Parameter vectors (weight (1 + scale), gate, post_weight) are kept in shared memory as floats, refreshed at the start of a batch.
// Measured (layer, gate and modulation, 16-bit): 16384 x 4608 205 us, 4.4 TB/s; 16384 x 1024 81 us; rms around rms, 6000 x 12288 in
// clusters of four 480 us, 1.8 TB/s (every row waits for an exchange between CTAs); 16384 x 2241 (element copies) 344 us.
// Rows that bulk copies cannot take (16-byte alignment) are copied into the same place by the threads, element by element.
constexpr int kNormStageMax = 6;
constexpr int kNormThreads = 576;
constexpr int kNormMaxCluster = 4;
constexpr int kNormRedOff = 128;                                    // barriers and the abort word in front
constexpr int kNormRedFloats = kNormMaxCluster * (kNormThreads / 32) * 8;
constexpr int kNormHeadBytes = kNormRedOff + 4 * kNormRedFloats * 4;   // two sets of statistics used in turn, two of the second phase

typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
    f32x2 d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float2 unpack2(f32x2 v) {
    float2 d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(v));
    return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float sum2(f32x2 v) { const float2 f = unpack2(v); return f.x + f.y; }

// two 16-bit elements -> a pair
template <typename T>
__device__ __forceinline__ f32x2 widen2(uint32_t w) {
    if constexpr (__is_same(T, __half)) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
        return pack2(f.x, f.y);
    } else {
        return pack2(bf16lo_to_f32(w), bf16hi_to_f32(w));
    }
}
// the eight elements of a group of a row in shared memory
template <typename T>
__device__ __forceinline__ void lds8(const uint8_t* row, int group, f32x2 (&v)[4]) {
    if constexpr (sizeof(T) == 4) {
        const ulonglong2 a = reinterpret_cast<const ulonglong2*>(row)[2 * group], b = reinterpret_cast<const ulonglong2*>(row)[2 * group + 1];
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
    } else {
        const uint4 a = reinterpret_cast<const uint4*>(row)[group];
        v[0] = widen2<T>(a.x); v[1] = widen2<T>(a.y); v[2] = widen2<T>(a.z); v[3] = widen2<T>(a.w);
    }
}
template <typename T>
__device__ __forceinline__ void store_pairs(T* p, int count, bool vec, const f32x2 (&w)[4]) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2(w[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
    store8(p, count, vec, 1, v);
}
// `d` columns of the four rows of an iteration that are not 16-byte aligned, into shared memory: sixteen loads in flight per
// thread; the tail of the last group is 0
template <typename S, typename Y>
__device__ __noinline__ void copy_rows(uint8_t* stage, const NormBackward& p, int64_t row, int c0, int d) {
    const S* src_s[2] = {static_cast<const S*>(p.h) + row * p.ld_h + c0, static_cast<const S*>(p.dh) + row * p.ld_dh + c0};
    const Y* src_y[2] = {static_cast<const Y*>(p.dn) + row * p.ld_dn + c0, static_cast<const Y*>(p.y) + row * p.ld_y + c0};
    S* dst_s[2] = {reinterpret_cast<S*>(stage), reinterpret_cast<S*>(stage + p.off_dh)};
    Y* dst_y[2] = {reinterpret_cast<Y*>(stage + p.off_dn), reinterpret_cast<Y*>(stage + p.off_y)};
    const bool have_s[2] = {true, p.dh != nullptr}, have_y[2] = {p.dn != nullptr, p.y != nullptr};
    const int T = (int)blockDim.x, padded = (d + 7) / 8 * 8;
    for (int c = (int)threadIdx.x; c < padded; c += 4 * T) {
        S a[2][4];
        Y b[2][4];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = c + i * T < d;
                a[q][i] = have_s[q] && in ? src_s[q][c + i * T] : Elem<S>::from_f32(0.f);
                b[q][i] = have_y[q] && in ? src_y[q][c + i * T] : Elem<Y>::from_f32(0.f);
            }
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i * T < padded) {
                    if (have_s[q]) dst_s[q][c + i * T] = a[q][i];
                    if (have_y[q]) dst_y[q][c + i * T] = b[q][i];
                }
    }
}

// VEC: every row on 16-byte boundaries (bulk copies, whole groups); else any alignment and any d.
template <typename S, typename Y, bool POST, bool VEC>
__global__ void __launch_bounds__(kNormThreads, 1) norm_residual_backward(const __grid_constant__ NormBackward p) {
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + 120);
    float* red = reinterpret_cast<float*>(smem + kNormRedOff);
    const int t = (int)threadIdx.x, warp = t >> 5, lane = t & 31, warps = (int)blockDim.x >> 5;
    const int rank = p.cluster > 1 ? (int)cluster_rank() : 0;
    const int64_t worker = blockIdx.x / (unsigned)p.cluster;
    const int c0 = rank * p.columns;                                  // this CTA's columns: c0 .. c0 + d - 1
    const int d = p.d - c0 < p.columns ? p.d - c0 : p.columns;
    float* par_m = reinterpret_cast<float*>(smem + kNormHeadBytes);
    float* par_gate = par_m + (p.cache_m ? p.columns : 0);
    float* par_post = par_gate + (p.cache_gate ? p.columns : 0);
    const int stage0 = kNormHeadBytes + 4 * p.columns * (p.cache_m + p.cache_gate + p.cache_post);
    const int64_t first = worker * p.rows_per_worker;
    const int rows = (int)(first + p.rows_per_worker < p.rows ? p.rows_per_worker : p.rows - first);
    constexpr bool vec = VEC;
    const float inv_d = 1.0f / (float)p.d;
    const bool layer_h = p.norm == kNormLayer, layer_y = POST && p.post == kNormLayer, norm = p.norm != kNormNone;
    // What the warps of a worker exchange: in one CTA by a barrier; in a cluster every warp sends its values to all CTAs and
    // an mbarrier counts their bytes.  Four sets of values, each with its barrier: statistics (two, used in turn, so that a
    // set is not written before all have read what it held), second phase (of the first and the second row of an iteration).
    auto exchange = [&](int set, float* at, const float4& a) {
        if (p.cluster == 1) *reinterpret_cast<float4*>(at) = a;
        else
            for (int q = 0; q < p.cluster; ++q) st_async_v4(smem_u32(at), base + 8u * (kNormStageMax + set), (uint32_t)q, a);
    };
    uint32_t set_parity = 0;                                          // bit = parity of a set's next phase
    auto exchanged_all = [&](int set, int bytes) {
        if (p.cluster == 1) {
            __syncthreads();
            return;
        }
        const uint32_t bar = base + 8u * (kNormStageMax + set);
        if (t == 0) mbar_expect_tx(bar, (uint32_t)bytes);
        if (!mbar_wait(bar, (set_parity >> set) & 1u, abort_flag) && !*abort_flag) {
            atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_NORM);
            *abort_flag = 1;
        }
        set_parity ^= 1u << set;
    };
    const int all_warps = warps * p.cluster, my_warp = warp + rank * warps;
    if (t == 0) {
        for (int s = 0; s < kNormStageMax + 4; ++s) mbar_init(base + 8u * s, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (p.cluster > 1) cluster_barrier(); else __syncthreads();
    pdl_wait_prior_grid();
    auto issue = [&](int r, int s) {                                  // thread 0: row `r` of this worker into stage s
        const int64_t row = first + r;
        const uint32_t bar = base + 8u * s, dst = base + (uint32_t)(stage0 + s * p.stage_bytes);
        const uint32_t bytes_s = (uint32_t)d * sizeof(S), bytes_y = (uint32_t)d * sizeof(Y);
        mbar_expect_tx(bar, bytes_s * (p.dh ? 2 : 1) + bytes_y * ((p.dn ? 1 : 0) + (p.y ? 1 : 0)));
        bulk_load(dst, static_cast<const S*>(p.h) + row * p.ld_h + c0, bytes_s, bar);
        if (p.dh) bulk_load(dst + p.off_dh, static_cast<const S*>(p.dh) + row * p.ld_dh + c0, bytes_s, bar);
        if (p.dn) bulk_load(dst + p.off_dn, static_cast<const Y*>(p.dn) + row * p.ld_dn + c0, bytes_y, bar);
        if (p.y) bulk_load(dst + p.off_y, static_cast<const Y*>(p.y) + row * p.ld_y + c0, bytes_y, bar);
    };
    if (vec && t == 0)
        for (int r = 0; r < p.stages && r < rows; ++r) issue(r, r);
    const int c = t * 8, count = VEC ? (c < d ? 8 : 0) : owned(d, c, 1);                       // this thread's channels in the CTA's columns
    f32x2 sum[3][4];
    auto clear = [&]() {
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[q][i] = 0ull;
    };
    auto flush = [&](int64_t slot) {
        float* out = p.partial + slot * 3 * p.d + c0 + c;
#pragma unroll
        for (int q = 0; q < 3; ++q)
            if (count > 0) store_pairs(out + (int64_t)q * p.d, count, vec, sum[q]);
        clear();
    };
    clear();
    int64_t batch = first / p.rows_per_batch;
    // rows of this worker before the next batch begins
    auto rows_left = [&](int64_t row) { const int64_t n = (batch + 1) * p.rows_per_batch - row; return (int)(n < rows ? n : rows); };
    int batch_end = rows_left(first);
    auto keep = [&](float* vector, const float (&v)[8]) {
        reinterpret_cast<float4*>(vector)[t] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(vector + (p.columns >> 1))[t] = make_float4(v[4], v[5], v[6], v[7]);
    };
    auto refresh = [&]() {
        if (count > 0) {
            float m[8], a[8];
            if (p.cache_m) {
                load_param(p.weight, 0, c0 + c, count, vec, 1, 1.f, m);
                load_param(p.scale, batch, c0 + c, count, vec, 1, 0.f, a);
#pragma unroll
                for (int i = 0; i < 8; ++i) m[i] = fmaf(m[i], a[i], m[i]);
                keep(par_m, m);
            }
            if (p.cache_gate) {
                load_param(p.gate, batch, c0 + c, count, vec, 1, 1.f, m);
                keep(par_gate, m);
            }
            if (p.cache_post) {
                load_param(p.post_weight, 0, c0 + c, count, vec, 1, 1.f, m);
                keep(par_post, m);
            }
        }
    };
    refresh();
    __syncthreads();
    const f32x2 one2 = pack2(1.f, 1.f), alpha2 = pack2(p.alpha, p.alpha);
    // a vector lies in two planes, the first and the last four entries of every group (no bank conflicts either way)
    const int plane = p.columns >> 1;
    auto parameters = [&](int have, const float* vector, int group, f32x2 (&m)[4]) {
        ulonglong2 a = make_ulonglong2(one2, one2), b = a;
        if (have) {
            a = reinterpret_cast<const ulonglong2*>(vector)[group];
            b = reinterpret_cast<const ulonglong2*>(vector + plane)[group];
        }
        m[0] = a.x; m[1] = a.y; m[2] = b.x; m[3] = b.y;
    };
    S* dx = static_cast<S*>(p.dx) + first * p.ld_dx + c0 + c;
    Y* dy = static_cast<Y*>(p.dy) + first * p.ld_dy + c0 + c;
    int s = 0, next = p.stages < rows ? p.stages : rows;              // stage of row r; next row to be fetched (thread 0)
    uint32_t parity = 0;
    int turn = 0;
    for (int r = 0, nr; r < rows; r += nr) {
        if (r == batch_end) {
            __syncthreads();                                          // other threads read this thread's parameters too
            if (p.partial) flush(worker + batch);
            ++batch;
            batch_end = r + rows_left(first + r);
            refresh();
            __syncthreads();
        }
        // two rows of one batch at a time where the stages leave two more in flight
        nr = p.stages >= 4 && r + 1 < rows && r + 1 < batch_end ? 2 : 1;
        uint8_t* stages[2];
        stages[0] = smem + stage0 + s * p.stage_bytes;
        stages[1] = smem + stage0 + (s + 1 < p.stages ? s + 1 : 0) * p.stage_bytes;
        if (vec) {
            // a wait that gives up records it and goes on (the barriers below stay matched)
            bool ok = mbar_wait(base + 8u * s, parity, abort_flag);
            if (nr == 2) ok = ok && mbar_wait(base + 8u * (s + 1 < p.stages ? s + 1 : 0), s + 1 < p.stages ? parity : parity ^ 1u, abort_flag);
            if (!ok && !*abort_flag) {
                atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_NORM);
                *abort_flag = 1;
            }
        } else {
            __syncthreads();
            for (int j = 0; j < nr; ++j) copy_rows<S, Y>(stages[j], p, first + r + j, c0, d);
            __syncthreads();
        }
        // ---- statistics: with two rows, half of the warps take one row each and a warp 512 columns, else 256 ----
        const int per_row = nr == 2 ? warps >> 1 : warps;
        const int my_row = nr == 2 && warp >= per_row ? 1 : 0, part = warp - my_row * per_row;
        {
            const uint8_t* stage = my_row ? stages[1] : stages[0];
            float pivot_h = 0.f, pivot_y = 0.f;                       // means of the first (up to) 256 of this warp's columns
            const int exist = d - part * nr * 256;
            const float share = exist >= 256 ? 0.00390625f : 1.f / (float)(exist > 0 ? exist : 1);
            if (layer_h || layer_y) {
                const int gi = part * nr * 32 + lane;
                float q[2] = {0.f, 0.f};
                if (gi * 8 < d) {                                    // (a ragged end of a row is filled up with zeros)
                    f32x2 v[4];
                    if (layer_h) {
                        lds8<S>(stage, gi, v);
                        q[0] = sum2(add2(add2(v[0], v[1]), add2(v[2], v[3])));
                    }
                    if (layer_y) {
                        lds8<Y>(stage + p.off_y, gi, v);
                        q[1] = sum2(add2(add2(v[0], v[1]), add2(v[2], v[3])));
                    }
                }
                if (POST) {
                    warp_sum2(q, lane);
                } else {
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) q[0] += __shfl_xor_sync(0xFFFFFFFFu, q[0], o);
                }
                pivot_h = q[0] * share;
                pivot_y = q[1] * share;
            }
            f32x2 s1 = 0ull, s2 = 0ull, g0 = 0ull, g1 = 0ull, y1 = 0ull, y2 = 0ull;
#pragma unroll 1
            for (int k = 0; k < nr; ++k) {
                const int gi = (part * nr + k) * 32 + lane, have = VEC ? (gi * 8 < d ? 8 : 0) : owned(d, gi * 8, 1);
                if (have == 8) {
                    if (POST) {
                        const f32x2 minus = pack2(-pivot_y, -pivot_y);
                        f32x2 v[4];
                        lds8<Y>(stage + p.off_y, gi, v);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const f32x2 u = add2(v[i], minus);
                            y1 = add2(y1, u);
                            y2 = fma2(u, u, y2);
                        }
                    }
                    if (norm) {
                        const f32x2 minus = pack2(-pivot_h, -pivot_h);
                        f32x2 v[4], g[4], m[4];
                        lds8<S>(stage, gi, v);
                        lds8<Y>(stage + p.off_dn, gi, g);
                        parameters(p.cache_m, par_m, gi, m);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const f32x2 u = add2(v[i], minus), w = mul2(g[i], m[i]);
                            s1 = add2(s1, u);
                            s2 = fma2(u, u, s2);
                            g0 = add2(g0, w);
                            g1 = fma2(w, u, g1);
                        }
                    }
                }
                if (!VEC && have < 8) {                              // the ragged end of a row: one thread, one by one
#pragma unroll 1
                    for (int i = gi * 8; i < gi * 8 + have; ++i) {
                        if (norm) {
                            const float u = Elem<S>::to_f32(reinterpret_cast<const S*>(stage)[i]) - pivot_h;
                            const float w = Elem<Y>::to_f32(reinterpret_cast<const Y*>(stage + p.off_dn)[i]) * (p.cache_m ? par_m[(i & 4 ? plane : 0) + (i >> 3) * 4 + (i & 3)] : 1.f);
                            s1 = add2(s1, pack2(u, 0.f));
                            s2 = add2(s2, pack2(u * u, 0.f));
                            g0 = add2(g0, pack2(w, 0.f));
                            g1 = add2(g1, pack2(w * u, 0.f));
                        }
                        if (POST) {
                            const float u = Elem<Y>::to_f32(reinterpret_cast<const Y*>(stage + p.off_y)[i]) - pivot_y;
                            y1 = add2(y1, pack2(u, 0.f));
                            y2 = add2(y2, pack2(u * u, 0.f));
                        }
                    }
                }
            }
            float st[4] = {sum2(s1), sum2(s2), sum2(g0), sum2(g1)}, sty[4] = {sum2(y1), sum2(y2), 0.f, 0.f};
            warp_sum4(st, lane);
            if (POST) warp_sum4(sty, lane);
            if (lane == 0) {
                // mean and squares about it of this warp's columns, sum g, sum g (h - mean)
                float n = 0.f;
                if (layer_h || layer_y) {
                    const int left = d - part * nr * 256;
                    n = left >= 256 * nr ? 256.f * nr : (float)(left > 0 ? left : 0);
                    const float one_nth = left >= 256 * nr ? (nr == 2 ? 0.001953125f : 0.00390625f) : (left > 0 ? 1.f / n : 0.f);
                    const float dh = st[0] * one_nth, dy = sty[0] * one_nth;
                    if (layer_h) {
                        st[1] = fmaf(-dh, st[0], st[1]);
                        st[3] = fmaf(-dh, st[2], st[3]);
                        pivot_h += dh;
                    }
                    if (layer_y) {
                        sty[1] = fmaf(-dy, sty[0], sty[1]);
                        pivot_y += dy;
                    }
                }
                float* at = red + turn * kNormRedFloats + (my_row * p.cluster * per_row + rank * per_row + part) * 8;
                exchange(turn, at, make_float4(pivot_h, st[1], st[2], st[3]));
                exchange(turn, at + 4, make_float4(pivot_y, sty[1], n, 0.f));
            }
        }
        exchanged_all(turn, all_warps * 32);
        // every thread is done with the rows before r: their stages take the rows that follow
        if (vec && t == 0)
            for (; next < rows && next < r + p.stages; ++next) issue(next, next % p.stages);
        const float* exchanged = red + turn * kNormRedFloats;        // (the other set may be written before all have read this one)
        turn ^= 1;
        // Chan's update over the warps: first the means, as offsets from the first warp's, then the sums moved to them,
        // sum (v - mean)^2 = M2 + n e^2 and sum g (h - mean) = g1 + e g0 with e = the warp's mean - mean.  Half a warp for each row.
        float half_mean_h = 0.f, half_mean_g = 0.f, half_mean_y = 0.f, half_inv_h, half_along_h, half_inv_y = 1.f;
        {
            const int parts = p.cluster * per_row;
            const float4* of_row = reinterpret_cast<const float4*>(exchanged + (nr == 2 && lane >= 16 ? parts * 8 : 0));
            auto each = [&](auto&& f) {                               // the warps of this lane
                int w = lane & 15;
                const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
                f(w < parts ? of_row[2 * w] : none, w < parts ? of_row[2 * w + 1] : none);
                if (parts > 16)
                    for (w += 16; w < parts; w += 16) f(of_row[2 * w], of_row[2 * w + 1]);
            };
            auto half_sum = [](float v) {
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
                return v;
            };
            if (layer_h || layer_y) {
                const float base_h = of_row[0].x, base_y = of_row[1].x;
                float mu = 0.f, mu_g = 0.f, mu_y = 0.f;
                each([&](const float4& a, const float4& b) {
                    mu = fmaf(b.z, a.x - base_h, mu);
                    mu_g += a.z;
                    if (POST) mu_y = fmaf(b.z, b.x - base_y, mu_y);
                });
                mu = half_sum(mu);
                mu_g = half_sum(mu_g);
                if (POST) mu_y = half_sum(mu_y);
                if (layer_h) {
                    half_mean_h = fmaf(mu, inv_d, base_h);
                    half_mean_g = mu_g * inv_d;
                }
                if (layer_y) half_mean_y = fmaf(mu_y, inv_d, base_y);
            }
            float sq = 0.f, sq_g = 0.f, sq_y = 0.f;
            each([&](const float4& a, const float4& b) {
                const float eh = a.x - half_mean_h, ey = b.x - half_mean_y;
                sq += fmaf(b.z * eh, eh, a.y);
                sq_g += fmaf(eh, a.z, a.w);
                if (POST) sq_y += fmaf(b.z * ey, ey, b.y);
            });
            sq = half_sum(sq);
            sq_g = half_sum(sq_g);
            if (POST) sq_y = half_sum(sq_y);
            half_inv_h = norm ? rsqrtf(fmaf(sq, inv_d, p.eps)) : 0.f;
            half_along_h = sq_g * inv_d * half_inv_h;
            if (POST) half_inv_y = rsqrtf(fmaf(sq_y, inv_d, p.eps));
        }
        // ---- gradients: H = dh + inv_h (g m - mean_g - xhat along_h) ----
#pragma unroll 1
        for (int j = 0; j < nr; ++j) {
        uint8_t* stage = j ? stages[1] : stages[0];
        auto of_this = [&](float v) { return __shfl_sync(0xFFFFFFFFu, v, 16 * j); };
        const float mean_h = of_this(half_mean_h), mean_g = of_this(half_mean_g), inv_h = of_this(half_inv_h), along_h = of_this(half_along_h);
        const float mean_y = POST ? of_this(half_mean_y) : 0.f, inv_y = POST ? of_this(half_inv_y) : 1.f;
        const f32x2 inv_h2 = pack2(inv_h, inv_h), off_h2 = pack2(-mean_h, -mean_h), along2 = pack2(-along_h, -along_h), mean_g2 = pack2(-mean_g, -mean_g);
        const f32x2 inv_y2 = pack2(inv_y, inv_y), off_y2 = pack2(-mean_y, -mean_y);
        f32x2 back0 = 0ull, back1 = 0ull;
        if (count > 0) {
            f32x2 H[4] = {0ull, 0ull, 0ull, 0ull}, v[4], m[4];
            if (p.dh) lds8<S>(stage + p.off_dh, t, H);
            if (norm) {
                f32x2 g[4];
                lds8<S>(stage, t, v);
                lds8<Y>(stage + p.off_dn, t, g);
                parameters(p.cache_m, par_m, t, m);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x2 xhat = mul2(add2(v[i], off_h2), inv_h2);
                    sum[0][i] = fma2(g[i], xhat, sum[0][i]);
                    sum[1][i] = add2(sum[1][i], g[i]);
                    H[i] = fma2(inv_h2, fma2(xhat, along2, fma2(g[i], m[i], mean_g2)), H[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = mul2(alpha2, H[i]);
            store_pairs(dx, count, vec, v);
            if (p.y) {
                lds8<Y>(stage + p.off_y, t, v);
                parameters(p.cache_gate, par_gate, t, m);
                if (!POST) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        sum[2][i] = fma2(H[i], v[i], sum[2][i]);
                        H[i] = mul2(H[i], m[i]);
                    }
                    store_pairs(dy, count, vec, H);
                } else {
                    f32x2 w[4];
                    parameters(p.cache_post, par_post, t, w);
                    if (!VEC && count < 8) {                                               // nothing beyond the row in the sums below
#pragma unroll
                        for (int i = 0; i < 4; ++i) H[i] = pack2(2 * i < count ? unpack2(H[i]).x : 0.f, 2 * i + 1 < count ? unpack2(H[i]).y : 0.f);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x2 yhat = mul2(add2(v[i], off_y2), inv_y2);
                        sum[2][i] = fma2(H[i], yhat, sum[2][i]);
                        H[i] = mul2(mul2(H[i], m[i]), w[i]);                       // the gradient at yhat
                        back0 = add2(back0, H[i]);
                        back1 = fma2(H[i], yhat, back1);
                    }
                    // kept for the second phase in the place of these channels' h (32 bits) or h and dh (16), which have been read
                    reinterpret_cast<ulonglong2*>(stage)[sizeof(S) == 4 ? 2 * t : t] = make_ulonglong2(H[0], H[1]);
                    (sizeof(S) == 4 ? reinterpret_cast<ulonglong2*>(stage) + 2 * t + 1 : reinterpret_cast<ulonglong2*>(stage + p.off_dh) + t)[0] = make_ulonglong2(H[2], H[3]);
                }
            }
        }
        if (POST) {
            float b0 = sum2(back0), b1 = sum2(back1);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                b0 += __shfl_xor_sync(0xFFFFFFFFu, b0, o);
                b1 += __shfl_xor_sync(0xFFFFFFFFu, b1, o);
            }
            float* at = red + (2 + j) * kNormRedFloats;
            if (lane == 0) exchange(2 + j, at + my_warp * 4, make_float4(b0, b1, 0.f, 0.f));
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the kept values lie where the next copy lands
            exchanged_all(2 + j, all_warps * 16);
            b0 = b1 = 0.f;
            for (int w = lane; w < all_warps; w += 32) {
                b0 += at[w * 4];
                b1 += at[w * 4 + 1];
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                b0 += __shfl_xor_sync(0xFFFFFFFFu, b0, o);
                b1 += __shfl_xor_sync(0xFFFFFFFFu, b1, o);
            }
            // dy = (a - mean_a - yhat along_y) inv_y
            const float mean_a = layer_y ? b0 * inv_d : 0.f, along_y = b1 * inv_d;
            const f32x2 mean_a2 = pack2(-mean_a, -mean_a), along_y2 = pack2(-along_y, -along_y);
            if (count > 0) {
                f32x2 v[4];
                lds8<Y>(stage + p.off_y, t, v);
                const ulonglong2 lo = reinterpret_cast<const ulonglong2*>(stage)[sizeof(S) == 4 ? 2 * t : t];
                const ulonglong2 hi = (sizeof(S) == 4 ? reinterpret_cast<const ulonglong2*>(stage) + 2 * t + 1 : reinterpret_cast<const ulonglong2*>(stage + p.off_dh) + t)[0];
                const f32x2 H[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[i] = mul2(fma2(mul2(add2(v[i], off_y2), inv_y2), along_y2, add2(H[i], mean_a2)), inv_y2);
                store_pairs(dy, count, vec, v);
            }
        }
        dx += p.ld_dx;
        dy += p.ld_dy;
        if (++s == p.stages) { s = 0; parity ^= 1u; }
        }
    }
    if (p.partial) flush(worker + batch);
    if (p.cluster > 1) cluster_barrier();                             // nobody's shared memory goes away while a peer writes to it
}

// ---- forward, many wide rows: persistent CTAs, rows staged in shared memory --------------------------------
// The kernel above starts a CTA per row, whose load latency, two reductions and parameter reads follow one another; with many
// rows that is what it costs (8192 x 2240, layer norm, gate and modulation: 44 us).  Here a CTA keeps its threads, its parameter
// vectors (shared memory) and two rows at a time, which share every barrier and every sum over a warp, while the next rows
// arrive by bulk copies.  Every warp takes the mean of its own values, then their squares about it (h in registers, y read again
// from shared memory), and Chan's update joins the warps behind one barrier.
// Measured: the same 33 us (4.5 TB/s; instructions and their latency with 27 warps per SM, neither memory nor issue alone);
// 16385 x 5600, rms around rms with a 32-bit stream, 206 to 215 us (5.1 to 5.3 TB/s, bound by memory).
constexpr int kNormFwdRedOff = 128;
constexpr int kNormFwdHead = kNormFwdRedOff + 4 * 32 * 16;            // two sets of sums for each of the two norms, used in turn
enum { kCacheGate = 1, kCachePost = 2, kCacheMul = 4, kCacheShift = 8 };

template <typename S, typename Y, int VPT, bool POST>
__global__ void __launch_bounds__(1024, 1) norm_residual_forward_rows(const __grid_constant__ NormForward p) {
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + 120);
    float4* red = reinterpret_cast<float4*>(smem + kNormFwdRedOff);
    const int T = (int)blockDim.x, t = (int)threadIdx.x, warp = t >> 5, lane = t & 31, warps = T >> 5;
    const int plane = p.d >> 1;                                       // a vector: the first, then the last four entries of every group
    float* at_vec = reinterpret_cast<float*>(smem + kNormFwdHead);
    float* par_gate = at_vec;
    float* par_post = par_gate + (p.cache & kCacheGate ? p.d : 0);
    float* par_mul = par_post + (p.cache & kCachePost ? p.d : 0);
    float* par_shift = par_mul + (p.cache & kCacheMul ? p.d : 0);
    const int stage0 = kNormFwdHead + 4 * p.d * __popc((unsigned)p.cache);
    const int64_t first = (int64_t)blockIdx.x * p.rows_per_worker;
    const int rows = (int)(first + p.rows_per_worker < p.rows ? p.rows_per_worker : p.rows - first);
    const float inv_d = 1.0f / (float)p.d;
    const bool layer_h = p.norm == kNormLayer, layer_y = POST && p.post == kNormLayer, norm = p.norm != kNormNone;
    if (t == 0) {
        for (int s = 0; s < p.stages; ++s) mbar_init(base + 8u * s, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    pdl_wait_prior_grid();
    auto issue = [&](int r, int s) {                                  // thread 0: row `r` of this worker into stage s
        const uint32_t bar = base + 8u * s, dst = base + (uint32_t)(stage0 + s * p.stage_bytes);
        mbar_expect_tx(bar, (uint32_t)p.d * (uint32_t)(sizeof(S) + (p.y ? sizeof(Y) : 0)));
        bulk_load(dst, static_cast<const S*>(p.x) + (first + r) * p.ld_x, (uint32_t)p.d * sizeof(S), bar);
        if (p.y) bulk_load(dst + p.off_y, static_cast<const Y*>(p.y) + (first + r) * p.ld_y, (uint32_t)p.d * sizeof(Y), bar);
    };
    int next = p.stages < rows ? p.stages : rows;
    if (t == 0)
        for (int r = 0; r < next; ++r) issue(r, r);
    int64_t batch = first / p.rows_per_batch;
    auto rows_left = [&](int64_t row) { const int64_t n = (batch + 1) * p.rows_per_batch - row; return (int)(n < rows ? n : rows); };
    int batch_end = rows_left(first);
    bool have[VPT];
#pragma unroll
    for (int k = 0; k < VPT; ++k) have[k] = (t + k * T) * 8 < p.d;
    // channels of a warp: its own as a reciprocal; those of warp `lane`
    auto channels = [&](int w) {
        int n = 0;
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int left = (p.d >> 3) - k * T - 32 * w;
            n += left < 0 ? 0 : (left > 32 ? 32 : left);
        }
        return 8 * n;
    };
    const float own_share = 1.f / (float)channels(warp), n_lane = lane < warps ? (float)channels(lane) : 0.f;
    auto refresh = [&]() {                                            // every thread its own groups
#pragma unroll
        for (int k = 0; k < VPT; ++k)
            if (have[k]) {
                const int gi = t + k * T, c = gi * 8;
                float m[8], a[8];
                auto keep = [&](float* vector) {
                    reinterpret_cast<float4*>(vector)[gi] = make_float4(m[0], m[1], m[2], m[3]);
                    reinterpret_cast<float4*>(vector + plane)[gi] = make_float4(m[4], m[5], m[6], m[7]);
                };
                if (p.cache & kCacheGate) { load_param(p.gate, batch, c, 8, true, 1, 1.f, m); keep(par_gate); }
                if (p.cache & kCachePost) { load_param(p.post_weight, 0, c, 8, true, 1, 1.f, m); keep(par_post); }
                if (p.cache & kCacheShift) { load_param(p.shift, batch, c, 8, true, 1, 0.f, m); keep(par_shift); }
                if (p.cache & kCacheMul) {
                    load_param(p.weight, 0, c, 8, true, 1, 1.f, m);
                    load_param(p.scale, batch, c, 8, true, 1, 0.f, a);
#pragma unroll
                    for (int i = 0; i < 8; ++i) m[i] = fmaf(m[i], a[i], m[i]);
                    keep(par_mul);
                }
            }
    };
    refresh();
    // eight entries of a vector: kept, read through the caches, or absent
    auto entries = [&](int bit, const float* vector, const NormVec& v, int64_t which, int gi, float none, f32x2 (&m)[4]) {
        if (p.cache & bit) {
            const ulonglong2 a = reinterpret_cast<const ulonglong2*>(vector)[gi], b = reinterpret_cast<const ulonglong2*>(vector + plane)[gi];
            m[0] = a.x; m[1] = a.y; m[2] = b.x; m[3] = b.y;
        } else {
            float f[8];
            load_param(v, which, gi * 8, 8, true, 1, none, f);
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] = pack2(f[2 * i], f[2 * i + 1]);
        }
    };
    // mean (layer, else 0) and sum of squares about it of both rows, over the CTA: every warp about the mean of its own values, joined by
    // Chan's update
    auto statistics = [&](auto&& values, bool layer, int set, float (&mean)[2], float (&m2)[2]) {      // values(j, k, v): group k of row j
        float own[2] = {0.f, 0.f};
        if (layer) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                f32x2 a = 0ull;
#pragma unroll
                for (int k = 0; k < VPT; ++k)
                    if (have[k]) {
                        f32x2 v[4];
                        values(j, k, v);
                        a = add2(a, add2(add2(v[0], v[1]), add2(v[2], v[3])));
                    }
                own[j] = sum2(a);
            }
            warp_sum2(own, lane);
            own[0] *= own_share;
            own[1] *= own_share;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const f32x2 minus = pack2(-own[j], -own[j]);
            f32x2 a = 0ull;
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (have[k]) {
                    f32x2 v[4];
                    values(j, k, v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x2 u = layer ? add2(v[i], minus) : v[i];
                        a = fma2(u, u, a);
                    }
                }
            m2[j] = sum2(a);
        }
        warp_sum2(m2, lane);
        float4* at = red + set * 32;
        if (lane == 0) at[warp] = make_float4(own[0], own[1], m2[0], m2[1]);
        __syncthreads();
        const float4 a = lane < warps ? at[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
        m2[0] = a.z;
        m2[1] = a.w;
        mean[0] = mean[1] = 0.f;
        if (layer) {
            const float base0 = at[0].x, base1 = at[0].y;            // (means as offsets from the first warp's)
            mean[0] = n_lane * (a.x - base0);
            mean[1] = n_lane * (a.y - base1);
            warp_sum2(mean, lane);
            mean[0] = fmaf(mean[0], inv_d, base0);
            mean[1] = fmaf(mean[1], inv_d, base1);
            m2[0] = fmaf(n_lane * (a.x - mean[0]), a.x - mean[0], m2[0]);
            m2[1] = fmaf(n_lane * (a.y - mean[1]), a.y - mean[1], m2[1]);
        }
        warp_sum2(m2, lane);
    };
    const f32x2 alpha2 = pack2(p.alpha, p.alpha);
    int s = 0, turn = 0;
    uint32_t parity = 0;
    for (int r = 0, nr; r < rows; r += nr) {
        if (r == batch_end) {
            ++batch;
            batch_end = r + rows_left(first + r);
            refresh();
        }
        nr = r + 1 < rows && r + 1 < batch_end ? 2 : 1;
        const uint8_t* stage[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            stage[j] = smem + stage0 + s * p.stage_bytes;
            if (j < nr) {
                // a wait that gives up records it and goes on (the barriers below stay matched)
                if (!mbar_wait(base + 8u * s, parity, abort_flag) && !*abort_flag) {
                    atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_NORM);
                    *abort_flag = 1;
                }
                if (++s == p.stages) { s = 0; parity ^= 1u; }
            }
        }
        if (nr == 1) stage[1] = stage[0];                            // (computed twice, stored once)
        float mean_y[2] = {0.f, 0.f}, inv_y[2] = {1.f, 1.f};
        if (POST) {
            float m2[2];
            // (read again for every pass: kept, they would spill)
            statistics([&](int j, int k, f32x2 (&v)[4]) {
                asm volatile("" ::: "memory");
                lds8<Y>(stage[j] + p.off_y, t + k * T, v);
            }, layer_y, turn, mean_y, m2);
#pragma unroll
            for (int j = 0; j < 2; ++j) inv_y[j] = rsqrtf(fmaf(m2[j], inv_d, p.eps));
        }
        f32x2 h[2][VPT][4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const f32x2 off_y = pack2(-mean_y[j] * inv_y[j], -mean_y[j] * inv_y[j]), inv_y2 = pack2(inv_y[j], inv_y[j]);
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (have[k]) {
                    const int gi = t + k * T;
                    f32x2 x[4], m[4];
                    lds8<S>(stage[j], gi, x);
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[j][k][i] = x[i];
                    if (p.alpha != 1.f) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) h[j][k][i] = mul2(alpha2, x[i]);
                    }
                    if (p.y) {
                        lds8<Y>(stage[j] + p.off_y, gi, x);
                        if (POST) {
                            entries(kCachePost, par_post, p.post_weight, 0, gi, 1.f, m);
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[i] = mul2(fma2(x[i], inv_y2, off_y), m[i]);
                        }
                        entries(kCacheGate, par_gate, p.gate, batch, gi, 1.f, m);
#pragma unroll
                        for (int i = 0; i < 4; ++i) h[j][k][i] = fma2(m[i], x[i], h[j][k][i]);
                    }
                    if (p.h && j < nr) store_pairs(static_cast<S*>(p.h) + (first + r + j) * p.ld_h + gi * 8, 8, true, h[j][k]);
                }
        }
        float mean[2], m2[2];
        statistics([&](int j, int k, f32x2 (&v)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = h[j][k][i];
        }, layer_h, 2 + turn, mean, m2);
        turn ^= 1;
        // every thread has read its part of these rows: their stages take the rows that follow
        if (t == 0)
            for (; next < rows && next < r + nr + p.stages; ++next) issue(next, next % p.stages);
        if (!norm) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (j < nr) {
                const float inv = rsqrtf(fmaf(m2[j], inv_d, p.eps));
                const f32x2 off = pack2(-mean[j], -mean[j]), inv2 = pack2(inv, inv);
#pragma unroll
                for (int k = 0; k < VPT; ++k)
                    if (have[k]) {
                        const int gi = t + k * T;
                        f32x2 m[4], a[4];
                        if (p.cache & kCacheMul) {
                            entries(kCacheMul, par_mul, p.weight, 0, gi, 1.f, m);
                        } else {
                            entries(0, par_mul, p.weight, 0, gi, 1.f, m);
                            entries(0, par_mul, p.scale, batch, gi, 0.f, a);
#pragma unroll
                            for (int i = 0; i < 4; ++i) m[i] = fma2(m[i], a[i], m[i]);
                        }
                        entries(kCacheShift, par_shift, p.shift, batch, gi, 0.f, a);
#pragma unroll
                        for (int i = 0; i < 4; ++i) a[i] = fma2(mul2(add2(h[j][k][i], off), inv2), m[i], a[i]);
                        store_pairs(static_cast<Y*>(p.n) + (first + r + j) * p.ld_n + gi * 8, 8, true, a);
                    }
            }
    }
}

struct NormVecGrads {
    int64_t rows;
    int d;
    int64_t rows_per_batch, rows_per_worker, batches;
    const float* partial;
    NormVec gate, post_weight, weight, scale;
    // outputs, float; the strides say whether a gradient is per batch (d or more) or summed over all batches (0)
    float *dgate, *dscale, *dshift, *dweight, *dpost_weight;
    int64_t dgate_stride, dscale_stride, dshift_stride;
};

// blockDim = (32 columns, kSlotLanes): lane l of a column adds slots l, l + kSlotLanes, ...; lane 0 adds the lanes' sums in order.
// Batches follow one another, which a few of them hide; with a vector row for each of 16384 rows of 2240 the gradients take 36 ms.
constexpr int kSlotLanes = 16;
__global__ void __launch_bounds__(32 * kSlotLanes) norm_vector_gradients(const __grid_constant__ NormVecGrads p) {
    __shared__ float part[3][kSlotLanes][32];
    pdl_wait_prior_grid();
    const int c = (int)blockIdx.x * 32 + (int)threadIdx.x;
    const bool live = c < p.d;
    float t_gate = 0.f, t_scale = 0.f, t_shift = 0.f, t_weight = 0.f, t_post = 0.f;      // over all batches
    for (int64_t b = 0; b < p.batches; ++b) {
        const int64_t r0 = b * p.rows_per_batch, r1 = (r0 + p.rows_per_batch < p.rows ? r0 + p.rows_per_batch : p.rows) - 1;
        const int64_t w1 = r1 / p.rows_per_worker;
        float sp = 0.f, ss = 0.f, sq = 0.f;
        if (live) {
#pragma unroll 4
            for (int64_t w = r0 / p.rows_per_worker + threadIdx.y; w <= w1; w += kSlotLanes) {
                const float* at = p.partial + (w + b) * 3 * p.d + c;
                sp += at[0];
                ss += at[p.d];
                sq += at[2 * p.d];
            }
        }
        __syncthreads();                                      // the previous batch's sums have been read
        part[0][threadIdx.y][threadIdx.x] = sp;
        part[1][threadIdx.y][threadIdx.x] = ss;
        part[2][threadIdx.y][threadIdx.x] = sq;
        __syncthreads();
        if (threadIdx.y == 0 && live) {
            for (int l = 1; l < kSlotLanes; ++l) {
                sp += part[0][l][threadIdx.x];
                ss += part[1][l][threadIdx.x];
                sq += part[2][l][threadIdx.x];
            }
            const float dgate = vec_entry(p.post_weight, 0, c, 1.f) * sq, dscale = vec_entry(p.weight, 0, c, 1.f) * sp;
            if (p.dgate && p.dgate_stride) p.dgate[b * p.dgate_stride + c] = dgate;
            if (p.dscale && p.dscale_stride) p.dscale[b * p.dscale_stride + c] = dscale;
            if (p.dshift && p.dshift_stride) p.dshift[b * p.dshift_stride + c] = ss;
            t_gate += dgate;
            t_scale += dscale;
            t_shift += ss;
            t_weight = fmaf(1.f + vec_entry(p.scale, b, c, 0.f), sp, t_weight);
            t_post = fmaf(vec_entry(p.gate, b, c, 1.f), sq, t_post);
        }
    }
    if (threadIdx.y == 0 && live) {
        if (p.dgate && !p.dgate_stride) p.dgate[c] = t_gate;
        if (p.dscale && !p.dscale_stride) p.dscale[c] = t_scale;
        if (p.dshift && !p.dshift_stride) p.dshift[c] = t_shift;
        if (p.dweight) p.dweight[c] = t_weight;
        if (p.dpost_weight) p.dpost_weight[c] = t_post;
    }
}

}  // namespace kq
