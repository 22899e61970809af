// Norms before and after a transformer block, fused with the block's gate and residual scale, and their backward pass.
//
// Forward, one row t of d channels, b = t / rows_per_batch:
//     r = post(y) post_weight          post, norm in {none, rms, layer}:  v -> (v - mean) / sqrt(mean((v - mean)^2) + eps)
//     h = alpha x + gate_b r                                              (rms: mean taken as 0)
//     n = norm(h) weight (1 + scale_b) + shift_b
// The row stays in registers between its one read and its one write; h enters the norm unrounded (32 bits), so n does
// not carry the rounding of h to the stream's type.  All statistics are 32-bit sums, the variance is taken about the mean
// (two reductions) because E[v^2] - E[v]^2 loses what a large mean leaves.
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
// All kernels are bound by memory: 2 reads and 2 writes (forward), 4 reads and 2 writes (backward) per element.
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
        const float* q = static_cast<const float*>(p.ptr) + at;
        if (vec) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(q)), b = __ldg(reinterpret_cast<const float4*>(q) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < count ? __ldg(q + i * step) : 0.f;
        }
    } else {
        const uint16_t* q = static_cast<const uint16_t*>(p.ptr) + at;
        uint4 u;
        if (vec) {
            u = __ldg(reinterpret_cast<const uint4*>(q));
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = 2 * i < count ? __ldg(q + 2 * i * step) : 0u, hi = 2 * i + 1 < count ? __ldg(q + (2 * i + 1) * step) : 0u;
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
};

// blockDim = (threads of a row, rows of a CTA): one warp per row and several rows for narrow d, else one row per CTA.
// Thread i owns the 8-channel groups i, i + blockDim.x, ...: VPT of them.
template <typename S, typename Y, int VPT>
__global__ void norm_residual_forward(const NormForward p) {
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
        inv_y = 1.0f / sqrtf(s[0] * inv_d + p.eps);
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
    const float inv = 1.0f / sqrtf(s[0] * inv_d + p.eps);
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
    // staged kernel: stages, bytes of a stage, whether dh is staged, offsets of the rows, which parameter vectors are kept in shared memory
    int stages, stage_bytes, stage_dh, off_dh, off_dn, off_y, cache_m, cache_gate, cache_post;
};

// ---- backward, narrow rows: one warp per row --------------------------------------------------------
// Worker w = blockIdx.x * blockDim.y + threadIdx.y takes rows [w rows_per_worker, ...); d <= 256 VPT, rows in registers.
template <typename S, typename Y, int VPT>
__global__ void __launch_bounds__(256) norm_residual_backward_warp(const NormBackward p) {
    const int64_t worker = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int64_t first = worker * p.rows_per_worker;
    const int64_t last = first + p.rows_per_worker < p.rows ? first + p.rows_per_worker : p.rows;
    pdl_wait_prior_grid();
    if (first >= last) return;
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
    auto flush = [&](int64_t slot) {
        float* out = p.partial + slot * 3 * p.d;
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int k = 0; k < VPT; ++k) {
                if (count[k] > 0) store8(out + (int64_t)q * p.d + column(k), count[k], vec, step, sum[q][k]);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[q][k][i] = 0.f;
            }
    };
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int k = 0; k < VPT; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[q][k][i] = 0.f;
    int64_t batch = first / p.rows_per_batch;
    for (int64_t row = first; row < last; ++row) {
        if (row >= (batch + 1) * p.rows_per_batch) {
            if (p.partial) flush(worker + batch);
            batch = row / p.rows_per_batch;
        }
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
        const float inv_h = 1.0f / sqrtf(sq[0] * inv_d + p.eps);
        const float along_h = sq[1] * inv_d * inv_h;
        const float inv_y = post ? 1.0f / sqrtf(sq[2] * inv_d + p.eps) : 1.f;
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
    if (p.partial) flush(worker + batch);
}

// ---- backward, wide rows: one CTA per row, rows staged in shared memory ---------------------------------
// A CTA is a worker.  The four rows of an iteration arrive in shared memory by bulk copies issued `stages` rows ahead, so
// that nothing waits for a load latency and a row needs no registers; a thread owns the 8-channel groups t, t + T, ... and
// reads them again in every phase.  What a thread writes to shared memory (parameters, see below) only it reads.
// One barrier for all statistics of a row: each warp takes its means, then its squares about ITS means, and every warp
// combines the warps' (mean, sum of squares) pairs by Chan's update, exact in the sense that nothing cancels:
//     M2 = sum_w M2_w + n_w (mean_w - mean)^2,    sum g (h - mean) = sum_w [G1_w + (mean_w - mean) G0_w].
// Parameter vectors (weight (1 + scale), gate, post_weight) are kept in shared memory as floats where they fit, refreshed
// at the start of a batch; else they are read through the caches.
// Rows that bulk copies cannot take (16-byte alignment) are copied into the same place by the threads, element by element.
constexpr int kNormStageMax = 4;
constexpr int kNormRedOff = 128;                                    // barriers and the abort word in front
constexpr int kNormHeadBytes = kNormRedOff + 2 * 32 * 8 * 4;

template <typename T>
__device__ __forceinline__ void lds_widen(const uint8_t* row, int group, float (&v)[8]) {
    Pack8<T> q;
    const uint4* at = reinterpret_cast<const uint4*>(row) + group * (sizeof(T) / 2);
    const uint4 a = at[0];
    q.w[0] = a.x; q.w[1] = a.y; q.w[2] = a.z; q.w[3] = a.w;
    if constexpr (sizeof(T) == 4) {
        const uint4 b = at[1];
        q.w[4] = b.x; q.w[5] = b.y; q.w[6] = b.z; q.w[7] = b.w;
    }
    pack_widen(q, v);
}
__device__ __forceinline__ void lds_floats(const float* at, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4*>(at)[0], b = reinterpret_cast<const float4*>(at)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void sts_floats(float* at, const float (&v)[8]) {
    reinterpret_cast<float4*>(at)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(at)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
// a row that is not 16-byte aligned, into shared memory; the tail of the last group becomes 0
template <typename T>
__device__ __forceinline__ void copy_row(uint8_t* dst, const T* src, int d) {
    T* out = reinterpret_cast<T*>(dst);
    for (int c = (int)threadIdx.x; c < (d + 7) / 8 * 8; c += (int)blockDim.x) out[c] = c < d ? src[c] : Elem<T>::from_f32(0.f);
}

template <typename S, typename Y, int VPT>
__global__ void __launch_bounds__(VPT == 2 ? 576 : 512, 1) norm_residual_backward(const NormBackward p) {
    extern __shared__ __align__(128) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + 64);
    float* red = reinterpret_cast<float*>(smem + kNormRedOff);
    const int T = (int)blockDim.x, t = (int)threadIdx.x, warp = t >> 5, lane = t & 31, warps = T >> 5;
    const int padded = (p.d + 7) / 8 * 8;
    float* par_m = reinterpret_cast<float*>(smem + kNormHeadBytes);
    float* par_gate = par_m + (p.cache_m ? padded : 0);
    float* par_post = par_gate + (p.cache_gate ? padded : 0);
    const int stage0 = kNormHeadBytes + 4 * padded * (p.cache_m + p.cache_gate + p.cache_post);
    const int64_t worker = blockIdx.x, first = worker * p.rows_per_worker;
    const int64_t last = first + p.rows_per_worker < p.rows ? first + p.rows_per_worker : p.rows;
    const bool vec = p.vec != 0;
    const float inv_d = 1.0f / (float)p.d;
    const bool layer_h = p.norm == kNormLayer, layer_y = p.post == kNormLayer, post = p.y && p.post != kNormNone;
    if (t == 0) {
        for (int s = 0; s < p.stages; ++s) mbar_init(base + 8u * s, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    pdl_wait_prior_grid();
    auto issue = [&](int64_t row) {                                  // thread 0
        const int s = (int)((row - first) % p.stages);
        const uint32_t bar = base + 8u * s, dst = base + (uint32_t)(stage0 + s * p.stage_bytes);
        const uint32_t bytes_s = (uint32_t)p.d * sizeof(S), bytes_y = (uint32_t)p.d * sizeof(Y);
        mbar_expect_tx(bar, bytes_s * (p.stage_dh ? 2 : 1) + bytes_y * ((p.dn ? 1 : 0) + (p.y ? 1 : 0)));
        bulk_load(dst, static_cast<const S*>(p.h) + row * p.ld_h, bytes_s, bar);
        if (p.stage_dh) bulk_load(dst + p.off_dh, static_cast<const S*>(p.dh) + row * p.ld_dh, bytes_s, bar);
        if (p.dn) bulk_load(dst + p.off_dn, static_cast<const Y*>(p.dn) + row * p.ld_dn, bytes_y, bar);
        if (p.y) bulk_load(dst + p.off_y, static_cast<const Y*>(p.y) + row * p.ld_y, bytes_y, bar);
    };
    if (vec && t == 0)
        for (int64_t r = first; r < first + p.stages && r < last; ++r) issue(r);
    int count[VPT];
    int mine = 0;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        count[k] = owned(p.d, (t + k * T) * 8, 1);
        mine += count[k];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
    const float n_w = (float)mine, inv_n = 1.f / (mine ? (float)mine : 1.f);
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
        float* out = p.partial + slot * 3 * p.d;
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) store8(out + (int64_t)q * p.d + (t + k * T) * 8, count[k], vec, 1, sum[q][k]);
        clear();
    };
    clear();
    int64_t batch = first / p.rows_per_batch;
    auto multiplier = [&](int k, float (&m)[8]) {
        if (p.cache_m) {
            lds_floats(par_m + (t + k * T) * 8, m);
        } else {
            float a[8];
            load_param(p.weight, 0, (t + k * T) * 8, count[k], vec, 1, 1.f, m);
            load_param(p.scale, batch, (t + k * T) * 8, count[k], vec, 1, 0.f, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) m[i] = fmaf(m[i], a[i], m[i]);
        }
    };
    auto refresh = [&]() {
#pragma unroll
        for (int k = 0; k < VPT; ++k)
            if (count[k] > 0) {
                const int c = (t + k * T) * 8;
                float m[8], a[8];
                if (p.cache_m) {
                    load_param(p.weight, 0, c, count[k], vec, 1, 1.f, m);
                    load_param(p.scale, batch, c, count[k], vec, 1, 0.f, a);
#pragma unroll
                    for (int i = 0; i < 8; ++i) m[i] = fmaf(m[i], a[i], m[i]);
                    sts_floats(par_m + c, m);
                }
                if (p.cache_gate) {
                    load_param(p.gate, batch, c, count[k], vec, 1, 1.f, m);
                    sts_floats(par_gate + c, m);
                }
                if (p.cache_post) {
                    load_param(p.post_weight, 0, c, count[k], vec, 1, 1.f, m);
                    sts_floats(par_post + c, m);
                }
            }
    };
    refresh();
    for (int64_t row = first; row < last; ++row) {
        const int64_t i_row = row - first;
        const int s = (int)(i_row % p.stages);
        uint8_t* stage = smem + stage0 + s * p.stage_bytes;
        if (row >= (batch + 1) * p.rows_per_batch) {
            if (p.partial) flush(worker + batch);
            batch = row / p.rows_per_batch;
            refresh();
        }
        if (vec) {
            if (p.stages == 1 && i_row > 0) {                        // no second slot: the next row starts when this one is done
                __syncthreads();
                if (t == 0) issue(row);
            }
            // a wait that gives up records it and goes on (the barriers below stay matched)
            if (!mbar_wait(base + 8u * s, (uint32_t)(i_row / p.stages) & 1u, abort_flag) && !*abort_flag) {
                atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_NORM);
                *abort_flag = 1;
            }
        } else {
            __syncthreads();
            copy_row(stage, static_cast<const S*>(p.h) + row * p.ld_h, p.d);
            if (p.stage_dh) copy_row(stage + p.off_dh, static_cast<const S*>(p.dh) + row * p.ld_dh, p.d);
            if (p.dn) copy_row(stage + p.off_dn, static_cast<const Y*>(p.dn) + row * p.ld_dn, p.d);
            if (p.y) copy_row(stage + p.off_y, static_cast<const Y*>(p.y) + row * p.ld_y, p.d);
            __syncthreads();
        }
        // this warp's means of h and y and its sum of g (layer)
        float mu[4] = {0.f, 0.f, 0.f, 0.f};
        if (layer_h || layer_y) {
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) {
                    float v[8], m[8];
                    if (layer_h) {
                        lds_widen<S>(stage, t + k * T, v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) mu[0] += v[i];
                        lds_widen<Y>(stage + p.off_dn, t + k * T, v);
                        multiplier(k, m);
#pragma unroll
                        for (int i = 0; i < 8; ++i) mu[1] = fmaf(v[i], m[i], mu[1]);
                    }
                    if (layer_y) {
                        lds_widen<Y>(stage + p.off_y, t + k * T, v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) mu[2] += v[i];
                    }
                }
            warp_sum4(mu, lane);
            mu[0] *= inv_n;
            mu[2] *= inv_n;
        }
        // squares about them
        float sq[4] = {0.f, 0.f, 0.f, 0.f};
        if (p.norm != kNormNone || post) {
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) {
                    float v[8], m[8], g[8];
                    if (p.norm != kNormNone) {
                        lds_widen<S>(stage, t + k * T, v);
                        lds_widen<Y>(stage + p.off_dn, t + k * T, g);
                        multiplier(k, m);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float u = i < count[k] ? v[i] - mu[0] : 0.f;
                            sq[0] = fmaf(u, u, sq[0]);
                            sq[1] = fmaf(g[i] * m[i], u, sq[1]);
                        }
                    }
                    if (post) {
                        lds_widen<Y>(stage + p.off_y, t + k * T, v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float u = i < count[k] ? v[i] - mu[2] : 0.f;
                            sq[2] = fmaf(u, u, sq[2]);
                        }
                    }
                }
            warp_sum4(sq, lane);
        }
        if (lane == 0) {
            float4* at = reinterpret_cast<float4*>(red + warp * 8);
            at[0] = make_float4(n_w, mu[0], mu[1], mu[2]);
            at[1] = make_float4(sq[0], sq[1], sq[2], 0.f);
        }
        __syncthreads();
        // every thread is done with the row before: its slot takes the row `stages` further on
        if (vec && t == 0 && p.stages > 1 && i_row > 0 && row - 1 + p.stages < last) issue(row - 1 + p.stages);
        float mean_h = 0.f, mean_g = 0.f, mean_y = 0.f;
        {
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
            if (lane < warps) {
                a = reinterpret_cast<const float4*>(red + lane * 8)[0];
                b = reinterpret_cast<const float4*>(red + lane * 8)[1];
            }
            if (layer_h || layer_y) {
                float tot[4] = {a.x * a.y, a.z, a.x * a.w, 0.f};
                warp_sum4(tot, lane);
                mean_h = tot[0] * inv_d;
                mean_g = tot[1] * inv_d;
                mean_y = tot[2] * inv_d;
            }
            const float dh_ = a.y - mean_h, dy_ = a.w - mean_y;
            sq[0] = fmaf(a.x * dh_, dh_, b.x);
            sq[1] = fmaf(dh_, a.z, b.y);
            sq[2] = fmaf(a.x * dy_, dy_, b.z);
            sq[3] = 0.f;
            warp_sum4(sq, lane);
        }
        const float inv_h = 1.0f / sqrtf(sq[0] * inv_d + p.eps);
        const float along_h = sq[1] * inv_d * inv_h;
        const float inv_y = post ? 1.0f / sqrtf(sq[2] * inv_d + p.eps) : 1.f;
        float back[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < VPT; ++k)
            if (count[k] > 0) {
                asm volatile("" ::: "memory");                     // one group at a time: the registers hold the column sums
                const int gi = t + k * T, c = gi * 8;
                float Hk[8], v[8], m[8];
                if (p.stage_dh) {
                    lds_widen<S>(stage + p.off_dh, gi, Hk);
                } else if (p.dh) {
                    Pack8<S> q;
                    load_pack(static_cast<const S*>(p.dh) + row * p.ld_dh + c, count[k], vec, 1, q);
                    pack_widen(q, Hk);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) Hk[i] = 0.f;
                }
                if (p.norm != kNormNone) {
                    float g[8];
                    lds_widen<S>(stage, gi, v);
                    lds_widen<Y>(stage + p.off_dn, gi, g);
                    multiplier(k, m);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float xhat = (v[i] - mean_h) * inv_h;
                        sum[0][k][i] = fmaf(g[i], xhat, sum[0][k][i]);
                        sum[1][k][i] += g[i];
                        Hk[i] = fmaf(inv_h, fmaf(g[i], m[i], -mean_g) - xhat * along_h, Hk[i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = p.alpha * Hk[i];
                store8(static_cast<S*>(p.dx) + row * p.ld_dx + c, count[k], vec, 1, v);
                if (p.y) {
                    float a[8];
                    lds_widen<Y>(stage + p.off_y, gi, v);
                    if (p.cache_gate) lds_floats(par_gate + c, m); else load_param(p.gate, batch, c, count[k], vec, 1, 1.f, m);
                    if (post) {
                        if (p.cache_post) lds_floats(par_post + c, a); else load_param(p.post_weight, 0, c, count[k], vec, 1, 1.f, a);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float yhat = (v[i] - mean_y) * inv_y;
                        sum[2][k][i] = fmaf(Hk[i], yhat, sum[2][k][i]);
                        Hk[i] *= m[i];                          // from here on the gradient at the branch
                        if (post) {
                            Hk[i] = i < count[k] ? Hk[i] * a[i] : 0.f;
                            back[0] += Hk[i];
                            back[1] = fmaf(Hk[i], yhat, back[1]);
                        }
                    }
                    if (!post) store8(static_cast<Y*>(p.dy) + row * p.ld_dy + c, count[k], vec, 1, Hk);
                    else {
                        // kept for the second phase in the place of this group's h and dh, which have been read
                        uint4* lo = reinterpret_cast<uint4*>(stage) + gi * (sizeof(S) / 2);
                        uint4* hi = sizeof(S) == 4 ? lo + 1 : reinterpret_cast<uint4*>(stage + p.off_dh) + gi;
                        *reinterpret_cast<float4*>(lo) = make_float4(Hk[0], Hk[1], Hk[2], Hk[3]);
                        *reinterpret_cast<float4*>(hi) = make_float4(Hk[4], Hk[5], Hk[6], Hk[7]);
                    }
                }
            }
        if (post) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                back[0] += __shfl_xor_sync(0xFFFFFFFFu, back[0], o);
                back[1] += __shfl_xor_sync(0xFFFFFFFFu, back[1], o);
            }
            float* at = red + 32 * 8;
            if (lane == 0) { at[warp * 2] = back[0]; at[warp * 2 + 1] = back[1]; }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // H lies where the next copy lands
            __syncthreads();
            back[0] = lane < warps ? at[lane * 2] : 0.f;
            back[1] = lane < warps ? at[lane * 2 + 1] : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                back[0] += __shfl_xor_sync(0xFFFFFFFFu, back[0], o);
                back[1] += __shfl_xor_sync(0xFFFFFFFFu, back[1], o);
            }
            const float mean_a = layer_y ? back[0] * inv_d : 0.f, along_y = back[1] * inv_d;
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) {
                    const int gi = t + k * T;
                    float v[8], a[8];
                    lds_widen<Y>(stage + p.off_y, gi, v);
                    const uint4* lo = reinterpret_cast<const uint4*>(stage) + gi * (sizeof(S) / 2);
                    const uint4* hi = sizeof(S) == 4 ? lo + 1 : reinterpret_cast<const uint4*>(stage + p.off_dh) + gi;
                    const float4 x = *reinterpret_cast<const float4*>(lo), z = *reinterpret_cast<const float4*>(hi);
                    a[0] = x.x; a[1] = x.y; a[2] = x.z; a[3] = x.w; a[4] = z.x; a[5] = z.y; a[6] = z.z; a[7] = z.w;
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = (a[i] - mean_a - (v[i] - mean_y) * inv_y * along_y) * inv_y;
                    store8(static_cast<Y*>(p.dy) + row * p.ld_dy + gi * 8, count[k], vec, 1, v);
                }
        }
    }
    if (p.partial && first < last) flush(worker + batch);
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

__device__ __forceinline__ float vec_entry(const NormVec& p, int64_t which, int at, float none) {
    if (!p.ptr) return none;
    const int64_t i = which * p.stride + at;
    if (p.type == kTypeF32) return static_cast<const float*>(p.ptr)[i];
    if (p.type == kTypeF16) return __half2float(static_cast<const __half*>(p.ptr)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p.ptr)[i]);
}
// blockDim = (32 columns, kSlotLanes): lane l of a column adds slots l, l + kSlotLanes, ...; lane 0 adds the lanes' sums in order.
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
