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
// Both kernels are bound by memory: 2 reads and 2 writes (forward), 4 reads and 2 writes (backward) per element.
#pragma once
#include "kq_common.cuh"

namespace kq {

enum { kNormNone = 0, kNormRms = 1, kNormLayer = 2 };
enum { kTypeF32 = 0, kTypeBf16 = 1, kTypeF16 = 2 };
constexpr int kNormMaxD = 16384;

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
// `count` of the eight elements exist (8 on the vector path; the others read as 0)
template <typename T>
__device__ __forceinline__ void load_pack(const T* p, int count, bool vec, Pack8<T>& out) {
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
        for (int i = 0; i < 8; ++i) out.w[i] = i < count ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
    } else {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = 2 * i < count ? q[2 * i] : 0u, hi = 2 * i + 1 < count ? q[2 * i + 1] : 0u;
            out.w[i] = lo | (hi << 16);
        }
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int count, bool vec, const float (&v)[8]) {
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
            if (i < count) p[i] = Elem<T>::from_f32(v[i]);
    }
}
// eight entries of a parameter vector at channel c (absent: `none`)
__device__ __forceinline__ void load_param(const NormVec& p, int64_t batch, int c, int count, bool vec, float none, float (&v)[8]) {
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
            for (int i = 0; i < 8; ++i) v[i] = i < count ? __ldg(q + i) : 0.f;
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
                const uint32_t lo = 2 * i < count ? __ldg(q + 2 * i) : 0u, hi = 2 * i + 1 < count ? __ldg(q + 2 * i + 1) : 0u;
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
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (row >= p.rows) return;        // whole warps: a CTA with more than one row has one warp per row
    const int64_t batch = row / p.rows_per_batch;
    const bool vec = p.vec != 0;
    const float inv_d = 1.0f / (float)p.d;
    int phase = 0;
    Pack8<S> xs[VPT];
    Pack8<Y> ys[VPT];
    int count[VPT];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int c = ((int)threadIdx.x + k * (int)blockDim.x) * 8;
        count[k] = p.d - c < 0 ? 0 : (p.d - c > 8 ? 8 : p.d - c);
        if (count[k] > 0) {
            load_pack(static_cast<const S*>(p.x) + row * p.ld_x + c, count[k], vec, xs[k]);
            if (p.y) load_pack(static_cast<const Y*>(p.y) + row * p.ld_y + c, count[k], vec, ys[k]);
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
            const int c = ((int)threadIdx.x + k * (int)blockDim.x) * 8;
            pack_widen(xs[k], h[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[k][i] *= p.alpha;
            if (p.y) {
                float v[8], g[8];
                pack_widen(ys[k], v);
                if (p.post != kNormNone) {
                    load_param(p.post_weight, 0, c, count[k], vec, 1.f, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = (v[i] - mean_y) * inv_y * g[i];
                }
                load_param(p.gate, batch, c, count[k], vec, 1.f, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[k][i] = i < count[k] ? fmaf(g[i], v[i], h[k][i]) : 0.f;
            }
            if (p.h) store8(static_cast<S*>(p.h) + row * p.ld_h + c, count[k], vec, h[k]);
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
            const int c = ((int)threadIdx.x + k * (int)blockDim.x) * 8;
            float a[8], w[8];
            load_param(p.weight, 0, c, count[k], vec, 1.f, w);
            load_param(p.scale, batch, c, count[k], vec, 0.f, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = fmaf(w[i], a[i], w[i]);
            load_param(p.shift, batch, c, count[k], vec, 0.f, a);
#pragma unroll
            for (int i = 0; i < 8; ++i) a[i] = fmaf((h[k][i] - mean) * inv, w[i], a[i]);
            store8(static_cast<Y*>(p.n) + row * p.ld_n + c, count[k], vec, a);
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
};

// One batch's column sums of this worker -> slot (worker + batch); the sums start again from zero.
template <int VPT>
__device__ __forceinline__ void flush_sums(const NormBackward& p, int64_t slot, float (&sum)[3][VPT][8], const int (&count)[VPT]) {
    float* out = p.partial + slot * 3 * p.d;
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int c = ((int)threadIdx.x + k * (int)blockDim.x) * 8;
            if (count[k] > 0) store8(out + (int64_t)q * p.d + c, count[k], p.vec != 0, sum[q][k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[q][k][i] = 0.f;
        }
}

// Worker w = blockIdx.x * blockDim.y + threadIdx.y takes rows [w rows_per_worker, ...).
template <typename S, typename Y, int VPT>
__global__ void __launch_bounds__(VPT == 1 ? 256 : 512)
norm_residual_backward(const NormBackward p) {
    __shared__ float red[2 * 128];
    const int64_t worker = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int64_t first = worker * p.rows_per_worker;
    int64_t last = first + p.rows_per_worker;
    if (last > p.rows) last = p.rows;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (first >= last) return;
    const bool vec = p.vec != 0;
    const float inv_d = 1.0f / (float)p.d;
    const bool layer_h = p.norm == kNormLayer, layer_y = p.post == kNormLayer, post = p.y && p.post != kNormNone;
    int phase = 0;
    int count[VPT];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int left = p.d - ((int)threadIdx.x + k * (int)blockDim.x) * 8;
        count[k] = left < 0 ? 0 : (left > 8 ? 8 : left);
    }
    float sum[3][VPT][8];
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int k = 0; k < VPT; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[q][k][i] = 0.f;
    int64_t batch = first / p.rows_per_batch;
    int64_t batch_end = (batch + 1) * p.rows_per_batch;
    for (int64_t row = first; row < last; ++row) {
        if (row >= batch_end) {
            if (p.partial) flush_sums<VPT>(p, worker + batch, sum, count);
            batch = row / p.rows_per_batch;
            batch_end = (batch + 1) * p.rows_per_batch;
        }
        Pack8<S> hs[VPT], dhs[VPT];
        Pack8<Y> ys[VPT], dns[VPT];
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int c = ((int)threadIdx.x + k * (int)blockDim.x) * 8;
            if (count[k] > 0) {
                load_pack(static_cast<const S*>(p.h) + row * p.ld_h + c, count[k], vec, hs[k]);
                if (p.dn) load_pack(static_cast<const Y*>(p.dn) + row * p.ld_dn + c, count[k], vec, dns[k]);
                if (p.dh) load_pack(static_cast<const S*>(p.dh) + row * p.ld_dh + c, count[k], vec, dhs[k]);
                if (p.y) load_pack(static_cast<const Y*>(p.y) + row * p.ld_y + c, count[k], vec, ys[k]);
            }
        }
        // means (layer only): of h, of g, of y
        float mu[3] = {0.f, 0.f, 0.f};
        if (layer_h || layer_y) {
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) {
                    const int c = ((int)threadIdx.x + k * (int)blockDim.x) * 8;
                    float v[8], w[8], a[8];
                    if (layer_h) {
                        pack_widen(hs[k], v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) mu[0] += v[i];
                        pack_widen(dns[k], v);
                        load_param(p.weight, 0, c, count[k], vec, 1.f, w);
                        load_param(p.scale, batch, c, count[k], vec, 0.f, a);
#pragma unroll
                        for (int i = 0; i < 8; ++i) mu[1] = fmaf(v[i], fmaf(w[i], a[i], w[i]), mu[1]);
                    }
                    if (layer_y) {
                        pack_widen(ys[k], v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) mu[2] += v[i];
                    }
                }
            row_sum<3>(mu, red, phase);
            mu[0] *= inv_d; mu[1] *= inv_d; mu[2] *= inv_d;
        }
        // squares about the means and g . (h - mean)
        float sq[3] = {0.f, 0.f, 0.f};
        if (p.norm != kNormNone || post) {
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) {
                    const int c = ((int)threadIdx.x + k * (int)blockDim.x) * 8;
                    float v[8], w[8], a[8], g[8];
                    if (p.norm != kNormNone) {
                        pack_widen(hs[k], v);
                        pack_widen(dns[k], g);
                        load_param(p.weight, 0, c, count[k], vec, 1.f, w);
                        load_param(p.scale, batch, c, count[k], vec, 0.f, a);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (i < count[k]) {
                                const float u = v[i] - mu[0];
                                sq[0] = fmaf(u, u, sq[0]);
                                sq[1] = fmaf(g[i] * fmaf(w[i], a[i], w[i]), u, sq[1]);
                            }
                    }
                    if (post) {
                        pack_widen(ys[k], v);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (i < count[k]) sq[2] = fmaf(v[i] - mu[2], v[i] - mu[2], sq[2]);
                    }
                }
            row_sum<3>(sq, red, phase);
        }
        const float inv_h = 1.0f / sqrtf(sq[0] * inv_d + p.eps);
        const float along_h = sq[1] * inv_d * inv_h;            // mean(g xhat)
        const float inv_y = post ? 1.0f / sqrtf(sq[2] * inv_d + p.eps) : 1.f;
        const float mean_y = mu[2];
        // H, dx, the column sums; without a post norm also dy
        float H[VPT][8];
        float back[2] = {0.f, 0.f};                             // sum a, sum a yhat
#pragma unroll
        for (int k = 0; k < VPT; ++k)
            if (count[k] > 0) {
                const int c = ((int)threadIdx.x + k * (int)blockDim.x) * 8;
                float v[8], w[8], a[8];
                if (p.dh) pack_widen(dhs[k], H[k]);
                else
#pragma unroll
                    for (int i = 0; i < 8; ++i) H[k][i] = 0.f;
                if (p.norm != kNormNone) {
                    float g[8];
                    pack_widen(hs[k], v);
                    pack_widen(dns[k], g);
                    load_param(p.weight, 0, c, count[k], vec, 1.f, w);
                    load_param(p.scale, batch, c, count[k], vec, 0.f, a);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float xhat = (v[i] - mu[0]) * inv_h;
                        if (i < count[k]) {
                            sum[0][k][i] = fmaf(g[i], xhat, sum[0][k][i]);
                            sum[1][k][i] += g[i];
                        }
                        H[k][i] = fmaf(inv_h, g[i] * fmaf(w[i], a[i], w[i]) - mu[1] - xhat * along_h, H[k][i]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = p.alpha * H[k][i];
                store8(static_cast<S*>(p.dx) + row * p.ld_dx + c, count[k], vec, v);
                if (p.y) {
                    pack_widen(ys[k], v);
                    load_param(p.gate, batch, c, count[k], vec, 1.f, w);
                    if (post) load_param(p.post_weight, 0, c, count[k], vec, 1.f, a);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float yhat = (v[i] - mean_y) * inv_y;
                        if (i < count[k]) sum[2][k][i] = fmaf(H[k][i], yhat, sum[2][k][i]);
                        H[k][i] *= w[i];                        // from here on the gradient at the branch
                        if (post) {
                            H[k][i] *= a[i];
                            if (i < count[k]) {
                                back[0] += H[k][i];
                                back[1] = fmaf(H[k][i], yhat, back[1]);
                            }
                        }
                    }
                    if (!post) store8(static_cast<Y*>(p.dy) + row * p.ld_dy + c, count[k], vec, H[k]);
                }
            }
        if (post) {
            row_sum<2>(back, red, phase);
            const float mean_a = layer_y ? back[0] * inv_d : 0.f, along_y = back[1] * inv_d;
#pragma unroll
            for (int k = 0; k < VPT; ++k)
                if (count[k] > 0) {
                    const int c = ((int)threadIdx.x + k * (int)blockDim.x) * 8;
                    float v[8];
                    pack_widen(ys[k], v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = (H[k][i] - mean_a - (v[i] - mean_y) * inv_y * along_y) * inv_y;
                    store8(static_cast<Y*>(p.dy) + row * p.ld_dy + c, count[k], vec, v);
                }
        }
    }
    if (p.partial) flush_sums<VPT>(p, worker + batch, sum, count);
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

// blockDim = (32 columns, 32 slot lanes); lane 0 adds the lanes' sums in order and writes.
__global__ void __launch_bounds__(1024) norm_vector_gradients(const NormVecGrads p) {
    __shared__ float part[3][32][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int c = (int)blockIdx.x * 32 + (int)threadIdx.x;
    const bool live = c < p.d;
    float total[5] = {0.f, 0.f, 0.f, 0.f, 0.f};              // dgate, dscale, dshift over all batches; dweight, dpost_weight
    for (int64_t b = 0; b < p.batches; ++b) {
        const int64_t r0 = b * p.rows_per_batch, r1 = (r0 + p.rows_per_batch < p.rows ? r0 + p.rows_per_batch : p.rows) - 1;
        const int64_t w0 = r0 / p.rows_per_worker, w1 = r1 / p.rows_per_worker;
        float s[3] = {0.f, 0.f, 0.f};
        if (live)
            for (int64_t w = w0 + threadIdx.y; w <= w1; w += 32) {
                const float* at = p.partial + (w + b) * 3 * p.d + c;
                s[0] += at[0];
                s[1] += at[p.d];
                s[2] += at[2 * (int64_t)p.d];
            }
        __syncthreads();                                      // the previous batch's sums have been read
#pragma unroll
        for (int q = 0; q < 3; ++q) part[q][threadIdx.y][threadIdx.x] = s[q];
        __syncthreads();
        if (threadIdx.y == 0 && live) {
            float t[3] = {0.f, 0.f, 0.f};
#pragma unroll 4
            for (int l = 0; l < 32; ++l)
#pragma unroll
                for (int q = 0; q < 3; ++q) t[q] += part[q][l][threadIdx.x];
            auto entry = [&](const NormVec& v, float none) {
                if (!v.ptr) return none;
                const int64_t at = b * v.stride + c;
                if (v.type == kTypeF32) return static_cast<const float*>(v.ptr)[at];
                if (v.type == kTypeF16) return __half2float(static_cast<const __half*>(v.ptr)[at]);
                return __bfloat162float(static_cast<const __nv_bfloat16*>(v.ptr)[at]);
            };
            const float dgate = entry(p.post_weight, 1.f) * t[2], dscale = entry(p.weight, 1.f) * t[0], dshift = t[1];
            if (p.dgate && p.dgate_stride) p.dgate[b * p.dgate_stride + c] = dgate;
            if (p.dscale && p.dscale_stride) p.dscale[b * p.dscale_stride + c] = dscale;
            if (p.dshift && p.dshift_stride) p.dshift[b * p.dshift_stride + c] = dshift;
            total[0] += dgate;
            total[1] += dscale;
            total[2] += dshift;
            total[3] = fmaf(1.f + entry(p.scale, 0.f), t[0], total[3]);
            total[4] = fmaf(entry(p.gate, 1.f), t[2], total[4]);
        }
    }
    if (threadIdx.y == 0 && live) {
        if (p.dgate && !p.dgate_stride) p.dgate[c] = total[0];
        if (p.dscale && !p.dscale_stride) p.dscale[c] = total[1];
        if (p.dshift && !p.dshift_stride) p.dshift[c] = total[2];
        if (p.dweight) p.dweight[c] = total[3];
        if (p.dpost_weight) p.dpost_weight[c] = total[4];
    }
}

}  // namespace kq
