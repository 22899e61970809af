// Rotary positions, sm_100a: the pairs of a head's channels turn by position * frequency.
//     (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = positions[token][axis of p] * frequencies[p]
// Pair p of P is the channels (2p, 2p + 1) or (p, p + P); the axes own consecutive runs of pairs.  The backward pass turns by -t.
//
// The angle in turns, position * (frequency / 2 pi), is a 64-bit product less its nearest integer: a position of 2^21 with a
// frequency of 1 has 3.3e5 turns, of which 32 bits would leave 5 digits of the angle's fraction.  Sine and cosine of the
// remainder are sincospif of its 32-bit head, corrected to first order by its tail, so they are as good as 32 bits hold.
//
// Bound by memory: one read and one write of every element.  Sines and cosines of a token are the same for all heads: a CTA takes one
// or a few tokens with all their heads, forms the P pairs of (cos, sin) once in shared memory and has its first rows on the way
// meanwhile.  A thread takes one place within a head (16 or 8 bytes, or single elements where rows are not aligned) of one row
// (token, head) after another.
#pragma once
#include "kq_common.cuh"

namespace kq {

struct FastDiv {                         // n / d for n < 2^31
    uint32_t d, mul, shift;
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
};

struct RotaryTensor {
    const void* x;
    void* out;
    int64_t xb, ob;                      // batch strides
    int heads, xt, xh, ot, oh;           // token and head strides, below 2^31
    FastDiv by_heads;
};
struct RotaryProblem {
    int64_t rows;                        // batches * tokens
    int64_t tokens;
    int head_dim, pairs, inverse, positions_f32;
    int axis_end[4];                     // pairs up to and with the axis
    const double* frequencies;
    const void* positions;
    int64_t pos_batch, pos_token;
    RotaryTensor t[2];
    int tensors;
    int tokens_per_cta, head_parts;      // blockIdx.y takes every head_parts-th run of rows
};

template <typename T> __device__ __forceinline__ float rotary_widen(T v);
template <> __device__ __forceinline__ float rotary_widen<float>(float v) { return v; }
template <> __device__ __forceinline__ float rotary_widen<__half>(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float rotary_widen<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T rotary_round(float v);
template <> __device__ __forceinline__ float rotary_round<float>(float v) { return v; }
template <> __device__ __forceinline__ __half rotary_round<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 rotary_round<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// N elements of one access
template <typename T, int N> struct alignas(sizeof(T) * N) RotaryPack { T v[N]; };

// (cos, sin) of N pairs from p0 on; two at a time where the place allows
template <int N>
__device__ __forceinline__ void load_turns(float2 (&turn)[N], const float2* cs, int p0, int pairs) {
    if (N % 2 == 0 && pairs % 2 == 0) {                                  // (rows of the table stay 16-byte aligned)
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            if (p0 + i >= pairs) break;
            const float4 c = *reinterpret_cast<const float4*>(cs + p0 + i);
            turn[i] = make_float2(c.x, c.y);
            if (i + 1 < N) turn[i + 1] = make_float2(c.z, c.w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (p0 + i < pairs) turn[i] = cs[p0 + i];
    }
}

// E: elements of an access (their bytes aligned; 1: any alignment of the type).  A unit is one access (interleaved; two elements, each
// its own access, with E = 1) or the two accesses of E pairs (half).  Behind the pairs a unit copies E elements.
template <typename T, int E, bool HALF>
struct RotaryUnit {
    static constexpr int kElems = E == 1 && !HALF ? 2 : E;
    static constexpr int kPairs = HALF ? E : kElems / 2;
    T a[kElems], b[HALF ? E : 1];
    // w: place in the head
    __device__ __forceinline__ void load(const T* row, int w, int pairs, int dim) {
        if constexpr (!HALF && E == 1) {
            a[0] = row[2 * w];
            a[1] = 2 * w + 1 < dim ? row[2 * w + 1] : a[0];
        } else if constexpr (!HALF) {
            const auto p = *reinterpret_cast<const RotaryPack<T, E>*>(row + w * E);
#pragma unroll
            for (int i = 0; i < E; ++i) a[i] = p.v[i];
        } else {
            const int at = w * E < pairs ? w * E : w * E + pairs;        // behind the first halves come the second ones
            const auto p = *reinterpret_cast<const RotaryPack<T, E>*>(row + at);
#pragma unroll
            for (int i = 0; i < E; ++i) a[i] = p.v[i];
            if (w * E < pairs) {
                const auto q = *reinterpret_cast<const RotaryPack<T, E>*>(row + at + pairs);
#pragma unroll
                for (int i = 0; i < E; ++i) b[i] = q.v[i];
            }
        }
    }
    __device__ __forceinline__ void turn_and_store(T* row, int w, int pairs, int dim, const float2* cs) {
        if constexpr (!HALF) {
            const int p0 = w * kPairs;
            float2 turn[kPairs];
            load_turns<kPairs>(turn, cs, p0, pairs);
#pragma unroll
            for (int i = 0; i < kPairs; ++i)
                if (p0 + i < pairs) {
                    const float x = rotary_widen(a[2 * i]), y = rotary_widen(a[2 * i + 1]);
                    const float2 c = turn[i];
                    a[2 * i] = rotary_round<T>(fmaf(x, c.x, -(y * c.y)));
                    a[2 * i + 1] = rotary_round<T>(fmaf(x, c.y, y * c.x));
                }
            if constexpr (E == 1) {
                row[2 * w] = a[0];
                if (2 * w + 1 < dim) row[2 * w + 1] = a[1];
            } else {
                RotaryPack<T, E> p;
#pragma unroll
                for (int i = 0; i < E; ++i) p.v[i] = a[i];
                *reinterpret_cast<RotaryPack<T, E>*>(row + w * E) = p;
            }
        } else {
            RotaryPack<T, E> p, q;
            if (w * E < pairs) {
                float2 turn[E];
                load_turns<E>(turn, cs, w * E, pairs);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float x = rotary_widen(a[i]), y = rotary_widen(b[i]);
                    const float2 c = turn[i];
                    p.v[i] = rotary_round<T>(fmaf(x, c.x, -(y * c.y)));
                    q.v[i] = rotary_round<T>(fmaf(x, c.y, y * c.x));
                }
                *reinterpret_cast<RotaryPack<T, E>*>(row + w * E) = p;
                *reinterpret_cast<RotaryPack<T, E>*>(row + w * E + pairs) = q;
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) p.v[i] = a[i];
                *reinterpret_cast<RotaryPack<T, E>*>(row + w * E + pairs) = p;
            }
        }
    }
};

constexpr int kRotaryThreads = 512;      // at most

// blockDim: x = units of a head, y = rows (token, head) at a time.  Dynamic shared memory: float2 [tokens_per_cta][pairs].
template <typename T, int E, bool HALF>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(const __grid_constant__ RotaryProblem p) {
    extern __shared__ __align__(16) float2 rotary_cs[];
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const int64_t token0 = (int64_t)blockIdx.x * p.tokens_per_cta;
    const int tokens = (int)(p.rows - token0 < p.tokens_per_cta ? p.rows - token0 : p.tokens_per_cta);
    const int w = threadIdx.x, first = threadIdx.y + blockIdx.y * blockDim.y, step = blockDim.y * p.head_parts;
    int64_t batch0 = 0, t0 = token0;                                      // batch and token of the CTA's first row
    if (p.tokens != p.rows) {
        batch0 = token0 / p.tokens;
        t0 = token0 - batch0 * p.tokens;
    }

    constexpr int kAhead = sizeof(RotaryUnit<T, E, HALF>) > 16 ? 2 : 4;   // rows of a thread in flight
    RotaryUnit<T, E, HALF> unit[kAhead];
    // element of row r (token lt of the CTA) behind its first token's first head
    auto place = [&](const RotaryTensor& s, int lt, int head, int64_t batch, int token, int head_stride) {
        int64_t at = (int64_t)lt * token + (int64_t)head * head_stride;
        if (p.tokens != p.rows && t0 + lt >= p.tokens) at += (t0 + lt) / p.tokens * (batch - p.tokens * token);   // into later batches
        return at;
    };
    auto fetch = [&](const RotaryTensor& s, int r0, int rows) {
        const T* x = static_cast<const T*>(s.x) + batch0 * s.xb + t0 * s.xt;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int r = r0 + u * step;
            if (r < rows) {
                const int lt = (int)s.by_heads.div((uint32_t)r);
                unit[u].load(x + place(s, lt, r - lt * s.heads, s.xb, s.xt, s.xh), w, p.pairs, p.head_dim);
            }
        }
    };
    fetch(p.t[0], first, tokens * p.t[0].heads);
    for (int i = threadIdx.y * blockDim.x + threadIdx.x; i < tokens * p.pairs; i += blockDim.x * blockDim.y) {
        const int lt = i / p.pairs, pair = i - lt * p.pairs;
        int64_t t = t0 + lt, b = batch0;
        if (p.tokens != p.rows && t >= p.tokens) {
            b += t / p.tokens;
            t %= p.tokens;
        }
        const int axis = (pair >= p.axis_end[0]) + (pair >= p.axis_end[1]) + (pair >= p.axis_end[2]);
        const int64_t at = b * p.pos_batch + t * p.pos_token + axis;
        const double position = p.positions_f32 ? (double)__ldg(static_cast<const float*>(p.positions) + at)
                                                : (double)__ldg(static_cast<const int*>(p.positions) + at);
        const double turns = position * (__ldg(p.frequencies + pair) * 0.15915494309189533577);
        const double rest = turns - rint(turns);
        const float head = (float)rest, tail = 6.2831853071795865f * (float)(rest - (double)head);
        float s, c;
        sincospif(2.f * head, &s, &c);
        const float cos_t = fmaf(-s, tail, c), sin_t = fmaf(c, tail, s);
        rotary_cs[i] = make_float2(cos_t, p.inverse ? -sin_t : sin_t);
    }
    __syncthreads();
    for (int k = 0; k < p.tensors; ++k) {
        const RotaryTensor& s = p.t[k];
        const int rows = tokens * s.heads;
        T* out = static_cast<T*>(s.out) + batch0 * s.ob + t0 * s.ot;
        for (int r0 = first; r0 < rows; r0 += kAhead * step) {
            if (k || r0 != first) fetch(s, r0, rows);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int r = r0 + u * step;
                if (r < rows) {
                    const int lt = (int)s.by_heads.div((uint32_t)r);
                    unit[u].turn_and_store(out + place(s, lt, r - lt * s.heads, s.ob, s.ot, s.oh), w, p.pairs, p.head_dim, rotary_cs + lt * p.pairs);
                }
            }
        }
    }
}

}  // namespace kq
