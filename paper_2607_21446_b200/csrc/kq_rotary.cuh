// Rotary positions, sm_100a: the pairs of a head's channels turn by position * frequency.
//     (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = positions[token][axis of p] * frequencies[p]
// Pair p of P is the channels (2p, 2p + 1) or (p, p + P); the axes own consecutive runs of pairs.  The backward pass turns by -t.
//
// The angle in turns, position * (frequency / 2 pi), is a 64-bit product less its nearest integer: a position of 2^21 with a
// frequency of 1 has 3.3e5 turns, of which 32 bits would leave 5 digits of the angle's fraction.  Sine and cosine of the
// remainder are sincospif of its 32-bit head, corrected to first order by its tail, so they are as good as 32 bits hold.
//
// Bound by memory: one read and one write of every element.  Sines and cosines of a token are the same for all heads: a CTA takes
// a few tokens with all their heads, forms the P pairs of (cos, sin) once in shared memory and has its first rows on the way
// meanwhile.  A thread takes one place within a head (16 or 8 bytes, or single elements where rows are not aligned) of one row
// (token, head) after another and has eight rows on the way, by asynchronous copies to shared memory that only it reads.
// Measured: 4608 tokens x 72 heads x 128, bf16, 34.8 us (4.9 TB/s, 0.75 of the copy rate; 47 with the rows
// in registers, an address computed for each and CTAs of more than one wave); 10007 x 32 x 72, fp16, 23.2 us (0.61); one token 2.8.  The instructions take 0.7 of the issue slots then.
#pragma once
#include "kq_mma16.cuh"

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

// two 16-bit values of a word, and back
template <typename T> __device__ __forceinline__ float2 rotary_widen2(uint32_t w);
template <> __device__ __forceinline__ float2 rotary_widen2<__nv_bfloat16>(uint32_t w) { return make_float2(bf16lo_to_f32(w), bf16hi_to_f32(w)); }
template <> __device__ __forceinline__ float2 rotary_widen2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
template <typename T> __device__ __forceinline__ uint32_t rotary_round2(float x, float y);
template <> __device__ __forceinline__ uint32_t rotary_round2<__nv_bfloat16>(float x, float y) { return pack_bf16(x, y); }
template <> __device__ __forceinline__ uint32_t rotary_round2<__half>(float x, float y) { return pack_f16(x, y); }
// (x, y) turned by (cos, sin)
__device__ __forceinline__ void rotary_turn(float& x, float& y, const float2& c) {
    const float u = fmaf(x, c.x, -(y * c.y));
    y = fmaf(x, c.y, y * c.x);
    x = u;
}
template <int WORDS>
__device__ __forceinline__ void rotary_load(uint32_t (&w)[WORDS], const void* at) {
    if constexpr (WORDS == 4) {
        const uint4 v = *static_cast<const uint4*>(at);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
        const uint2 v = *static_cast<const uint2*>(at);
        w[0] = v.x; w[1] = v.y;
    }
}
template <int BYTES>
__device__ __forceinline__ void rotary_copy(uint32_t to, const void* from) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
}
template <int WORDS>
__device__ __forceinline__ void rotary_store(void* at, const uint32_t (&w)[WORDS]) {
    if constexpr (WORDS == 4) *static_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
    else *static_cast<uint2*>(at) = make_uint2(w[0], w[1]);
}

// E: elements of an access of 16 or 8 bytes (1: any alignment of the type).  A unit is one access (interleaved; two elements, each its own
// access, with E = 1) or the two accesses of E pairs (half).  Behind the pairs a unit copies E elements.
template <typename T, int E, bool HALF>
struct RotaryUnit {
    static constexpr int kWords = E * (int)sizeof(T) / 4;
    uint32_t a[kWords], b[HALF ? kWords : 1];
    static constexpr int kBytes = 4 * kWords;                            // of an access
    // w: place in the head.  Copies the unit to `slot` in shared memory, its second access `second` bytes behind it.
    static __device__ __forceinline__ void copy(uint32_t slot, uint32_t second, const T* row, int w, int pairs) {
        const int at = !HALF || w * E < pairs ? w * E : w * E + pairs;   // (half: behind the first members come the second ones)
        rotary_copy<kBytes>(slot, row + at);
        if constexpr (HALF)
            if (w * E < pairs) rotary_copy<kBytes>(slot + second, row + at + pairs);
    }
    __device__ __forceinline__ void take(const uint8_t* slot, int second) {
        rotary_load(a, slot);
        if constexpr (HALF) rotary_load(b, slot + second);
    }
    __device__ __forceinline__ void turn_and_store(T* row, int w, int pairs, int, const float2* cs) {
        if constexpr (!HALF) {
            constexpr int kPairs = E / 2;
            const int p0 = w * kPairs;
            float2 turn[kPairs];
            load_turns<kPairs>(turn, cs, p0, pairs);
            auto pair = [&](int i) {
                if constexpr (sizeof(T) == 2) {
                    float2 v = rotary_widen2<T>(a[i]);
                    rotary_turn(v.x, v.y, turn[i]);
                    a[i] = rotary_round2<T>(v.x, v.y);
                } else {
                    float x = __uint_as_float(a[2 * i]), y = __uint_as_float(a[2 * i + 1]);
                    rotary_turn(x, y, turn[i]);
                    a[2 * i] = __float_as_uint(x);
                    a[2 * i + 1] = __float_as_uint(y);
                }
            };
            if (p0 + kPairs <= pairs) {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) pair(i);
            } else {
#pragma unroll
                for (int i = 0; i < kPairs; ++i)
                    if (p0 + i < pairs) pair(i);
            }
            rotary_store(row + w * E, a);
        } else if (w * E < pairs) {
            float2 turn[E];
            load_turns<E>(turn, cs, w * E, pairs);
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if constexpr (sizeof(T) == 2) {
                    float2 x = rotary_widen2<T>(a[i]), y = rotary_widen2<T>(b[i]);
                    rotary_turn(x.x, y.x, turn[2 * i]);
                    rotary_turn(x.y, y.y, turn[2 * i + 1]);
                    a[i] = rotary_round2<T>(x.x, x.y);
                    b[i] = rotary_round2<T>(y.x, y.y);
                } else {
                    float x = __uint_as_float(a[i]), y = __uint_as_float(b[i]);
                    rotary_turn(x, y, turn[i]);
                    a[i] = __float_as_uint(x);
                    b[i] = __float_as_uint(y);
                }
            }
            rotary_store(row + w * E, a);
            rotary_store(row + w * E + pairs, b);
        } else {
            rotary_store(row + w * E + pairs, a);
        }
    }
};
template <typename T, bool HALF>
struct RotaryUnit<T, 1, HALF> {
    T a, b;
    __device__ __forceinline__ void load(const T* row, int w, int pairs, int dim) {
        if constexpr (HALF) {
            a = row[w < pairs ? w : w + pairs];
            if (w < pairs) b = row[w + pairs];
        } else {
            a = row[2 * w];
            if (2 * w + 1 < dim) b = row[2 * w + 1];
        }
    }
    __device__ __forceinline__ void turn_and_store(T* row, int w, int pairs, int dim, const float2* cs) {
        if (w < pairs) {
            float x = rotary_widen(a), y = rotary_widen(b);
            rotary_turn(x, y, cs[w]);
            a = rotary_round<T>(x);
            b = rotary_round<T>(y);
        }
        if constexpr (HALF) {
            row[w < pairs ? w : w + pairs] = a;
            if (w < pairs) row[w + pairs] = b;
        } else {
            row[2 * w] = a;
            if (2 * w + 1 < dim) row[2 * w + 1] = b;
        }
    }
};

constexpr int kRotaryThreads = 512;      // at most
// Rows of a thread on the way: copies to shared memory of its own (aligned rows), or registers.
template <typename T, int E, bool HALF>
__host__ __device__ constexpr int rotary_ahead() { return E == 1 || (HALF && E * sizeof(T) == 16) ? 4 : 8; }
template <typename T, int E, bool HALF>
__host__ __device__ constexpr int rotary_slot_bytes() { return E == 1 ? 0 : E * (int)sizeof(T) * (HALF ? 2 : 1) * rotary_ahead<T, E, HALF>(); }   // of a thread

// blockDim: x = units of a head, y = rows (token, head) at a time.  Dynamic shared memory: the slots of the copies, then
// float2 [tokens_per_cta][pairs].
template <typename T, int E, bool HALF>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(const __grid_constant__ RotaryProblem p) {
    extern __shared__ __align__(16) uint8_t rotary_smem[];
    const int thread = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
    float2* rotary_cs = reinterpret_cast<float2*>(rotary_smem + (threads * rotary_slot_bytes<T, E, HALF>() + 15) / 16 * 16);
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

    constexpr int kAhead = rotary_ahead<T, E, HALF>();
    const bool crosses = p.tokens != p.rows && t0 + tokens > p.tokens;   // into later batches
    // element of a token (counted within the CTA) and head
    auto place = [&](int lt, int head, int64_t batch, int token, int head_stride) {
        int64_t at = batch0 * batch + t0 * token + ((int64_t)lt * token + (int64_t)head * head_stride);
        if (crosses && t0 + lt >= p.tokens) at += (t0 + lt) / p.tokens * (batch - p.tokens * token);
        return at;
    };
    auto source = [&](const RotaryTensor& s, int r) -> const T* {
        const int lt = (int)s.by_heads.div((uint32_t)r);
        return static_cast<const T*>(s.x) + place(lt, r - lt * s.heads, s.xb, s.xt, s.xh);
    };
    auto finish = [&](const RotaryTensor& s, RotaryUnit<T, E, HALF>& unit, int r) {
        const int lt = (int)s.by_heads.div((uint32_t)r);
        unit.turn_and_store(static_cast<T*>(s.out) + place(lt, r - lt * s.heads, s.ob, s.ot, s.oh), w, p.pairs, p.head_dim, rotary_cs + lt * p.pairs);
    };

    // Aligned rows: a pipeline of copies.  From one row of a thread to its next, x and out move on by the same step, and by another
    // one more where the head passes the last: no row's address is formed anew.
    constexpr int kUnitBytes = E * (int)sizeof(T);
    const uint32_t slot0 = (uint32_t)__cvta_generic_to_shared(rotary_smem) + thread * kUnitBytes, second = threads * kUnitBytes;
    const uint32_t slot_step = second * (HALF ? 2 : 1);
    const T* from = nullptr;                                              // the next row to copy: its address, head and number
    int from_head = 0, from_row = 0, fill = 0;
    auto copy_next = [&](const RotaryTensor& s, int rows, int dt, int dh) {
        if constexpr (E > 1) {
            if (from_row < rows) {
                RotaryUnit<T, E, HALF>::copy(slot0 + fill * slot_step, second, crosses ? source(s, from_row) : from, w, p.pairs);
                from_row += step;
                from_head += dh;
                from += (int64_t)dt * s.xt + (int64_t)dh * s.xh;
                if (from_head >= s.heads) {
                    from_head -= s.heads;
                    from += s.xt - (int64_t)s.heads * s.xh;
                }
            }
            fill = fill + 1 == kAhead ? 0 : fill + 1;
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    auto begin = [&](const RotaryTensor& s, int rows, int dt, int dh) {
        if constexpr (E > 1) {
            from_row = first;
            if (first < rows) {
                from_head = first - (int)s.by_heads.div((uint32_t)first) * s.heads;
                from = source(s, first);
            }
#pragma unroll
            for (int u = 0; u < kAhead - 1; ++u) copy_next(s, rows, dt, dh);
        }
    };
    const int dt0 = (int)p.t[0].by_heads.div((uint32_t)step), dh0 = step - dt0 * p.t[0].heads;
    begin(p.t[0], tokens * p.t[0].heads, dt0, dh0);
    for (int i = thread; i < tokens * p.pairs; i += threads) {
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
    auto run = [&](const RotaryTensor& s, int dt, int dh) {
        const int rows = tokens * s.heads;
        if constexpr (E > 1) {
            if (first >= rows) return;
            RotaryUnit<T, E, HALF> unit;
            const int lt = (int)s.by_heads.div((uint32_t)first);
            int head = first - lt * s.heads;
            const float2* cs = rotary_cs + lt * p.pairs;
            T* to = static_cast<T*>(s.out) + place(lt, head, s.ob, s.ot, s.oh);
            const int64_t ahead = (int64_t)dt * s.ot + (int64_t)dh * s.oh, wrap = s.ot - (int64_t)s.heads * s.oh;
            for (int r = first; r < rows; r += step) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 2) : "memory");
                const int slot = fill + 1 == kAhead ? 0 : fill + 1;      // (the one behind the slot to fill next, which is the row before's)
                copy_next(s, rows, dt, dh);
                unit.take(rotary_smem + thread * kUnitBytes + slot * slot_step, (int)second);
                if (crosses) {
                    finish(s, unit, r);
                    continue;
                }
                unit.turn_and_store(to, w, p.pairs, p.head_dim, cs);
                to += ahead;
                cs += dt * p.pairs;
                head += dh;
                if (head >= s.heads) {
                    head -= s.heads;
                    to += wrap;
                    cs += p.pairs;
                }
            }
        } else {
            RotaryUnit<T, E, HALF> unit[kAhead];
            for (int r0 = first; r0 < rows; r0 += kAhead * step) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (r0 + u * step < rows) unit[u].load(source(s, r0 + u * step), w, p.pairs, p.head_dim);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (r0 + u * step < rows) finish(s, unit[u], r0 + u * step);
            }
        }
    };
    run(p.t[0], dt0, dh0);
    if (p.tensors > 1) {
        const int dt = (int)p.t[1].by_heads.div((uint32_t)step), dh = step - dt * p.t[1].heads;
        begin(p.t[1], tokens * p.t[1].heads, dt, dh);
        run(p.t[1], dt, dh);
    }
}

}  // namespace kq
