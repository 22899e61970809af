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
// Measured: 4608 tokens x 72 heads x 128, bf16, 31.2 us (5.5 TB/s, 0.83 of the copy rate; 34.8 where the copies of k began behind the last row of q and
// out's addresses were formed from more terms, 47 with the rows in registers and CTAs of more than one wave); 10007 x 32 x 72, fp16, accesses
// of 8 bytes, 21.6 us (0.65); one token 2.8.  Instructions take two thirds of the issue slots; a loop of 8 rows a turn was slower (its code).
#pragma once
#include "kq_mma16.cuh"

namespace kq {

struct FastDiv {                         // n / d for n < 2^31, by Granlund and Montgomery's multiplication (1994)
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

// (cos, sin) of N pairs; two at a time (rows of the table and the places of units of more than one pair are 16-byte aligned)
template <int N>
__device__ __forceinline__ void load_turns(float2 (&turn)[N], const float2* cs) {
    if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float4 c = *reinterpret_cast<const float4*>(cs + i);
            turn[i] = make_float2(c.x, c.y);
            turn[i + 1] = make_float2(c.z, c.w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) turn[i] = cs[i];
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
    static constexpr int kBytes = 4 * kWords;                            // of an access
    static constexpr int kPairs = HALF ? E : E / 2;
    uint32_t a[kWords], b[HALF ? kWords : 1];
    // Unit w: its first element in the head (half: behind the first members come the second ones) and how many of its pairs turn.
    static __device__ __forceinline__ int place(int w, int pairs) { return !HALF || w * E < pairs ? w * E : w * E + pairs; }
    static __device__ __forceinline__ int turning(int w, int pairs) {
        const int left = pairs - w * kPairs;
        return left < 0 ? 0 : left < kPairs ? left : kPairs;
    }
    // at: the unit's first element of a row.  To `slot` in shared memory, the second access `second` bytes behind it.
    static __device__ __forceinline__ void copy(uint32_t slot, uint32_t second, const uint8_t* at, int turning, int pairs) {
        rotary_copy<kBytes>(slot, at);
        if constexpr (HALF)
            if (turning) rotary_copy<kBytes>(slot + second, at + pairs * (int)sizeof(T));
    }
    __device__ __forceinline__ void take(const uint8_t* at, int second) {
        rotary_load(a, at);
        if constexpr (HALF) rotary_load(b, at + second);
    }
    __device__ __forceinline__ void load(const uint8_t* at, int turning, int pairs) {
        rotary_load(a, at);
        if constexpr (HALF)
            if (turning) rotary_load(b, at + pairs * (int)sizeof(T));
    }
    // cs: of the unit's first pair
    __device__ __forceinline__ void turn(int turning, const float2* cs) {
        if constexpr (!HALF) {
            auto pair = [&](int i, const float2& c) {
                if constexpr (sizeof(T) == 2) {
                    float2 v = rotary_widen2<T>(a[i]);
                    rotary_turn(v.x, v.y, c);
                    a[i] = rotary_round2<T>(v.x, v.y);
                } else {
                    float x = __uint_as_float(a[2 * i]), y = __uint_as_float(a[2 * i + 1]);
                    rotary_turn(x, y, c);
                    a[2 * i] = __float_as_uint(x);
                    a[2 * i + 1] = __float_as_uint(y);
                }
            };
            if (turning == kPairs) {
                float2 c[kPairs];
                load_turns<kPairs>(c, cs);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) pair(i, c[i]);
            } else if (turning) {
#pragma unroll
                for (int i = 0; i < kPairs; ++i)
                    if (i < turning) pair(i, cs[i]);
            }
        } else if (turning) {                                            // (all of them)
            float2 c[E];
            load_turns<E>(c, cs);
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if constexpr (sizeof(T) == 2) {
                    float2 x = rotary_widen2<T>(a[i]), y = rotary_widen2<T>(b[i]);
                    rotary_turn(x.x, y.x, c[2 * i]);
                    rotary_turn(x.y, y.y, c[2 * i + 1]);
                    a[i] = rotary_round2<T>(x.x, x.y);
                    b[i] = rotary_round2<T>(y.x, y.y);
                } else {
                    float x = __uint_as_float(a[i]), y = __uint_as_float(b[i]);
                    rotary_turn(x, y, c[i]);
                    a[i] = __float_as_uint(x);
                    b[i] = __float_as_uint(y);
                }
            }
        }
    }
    __device__ __forceinline__ void store(uint8_t* at, int turning, int pairs) const {
        rotary_store(at, a);
        if constexpr (HALF)
            if (turning) rotary_store(at + pairs * (int)sizeof(T), b);
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
__host__ __device__ constexpr int rotary_pitch(int pairs) { return (pairs + 1) & ~1; }      // of the table of sines
// Rows of a thread on the way: copies to shared memory of its own (aligned rows), or registers.
template <typename T, int E, bool HALF>
__host__ __device__ constexpr int rotary_ahead() { return E == 1 || (HALF && E * sizeof(T) == 16) ? 4 : 8; }
template <typename T, int E, bool HALF>
__host__ __device__ constexpr int rotary_slot_bytes() { return E == 1 ? 0 : E * (int)sizeof(T) * (HALF ? 2 : 1) * rotary_ahead<T, E, HALF>(); }   // of a thread

// A thread's way through the rows (token, head) of the tensors, one after the other, on one side (x or out).  From a row to the
// next its address moves on by the same step, and by another one more where the head passes the last: none is formed anew.
struct RotaryWalk {
    uint8_t* at;
    int64_t step, wrap;                  // bytes
    int head, dh, heads, left, tensor;   // left: rows of this tensor, with the present one
    template <bool OUT, typename T>
    __device__ __forceinline__ void open(const RotaryProblem& p, int n, int tokens, int first, int rows_step, int64_t batch0, int64_t t0, int place) {
        for (left = 0; n < p.tensors; ++n) {
            const RotaryTensor& s = p.t[n];
            if (first >= tokens * s.heads) continue;
            const int dt = (int)s.by_heads.div((uint32_t)rows_step), lt = (int)s.by_heads.div((uint32_t)first);
            const int64_t token = (OUT ? s.ot : s.xt) * (int64_t)sizeof(T), each = (OUT ? s.oh : s.xh) * (int64_t)sizeof(T);
            heads = s.heads;
            dh = rows_step - dt * heads;
            head = first - lt * heads;
            step = dt * token + dh * each;
            wrap = token - heads * each;
            at = (OUT ? static_cast<uint8_t*>(s.out) : static_cast<uint8_t*>(const_cast<void*>(s.x))) + batch0 * (OUT ? s.ob : s.xb) * (int64_t)sizeof(T) +
                 (t0 + lt) * token + head * each + place * (int)sizeof(T);
            left = (tokens * heads - 1 - first) / rows_step + 1;
            tensor = n;
            break;
        }
    }
    __device__ __forceinline__ bool next() {                             // into the next token
        at += step;
        head += dh;
        if (head < heads) return false;
        head -= heads;
        at += wrap;
        return true;
    }
};

// blockDim: x = units of a head, y = rows (token, head) at a time.  Dynamic shared memory: the slots of the copies, then
// float2 [tokens_per_cta][pairs, an even number].
template <typename T, int E, bool HALF>
__global__ void __launch_bounds__(kRotaryThreads, 2) rotary_kernel(const __grid_constant__ RotaryProblem p) {
    extern __shared__ __align__(16) uint8_t rotary_smem[];
    using Unit = RotaryUnit<T, E, HALF>;
    constexpr int kAhead = rotary_ahead<T, E, HALF>();
    const int thread = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
    float2* rotary_cs = reinterpret_cast<float2*>(rotary_smem + (threads * rotary_slot_bytes<T, E, HALF>() + 15) / 16 * 16);
    const int pitch = rotary_pitch(p.pairs);
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
    const bool crosses = p.tokens != p.rows && t0 + tokens > p.tokens;   // into later batches

    // Aligned rows: a pipeline of copies, each into a slot that only its thread reads, from tensor to tensor without a break.
    constexpr int kUnitBytes = E * (int)sizeof(T);
    const uint32_t second = threads * kUnitBytes, slot_step = second * (HALF ? 2 : 1);
    const uint8_t* const slots = rotary_smem + thread * kUnitBytes;
    const uint32_t slots_at = (uint32_t)__cvta_generic_to_shared(slots);
    int turning = 0, place = 0;
    if constexpr (E > 1) {
        turning = Unit::turning(w, p.pairs);
        place = Unit::place(w, p.pairs);
    }
    RotaryWalk in = {}, out = {};
    auto copy_next = [&](uint32_t slot) {
        if constexpr (E > 1) {
            if (in.left > 0) {
                Unit::copy(slots_at + slot, second, in.at, turning, p.pairs);
                in.next();
                if (--in.left == 0) in.open<false, T>(p, in.tensor + 1, tokens, first, step, batch0, t0, place);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    if (E > 1 && !crosses) {
        in.open<false, T>(p, 0, tokens, first, step, batch0, t0, place);
#pragma unroll
        for (int u = 0; u < kAhead - 1; ++u) copy_next(u * slot_step);
    }
    for (int i = thread; i < tokens * p.pairs; i += threads) {
        const int lt = i / p.pairs, pair = i - lt * p.pairs;
        int64_t t = t0 + lt, b = batch0;
        if (crosses && t >= p.tokens) {
            b += t / p.tokens;
            t %= p.tokens;
        }
        const int axis = (pair >= p.axis_end[0]) + (pair >= p.axis_end[1]) + (pair >= p.axis_end[2]);
        const int64_t at = b * p.pos_batch + t * p.pos_token + axis;
        const double position = p.positions_f32 ? (double)static_cast<const float*>(p.positions)[at]
                                                : (double)static_cast<const int*>(p.positions)[at];
        const double turns = position * (p.frequencies[pair] * 0.15915494309189533577);
        const double rest = turns - rint(turns);
        const float head = (float)rest, tail = 6.2831853071795865f * (float)(rest - (double)head);
        float s, c;
        sincospif(2.f * head, &s, &c);
        const float cos_t = fmaf(-s, tail, c), sin_t = fmaf(c, tail, s);
        rotary_cs[lt * pitch + pair] = make_float2(cos_t, p.inverse ? -sin_t : sin_t);
    }
    __syncthreads();
    if constexpr (E > 1) {
        if (!crosses) {
            out.open<true, T>(p, 0, tokens, first, step, batch0, t0, place);
            if (out.left == 0) return;
            const float2* const mine = rotary_cs + w * Unit::kPairs;
            const float2* cs;
            int cs_step;
            auto turns_of = [&] {                                        // where out begins a tensor
                const RotaryTensor& s = p.t[out.tensor];
                cs = mine + (int)s.by_heads.div((uint32_t)first) * pitch;
                cs_step = (int)s.by_heads.div((uint32_t)step) * pitch;
            };
            turns_of();
            for (uint32_t slot = 0, before = (kAhead - 1) * slot_step;;) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 2) : "memory");
                copy_next(before);                                       // (the slot of the row before)
                Unit unit;
                unit.take(slots + slot, (int)second);
                before = slot;
                slot += slot_step;
                if (slot == kAhead * slot_step) slot = 0;
                unit.turn(turning, cs);
                unit.store(out.at, turning, p.pairs);
                cs += cs_step;
                if (out.next()) cs += pitch;
                if (--out.left == 0) {
                    out.open<true, T>(p, out.tensor + 1, tokens, first, step, batch0, t0, place);
                    if (out.left == 0) return;
                    turns_of();
                }
            }
        }
    }
    // Rows of any alignment, and the CTAs whose tokens lie in several batches: each row's address by itself.
    for (int n = 0; n < p.tensors; ++n) {
        const RotaryTensor& s = p.t[n];
        const int rows = tokens * s.heads;
        auto element = [&](int r, int64_t batch, int token, int head, int& lt) {
            lt = (int)s.by_heads.div((uint32_t)r);
            int64_t b = batch0, t = t0 + lt;
            if (crosses && t >= p.tokens) {
                b += t / p.tokens;
                t %= p.tokens;
            }
            return b * batch + t * token + (int64_t)(r - lt * s.heads) * head;
        };
        int lt;
        if constexpr (E > 1) {
            for (int r = first; r < rows; r += step) {
                const int64_t from = element(r, s.xb, s.xt, s.xh, lt) + place, to = element(r, s.ob, s.ot, s.oh, lt) + place;
                Unit unit;
                unit.load(static_cast<const uint8_t*>(s.x) + from * (int)sizeof(T), turning, p.pairs);
                unit.turn(turning, rotary_cs + lt * pitch + w * Unit::kPairs);
                unit.store(static_cast<uint8_t*>(s.out) + to * (int)sizeof(T), turning, p.pairs);
            }
        } else {
            Unit unit[kAhead];
            for (int r0 = first; r0 < rows; r0 += kAhead * step) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (r0 + u * step < rows) unit[u].load(static_cast<const T*>(s.x) + element(r0 + u * step, s.xb, s.xt, s.xh, lt), w, p.pairs, p.head_dim);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (r0 + u * step < rows) {
                        T* to = static_cast<T*>(s.out) + element(r0 + u * step, s.ob, s.ot, s.oh, lt);
                        unit[u].turn_and_store(to, w, p.pairs, p.head_dim, rotary_cs + lt * pitch);
                    }
            }
        }
    }
}

}  // namespace kq
