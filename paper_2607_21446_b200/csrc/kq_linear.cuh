// The linear layers around the MXFP4 product, sm_100a:
//     acc[m][r] = sum_k a[m][k] 2^(sa[m][k/32]-127) * w[r][k] 2^(sw[r][k/32]-127)          (r: rows of the stored weight)
//     v[m][n]   = act(acc + bias)                     or, gated:  act(acc_g + bias_g) * (acc_u + bias_u)
//     out[m][n] = residual_scale * residual[m][n] + row_scale[m] * gate[m / rows_per_gate][n] * v[m][n]
// and the same with one weight per expert: group e of the rows of A, [offsets[e], offsets[e+1]), meets weight e.
//
// A gated weight stores its rows interleaved, 32 gate rows then their 32 value rows, so that both halves of a product
// lie in the same tile of the accumulator: no second pass and no second operand.
//
// Groups are not padded.  The scale bytes of A live in tiles of 128 rows, so the kernels cut A into aligned row tiles and
// an item of work is (expert, row tile that the group touches, weight tile): a tile that two groups share is multiplied
// by both weights and each epilogue stores only the rows of its own group.  At most one more item per expert and
// weight tile than padding would give, no copy of A, and the group sizes are never needed on the host.
//
// Two kernels.
//   linear_mxfp4_pair    CTA pairs on 256 rows x 192 weight rows (tcgen05.mma.cta_group::2): many rows per weight.
//   linear_mxfp4_narrow  the weight as the 128-row operand and up to 128 rows of A as the narrow one: few rows per
//                        weight, bound by reading the weights; K split over a cluster when there are few weight tiles.
// The tensor-core path is that of kq_gemm_fp4_pair.cuh: codes by TMA, scale tiles copied to tensor memory.
#pragma once
#include "kq_gemm_fp4_pair.cuh"
#include "kq_norm.cuh"

namespace kq {

enum { kActNone = 0, kActRelu = 1, kActSilu = 2, kActGelu = 3, kActGeluTanh = 4 };
constexpr int kMaxExperts = 1024;

struct LinearEpilogue {
    int N, act;                          // columns of out
    NormVec bias;                        // [weight rows], stride: between experts
    NormVec gate;                        // [N], stride: between gate rows
    int rows_per_gate;
    const float* row_scale;              // [M] or null
    const void* residual; int residual_type; int64_t ld_residual; float residual_scale;
    void* out; int out_type; int64_t ld_out;
    int vec, wide;                       // residual and out allow 16-byte accesses; out 32-byte ones
};

struct LinearProblem {
    int M, R;                            // rows of A, rows of one weight
    int k_blocks;                        // pipeline stages of 256 K-elements
    int tiles_m, tiles_n;                // row tiles (dense only), weight tiles
    int sf_row_tiles;                    // 128-row scale tiles of one weight
    int experts;                         // 0: dense
    const int32_t* offsets;              // device [experts + 1]
    LinearEpilogue epi;
};

// ---- activations ---------------------------------------------------------------------------------
// silu and the tanh form of gelu as v / (1 + e^-z): gelu_tanh(v) = v sigmoid(2 sqrt(2/pi) (v + 0.044715 v^3)).
// gelu with erf: v Phi(v), with q = Phi(-|v|) as 2^R(|v|).  R(a) = log2 Phi(-a) is smooth and runs from -1 at 0 to -50.5 at 8: a
// polynomial of degree 12 with R(0) = -1, fitted to Phi itself with the weight that its error has in v (1 - q) and v q.  Nothing
// cancels where q is large: the result is off by at most 1.5 * 2^-23 |v|, its own rounding and the hardware exponential's 1.2 * 2^-23 q
// included (measured over [-8, 8]: 1.0; 0.5 v (1 + erf) in 32 bits: 0.9), and the negative tail keeps a relative accuracy, 2^-19 down
// to -4, 2^-17 to -6, 2^-14 to -8; below that the result, above -5e-15, is taken as 0.  On pairs (f32x2): 8192 x 1152 -> 4608 takes
// 59.6 us, element by element 76.
// (ex2 and rcp directly, denormals as zero: the ordinary functions spend three instructions on results below 2^-126, which
// change nothing next to the 1 of 1 + e^x, and make silu below -87.3 zero instead of 1e-36.)
__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <int ACT>
__device__ __forceinline__ float act_fn(float v) {
    constexpr float kLog2e = 1.4426950408889634f;
    if constexpr (ACT == kActRelu) return v < 0.f ? 0.f : v;         // (NaN stays)
    if constexpr (ACT == kActSilu) return v * rcp_approx(1.f + ex2_approx(-kLog2e * v));
    if constexpr (ACT == kActGeluTanh) return v * rcp_approx(1.f + ex2_approx(-kLog2e * 1.5957691216057308f * fmaf(0.044715f * v * v, v, v)));
    return v;
}
// a pair of values at a time
__device__ __forceinline__ void gelu2(float& v0, float& v1) {
    const f32x2 a = pack2(fabsf(v0), fabsf(v1));
    auto both = [](float c) { return pack2(c, c); };
    f32x2 r = fma2(both(-1.1298189467323638e-10f), a, both(5.902352384623555e-09f));
    r = fma2(r, a, both(-1.371750073531075e-07f));
    r = fma2(r, a, both(1.8654657196748303e-06f));
    r = fma2(r, a, both(-1.6329351637978107e-05f));
    r = fma2(r, a, both(9.349935135105625e-05f));
    r = fma2(r, a, both(-0.0003115577856078744f));
    r = fma2(r, a, both(3.248723805882037e-05f));
    r = fma2(r, a, both(0.0069331880658864975f));
    r = fma2(r, a, both(-0.05244309455156326f));
    r = fma2(r, a, both(-0.4592180848121643f));
    r = fma2(r, a, both(-1.1511045694351196f));
    r = fma2(r, a, both(-1.f));
    const float2 e = unpack2(r);
    const float q0 = fabsf(v0) < 8.f ? ex2_approx(e.x) : 0.f, q1 = fabsf(v1) < 8.f ? ex2_approx(e.y) : 0.f;
    v0 *= v0 >= 0.f ? 1.f - q0 : q0;
    v1 *= v1 >= 0.f ? 1.f - q1 : q1;
}
template <int COUNT>
__device__ __forceinline__ void act_apply(int act, float (&v)[COUNT]) {
    switch (act) {
        case kActRelu:
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = act_fn<kActRelu>(v[i]);
            break;
        case kActSilu:
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = act_fn<kActSilu>(v[i]);
            break;
        case kActGelu:
            static_assert(COUNT % 2 == 0, "pairs");
#pragma unroll
            for (int i = 0; i < COUNT; i += 2) gelu2(v[i], v[i + 1]);
            break;
        case kActGeluTanh:
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = act_fn<kActGeluTanh>(v[i]);
            break;
        default: break;
    }
}

// eight words to one row: one 32-byte store where the address allows it, else two of 16
template <int N>
__device__ __forceinline__ void store_words(void* p, const uint32_t (&w)[N], int wide) {
    if (wide) {
        st_global_32(p, w);
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// ---- scalar access by runtime type ------------------------------------------------------------------
__device__ __forceinline__ float load_typed(const void* p, int type, int64_t at) {
    if (type == kTypeF32) return static_cast<const float*>(p)[at];
    if (type == kTypeF16) return __half2float(static_cast<const __half*>(p)[at]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
}

// Arrival on the barrier of a CTA of the cluster, and the wait for it, that hand over tensor memory only: what orders the loads before
// and the products behind them are the tcgen05 fences at both ends and the completed loads, so both are relaxed, at cluster scope.  (A
// release there would wait for the global stores of the item before, 2 to 3 us behind the operand loads.)
__device__ __forceinline__ void mbar_arrive_relaxed(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait_relaxed(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_relaxed(uint32_t bar, uint32_t parity, volatile int* abort_flag) {      // bounded as mbar_wait
    uint64_t t0 = 0;
    for (uint32_t i = 1; i < (1u << 30); ++i) {
        if (mbar_try_wait_relaxed(bar, parity)) return true;
        if ((i & 4095u) == 0u) {
            if (*abort_flag) return false;
            const uint64_t now = global_timer_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > kWaitLimitNs) return false;
        }
    }
    return false;
}
// sixteen columns of this warp's 32 TMEM lanes, without the completion wait
__device__ __forceinline__ void tc_ld_32x16_nowait(uint32_t taddr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}

// ---- items of work --------------------------------------------------------------------------------
struct LinearItem { int expert, tile_m, tile_n, lo, hi; };

// A group's rows, clamped so that no offsets, whatever they hold, lead outside A.
__device__ __forceinline__ void clamp_rows(int M, int& lo, int& hi) {
    lo = lo < 0 ? 0 : (lo > M ? M : lo);
    hi = hi < lo ? lo : (hi > M ? M : hi);
}
// Groups of offsets that decrease somewhere could overlap and make more items than the host allows for (a K split has memory for
// one item per cluster), so a group then begins no earlier than the groups before it end: the end of those before `expert`.
// (Not a function of its own: around a call the loads of the next item's bounds lost their lead, 48 -> 54 us with 32 small groups.)
__device__ __forceinline__ int rows_taken(const int32_t* offsets, int M, int expert) {
    int end = 0;
#pragma unroll 1
    for (int e = 0; e < expert; ++e) {
        int lo = offsets[e], hi = offsets[e + 1];
        clamp_rows(M, lo, hi);
        if (hi > lo && hi > end) end = hi;
    }
    return end;
}
// cum[e] = items of the experts before e, cum[experts + 1] = whether the offsets decrease somewhere; one warp.  ROWS: rows of a row tile.
template <int ROWS>
__device__ __forceinline__ void build_item_table(const LinearProblem& p, int* cum, int lane) {
    int base = 0, wild = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 32) {
        const int e = e0 + lane;
        int items = 0, decreases = 0;
        if (e < p.experts) {
            int lo = p.offsets[e], hi = p.offsets[e + 1];
            decreases = hi < lo;
            clamp_rows(p.M, lo, hi);
            if (hi > lo) items = ((hi - 1) / ROWS - lo / ROWS + 1) * p.tiles_n;
        }
        wild |= __any_sync(0xFFFFFFFFu, decreases);
        int scan = items;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xFFFFFFFFu, scan, o);
            if (lane >= o) scan += t;
        }
        if (e < p.experts) cum[e] = base + scan - items;
        base += __shfl_sync(0xFFFFFFFFu, scan, 31);
    }
    __syncwarp();
    if (lane == 0) {
        if (wild) {
            int end = 0;
            base = 0;
            for (int e = 0; e < p.experts; ++e) {
                int lo = p.offsets[e], hi = p.offsets[e + 1];
                clamp_rows(p.M, lo, hi);
                cum[e] = base;
                if (hi <= lo || hi <= end) continue;
                if (lo < end) lo = end;
                end = hi;
                base += ((hi - 1) / ROWS - lo / ROWS + 1) * p.tiles_n;
            }
        }
        cum[p.experts] = base;
        cum[p.experts + 1] = wild;
    }
}
// Row tiles in groups of `group` sweep all weight tiles, so that the CTAs running at one time share a few panels in L2.
__device__ __forceinline__ void raster(int t, int rows, int cols, int group, int& r, int& c) {
    const int per_group = group * cols;
    const int g = t / per_group, in = t - g * per_group;
    const int first = g * group, count = rows - first < group ? rows - first : group;
    r = first + in % count;
    c = in / count;
}
// Item t in two steps: its expert (shared memory) and the loads of the group's bounds, then the rest.  A load waits some 2 us
// behind the operand stages in flight, so a role takes the first step for its next item when it begins one.
struct ItemAhead { int t, expert, lo, hi; };
__device__ __forceinline__ ItemAhead item_ahead(const LinearProblem& p, const int* cum, int t, int n_items) {
    ItemAhead a = {t, 0, 0, p.M};
    if (p.experts && t < n_items) {
        int lo = 0, hi = p.experts;               // cum[lo] <= t < cum[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cum[mid] <= t) lo = mid; else hi = mid;
        }
        a.expert = lo;
        a.lo = p.offsets[lo];
        a.hi = p.offsets[lo + 1];
    }
    return a;
}
template <int ROWS>
__device__ __forceinline__ LinearItem linear_item(const LinearProblem& p, const int* cum, const ItemAhead& a, int group) {
    LinearItem it;
    it.expert = a.expert;
    it.lo = a.lo;
    it.hi = a.hi;
    if (!p.experts) {
        raster(a.t, p.tiles_m, p.tiles_n, group, it.tile_m, it.tile_n);
        return it;
    }
    clamp_rows(p.M, it.lo, it.hi);
    if (cum[p.experts + 1]) {                     // (here, where the bounds are used: in the step before it would wait for their loads)
        const int taken = rows_taken(p.offsets, p.M, a.expert);
        if (it.lo < taken) it.lo = taken;
    }
    const int first = it.lo / ROWS, rows = (it.hi - 1) / ROWS - first + 1;
    raster(a.t - cum[a.expert], rows, p.tiles_n, group, it.tile_m, it.tile_n);
    it.tile_m += first;
    return it;
}

// ---- pair kernel ------------------------------------------------------------------------------------
// Clusters of two CTAs on 256 rows x 192 weight rows (tcgen05.mma.cta_group::2): CTA r holds rows 128 r .. of the A tile with
// their scale tile, weight rows 96 r .. of the tile, and the scale tiles of all 192.  192 columns and not 256 because two
// accumulators (384 columns) and the scales of five stages (24 columns each) fit tensor memory: an item's epilogue has
// the main loop of the next one to run in, and the next main loop starts without waiting for it.  (One accumulator of 256
// columns costs 2 us between two items, 12 x 0.46 us of main loop at K = 3072.)  A weight tile of 192 rows starts in the middle
// of a 128-row scale tile every other time; the instruction then finds its scales two columns (64 rows) further on.
// The stages in flight are also a queue in front of every load of the epilogue (some 3000 cycles), so nothing is loaded
// when it is needed: before a warp waits for its accumulator it fetches its 64 columns' bias and gate and its part of the
// residual (a bulk copy per row) into shared memory.
// Barriers as in gemm_mxfp4_umma_pair; 12 epilogue warps per CTA, one for each 32 rows x 64 columns.
// Bound by the operands' way from L2 to the SMs (11 to 13 TB/s over all SMs) and, on long runs, by the power limit.  Measured: 16384 x
// 4608 -> 12288 with bias, gate and residual 455 to 530 us (3.5 to 4.1 PFLOP/s; the upper end in sustained runs), 8192 x 8192 -> 8192
// plain 225 to 235 us (4.8), where the 256 x 256 tiles of gemm_mxfp4_umma_pair, which move a seventh less per operation, take 191;
// 8 gated experts of 4096 -> 5632 on 16384 rows 363 to 435 us, 4099 x 2240 -> 5601 with gelu_tanh and an odd pitch 58 us.
constexpr int kLinN = 192;
constexpr int kLinStages = 5;
constexpr int kLinABytes = 128 * 128;
constexpr int kLinBBytes = kLinN / 2 * 128;
constexpr int kLinSfaOff = kLinABytes + kLinBBytes;                  // 1 KB: [k tile]
constexpr int kLinSfbOff = kLinSfaOff + 1024;                        // 2 KB: [row tile][k tile]
constexpr int kLinStageBytes = kLinSfbOff + 2048;
constexpr int kLinSfCol0 = 2 * kLinN;
constexpr int kLinEpiWarps = 12;
constexpr int kLinCols = 64;                                         // accumulator columns of a warp
constexpr int kLinThreads = 32 * (3 + kLinEpiWarps);
constexpr int kLinRowBytes = 128;                                    // of the residual, per row and copy
constexpr int kLinRowStride = kLinRowBytes + 16;                     // rows of a warp's copy: no bank conflicts, a lane per row
constexpr int kLinTileStride = 36;                                   // floats between the rows when the same place turns rows into columns
constexpr int kLinVecOff = 32 * kLinRowStride;                       // floats [2][64]: bias by accumulator column, gate by column of out
constexpr int kLinWarpBytes = kLinVecOff + 2 * kLinCols * 4;
constexpr int kLinWarpOff = kLinStages * kLinStageBytes;
constexpr int kLinBarOff = kLinWarpOff + kLinEpiWarps * kLinWarpBytes;
constexpr int kLinNumBars = 3 * kLinStages + 4 + kLinEpiWarps;       // full, empty, sfready, tfull[2], tempty[2], residual of each warp
constexpr int kLinSlotOff = kLinBarOff + 8 * kLinNumBars;
constexpr int kLinAbortOff = kLinSlotOff + 4;
constexpr int kLinCumOff = kLinAbortOff + 4;
constexpr int kLinDynBytes = kLinCumOff + 4 * (kMaxExperts + 2) + 1024;
static_assert(kLinSfCol0 + 24 * kLinStages <= 512, "tensor memory");
static_assert(kLinStageBytes % 1024 == 0 && kLinWarpBytes % 16 == 0 && 32 * kLinTileStride * 4 <= kLinVecOff && kLinDynBytes <= 227 * 1024, "shared memory");

__device__ __forceinline__ uint32_t idesc_mxf4_192(uint32_t sf_id) {
    return (sf_id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kLinN >> 3) << 17) | (1u << 23) | ((256u >> 4) << 24) | (sf_id << 29);
}

// ---- epilogue of 32 rows x 32 accumulator columns, a lane per row ----
// Bias, activation, gate and row scale act on the lane's own registers: 32 independent elements, vectors read from shared
// memory by all lanes at once.  out: whole vectors of the lane's row where the alignment allows it (a chunk is 64 bytes of 16-bit
// elements, full sectors); at other pitches, and at the ragged end of a row, the chunk goes through a tile of shared memory and
// a lane takes a column, so that a warp's accesses stay neighbours in memory.  Gated: 16 features, gate half first.
struct EpiChunk {
    int row0, lo, hi;                    // first row of the warp, rows of the group
    int col, at;                         // first column of out; the chunk's first entry in the warp's bias and gate
    int which;                           // gate row of this lane's row; uniform: the whole warp's, in shared memory
    bool uniform;
    float scale;                         // row scale of this lane's row
    int res_at;                          // byte of the residual within the warp's copied rows
};
template <int C, bool MUL>
__device__ __forceinline__ void apply_shared(const float* vector, float (&v)[C]) {
#pragma unroll
    for (int q = 0; q < C / 4; ++q) {
        const float4 b = reinterpret_cast<const float4*>(vector)[q];
        v[4 * q] = MUL ? v[4 * q] * b.x : v[4 * q] + b.x;
        v[4 * q + 1] = MUL ? v[4 * q + 1] * b.y : v[4 * q + 1] + b.y;
        v[4 * q + 2] = MUL ? v[4 * q + 2] * b.z : v[4 * q + 2] + b.z;
        v[4 * q + 3] = MUL ? v[4 * q + 3] * b.w : v[4 * q + 3] + b.w;
    }
}

template <bool GLU>
__device__ __forceinline__ void epilogue_chunk(const LinearEpilogue& p, const uint32_t (&r)[32], uint8_t* mem, const EpiChunk& c, int lane) {
    constexpr int C = GLU ? 16 : 32;                                 // columns of out
    const int row = c.row0 + lane, have = p.N - c.col;
    const bool mine = row >= c.lo && row < c.hi;
    const float* vec = reinterpret_cast<const float*>(mem + kLinVecOff);
    float v[C];
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] = __uint_as_float(r[i]);
    if (p.bias.ptr) apply_shared<C, false>(vec + c.at, v);
    act_apply<C>(p.act, v);
    if (GLU) {
        float u[C];
#pragma unroll
        for (int i = 0; i < C; ++i) u[i] = __uint_as_float(r[(C + i) & 31]);
        if (p.bias.ptr) apply_shared<C, false>(vec + c.at + 32, u);
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] *= u[i];
    }
    if (p.gate.ptr) {
        if (c.uniform) {
            apply_shared<C, true>(vec + kLinCols + c.at, v);
        } else {                                                     // rows of several gate rows in one warp
#pragma unroll
            for (int i = 0; i < C; ++i) v[i] *= i < have ? vec_entry(p.gate, c.which, c.col + i, 1.f) : 1.f;
        }
    }
    if (p.row_scale) {
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] *= c.scale;
    }
    if (p.vec && have >= C) {
        if (p.residual) {
            const uint8_t* res = mem + lane * kLinRowStride + c.res_at;
            if (p.residual_type == kTypeF32) {
#pragma unroll
                for (int i = 0; i < C / 4; ++i) {
                    const float4 t = reinterpret_cast<const float4*>(res)[i];
                    v[4 * i] = fmaf(p.residual_scale, t.x, v[4 * i]);
                    v[4 * i + 1] = fmaf(p.residual_scale, t.y, v[4 * i + 1]);
                    v[4 * i + 2] = fmaf(p.residual_scale, t.z, v[4 * i + 2]);
                    v[4 * i + 3] = fmaf(p.residual_scale, t.w, v[4 * i + 3]);
                }
            } else if (p.residual_type == kTypeF16) {
#pragma unroll
                for (int i = 0; i < C / 8; ++i) {
                    float t[8];
                    widen8_f16(reinterpret_cast<const uint4*>(res)[i], t);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[8 * i + e] = fmaf(p.residual_scale, t[e], v[8 * i + e]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < C / 8; ++i) {
                    float t[8];
                    widen8(reinterpret_cast<const uint4*>(res)[i], t);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[8 * i + e] = fmaf(p.residual_scale, t[e], v[8 * i + e]);
                }
            }
        }
        if (!mine) return;
        const int64_t at = (int64_t)row * p.ld_out + c.col;
        if (p.out_type == kTypeF32) {
            float* o = static_cast<float*>(p.out) + at;
#pragma unroll
            for (int q = 0; q < C / 8; ++q) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[8 * q + i]);
                store_words<8>(o + 8 * q, w, p.wide);
            }
        } else if (p.out_type == kTypeF16) {
#pragma unroll
            for (int q = 0; q < C / 16; ++q) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const __half2 h = __floats2half2_rn(v[16 * q + 2 * i], v[16 * q + 2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t*>(&h);
                }
                store_words<8>(static_cast<uint16_t*>(p.out) + at + 16 * q, w, p.wide);
            }
        } else {
#pragma unroll
            for (int q = 0; q < C / 16; ++q) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v[16 * q + 2 * i], v[16 * q + 2 * i + 1]);
                    w[i] = *reinterpret_cast<const uint32_t*>(&h);
                }
                store_words<8>(static_cast<uint16_t*>(p.out) + at + 16 * q, w, p.wide);
            }
        }
        return;
    }
    // (an unaligned residual has not been copied: it is read in the column layout)
    float* tile = reinterpret_cast<float*>(mem);
    __syncwarp();                                                    // the chunk before has been read
    float4* at4 = reinterpret_cast<float4*>(tile + lane * kLinTileStride);
#pragma unroll
    for (int i = 0; i < C / 4; ++i) at4[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    __syncwarp();
    constexpr int kRows = 32 / C;                                    // rows of an access
    const int x = lane % C, first = lane / C;
    if (x < have) {
        // rows of the warp's 32 that are in the group
        const int begin = c.lo - c.row0 > 0 ? c.lo - c.row0 : 0, end = c.hi - c.row0 < 32 ? c.hi - c.row0 : 32;
        const int64_t pitch = p.ld_out * kRows, pitch_r = p.ld_residual * kRows;
        int64_t at = (int64_t)(c.row0 + first) * p.ld_out + c.col + x, at_r = (int64_t)(c.row0 + first) * p.ld_residual + c.col + x;
#pragma unroll 1
        for (int in = first; in < 32; in += 8 * kRows) {             // eight rows of a column at a time
            float t[8];
            bool ok[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                t[i] = tile[(in + i * kRows) * kLinTileStride + x];
                ok[i] = in + i * kRows >= begin && in + i * kRows < end;
            }
            if (p.residual) {
                float q[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) q[i] = ok[i] ? load_typed(p.residual, p.residual_type, at_r + i * pitch_r) : 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) t[i] = fmaf(p.residual_scale, q[i], t[i]);
            }
            if (p.out_type == kTypeF32) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (ok[i]) static_cast<float*>(p.out)[at + i * pitch] = t[i];
            } else if (p.out_type == kTypeF16) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (ok[i]) static_cast<__half*>(p.out)[at + i * pitch] = __float2half_rn(t[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (ok[i]) static_cast<__nv_bfloat16*>(p.out)[at + i * pitch] = __float2bfloat16_rn(t[i]);
            }
            at += 8 * pitch;
            at_r += 8 * pitch_r;
        }
    }
}

// Before the accumulator is there: the warp's bias (64 accumulator columns from weight row wrow on) and gate (columns of out
// from col on), zero where they end, into shared memory.  Floats go there by asynchronous copies, which nothing waits for here.
__device__ __forceinline__ void fetch_entry(const NormVec& p, int64_t which, int at, bool exists, float* dst) {
    if (p.type == kTypeF32) {
        const float* src = static_cast<const float*>(p.ptr) + (exists ? which * p.stride + at : 0);
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(exists ? 4 : 0) : "memory");
    } else {
        *dst = exists ? vec_entry(p, which, at, 0.f) : 0.f;
    }
}
template <bool GLU>
__device__ __forceinline__ void fetch_vectors(const LinearEpilogue& p, float* vec, int expert, int wrow, int rows, int col, int which, bool gate, int lane) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int x = lane + 32 * i;
        if (p.bias.ptr) fetch_entry(p.bias, expert, wrow + x, wrow + x < rows, vec + x);
        if (gate && (!GLU || i == 0)) fetch_entry(p.gate, which, col + x, col + x < p.N, vec + kLinCols + x);
    }
}
// This lane's row of the residual from column `col` on, up to kLinRowBytes of it, and the warp's barrier armed with all of them.
// (Only whole 16-byte pieces: what a ragged last chunk needs is read in the column layout.  A gated product takes half of what is
// copied of a 16-bit residual: 32 columns a warp.)
__device__ __forceinline__ void fetch_residual(const LinearEpilogue& p, uint8_t* mem, uint32_t bar, int row, int lo, int hi, int col, int lane) {
    const int size = p.residual_type == kTypeF32 ? 4 : 2;
    const int bytes = (p.N - col) * size < kLinRowBytes ? (p.N - col) * size & ~15 : kLinRowBytes;
    const bool mine = row >= lo && row < hi && bytes > 0;
    const int rows = __popc(__ballot_sync(0xFFFFFFFFu, mine));
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the place may have held a tile of columns
    __syncwarp();
    if (lane == 0) mbar_expect_tx(bar, (uint32_t)(bytes > 0 ? rows * bytes : 0));
    __syncwarp();
    if (mine)
        bulk_load(smem_u32(mem) + lane * kLinRowStride, static_cast<const char*>(p.residual) + ((int64_t)row * p.ld_residual + col) * size, (uint32_t)bytes, bar);
}

// tmap_a: codes [M][K/2]; tmap_b: codes [experts][R][K/2]; tmap_sfa / tmap_sfb: scale tiles [row tiles][k tiles][128 x u32].
template <bool GLU>
__global__ void __launch_bounds__(kLinThreads, 1)
linear_mxfp4_pair(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
                  const __grid_constant__ CUtensorMap tmap_sfa, const __grid_constant__ CUtensorMap tmap_sfb,
                  const __grid_constant__ LinearProblem p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - raw);
    const uint32_t bar0 = base + kLinBarOff;
    auto bar_full = [&](int s) { return bar0 + 8u * s; };
    auto bar_empty = [&](int s) { return bar0 + 8u * (kLinStages + s); };
    auto bar_sfready = [&](int s) { return bar0 + 8u * (2 * kLinStages + s); };
    auto bar_tfull = [&](int a) { return bar0 + 8u * (3 * kLinStages + a); };
    auto bar_tempty = [&](int a) { return bar0 + 8u * (3 * kLinStages + 2 + a); };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + kLinSlotOff);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + kLinAbortOff);
    int* cum = reinterpret_cast<int*>(base_ptr + kLinCumOff);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = (int)(blockIdx.x >> 1), n_pairs = (int)(gridDim.x >> 1);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kLinStages; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); mbar_init(bar_sfready(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(bar_tfull(a), 1); mbar_init(bar_tempty(a), 2 * kLinEpiWarps); }
        for (int e = 0; e < kLinEpiWarps; ++e) mbar_init(bar0 + 8u * (3 * kLinStages + 4 + e), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_b) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_sfa) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_sfb) : "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(base + (uint32_t)kLinSlotOff), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (warp == 2 && p.experts) {
        pdl_wait_prior_grid();                   // the offsets may come from the kernel before
        build_item_table<256>(p, cum, lane);
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const int n_items = p.experts ? cum[p.experts] : p.tiles_m * p.tiles_n;
    const int my_items = pair < n_items ? (n_items - pair + n_pairs - 1) / n_pairs : 0;

    int issued = 0;
    if (warp == 0) {
        // ---------------- producer (both CTAs) ----------------
        if (lane == 0) {
            pdl_wait_prior_grid();
            int it = 0;
            ItemAhead ahead = item_ahead(p, cum, pair, n_items);
            for (int i = 0; i < my_items && !*abort_flag; ++i) {
                const LinearItem w = linear_item<256>(p, cum, ahead, kGemmGroupM);
                ahead = item_ahead(p, cum, pair + (i + 1) * n_pairs, n_items);
                const int sf_tile = w.expert * p.sf_row_tiles + w.tile_n * kLinN / 128;
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const int s = it % kLinStages;
                    if (it >= kLinStages && !mbar_wait(bar_empty(s), ((it / kLinStages) - 1) & 1, abort_flag)) {
                        if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_PRODUCER); *abort_flag = 1; }
                        break;
                    }
                    const uint32_t dst = base + s * kLinStageBytes;
                    const uint32_t leader_full = mapa_shared(bar_full(s), 0);
                    if (rank == 0) mbar_expect_tx(bar_full(s), 2 * kLinStageBytes);
                    tma_load_2d_pair(dst, &tmap_a, kb * 128, w.tile_m * 256 + (int)rank * 128, leader_full);
                    tma_load_3d_pair(dst + kLinABytes, &tmap_b, kb * 128, w.tile_n * kLinN + (int)rank * (kLinN / 2), w.expert, leader_full);
                    tma_load_3d_pair(dst + kLinSfaOff, &tmap_sfa, 0, 2 * kb, w.tile_m * 2 + (int)rank, leader_full);
                    tma_load_3d_pair(dst + kLinSfbOff, &tmap_sfb, 0, 2 * kb, sf_tile, leader_full);
                    issued = it + 1;
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (leader CTA only) ----------------
        if (lane == 0 && rank == 0) {
            const uint64_t a_desc0 = smem_desc_sw128(base);
            const uint64_t b_desc0 = smem_desc_sw128(base + kLinABytes);
            int it = 0;
            bool ok = true;
            ItemAhead ahead = item_ahead(p, cum, pair, n_items);
            for (int i = 0; ok && i < my_items; ++i) {
                const int acc = i & 1;
                if (i >= 2 && !mbar_wait_relaxed(bar_tempty(acc), ((i >> 1) - 1) & 1, abort_flag)) {
                    if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                    break;
                }
                tc_fence_after();
                const LinearItem w = linear_item<256>(p, cum, ahead, kGemmGroupM);
                ahead = item_ahead(p, cum, pair + (i + 1) * n_pairs, n_items);
                const uint32_t d_addr = tmem_base + (uint32_t)(acc * kLinN), shift = (w.tile_n & 1) ? 2u : 0u;
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const int s = it % kLinStages;
                    if (!mbar_wait(bar_sfready(s), (it / kLinStages) & 1, abort_flag)) {
                        if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t off = (uint64_t)((s * kLinStageBytes) >> 4);
                    const uint32_t t_sfa = tmem_base + (uint32_t)(kLinSfCol0 + 24 * s);
                    const uint32_t t_sfb = t_sfa + 8 + shift;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma_mxf4_pair(d_addr, a_desc0 + off + (uint64_t)(2 * k), b_desc0 + off + (uint64_t)(2 * k),
                                         idesc_mxf4_192(2u * (k & 1)), t_sfa + 4 * (k >> 1), t_sfb + 8 * (k >> 1), (uint32_t)((kb | k) != 0));
                    tc_commit_pair(bar_empty(s));
                }
                if (ok) tc_commit_pair(bar_tfull(acc));
            }
        }
    } else if (warp == 2) {
        // ---------------- scale tiles: shared memory -> TMEM of both CTAs (leader CTA only) ----------------
        if (lane == 0 && rank == 0) {
            const uint64_t sfa_desc0 = smem_desc_sf(base + kLinSfaOff);
            const uint64_t sfb_desc0 = smem_desc_sf(base + kLinSfbOff);
            const int total = my_items * p.k_blocks;
            for (int it = 0; it < total; ++it) {
                const int s = it % kLinStages;
                if (!mbar_wait(bar_full(s), (it / kLinStages) & 1, abort_flag)) {
                    if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                    break;
                }
                tc_fence_after();
                const uint64_t off = (uint64_t)((s * kLinStageBytes) >> 4);
                const uint32_t t_sfa = tmem_base + (uint32_t)(kLinSfCol0 + 24 * s);
                const uint32_t t_sfb = t_sfa + 8;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    tc_cp_sf_pair(t_sfa + 4 * y, sfa_desc0 + off + (uint64_t)((512 * y) >> 4));
                    tc_cp_sf_pair(t_sfb + 8 * y, sfb_desc0 + off + (uint64_t)((512 * y) >> 4));
                    tc_cp_sf_pair(t_sfb + 8 * y + 4, sfb_desc0 + off + (uint64_t)((512 * (2 + y)) >> 4));
                }
                asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];"
                             ::"r"(bar_sfready(s)) : "memory");
            }
        }
    } else {
        // ---------------- epilogue: warp = lane quarter x third of the columns ----------------
        const int quarter = warp & 3;            // the lanes of TMEM that this warp may read
        const int third = (warp - 3) >> 2;
        uint8_t* mem = base_ptr + kLinWarpOff + (warp - 3) * kLinWarpBytes;
        const uint32_t bar_res = bar0 + 8u * (3 * kLinStages + 4 + (warp - 3));
        const bool copied = p.epi.residual && p.epi.vec;
        uint32_t res_parity = 0;
        pdl_wait_prior_grid();
        for (int i = 0; i < my_items; ++i) {
            const LinearItem w = linear_item<256>(p, cum, item_ahead(p, cum, pair + i * n_pairs, n_items), kGemmGroupM);
            EpiChunk c;
            c.row0 = w.tile_m * 256 + (int)rank * 128 + quarter * 32;
            c.lo = w.lo;
            c.hi = w.hi;
            const int wrow = w.tile_n * kLinN + third * kLinCols, col = GLU ? wrow / 2 : wrow;
            const bool live = c.row0 < c.hi && c.row0 + 32 > c.lo && wrow < p.R;    // warp-uniform
            if (live) {
                const int row = c.row0 + lane < c.hi ? (c.row0 + lane > c.lo ? c.row0 + lane : c.lo) : c.hi - 1;
                c.which = p.epi.gate.ptr ? row / p.epi.rows_per_gate : 0;
                c.uniform = __all_sync(0xFFFFFFFFu, c.which == __shfl_sync(0xFFFFFFFFu, c.which, 0));
                c.scale = p.epi.row_scale ? p.epi.row_scale[row] : 1.f;
                __syncwarp();                                                       // the vectors of the item before have been read
                if (copied) fetch_residual(p.epi, mem, bar_res, c.row0 + lane, c.lo, c.hi, col, lane);
                fetch_vectors<GLU>(p.epi, reinterpret_cast<float*>(mem + kLinVecOff), w.expert, wrow, p.R, col, c.which, p.epi.gate.ptr && c.uniform, lane);
            }
            const int acc = i & 1;
            const bool ok = mbar_wait(bar_tfull(acc), (i >> 1) & 1, abort_flag);
            if (live && copied) {                                                   // (also when giving up: no copy may outlive the CTA)
                int never = 0;
                if (!mbar_wait(bar_res, res_parity, &never) && !*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_EPILOGUE); *abort_flag = 1; }
                res_parity ^= 1u;
            }
            if (!ok) {
                if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_EPILOGUE); *abort_flag = 1; }
                break;
            }
            tc_fence_after();
            // 32 lanes x 64 columns to registers in one sweep, as two chunks: 32 columns each or, gated, 16 gate columns and
            // their 16 value columns; then the accumulator goes back to the issuer
            uint32_t r[2][32];
            if (live) {
                const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * kLinN + third * kLinCols);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const uint32_t lo = taddr + (uint32_t)(GLU ? 16 * q : 32 * q);
                    tc_ld_32x16_nowait(lo, r[q]);
                    tc_ld_32x16_nowait(lo + (GLU ? 32 : 16), r[q] + 16);
                }
                tc_wait_ld();
#pragma unroll
                for (int q = 0; q < 2; ++q) pin_after_wait(r[q]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_relaxed(mapa_shared(bar_tempty(acc), 0));
            if (!live) continue;
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();                                                           // every lane's entries are there
            // one copy of the epilogue's code for both chunks (two copies of all its variants do not fit the instruction cache): the
            // registers of the next chunk move up
#pragma unroll 1
            for (int q = 0; q < 2; ++q) {
                c.at = GLU ? 16 * q : 32 * q;
                c.col = col + c.at;
                c.res_at = c.at * (p.epi.residual_type == kTypeF32 ? 4 : 2) % kLinRowBytes;
                if (copied && c.res_at == 0 && q > 0 && c.col < p.epi.N) {          // 32-bit residual: the other half of the columns
                    fetch_residual(p.epi, mem, bar_res, c.row0 + lane, c.lo, c.hi, c.col, lane);
                    if (!mbar_wait(bar_res, res_parity, abort_flag) && !*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_EPILOGUE); *abort_flag = 1; }
                    res_parity ^= 1u;
                }
                if (c.col < p.epi.N) epilogue_chunk<GLU>(p.epi, r[0], mem, c, lane);
#pragma unroll
                for (int x = 0; x < 32; ++x) r[0][x] = r[1][x];
            }
        }
    }

    // ---------------- teardown ----------------
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0 && rank == 0) {
        int never = 0;
        for (int m = (issued > kLinStages ? issued - kLinStages : 0); m < issued; ++m)
            if (!mbar_wait(bar_full(m % kLinStages), (m / kLinStages) & 1, &never))
                atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_DRAIN);
    }
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

// ---- narrow kernel ------------------------------------------------------------------------------------
// D[128 weight rows][TB rows of A]: the weight is the M operand, so its tiles are read once, by as many CTAs as there are
// tiles (times the K split), and a few rows of A cost a narrow instruction instead of a mostly empty one.  TB = 32, 64
// (all of A in one tile of that many rows) or 128.  Stages of 256 K-elements: 16 KB of weight codes, 1 KB of their scales,
// TB x 128 bytes of A (of a tile of 128 only the boxes of 32 rows that the group touches), 1 KB of A's scales.  Bound by
// reading the weights: what counts is the bytes in flight, so nearly all shared memory is stages and the epilogue turns 32
// rows of A at a time through 16 KB.
// Cluster of `splits` CTAs: CTA r takes the K-stages [r, r + 1) * k_blocks / splits of one item; partial accumulators meet in
// shared memory and every CTA adds its share of the elements in rank order (the same bits every time).  With splits > 1 a
// cluster has exactly one item, so the partials use the pipeline's memory after its last read; with one CTA per item the
// kernel is persistent.
// Measured: 8 gated experts of 4096 -> 5632 with 16 rows 30 us (4.9 TB/s, 0.76 of what a copy reaches), 32 experts of 5600 -> 2240
// with 1030 rows 48 to 49 us, 24 rows x 4096 -> 4096 8.7 us, one row x 1152 -> 6912 7.4 us (start of a kernel, not bytes).
constexpr int kNarrowThreads = 352;                                      // producer, MMA issuer, 8 epilogue warps, scale copies
template <int TB>
struct NarrowSmem {
    static constexpr int kStages = TB == 32 ? 9 : (TB == 64 ? 7 : 6);
    static constexpr int kWBytes = 128 * 128;
    static constexpr int kABytes = TB * 128;
    static constexpr int kSfwOff = kWBytes + kABytes;
    static constexpr int kSfaOff = kSfwOff + 1024;
    static constexpr int kStageBytes = kSfaOff + 1024;
    static constexpr int kAccOff = kStages * kStageBytes;                 // [32][128] float
    static constexpr int kScalesOff = kAccOff + 32 * 512;                 // [128] float: row scales of the tile
    static constexpr int kBarOff = kScalesOff + 512;
    static constexpr int kNumBars = 3 * kStages + 4;                      // full, empty, sfready, tfull[2], tempty[2]
    static constexpr int kSlotOff = kBarOff + 8 * kNumBars;
    static constexpr int kAbortOff = kSlotOff + 4;
    static constexpr int kEpiFailOff = kAbortOff + 4;
    static constexpr int kCumOff = kEpiFailOff + 4;
    static constexpr int kDynBytes = kCumOff + 4 * (kMaxExperts + 2) + 1024;
    static constexpr int kSfCol0 = 256;                                   // two accumulators of up to 128 columns in front
    static_assert(kStageBytes % 1024 == 0 && TB * 512 <= kStages * kStageBytes && kDynBytes <= 227 * 1024, "shared memory");
    static_assert(kSfCol0 + 16 * kStages <= 512, "tensor memory");
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tmap, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                 " [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t cluster_addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr));      // (no memory clobber: several in flight)
    return v;
}
// M = 128, N = TB, scales of 32-element blocks `id` and `id + 1` of the 128-element scale tile
template <int TB>
__device__ __forceinline__ uint32_t idesc_mxf4_narrow(uint32_t sf_id) {
    return (sf_id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TB >> 3) << 17) | (1u << 23) | ((128u >> 4) << 24) | (sf_id << 29);
}

// A thread's column of out in an item of the narrow kernel and the rows it takes: first, first + kStep, ...
template <bool GLU>
struct NarrowColumn {
    static constexpr int kCols = GLU ? 64 : 128, kStep = 256 / kCols;
    int first, r, n;                     // first row, accumulator lane (gate half), column of out
    float bias, bias_u;
    bool live;
    __device__ __forceinline__ void open(const LinearProblem& p, const LinearItem& w, int thread) {
        const int f = thread % kCols;
        first = thread / kCols;
        r = GLU ? f / 32 * 64 + f % 32 : f;
        n = w.tile_n * kCols + f;
        live = n < p.epi.N;
        bias = live ? vec_entry(p.epi.bias, w.expert, w.tile_n * 128 + r, 0.f) : 0.f;
        bias_u = GLU && live ? vec_entry(p.epi.bias, w.expert, w.tile_n * 128 + r + 32, 0.f) : 0.f;
    }
    // J rows of the column: row0, row0 + stride, ..., `count` of them; all loads go out before the first is used.  row_scale:
    // entries of the rows in shared memory from the first on (null: read here).
    template <int J>
    __device__ __forceinline__ void write(const LinearEpilogue& p, int row0, int stride, int count, const float* row_scale, float (&v)[J], float (&u)[J]) const {
        if (!live) return;
        float res[J], scale[J], gate[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int row = row0 + j * stride;
            const bool ok = j < count;
            res[j] = p.residual && ok ? load_typed(p.residual, p.residual_type, (int64_t)row * p.ld_residual + n) : 0.f;
            gate[j] = p.gate.ptr && ok ? vec_entry(p.gate, row / p.rows_per_gate, n, 1.f) : 1.f;
            scale[j] = !p.row_scale || !ok ? 1.f : (row_scale ? row_scale[j * stride] : p.row_scale[row]);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) v[j] += bias;
        act_apply<J>(p.act, v);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (GLU) v[j] *= u[j] + bias_u;
            if (p.gate.ptr) v[j] *= gate[j];
            if (p.row_scale) v[j] *= scale[j];
            if (p.residual) v[j] = fmaf(p.residual_scale, res[j], v[j]);
        }
        const int64_t at = (int64_t)row0 * p.ld_out + n, step = (int64_t)stride * p.ld_out;
        if (p.out_type == kTypeF32) {
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (j < count) static_cast<float*>(p.out)[at + j * step] = v[j];
        } else if (p.out_type == kTypeF16) {
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (j < count) static_cast<__half*>(p.out)[at + j * step] = __float2half_rn(v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (j < count) static_cast<__nv_bfloat16*>(p.out)[at + j * step] = __float2bfloat16_rn(v[j]);
        }
    }
};

template <bool GLU, int TB>
__global__ void __launch_bounds__(kNarrowThreads, 1)
linear_mxfp4_narrow(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_a,
                    const __grid_constant__ CUtensorMap tmap_sfw, const __grid_constant__ CUtensorMap tmap_sfa,
                    const __grid_constant__ LinearProblem p, const int splits) {
    using L = NarrowSmem<TB>;
    constexpr int NS = L::kStages, kBox = TB == 128 ? 32 : TB;          // rows of a TMA box of A
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - raw);
    const uint32_t bar0 = base + L::kBarOff;
    auto bar_full = [&](int s) { return bar0 + 8u * s; };
    auto bar_empty = [&](int s) { return bar0 + 8u * (NS + s); };
    auto bar_sfready = [&](int s) { return bar0 + 8u * (2 * NS + s); };
    auto bar_tfull = [&](int a) { return bar0 + 8u * (3 * NS + a); };
    auto bar_tempty = [&](int a) { return bar0 + 8u * (3 * NS + 2 + a); };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + L::kSlotOff);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + L::kAbortOff);
    volatile int* epi_fail = reinterpret_cast<volatile int*>(base_ptr + L::kEpiFailOff);
    int* cum = reinterpret_cast<int*>(base_ptr + L::kCumOff);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const int rank = splits > 1 ? (int)cluster_ctarank() : 0;
    const int first = (int)blockIdx.x / splits, step = (int)gridDim.x / splits;
    const int kb0 = (int)((int64_t)p.k_blocks * rank / splits), kb1 = (int)((int64_t)p.k_blocks * (rank + 1) / splits);

    if (threadIdx.x == 0) {
        for (int s = 0; s < NS; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); mbar_init(bar_sfready(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(bar_tfull(a), 1); mbar_init(bar_tempty(a), 8); }
        *abort_flag = 0;
        *epi_fail = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_w) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_sfw) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_sfa) : "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(base + (uint32_t)L::kSlotOff), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == 2 && p.experts) {
        pdl_wait_prior_grid();
        build_item_table<128>(p, cum, lane);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const int n_items = p.experts ? cum[p.experts] : p.tiles_m * p.tiles_n;
    const int my_items = first < n_items ? (n_items - first + step - 1) / step : 0;

    int issued = 0;
    if (warp == 0) {
        // ---------------- producer ----------------
        if (lane == 0) {
            pdl_wait_prior_grid();
            int it = 0;
            ItemAhead ahead = item_ahead(p, cum, first, n_items);
            for (int i = 0; i < my_items && !*abort_flag; ++i) {
                const LinearItem w = linear_item<128>(p, cum, ahead, 4);
                ahead = item_ahead(p, cum, first + (i + 1) * step, n_items);
                int box0 = 0, box1 = 1;
                if (TB == 128) {
                    const int lo = w.lo - w.tile_m * 128, hi = w.hi - w.tile_m * 128;
                    box0 = lo > 0 ? lo / kBox : 0;
                    box1 = hi < 128 ? (hi + kBox - 1) / kBox : 4;
                }
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const int s = it % NS;
                    if (it >= NS && !mbar_wait(bar_empty(s), ((it / NS) - 1) & 1, abort_flag)) {
                        if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_PRODUCER); *abort_flag = 1; }
                        break;
                    }
                    const uint32_t dst = base + s * L::kStageBytes;
                    mbar_expect_tx(bar_full(s), (uint32_t)(L::kWBytes + 2048 + (box1 - box0) * kBox * 128));
                    tma_load_3d(dst, &tmap_w, kb * 128, w.tile_n * 128, w.expert, bar_full(s));
                    for (int b = box0; b < box1; ++b)
                        tma_load_2d(dst + L::kWBytes + b * kBox * 128, &tmap_a, kb * 128, w.tile_m * 128 + b * kBox, bar_full(s));
                    tma_load_3d(dst + L::kSfwOff, &tmap_sfw, 0, 2 * kb, w.expert * p.sf_row_tiles + w.tile_n, bar_full(s));
                    tma_load_3d(dst + L::kSfaOff, &tmap_sfa, 0, 2 * kb, w.tile_m, bar_full(s));
                    issued = it + 1;
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0) {
            const uint64_t w_desc0 = smem_desc_sw128(base);
            const uint64_t a_desc0 = smem_desc_sw128(base + L::kWBytes);
            int it = 0;
            bool ok = true;
            for (int i = 0; ok && i < my_items; ++i) {
                const int acc = i & 1;
                if (i >= 2 && !mbar_wait(bar_tempty(acc), ((i >> 1) - 1) & 1, abort_flag)) {
                    if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                    break;
                }
                tc_fence_after();
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const int s = it % NS;
                    // sfready[s]: the stage's codes have landed and its scales are in TMEM
                    if (!mbar_wait(bar_sfready(s), (it / NS) & 1, abort_flag)) {
                        if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t off = (uint64_t)((s * L::kStageBytes) >> 4);
                    const uint32_t t_sfw = tmem_base + (uint32_t)(L::kSfCol0 + 16 * s);
                    const uint32_t t_sfa = t_sfw + 8;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma_mxf4(tmem_base + (uint32_t)(acc * 128), w_desc0 + off + (uint64_t)(2 * k), a_desc0 + off + (uint64_t)(2 * k),
                                    idesc_mxf4_narrow<TB>(2u * (k & 1)), t_sfw + 4 * (k >> 1), t_sfa + 4 * (k >> 1),
                                    (uint32_t)((kb > kb0) || k));
                    tc_commit(bar_empty(s));
                }
                if (ok) tc_commit(bar_tfull(acc));
            }
        }
    } else if (warp == 10) {
        // ---------------- scale tiles: shared memory -> TMEM (from a thread of their own they overlap the products) ----------------
        if (lane == 0) {
            const uint64_t sfw_desc0 = smem_desc_sf(base + L::kSfwOff);
            const uint64_t sfa_desc0 = smem_desc_sf(base + L::kSfaOff);
            const int total = my_items * (kb1 - kb0);
            for (int it = 0; it < total; ++it) {
                const int s = it % NS;
                if (!mbar_wait(bar_full(s), (it / NS) & 1, abort_flag)) {
                    if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                    break;
                }
                tc_fence_after();
                const uint64_t off = (uint64_t)((s * L::kStageBytes) >> 4);
                const uint32_t t_sfw = tmem_base + (uint32_t)(L::kSfCol0 + 16 * s);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    tc_cp_sf(t_sfw + 4 * y, sfw_desc0 + off + (uint64_t)((512 * y) >> 4));
                    tc_cp_sf(t_sfw + 8 + 4 * y, sfa_desc0 + off + (uint64_t)((512 * y) >> 4));
                }
                tc_commit(bar_sfready(s));
            }
        }
    } else {
        // ---------------- epilogue: warps 2..9 ----------------
        const int quarter = warp & 3;
        const int chalf = (warp - 2) >> 2;
        float* part = reinterpret_cast<float*>(base_ptr + (splits > 1 ? 0 : L::kAccOff));
        float* scales = reinterpret_cast<float*>(base_ptr + L::kScalesOff);
        pdl_wait_prior_grid();
        ItemAhead ahead = item_ahead(p, cum, first, n_items);
        for (int i = 0; i < my_items; ++i) {
            const LinearItem w = linear_item<128>(p, cum, ahead, 4);
            ahead = item_ahead(p, cum, first + (i + 1) * step, n_items);
            const int acc = i & 1;
            // loads wait behind the operand stages in flight (2 us): the row scales come while the item is multiplied
            if (p.epi.row_scale && threadIdx.x < 64 + 128) {
                const int row = w.tile_m * 128 + (int)threadIdx.x - 64;
                scales[threadIdx.x - 64] = row < p.M ? p.epi.row_scale[row] : 0.f;
            }
            // A wait that gives up must not keep this warp from the barriers below: the decision to stop is taken by all
            // epilogue warps together, from a word that is only written before the first of them.
            const bool ok = mbar_wait(bar_tfull(acc), (i >> 1) & 1, abort_flag);
            if (!ok) {
                if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_EPILOGUE); *abort_flag = 1; }
                *epi_fail = 1;
            }
            tc_fence_after();
            const int c0 = w.lo > w.tile_m * 128 ? w.lo - w.tile_m * 128 : 0;                // columns = rows of A in the group
            const int c1 = w.hi < w.tile_m * 128 + 128 ? w.hi - w.tile_m * 128 : 128;
            NarrowColumn<GLU> col;
            if (splits == 1) col.open(p, w, (int)threadIdx.x - 64);                          // (its loads overlap the accumulator's)
            bool stop = false;
            for (int base_c = c0 & ~31; base_c < c1 && !stop; base_c += 32) {
                if (ok && base_c + 16 * chalf < c1) {
                    uint32_t r[16];
                    tc_ld_32x16_nowait(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * 128 + base_c + 16 * chalf), r);
                    tc_wait_ld();
#pragma unroll
                    for (int q = 0; q < 16; ++q) asm volatile("" : "+r"(r[q]));
                    float* at = part + ((splits > 1 ? base_c : 0) + 16 * chalf) * 128 + quarter * 32 + lane;
#pragma unroll
                    for (int q = 0; q < 16; ++q) at[q * 128] = __uint_as_float(r[q]);
                }
                if (base_c + 32 >= c1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_tempty(acc));
                }
                if (splits > 1) continue;                                                    // the rest follows the cluster barrier
                named_barrier_sync(1, 256);
                stop = *epi_fail != 0;
                const int from = c0 > base_c ? c0 : base_c, to = c1 < base_c + 32 ? c1 : base_c + 32;
                constexpr int kStep = NarrowColumn<GLU>::kStep;
                if (!stop)
                    for (int c = from + col.first; c < to; c += 4 * kStep) {
                        float v[4], u[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float* at = part + ((c + j * kStep - base_c) & 31) * 128 + col.r;
                            v[j] = at[0];
                            u[j] = GLU ? at[32] : 0.f;
                        }
                        col.template write<4>(p.epi, w.tile_m * 128 + c, kStep, (to - c + kStep - 1) / kStep, scales + c, v, u);
                    }
                named_barrier_sync(1, 256);                                                  // before the next rows' partials
            }
            if (stop || splits > 1) break;
        }
    }

    tc_fence_before();
    __syncthreads();
    if (splits > 1) {
        cluster_sync_all();
        if (my_items && warp >= 2 && warp < 10 && !*abort_flag) {
            const LinearItem w = linear_item<128>(p, cum, item_ahead(p, cum, first, n_items), 4);
            const int c0 = w.lo > w.tile_m * 128 ? w.lo - w.tile_m * 128 : 0;
            const int c1 = w.hi < w.tile_m * 128 + 128 ? w.hi - w.tile_m * 128 : 128;
            NarrowColumn<GLU> col;
            col.open(p, w, (int)threadIdx.x - 64);
            // four rows and four CTAs' partials in flight; the sum goes in rank order
            const int stride = NarrowColumn<GLU>::kStep * splits;
            for (int c = c0 + col.first + rank * NarrowColumn<GLU>::kStep; c < c1; c += 4 * stride) {
                float sum[4] = {0.f, 0.f, 0.f, 0.f}, sum_u[4] = {0.f, 0.f, 0.f, 0.f};
                for (int q0 = 0; q0 < splits; q0 += 4) {
                    float x[4][4], y[4][4];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            x[q][j] = y[q][j] = 0.f;
                            if (q0 + q < splits && c + j * stride < c1) {
                                const uint32_t at = mapa_shared(base + (uint32_t)((c + j * stride) * 128 + col.r) * 4u, (uint32_t)(q0 + q));
                                x[q][j] = ld_cluster_f32(at);
                                if (GLU) y[q][j] = ld_cluster_f32(at + 128u);
                            }
                        }
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            sum[j] += x[q][j];
                            if (GLU) sum_u[j] += y[q][j];
                        }
                }
                col.template write<4>(p.epi, w.tile_m * 128 + c, stride, (c1 - c + stride - 1) / stride, nullptr, sum, sum_u);
            }
        }
    }

    // ---------------- teardown ----------------
    if (*abort_flag && threadIdx.x == 0) {
        int never = 0;
        for (int m = (issued > NS ? issued - NS : 0); m < issued; ++m)
            if (!mbar_wait(bar_full(m % NS), (m / NS) & 1, &never)) atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_DRAIN);
    }
    __syncthreads();
    if (splits > 1) cluster_sync_all();              // nobody's partials go away while a peer reads them
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

}  // namespace kq
