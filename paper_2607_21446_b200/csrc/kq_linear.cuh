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
//   linear_mxfp4_pair    CTA pairs on 256 rows x 256 weight rows (tcgen05.mma.cta_group::2): many rows per weight.
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
    int M, N;                            // rows of A; columns of out
    int act;
    NormVec bias;                        // [weight rows], stride: between experts
    NormVec gate;                        // [N], stride: between gate rows
    int rows_per_gate;
    const float* row_scale;              // [M] or null
    const void* residual; int residual_type; int64_t ld_residual; float residual_scale;
    void* out; int out_type; int64_t ld_out;
    int vec;                             // bias, gate, residual, out: full 32-column chunks allow 16-byte accesses
    int wide;                            // out: and 32-byte stores
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
// gelu with erf by Abramowitz and Stegun 7.1.26, |error of erf| <= 1.5e-7 (absolute): the result's error stays below
// 1e-7 |v|, one 24-bit rounding.  e^x by the hardware exponential.
template <int ACT>
__device__ __forceinline__ float act_fn(float v) {
    if constexpr (ACT == kActRelu) return v > 0.f ? v : 0.f;
    if constexpr (ACT == kActSilu) return __fdividef(v, 1.f + __expf(-v));
    if constexpr (ACT == kActGeluTanh)
        return __fdividef(v, 1.f + __expf(-1.5957691216057308f * fmaf(0.044715f * v * v, v, v)));
    if constexpr (ACT == kActGelu) {
        const float x = fabsf(v) * 0.70710678118654752f;
        const float t = __fdividef(1.f, fmaf(0.3275911f, x, 1.f));
        const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
        const float q = 0.5f * poly * __expf(-x * x);               // half of erfc(|v| / sqrt 2)
        return v * (v >= 0.f ? 1.f - q : q);
    }
    return v;
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
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = act_fn<kActGelu>(v[i]);
            break;
        case kActGeluTanh:
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = act_fn<kActGeluTanh>(v[i]);
            break;
        default: break;
    }
}

// ---- scalar access by runtime type ------------------------------------------------------------------
__device__ __forceinline__ float load_typed(const void* p, int type, int64_t at) {
    if (type == kTypeF32) return static_cast<const float*>(p)[at];
    if (type == kTypeF16) return __half2float(static_cast<const __half*>(p)[at]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
}
__device__ __forceinline__ void store_typed(void* p, int type, int64_t at, float v) {
    if (type == kTypeF32) static_cast<float*>(p)[at] = v;
    else if (type == kTypeF16) static_cast<__half*>(p)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
}

// One output element from its accumulator(s): feature n, weight row r (the gate row; its value row is r + 32).
template <bool GLU>
__device__ __forceinline__ float linear_element(const LinearEpilogue& p, int expert, int row, int n, int r, float acc, float acc_u,
                                                float bias, float bias_u) {
    float v[1] = {acc + bias};
    act_apply<1>(p.act, v);
    if (GLU) v[0] *= acc_u + bias_u;
    if (p.gate.ptr) v[0] *= vec_entry(p.gate, row / p.rows_per_gate, n, 1.f);
    if (p.row_scale) v[0] *= __ldg(p.row_scale + row);
    return v[0];
}

// ---- items of work --------------------------------------------------------------------------------
struct LinearItem { int expert, tile_m, tile_n, lo, hi; };

// Rows of group e, clamped so that no offsets, whatever they hold, lead outside A.
__device__ __forceinline__ void group_rows(const LinearProblem& p, int e, int& lo, int& hi) {
    lo = __ldg(p.offsets + e);
    hi = __ldg(p.offsets + e + 1);
    lo = lo < 0 ? 0 : (lo > p.M ? p.M : lo);
    hi = hi < lo ? lo : (hi > p.M ? p.M : hi);
}
// cum[e] = items of the experts before e; one warp.  ROWS: rows of a row tile.
template <int ROWS>
__device__ __forceinline__ void build_item_table(const LinearProblem& p, int* cum, int lane) {
    int base = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 32) {
        const int e = e0 + lane;
        int items = 0;
        if (e < p.experts) {
            int lo, hi;
            group_rows(p, e, lo, hi);
            if (hi > lo) items = ((hi - 1) / ROWS - lo / ROWS + 1) * p.tiles_n;
        }
        int scan = items;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xFFFFFFFFu, scan, o);
            if (lane >= o) scan += t;
        }
        if (e < p.experts) cum[e] = base + scan - items;
        base += __shfl_sync(0xFFFFFFFFu, scan, 31);
    }
    if (lane == 0) cum[p.experts] = base;
}
// Row tiles in groups of `group` sweep all weight tiles, so that the CTAs running at one time share a few panels in L2.
__device__ __forceinline__ void raster(int t, int rows, int cols, int group, int& r, int& c) {
    const int per_group = group * cols;
    const int g = t / per_group, in = t - g * per_group;
    const int first = g * group, count = rows - first < group ? rows - first : group;
    r = first + in % count;
    c = in / count;
}
template <int ROWS>
__device__ __forceinline__ LinearItem linear_item(const LinearProblem& p, const int* cum, int t, int group) {
    LinearItem it;
    if (!p.experts) {
        it.expert = 0;
        raster(t, p.tiles_m, p.tiles_n, group, it.tile_m, it.tile_n);
        it.lo = 0;
        it.hi = p.M;
        return it;
    }
    int a = 0, b = p.experts;                     // cum[a] <= t < cum[b]
    while (b - a > 1) {
        const int mid = (a + b) >> 1;
        if (cum[mid] <= t) a = mid; else b = mid;
    }
    it.expert = a;
    group_rows(p, a, it.lo, it.hi);
    const int first = it.lo / ROWS, rows = (it.hi - 1) / ROWS - first + 1;
    raster(t - cum[a], rows, p.tiles_n, group, it.tile_m, it.tile_n);
    it.tile_m += first;
    return it;
}

// ---- pair kernel ------------------------------------------------------------------------------------
// Stage layout, barriers and roles are those of gemm_mxfp4_umma_pair; what is new: items instead of tiles, the 3-D map of
// the weights (experts), and the epilogue.
constexpr int kLinPStages = kF4PStages;
constexpr int kLinPBarOff = kLinPStages * kF4PStageBytes;
constexpr int kLinPNumBars = 3 * kLinPStages + 2;
constexpr int kLinPSlotOff = kLinPBarOff + 8 * kLinPNumBars;
constexpr int kLinPAbortOff = kLinPSlotOff + 4;
constexpr int kLinPCumOff = kLinPAbortOff + 4;
constexpr int kLinPDynBytes = kLinPCumOff + 4 * (kMaxExperts + 1) + 1024;

// lane l, register i  <->  lane i, register l
__device__ __forceinline__ void warp_transpose(float (&v)[32], int lane) {
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1)
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (!(i & s)) {
                const bool up = lane & s;
                const float got = __shfl_xor_sync(0xFFFFFFFFu, up ? v[i] : v[i | s], s);
                if (up) v[i] = got; else v[i | s] = got;
            }
}

// 32 columns of one row held by one thread; every access of the chunk is a vector (epi.vec, all 32 columns exist).
template <bool GLU>
__device__ __forceinline__ void epilogue_row(const LinearEpilogue& p, float (&v)[32], float (&u)[32], int expert, int row, int col, int r) {
    if (p.bias.ptr) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float b[8];
            load_param(p.bias, expert, r + 8 * q, 8, true, 1, 0.f, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[8 * q + i] += b[i];
            if (GLU) {
                load_param(p.bias, expert, r + 32 + 8 * q, 8, true, 1, 0.f, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) u[8 * q + i] += b[i];
            }
        }
    }
    act_apply<32>(p.act, v);
    if (GLU) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= u[i];
    }
    if (p.gate.ptr) {
        const int which = row / p.rows_per_gate;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float b[8];
            load_param(p.gate, which, col + 8 * q, 8, true, 1, 1.f, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[8 * q + i] *= b[i];
        }
    }
    if (p.row_scale) {
        const float s = __ldg(p.row_scale + row);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= s;
    }
    if (p.residual) {
        const int64_t at = (int64_t)row * p.ld_residual + col;
        if (p.residual_type == kTypeF32) {
            const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p.residual) + at);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 t = q[i];
                v[4 * i] = fmaf(p.residual_scale, t.x, v[4 * i]);
                v[4 * i + 1] = fmaf(p.residual_scale, t.y, v[4 * i + 1]);
                v[4 * i + 2] = fmaf(p.residual_scale, t.z, v[4 * i + 2]);
                v[4 * i + 3] = fmaf(p.residual_scale, t.w, v[4 * i + 3]);
            }
        } else {
            const uint4* q = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.residual) + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float t[8];
                if (p.residual_type == kTypeF16) widen8_f16(q[i], t); else widen8(q[i], t);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[8 * i + e] = fmaf(p.residual_scale, t[e], v[8 * i + e]);
            }
        }
    }
    const int64_t at = (int64_t)row * p.ld_out + col;
    if (p.out_type == kTypeF32) {
        float* o = static_cast<float*>(p.out) + at;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (p.wide) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(v[8 * q + i]);
                st_global_32(o + 8 * q, w);
            } else {
                reinterpret_cast<float4*>(o)[2 * q] = make_float4(v[8 * q], v[8 * q + 1], v[8 * q + 2], v[8 * q + 3]);
                reinterpret_cast<float4*>(o)[2 * q + 1] = make_float4(v[8 * q + 4], v[8 * q + 5], v[8 * q + 6], v[8 * q + 7]);
            }
        }
    } else {
        uint16_t* o = static_cast<uint16_t*>(p.out) + at;
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (p.out_type == kTypeF16) {
                const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
        if (p.wide) {
            const uint32_t lo[8] = {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]};
            const uint32_t hi[8] = {w[8], w[9], w[10], w[11], w[12], w[13], w[14], w[15]};
            st_global_32(o, lo);
            st_global_32(o + 16, hi);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) reinterpret_cast<uint4*>(o)[q] = make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
        }
    }
}

// 32 rows x 32 columns of a warp, lane = column after the transpose: any alignment, any pitch, a ragged last chunk.
template <bool GLU>
__device__ __forceinline__ void epilogue_column(const LinearEpilogue& p, float (&v)[32], float (&u)[32], int expert, int row0, int lo, int hi,
                                                int col0, int r0, int lane) {
    warp_transpose(v, lane);
    if (GLU) warp_transpose(u, lane);
    const int n = col0 + lane, r = r0 + lane;
    if (n >= p.N) return;
    const float bias = vec_entry(p.bias, expert, r, 0.f), bias_u = GLU ? vec_entry(p.bias, expert, r + 32, 0.f) : 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] += bias;
    act_apply<32>(p.act, v);
    if (GLU) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= u[i] + bias_u;
    }
    if (p.gate.ptr) {
        // one load per change of the gate row
        int which = -1;
        float g = 1.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int w = (row0 + i < hi ? row0 + i : hi - 1) / p.rows_per_gate;
            if (w != which) { which = w; g = vec_entry(p.gate, w, n, 1.f); }
            v[i] *= g;
        }
    }
    if (p.row_scale) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (row0 + i < hi) v[i] *= __ldg(p.row_scale + row0 + i);
    }
    if (p.residual) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (row0 + i >= lo && row0 + i < hi)
                v[i] = fmaf(p.residual_scale, load_typed(p.residual, p.residual_type, (int64_t)(row0 + i) * p.ld_residual + n), v[i]);
    }
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (row0 + i >= lo && row0 + i < hi) store_typed(p.out, p.out_type, (int64_t)(row0 + i) * p.ld_out + n, v[i]);
}

// tmap_a: codes [M][K/2]; tmap_b: codes [experts][R][K/2]; tmap_sfa / tmap_sfb: scale tiles [row tiles][k tiles][128 x u32].
template <bool GLU>
__global__ void __launch_bounds__(kF4PThreads, 1)
linear_mxfp4_pair(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
                  const __grid_constant__ CUtensorMap tmap_sfa, const __grid_constant__ CUtensorMap tmap_sfb,
                  const __grid_constant__ LinearProblem p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - raw);
    const uint32_t bar0 = base + kLinPBarOff;
    auto bar_full = [&](int s) { return bar0 + 8u * s; };
    auto bar_empty = [&](int s) { return bar0 + 8u * (kLinPStages + s); };
    auto bar_sfready = [&](int s) { return bar0 + 8u * (2 * kLinPStages + s); };
    const uint32_t bar_tfull = bar0 + 8u * (3 * kLinPStages);
    const uint32_t bar_tempty = bar0 + 8u * (3 * kLinPStages + 1);
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + kLinPSlotOff);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + kLinPAbortOff);
    int* cum = reinterpret_cast<int*>(base_ptr + kLinPCumOff);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int pair = (int)(blockIdx.x >> 1), n_pairs = (int)(gridDim.x >> 1);

    if (threadIdx.x == 0) {
        for (int s = 0; s < kLinPStages; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); mbar_init(bar_sfready(s), 1); }
        mbar_init(bar_tfull, 1);
        mbar_init(bar_tempty, 16);
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
                     ::"r"(base + (uint32_t)kLinPSlotOff), "r"(512u) : "memory");
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
            for (int i = 0; i < my_items && !*abort_flag; ++i) {
                const LinearItem w = linear_item<256>(p, cum, pair + i * n_pairs, kGemmGroupM);
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const int s = it % kLinPStages;
                    if (it >= kLinPStages && !mbar_wait(bar_empty(s), ((it / kLinPStages) - 1) & 1, abort_flag)) {
                        if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_PRODUCER); *abort_flag = 1; }
                        break;
                    }
                    const uint32_t dst = base + s * kF4PStageBytes;
                    const uint32_t leader_full = mapa_shared(bar_full(s), 0);
                    if (rank == 0) mbar_expect_tx(bar_full(s), 2 * kF4PLoadBytes);
                    tma_load_2d_pair(dst, &tmap_a, kb * kF4PKBytes, w.tile_m * 256 + (int)rank * 128, leader_full);
                    tma_load_3d_pair(dst + kF4PABytes, &tmap_b, kb * kF4PKBytes, w.tile_n * 256 + (int)rank * 128, w.expert, leader_full);
                    tma_load_3d_pair(dst + kF4PSfaOff, &tmap_sfa, 0, 2 * kb, w.tile_m * 2 + (int)rank, leader_full);
                    tma_load_3d_pair(dst + kF4PSfbOff, &tmap_sfb, 0, 2 * kb, w.expert * p.sf_row_tiles + w.tile_n * 2, leader_full);
                    issued = it + 1;
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (leader CTA only) ----------------
        if (lane == 0 && rank == 0) {
            const uint64_t a_desc0 = smem_desc_sw128(base);
            const uint64_t b_desc0 = smem_desc_sw128(base + kF4PABytes);
            int it = 0;
            bool ok = true;
            for (int i = 0; ok && i < my_items; ++i) {
                if (i >= 1 && !mbar_wait(bar_tempty, (i - 1) & 1, abort_flag)) {
                    if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                    break;
                }
                tc_fence_after();
                for (int kb = 0; kb < p.k_blocks; ++kb, ++it) {
                    const int s = it % kLinPStages;
                    if (!mbar_wait(bar_sfready(s), (it / kLinPStages) & 1, abort_flag)) {
                        if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t off = (uint64_t)((s * kF4PStageBytes) >> 4);
                    const uint32_t t_sfa = tmem_base + (uint32_t)(kF4PSfCol0 + 24 * s);
                    const uint32_t t_sfb = t_sfa + 8;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma_mxf4_pair(tmem_base, a_desc0 + off + (uint64_t)(2 * k), b_desc0 + off + (uint64_t)(2 * k),
                                         idesc_mxf4_pair(2u * (k & 1), 2u * (k & 1)), t_sfa + 4 * (k >> 1), t_sfb + 8 * (k >> 1),
                                         (uint32_t)((kb | k) != 0));
                    tc_commit_pair(bar_empty(s));
                }
                if (ok) tc_commit_pair(bar_tfull);
            }
        }
    } else if (warp == 10) {
        // ---------------- scale tiles: shared memory -> TMEM of both CTAs (leader CTA only) ----------------
        if (lane == 0 && rank == 0) {
            const uint64_t sfa_desc0 = smem_desc_sf(base + kF4PSfaOff);
            const uint64_t sfb_desc0 = smem_desc_sf(base + kF4PSfbOff);
            const int total = my_items * p.k_blocks;
            for (int it = 0; it < total; ++it) {
                const int s = it % kLinPStages;
                if (!mbar_wait(bar_full(s), (it / kLinPStages) & 1, abort_flag)) {
                    if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                    break;
                }
                tc_fence_after();
                const uint64_t off = (uint64_t)((s * kF4PStageBytes) >> 4);
                const uint32_t t_sfa = tmem_base + (uint32_t)(kF4PSfCol0 + 24 * s);
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
        // ---------------- epilogue: warps 2..9 of both CTAs; warp = lane quarter x column half ----------------
        const int quarter = warp & 3;
        const int chalf = (warp - 2) >> 2;
        pdl_wait_prior_grid();
        for (int i = 0; i < my_items; ++i) {
            const LinearItem w = linear_item<256>(p, cum, pair + i * n_pairs, kGemmGroupM);
            if (!mbar_wait(bar_tfull, i & 1, abort_flag)) {
                if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_EPILOGUE); *abort_flag = 1; }
                break;
            }
            tc_fence_after();
            // 32 lanes x 128 columns to registers in one sweep; the accumulator goes back to the issuer at once
            uint32_t r[4][32];
#pragma unroll
            for (int cc = 0; cc < 4; ++cc)
                tc_ld_32x32_nowait(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)((chalf * 4 + cc) * 32), r[cc]);
            tc_wait_ld();
#pragma unroll
            for (int cc = 0; cc < 4; ++cc) pin_after_wait(r[cc]);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(mapa_shared(bar_tempty, 0));
            const int row0 = w.tile_m * 256 + (int)rank * 128 + quarter * 32;
            const int row = row0 + lane;
            const int wrow = w.tile_n * 256 + chalf * 128;           // weight row of r[0][0]
            if (row0 >= w.hi || row0 + 32 <= w.lo) continue;         // warp-uniform: no row of this warp is in the group
#pragma unroll
            for (int cc = 0; cc < 4; cc += GLU ? 2 : 1) {
                const int col = GLU ? (wrow + cc * 32) / 2 : wrow + cc * 32;
                if (col < p.epi.N) {
                    float v[32], u[32];
#pragma unroll
                    for (int q = 0; q < 32; ++q) {
                        v[q] = __uint_as_float(r[cc][q]);
                        if (GLU) u[q] = __uint_as_float(r[cc + (GLU ? 1 : 0)][q]);
                    }
                    if (p.epi.vec && col + 32 <= p.epi.N) {
                        if (row >= w.lo && row < w.hi) epilogue_row<GLU>(p.epi, v, u, w.expert, row, col, wrow + cc * 32);
                        __syncwarp();
                    } else {
                        epilogue_column<GLU>(p.epi, v, u, w.expert, row0, w.lo, w.hi, col, wrow + cc * 32, lane);
                        __syncwarp();
                    }
                }
            }
        }
    }

    // ---------------- teardown ----------------
    tc_fence_before();
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0 && rank == 0) {
        int never = 0;
        for (int m = (issued > kLinPStages ? issued - kLinPStages : 0); m < issued; ++m)
            if (!mbar_wait(bar_full(m % kLinPStages), (m / kLinPStages) & 1, &never))
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
// TB x 128 bytes of A, 1 KB of A's scales.  Cluster of `splits` CTAs: CTA r takes the K-stages [r, r + 1) * k_blocks /
// splits of one item; partial accumulators meet in shared memory and every CTA adds its share of the elements in rank
// order (the same bits every time).  With splits > 1 a cluster has exactly one item, so the partials use the pipeline's
// memory after its last read; with one CTA per item the kernel is persistent and they have their own.
template <int TB>
struct NarrowSmem {
    static constexpr int kStages = TB == 32 ? 8 : (TB == 64 ? 6 : 4);
    static constexpr int kWBytes = 128 * 128;
    static constexpr int kABytes = TB * 128;
    static constexpr int kSfwOff = kWBytes + kABytes;
    static constexpr int kSfaOff = kSfwOff + 1024;
    static constexpr int kLoadBytes = kSfaOff + 1024;
    static constexpr int kStageBytes = (kLoadBytes + 1023) / 1024 * 1024;
    static constexpr int kAccOff = kStages * kStageBytes;                 // [TB][128] float
    static constexpr int kBarOff = kAccOff + TB * 512;
    static constexpr int kNumBars = 2 * kStages + 4;                      // full, empty, tfull[2], tempty[2]
    static constexpr int kSlotOff = kBarOff + 8 * kNumBars;
    static constexpr int kAbortOff = kSlotOff + 4;
    static constexpr int kEpiFailOff = kAbortOff + 4;
    static constexpr int kCumOff = kEpiFailOff + 4;
    static constexpr int kDynBytes = kCumOff + 4 * (kMaxExperts + 1) + 1024;
    static constexpr int kSfCol0 = 256;                                   // two accumulators of up to 128 columns in front
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tmap, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
                 " [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(tmap), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t cluster_addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr) : "memory");
    return v;
}
// M = 128, N = TB, scales of 32-element blocks `id` and `id + 1` of the 128-element scale tile
template <int TB>
__device__ __forceinline__ uint32_t idesc_mxf4_narrow(uint32_t sf_id) {
    return (sf_id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TB >> 3) << 17) | (1u << 23) | ((128u >> 4) << 24) | (sf_id << 29);
}

template <bool GLU, int TB>
__global__ void __launch_bounds__(kGemmThreads, 1)
linear_mxfp4_narrow(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_a,
                    const __grid_constant__ CUtensorMap tmap_sfw, const __grid_constant__ CUtensorMap tmap_sfa,
                    const __grid_constant__ LinearProblem p, const int splits) {
    using L = NarrowSmem<TB>;
    constexpr int NS = L::kStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - raw);
    const uint32_t bar0 = base + L::kBarOff;
    auto bar_full = [&](int s) { return bar0 + 8u * s; };
    auto bar_empty = [&](int s) { return bar0 + 8u * (NS + s); };
    auto bar_tfull = [&](int a) { return bar0 + 8u * (2 * NS + a); };
    auto bar_tempty = [&](int a) { return bar0 + 8u * (2 * NS + 2 + a); };
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
        for (int s = 0; s < NS; ++s) { mbar_init(bar_full(s), 1); mbar_init(bar_empty(s), 1); }
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
            for (int i = 0; i < my_items && !*abort_flag; ++i) {
                const LinearItem w = linear_item<128>(p, cum, first + i * step, 4);
                for (int kb = kb0; kb < kb1; ++kb, ++it) {
                    const int s = it % NS;
                    if (it >= NS && !mbar_wait(bar_empty(s), ((it / NS) - 1) & 1, abort_flag)) {
                        if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_PRODUCER); *abort_flag = 1; }
                        break;
                    }
                    const uint32_t dst = base + s * L::kStageBytes;
                    mbar_expect_tx(bar_full(s), L::kLoadBytes);
                    tma_load_3d(dst, &tmap_w, kb * 128, w.tile_n * 128, w.expert, bar_full(s));
                    tma_load_2d(dst + L::kWBytes, &tmap_a, kb * 128, w.tile_m * 128, bar_full(s));
                    tma_load_3d(dst + L::kSfwOff, &tmap_sfw, 0, 2 * kb, w.expert * p.sf_row_tiles + w.tile_n, bar_full(s));
                    tma_load_3d(dst + L::kSfaOff, &tmap_sfa, 0, 2 * kb, w.tile_m, bar_full(s));
                    issued = it + 1;
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- scale copies and MMA ----------------
        if (lane == 0) {
            const uint64_t w_desc0 = smem_desc_sw128(base);
            const uint64_t a_desc0 = smem_desc_sw128(base + L::kWBytes);
            const uint64_t sfw_desc0 = smem_desc_sf(base + L::kSfwOff);
            const uint64_t sfa_desc0 = smem_desc_sf(base + L::kSfaOff);
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
                    if (!mbar_wait(bar_full(s), (it / NS) & 1, abort_flag)) {
                        if (!*abort_flag) { atomicExch(&g_kq_device_error, KQ_DEV_TIMEOUT_GEMM_MMA); *abort_flag = 1; }
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t off = (uint64_t)((s * L::kStageBytes) >> 4);
                    const uint32_t t_sfw = tmem_base + (uint32_t)(L::kSfCol0 + 16 * s);
                    const uint32_t t_sfa = t_sfw + 8;
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        tc_cp_sf(t_sfw + 4 * y, sfw_desc0 + off + (uint64_t)((512 * y) >> 4));
                        tc_cp_sf(t_sfa + 4 * y, sfa_desc0 + off + (uint64_t)((512 * y) >> 4));
                    }
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
    } else {
        // ---------------- epilogue: warps 2..9 ----------------
        const int quarter = warp & 3;
        const int chalf = (warp - 2) >> 2;
        float* part = reinterpret_cast<float*>(base_ptr + (splits > 1 ? 0 : L::kAccOff));
        pdl_wait_prior_grid();
        for (int i = 0; i < my_items; ++i) {
            const LinearItem w = linear_item<128>(p, cum, first + i * step, 4);
            const int acc = i & 1;
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
            for (int c = (c0 / 8 + chalf) * 8; ok && c < c1; c += 16) {
                uint32_t r[8];
                tc_ld_32x8_nowait(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(acc * 128 + c), r);
                tc_wait_ld();
#pragma unroll
                for (int q = 0; q < 8; ++q) asm volatile("" : "+r"(r[q]));
#pragma unroll
                for (int q = 0; q < 8; ++q) part[(c + q) * 128 + quarter * 32 + lane] = __uint_as_float(r[q]);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_tempty(acc));
            if (splits > 1) break;                                                           // the rest follows the cluster barrier
            named_barrier_sync(1, 256);
            if (*epi_fail) break;
            constexpr int kCols = GLU ? 64 : 128;
            for (int x = (int)threadIdx.x - 64; x < (c1 - c0) * kCols; x += 256) {
                const int c = c0 + x / kCols, f = x % kCols;
                const int r = GLU ? f / 32 * 64 + f % 32 : f;
                const int n = GLU ? w.tile_n * 64 + f : w.tile_n * 128 + f, wrow = w.tile_n * 128 + r, row = w.tile_m * 128 + c;
                if (n < p.epi.N) {
                    float v = linear_element<GLU>(p.epi, w.expert, row, n, wrow, part[c * 128 + r], GLU ? part[c * 128 + r + 32] : 0.f,
                                                  vec_entry(p.epi.bias, w.expert, wrow, 0.f), GLU ? vec_entry(p.epi.bias, w.expert, wrow + 32, 0.f) : 0.f);
                    if (p.epi.residual)
                        v = fmaf(p.epi.residual_scale, load_typed(p.epi.residual, p.epi.residual_type, (int64_t)row * p.epi.ld_residual + n), v);
                    store_typed(p.epi.out, p.epi.out_type, (int64_t)row * p.epi.ld_out + n, v);
                }
            }
            named_barrier_sync(1, 256);                                                      // before the next item's partials
        }
    }

    tc_fence_before();
    __syncthreads();
    if (splits > 1) {
        cluster_sync_all();
        if (my_items && warp >= 2 && !*abort_flag) {
            const LinearItem w = linear_item<128>(p, cum, first, 4);
            const int c0 = w.lo > w.tile_m * 128 ? w.lo - w.tile_m * 128 : 0;
            const int c1 = w.hi < w.tile_m * 128 + 128 ? w.hi - w.tile_m * 128 : 128;
            constexpr int kCols = GLU ? 64 : 128;
            for (int x = rank * 256 + (int)threadIdx.x - 64; x < (c1 - c0) * kCols; x += 256 * splits) {
                const int c = c0 + x / kCols, f = x % kCols;
                const int r = GLU ? f / 32 * 64 + f % 32 : f;
                const int n = GLU ? w.tile_n * 64 + f : w.tile_n * 128 + f, wrow = w.tile_n * 128 + r, row = w.tile_m * 128 + c;
                if (n < p.epi.N) {
                    float acc = 0.f, acc_u = 0.f;
                    for (int q = 0; q < splits; ++q) {
                        const uint32_t at = mapa_shared(base + (uint32_t)(c * 128 + r) * 4u, (uint32_t)q);
                        acc += ld_cluster_f32(at);
                        if (GLU) acc_u += ld_cluster_f32(at + 128u);
                    }
                    float v = linear_element<GLU>(p.epi, w.expert, row, n, wrow, acc, acc_u, vec_entry(p.epi.bias, w.expert, wrow, 0.f),
                                                  GLU ? vec_entry(p.epi.bias, w.expert, wrow + 32, 0.f) : 0.f);
                    if (p.epi.residual)
                        v = fmaf(p.epi.residual_scale, load_typed(p.epi.residual, p.epi.residual_type, (int64_t)row * p.epi.ld_residual + n), v);
                    store_typed(p.epi.out, p.epi.out_type, (int64_t)row * p.epi.ld_out + n, v);
                }
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
