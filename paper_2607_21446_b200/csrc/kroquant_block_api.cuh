// Host side of the transformer block's operators (contract: include/kroquant.h): the linear layers around the MXFP4
// product and the norm / gate / residual step with its backward pass.  Included at the end of kroquant_api.cu: one
// translation unit, one device error word.
#pragma once
#include "kq_linear.cuh"
#include "kq_norm.cuh"

namespace {

int type_size(int t) { return t == KQ_OUT_F32 ? 4 : 2; }
bool known_type(int t) { return t == KQ_OUT_F32 || t == KQ_OUT_BF16 || t == KQ_OUT_FP16; }
bool element_aligned(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % type_size(type) == 0; }
// pointer and pitch (in elements) both keep rows on `bytes`-byte boundaries
bool rows_aligned(const void* p, int64_t pitch, int type, int bytes) {
    return !p || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && pitch * type_size(type) % bytes == 0);
}

// a launch that may set up while the kernel before it drains (every kernel here waits for it before it touches memory)
void launch_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* attr, dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st) {
    *cfg = {};
    cfg->gridDim = grid;
    cfg->blockDim = block;
    cfg->dynamicSmemBytes = smem;
    cfg->stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg->attrs = attr;
    cfg->numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg->numAttrs = 2;
    }
}
template <typename... Params, typename... Args>
kq_status_t launch(const cudaLaunchConfig_t& cfg, void (*kernel)(Params...), Args&&... args) {
    if (cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...) != cudaSuccess) {
        (void)cudaGetLastError();
        return KQ_ERR_CUDA;
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return KQ_OK;
}

bool encode_map(EncodeTiledFn enc, CUtensorMap* tm, CUtensorMapDataType type, int rank, const void* ptr, const cuuint64_t* dims,
                const cuuint64_t* strides, const cuuint32_t* box, CUtensorMapSwizzle swizzle, CUtensorMapL2promotion promote) {
    const cuuint32_t one[3] = {1, 1, 1};
    return enc(tm, type, (cuuint32_t)rank, const_cast<void*>(ptr), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
               promote, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// packed codes [count][rows][K/2]: boxes of 128 bytes x box_rows rows
bool code_map(EncodeTiledFn enc, CUtensorMap* tm, const uint8_t* codes, int K, int64_t rows, int count, int box_rows) {
    const cuuint64_t dims[3] = {(cuuint64_t)(K / 2), (cuuint64_t)rows, (cuuint64_t)count};
    const cuuint64_t strides[2] = {(cuuint64_t)(K / 2), (cuuint64_t)(K / 2) * (cuuint64_t)rows};
    const cuuint32_t box[3] = {128, (cuuint32_t)box_rows, 1};
    return encode_map(enc, tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, count ? 3 : 2, codes, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}
// tiled scale bytes as [row tiles][k tiles][128 x u32]: boxes of 2 k tiles x box_tiles row tiles
bool scale_map(EncodeTiledFn enc, CUtensorMap* tm, const uint8_t* scales, int K, int64_t row_tiles, int box_tiles) {
    const cuuint64_t k_tiles = (cuuint64_t)((K + 127) / 128);
    const cuuint64_t dims[3] = {128, k_tiles, (cuuint64_t)row_tiles}, strides[2] = {512, k_tiles * 512};
    const cuuint32_t box[3] = {128, 2, (cuuint32_t)box_tiles};
    return encode_map(enc, tm, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, scales, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE,
                      CU_TENSOR_MAP_L2_PROMOTION_NONE);
}

struct LinearLaunch {
    const uint8_t *a_codes, *a_scales, *b_codes, *b_scales;
    int K, count;                      // count: weights (1 for the dense call)
    kq::LinearProblem p;
};

template <bool GLU>
kq_status_t launch_pair(LinearLaunch& l, EncodeTiledFn enc, int sms, cudaStream_t st) {
    static DeviceOnce attr_done;
    if (attr_done.needed()) {
        if (cudaFuncSetAttribute(kq::linear_mxfp4_pair<GLU>, cudaFuncAttributeMaxDynamicSharedMemorySize, kq::kLinDynBytes) != cudaSuccess) {
            (void)cudaGetLastError();
            return KQ_ERR_CUDA;
        }
        attr_done.done();
    }
    kq::LinearProblem& p = l.p;
    CUtensorMap ta, tb, tsa, tsb;
    const int64_t a_tiles = ((int64_t)p.M + 127) / 128;
    if (!code_map(enc, &ta, l.a_codes, l.K, p.M, 0, 128) || !code_map(enc, &tb, l.b_codes, l.K, p.R, l.count, kq::kLinN / 2) ||
        !scale_map(enc, &tsa, l.a_scales, l.K, a_tiles, 1) || !scale_map(enc, &tsb, l.b_scales, l.K, (int64_t)p.sf_row_tiles * l.count, 2))
        return KQ_ERR_CUDA;
    p.tiles_m = (p.M + 255) / 256;
    p.tiles_n = (p.R + kq::kLinN - 1) / kq::kLinN;
    // an upper bound of the items: every boundary between two groups can add one row tile
    const int64_t items = ((int64_t)p.tiles_m + (p.experts ? l.count - 1 : 0)) * p.tiles_n;
    const int pairs = (int)(items < sms / 2 ? items : sms / 2);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    launch_config(&cfg, attr, dim3((unsigned)(2 * pairs)), dim3(kq::kLinThreads), kq::kLinDynBytes, 2, st);
    return launch(cfg, kq::linear_mxfp4_pair<GLU>, ta, tb, tsa, tsb, p);
}

template <bool GLU, int TB>
kq_status_t launch_narrow(LinearLaunch& l, EncodeTiledFn enc, int sms, cudaStream_t st) {
    using L = kq::NarrowSmem<TB>;
    static DeviceOnce attr_done;
    if (attr_done.needed()) {
        if (cudaFuncSetAttribute(kq::linear_mxfp4_narrow<GLU, TB>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynBytes) != cudaSuccess) {
            (void)cudaGetLastError();
            return KQ_ERR_CUDA;
        }
        attr_done.done();
    }
    kq::LinearProblem& p = l.p;
    CUtensorMap tw, ta, tsw, tsa;
    const int64_t a_tiles = ((int64_t)p.M + 127) / 128;
    if (!code_map(enc, &tw, l.b_codes, l.K, p.R, l.count, 128) || !code_map(enc, &ta, l.a_codes, l.K, p.M, 0, TB == 128 ? 32 : TB) ||
        !scale_map(enc, &tsw, l.b_scales, l.K, (int64_t)p.sf_row_tiles * l.count, 1) || !scale_map(enc, &tsa, l.a_scales, l.K, a_tiles, 1))
        return KQ_ERR_CUDA;
    p.tiles_m = (int)a_tiles;
    p.tiles_n = (p.R + 127) / 128;
    const int64_t live = p.experts ? (l.count < p.M ? l.count : p.M) : 1;         // experts that can have rows
    const int64_t items = (a_tiles + live - 1) * p.tiles_n;
    // K split: doubled while the CTAs fit the SMs and keep two stages each.  A cluster of four or eight needs as many free SMs of one
    // GPC (16 to 20 of them), so fewer SMs can be filled with those: 7/8, and 16 less (18 clusters of eight ran in two waves: 14.4 us
    // instead of the 11 of 18 clusters of four).
    const int room[3] = {sms, sms * 7 / 8, sms * 7 / 8 - 16};                     // SMs for clusters of 2, 4, 8
    int splits = 1;
    for (int i = 0; i < 3 && items * splits * 2 <= room[i] && p.k_blocks >= 4 * splits; ++i) splits *= 2;
    const int64_t ctas = items * splits;
    const int grid = (int)(ctas < sms ? ctas : sms);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    launch_config(&cfg, attr, dim3((unsigned)grid), dim3(kq::kNarrowThreads), L::kDynBytes, splits, st);
    return launch(cfg, kq::linear_mxfp4_narrow<GLU, TB>, tw, ta, tsw, tsa, p, splits);
}

kq_status_t run_linear(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales,
                       const int32_t* offsets, int experts, int64_t M, int N, int K, const kq_epilogue_t* epilogue, void* out,
                       kq_dtype_t out_dtype, int64_t ld_out, void* stream) {
    kq_epilogue_t e;
    if (epilogue) e = *epilogue; else kroquant_epilogue_default(&e);
    if (!b_codes || !b_scales || (M > 0 && (!a_codes || !a_scales || !out))) return KQ_ERR_NULL;
    if (M < 0 || M > (1 << 24) || N <= 0 || N > (1 << 26) || K <= 0 || K % 32 || ld_out < N) return KQ_ERR_SHAPE;
    if (e.activation < KQ_ACT_NONE || e.activation > KQ_ACT_GELU_TANH || (e.glu | 1) != 1 || !known_type(out_dtype) ||
        (e.bias && !known_type(e.bias_dtype)) || (e.gate && !known_type(e.gate_dtype)) || (e.residual && !known_type(e.residual_dtype)))
        return KQ_ERR_UNSUPPORTED;
    if ((e.gate && (e.rows_per_gate < 1 || (e.gate_stride != 0 && e.gate_stride < N))) || (e.residual && e.ld_residual < N)) return KQ_ERR_SHAPE;
    if (!aligned16(a_codes) || !aligned16(a_scales) || !aligned16(b_codes) || !aligned16(b_scales) || !element_aligned(out, out_dtype) ||
        (e.bias && !element_aligned(e.bias, e.bias_dtype)) || (e.gate && !element_aligned(e.gate, e.gate_dtype)) ||
        (e.residual && !element_aligned(e.residual, e.residual_dtype)) || reinterpret_cast<uintptr_t>(e.row_scale) % 4)
        return KQ_ERR_ALIGN;
    const int64_t R = e.glu ? (int64_t)64 * ((N + 31) / 32) : N;
    const int count = experts ? experts : 1;
    if ((M / 128 + 1 + count) * ((R + 127) / 128) >= ((int64_t)1 << 31) || ((R + 127) / 128) * count >= ((int64_t)1 << 31)) return KQ_ERR_SHAPE;
    if (M == 0) return KQ_OK;
    EncodeTiledFn enc = get_encode_tiled();
    const int sms = sm_count();
    if (!enc || sms <= 0) return KQ_ERR_CUDA;
    LinearLaunch l;
    l.a_codes = a_codes; l.a_scales = a_scales; l.b_codes = b_codes; l.b_scales = b_scales;
    l.K = K;
    l.count = count;
    kq::LinearProblem& p = l.p;
    p = {};
    p.M = (int)M;
    p.R = (int)R;
    p.k_blocks = (K + 255) / 256;
    p.sf_row_tiles = (int)((R + 127) / 128);
    p.experts = experts;
    p.offsets = offsets;
    kq::LinearEpilogue& ep = p.epi;
    ep.N = N;
    ep.act = e.activation;
    ep.bias = {e.bias, experts ? R : 0, e.bias_dtype};
    ep.gate = {e.gate, e.gate_stride, e.gate_dtype};
    // (one gate row for all is one gate row, whatever rows_per_gate says: a warp then reads it once instead of a lane each for its row)
    ep.rows_per_gate = !e.gate || !e.gate_stride || e.rows_per_gate > M ? (int)M : (int)e.rows_per_gate;
    ep.row_scale = e.row_scale;
    ep.residual = e.residual; ep.residual_type = e.residual_dtype; ep.ld_residual = e.ld_residual; ep.residual_scale = e.residual_scale;
    ep.out = out; ep.out_type = out_dtype; ep.ld_out = ld_out;
    ep.vec = rows_aligned(out, ld_out, out_dtype, 16) && rows_aligned(e.residual, e.ld_residual, e.residual_dtype, 16);
    ep.wide = rows_aligned(out, ld_out, out_dtype, 32);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    // Few rows per weight: the weight is the wide operand and is what is read.  Narrow against pair kernel, us: dense N x K = 4096 x
    // 4096 8.3 / 11.6 (1 row), 9.0 / 11.4 (32), 11.0 / 11.7 (64), 15.5 / 12.7 (128); 12288 x 2240 7.3 / 11.9, 11.7 / 10.7 (32), 16.8 / 11.1;
    // 8 gated experts of 4096 x 4096 29 / 44 (4 rows each), 33 / 41 (32), 40 / 46 (64), 58 / 52 (128); 32 of 1024 x 2048 16 / 22,
    // 26 / 25 (32), 35 / 30 (64).  The rule goes by rows per weight alone, between these: it gives away 1 us at 12288 x 2240 with 32
    // rows and 6 us with 64 rows for each of the 8 experts.  It takes the mean over the experts (the sizes are on the device): all 2560
    // rows on one of 64 experts of 1024 x 2048 take 29 us, spread evenly 34.
    const bool narrow = M <= (experts ? 40 : 32) * (int64_t)count;
    if (!narrow) return e.glu ? launch_pair<true>(l, enc, sms, st) : launch_pair<false>(l, enc, sms, st);
    if (M <= 32) return e.glu ? launch_narrow<true, 32>(l, enc, sms, st) : launch_narrow<false, 32>(l, enc, sms, st);
    if (M <= 64) return e.glu ? launch_narrow<true, 64>(l, enc, sms, st) : launch_narrow<false, 64>(l, enc, sms, st);
    return e.glu ? launch_narrow<true, 128>(l, enc, sms, st) : launch_narrow<false, 128>(l, enc, sms, st);
}

// ---- norms ------------------------------------------------------------------------------------------

struct NormShape {
    int threads, rows;          // block: threads of a row, rows of a CTA
    int vpt;                    // 8-channel groups per thread
};
// Forward: one warp per row while a lane's share is at most four groups (d <= 1024), else one CTA per row with two.
NormShape forward_shape(int d) {
    const int groups = (d + 7) / 8;
    if (groups <= 128) return {32, 8, groups <= 32 ? 1 : (groups <= 64 ? 2 : 4)};
    return {((groups + 1) / 2 + 31) / 32 * 32, 1, 2};
}
// Backward: one warp per row for d <= 512, else one group per thread in one CTA per row, above d = 4608 in a cluster of two or four.
NormShape backward_shape(int d, int* cluster) {
    const int groups = (d + 7) / 8;
    *cluster = 1;
    if (groups <= 64) return {32, kq::kNormWarps, groups <= 32 ? 1 : 2};
    while (groups > *cluster * kq::kNormThreads) *cluster *= 2;
    return {((groups + *cluster - 1) / *cluster + 63) / 64 * 64, 1, 1};        // an even number of warps
}
bool vec_row(const void* p, int64_t ld, int type) { return rows_aligned(p, ld, type, 16); }

kq_status_t check_norm(const kq_norm_args_t& a, bool backward) {
    if (a.rows < 0 || a.d <= 0 || a.d > kq::kNormMaxD || a.rows_per_batch < 1 || a.rows > ((int64_t)1 << 31) - 1) return KQ_ERR_SHAPE;
    if (a.norm < KQ_NORM_NONE || a.norm > KQ_NORM_LAYER || a.post_norm < KQ_NORM_NONE || a.post_norm > KQ_NORM_LAYER ||
        !known_type(a.stream_dtype) || !known_type(a.branch_dtype) || !known_type(a.vec_dtype) ||
        (a.stream_dtype != a.branch_dtype && a.stream_dtype != KQ_OUT_F32) || (a.post_weight && a.post_norm == KQ_NORM_NONE) ||
        ((a.weight || a.scale || a.shift) && a.norm == KQ_NORM_NONE))
        return KQ_ERR_UNSUPPORTED;
    const int s = a.stream_dtype, b = a.branch_dtype, v = a.vec_dtype;
    struct { const void* p; int64_t ld; int type; } rows[] = {{a.x, a.ld_x, s}, {a.y, a.ld_y, b}, {a.h, a.ld_h, s}, {a.n, a.ld_n, b},
                                                             {a.dn, a.ld_dn, b}, {a.dh, a.ld_dh, s}, {a.dx, a.ld_dx, s}, {a.dy, a.ld_dy, b}};
    const bool used[] = {!backward, true, true, !backward, backward, backward, backward, backward};
    for (int i = 0; i < 8; ++i)
        if (used[i] && rows[i].p) {
            if (rows[i].ld < a.d) return KQ_ERR_SHAPE;
            if (!element_aligned(rows[i].p, rows[i].type)) return KQ_ERR_ALIGN;
        }
    const void* vecs[] = {a.gate, a.post_weight, a.weight, a.scale, a.shift};
    const int64_t strides[] = {a.gate_stride, 0, 0, a.scale_stride, a.shift_stride};
    for (int i = 0; i < 5; ++i) {
        if (vecs[i] && !element_aligned(vecs[i], v)) return KQ_ERR_ALIGN;
        if (strides[i] != 0 && strides[i] < a.d) return KQ_ERR_SHAPE;
    }
    return KQ_OK;
}
// Rows of a batch, never more than there are rows (the caller may say "all of them" with any large number; rows >= 1).  Vectors that
// are all shared make one batch: the boundaries of others would only cost (a flush, a slot of the scratch space and a step of the
// gradients' sum each).
int64_t batch_rows(const kq_norm_args_t& a) {
    if (!a.gate_stride && !a.scale_stride && !a.shift_stride) return a.rows;
    return a.rows_per_batch < a.rows ? a.rows_per_batch : a.rows;
}
bool norm_vectors_vec(const kq_norm_args_t& a) {
    const int v = a.vec_dtype;
    return a.d % 8 == 0 && rows_aligned(a.gate, a.gate_stride, v, 16) && rows_aligned(a.post_weight, 0, v, 16) &&
           rows_aligned(a.weight, 0, v, 16) && rows_aligned(a.scale, a.scale_stride, v, 16) && rows_aligned(a.shift, a.shift_stride, v, 16);
}

constexpr int kSmemPerSm = 228 * 1024, kSmemPerCta = 227 * 1024;

template <typename S, typename Y, int VPT, bool POST>
kq_status_t launch_norm_rows(kq::NormForward& p, int threads, int sms, cudaStream_t st) {
    static DeviceOnce attr_done;
    if (attr_done.needed()) {
        if (cudaFuncSetAttribute(kq::norm_residual_forward_rows<S, Y, VPT, POST>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemPerCta) != cudaSuccess) {
            (void)cudaGetLastError();
            return KQ_ERR_CUDA;
        }
        attr_done.done();
    }
    int per_sm = 1024 / threads;                                     // 64 registers a thread
    if (per_sm > 4) per_sm = 4;
    p.off_y = p.d * (int)sizeof(S);
    p.stage_bytes = p.off_y + (p.y ? p.d * (int)sizeof(Y) : 0);
    auto room = [&]() { return (per_sm == 1 ? kSmemPerCta : kSmemPerSm / per_sm - 1024) - kq::kNormFwdHead; };
    auto params = [&]() { return 4 * p.d * __builtin_popcount((unsigned)p.cache); };
    p.cache = (p.y && p.gate.ptr ? kq::kCacheGate : 0) | (POST && p.post_weight.ptr ? kq::kCachePost : 0) |
              (p.norm != KQ_NORM_NONE && (p.weight.ptr || p.scale.ptr) ? kq::kCacheMul : 0) | (p.norm != KQ_NORM_NONE && p.shift.ptr ? kq::kCacheShift : 0);
    // four rows in flight come before the vectors, those before a second CTA
    while (per_sm > 1 && params() + 4 * p.stage_bytes > room()) --per_sm;
    if (params() + 4 * p.stage_bytes > room()) p.cache = 0;
    int stages = (room() - params()) / p.stage_bytes;
    p.stages = stages > 8 ? 8 : stages;
    const int64_t most = (int64_t)sms * per_sm;
    p.rows_per_worker = (p.rows + most - 1) / most;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    launch_config(&cfg, attr, dim3((unsigned)((p.rows + p.rows_per_worker - 1) / p.rows_per_worker)), dim3((unsigned)threads),
                  (size_t)(kq::kNormFwdHead + params() + p.stages * p.stage_bytes), 1, st);
    return launch(cfg, kq::norm_residual_forward_rows<S, Y, VPT, POST>, p);
}

template <typename S, typename Y>
kq_status_t launch_norm_forward(kq::NormForward& p, cudaStream_t st) {
    const int sms = sm_count(), groups = p.d / 8;
    if (sms <= 0) return KQ_ERR_CUDA;
    // Rows of more than 1024 channels, two or more per SM: persistent CTAs.  Few rows: a CTA each, which has the shorter way (one token:
    // 3.2 us).  CTA per row against persistent, us, with 148, 296, 1184, 2368 rows: d = 1152 4.3 / 3.9, 4.5 / 4.2, 5.3 / 4.9, 10.3 / 7.3;
    // 2240 4.5 / 4.2, 4.6 / 4.5, 10.7 / 8.0, 15.9 / 14.1; 5600 with a 32-bit stream and two norms 5.1 / 5.6, 7.0 / 6.2, 24.0 / 21.2, 43.1 / 36.4.
    // Two stages need two rows in 225 KB.
    if (p.vec && p.d > 1024 && p.rows >= 2 * (int64_t)sms && 2 * p.d * (int)(sizeof(S) + (p.y ? sizeof(Y) : 0)) <= kSmemPerCta - kq::kNormFwdHead) {
        const bool post = p.y && p.post != KQ_NORM_NONE;
        if (groups <= 1024) {
            const int threads = (groups + 31) / 32 * 32;
            return post ? launch_norm_rows<S, Y, 1, true>(p, threads, sms, st) : launch_norm_rows<S, Y, 1, false>(p, threads, sms, st);
        }
        const int threads = ((groups + 1) / 2 + 31) / 32 * 32;
        return post ? launch_norm_rows<S, Y, 2, true>(p, threads, sms, st) : launch_norm_rows<S, Y, 2, false>(p, threads, sms, st);
    }
    const NormShape s = forward_shape(p.d);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    launch_config(&cfg, attr, dim3((unsigned)((p.rows + s.rows - 1) / s.rows)), dim3((unsigned)s.threads, (unsigned)s.rows), 0, 1, st);
    switch (s.vpt) {
        case 1: return launch(cfg, kq::norm_residual_forward<S, Y, 1>, p);
        case 2: return launch(cfg, kq::norm_residual_forward<S, Y, 2>, p);
        default: return launch(cfg, kq::norm_residual_forward<S, Y, 4>, p);
    }
}

// Workers of the backward pass: as many as run at once, and no more than there are rows; the staged kernel's use of
// shared memory.
struct NormWorkers {
    NormShape shape;
    int64_t workers, rows_per_worker, batches;
    int cluster, smem;          // CTAs of a worker and dynamic shared memory (staged kernel)
};
NormWorkers norm_workers(const kq_norm_args_t& a, int sms, kq::NormBackward* p) {
    NormWorkers w = {};
    w.shape = backward_shape(a.d, &w.cluster);
    int per_sm = w.shape.vpt == 1 ? 2 : 1;                           // narrow rows: 110 to 183 registers
    w.smem = kq::kNormWarps * 3 * a.d * (int)sizeof(float);          // at most 48 KB
    if (w.shape.rows == 1) {
        per_sm = 20 * 32 / w.shape.threads;                          // 96 registers: five warps per scheduler
        const int columns = ((a.d + 7) / 8 + w.cluster - 1) / w.cluster * 8;      // of a CTA; the last one's may be fewer
        const int ss = type_size(a.stream_dtype), sb = type_size(a.branch_dtype);
        const bool post = a.y && a.post_norm != KQ_NORM_NONE, dn = a.norm != KQ_NORM_NONE;
        // the second phase's values take the place of h and dh: both rows must exist (a 32-bit stream has the room in h's)
        const int rows_s = a.dh || (post && ss == 2) ? 2 : 1;
        const int off_dh = columns * ss, off_dn = off_dh * rows_s;
        const int off_y = off_dn + (dn ? columns * sb : 0), stage = off_y + (a.y ? columns * sb : 0);
        const int cache_m = dn && (a.weight || a.scale) ? 1 : 0, cache_gate = a.y && a.gate ? 1 : 0, cache_post = post && a.post_weight ? 1 : 0;
        const int params = 4 * columns * (cache_m + cache_gate + cache_post);
        auto room = [&]() { return (per_sm == 1 ? kSmemPerCta : kSmemPerSm / per_sm - 1024) - kq::kNormHeadBytes; };
        // two stages at least: 4608 columns of four 32-bit rows, twice, and three vectors are 198 KB
        while (per_sm > 1 && params + 2 * stage > room()) --per_sm;
        int stages = (room() - params) / stage;
        stages = stages > kq::kNormStageMax ? kq::kNormStageMax : stages;
        w.smem = kq::kNormHeadBytes + params + stages * stage;
        if (p) {
            p->cluster = w.cluster; p->columns = columns; p->stages = stages; p->stage_bytes = stage;
            p->off_dh = off_dh; p->off_dn = off_dn; p->off_y = off_y;
            p->cache_m = cache_m; p->cache_gate = cache_gate; p->cache_post = cache_post;
        }
    }
    // a cluster of four needs four SMs of one GPC: 32 of them fit (8 GPCs of 16 to 20 SMs), not 37
    int64_t most = (int64_t)(sms > 3 ? sms : 4) * per_sm / w.cluster;
    if (w.cluster > 2) most = most * 7 / 8;
    w.rows_per_worker = (a.rows + most - 1) / most;
    if (w.rows_per_worker < 1) w.rows_per_worker = 1;
    w.workers = (a.rows + w.rows_per_worker - 1) / w.rows_per_worker;
    w.batches = (a.rows + batch_rows(a) - 1) / batch_rows(a);
    return w;
}
bool wants_vector_gradients(const kq_norm_args_t& a) { return a.dgate || a.dpost_weight || a.dweight || a.dscale || a.dshift; }

template <typename S, typename Y, bool POST, bool VEC>
kq_status_t launch_norm_staged(const kq::NormBackward& p, const NormWorkers& w, cudaStream_t st) {
    static DeviceOnce attr_done;
    if (attr_done.needed()) {
        if (cudaFuncSetAttribute(kq::norm_residual_backward<S, Y, POST, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemPerCta) != cudaSuccess) {
            (void)cudaGetLastError();
            return KQ_ERR_CUDA;
        }
        attr_done.done();
    }
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    launch_config(&cfg, attr, dim3((unsigned)(w.workers * w.cluster)), dim3((unsigned)w.shape.threads), (size_t)w.smem, w.cluster, st);
    return launch(cfg, kq::norm_residual_backward<S, Y, POST, VEC>, p);
}
template <typename S, typename Y>
kq_status_t launch_norm_backward(const kq::NormBackward& p, const NormWorkers& w, cudaStream_t st) {
    if (w.shape.rows == 1) {
        if (p.y && p.post != KQ_NORM_NONE) return p.vec ? launch_norm_staged<S, Y, true, true>(p, w, st) : launch_norm_staged<S, Y, true, false>(p, w, st);
        return p.vec ? launch_norm_staged<S, Y, false, true>(p, w, st) : launch_norm_staged<S, Y, false, false>(p, w, st);
    }
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    launch_config(&cfg, attr, dim3((unsigned)w.workers), dim3((unsigned)w.shape.threads, (unsigned)w.shape.rows), (size_t)w.smem, 1, st);
    return w.shape.vpt == 1 ? launch(cfg, kq::norm_residual_backward_warp<S, Y, 1>, p) : launch(cfg, kq::norm_residual_backward_warp<S, Y, 2>, p);
}

}  // namespace

extern "C" {

void kroquant_epilogue_default(kq_epilogue_t* e) {
    if (!e) return;
    std::memset(e, 0, sizeof(*e));
    e->rows_per_gate = 1;
    e->residual_scale = 1.0f;
}

kq_status_t kroquant_linear_mxfp4(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales,
                                  int64_t M, int N, int K, const kq_epilogue_t* epilogue, void* out, kq_dtype_t out_dtype, int64_t ld_out,
                                  void* stream) {
    return run_linear(a_codes, a_scales, b_codes, b_scales, nullptr, 0, M, N, K, epilogue, out, out_dtype, ld_out, stream);
}

kq_status_t kroquant_linear_mxfp4_grouped(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales,
                                          const int32_t* offsets, int experts, int64_t M, int N, int K, const kq_epilogue_t* epilogue,
                                          void* out, kq_dtype_t out_dtype, int64_t ld_out, void* stream) {
    if (!offsets) return KQ_ERR_NULL;
    if (experts < 1 || experts > kq::kMaxExperts) return KQ_ERR_SHAPE;
    if (reinterpret_cast<uintptr_t>(offsets) % 4) return KQ_ERR_ALIGN;
    return run_linear(a_codes, a_scales, b_codes, b_scales, offsets, experts, M, N, K, epilogue, out, out_dtype, ld_out, stream);
}

void kroquant_norm_args_default(kq_norm_args_t* a) {
    if (!a) return;
    std::memset(a, 0, sizeof(*a));
    a->residual_scale = 1.0f;
    a->eps = 1e-6f;
    a->rows_per_batch = 1;
}

kq_status_t kroquant_norm_residual(const kq_norm_args_t* args, void* stream) {
    if (!args) return KQ_ERR_NULL;
    const kq_norm_args_t& a = *args;
    const kq_status_t rc = check_norm(a, false);
    if (rc != KQ_OK) return rc;
    if (a.rows == 0) return KQ_OK;
    if (!a.x || (a.norm != KQ_NORM_NONE && !a.n) || (a.norm == KQ_NORM_NONE && !a.h)) return KQ_ERR_NULL;
    kq::NormForward p = {};
    p.rows = a.rows; p.d = a.d; p.rows_per_batch = batch_rows(a);
    p.x = a.x; p.ld_x = a.ld_x; p.y = a.y; p.ld_y = a.ld_y; p.h = a.h; p.ld_h = a.ld_h; p.n = a.n; p.ld_n = a.ld_n;
    p.gate = {a.gate, a.gate_stride, a.vec_dtype};
    p.post_weight = {a.post_weight, 0, a.vec_dtype};
    p.weight = {a.weight, 0, a.vec_dtype};
    p.scale = {a.scale, a.scale_stride, a.vec_dtype};
    p.shift = {a.shift, a.shift_stride, a.vec_dtype};
    p.alpha = a.residual_scale; p.eps = a.eps; p.norm = a.norm; p.post = a.post_norm;
    p.vec = norm_vectors_vec(a) && vec_row(a.x, a.ld_x, a.stream_dtype) && vec_row(a.y, a.ld_y, a.branch_dtype) &&
            vec_row(a.h, a.ld_h, a.stream_dtype) && vec_row(a.n, a.ld_n, a.branch_dtype);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    if (a.stream_dtype == KQ_OUT_BF16) return launch_norm_forward<__nv_bfloat16, __nv_bfloat16>(p, st);
    if (a.stream_dtype == KQ_OUT_FP16) return launch_norm_forward<__half, __half>(p, st);
    if (a.branch_dtype == KQ_OUT_BF16) return launch_norm_forward<float, __nv_bfloat16>(p, st);
    if (a.branch_dtype == KQ_OUT_FP16) return launch_norm_forward<float, __half>(p, st);
    return launch_norm_forward<float, float>(p, st);
}

int64_t kroquant_norm_residual_grad_scratch_bytes(const kq_norm_args_t* args) {
    if (!args || check_norm(*args, true) != KQ_OK || args->rows == 0 || !wants_vector_gradients(*args)) return 0;
    const NormWorkers w = norm_workers(*args, sm_count(), nullptr);
    return (w.workers + w.batches - 1) * 3 * args->d * (int64_t)sizeof(float);
}

kq_status_t kroquant_norm_residual_grad(const kq_norm_args_t* args, void* scratch, int64_t scratch_bytes, void* stream) {
    if (!args) return KQ_ERR_NULL;
    const kq_norm_args_t& a = *args;
    kq_status_t rc = check_norm(a, true);
    if (rc != KQ_OK) return rc;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool vectors = wants_vector_gradients(a);
    if (a.rows == 0) {
        float* zero[] = {a.gate_stride ? nullptr : a.dgate, a.dpost_weight, a.dweight, a.scale_stride ? nullptr : a.dscale,
                         a.shift_stride ? nullptr : a.dshift};
        for (float* z : zero)
            if (z && cudaMemsetAsync(z, 0, (size_t)a.d * sizeof(float), st) != cudaSuccess) {
                (void)cudaGetLastError();
                return KQ_ERR_CUDA;
            }
        return KQ_OK;
    }
    if (!a.h || !a.dx || (a.norm != KQ_NORM_NONE && !a.dn) || (a.y && !a.dy)) return KQ_ERR_NULL;
    const int sms = sm_count();
    if (sms <= 0) return KQ_ERR_CUDA;
    kq::NormBackward p = {};
    const NormWorkers w = norm_workers(a, sms, &p);
    if (vectors) {
        if (!scratch) return KQ_ERR_NULL;
        if (!aligned16(scratch)) return KQ_ERR_ALIGN;
        if (scratch_bytes < kroquant_norm_residual_grad_scratch_bytes(args)) return KQ_ERR_SHAPE;
    }
    p.rows = a.rows; p.d = a.d; p.rows_per_batch = batch_rows(a); p.rows_per_worker = w.rows_per_worker;
    p.dn = a.norm == KQ_NORM_NONE ? nullptr : a.dn; p.ld_dn = a.ld_dn; p.dh = a.dh; p.ld_dh = a.ld_dh;
    p.h = a.h; p.ld_h = a.ld_h; p.y = a.y; p.ld_y = a.ld_y; p.dx = a.dx; p.ld_dx = a.ld_dx; p.dy = a.dy; p.ld_dy = a.ld_dy;
    p.gate = {a.gate, a.gate_stride, a.vec_dtype};
    p.post_weight = {a.post_weight, 0, a.vec_dtype};
    p.weight = {a.weight, 0, a.vec_dtype};
    p.scale = {a.scale, a.scale_stride, a.vec_dtype};
    p.alpha = a.residual_scale; p.eps = a.eps; p.norm = a.norm; p.post = a.post_norm;
    p.vec = norm_vectors_vec(a) && vec_row(a.h, a.ld_h, a.stream_dtype) && vec_row(a.y, a.ld_y, a.branch_dtype) &&
            vec_row(p.dn, a.ld_dn, a.branch_dtype) && vec_row(a.dh, a.ld_dh, a.stream_dtype) && vec_row(a.dx, a.ld_dx, a.stream_dtype) &&
            vec_row(a.dy, a.ld_dy, a.branch_dtype);
    p.partial = vectors ? static_cast<float*>(scratch) : nullptr;
    if (a.stream_dtype == KQ_OUT_BF16) rc = launch_norm_backward<__nv_bfloat16, __nv_bfloat16>(p, w, st);
    else if (a.stream_dtype == KQ_OUT_FP16) rc = launch_norm_backward<__half, __half>(p, w, st);
    else if (a.branch_dtype == KQ_OUT_BF16) rc = launch_norm_backward<float, __nv_bfloat16>(p, w, st);
    else if (a.branch_dtype == KQ_OUT_FP16) rc = launch_norm_backward<float, __half>(p, w, st);
    else rc = launch_norm_backward<float, float>(p, w, st);
    if (rc != KQ_OK || !vectors) return rc;
    kq::NormVecGrads g = {};
    g.rows = a.rows; g.d = a.d; g.rows_per_batch = p.rows_per_batch; g.rows_per_worker = w.rows_per_worker; g.batches = w.batches;
    g.partial = p.partial;
    g.gate = p.gate; g.post_weight = p.post_weight; g.weight = p.weight; g.scale = p.scale;
    g.dgate = a.dgate; g.dscale = a.dscale; g.dshift = a.dshift; g.dweight = a.dweight; g.dpost_weight = a.dpost_weight;
    // gradients of batched vectors are stored [batches][d]
    g.dgate_stride = a.gate_stride ? a.d : 0;
    g.dscale_stride = a.scale_stride ? a.d : 0;
    g.dshift_stride = a.shift_stride ? a.d : 0;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    launch_config(&cfg, attr, dim3((unsigned)((a.d + 31) / 32)), dim3(32, kq::kSlotLanes), 0, 1, st);
    return launch(cfg, kq::norm_vector_gradients, g);
}

}  // extern "C"
