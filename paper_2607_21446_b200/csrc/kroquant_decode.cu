// Host side of the operators of one step over new tokens (contract: include/kroquant.h): rotary positions, the paged cache and the
// attention over it.  Argument checks, variant rules, launches; nothing here allocates, synchronizes or throws.
#include <cstring>

#include "kq_host.cuh"

#include "kq_cache_attention.cuh"

namespace {

kq::FastDiv fast_div(uint32_t d) {       // 1 <= d < 2^31
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return {d, (uint32_t)(((1ull << 32) * ((1ull << s) - d)) / d + 1), s};
}
bool sixteen_bit(int t) { return t == KQ_OUT_BF16 || t == KQ_OUT_FP16; }

template <typename Kernel>
kq_status_t allow_shared(DeviceOnce& once, Kernel* kernel, int bytes) {
    if (bytes <= 48 * 1024 || !once.needed()) return KQ_OK;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return KQ_ERR_CUDA;
    }
    once.done();
    return KQ_OK;
}

// ---- rotary ------------------------------------------------------------------------------------------

template <typename T, int E, bool HALF>
kq_status_t launch_rotary(kq::RotaryProblem& p, int sms, cudaStream_t st) {
    const int units = HALF ? (E == 1 ? p.head_dim - p.pairs : (p.head_dim - p.pairs) / E) : (E == 1 ? (p.head_dim + 1) / 2 : p.head_dim / E);
    int rows = 192 / units;                                          // at a time
    if (rows < 1) rows = 1;
    int heads = p.t[0].heads + (p.tensors > 1 ? p.t[1].heads : 0);
    // Tokens of a CTA: all CTAs run at once (five on an SM), since a second wave that is not full costs as much as the first.  One token of
    // many heads goes over several CTAs, each of which forms the token's sines again.
    int64_t per_cta = (p.rows + 5 * sms - 1) / (5 * sms);
    if (per_cta * p.pairs > 2048) per_cta = 2048 / p.pairs;          // 16 KB
    if (per_cta * heads > (1 << 24)) per_cta = (1 << 24) / heads;    // (rows are counted in 32 bits)
    if (per_cta < 1) per_cta = 1;
    p.tokens_per_cta = (int)per_cta;
    const int64_t tiles = (p.rows + per_cta - 1) / per_cta, taken = heads * per_cta;
    const int64_t spare = tiles < sms ? (2 * sms + tiles - 1) / tiles : 1, runs = (taken + rows - 1) / rows;
    p.head_parts = (int)(spare < runs ? spare : runs);
    if (rows > taken) rows = (int)taken;
    const int smem = (units * rows * kq::rotary_slot_bytes<T, E, HALF>() + 15) / 16 * 16 + (int)per_cta * kq::rotary_pitch(p.pairs) * (int)sizeof(float2);
    static DeviceOnce attr_done;
    const kq_status_t rc = allow_shared(attr_done, kq::rotary_kernel<T, E, HALF>, 100 * 1024);
    if (rc != KQ_OK) return rc;
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    launch_config(&cfg, attr, dim3((unsigned)tiles, (unsigned)p.head_parts), dim3((unsigned)units, (unsigned)rows),
                  (size_t)smem, 1, st);
    return launch(cfg, kq::rotary_kernel<T, E, HALF>, p);
}
template <typename T>
kq_status_t launch_rotary_type(kq::RotaryProblem& p, bool half, int bytes, int sms, cudaStream_t st) {
    constexpr int kWide = 16 / sizeof(T), kNarrow = 8 / sizeof(T);
    if (half) {
        if (bytes == 16) return launch_rotary<T, kWide, true>(p, sms, st);
        if (bytes == 8) return launch_rotary<T, kNarrow, true>(p, sms, st);
        return launch_rotary<T, 1, true>(p, sms, st);
    }
    if (bytes == 16) return launch_rotary<T, kWide, false>(p, sms, st);
    if (bytes == 8) return launch_rotary<T, kNarrow, false>(p, sms, st);
    return launch_rotary<T, 1, false>(p, sms, st);
}

// ---- cache -------------------------------------------------------------------------------------------

kq_status_t check_cache(const kq_cache_t& c) {
    if (c.format < KQ_CACHE_16BIT || c.format > KQ_CACHE_MXFP4 || (c.format == KQ_CACHE_16BIT && !sixteen_bit(c.dtype))) return KQ_ERR_UNSUPPORTED;
    if (c.pages < 1 || c.page_size < 1 || c.heads < 1 || c.head_dim < 1 || c.head_dim > 256 || c.pages > ((int64_t)1 << 31) - 1 ||
        (int64_t)c.heads * c.page_size > ((int64_t)1 << 32) - 1 || c.pages > (((int64_t)1 << 32) - 1) / ((int64_t)c.heads * c.page_size))
        return KQ_ERR_SHAPE;
    if (!c.k || !c.v || (c.format != KQ_CACHE_16BIT && (!c.k_scales || !c.v_scales))) return KQ_ERR_NULL;
    if (!aligned16(c.k) || !aligned16(c.v) ||
        (c.format != KQ_CACHE_16BIT && (reinterpret_cast<uintptr_t>(c.k_scales) % 8 || reinterpret_cast<uintptr_t>(c.v_scales) % 8)))
        return KQ_ERR_ALIGN;
    return KQ_OK;
}
kq::CacheRef cache_ref(const kq_cache_t& c) {
    kq::CacheRef r = {};
    r.format = c.format;
    r.pages = c.pages;
    r.page_size = c.page_size;
    r.heads = c.heads;
    r.head_dim = c.head_dim;
    r.blocks = (c.head_dim + 31) / 32;
    r.scale_row = (r.blocks + 3) / 4 * 4;
    r.k = static_cast<uint8_t*>(c.k);
    r.v = static_cast<uint8_t*>(c.v);
    r.k_scales = c.k_scales;
    r.v_scales = c.v_scales;
    r.by_page = fast_div((uint32_t)c.page_size);
    return r;
}

kq_status_t check_rows(const kq_cache_t& c, const kq_cache_rows_t& r, bool write) {
    if (!known_type(r.dtype) || (write && (!sixteen_bit(r.dtype) || (c.format == KQ_CACHE_16BIT && r.dtype != c.dtype)))) return KQ_ERR_UNSUPPORTED;
    if (r.rows < 0 || r.rows > ((int64_t)1 << 31) - 1 || r.sequences < 0 || r.table_width < 0 || r.table_stride < 0 || (!r.offsets && r.rows != r.sequences))
        return KQ_ERR_SHAPE;
    if (r.rows > 0 && r.sequences > 0) {
        if (!r.k || !r.v || (!r.table && r.table_width > 0)) return KQ_ERR_NULL;
        if (!element_aligned(r.k, r.dtype) || !element_aligned(r.v, r.dtype) || reinterpret_cast<uintptr_t>(r.table) % 4 ||
            reinterpret_cast<uintptr_t>(r.offsets) % 4 || reinterpret_cast<uintptr_t>(r.starts) % 4)
            return KQ_ERR_ALIGN;
    }
    return KQ_OK;
}

kq_status_t run_cache(const kq_cache_t* cache, const kq_cache_rows_t* rows, void* stream, bool write) {
    if (!cache || !rows) return KQ_ERR_NULL;
    const kq_cache_t& c = *cache;
    const kq_cache_rows_t& r = *rows;
    kq_status_t rc = check_cache(c);
    if (rc == KQ_OK) rc = check_rows(c, r, write);
    if (rc != KQ_OK || r.rows == 0 || r.sequences == 0) return rc;
    const int sms = sm_count();
    if (sms <= 0) return KQ_ERR_CUDA;
    const kq::CacheRef ref = cache_ref(c);
    kq::CacheRows p = {};
    p.rows = r.rows; p.sequences = r.sequences; p.table = r.table; p.table_stride = r.table_stride; p.table_width = r.table_width;
    p.offsets = r.offsets; p.starts = r.starts;
    p.k = r.k; p.v = r.v; p.k_row = r.k_row_stride; p.k_head = r.k_head_stride; p.v_row = r.v_row_stride; p.v_head = r.v_head_stride;
    const int groups = write ? 2 * ref.blocks : (c.head_dim + 15) / 16;
    if ((int64_t)c.heads * groups > (1 << 30)) return KQ_ERR_SHAPE;
    p.units = c.heads * groups;
    p.by_groups = fast_div((uint32_t)groups);
    // Rows of a CTA: as many as let all CTAs run at once (four of them on an SM: the rows' cells, which the others wait for, are then found
    // once), up to the room for their cells.
    const int across = p.units < kq::kCacheThreads ? p.units : kq::kCacheThreads;
    int at_once = kq::kCacheThreads / across;
    int64_t per_cta = (2 * r.rows + 4 * sms - 1) / (4 * sms);        // (keys and values: two grids of CTAs)
    if (per_cta > kq::kCacheRowsMax) per_cta = kq::kCacheRowsMax;
    if (at_once > per_cta) at_once = (int)per_cta;
    p.rows_per_cta = (int)per_cta;
    auto allows = [&](int bytes) {
        return rows_aligned(r.k, r.k_row_stride, r.dtype, bytes) && rows_aligned(r.k, r.k_head_stride, r.dtype, bytes) &&
               rows_aligned(r.v, r.v_row_stride, r.dtype, bytes) && rows_aligned(r.v, r.v_head_stride, r.dtype, bytes);
    };
    const bool vec = c.head_dim % 8 == 0 && allows(16);
    const int width = !vec ? 0 : (c.head_dim % 16 == 0 && allows(32) ? 32 : 16);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    launch_config(&cfg, attr, dim3((unsigned)((r.rows + per_cta - 1) / per_cta), 2), dim3((unsigned)across, (unsigned)at_once), 0, 1, st);
    if (write) {
        auto go = [&](auto type, auto format) {
            using T = decltype(type);
            constexpr int F = decltype(format)::value;
            return vec ? launch(cfg, kq::cache_write_kernel<T, F, true>, ref, p) : launch(cfg, kq::cache_write_kernel<T, F, false>, ref, p);
        };
        auto by_format = [&](auto type) {
            if (c.format == KQ_CACHE_MXFP4) return go(type, std::integral_constant<int, kq::kCacheFp4>{});
            if (c.format == KQ_CACHE_MXFP8) return go(type, std::integral_constant<int, kq::kCacheFp8>{});
            return go(type, std::integral_constant<int, kq::kCache16>{});
        };
        return r.dtype == KQ_OUT_FP16 ? by_format(__half{}) : by_format(__nv_bfloat16{});
    }
    auto by_format = [&](auto type) {
        using T = decltype(type);
        if (c.format == KQ_CACHE_MXFP4) return launch(cfg, kq::cache_read_kernel<T, kq::kCacheFp4, false>, ref, p, width);
        if (c.format == KQ_CACHE_MXFP8) return launch(cfg, kq::cache_read_kernel<T, kq::kCacheFp8, false>, ref, p, width);
        if (c.dtype == KQ_OUT_FP16) return launch(cfg, kq::cache_read_kernel<T, kq::kCache16, true>, ref, p, width);
        return launch(cfg, kq::cache_read_kernel<T, kq::kCache16, false>, ref, p, width);
    };
    if (r.dtype == KQ_OUT_FP16) return by_format(__half{});
    if (r.dtype == KQ_OUT_BF16) return by_format(__nv_bfloat16{});
    return by_format(float{});
}

// ---- attention ---------------------------------------------------------------------------------------

// How a call is laid out: what the kernel instance fixes and the host can know without the lengths.
struct AttentionPlan {
    int columns;                         // query heads of a pass (NQ)
    int channels;                        // channels of the instance (D)
    int tile;                            // positions of a tile
    int per_sm;
    int64_t items, most_tiles;           // most_tiles: of an item
    int ctas, min_run;
    bool whole;                          // no item is split
    int64_t partial_floats() const { return (int64_t)2 * ctas * (columns * channels + 2 * columns); }
    int64_t scratch_bytes() const { return whole ? 0 : partial_floats() * (int64_t)sizeof(float) + items * (int64_t)sizeof(int2); }
};

template <typename F>
auto with_shape(int format, int dtype, int channels, int columns, F f) {
    auto by_columns = [&](auto fmt, auto d) {
        constexpr int FMT = decltype(fmt)::value, D = decltype(d)::value;
        return columns == 8 ? f(kq::AttnShape<FMT, D, 8>{}, fmt, d, std::integral_constant<int, 8>{})
                            : f(kq::AttnShape<FMT, D, 16>{}, fmt, d, std::integral_constant<int, 16>{});
    };
    auto by_channels = [&](auto fmt) {
        if (channels == 64) return by_columns(fmt, std::integral_constant<int, 64>{});
        if (channels == 128) return by_columns(fmt, std::integral_constant<int, 128>{});
        return by_columns(fmt, std::integral_constant<int, 256>{});
    };
    if (format == KQ_CACHE_MXFP4) return by_channels(std::integral_constant<int, kq::kAttnFp4>{});
    if (format == KQ_CACHE_MXFP8) return by_channels(std::integral_constant<int, kq::kAttnFp8>{});
    if (dtype == KQ_OUT_FP16) return by_channels(std::integral_constant<int, kq::kAttnF16>{});
    return by_channels(std::integral_constant<int, kq::kAttnBf16>{});
}

kq_status_t check_attention(const kq_cache_t& c, const kq_attention_args_t& a) {
    kq_status_t rc = check_cache(c);
    if (rc != KQ_OK) return rc;
    if (!sixteen_bit(a.q_dtype) || !known_type(a.out_dtype) || (c.format == KQ_CACHE_16BIT && a.q_dtype != c.dtype)) return KQ_ERR_UNSUPPORTED;
    if (a.sequences < 0 || a.q_heads < 1 || a.q_heads % c.heads || a.table_width < 0 || a.table_stride < 0 || a.window < 0 ||
        (int64_t)a.table_width * c.page_size > (1 << 30) || (int64_t)a.sequences * a.q_heads > ((int64_t)1 << 31) - 1)
        return KQ_ERR_SHAPE;
    return KQ_OK;
}
AttentionPlan plan_attention(const kq_cache_t& c, const kq_attention_args_t& a, int sms) {
    AttentionPlan p = {};
    const int group = a.q_heads / c.heads;
    p.columns = group <= 8 ? 8 : 16;
    p.channels = c.head_dim <= 64 ? 64 : (c.head_dim <= 128 ? 128 : 256);
    with_shape(c.format, c.dtype, p.channels, p.columns, [&](auto shape, auto, auto, auto) {
        using L = decltype(shape);
        p.tile = L::kTile;
        p.per_sm = L::kPerSm;
        return 0;
    });
    p.items = (int64_t)a.sequences * c.heads * ((group + p.columns - 1) / p.columns);
    int64_t most = (int64_t)a.table_width * c.page_size;
    if (a.window > 0 && most > a.window) most = a.window;
    p.most_tiles = most <= p.tile ? 1 : (most - 1) / p.tile + 1;
    p.min_run = 3;
    p.whole = p.most_tiles <= 8;
    int64_t ctas = (int64_t)sms * p.per_sm;
    const int64_t useful = p.whole ? p.items : (p.items * (p.most_tiles + kq::kLead) + p.min_run - 1) / p.min_run;
    p.ctas = (int)(ctas < useful ? ctas : useful);
    return p;
}

}  // namespace

extern "C" {

void kroquant_rotary_args_default(kq_rotary_args_t* a) {
    if (!a) return;
    std::memset(a, 0, sizeof(*a));
    a->batches = 1;
    a->axes = 1;
}

kq_status_t kroquant_rotary(const kq_rotary_args_t* args, void* stream) {
    if (!args) return KQ_ERR_NULL;
    const kq_rotary_args_t& a = *args;
    if (!known_type(a.dtype) || a.layout < KQ_ROTARY_INTERLEAVED || a.layout > KQ_ROTARY_HALF || (a.inverse | 1) != 1 || (a.positions_f32 | 1) != 1)
        return KQ_ERR_UNSUPPORTED;
    if (a.batches < 0 || a.tokens < 0 || a.head_dim < 1 || a.head_dim > 512 || a.axes < 1 || a.axes > 4) return KQ_ERR_SHAPE;
    if (a.tokens > 0 && a.batches > (((int64_t)1 << 31) - 1) / a.tokens) return KQ_ERR_SHAPE;
    kq::RotaryProblem p = {};
    for (int i = 0; i < 4; ++i) {
        if (i < a.axes) {
            if (a.axis_channels[i] < 0 || a.axis_channels[i] % 2 || a.axis_channels[i] > a.head_dim) return KQ_ERR_SHAPE;
            p.pairs += a.axis_channels[i] / 2;
        }
        p.axis_end[i] = i < a.axes - 1 ? p.pairs : 0x7FFFFFFF;       // (the last axis takes what is left)
    }
    if (2 * p.pairs > a.head_dim || p.pairs < 1) return KQ_ERR_SHAPE;
    const int tensors = a.x[1] || a.out[1] ? 2 : 1;
    int bytes = 16;
    const int64_t far = (int64_t)1 << 31;
    for (int i = 0; i < tensors; ++i) {
        if (a.heads[i] < 1 || a.heads[i] > (1 << 20)) return KQ_ERR_SHAPE;
        const int64_t strides[] = {a.x_token_stride[i], a.x_head_stride[i], a.out_token_stride[i], a.out_head_stride[i]};
        for (int64_t stride : strides)
            if (stride >= far || stride <= -far) return KQ_ERR_SHAPE;
    }
    const int64_t rows = a.batches * a.tokens;
    if (rows == 0) return KQ_OK;
    if (!a.frequencies || !a.positions) return KQ_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(a.frequencies) % 8 || reinterpret_cast<uintptr_t>(a.positions) % 4) return KQ_ERR_ALIGN;
    const int size = type_size(a.dtype);
    for (int i = 0; i < tensors; ++i) {
        if (!a.x[i] || !a.out[i]) return KQ_ERR_NULL;
        if (!element_aligned(a.x[i], a.dtype) || !element_aligned(a.out[i], a.dtype)) return KQ_ERR_ALIGN;
        p.t[i] = {a.x[i], a.out[i], a.x_batch_stride[i], a.out_batch_stride[i], a.heads[i], (int)a.x_token_stride[i], (int)a.x_head_stride[i],
                  (int)a.out_token_stride[i], (int)a.out_head_stride[i], fast_div((uint32_t)a.heads[i])};
        const int64_t strides[] = {a.x_batch_stride[i], a.x_token_stride[i], a.x_head_stride[i], a.out_batch_stride[i], a.out_token_stride[i], a.out_head_stride[i]};
        const int64_t used[] = {a.batches, a.tokens, a.heads[i], a.batches, a.tokens, a.heads[i]};
        for (int width = 16; width >= 8; width /= 2) {
            bool ok = reinterpret_cast<uintptr_t>(a.x[i]) % width == 0 && reinterpret_cast<uintptr_t>(a.out[i]) % width == 0 && a.head_dim * size % width == 0 &&
                      (a.layout == KQ_ROTARY_INTERLEAVED || p.pairs * size % width == 0);
            for (int k = 0; k < 6; ++k) ok = ok && (used[k] <= 1 || strides[k] * size % width == 0);
            if (!ok && bytes >= width) bytes = width / 2;
        }
    }
    const int sms = sm_count();
    if (sms <= 0) return KQ_ERR_CUDA;
    p.tensors = tensors; p.rows = rows; p.tokens = a.tokens; p.head_dim = a.head_dim; p.inverse = a.inverse; p.positions_f32 = a.positions_f32;
    p.frequencies = a.frequencies; p.positions = a.positions; p.pos_batch = a.position_batch_stride; p.pos_token = a.position_token_stride;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool half = a.layout == KQ_ROTARY_HALF;
    if (a.dtype == KQ_OUT_F32) return launch_rotary_type<float>(p, half, bytes, sms, st);
    if (a.dtype == KQ_OUT_FP16) return launch_rotary_type<__half>(p, half, bytes, sms, st);
    return launch_rotary_type<__nv_bfloat16>(p, half, bytes, sms, st);
}

kq_status_t kroquant_cache_write(const kq_cache_t* cache, const kq_cache_rows_t* rows, void* stream) { return run_cache(cache, rows, stream, true); }
kq_status_t kroquant_cache_read(const kq_cache_t* cache, const kq_cache_rows_t* rows, void* stream) { return run_cache(cache, rows, stream, false); }

int64_t kroquant_cache_attention_scratch_bytes(const kq_cache_t* cache, const kq_attention_args_t* args) {
    if (!cache || !args || check_attention(*cache, *args) != KQ_OK || args->sequences == 0) return 0;
    return plan_attention(*cache, *args, sm_count()).scratch_bytes();
}

kq_status_t kroquant_cache_attention(const kq_cache_t* cache, const kq_attention_args_t* args, void* scratch, int64_t scratch_bytes, void* stream) {
    if (!cache || !args) return KQ_ERR_NULL;
    const kq_cache_t& c = *cache;
    const kq_attention_args_t& a = *args;
    const kq_status_t rc = check_attention(c, a);
    if (rc != KQ_OK || a.sequences == 0) return rc;
    if (!a.q || !a.out || !a.lengths || (!a.table && a.table_width > 0)) return KQ_ERR_NULL;
    if (!element_aligned(a.q, a.q_dtype) || !element_aligned(a.out, a.out_dtype) || reinterpret_cast<uintptr_t>(a.table) % 4 ||
        reinterpret_cast<uintptr_t>(a.lengths) % 4 || reinterpret_cast<uintptr_t>(a.lse) % 4)
        return KQ_ERR_ALIGN;
    const int sms = sm_count();
    if (sms <= 0) return KQ_ERR_CUDA;
    const AttentionPlan plan = plan_attention(c, a, sms);
    if (!plan.whole) {
        if (!scratch) return KQ_ERR_NULL;
        if (!aligned16(scratch)) return KQ_ERR_ALIGN;
        if (scratch_bytes < plan.scratch_bytes()) return KQ_ERR_SHAPE;
    }
    kq::AttentionProblem p = {};
    p.c = cache_ref(c);
    p.sequences = a.sequences; p.q_heads = a.q_heads; p.group = a.q_heads / c.heads; p.chunks = (p.group + plan.columns - 1) / plan.columns;
    p.q = a.q; p.q_f16 = a.q_dtype == KQ_OUT_FP16;
    p.q_vec = reinterpret_cast<uintptr_t>(a.q) % 8 == 0 && a.q_row_stride % 4 == 0 && a.q_head_stride % 4 == 0 && c.head_dim % 4 == 0;
    p.q_row = a.q_row_stride; p.q_head = a.q_head_stride;
    p.out = a.out; p.out_type = a.out_dtype; p.out_row = a.out_row_stride; p.out_head = a.out_head_stride;
    p.table = a.table; p.table_stride = a.table_stride; p.table_width = a.table_width; p.lengths = a.lengths; p.window = a.window;
    p.scale_log2e = a.scale * 1.4426950408889634f;
    p.lse = a.lse;
    p.partial = plan.whole ? nullptr : static_cast<float*>(scratch);
    p.parts = plan.whole ? nullptr : reinterpret_cast<int2*>(p.partial + plan.partial_floats());
    p.ctas = plan.ctas;
    p.min_run = plan.min_run;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return with_shape(c.format, c.dtype, plan.channels, plan.columns, [&](auto shape, auto fmt, auto d, auto nq) {
        using L = decltype(shape);
        constexpr int FMT = decltype(fmt)::value, D = decltype(d)::value, NQ = decltype(nq)::value;
        static DeviceOnce attr_done;
        kq_status_t r = allow_shared(attr_done, kq::cache_attention_kernel<FMT, D, NQ>, L::kBytes);
        if (r != KQ_OK) return r;
        cudaLaunchConfig_t cfg;
        cudaLaunchAttribute attr[2];
        launch_config(&cfg, attr, dim3((unsigned)plan.ctas), dim3(kq::kAttnThreads), (size_t)L::kBytes, 1, st);
        r = launch(cfg, kq::cache_attention_kernel<FMT, D, NQ>, p);
        if (r != KQ_OK || plan.whole) return r;
        const unsigned queries = (unsigned)(p.group < NQ ? p.group : NQ);
        launch_config(&cfg, attr, dim3((unsigned)plan.items, queries), dim3(plan.items * queries <= 2 * sms ? kq::kJoinThreads : 256), 0, 1, st);
        return launch(cfg, kq::cache_attention_join<D, NQ>, p);
    });
}

}  // extern "C"
