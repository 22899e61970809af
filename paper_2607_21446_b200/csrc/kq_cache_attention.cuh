// Attention of one new token per sequence over the paged cache, sm_100a:
//     out[s][h] = sum_t w_t v_t / sum_t w_t,    w_t = exp(scale q[s][h] . k_t - m),   m the largest score so far
// One pass over the positions with a running maximum and sum: when m grows, the sum and the accumulated values are scaled down.
//
// The cache is read once (for each 16 query heads of a cache head, where it has more), by 4 warps of a CTA that each take every fourth step of 16 (16-bit) or 32 positions, with rings of their own
// in shared memory (cp.async; no barrier between the warps until the end of a segment).  A warp multiplies with mma.sync, positions
// as the 16 rows of the product and the query heads of one cache head as its 8 (or twice 8) columns:
//     S^T [position][query] = K Q^T,     O^T [channel][query] += V^T P^T.
// So nothing is padded to 128 rows, and codes go from shared memory through the converter into the operand registers, never back.  For V^T P^T
// tcgen05 would want V written to shared memory again in 16 bits, as its scale blocks do not run along the positions; keys in E4M3 could be a
// block-scaled operand as they lie (not built).
// Measured (us, and the time of the bytes at the copy rate): one sequence of 300 in 16 bits 7.1 (0.2; 10.0 under a table with room for 8192, whose
// items may be split), 24 of 341 to 8192 in MXFP8 43.5 (30), one of 131071 in MXFP4 44 (22), 5 with a window of 4096 in 16 bits, 20 heads of 112, 41 (28;
// 32 with the channels that fill the rows up); 8 of 8192 in MXFP8 with 8, 12 and 16 query heads a cache head 35, 46, 46 (21).  The formats of codes are
// bound by instructions (some 750 per 32 positions of a head; converter, extraction of its byte and scale are nearly half of them), 16 bits by memory.
//
// Operand order.  Any order of channels serves K Q^T, and any order of positions P^T as long as both products use the same, so that a
// lane takes what lies together: of K, with j = lane % 4, whole 16-byte chunks of the rows of positions lane / 4 and lane / 4 + 8; of V,
// with g = lane / 4, D/8 consecutive channels of four positions.  P^T is S^T with rows and columns of 8 x 8 blocks exchanged (movmatrix).
// Rows of codes are stored with pairs of chunks exchanged, rows of 16-bit values 16 bytes further apart, so that both kinds of access take
// all banks (an asynchronous copy that puts the halves of 32 bytes apart takes several times as long).
//
// Scales.  A code times 2^(S - 127) would leave fp16, so K is taken relative to the largest scale byte of its position (a factor of the
// score, fp32) and V relative to the largest of its position, which goes into P: p 2^(S_t - R + 9), R the largest S_t so far (a
// running maximum that rescales the accumulator as m does).  Code times 2^(S - S_t + kLift) has at most 4 significant bits and is exact in
// fp16; a block whose scale is 2^-28 (E2M1) or 2^-21 (E4M3) of its position's largest, or less, counts as zero.  The queries of a CTA are
// fp16 times one power of two, or one each where their sizes differ much, so that none costs another its digits: exact for both 16-bit types
// down to values 2^-21 of the query's largest.  P is rounded to fp16: 11 bits, down to 2^-23 of the largest weight where a position's S_t is R, 2^(R - S_t)
// above that where it is less; what is lost below is 2^-34 of the largest value at most.  With 16-bit values, where memory leaves the time, P is
// two terms of their type (16 and 22 bits).  Two terms with codes as well: 3 to 8 % slower (131071 in MXFP4 44 -> 47), the error against 64 bits
// 1.7e-4 -> 3e-7 in float32, and no other in 16 bits (1.7e-3 in bf16 either way, by out's own rounding).
//
// Work.  Tiles (4 steps) of all (sequence, head) items are laid end to end, each item led by kLead tiles' worth of nothing for what
// beginning and ending it costs, and every CTA takes an equal run: ragged batches balance, one long sequence fills the GPU.  An
// item that lies within one CTA is written; the parts of others go to the scratch space (at most two per CTA) and a second
// kernel joins them in order.  Lengths are read on the device.
#pragma once
#include "kq_cache.cuh"

namespace kq {

// The running maximum follows the scores only when one exceeds it by more than kSlack (in powers of two), so that the accumulator is seldom
// rescaled: weights are then up to 2^kSlack, times 2^kPLift below fp16's largest.
constexpr float kSlack = 6;
constexpr int kPLift = 9;

// Queries of a CTA share one power of two unless the largest values of two of them are further apart than 2^kQueryRange.  (A power for each in every
// call: one sequence of 131071 in MXFP4 46 us, with it 45.)
constexpr int kQueryRange = 8;

enum { kAttnBf16 = 0, kAttnF16 = 1, kAttnFp8 = 2, kAttnFp4 = 3 };
constexpr int kAttnWarps = 4;
constexpr int kAttnThreads = 32 * kAttnWarps;

struct AttentionProblem {
    CacheRef c;
    int sequences, q_heads, group, chunks;       // group: query heads of a cache head, taken in `chunks` runs
    const void* q;
    int q_f16, q_vec;                    // q_vec: 8-byte loads of four channels
    int64_t q_row, q_head;
    void* out;
    int out_type;
    int64_t out_row, out_head;
    const int32_t* table;
    int64_t table_stride;
    int table_width;
    const int32_t* lengths;
    int window;
    float scale_log2e;
    float* lse;
    float* partial;                      // [2 per CTA][NQ][D], then [2 per CTA][2][NQ]: maximum, sum.  null: items are taken whole
    int2* parts;                         // of each item: first CTA and number of CTAs that took it; {., 1}: written
    int ctas;                            // of the attention kernel
    int min_run;                         // smallest run of a CTA
};

// What an item costs besides its tiles, in tiles: queries, first copies, joining the warps.  24 sequences of 341 to 8192 positions: 63 us with 0,
// 50 with 1, 49 with 2.
constexpr int kLead = 1;

// Positions of a sequence that its token sees, and their tiles (at least one, so that an empty row is written).
struct VisibleRange { int begin, end; };
__device__ __forceinline__ VisibleRange visible_range(const AttentionProblem& p, int s) {
    const int64_t room = (int64_t)p.table_width * p.c.page_size;
    int n = p.lengths[s];
    n = n < 0 ? 0 : (n > room ? (int)room : n);
    return {p.window > 0 && n > p.window ? n - p.window : 0, n};
}
template <int TN>
__device__ __forceinline__ int tiles_of(const VisibleRange& v) {
    const int n = v.end - v.begin;
    return n <= TN ? 1 : (n - 1) / TN + 1;
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t shared_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes of which the first `size` are copied and the others zero; 4 or 8 bytes, zeros where `exists` does not hold
__device__ __forceinline__ void copy_async_16(uint32_t dst, const uint8_t* src, uint32_t size) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
}
template <int N>
__device__ __forceinline__ void copy_async_small(uint32_t dst, const uint8_t* src, bool exists) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(exists ? N : 0), "n"(N) : "memory");
}

template <int FMT, int D, int NQ>
struct AttnShape {
    static constexpr bool kCodes = FMT >= kAttnFp8;
    static constexpr int kBits = FMT == kAttnFp4 ? 4 : (FMT == kAttnFp8 ? 8 : 16);
    static constexpr int kStep = kCodes ? 32 : 16;               // positions of a step
    static constexpr int kTile = kStep * kAttnWarps;
    static constexpr int kChunks = D * kBits / 128;              // of 16 bytes in a row
    static constexpr int kRow = 16 * kChunks + (kCodes ? 0 : 16);    // from row to row in shared memory
    static constexpr int kScaleRow = kCodes ? (D > 128 ? 8 : 4) : 0;
    static constexpr int kScaleOff = 2 * kStep * kRow;
    static constexpr int kMaskOff = kScaleOff + 2 * kStep * kScaleRow;
    static constexpr int kStageBytes = kMaskOff + 16;
    // Two stages: a third in the place of a CTA is slower (24 sequences, MXFP8: 57 us with two CTAs of three stages, 50 with three of two).
    static constexpr int kStages = 2;
    static constexpr int kLift = FMT == kAttnFp4 ? 13 : 6;       // largest code 2^kLift stays below 2^16
    static constexpr int kMulBytes = kCodes ? 2 * (D / 32) * kStep * 2 : 0;      // fp16 multipliers [K, V][block][position]
    static constexpr int kRing = kStages * kStageBytes;
    static constexpr int kWarpBytes = kRing + kMulBytes;
    static constexpr int kJoinStride = D + 4;                    // floats
    static constexpr int kJoinBytes = kAttnWarps * NQ * kJoinStride * 4;
    static constexpr int kStatsOff = kAttnWarps * kWarpBytes > kJoinBytes ? kAttnWarps * kWarpBytes : kJoinBytes;
    static constexpr int kBytes = kStatsOff + kAttnWarps * NQ * 2 * 4;
    // CTAs of an SM: what registers (operands and accumulators of a lane, some 60 besides) and shared memory allow
    static constexpr int kRegs = D * NQ / 32 + D * NQ / 64;
    static constexpr int kByRegs = kRegs <= 48 ? 4 : (kRegs <= 96 ? 3 : 2);
    static constexpr int kBySmem = 227 * 1024 / (kBytes + 1024);
    static constexpr int kPerSm = kByRegs < kBySmem ? kByRegs : kBySmem;
    static_assert(kPerSm >= 1 && kStageBytes % 16 == 0 && kWarpBytes % 16 == 0, "shared memory");

    // where chunk c of a step's row r lies
    static __device__ __forceinline__ int chunk_at(int r, int c) {
        if constexpr (!kCodes) return c;
        else if constexpr (kChunks >= 8) return c ^ (2 * (r & 3));
        else if constexpr (kChunks == 4) return c ^ (r & 2);
        else return c;
    }
    // row of a step that is position k of the products
    static __device__ __forceinline__ int row_of(int k) {
        if constexpr (!kCodes) return k;
        const int j = (k & 7) >> 1;
        return (k & ~7) | ((k & 1) ? 4 + (j ^ (kChunks >= 8 ? 2 : 1)) : j);
    }
    // first of the four channels that lane quarter j holds for product m of K Q^T
    static __device__ __forceinline__ int k_channel(int m, int j) {
        if constexpr (!kCodes) {
            const int l = m >> 1;
            return 8 * (2 * j + (l & 1) + 8 * (l >> 1)) + 4 * (m & 1);
        } else if constexpr (FMT == kAttnFp8) {
            return 16 * (j + 4 * (m >> 2)) + 4 * (m & 3);
        } else if constexpr (kChunks >= 4) {
            return 32 * (j + 4 * (m >> 3)) + 4 * (m & 7);
        } else {
            return 16 * j + 4 * m;
        }
    }
};

template <int FMT, int D, int NQ>
__global__ void __launch_bounds__(kAttnThreads, (AttnShape<FMT, D, NQ>::kPerSm)) cache_attention_kernel(const __grid_constant__ AttentionProblem p) {
    using L = AttnShape<FMT, D, NQ>;
    constexpr int NT = NQ / 8, kM = D / 16;                              // column tiles; products of K Q^T = row tiles of O^T
    constexpr int kMt = L::kStep / 16;                                   // row tiles of S^T
    constexpr float kMinus = -INFINITY;
    extern __shared__ __align__(16) uint8_t attn_smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
    uint8_t* ring = attn_smem + warp * L::kWarpBytes;
    uint16_t* mul = reinterpret_cast<uint16_t*>(ring + L::kRing);
    const int row_lane = L::row_of(lane & (L::kStep - 1));
    float* join = reinterpret_cast<float*>(attn_smem);
    float* stats = reinterpret_cast<float*>(attn_smem + L::kStatsOff);
    const int real_chunks = p.c.row_bytes() / 16, blocks = p.c.blocks;
    const bool padded = real_chunks < L::kChunks;
    // what a lane copies: chunk lane % kChunks of every row
    const bool lane_copies = lane % L::kChunks < real_chunks;
    const uint32_t ring_at = shared_u32(ring), copy_row = lane / L::kChunks * L::kRow;
    const uint8_t *k_lane = p.c.k + 16 * (lane % L::kChunks), *v_lane = p.c.v + 16 * (lane % L::kChunks);
    const uint32_t row_bytes = (uint32_t)p.c.row_bytes(), pages = (uint32_t)p.c.pages, heads = (uint32_t)p.c.heads, page_size = (uint32_t)p.c.page_size;
    constexpr uint32_t kFull = L::kStep == 32 ? 0xFFFFFFFFu : (1u << L::kStep) - 1u;
    const uint32_t byte_mask0 = blocks >= 4 ? 0xFFFFFFFFu : (1u << (8 * blocks)) - 1u;
    const uint32_t byte_mask1 = blocks >= 8 ? 0xFFFFFFFFu : (blocks <= 4 ? 0u : (1u << (8 * (blocks - 4))) - 1u);
    pdl_launch_dependents();
    pdl_wait_prior_grid();

    // ---- this CTA's run ----
    const int per_seq = p.c.heads * p.chunks;
    int64_t at = 0, stop = 0, quota = 0;
    int seq = 0, item = 0, unit = 0;                                     // unit: of the item, kLead and then its tiles
    if (p.partial) {
        // units of the sequences 0 .. 31, a lane each: most calls need no others
        const int n0 = lane < p.sequences ? tiles_of<L::kTile>(visible_range(p, lane)) + kLead : 0;
        int64_t sum = n0;
        for (int s = lane + 32; s < p.sequences; s += 32) sum += tiles_of<L::kTile>(visible_range(p, s)) + kLead;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        const int64_t total = sum * per_seq, rounded = total + p.ctas - 1;
        quota = rounded < 0x7FFFFFFF ? (uint32_t)rounded / (uint32_t)p.ctas : rounded / p.ctas;      // (32 bits divide in a third of the time)
        if (quota < p.min_run) quota = p.min_run;
        at = blockIdx.x * quota;
        stop = at + quota < total ? at + quota : total;
        if (at >= stop) return;
        int64_t before = 0;                                              // units per head of the sequences before
        for (int s0 = 0;; s0 += 32) {
            const int n = s0 == 0 ? n0 : s0 + lane < p.sequences ? tiles_of<L::kTile>(visible_range(p, s0 + lane)) + kLead : 0;
            int64_t upto = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
                if (lane >= o) upto += v;
            }
            const uint32_t past = __ballot_sync(0xFFFFFFFFu, (before + upto) * per_seq > at);
            if (past) {
                const int first = __ffs(past) - 1;
                seq = s0 + first;
                const int units = __shfl_sync(0xFFFFFFFFu, n, first);
                const int64_t rest = at - (before + __shfl_sync(0xFFFFFFFFu, upto, first) - units) * per_seq;
                item = (int)(rest < 0x7FFFFFFF ? (uint32_t)rest / (uint32_t)units : rest / units);
                unit = (int)(rest - (int64_t)item * units);
                break;
            }
            before += __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
    } else {
        at = blockIdx.x;
        stop = (int64_t)p.sequences * per_seq;
    }

    bool first_segment = true;
    while (at < stop) {
        if (!p.partial) {
            seq = (int)(at / per_seq);
            item = (int)(at - (int64_t)seq * per_seq);
        }
        int s_seq, s_item;                                               // what is done here (seq and item move on)
        const VisibleRange range = visible_range(p, seq);
        const int tiles = tiles_of<L::kTile>(range);
        // tiles tile .. tile + count - 1 of the item
        int tile = 0, count = tiles;
        if (p.partial) {
            const int64_t left = stop - at;
            const int units = left < tiles + kLead - unit ? (int)left : tiles + kLead - unit, last = unit + units - kLead;
            tile = unit > kLead ? unit - kLead : 0;
            count = last > tile ? last - tile : 0;
            const int64_t item_at = at - unit;
            at += units;
            const int item_now = item, seq_now = seq;
            unit = 0;
            if (++item == per_seq) {
                item = 0;
                ++seq;
            }
            if (count == 0) continue;                                    // (the item's lead alone)
            const bool whole_run = count == tiles;
            if (tile == 0 && threadIdx.x == 0)
                p.parts[(int64_t)seq_now * per_seq + item_now] =
                    make_int2((int)blockIdx.x, whole_run ? 1 : (int)((item_at + kLead + tiles - 1) / quota) - (int)blockIdx.x + 1);
            s_seq = seq_now;
            s_item = item_now;
        } else {
            s_seq = seq;
            s_item = item;
            at += gridDim.x;
        }
        const bool whole = tile == 0 && count == tiles;
        const int slot = 2 * (int)blockIdx.x + (tile == 0 ? 1 : 0);
        const int head = s_item / p.chunks, chunk = s_item - head * p.chunks;
        const int token0 = range.begin + tile * L::kTile;
        const int64_t token_end = (int64_t)token0 + (int64_t)count * L::kTile;
        const int end = token_end < range.end ? (int)token_end : range.end;
        const int steps = end > token0 ? (end - token0 + L::kStep - 1) / L::kStep : 0;
        const int my_steps = steps > warp ? (steps - warp + kAttnWarps - 1) / kAttnWarps : 0;
        const int32_t* table = p.table + (int64_t)s_seq * p.table_stride;

        if (padded || first_segment) {                                   // columns behind the rows' channels stay zero
            if (padded)
                for (int i = lane; i < L::kRing / 16; i += 32) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
            first_segment = false;
            __syncwarp();
        }

        // ---- copies of a step ----
        // table entry and slot of position `lane` of step i of this warp; the entry is looked at when the step is copied, one step later
        int page_next = -1;
        uint32_t slot_next = 0;
        auto look_up = [&](int i) {
            const int t = token0 + (warp + i * kAttnWarps) * L::kStep + lane;
            page_next = -1;
            if (i >= my_steps || lane >= L::kStep || t >= end) return;
            const uint32_t entry = p.c.by_page.div((uint32_t)t);
            slot_next = (uint32_t)t - entry * page_size;
            page_next = table[entry];
        };
        look_up(0);
        int fill = 0;                                                    // stage of the next step to copy
        auto issue = [&](int i) {
            if (i < my_steps) {
                const bool live = (uint32_t)page_next < pages;
                const uint32_t cell = live ? ((uint32_t)page_next * heads + (uint32_t)head) * page_size + slot_next : 0u;
                const uint32_t mask = __ballot_sync(0xFFFFFFFFu, live);
                look_up(i + 1);
                const uint32_t base = ring_at + fill * L::kStageBytes;
                fill = fill + 1 == L::kStages ? 0 : fill + 1;
                constexpr int kRows = 32 / L::kChunks, kPasses = L::kStep / kRows;   // rows of a pass
#pragma unroll
                for (int x = 0; x < kPasses; ++x) {
                    const int r = x * kRows + lane / L::kChunks;
                    const uint64_t from = __shfl_sync(0xFFFFFFFFu, cell, r);
                    const uint32_t dst = base + copy_row + x * kRows * L::kRow + 16 * L::chunk_at(r, lane % L::kChunks);
                    const uint32_t size = mask == kFull ? 16u : ((mask >> r) & 1u) << 4;
                    if (lane_copies) {
                        copy_async_16(dst, k_lane + from * row_bytes, size);
                        copy_async_16(dst + L::kStep * L::kRow, v_lane + from * row_bytes, size);
                    }
                }
                if constexpr (L::kCodes) {
                    copy_async_small<L::kScaleRow>(base + L::kScaleOff + lane * L::kScaleRow, p.c.k_scales + (uint64_t)cell * L::kScaleRow, live);
                    copy_async_small<L::kScaleRow>(base + L::kScaleOff + (L::kStep + lane) * L::kScaleRow, p.c.v_scales + (uint64_t)cell * L::kScaleRow, live);
                }
                if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(base + L::kMaskOff), "r"(mask) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };

        // ---- queries: operand registers and their power of two ----
        uint32_t qf[kM][NT][2];
        float q_scale = p.scale_log2e;
        bool apart = false;                                              // the queries have a power of two each
        float* const powers = stats + warp * NQ;                         // then: those (the place of the warp's maxima)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = chunk * NQ + nt * 8 + g;                     // query head within the group
            const bool exists = row < p.group;
            const uint16_t* q = static_cast<const uint16_t*>(p.q) + (int64_t)s_seq * p.q_row + (int64_t)(head * p.group + (exists ? row : 0)) * p.q_head;
#pragma unroll
            for (int m = 0; m < kM; ++m) {
                const int ch = L::k_channel(m, j);
                if (p.q_vec) {                                           // four channels at a time; nothing waits for them yet
                    uint2 w = make_uint2(0, 0);
                    if (exists && ch < p.c.head_dim) w = *reinterpret_cast<const uint2*>(q + ch);
                    qf[m][nt][0] = w.x;
                    qf[m][nt][1] = w.y;
                } else {
                    uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (exists && ch + i < p.c.head_dim) v[i] = q[ch + i];
                    qf[m][nt][0] = v[0] | (v[1] << 16);
                    qf[m][nt][1] = v[2] | (v[3] << 16);
                }
            }
        }

        float o[kM][NT][4];
        float m_run[NT][2], l_run[NT][2];
        int v_run = 0;                                                   // R of the comment above
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int m = 0; m < kM; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[m][nt][i] = 0.f;
            m_run[nt][0] = m_run[nt][1] = kMinus;
            l_run[nt][0] = l_run[nt][1] = 0.f;
        }

#pragma unroll
        for (int i = 0; i < L::kStages - 1; ++i) issue(i);
        if constexpr (L::kCodes) {
            int e[NT], most = -100, least = 128;                         // exponent of the largest value of query 8 nt + g (-100 at least), of all queries'
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                uint32_t amax = 0;                                       // of the magnitude bits
#pragma unroll
                for (int m = 0; m < kM; ++m)
#pragma unroll
                    for (int i = 0; i < 2; ++i) amax = max(amax, max(qf[m][nt][i] & 0x7FFFu, (qf[m][nt][i] >> 16) & 0x7FFFu));
                amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
                amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
                const float top = p.q_f16 ? __half2float(__ushort_as_half((unsigned short)amax)) : __uint_as_float(amax << 16);
                e[nt] = max((int)(__float_as_uint(top) >> 23) - 127, -100);              // (infinity and NaN: 128)
                most = max(most, e[nt]);
                if (amax) least = min(least, e[nt]);                     // (queries that are zero, or that there are none of, go with any power)
            }
            most = __reduce_max_sync(0xFFFFFFFFu, most);
            apart = most - __reduce_min_sync(0xFFFFFFFFu, least) > kQueryRange;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (!apart) e[nt] = most;
                else if (j == 0) powers[nt * 8 + g] = exp2_int(e[nt]);
                const float up = exp2_int(14 - e[nt]);
#pragma unroll
                for (int m = 0; m < kM; ++m)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t w = qf[m][nt][i];
                        float lo, hi;
                        if (p.q_f16) {
                            lo = __half2float(__ushort_as_half((unsigned short)(w & 0xFFFFu)));
                            hi = __half2float(__ushort_as_half((unsigned short)(w >> 16)));
                        } else {
                            lo = bf16lo_to_f32(w);
                            hi = bf16hi_to_f32(w);
                        }
                        qf[m][nt][i] = pack_f16(lo * up, hi * up);
                    }
            }
            q_scale *= exp2_int((apart ? 0 : most) - 14 - L::kLift);
            __syncwarp();
        }

        int use = 0;
        uint32_t seen = 0;                                               // whether any position has had a place
        for (int it = 0; it < my_steps; ++it) {
            asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 2) : "memory");
            __syncwarp();
            issue(it + L::kStages - 1);                                  // (into the stage of the step before, which all lanes have left)
            const uint8_t* stage = ring + use * L::kStageBytes;
            use = use + 1 == L::kStages ? 0 : use + 1;
            const uint8_t* kst = stage;
            const uint8_t* vst = stage + L::kStep * L::kRow;
            const uint32_t mask = *reinterpret_cast<const uint32_t*>(stage + L::kMaskOff);
            seen |= mask;

            // ---- scales: lane = position of the products ----
            float k_factor = q_scale, v_factor = 1.f;
            int v_new = v_run;
            if constexpr (L::kCodes) {
                int top[2];
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    const uint8_t* s = stage + L::kScaleOff + (kv * L::kStep + row_lane) * L::kScaleRow;
                    uint32_t w[L::kScaleRow / 4];
                    w[0] = *reinterpret_cast<const uint32_t*>(s) & byte_mask0;
                    if constexpr (L::kScaleRow == 8) w[1] = *reinterpret_cast<const uint32_t*>(s + 4) & byte_mask1;
                    int S[D / 32], most = 0;
#pragma unroll
                    for (int b = 0; b < D / 32; ++b) {
                        S[b] = (int)((w[b / 4] >> (8 * (b & 3))) & 0xFFu);
                        most = max(most, S[b]);
                    }
                    top[kv] = most;
                    // fp16 bits of 2^(S - most + kLift), 0 below its normal range
#pragma unroll
                    for (int b = 0; b < D / 32; ++b)
                        mul[(kv * (D / 32) + b) * L::kStep + lane] = (uint16_t)(max(S[b] - most + 15 + L::kLift, 0) << 10);
                }
                k_factor *= __uint_as_float((uint32_t)top[0] << 23);     // 2^(S - 127)
                v_new = max(v_run, (int)__reduce_max_sync(0xFFFFFFFFu, top[1]));     // (0 where there is no position)
                v_factor = __uint_as_float((uint32_t)max(top[1] - v_new + 127 + kPLift, 0) << 23);
                __syncwarp();
            }

            // ---- S^T = K Q^T ----
            float s[kMt][NT][4];
#pragma unroll
            for (int mt = 0; mt < kMt; ++mt) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[mt][nt][i] = 0.f;
                const int r0 = L::row_of(16 * mt + g), r1 = r0 + 8;
                const uint8_t* a = kst + r0 * L::kRow;
                const uint8_t* b = kst + r1 * L::kRow;
                if constexpr (FMT == kAttnFp4 && L::kChunks == 2) {
                    const uint2 x = *reinterpret_cast<const uint2*>(a + 8 * j), y = *reinterpret_cast<const uint2*>(b + 8 * j);
                    const uint32_t xs = mul[(j >> 1) * L::kStep + 16 * mt + g] * 0x10001u, ys = mul[(j >> 1) * L::kStep + 16 * mt + g + 8] * 0x10001u;
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        uint32_t hx[4], hy[4];
                        e2m1x8_to_f16(w ? x.y : x.x, hx);
                        e2m1x8_to_f16(w ? y.y : y.x, hy);
#pragma unroll
                        for (int i = 0; i < 4; ++i) { hx[i] = mul_f16x2(hx[i], xs); hy[i] = mul_f16x2(hy[i], ys); }
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
                                mma_16816_f16(s[mt][nt], hx[2 * h], hy[2 * h], hx[2 * h + 1], hy[2 * h + 1], qf[2 * w + h][nt][0], qf[2 * w + h][nt][1]);
                    }
                } else {
#pragma unroll
                    for (int l = 0; l < L::kChunks / 4; ++l) {
                        const int c = L::kCodes ? j + 4 * l : 2 * j + (l & 1) + 8 * (l >> 1);
                        const uint4 x = *reinterpret_cast<const uint4*>(a + 16 * L::chunk_at(r0, c));
                        const uint4 y = *reinterpret_cast<const uint4*>(b + 16 * L::chunk_at(r1, c));
                        const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
                        if constexpr (!L::kCodes) {
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    if constexpr (FMT == kAttnBf16)
                                        mma_16816_bf16(s[mt][nt], xw[2 * h], yw[2 * h], xw[2 * h + 1], yw[2 * h + 1], qf[2 * l + h][nt][0], qf[2 * l + h][nt][1]);
                                    else
                                        mma_16816_f16(s[mt][nt], xw[2 * h], yw[2 * h], xw[2 * h + 1], yw[2 * h + 1], qf[2 * l + h][nt][0], qf[2 * l + h][nt][1]);
                                }
                        } else {
                            const int block = FMT == kAttnFp8 ? c >> 1 : c;
                            const uint32_t xs = mul[block * L::kStep + 16 * mt + g] * 0x10001u, ys = mul[block * L::kStep + 16 * mt + g + 8] * 0x10001u;
#pragma unroll
                            for (int w = 0; w < 4; ++w) {
                                if constexpr (FMT == kAttnFp8) {
                                    uint32_t x0, x1, y0, y1;
                                    e4m3x4_to_f16(xw[w], x0, x1);
                                    e4m3x4_to_f16(yw[w], y0, y1);
                                    x0 = mul_f16x2(x0, xs); x1 = mul_f16x2(x1, xs);
                                    y0 = mul_f16x2(y0, ys); y1 = mul_f16x2(y1, ys);
#pragma unroll
                                    for (int nt = 0; nt < NT; ++nt)
                                        mma_16816_f16(s[mt][nt], x0, y0, x1, y1, qf[4 * l + w][nt][0], qf[4 * l + w][nt][1]);
                                } else {
                                    uint32_t hx[4], hy[4];
                                    e2m1x8_to_f16(xw[w], hx);
                                    e2m1x8_to_f16(yw[w], hy);
#pragma unroll
                                    for (int i = 0; i < 4; ++i) { hx[i] = mul_f16x2(hx[i], xs); hy[i] = mul_f16x2(hy[i], ys); }
#pragma unroll
                                    for (int h = 0; h < 2; ++h)
#pragma unroll
                                        for (int nt = 0; nt < NT; ++nt)
                                            mma_16816_f16(s[mt][nt], hx[2 * h], hy[2 * h], hx[2 * h + 1], hy[2 * h + 1], qf[8 * l + 2 * w + h][nt][0], qf[8 * l + 2 * w + h][nt][1]);
                                }
                            }
                        }
                    }
                }
            }

            // ---- scores, running maximum and sum ----
            float vf[kMt][2];
            auto scores = [&](auto own) {                                // own: with the queries' own powers
                float power[NT][2];
                if constexpr (decltype(own)::value) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const float2 two = *reinterpret_cast<const float2*>(powers + nt * 8 + 2 * j);
                        power[nt][0] = two.x;
                        power[nt][1] = two.y;
                    }
                }
#pragma unroll
                for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int k = 16 * mt + 8 * h + g;
                        float kf = q_scale;
                        vf[mt][h] = FMT == kAttnF16 ? (float)(1 << kPLift) : 1.f;
                        if constexpr (L::kCodes) {
                            kf = __shfl_sync(0xFFFFFFFFu, k_factor, k);
                            vf[mt][h] = __shfl_sync(0xFFFFFFFFu, v_factor, k);
                        }
                        const float shut = (mask >> L::row_of(k)) & 1u ? 0.f : kMinus;   // (keys without a place were read as zeros)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                float f = kf;
                                if constexpr (decltype(own)::value) f *= power[nt][i];
                                s[mt][nt][2 * h + i] = fmaf(s[mt][nt][2 * h + i], f, shut);
                            }
                    }
            };
            if (L::kCodes && apart) scores(std::true_type{});
            else scores(std::false_type{});
            bool grown = v_new != v_run;
            float m_new[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float m = m_run[nt][i];
#pragma unroll
                    for (int mt = 0; mt < kMt; ++mt) m = fmaxf(m, fmaxf(s[mt][nt][i], s[mt][nt][2 + i]));
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
                    m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
                    m_new[nt][i] = m;
                    grown |= m > m_run[nt][i] + kSlack;
                }
            if (__any_sync(0xFFFFFFFFu, grown)) {                        // (seldom, thanks to the slack)
                const float v_down = exp2_int(v_run - v_new);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float down = m_run[nt][i] == kMinus ? 0.f : exp2_fast(m_run[nt][i] - m_new[nt][i]);
                        m_run[nt][i] = m_new[nt][i];
                        l_run[nt][i] *= down;
                        const float both = down * v_down;
#pragma unroll
                        for (int m = 0; m < kM; ++m) {
                            o[m][nt][i] *= both;
                            o[m][nt][2 + i] *= both;
                        }
                    }
                v_run = v_new;
            }
            // weights, as operand B of O^T += V^T P^T
            uint32_t pb[kMt][NT][2], pl[L::kCodes ? 1 : kMt][NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float m0 = m_run[nt][0] == kMinus ? 0.f : m_run[nt][0], m1 = m_run[nt][1] == kMinus ? 0.f : m_run[nt][1];
#pragma unroll
                for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float p0 = exp2_fast(s[mt][nt][2 * h] - m0), p1 = exp2_fast(s[mt][nt][2 * h + 1] - m1);
                        l_run[nt][0] += p0;
                        l_run[nt][1] += p1;
                        if constexpr (FMT == kAttnBf16) {
                            const uint32_t hi = pack_bf16(p0, p1);
                            pb[mt][nt][h] = transpose_8x8(hi);
                            pl[mt][nt][h] = transpose_8x8(pack_bf16(p0 - bf16lo_to_f32(hi), p1 - bf16hi_to_f32(hi)));
                        } else {
                            const float w0 = p0 * vf[mt][h], w1 = p1 * vf[mt][h];
                            const uint32_t hi = pack_f16(w0, w1);
                            pb[mt][nt][h] = transpose_8x8(hi);
                            if constexpr (FMT == kAttnF16) {
                                const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                                pl[mt][nt][h] = transpose_8x8(pack_f16(w0 - back.x, w1 - back.y));
                            }
                        }
                    }
            }

            // ---- O^T += V^T P^T ----
            if constexpr (!L::kCodes) {
                const int r = (lane & 7) + ((lane >> 4) & 1) * 8;
                const uint32_t row = shared_u32(vst) + r * L::kRow;
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                    uint32_t a0, a1, a2, a3;
                    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(a0), "=r"(a1), "=r"(a2), "=r"(a3) : "r"(row + 16 * L::chunk_at(r, 2 * m + ((lane >> 3) & 1))) : "memory");
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if constexpr (FMT == kAttnBf16) {
                            mma_16816_bf16(o[m][nt], a0, a1, a2, a3, pb[0][nt][0], pb[0][nt][1]);
                            mma_16816_bf16(o[m][nt], a0, a1, a2, a3, pl[0][nt][0], pl[0][nt][1]);
                        } else {
                            mma_16816_f16(o[m][nt], a0, a1, a2, a3, pb[0][nt][0], pb[0][nt][1]);
                            mma_16816_f16(o[m][nt], a0, a1, a2, a3, pl[0][nt][0], pl[0][nt][1]);
                        }
                    }
                }
            } else {
                constexpr int kBytesV = 2 * L::kChunks, kWords = kBytesV / 4;   // of a lane's channels at one position
                const int block = g * (D / 8) / 32;
#pragma unroll
                for (int mt = 0; mt < kMt; ++mt) {
                    uint32_t w[4][kWords];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {                        // positions 2j, 2j + 1, 2j + 8, 2j + 9
                        const int r = L::row_of(16 * mt + 2 * j + (i & 1) + 8 * (i >> 1));
                        const uint8_t* row = vst + r * L::kRow;
                        if constexpr (kBytesV == 4) {
                            w[i][0] = *reinterpret_cast<const uint32_t*>(row + 16 * L::chunk_at(r, g >> 2) + 4 * (g & 3));
                        } else if constexpr (kBytesV == 8) {
                            const uint2 x = *reinterpret_cast<const uint2*>(row + 16 * L::chunk_at(r, g >> 1) + 8 * (g & 1));
                            w[i][0] = x.x; w[i][1] = x.y;
                        } else {
#pragma unroll
                            for (int c = 0; c < kBytesV / 16; ++c) {
                                const uint4 x = *reinterpret_cast<const uint4*>(row + 16 * L::chunk_at(r, g * (kBytesV / 16) + c));
                                w[i][4 * c] = x.x; w[i][4 * c + 1] = x.y; w[i][4 * c + 2] = x.z; w[i][4 * c + 3] = x.w;
                            }
                        }
                    }
                    const uint16_t* mv = mul + (D / 32 + block) * L::kStep + 16 * mt + 2 * j;
                    const uint32_t m01 = *reinterpret_cast<const uint32_t*>(mv), m23 = *reinterpret_cast<const uint32_t*>(mv + 8);
#pragma unroll
                    for (int x = 0; x < kWords; ++x) {
                        if constexpr (FMT == kAttnFp8) {                 // four channels: the same channel of two positions side by side
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                uint32_t a0, a1, a2, a3;
                                e4m3x4_to_f16(__byte_perm(w[0][x], w[1][x], h ? 0x7362 : 0x5140), a0, a1);
                                e4m3x4_to_f16(__byte_perm(w[2][x], w[3][x], h ? 0x7362 : 0x5140), a2, a3);
                                a0 = mul_f16x2(a0, m01); a1 = mul_f16x2(a1, m01);
                                a2 = mul_f16x2(a2, m23); a3 = mul_f16x2(a3, m23);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) mma_16816_f16(o[2 * x + h][nt], a0, a1, a2, a3, pb[mt][nt][0], pb[mt][nt][1]);
                            }
                        } else {                                         // eight channels
                            constexpr uint32_t kLow = 0x0F0F0F0Fu;
                            uint32_t e01[4], o01[4], e23[4], o23[4];     // even and odd channels of the pairs of positions
                            e2m1x8_to_f16((w[0][x] & kLow) | ((w[1][x] << 4) & ~kLow), e01);
                            e2m1x8_to_f16(((w[0][x] >> 4) & kLow) | (w[1][x] & ~kLow), o01);
                            e2m1x8_to_f16((w[2][x] & kLow) | ((w[3][x] << 4) & ~kLow), e23);
                            e2m1x8_to_f16(((w[2][x] >> 4) & kLow) | (w[3][x] & ~kLow), o23);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t a0 = mul_f16x2(e01[i], m01), a1 = mul_f16x2(o01[i], m01);
                                const uint32_t a2 = mul_f16x2(e23[i], m23), a3 = mul_f16x2(o23[i], m23);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) mma_16816_f16(o[4 * x + i][nt], a0, a1, a2, a3, pb[mt][nt][0], pb[mt][nt][1]);
                            }
                        }
                    }
                }
            }
            __syncwarp();                                                // the multipliers' place is free again
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");

        // ---- the warps' parts together ----
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float l = l_run[nt][i];
                l += __shfl_xor_sync(0xFFFFFFFFu, l, 4);
                l += __shfl_xor_sync(0xFFFFFFFFu, l, 8);
                l += __shfl_xor_sync(0xFFFFFFFFu, l, 16);
                if (seen == 0) l = 0.f;                                  // (a query that is not finite has met no position)
                if (g == 0) {
                    stats[warp * NQ + nt * 8 + 2 * j + i] = m_run[nt][i];
                    stats[(kAttnWarps + warp) * NQ + nt * 8 + 2 * j + i] = l;
                }
            }
        __syncthreads();                                                 // all warps have left their rings
        const float unit = L::kCodes ? exp2_int(v_run - 127 - kPLift - L::kLift) : (FMT == kAttnF16 ? 1.f / (1 << kPLift) : 1.f);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int col = nt * 8 + 2 * j + i;
                float top = kMinus;
#pragma unroll
                for (int w = 0; w < kAttnWarps; ++w) top = fmaxf(top, stats[w * NQ + col]);
                const float f = m_run[nt][i] == kMinus ? 0.f : exp2_fast(m_run[nt][i] - top) * unit;
                float* to = join + (warp * NQ + col) * L::kJoinStride;
#pragma unroll
                for (int m = 0; m < kM; ++m) {
                    if constexpr (L::kCodes) {
                        *reinterpret_cast<float2*>(to + g * (D / 8) + 2 * m) = make_float2(o[m][nt][i] * f, o[m][nt][2 + i] * f);
                    } else {
                        to[16 * m + g] = o[m][nt][i] * f;
                        to[16 * m + 8 + g] = o[m][nt][2 + i] * f;
                    }
                }
            }
        __syncthreads();
        const int live_q = p.group - chunk * NQ < NQ ? p.group - chunk * NQ : NQ;
        for (int i = threadIdx.x; i < live_q * D; i += kAttnThreads) {
            const int col = i / D, ch = i - col * D;
            float top = kMinus, sum = 0.f, l = 0.f;
#pragma unroll
            for (int w = 0; w < kAttnWarps; ++w) top = fmaxf(top, stats[w * NQ + col]);
            const float ref = top == kMinus ? 0.f : top;
#pragma unroll
            for (int w = 0; w < kAttnWarps; ++w) {
                sum += join[(w * NQ + col) * L::kJoinStride + ch];
                l += stats[(kAttnWarps + w) * NQ + col] * exp2_fast(stats[w * NQ + col] - ref);
            }
            if (whole) {
                const int q_head = head * p.group + chunk * NQ + col;
                const float v = l == 0.f ? 0.f : sum / l;
                if (ch < p.c.head_dim) {
                    const int64_t to = (int64_t)s_seq * p.out_row + (int64_t)q_head * p.out_head + ch;
                    if (p.out_type == 0) static_cast<float*>(p.out)[to] = v;
                    else if (p.out_type == 2) static_cast<__half*>(p.out)[to] = __float2half_rn(v);
                    else static_cast<__nv_bfloat16*>(p.out)[to] = __float2bfloat16_rn(v);
                }
                if (p.lse && ch == 0) p.lse[(int64_t)s_seq * p.q_heads + q_head] = l == 0.f ? kMinus : (top + log2f(l)) * 0.6931471805599453f;
            } else {
                p.partial[((int64_t)slot * NQ + col) * D + ch] = sum;
                if (ch == 0) {
                    float* st = p.partial + (int64_t)2 * p.ctas * NQ * D + (int64_t)slot * 2 * NQ;
                    st[col] = top;
                    st[NQ + col] = l;
                }
            }
        }
        __syncthreads();                                                 // the rings are free again
    }
}

constexpr int kJoinThreads = 1024;       // at most; 256 where there are many items, most of which have a few parts

// Joins the parts of an item that several CTAs took: blockIdx.x = item, blockIdx.y = query of the chunk.  The threads are D/4 groups of
// four channels times lanes that take every so many parts with a running maximum; the lanes' sums are added in order.
template <int D, int NQ>
__global__ void __launch_bounds__(kJoinThreads) cache_attention_join(const __grid_constant__ AttentionProblem p) {
    constexpr int kCols = D / 4;
    __shared__ float4 sums[kJoinThreads];
    __shared__ float tops[kJoinThreads / kCols], weights[kJoinThreads / kCols];
    const int every = (int)blockDim.x / kCols;
    pdl_launch_dependents();
    const int per_seq = p.c.heads * p.chunks;
    const int seq = (int)blockIdx.x / per_seq, item = (int)blockIdx.x - seq * per_seq;
    const int head = item / p.chunks, col = blockIdx.y, row = (item - head * p.chunks) * NQ + col;
    if (row >= p.group) return;
    pdl_wait_prior_grid();
    const int2 parts = p.parts[blockIdx.x];
    if (parts.y <= 1) return;                                            // written by its CTA
    const float* st = p.partial + (int64_t)2 * p.ctas * NQ * D;
    const int x = threadIdx.x % kCols, y = threadIdx.x / kCols;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f, top = -INFINITY;
    constexpr int kAhead = 8;
    for (int c = y; c < parts.y; c += kAhead * every) {
        float4 v[kAhead];
        float m[kAhead], w[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = c + i * every;
            const int64_t slot = 2 * (int64_t)(parts.x + (k < parts.y ? k : 0)) + (k == 0 || k >= parts.y ? 1 : 0);
            v[i] = *reinterpret_cast<const float4*>(p.partial + (slot * NQ + col) * D + 4 * x);
            m[i] = k < parts.y ? st[slot * 2 * NQ + col] : -INFINITY;
            w[i] = st[slot * 2 * NQ + NQ + col];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (c + i * every >= parts.y) break;
            const float up = fmaxf(top, m[i]), ref = up == -INFINITY ? 0.f : up;
            const float f = exp2_fast(top - ref), e = exp2_fast(m[i] - ref);
            top = up;
            l = l * f + w[i] * e;
            sum.x = sum.x * f + v[i].x * e;
            sum.y = sum.y * f + v[i].y * e;
            sum.z = sum.z * f + v[i].z * e;
            sum.w = sum.w * f + v[i].w * e;
        }
    }
    sums[threadIdx.x] = sum;
    if (x == 0) {
        tops[y] = top;
        weights[y] = l;
    }
    __syncthreads();
    if (y != 0) return;
    const int lanes = parts.y < every ? parts.y : every;
    top = tops[0];
    for (int k = 1; k < lanes; ++k) top = fmaxf(top, tops[k]);
    const float ref = top == -INFINITY ? 0.f : top;
    sum = make_float4(0.f, 0.f, 0.f, 0.f);
    l = 0.f;
    for (int k = 0; k < lanes; ++k) {
        const float4 v = sums[k * kCols + x];
        const float e = exp2_fast(tops[k] - ref);
        sum.x += v.x * e; sum.y += v.y * e; sum.z += v.z * e; sum.w += v.w * e;
        l += weights[k] * e;
    }
    const int q_head = head * p.group + row;
    const float all[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int ch = 4 * x + i;
        if (ch >= p.c.head_dim) continue;
        const float v = l == 0.f ? 0.f : all[i] / l;
        const int64_t to = (int64_t)seq * p.out_row + (int64_t)q_head * p.out_head + ch;
        if (p.out_type == 0) static_cast<float*>(p.out)[to] = v;
        else if (p.out_type == 2) static_cast<__half*>(p.out)[to] = __float2half_rn(v);
        else static_cast<__nv_bfloat16*>(p.out)[to] = __float2bfloat16_rn(v);
    }
    if (p.lse && x == 0) p.lse[(int64_t)seq * p.q_heads + q_head] = l == 0.f ? -INFINITY : (top + log2f(l)) * 0.6931471805599453f;
}

}  // namespace kq
