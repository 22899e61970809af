// The linear layer of kq_linear.cuh for a few rows in 16 bits and a weight in MXFP4, sm_100a:
//     acc[m][r] = sum_k x[m][k] w[r][k] 2^(sw[r][k/32] - 127),     then the same epilogue
//
// Bound by reading the weight (half a byte per element and a scale byte per 32): nothing else grows with N K.  With so few rows
// the tensor cores are there to keep up with memory, not for their rate, and mma.sync takes its operands from registers: weight rows as the
// 16 rows of the product, rows of x as its 8 columns, so that codes go from memory through the converter into the operand and are never
// stored again (an operand for tcgen05 has to lie in shared memory, in 16 bits: four times the bytes of the codes written and read).
//
// Eight warps take 128 weight rows, one tile of the scale layout (a CTA has one such tile, or two and x for both).  Warp w takes rows 32 q + 8 (w % 4) + g, q = 0..3, g = lane / 4, so that the 16
// scale bytes a lane loads are those of its four rows and no scale is fetched twice; lane j = lane % 4 of a quad takes block j of 128
// channels, 16 bytes of codes of each row.  The channels' order within the products is the lanes', which x follows in shared memory.
// The two halves of the warps take every other 128 channels, and the CTAs of a cluster runs of them; the partial sums
// meet in shared memory and are added in a fixed order.
//
// x in fp16: 128 channels of a row are scaled by a power of two that brings the largest to [2^14, 2^15).  fp16 then holds every bf16 and
// fp16 value exactly that is larger than 2^-28 of it; smaller ones are off by 2^-40 of it.  A weight's value is code times 2^(S - S0 + 13), S0 the
// largest of the row's four scale bytes: at most 2 significant bits, exact; a block whose scale is 2^-28 of S0's, or less, counts as zero.
// 2^(S0 - 127 - 13) and x's power multiply the fp32 sum of 128 channels.
//
// Measured (us, and the time of the bytes at the copy rate): one row 1152 -> 6912 5.5 (0.7), 5 rows 4096 -> 2 x 5632 gated 12.2 (3.8), 16 rows 12288 -> 4608
// 19.3, with a residual 20.1 (4.7).  The last runs as 18 clusters of six CTAs of two tiles, 8 units of 128 channels for each warp: some 7 us are theirs, the
// others go by until x is converted (mostly latencies) and waiting for the cluster's last CTA, its sums and the epilogue.  Runs of more than 16 rows
// read and decode the weight once for each 16: 33 and 64 rows 4608 -> 12288 37 and 69 (4.8), 16 rows 21.
#pragma once
#include "kq_linear.cuh"
#include "kq_mma16.cuh"

namespace kq {

struct W4A16Problem {
    LinearProblem lin;                   // M, R, epilogue
    const void* x;
    int64_t ld_x;
    int x_vec;                           // rows allow 16-byte loads
    int K, units;                        // units of 128 channels
    const uint8_t *codes, *scales;
};

constexpr int kW4Threads = 256;          // of a tile
constexpr int kW4Stages = 3;             // units of a warp on the way or in use
constexpr int kW4Lift = 13;              // 6 * 2^13 is the largest power-of-two multiple of a code in fp16
constexpr int kW4StageBytes = 2048 + 128;                                // [q][lane] x 16 bytes of codes, [g] x 16 scale bytes
template <int NT, int TILES> struct W4Smem {                            // (an SM has room for two tiles, in two CTAs or one)
    static constexpr int kUnits = (NT == 1 ? 24 : 14) * TILES;           // of x at a time (even: the halves of the warps take turns)
    static constexpr int kXOff = TILES * (kW4Threads / 32) * kW4Stages * kW4StageBytes;
    static constexpr int kXBytes = kUnits * NT * 2048;                   // [unit][row][128 channels]
    static constexpr int kPartBytes = TILES * 2 * 8 * NT * 128 * 4;      // [tile][half of the warps][row of x][weight row], from the start
    static constexpr int kScaleOff = kXOff + kXBytes;
    static constexpr int kBytes = kScaleOff + kUnits * 8 * NT * 4;
    static_assert(kPartBytes <= kXOff, "partial sums take the place of the stages");
};

// Place (16 bytes) of the k-th eight channels of block j within the 256 bytes of 128 channels of row m: neighbouring operands fill all banks.
__device__ __forceinline__ int w4_place(int m, int k, int j) { return (4 * k + j) ^ ((m & 1) << 2); }

// grid: x = TILES tiles of 128 weight rows times splits (a cluster), y = runs of 8 NT rows of x
template <bool GLU, int NT, bool XF16, int TILES>
__global__ void __launch_bounds__(kW4Threads * TILES, 2 / TILES) linear_w4a16_kernel(const __grid_constant__ W4A16Problem p, const int splits) {
    using L = W4Smem<NT, TILES>;
    constexpr int kThreads = kW4Threads * TILES;
    extern __shared__ __align__(16) uint8_t w4_smem[];
    uint4* x_smem = reinterpret_cast<uint4*>(w4_smem + L::kXOff);
    float* x_scale = reinterpret_cast<float*>(w4_smem + L::kScaleOff);
    const int own_tile = TILES > 1 ? threadIdx.x / kW4Threads : 0, thread = threadIdx.x - own_tile * kW4Threads;
    const int warp = thread >> 5, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
    const int rank = splits > 1 ? (int)cluster_ctarank() : 0;
    const int tile = (int)blockIdx.x / splits * TILES + own_tile, m0 = (int)blockIdx.y * 8 * NT;
    const int rows = p.lin.M - m0 < 8 * NT ? p.lin.M - m0 : 8 * NT;
    const int u0 = (int)((int64_t)p.units * rank / splits), u1 = (int)((int64_t)p.units * (rank + 1) / splits);
    const int half = warp >> 2, base_row = tile * 128 + 8 * (warp & 3) + g;
    const int blocks = p.K / 32;
    const int64_t pitch = p.K / 2;
    const bool exists = TILES == 1 || tile * 128 < p.lin.R;             // (a last tile alone: its neighbour's warps get zeros)
    const uint8_t* scales = p.scales + ((int64_t)(exists ? tile : 0) * p.units * 512) + (8 * (warp & 3) + g) * 16;
    const uint8_t* codes = p.codes + (int64_t)base_row * pitch + 16 * j;
    pdl_launch_dependents();
    pdl_wait_prior_grid();

    // A lane copies the codes that it will use itself, and lane 4 g the scales of its quad.
    uint8_t* ring = w4_smem + (threadIdx.x >> 5) * (kW4Stages * kW4StageBytes);
    const uint32_t ring_at = smem_u32(ring);
    int fill = 0;
    auto fetch = [&](int u) {
        if (u < u1) {
            const uint32_t to = ring_at + fill * kW4StageBytes;
            const uint8_t* from = codes + (int64_t)u * 64;
            const bool inside = 4 * u + j < blocks;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const bool row = inside && base_row + 32 * q < p.lin.R;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                             ::"r"(to + q * 512 + lane * 16), "l"(row ? from + (int64_t)(32 * q) * pitch : p.codes), "r"(row ? 16 : 0) : "memory");
            }
            if (j == 0) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 2048 + g * 16), "l"(scales + (int64_t)u * 512) : "memory");
            fill = fill + 1 == kW4Stages ? 0 : fill + 1;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int use = 0;

    float acc[2][NT][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][nt][i] = 0.f;

    NarrowColumn<GLU> col;
    const LinearItem item = {0, 0, tile, 0, p.lin.M};
    col.open(p.lin, item, thread);                             // (the bias is on its way meanwhile)
    if (p.lin.epi.residual && col.live)
        for (int c = col.first + rank * NarrowColumn<GLU>::kStep; c < rows; c += NarrowColumn<GLU>::kStep * splits)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const uint8_t*>(p.lin.epi.residual) +
                         ((int64_t)(m0 + c) * p.lin.epi.ld_residual + col.n) * (p.lin.epi.residual_type == kTypeF32 ? 4 : 2)));

    // A group of 16 lanes keeps one row of x and takes its 128 channels of every `turns`-th unit, a lane eight channels.
    const int piece = threadIdx.x & 15, group = threadIdx.x >> 4, turns = (kThreads / 16) / rows;
    const int m = group % rows, first = group < turns * rows ? group / rows : L::kUnits;
    const uint16_t* x_at = static_cast<const uint16_t*>(p.x) + (int64_t)(m0 + m) * p.ld_x + 8 * piece;
    uint4* const x_row = x_smem + m * 16;
    for (int p0 = u0; p0 < u1; p0 += L::kUnits) {
        const int p1 = p0 + L::kUnits < u1 ? p0 + L::kUnits : u1;
        if (p0 != u0) __syncthreads();
        // x of these units, as it is and in its order (asynchronous copies that put neighbouring 16 bytes apart take four times as long).
        // Columns of the products without a row of x hold what is there: they reach no output.
#pragma unroll 4
        for (int u = first; u < p1 - p0; u += turns) {
            const int ch = (p0 + u) * 128;
            const bool exists = ch + 8 * piece < p.K;
            if (p.x_vec) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                             ::"r"(smem_u32(x_row + u * 8 * NT * 16 + piece)), "l"(exists ? x_at + ch : static_cast<const uint16_t*>(p.x)), "r"(exists ? 16 : 0) : "memory");
            } else {
                uint32_t r[4] = {0, 0, 0, 0};
                if (exists)
#pragma unroll
                    for (int i = 0; i < 4; ++i) r[i] = (uint32_t)x_at[ch + 2 * i] | ((uint32_t)x_at[ch + 2 * i + 1] << 16);
                x_row[u * 8 * NT * 16 + piece] = make_uint4(r[0], r[1], r[2], r[3]);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (p0 == u0) {
#pragma unroll
            for (int i = 0; i < kW4Stages - 1; ++i) fetch(u0 + half + 2 * i);
            asm volatile("cp.async.wait_group %0;" ::"n"(kW4Stages - 1) : "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        // what a lane copied becomes fp16 times the power of two of its 128 channels and goes to its place among them
        const uint32_t lanes = 0xFFFFu << (lane & 16);
#pragma unroll 4
        for (int u = first; u < p1 - p0; u += turns) {
            uint4* row = x_row + u * 8 * NT * 16;
            float v[8];
            widen8_any<XF16>(row[piece], v);
            int e = (int)(__reduce_max_sync(lanes, __float_as_uint(absmax8(v))) >> 23) - 127;          // (and all have read)
            e = e < -112 ? -112 : e;
            const float up = exp2_int(14 - e);
            __syncwarp(lanes);
            row[w4_place(m, piece & 3, piece >> 2)] = make_uint4(pack_f16(v[0] * up, v[1] * up), pack_f16(v[2] * up, v[3] * up),
                                                                 pack_f16(v[4] * up, v[5] * up), pack_f16(v[6] * up, v[7] * up));
            if (piece == 0) x_scale[u * 8 * NT + m] = exp2_int(e - 14);
        }
        __syncthreads();
        for (int u = p0 + half; u < p1; u += 2) {                        // (the number of units is even: the order goes on over the passes)
            asm volatile("cp.async.wait_group %0;" ::"n"(kW4Stages - 2) : "memory");
            __syncwarp();
            fetch(u + 2 * (kW4Stages - 1));                              // into the stage that all lanes have left
            const uint8_t* stage = ring + use * kW4StageBytes;
            use = use + 1 == kW4Stages ? 0 : use + 1;
            uint4 w[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) w[q] = *reinterpret_cast<const uint4*>(stage + q * 512 + lane * 16);
            const uint4 sc = *reinterpret_cast<const uint4*>(stage + 2048 + g * 16);
            const int left = blocks - 4 * u;                             // blocks of this unit
            const uint32_t mask = left >= 4 ? 0xFFFFFFFFu : (1u << (8 * left)) - 1u;
            const uint32_t sw[4] = {sc.x & mask, sc.y & mask, sc.z & mask, sc.w & mask};
            uint32_t mul[4];
            float factor[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int s0 = (int)(sw[q] & 0xFFu), s1 = (int)((sw[q] >> 8) & 0xFFu), s2 = (int)((sw[q] >> 16) & 0xFFu), s3 = (int)(sw[q] >> 24);
                const int top = max(max(s0, s1), max(s2, s3));
                const int own = (int)((sw[q] >> (8 * j)) & 0xFFu);
                mul[q] = (uint32_t)max(own - top + 15 + kW4Lift, 0) * 0x04000400u;       // two fp16 2^(own - top + kW4Lift), 0 below the normal range
                factor[q] = exp2_int(top - 127 - kW4Lift);
            }
            float part[2][NT][4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) part[t][nt][i] = 0.f;
            const uint4* xs = x_smem + ((u - p0) * 8 * NT + g) * 16;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t xw[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint4 v = xs[nt * 128 + w4_place(g, k, j)];
                    xw[nt][0] = v.x; xw[nt][1] = v.y; xw[nt][2] = v.z; xw[nt][3] = v.w;
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    uint32_t lo[4], hi[4];
                    const uint4 &wl = w[2 * t], &wh = w[2 * t + 1];
                    e2m1x8_to_f16(k == 0 ? wl.x : k == 1 ? wl.y : k == 2 ? wl.z : wl.w, lo);
                    e2m1x8_to_f16(k == 0 ? wh.x : k == 1 ? wh.y : k == 2 ? wh.z : wh.w, hi);
#pragma unroll
                    for (int i = 0; i < 4; ++i) { lo[i] = mul_f16x2(lo[i], mul[2 * t]); hi[i] = mul_f16x2(hi[i], mul[2 * t + 1]); }
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            mma_16816_f16(part[t][nt], lo[2 * h], hi[2 * h], lo[2 * h + 1], hi[2 * h + 1], xw[nt][2 * h], xw[nt][2 * h + 1]);
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float2 xf = *reinterpret_cast<const float2*>(x_scale + (u - p0) * 8 * NT + nt * 8 + 2 * j);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        acc[t][nt][i] = fmaf(part[t][nt][i] * factor[2 * t + (i >> 1)], (i & 1) ? xf.y : xf.x, acc[t][nt][i]);
            }
        }
    }

    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    float* sums = reinterpret_cast<float*>(w4_smem) + own_tile * (2 * 8 * NT * 128);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sums[(half * 8 * NT + nt * 8 + 2 * j + (i & 1)) * 128 + 32 * (2 * t + (i >> 1)) + 8 * (warp & 3) + g] = acc[t][nt][i];
    if (splits > 1) cluster_sync_all(); else __syncthreads();

    // Two rows of a column at a time; the partial sums of four CTAs are on the way together and are added in order.  Peers may go on
    // with this CTA's shared memory gone once they have read it, so all meet again after the reads, not after the stores.
    const int stride = NarrowColumn<GLU>::kStep * splits;
    bool met = splits == 1;
    for (int c = col.first + rank * NarrowColumn<GLU>::kStep; c < rows; c += 2 * stride) {
        float v[2] = {0.f, 0.f}, u[2] = {0.f, 0.f};
        for (int q0 = 0; q0 < splits; q0 += 4) {
            float x[4][2][2], y[4][2][2];
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        x[q][h][k] = y[q][h][k] = 0.f;
                        if (q0 + q >= splits || c + k * stride >= rows) continue;
                        const float* at = sums + (h * 8 * NT + c + k * stride) * 128 + col.r;
                        if (splits > 1) {
                            const uint32_t far = mapa_shared(smem_u32(at), (uint32_t)(q0 + q));
                            x[q][h][k] = ld_cluster_f32(far);
                            if (GLU) y[q][h][k] = ld_cluster_f32(far + 128u);
                        } else {
                            x[q][h][k] = at[0];
                            if (GLU) y[q][h][k] = at[32];
                        }
                    }
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        v[k] += x[q][h][k];
                        if (GLU) u[k] += y[q][h][k];
                    }
        }
        if (c + 2 * stride >= rows && !met) {
            met = true;
            asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        }
        col.template write<2>(p.lin.epi, m0 + c, stride, (rows - c + stride - 1) / stride, nullptr, v, u);
    }
    if (splits > 1) {
        if (!met) asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
}

}  // namespace kq
