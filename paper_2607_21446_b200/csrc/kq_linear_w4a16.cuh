// The linear layer of kq_linear.cuh for a few rows in 16 bits and a weight in MXFP4, sm_100a:
//     acc[m][r] = sum_k x[m][k] w[r][k] 2^(sw[r][k/32] - 127),     then the same epilogue
//
// Bound by reading the weight (half a byte per element and a scale byte per 32): nothing else grows with N K.  With so few rows
// the tensor cores are there to keep up with memory, not for their rate, and mma.sync takes its operands from registers: weight rows as the
// 16 rows of the product, rows of x as its 8 columns, so that codes go from memory through the converter into the operand and are never
// stored again (an operand for tcgen05 has to lie in shared memory, in 16 bits: four times the bytes of the codes written and read).
//
// A CTA has 128 weight rows, one tile of the scale layout.  Warp w takes rows 32 q + 8 (w % 4) + g, q = 0..3, g = lane / 4, so that the 16
// scale bytes a lane loads are those of its four rows and no scale is fetched twice; lane j = lane % 4 of a quad takes block j of 128
// channels, 16 bytes of codes of each row.  The channels' order within the products is the lanes', which x follows in shared memory.
// The two halves of the warps take every other 128 channels, and the CTAs of a cluster runs of them; the partial sums
// meet in shared memory and are added in a fixed order.
//
// x in fp16: 128 channels of a row are scaled by a power of two that brings the largest to [2^14, 2^15).  fp16 then holds every bf16 and
// fp16 value exactly that is larger than 2^-28 of it; smaller ones are off by 2^-40 of it.  A weight's value is code times 2^(S - S0), S0 the largest of
// the row's four scale bytes: at most 2 significant bits, exact down to 2^-24.  2^(S0 - 127) and x's power multiply the fp32 sum of 128 channels.
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

constexpr int kW4Threads = 256;
constexpr int kW4Units = 24;             // of x in shared memory at a time
template <int NT> struct W4Smem {
    static constexpr int kXBytes = kW4Units * NT * 2048;                 // [unit][column tile][piece of 8 channels][lane] x 16 bytes
    static constexpr int kPartBytes = 2 * 8 * NT * 128 * 4;              // [half of the warps][row of x][weight row], in x's place
    static constexpr int kScaleOff = kXBytes > kPartBytes ? kXBytes : kPartBytes;
    static constexpr int kBytes = kScaleOff + kW4Units * 8 * NT * 4;
};

__device__ __forceinline__ uint4 w4_load(const uint8_t* p, bool exists) { return exists ? ld_stream_16(p) : make_uint4(0, 0, 0, 0); }

// grid: x = tiles of 128 weight rows times splits (a cluster), y = runs of 8 NT rows of x
template <bool GLU, int NT, bool XF16>
__global__ void __launch_bounds__(kW4Threads, 2) linear_w4a16_kernel(const __grid_constant__ W4A16Problem p, const int splits) {
    using L = W4Smem<NT>;
    extern __shared__ __align__(16) uint8_t w4_smem[];
    float* x_scale = reinterpret_cast<float*>(w4_smem + L::kScaleOff);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, j = lane & 3;
    const int rank = splits > 1 ? (int)cluster_ctarank() : 0;
    const int tile = (int)blockIdx.x / splits, m0 = (int)blockIdx.y * 8 * NT;
    const int rows = p.lin.M - m0 < 8 * NT ? p.lin.M - m0 : 8 * NT;
    const int u0 = (int)((int64_t)p.units * rank / splits), u1 = (int)((int64_t)p.units * (rank + 1) / splits);
    const int half = warp >> 2, base_row = tile * 128 + 8 * (warp & 3) + g;
    const int blocks = p.K / 32;
    const int64_t pitch = p.K / 2;
    const uint8_t* scales = p.scales + ((int64_t)tile * p.units * 512) + (8 * (warp & 3) + g) * 16;
    const uint8_t* codes = p.codes + (int64_t)base_row * pitch + 16 * j;
    pdl_launch_dependents();
    pdl_wait_prior_grid();

    uint4 w[2][4], sc[2];
    auto fetch = [&](int u, uint4 (&wr)[4], uint4& s) {
        const bool exists = u < u1 && 4 * u + j < blocks;
#pragma unroll
        for (int q = 0; q < 4; ++q) wr[q] = w4_load(codes + (int64_t)(32 * q) * pitch + (int64_t)u * 64, exists && base_row + 32 * q < p.lin.R);
        s = w4_load(scales + (int64_t)u * 512, u < u1);
    };
    fetch(u0 + half, w[0], sc[0]);
    fetch(u0 + half + 2, w[1], sc[1]);

    float acc[2][NT][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][nt][i] = 0.f;

    for (int p0 = u0; p0 < u1; p0 += kW4Units) {
        const int p1 = p0 + kW4Units < u1 ? p0 + kW4Units : u1;
        if (p0 != u0) __syncthreads();
        // x of these units: 16 lanes per row and unit, eight channels each
        for (int i = threadIdx.x; i < (p1 - p0) * 8 * NT * 16; i += kW4Threads) {
            const int piece = i & 15, m = (i >> 4) % (8 * NT), ul = (i >> 4) / (8 * NT);
            const int ch = (p0 + ul) * 128 + 8 * piece;
            uint32_t r[4] = {0, 0, 0, 0};
            if (m < rows && ch < p.K) {
                const uint16_t* at = static_cast<const uint16_t*>(p.x) + (int64_t)(m0 + m) * p.ld_x + ch;
                if (p.x_vec) {
                    const uint4 v = __ldg(reinterpret_cast<const uint4*>(at));
                    r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) r[k] = (uint32_t)at[2 * k] | ((uint32_t)at[2 * k + 1] << 16);
                }
            }
            float v[8];
            widen8_any<XF16>(make_uint4(r[0], r[1], r[2], r[3]), v);
            float amax = absmax8(v);
            const uint32_t group = 0xFFFFu << (lane & 16);
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(group, amax, o));
            int e = (int)(__float_as_uint(amax) >> 23) - 127;
            e = e < -112 ? -112 : e;
            const float up = exp2_int(14 - e);
            uint32_t h[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const __half2 two = __floats2half2_rn(v[2 * k] * up, v[2 * k + 1] * up);
                h[k] = *reinterpret_cast<const uint32_t*>(&two);
            }
            const int to = ((ul * NT + (m >> 3)) * 4 + (piece & 3)) * 32 + (m & 7) * 4 + (piece >> 2);
            reinterpret_cast<uint4*>(w4_smem)[to] = make_uint4(h[0], h[1], h[2], h[3]);
            if (piece == 0) x_scale[ul * 8 * NT + m] = exp2_int(e - 14);
        }
        __syncthreads();
        // (units of this warp in the pass: p0 + half, p0 + half + 2, ...; kW4Units is even, so the order goes on over passes)
        for (int u = p0 + half; u < p1; u += 4) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int uu = u + 2 * b;
                if (uu >= p1) break;
                const int left = blocks - 4 * uu;                        // blocks of this unit
                const uint32_t mask = left >= 4 ? 0xFFFFFFFFu : (1u << (8 * left)) - 1u;
                const uint32_t sw[4] = {sc[b].x & mask, sc[b].y & mask, sc[b].z & mask, sc[b].w & mask};
                uint32_t mul[4];
                float factor[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int s0 = (int)(sw[q] & 0xFFu), s1 = (int)((sw[q] >> 8) & 0xFFu), s2 = (int)((sw[q] >> 16) & 0xFFu), s3 = (int)(sw[q] >> 24);
                    const int top = max(max(s0, s1), max(s2, s3));
                    const int own = (int)((sw[q] >> (8 * j)) & 0xFFu);
                    const __half2 two = __half2half2(__float2half_rn(exp2_int(own - top)));
                    mul[q] = *reinterpret_cast<const uint32_t*>(&two);
                    factor[q] = exp2_int(top - 127);
                }
                float part[2][NT][4];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) part[t][nt][i] = 0.f;
                const uint4* xs = reinterpret_cast<const uint4*>(w4_smem) + (uu - p0) * NT * 128 + lane;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t xw[NT][4];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint4 v = xs[nt * 128 + k * 32];
                        xw[nt][0] = v.x; xw[nt][1] = v.y; xw[nt][2] = v.z; xw[nt][3] = v.w;
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        uint32_t lo[4], hi[4];
                        const uint4 &wl = w[b][2 * t], &wh = w[b][2 * t + 1];
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
                fetch(uu + 4, w[b], sc[b]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float2 xf = *reinterpret_cast<const float2*>(x_scale + (uu - p0) * 8 * NT + nt * 8 + 2 * j);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            acc[t][nt][i] = fmaf(part[t][nt][i] * factor[2 * t + (i >> 1)], (i & 1) ? xf.y : xf.x, acc[t][nt][i]);
                }
            }
        }
    }

    __syncthreads();
    float* sums = reinterpret_cast<float*>(w4_smem);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sums[(half * 8 * NT + nt * 8 + 2 * j + (i & 1)) * 128 + 32 * (2 * t + (i >> 1)) + 8 * (warp & 3) + g] = acc[t][nt][i];
    if (splits > 1) cluster_sync_all(); else __syncthreads();

    NarrowColumn<GLU> col;
    const LinearItem item = {0, 0, tile, 0, p.lin.M};
    col.open(p.lin, item, (int)threadIdx.x);
    const int stride = NarrowColumn<GLU>::kStep * splits;
    for (int c = col.first + rank * NarrowColumn<GLU>::kStep; c < rows; c += 2 * stride) {
        float v[2] = {0.f, 0.f}, u[2] = {0.f, 0.f};
        for (int q = 0; q < splits; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int m = c + k * stride;
                    if (m >= rows) continue;
                    const float* at = sums + (h * 8 * NT + m) * 128 + col.r;
                    if (splits > 1) {
                        const uint32_t far = mapa_shared(smem_u32(at), (uint32_t)q);
                        v[k] += ld_cluster_f32(far);
                        if (GLU) u[k] += ld_cluster_f32(far + 128u);
                    } else {
                        v[k] += at[0];
                        if (GLU) u[k] += at[32];
                    }
                }
        col.template write<2>(p.lin.epi, m0 + c, stride, (rows - c + stride - 1) / stride, nullptr, v, u);
    }
    if (splits > 1) cluster_sync_all();                                  // nobody's sums go away while a peer reads them
}

}  // namespace kq
