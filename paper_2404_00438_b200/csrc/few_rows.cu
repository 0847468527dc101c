// Products of one to eight rows (a serving step): every weight is read once and used at most eight times, so the only
// question is how fast the weights stream.  No shared-memory ring and no copy descriptors: the weights go from global memory
// straight into the fragments of the warp-level 16 x 8 x 16 matrix instruction, whose k (or n) indices are
// renamed so that each thread's fragment is 16 adjacent bytes.  (One row on fused multiply-adds would do, eight rows
// would not: 64 of them, and 8 conversions, for every 16 bytes against the 23 bytes a clock that an SM streams.)
#include "product_host.h"

namespace dlion {
namespace prod {

namespace {

constexpr int kFewThreads = 256, kFewWarps = 8, kTokens = 8;

__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// eight adjacent values, `valid` of them there (the rest, or all of a negative count, 0); p on 16 bytes
__device__ __forceinline__ uint4 load8(const __nv_bfloat16* p, int valid) {
    if (valid >= 8) return __ldg(reinterpret_cast<const uint4*>(p));
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i < valid) w[i / 2] |= static_cast<uint32_t>(__ldg(reinterpret_cast<const unsigned short*>(p) + i)) << (16 * (i % 2));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row's 32 columns, a lane each, through the rest of the product (see Finish).
__device__ __forceinline__ void finish_row(const Finish& f, int row, int64_t col, float v) {
    const bool in = col < f.n;
    if (f.scale != nullptr) v *= *f.scale;
    if (f.bias != nullptr && in) {
        v += f.bias_f32 ? static_cast<const float*>(f.bias)[col] : __bfloat162float(static_cast<const __nv_bfloat16*>(f.bias)[col]);
    }
    if (f.keep == DLION_KEEP_8BIT) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, in ? __float_as_uint(v) & 0x7fffffffu : 0u);
        const uint32_t e = block_exponent(top);
        if (threadIdx.x % 32 == 0 && in) f.kept_e[(col / 32) * f.kept_e_ld + row] = static_cast<uint8_t>(e);
        if (in) static_cast<int8_t*>(f.kept)[row * f.kept_ld + col] = static_cast<int8_t>(quantise8(v, block_inverse(e)));
    } else if (f.keep == DLION_KEEP_BF16 && in) {
        static_cast<__nv_bfloat16*>(f.kept)[row * f.kept_ld + col] = __float2bfloat16_rn(v);
    }
    if (!in) return;
    with_act(f.act, [&](auto kind) { v = act_value<decltype(kind)::value>(v); });
    if (f.slope != DLION_ACT_NONE) {
        float u;
        if (f.saved8) {
            u = static_cast<float>(static_cast<const int8_t*>(f.saved)[row * f.saved_ld + col]) *
                block_scale(f.saved_e[(col / 32) * f.saved_e_ld + row]);
        } else {
            u = __bfloat162float(static_cast<const __nv_bfloat16*>(f.saved)[row * f.saved_ld + col]);
        }
        with_act(f.slope, [&](auto kind) { v *= act_slope<decltype(kind)::value>(u); });
    }
    if (f.residual != nullptr) v += __bfloat162float(f.residual[row * f.residual_ld + col]);
    if (f.out_f32) {
        static_cast<float*>(f.out)[row * f.out_ld + col] = v;
    } else {
        static_cast<__nv_bfloat16*>(f.out)[row * f.out_ld + col] = __float2bfloat16_rn(v);
    }
}

// Weights [n][k], k adjacent.  A block has 32 of the n at a time and its eight warps every eighth 32 of k.  Thread (g, q) = (lane / 4,
// lane % 4) loads k = 8 q .. 8 q + 7 of rows g, g + 8, g + 16, g + 24 and of token g: as fragments these are k pairs q, and q + 4,
// of two instructions, the same pairs on both sides.
__global__ void __launch_bounds__(kFewThreads, 3)
few_rows_along_k_kernel(const __nv_bfloat16* x, int64_t x_ld, const __nv_bfloat16* w, int64_t w_ld, int k, const __grid_constant__ Finish f) {
    __shared__ float part[kFewWarps][32][kTokens + 1];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, q = lane % 4;
    tc::let_next_start();
    tc::wait_for_previous();
    const __nv_bfloat16* xg = x + g * x_ld;
    const bool token = g < f.m;
    {
        const int u = blockIdx.x;
        const __nv_bfloat16* rows[4];
        bool there[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            there[r] = u * 32 + g + 8 * r < f.n;
            rows[r] = w + static_cast<int64_t>(u * 32 + g + 8 * r) * w_ld;
        }
        float c[2][4] = {};
#pragma unroll 3
        for (int at = warp * 32 + q * 8; at < k + 31; at += kFewWarps * 32) {        // whole warps leave together: at - 8 q is a multiple of 32
            if (at - q * 8 >= k) break;
            const int valid = k - at;
            uint4 a[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) a[r] = load8(rows[r] + at, there[r] ? valid : 0);
            const uint4 b = load8(xg + at, token ? valid : 0);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                mma_16x8x16(c[t], a[2 * t].x, a[2 * t + 1].x, a[2 * t].y, a[2 * t + 1].y, b.x, b.y);
                mma_16x8x16(c[t], a[2 * t].z, a[2 * t + 1].z, a[2 * t].w, a[2 * t + 1].w, b.z, b.w);
            }
        }
        __syncthreads();                       // the previous columns' sums have been read
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) part[warp][t * 16 + g + 8 * (i / 2)][2 * q + i % 2] = c[t][i];
        }
        __syncthreads();
        if (warp < f.m) {
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < kFewWarps; ++i) v += part[i][lane][warp];
            finish_row(f, warp, static_cast<int64_t>(u) * 32 + lane, v);
        }
    }
}

// Weights [k][n], n adjacent.  A cluster has 64 of the n, its warps every so many 16 of k.  Thread (g, q) loads n = 8 g .. 8 g + 7 of k =
// 2 q, 2 q + 1, 2 q + 8, 2 q + 9; column g of the eight instructions' j-th is n = 8 g + j.
__global__ void __launch_bounds__(kFewThreads, 3)
few_rows_along_n_kernel(const __nv_bfloat16* x, int64_t x_ld, const __nv_bfloat16* w, int64_t w_ld, int k, const __grid_constant__ Finish f) {
    __shared__ float part[kFewWarps][kTokens][65];
    __shared__ float total[kTokens][64];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, q = lane % 4;
    const int rank = static_cast<int>(tc::cluster_rank()), blocks = static_cast<int>(tc::cluster_size());
    const int n0 = static_cast<int>(blockIdx.x) / blocks * 64, cols = f.n - n0 - g * 8;
    tc::let_next_start();
    tc::wait_for_previous();
    const __nv_bfloat16* xg = x + g * x_ld;
    const __nv_bfloat16* wg = w + n0 + g * 8;
    const bool token = g < f.m;
    float c[8][4] = {};
#pragma unroll 2
    for (int at = (rank * kFewWarps + warp) * 16; at < k; at += blocks * kFewWarps * 16) {
        uint4 b[4];
        uint32_t a[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k0 = at + 2 * q + 8 * h;
            b[2 * h] = load8(wg + static_cast<int64_t>(k0) * w_ld, k0 < k ? cols : 0);
            b[2 * h + 1] = load8(wg + static_cast<int64_t>(k0 + 1) * w_ld, k0 + 1 < k ? cols : 0);
            if (!token || k0 >= k) {
                a[h] = 0;
            } else if (k0 + 1 < k) {
                a[h] = __ldg(reinterpret_cast<const unsigned int*>(xg + k0));
            } else {
                a[h] = __ldg(reinterpret_cast<const unsigned short*>(xg + k0));
            }
        }
        const uint32_t r0[4] = {b[0].x, b[0].y, b[0].z, b[0].w}, r1[4] = {b[1].x, b[1].y, b[1].z, b[1].w};
        const uint32_t r2[4] = {b[2].x, b[2].y, b[2].z, b[2].w}, r3[4] = {b[3].x, b[3].y, b[3].z, b[3].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            mma_16x8x16(c[2 * i], a[0], 0u, a[1], 0u, __byte_perm(r0[i], r1[i], 0x5410), __byte_perm(r2[i], r3[i], 0x5410));
            mma_16x8x16(c[2 * i + 1], a[0], 0u, a[1], 0u, __byte_perm(r0[i], r1[i], 0x7632), __byte_perm(r2[i], r3[i], 0x7632));
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        part[warp][g][16 * q + j] = c[j][0];
        part[warp][g][16 * q + 8 + j] = c[j][1];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float v = 0.0f;
#pragma unroll
        for (int s = 0; s < kFewWarps; ++s) v += part[s][warp][i * 32 + lane];
        total[warp][i * 32 + lane] = v;
    }
    if (blocks > 1) {
        tc::cluster_sync();
    } else {
        __syncwarp();
    }
    if (warp < f.m && warp % blocks == rank) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float v = 0.0f;
            if (blocks == 1) {
                v = total[warp][i * 32 + lane];
            } else {
                const uint32_t mine = tc::smem_addr(&total[warp][i * 32 + lane]);
                for (int r = 0; r < blocks; ++r) v += tc::load_cluster(tc::map_to_rank(mine, static_cast<uint32_t>(r)));
            }
            if (n0 + i * 32 < f.n) finish_row(f, warp, static_cast<int64_t>(n0) + i * 32 + lane, v);
        }
    }
    if (blocks > 1) tc::cluster_sync();        // the sums stay until they are read
}

}  // namespace

// Rows of k adjacent on both the tokens' side and one of the weights' two orders; nothing accumulated.
bool few_rows(Call& c, const Matrix& a, const Matrix& b, const Finish& f) {
    if (a.rows > kTokens || (a.cs != 1 && a.cols != 1) || f.accumulated != nullptr) return false;
    if (!c.live()) return true;
    const auto* x = static_cast<const __nv_bfloat16*>(a.p);
    const auto* w = static_cast<const __nv_bfloat16*>(b.p);
    const int k = static_cast<int>(a.cols);
    if (b.cs == 1) {
        const int64_t units = parts(b.rows, 32);
        start(c, few_rows_along_k_kernel, dim3(static_cast<unsigned>(units)), dim3(kFewThreads), 0, 1, x, a.rs, w,
              b.rs, k, f);
    } else {
        // so many blocks a cluster that the SMs have one each, as long as a warp keeps 16 of k
        const int64_t units = parts(b.rows, 64);
        int blocks = 1;
        while (blocks < 8 && units * blocks < c.sms && k > blocks * kFewWarps * 16) blocks *= 2;
        start(c, few_rows_along_n_kernel, dim3(static_cast<unsigned>(units * blocks)), dim3(kFewThreads), 0, blocks, x, a.rs, w, b.cs, k, f);
    }
    return true;
}

}  // namespace prod
}  // namespace dlion
