// The product with its epilogue, its gradient, and the 8-bit form (include/dlion_layers.h).
#include <algorithm>

#include "product_host.h"

namespace {

using namespace dlion;
using namespace dlion::prod;

constexpr int64_t kMost = int64_t{1} << 30;

bool size_ok(int64_t v, int64_t least) { return v >= least && v <= kMost; }
constexpr int64_t kMostCols = 65535 * 256;   // blocks along a grid's second axis
bool type_ok(int t) { return t == DLION_GRAD_F32 || t == DLION_GRAD_BF16; }
int type_bytes(int t) { return t == DLION_GRAD_F32 ? 4 : 2; }
bool stride_ok(int64_t s) { return s >= 0 && s <= (int64_t{1} << 40); }
bool ld_ok(int64_t ld, int64_t rows, int64_t cols) { return stride_ok(ld) && (rows <= 1 || ld >= cols); }

// The element-wise kernels take 32 rows x 256 columns a block: a thread has eight columns of four rows, all
// loads under way at once, and the block's 8 x 32 exponents go through shared memory, because a row's neighbours in
// the exponents' array are the next rows, not the next blocks.
constexpr int kTileRows = 32, kTileCols = 256;

__device__ __forceinline__ uint32_t extent(int64_t left, int most) { return static_cast<uint32_t>(left < most ? (left > 0 ? left : 0) : most); }

__device__ __forceinline__ uint4 narrow(const float (&v)[8]) {
    return make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// eight bf16 values at p, `valid` of them there (the rest 0); off the 16-byte grid, in words where words begin
__device__ __forceinline__ uint4 take16(const __nv_bfloat16* at, uint32_t valid, bool wide) {
    if (wide && valid == 8) return *reinterpret_cast<const uint4*>(at);
    const uint16_t* p = reinterpret_cast<const uint16_t*>(at);
    if (valid == 8 && (reinterpret_cast<uintptr_t>(p) & 3u) == 0) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(p);
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (valid == 8) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(p + 1);
        const uint32_t first = p[0], a = w[0], b = w[1], c = w[2], last = p[7];
        return make_uint4(first | (a << 16), __funnelshift_r(a, b, 16), __funnelshift_r(b, c, 16), (c >> 16) | (last << 16));
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        if (static_cast<uint32_t>(i) < valid) w[i / 2] |= static_cast<uint32_t>(p[i]) << (16 * (i % 2));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ void give16(__nv_bfloat16* at, const uint4& v, uint32_t valid, bool wide) {
    if (wide && valid == 8) {
        *reinterpret_cast<uint4*>(at) = v;
        return;
    }
    uint16_t* p = reinterpret_cast<uint16_t*>(at);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if (valid == 8 && (reinterpret_cast<uintptr_t>(p) & 3u) == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
    } else if (valid == 8) {
        p[0] = static_cast<uint16_t>(v.x);
#pragma unroll
        for (int i = 0; i < 3; ++i) reinterpret_cast<uint32_t*>(p + 1)[i] = __funnelshift_r(w[i], w[i + 1], 16);
        p[7] = static_cast<uint16_t>(v.w >> 16);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i) {
            if (static_cast<uint32_t>(i) < valid) p[i] = static_cast<uint16_t>(w[i / 2] >> (16 * (i % 2)));
        }
    }
}

__device__ __forceinline__ uint2 take8(const int8_t* at, uint32_t valid, bool wide) {
    if (wide && valid == 8) return *reinterpret_cast<const uint2*>(at);
    const uint8_t* p = reinterpret_cast<const uint8_t*>(at);
    if (valid == 8 && (reinterpret_cast<uintptr_t>(p) & 1u) != 0) {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p + 1);
        const uint32_t first = p[0], a = h[0], b = h[1], c = h[2], last = p[7];
        return make_uint2(first | (a << 8) | (b << 24), (b >> 8) | (c << 8) | (last << 24));
    }
    if (valid == 8) {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
        return make_uint2(h[0] | (static_cast<uint32_t>(h[1]) << 16), h[2] | (static_cast<uint32_t>(h[3]) << 16));
    }
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        if (static_cast<uint32_t>(i) < valid) w[i / 4] |= static_cast<uint32_t>(p[i]) << (8 * (i % 4));
    }
    return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void give8(int8_t* at, const uint2& v, uint32_t valid, bool wide) {
    if (wide && valid == 8) {
        *reinterpret_cast<uint2*>(at) = v;
        return;
    }
    uint8_t* p = reinterpret_cast<uint8_t*>(at);
    if (valid == 8 && (reinterpret_cast<uintptr_t>(p) & 1u) != 0) {
        uint16_t* h = reinterpret_cast<uint16_t*>(p + 1);
        p[0] = static_cast<uint8_t>(v.x);
        h[0] = static_cast<uint16_t>(v.x >> 8);
        h[1] = static_cast<uint16_t>((v.x >> 24) | (v.y << 8));
        h[2] = static_cast<uint16_t>(v.y >> 8);
        p[7] = static_cast<uint8_t>(v.y >> 24);
    } else if (valid == 8) {
        uint16_t* h = reinterpret_cast<uint16_t*>(p);
        h[0] = static_cast<uint16_t>(v.x);
        h[1] = static_cast<uint16_t>(v.x >> 16);
        h[2] = static_cast<uint16_t>(v.y);
        h[3] = static_cast<uint16_t>(v.y >> 16);
    } else {
        const uint32_t w[2] = {v.x, v.y};
#pragma unroll
        for (int i = 0; i < 7; ++i) {
            if (static_cast<uint32_t>(i) < valid) p[i] = static_cast<uint8_t>(w[i / 4] >> (8 * (i % 4)));
        }
    }
}

// act(u) as a bf16 operand.  Bound by memory, 2 (or 33/32) + 2 bytes a value; issue slots are 70 % busy.  8192 x 8192 from 8
// bits: 35 us plain, launched again and again (203 MB, 5.7 TB/s); with gelu, whose two special functions a value the loads do not
// cover, 40 us more for a call than without the operand, 47 us alone from cold caches.  Rows off the 16-byte grid take
// accesses of 2 and 4 bytes: 8192 x 2047 19.5 us, 8192 x 2048 7.8 us (from L2).
template <bool EIGHT, int ACT>
__global__ void __launch_bounds__(256) operand_kernel(const void* u, int64_t u_ld, const uint8_t* e, int64_t e_ld, int64_t m, int64_t k,
                                                      __nv_bfloat16* out, int64_t out_ld, int wide, int wide_out) {
    __shared__ uint8_t ex[8][kTileRows];
    tc::let_next_start();
    tc::wait_for_previous();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kTileRows, col0 = static_cast<int64_t>(blockIdx.y) * kTileCols;
    const int64_t col = col0 + lane * 8;
    const uint32_t valid = extent(k - col, 8);
    if (EIGHT) {
        if (row0 + lane < m && col0 + warp * 32 < k) ex[warp][lane] = e[(col0 / 32 + warp) * e_ld + row0 + lane];
    }
    uint4 w[4];
    uint2 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = row0 + warp + 8 * i;
        const uint32_t n = row < m ? valid : 0;
        if (EIGHT) {
            q[i] = take8(static_cast<const int8_t*>(u) + row * u_ld + col, n, wide);
        } else {
            w[i] = take16(static_cast<const __nv_bfloat16*>(u) + row * u_ld + col, n, wide);
        }
    }
    if (EIGHT) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = warp + 8 * i;
        if (row0 + r >= m || valid == 0) continue;
        float v[8];
        if (EIGHT) {
            const float s = block_scale(ex[lane / 4][r]);
            float a[4], b[4];
            restore4(q[i].x, s, a);
            restore4(q[i].y, s, b);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = a[j];
                v[j + 4] = b[j];
            }
        } else {
            widen(w[i], v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = act_value<ACT>(v[j]);
        give16(out + (row0 + r) * out_ld + col, narrow(v), valid, wide_out);
    }
}

// Rows of x into the 8-bit form: a block of 32 values is four neighbouring threads.  Bound by memory, 2 + 33/32 bytes a value:
// 8192 x 8192 35 us (203 MB, 5.8 TB/s); off the 16-byte grid 8192 x 2047 14.4 us, 8192 x 2048 9.5 us (to L2).
__global__ void __launch_bounds__(256) checkpoint8_kernel(const __nv_bfloat16* x, int64_t x_ld, int64_t m, int64_t k, int8_t* q,
                                                          int64_t q_ld, uint8_t* e, int64_t e_ld, int wide, int wide_out) {
    __shared__ uint8_t ex[8][kTileRows];
    tc::let_next_start();
    tc::wait_for_previous();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kTileRows, col0 = static_cast<int64_t>(blockIdx.y) * kTileCols;
    const int64_t col = col0 + lane * 8;
    const uint32_t valid = extent(k - col, 8);
    uint4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = row0 + warp + 8 * i;
        w[i] = take16(x + row * x_ld + col, row < m ? valid : 0, wide);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = warp + 8 * i;
        // bf16 sizes order as integers, NaN and infinity last: two at a time
        const uint32_t mask = 0x7fff7fffu;
        uint32_t two = __vmaxu2(__vmaxu2(w[i].x & mask, w[i].y & mask), __vmaxu2(w[i].z & mask, w[i].w & mask));
        two = __vmaxu2(two, __shfl_xor_sync(0xffffffffu, two, 1));
        two = __vmaxu2(two, __shfl_xor_sync(0xffffffffu, two, 2));
        const uint32_t top = max(two << 16, two & 0xffff0000u);
        const uint32_t scale = block_exponent(top);
        const float inv = block_inverse(scale);
        if (lane % 4 == 0) ex[lane / 4][r] = static_cast<uint8_t>(scale);
        float v[8];
        widen(w[i], v);
        if (scale == kTop8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = within8(v[j]);
        }
        const uint32_t o[2] = {bytes4(quantise8(v[0], inv), quantise8(v[1], inv), quantise8(v[2], inv), quantise8(v[3], inv)),
                               bytes4(quantise8(v[4], inv), quantise8(v[5], inv), quantise8(v[6], inv), quantise8(v[7], inv))};
        if (row0 + r >= m || valid == 0) continue;
        give8(q + (row0 + r) * q_ld + col, make_uint2(o[0], o[1]), valid, wide_out);
    }
    __syncthreads();
    if (row0 + lane < m && col0 + warp * 32 < k) e[(col0 / 32 + warp) * e_ld + row0 + lane] = ex[warp][lane];
}

// Sums over rows: a cluster of eight blocks has 64 columns, each block an eighth of the rows; the first adds the
// others' sums, in their order.  Bound by memory (8192 x 8192: 134 MB in 25 us, 5.4 TB/s).
constexpr int kSumBlocks = 8;

__global__ void __cluster_dims__(kSumBlocks, 1, 1) __launch_bounds__(256)
column_sums_kernel(const __nv_bfloat16* a, int64_t rs, int64_t cs, int64_t rows, int64_t cols, void* out, int f32, int wide) {
    __shared__ float sum[32][65];
    __shared__ __align__(16) float total[64];
    const int lane = threadIdx.x % 8, line = threadIdx.x / 8;             // 32 lines of 8 x 8 columns
    const uint32_t rank = tc::cluster_rank();
    const int64_t c0 = static_cast<int64_t>(blockIdx.x / kSumBlocks) * 64 + lane * 8;
    tc::let_next_start();
    tc::wait_for_previous();
    float v[8] = {};
    const int64_t first = static_cast<int64_t>(rank) * 32 + line;
    if (wide && c0 < cols && (c0 + 8 <= cols || c0 + 8 <= rs)) {
        // a row's last columns may share their 16 bytes with what lies between it and the next row; after the last row may be nothing
        const bool ragged = c0 + 8 > cols;
        const int64_t whole = ragged ? rows - 1 : rows;
        const uint4* p = reinterpret_cast<const uint4*>(a + first * rs + c0);
        const int64_t step = rs * (kSumBlocks * 32 / 8);
        int64_t r = first;
        for (; r + 7 * kSumBlocks * 32 < whole; r += 8 * kSumBlocks * 32, p += 8 * step) {
            uint4 w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = p[i * step];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x[8];
                widen(w[i], x);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += x[j];
            }
        }
        for (; r < whole; r += kSumBlocks * 32, p += step) {
            float x[8];
            widen(*p, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += x[j];
        }
        if (ragged && r == rows - 1) {
#pragma unroll
            for (int j = 0; j < 7; ++j) {
                if (c0 + j < cols) v[j] += __bfloat162float(a[r * rs + c0 + j]);
            }
        }
    } else {
        for (int64_t r = first; r < rows; r += kSumBlocks * 32) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (c0 + j < cols) v[j] += __bfloat162float(a[r * rs + (c0 + j) * cs]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[line][lane * 8 + j] = v[j];
    __syncthreads();
    if (threadIdx.x < 64) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += sum[i][threadIdx.x];
        total[threadIdx.x] = t;
    }
    tc::cluster_sync();
    const int64_t c = static_cast<int64_t>(blockIdx.x / kSumBlocks) * 64 + threadIdx.x;
    if (rank == 0 && threadIdx.x < 64 && c < cols) {
        const uint32_t mine = tc::smem_addr(total + threadIdx.x);
        float w[kSumBlocks], t = 0.0f;
#pragma unroll
        for (int i = 0; i < kSumBlocks; ++i) w[i] = tc::load_cluster(tc::map_to_rank(mine, i));
#pragma unroll
        for (int i = 0; i < kSumBlocks; ++i) t += w[i];
        if (f32) {
            static_cast<float*>(out)[c] = t;
        } else {
            static_cast<__nv_bfloat16*>(out)[c] = __float2bfloat16_rn(t);
        }
    }
    tc::cluster_sync();                        // the sums stay until they are read
}

void column_sums(Call& c, const Matrix& a, void* out, int type) {
    if (!c.live()) return;
    const int wide = a.cs == 1 && aligned16(a.p) && a.rs % 8 == 0;
    start(c, column_sums_kernel, dim3(static_cast<unsigned>(parts(a.cols, 64) * kSumBlocks)), dim3(256), 0, 1,
          static_cast<const __nv_bfloat16*>(a.p), a.rs, a.cs, a.rows, a.cols, out, type == DLION_GRAD_F32, wide);
}

void operand(Call& c, const void* u, int64_t u_ld, const uint8_t* e, int64_t e_ld, int eight, int act, int64_t m, int64_t k,
             __nv_bfloat16* out, int64_t out_ld) {
    const int wide = aligned(u, eight ? 8 : 16) && u_ld % 8 == 0, wide_out = aligned16(out) && out_ld % 8 == 0;
    const dim3 grid(static_cast<unsigned>(parts(m, kTileRows)), static_cast<unsigned>(parts(k, kTileCols)));
    auto go = [&](auto* kernel) { start(c, kernel, grid, dim3(256), 0, 1, u, u_ld, e, e_ld, m, k, out, out_ld, wide, wide_out); };
    switch (act) {
        case DLION_ACT_RELU: eight ? go(operand_kernel<true, DLION_ACT_RELU>) : go(operand_kernel<false, DLION_ACT_RELU>); break;
        case DLION_ACT_GELU: eight ? go(operand_kernel<true, DLION_ACT_GELU>) : go(operand_kernel<false, DLION_ACT_GELU>); break;
        case DLION_ACT_SILU: eight ? go(operand_kernel<true, DLION_ACT_SILU>) : go(operand_kernel<false, DLION_ACT_SILU>); break;
        default: eight ? go(operand_kernel<true, DLION_ACT_NONE>) : go(operand_kernel<false, DLION_ACT_NONE>); break;
    }
}

dlion_status check_forward(const dlion_linear_fwd* p) {
    if (p == nullptr || !size_ok(p->m, 0) || !size_ok(p->k, 1) || !size_ok(p->n, 1)) return DLION_EINVAL;
    if (p->act < DLION_ACT_NONE || p->act > DLION_ACT_SILU || p->keep < DLION_KEEP_NONE || p->keep > DLION_KEEP_8BIT) return DLION_EINVAL;
    if (!type_ok(p->y_type) || (p->bias != nullptr && !type_ok(p->bias_type))) return DLION_EINVAL;
    if (!stride_ok(p->x_rs) || !stride_ok(p->x_cs) || !stride_ok(p->w_rs) || !stride_ok(p->w_cs)) return DLION_EINVAL;
    if (!ld_ok(p->y_ld, p->m, p->n) || (p->residual != nullptr && !ld_ok(p->r_ld, p->m, p->n))) return DLION_EINVAL;
    if (p->keep != DLION_KEEP_NONE && !ld_ok(p->kept_ld, p->m, p->n)) return DLION_EINVAL;
    if (p->keep == DLION_KEEP_8BIT && !ld_ok(p->kept_e_ld, parts(p->n, 32), p->m)) return DLION_EINVAL;
    if (p->m == 0) return DLION_OK;
    if (p->x == nullptr || p->w == nullptr || p->y == nullptr) return DLION_EINVAL;
    if (p->keep != DLION_KEEP_NONE && p->kept == nullptr) return DLION_EINVAL;
    if (p->keep == DLION_KEEP_8BIT && p->kept_e == nullptr) return DLION_EINVAL;
    if (!aligned(p->x, 2) || !aligned(p->w, 2) || !aligned(p->y, type_bytes(p->y_type)) || !aligned(p->residual, 2)) return DLION_EALIGN;
    if (p->bias != nullptr && !aligned(p->bias, type_bytes(p->bias_type))) return DLION_EALIGN;
    if (p->keep == DLION_KEEP_BF16 && !aligned(p->kept, 2)) return DLION_EALIGN;
    return DLION_OK;
}

void forward(Call& c, const dlion_linear_fwd& p) {
    if (p.m == 0) return;
    const Matrix x = readable(c, Matrix{p.x, p.m, p.k, p.x_rs, p.x_cs});
    const Matrix w = readable(c, Matrix{p.w, p.k, p.n, p.w_rs, p.w_cs});
    Finish f{};
    f.bias = p.bias;
    f.bias_f32 = p.bias_type == DLION_GRAD_F32;
    f.act = p.act;
    f.keep = p.keep;
    f.kept = p.kept;
    f.kept_ld = p.kept_ld;
    f.kept_e = p.kept_e;
    f.kept_e_ld = p.kept_e_ld;
    f.residual = static_cast<const __nv_bfloat16*>(p.residual);
    f.residual_ld = p.r_ld;
    f.out = p.y;
    f.out_ld = p.y_ld;
    f.out_f32 = p.y_type == DLION_GRAD_F32;
    product(c, x, transposed(w), f);
}

bool rows_of_dw(const dlion_linear_bwd& p) { return p.dw_cs == 1 && (p.k == 1 || p.dw_rs >= p.n); }
bool cols_of_dw(const dlion_linear_bwd& p) { return p.dw_rs == 1 && (p.n == 1 || p.dw_cs >= p.k); }

dlion_status check_backward(const dlion_linear_bwd* p) {
    if (p == nullptr || !size_ok(p->m, 0) || !size_ok(p->k, 1) || !size_ok(p->n, 1)) return DLION_EINVAL;
    if (p->act < DLION_ACT_NONE || p->act > DLION_ACT_SILU) return DLION_EINVAL;
    if (p->k > kMostCols || (p->saved != DLION_KEEP_BF16 && p->saved != DLION_KEEP_8BIT)) return DLION_EINVAL;
    if (!type_ok(p->grad_type)) return DLION_EINVAL;
    if (!stride_ok(p->dy_rs) || !stride_ok(p->dy_cs)) return DLION_EINVAL;
    const bool needs_u = p->dw != nullptr || (p->dx != nullptr && p->act != DLION_ACT_NONE);
    if (p->dx != nullptr) {
        if (!stride_ok(p->w_rs) || !stride_ok(p->w_cs) || !ld_ok(p->dx_ld, p->m, p->k)) return DLION_EINVAL;
        if (p->residual != nullptr && !ld_ok(p->r_ld, p->m, p->k)) return DLION_EINVAL;
        if (p->m != 0 && p->w == nullptr) return DLION_EINVAL;
        if (!aligned(p->w, 2) || !aligned(p->dx, 2) || !aligned(p->residual, 2)) return DLION_EALIGN;
    }
    if (p->dw != nullptr) {
        if (!stride_ok(p->dw_rs) || !stride_ok(p->dw_cs)) return DLION_EINVAL;
        if (!rows_of_dw(*p) && !cols_of_dw(*p)) return DLION_EINVAL;
        if (!aligned(p->dw, type_bytes(p->grad_type))) return DLION_EALIGN;
    }
    if (p->db != nullptr && !aligned(p->db, type_bytes(p->grad_type))) return DLION_EALIGN;
    if (needs_u) {
        if (!ld_ok(p->u_ld, p->m, p->k) || (p->saved == DLION_KEEP_8BIT && !ld_ok(p->u_e_ld, parts(p->k, 32), p->m))) return DLION_EINVAL;
        if (p->m != 0 && (p->u == nullptr || (p->saved == DLION_KEEP_8BIT && p->u_e == nullptr))) return DLION_EINVAL;
        if (p->saved == DLION_KEEP_BF16 && !aligned(p->u, 2)) return DLION_EALIGN;
    }
    if (p->m == 0) return DLION_OK;
    if (p->dy == nullptr) return DLION_EINVAL;
    return aligned(p->dy, 2) ? DLION_OK : DLION_EALIGN;
}

void backward(Call& c, const dlion_linear_bwd& p) {
    if (p.dx == nullptr && p.dw == nullptr && p.db == nullptr) return;
    if (p.m == 0) {                            // sums over no rows
        if (!c.live()) return;
        const size_t el = type_bytes(p.grad_type);
        if (p.dw != nullptr) {
            const bool rows = rows_of_dw(p);
            c.check(cudaMemset2DAsync(p.dw, std::max<int64_t>(1, rows ? std::max(p.dw_rs, p.n) : std::max(p.dw_cs, p.k)) * el, 0,
                                      (rows ? p.n : p.k) * el, rows ? p.k : p.n, c.stream));
        }
        if (p.db != nullptr) c.check(cudaMemsetAsync(p.db, 0, p.n * el, c.stream));
        return;
    }
    const Matrix dy = readable(c, Matrix{p.dy, p.m, p.n, p.dy_rs, p.dy_cs});
    Matrix w{nullptr, p.k, p.n, 0, 0}, a{nullptr, p.m, p.k, 0, 0};
    Finish fx{}, fw{};
    if (p.dx != nullptr) {
        w = readable(c, Matrix{p.w, p.k, p.n, p.w_rs, p.w_cs});
        fx.slope = p.act;
        fx.saved8 = p.saved == DLION_KEEP_8BIT;
        fx.saved = p.u;
        fx.saved_ld = p.u_ld;
        fx.saved_e = p.u_e;
        fx.saved_e_ld = p.u_e_ld;
        fx.residual = static_cast<const __nv_bfloat16*>(p.residual);
        fx.residual_ld = p.r_ld;
        fx.out = p.dx;
        fx.out_ld = p.dx_ld;
    }
    // dw's type and order say how the two products are divided, of which dx alone has the same share
    const bool rows = rows_of_dw(p) || (p.dw == nullptr && !cols_of_dw(p));
    fw.out_f32 = p.grad_type == DLION_GRAD_F32;
    if (p.dw != nullptr) {
        if (p.saved == DLION_KEEP_BF16 && p.act == DLION_ACT_NONE) {
            a = readable(c, Matrix{p.u, p.m, p.k, p.u_ld, 1});
        } else {
            const int64_t ld = round_up(p.k, 8);
            __nv_bfloat16* out = c.ws.take<__nv_bfloat16>(static_cast<uint64_t>(p.m) * ld);
            if (c.live()) operand(c, p.u, p.u_ld, p.u_e, p.u_e_ld, p.saved == DLION_KEEP_8BIT, p.act, p.m, p.k, out, ld);
            a = Matrix{out, p.m, p.k, ld, 1};
        }
        fw.out = p.dw;
        fw.out_ld = rows ? p.dw_rs : p.dw_cs;
    }
    Beside beside{static_cast<const __nv_bfloat16*>(dy.p), dy.rs, static_cast<int>(p.m), static_cast<int>(p.n), p.db, p.grad_type == DLION_GRAD_F32, 0};
    if (p.db == nullptr || dy.cs != 1 || !aligned16(dy.p) || dy.rs % 8 != 0) beside.out = nullptr;
    const bool summed = products(c, Part{dy, w, fx, p.dx != nullptr}, Part{transposed(rows ? a : dy), transposed(rows ? dy : a), fw, p.dw != nullptr}, beside);
    if (p.db != nullptr && !summed) column_sums(c, dy, p.db, p.grad_type);
}

}  // namespace

extern "C" {

uint64_t dlion_linear_forward_workspace(const dlion_linear_fwd* p) {
    return check_forward(p) == DLION_OK ? workspace_of(*p, forward) : 0;
}

dlion_status dlion_linear_forward(const dlion_linear_fwd* p, void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
    const dlion_status st = check_forward(p);
    return st != DLION_OK ? st : run(*p, forward, workspace, workspace_bytes, cuda_stream);
}

uint64_t dlion_linear_backward_workspace(const dlion_linear_bwd* p) {
    return check_backward(p) == DLION_OK ? workspace_of(*p, backward) : 0;
}

dlion_status dlion_linear_backward(const dlion_linear_bwd* p, void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
    const dlion_status st = check_backward(p);
    return st != DLION_OK ? st : run(*p, backward, workspace, workspace_bytes, cuda_stream);
}

dlion_status dlion_checkpoint8(const void* x, int64_t x_ld, int64_t m, int64_t k, int8_t* q, int64_t q_ld, uint8_t* e, int64_t e_ld,
                               void* cuda_stream) {
    if (!size_ok(m, 0) || !size_ok(k, 1) || k > kMostCols || !ld_ok(x_ld, m, k) || !ld_ok(q_ld, m, k) || !ld_ok(e_ld, parts(k, 32), m)) return DLION_EINVAL;
    if (m == 0) return DLION_OK;
    if (x == nullptr || q == nullptr || e == nullptr) return DLION_EINVAL;
    if (!aligned(x, 2)) return DLION_EALIGN;
    Call c;
    c.stream = static_cast<cudaStream_t>(cuda_stream);
    if (!device_of(c)) return DLION_ECUDA;
    const int wide = aligned16(x) && x_ld % 8 == 0, wide_out = aligned(q, 8) && q_ld % 8 == 0;
    const dim3 grid(static_cast<unsigned>(parts(m, kTileRows)), static_cast<unsigned>(parts(k, kTileCols)));
    start(c, checkpoint8_kernel, grid, dim3(256), 0, 1, static_cast<const __nv_bfloat16*>(x), x_ld, m, k, q, q_ld, e, e_ld, wide, wide_out);
    return c.status;
}

dlion_status dlion_restore8(const int8_t* q, int64_t q_ld, const uint8_t* e, int64_t e_ld, int64_t m, int64_t k, void* x, int64_t x_ld,
                            void* cuda_stream) {
    if (!size_ok(m, 0) || !size_ok(k, 1) || k > kMostCols || !ld_ok(x_ld, m, k) || !ld_ok(q_ld, m, k) || !ld_ok(e_ld, parts(k, 32), m)) return DLION_EINVAL;
    if (m == 0) return DLION_OK;
    if (x == nullptr || q == nullptr || e == nullptr) return DLION_EINVAL;
    if (!aligned(x, 2)) return DLION_EALIGN;
    Call c;
    c.stream = static_cast<cudaStream_t>(cuda_stream);
    if (!device_of(c)) return DLION_ECUDA;
    operand(c, q, q_ld, e, e_ld, 1, DLION_ACT_NONE, m, k, static_cast<__nv_bfloat16*>(x), x_ld);
    return c.status;
}

}  // extern "C"
