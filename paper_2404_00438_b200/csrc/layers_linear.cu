// The product with its epilogue, its gradient, and the 8-bit form (include/dlion_layers.h).
#include <algorithm>

#include "product_host.h"

namespace {

using namespace dlion;
using namespace dlion::prod;

constexpr int64_t kMost = int64_t{1} << 30;

bool size_ok(int64_t v, int64_t least) { return v >= least && v <= kMost; }
bool type_ok(int t) { return t == DLION_GRAD_F32 || t == DLION_GRAD_BF16; }
int type_bytes(int t) { return t == DLION_GRAD_F32 ? 4 : 2; }
bool stride_ok(int64_t s) { return s >= 0 && s <= (int64_t{1} << 40); }
bool ld_ok(int64_t ld, int64_t rows, int64_t cols) { return stride_ok(ld) && (rows <= 1 || ld >= cols); }

// act(u) as a bf16 operand, eight values a thread.  Bound by memory: 2 (or 33/32) + 2 bytes a value.
__global__ void __launch_bounds__(256) operand_kernel(const void* u, int64_t u_ld, const uint8_t* e, int64_t e_ld, int eight, int act,
                                                      int64_t m, int64_t k, __nv_bfloat16* out, int64_t out_ld, int wide) {
    const int64_t per_row = (k + 7) / 8;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = at / per_row, col = (at - row * per_row) * 8;
    if (row >= m) return;
    const int valid = static_cast<int>(k - col < 8 ? k - col : 8);
    float v[8];
    if (eight) {
        const int8_t* q = static_cast<const int8_t*>(u) + row * u_ld + col;
        const float s = block_scale(e[(col / 32) * e_ld + row]);
        int8_t b[8] = {};
        if (wide && valid == 8) {
            *reinterpret_cast<uint2*>(b) = *reinterpret_cast<const uint2*>(q);
        } else {
            for (int i = 0; i < valid; ++i) b[i] = q[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(b[i]) * s;
    } else {
        const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(u) + row * u_ld + col;
        if (wide && valid == 8) {
            const uint4 w = *reinterpret_cast<const uint4*>(p);
            const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = bf16_lo(x[i]);
                v[2 * i + 1] = bf16_hi(x[i]);
            }
        } else {
            for (int i = 0; i < 8; ++i) v[i] = i < valid ? __bfloat162float(p[i]) : 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_value(act, v[i]);
    __nv_bfloat16* o = out + row * out_ld + col;
    if (valid == 8 && on_grid(out, out_ld, 2)) {
        *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    } else {
        for (int i = 0; i < valid; ++i) o[i] = __float2bfloat16_rn(v[i]);
    }
}

// Rows of x into the 8-bit form: four threads a block of 32 values, eight values each.
__global__ void __launch_bounds__(256) checkpoint8_kernel(const __nv_bfloat16* x, int64_t x_ld, int64_t m, int64_t k, int8_t* q,
                                                          int64_t q_ld, uint8_t* e, int64_t e_ld, int wide) {
    const int64_t per_row = (k + 31) / 32 * 4;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t row = at / per_row, col = (at - row * per_row) * 8;
    const bool in = row < m;                    // whole groups of four threads
    const int valid = in && col < k ? static_cast<int>(k - col < 8 ? k - col : 8) : 0;
    float v[8] = {};
    if (valid != 0) {
        const __nv_bfloat16* p = x + row * x_ld + col;
        if (wide && valid == 8) {
            const uint4 w = *reinterpret_cast<const uint4*>(p);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = bf16_lo(u[i]);
                v[2 * i + 1] = bf16_hi(u[i]);
            }
        } else {
            for (int i = 0; i < valid; ++i) v[i] = __bfloat162float(p[i]);
        }
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    if (!in) return;
    const uint32_t ex = block_exponent(top);
    const float inv = block_inverse(ex);
    if (threadIdx.x % 4 == 0) e[(col / 32) * e_ld + row] = static_cast<uint8_t>(ex);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / 4] |= (static_cast<uint32_t>(quantise8(v[i], inv)) & 255u) << (8 * (i % 4));
    int8_t* o = q + row * q_ld + col;
    if (wide && valid == 8) {
        *reinterpret_cast<uint2*>(o) = make_uint2(w[0], w[1]);
    } else {
        for (int i = 0; i < valid; ++i) o[i] = static_cast<int8_t>(w[i / 4] >> (8 * (i % 4)));
    }
}

// Sums over rows in two steps, in a fixed order: a block has 256 columns and a run of rows.
__global__ void __launch_bounds__(256) column_sums_kernel(const __nv_bfloat16* a, int64_t rs, int64_t cs, int64_t rows, int64_t cols,
                                                          int64_t run, float* partial, int wide) {
    __shared__ float sum[8][257];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t c0 = static_cast<int64_t>(blockIdx.x) * 256 + lane * 8;
    const int64_t r0 = static_cast<int64_t>(blockIdx.y) * run, r1 = r0 + run < rows ? r0 + run : rows;
    float v[8] = {};
    if (wide && c0 + 8 <= cols) {
#pragma unroll 4
        for (int64_t r = r0 + warp; r < r1; r += 8) {
            const uint4 w = *reinterpret_cast<const uint4*>(a + r * rs + c0);
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] += bf16_lo(u[i]);
                v[2 * i + 1] += bf16_hi(u[i]);
            }
        }
    } else {
        for (int64_t r = r0 + warp; r < r1; r += 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (c0 + i < cols) v[i] += __bfloat162float(a[r * rs + (c0 + i) * cs]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[warp][lane * 8 + i] = v[i];
    __syncthreads();
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c >= cols) return;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) t += sum[i][threadIdx.x];
    partial[blockIdx.y * cols + c] = t;
}

__global__ void __launch_bounds__(256) join_sums_kernel(const float* partial, int runs, int64_t cols, void* out, int f32) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (c >= cols) return;
    float t = 0.0f;
#pragma unroll 8
    for (int i = 0; i < runs; ++i) t += partial[i * cols + c];
    if (f32) {
        static_cast<float*>(out)[c] = t;
    } else {
        static_cast<__nv_bfloat16*>(out)[c] = __float2bfloat16_rn(t);
    }
}

void column_sums(Call& c, const Matrix& a, void* out, int type) {
    const int64_t strips = parts(a.cols, 256);
    const int64_t runs = std::max<int64_t>(1, std::min<int64_t>(parts(4 * c.sms, strips), parts(a.rows, 64)));
    const int64_t run = std::max<int64_t>(1, parts(a.rows, runs));
    float* partial = c.ws.take<float>(static_cast<uint64_t>(runs) * a.cols);
    if (!c.live()) return;
    const int wide = a.cs == 1 && aligned16(a.p) && a.rs % 8 == 0;
    column_sums_kernel<<<dim3(static_cast<unsigned>(strips), static_cast<unsigned>(runs)), 256, 0, c.stream>>>(
        static_cast<const __nv_bfloat16*>(a.p), a.rs, a.cs, a.rows, a.cols, run, partial, wide);
    c.check(cudaGetLastError());
    join_sums_kernel<<<static_cast<unsigned>(strips), 256, 0, c.stream>>>(partial, static_cast<int>(runs), a.cols, out,
                                                                         type == DLION_GRAD_F32);
    c.check(cudaGetLastError());
}

void operand(Call& c, const void* u, int64_t u_ld, const uint8_t* e, int64_t e_ld, int eight, int act, int64_t m, int64_t k,
             __nv_bfloat16* out, int64_t out_ld) {
    const int wide = aligned(u, eight ? 8 : 16) && u_ld % 8 == 0;
    const int64_t blocks = parts(m * parts(k, 8), 256);
    operand_kernel<<<static_cast<unsigned>(blocks), 256, 0, c.stream>>>(u, u_ld, e, e_ld, eight, act, m, k, out, out_ld, wide);
    c.check(cudaGetLastError());
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

dlion_status check_backward(const dlion_linear_bwd* p) {
    if (p == nullptr || !size_ok(p->m, 0) || !size_ok(p->k, 1) || !size_ok(p->n, 1)) return DLION_EINVAL;
    if (p->act < DLION_ACT_NONE || p->act > DLION_ACT_SILU) return DLION_EINVAL;
    if (p->saved != DLION_KEEP_BF16 && p->saved != DLION_KEEP_8BIT) return DLION_EINVAL;
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
        const bool rows = p->dw_cs == 1 && (p->k == 1 || p->dw_rs >= p->n), cols = p->dw_rs == 1 && (p->n == 1 || p->dw_cs >= p->k);
        if (!rows && !cols) return DLION_EINVAL;
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
            const bool rows = p.dw_cs == 1 && (p.k == 1 || p.dw_rs >= p.n);
            c.check(cudaMemset2DAsync(p.dw, std::max<int64_t>(1, rows ? std::max(p.dw_rs, p.n) : std::max(p.dw_cs, p.k)) * el, 0,
                                      (rows ? p.n : p.k) * el, rows ? p.k : p.n, c.stream));
        }
        if (p.db != nullptr) c.check(cudaMemsetAsync(p.db, 0, p.n * el, c.stream));
        return;
    }
    const Matrix dy = readable(c, Matrix{p.dy, p.m, p.n, p.dy_rs, p.dy_cs});
    if (p.dx != nullptr) {
        const Matrix w = readable(c, Matrix{p.w, p.k, p.n, p.w_rs, p.w_cs});
        Finish f{};
        f.slope = p.act;
        f.saved8 = p.saved == DLION_KEEP_8BIT;
        f.saved = p.u;
        f.saved_ld = p.u_ld;
        f.saved_e = p.u_e;
        f.saved_e_ld = p.u_e_ld;
        f.residual = static_cast<const __nv_bfloat16*>(p.residual);
        f.residual_ld = p.r_ld;
        f.out = p.dx;
        f.out_ld = p.dx_ld;
        product(c, dy, w, f);
    }
    if (p.dw != nullptr) {
        Matrix a;
        if (p.saved == DLION_KEEP_BF16 && p.act == DLION_ACT_NONE) {
            a = readable(c, Matrix{p.u, p.m, p.k, p.u_ld, 1});
        } else {
            const int64_t ld = round_up(p.k, 8);
            __nv_bfloat16* out = c.ws.take<__nv_bfloat16>(static_cast<uint64_t>(p.m) * ld);
            if (c.live()) operand(c, p.u, p.u_ld, p.u_e, p.u_e_ld, p.saved == DLION_KEEP_8BIT, p.act, p.m, p.k, out, ld);
            a = Matrix{out, p.m, p.k, ld, 1};
        }
        Finish f{};
        f.out = p.dw;
        f.out_f32 = p.grad_type == DLION_GRAD_F32;
        if (p.dw_cs == 1 && (p.k == 1 || p.dw_rs >= p.n)) {
            f.out_ld = p.dw_rs;
            product(c, transposed(a), transposed(dy), f);
        } else {
            f.out_ld = p.dw_cs;
            product(c, transposed(dy), transposed(a), f);
        }
    }
    if (p.db != nullptr) column_sums(c, dy, p.db, p.grad_type);
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
    if (!size_ok(m, 0) || !size_ok(k, 1) || !ld_ok(x_ld, m, k) || !ld_ok(q_ld, m, k) || !ld_ok(e_ld, parts(k, 32), m)) return DLION_EINVAL;
    if (m == 0) return DLION_OK;
    if (x == nullptr || q == nullptr || e == nullptr) return DLION_EINVAL;
    if (!aligned(x, 2)) return DLION_EALIGN;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return DLION_ECUDA;
    const int wide = aligned16(x) && x_ld % 8 == 0 && aligned(q, 8) && q_ld % 8 == 0;
    checkpoint8_kernel<<<static_cast<unsigned>(parts(m * parts(k, 32) * 4, 256)), 256, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        static_cast<const __nv_bfloat16*>(x), x_ld, m, k, q, q_ld, e, e_ld, wide);
    return cudaGetLastError() == cudaSuccess ? DLION_OK : DLION_ECUDA;
}

dlion_status dlion_restore8(const int8_t* q, int64_t q_ld, const uint8_t* e, int64_t e_ld, int64_t m, int64_t k, void* x, int64_t x_ld,
                            void* cuda_stream) {
    if (!size_ok(m, 0) || !size_ok(k, 1) || !ld_ok(x_ld, m, k) || !ld_ok(q_ld, m, k) || !ld_ok(e_ld, parts(k, 32), m)) return DLION_EINVAL;
    if (m == 0) return DLION_OK;
    if (x == nullptr || q == nullptr || e == nullptr) return DLION_EINVAL;
    if (!aligned(x, 2)) return DLION_EALIGN;
    Call c;
    if (cudaGetDevice(&c.device) != cudaSuccess) return DLION_ECUDA;
    c.stream = static_cast<cudaStream_t>(cuda_stream);
    operand(c, q, q_ld, e, e_ld, 1, DLION_ACT_NONE, m, k, static_cast<__nv_bfloat16*>(x), x_ld);
    return c.status;
}

}  // extern "C"
