// Layer norm and its gradient (include/dlion_layers.h).
//
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(var + eps)
//   with h = (x - mean) rstd and u = w dy:  dx = rstd (u - mean(u) - h mean(u h)) + r,  dw = sum dy h,  db = sum dy
//
// Bound by memory: every value is read once and stays in registers, all arithmetic is binary32.
#include <climits>

#include "layers_math.cuh"
#include "product_host.h"

namespace {

using namespace dlion;
using namespace dlion::prod;
using bf16 = __nv_bfloat16;

constexpr int64_t kMost = int64_t{1} << 30;
constexpr int kBlock = 256;

bool type_ok(int t) { return t == DLION_GRAD_F32 || t == DLION_GRAD_BF16; }
int type_bytes(int t) { return t == DLION_GRAD_F32 ? 4 : 2; }
bool ld_ok(int64_t ld, int64_t rows, int64_t cols) { return ld >= 0 && ld <= (int64_t{1} << 40) && (rows <= 1 || ld >= cols); }

// Eight values of a row, as a thread holds them until they are used.
template <class T>
struct Eight;
template <>
struct Eight<bf16> {
    uint4 w;
    __device__ __forceinline__ void get(float (&v)[8]) const { widen(w, v); }
};
template <>
struct Eight<float> {
    float v8[8];
    __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v8[i];
    }
};

// The columns of thread t of a row's g threads.  WIDE: eight adjacent ones at a time, by 16-byte accesses.  Otherwise (rows off the
// 16-byte grid) single ones, g apart, so that a warp's accesses are adjacent.
template <bool WIDE>
struct Columns {
    int64_t n;
    int t, g;
    __device__ __forceinline__ int64_t at(int c, int e) const { return WIDE ? (static_cast<int64_t>(c) * g + t) * 8 + e : (static_cast<int64_t>(c) * 8 + e) * g + t; }

    __device__ __forceinline__ void load(const bf16* p, int c, Eight<bf16>& o) const {
        if (WIDE) {
            o.w = at(c, 0) < n ? *reinterpret_cast<const uint4*>(p + at(c, 0)) : make_uint4(0, 0, 0, 0);
        } else {
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = at(c, e) < n ? reinterpret_cast<const uint16_t*>(p)[at(c, e)] : 0u;
            o.w = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
    }
    __device__ __forceinline__ void load(const float* p, int c, Eight<float>& o) const {
        if (WIDE) {
            const bool in = at(c, 0) < n;
            const float4* q = reinterpret_cast<const float4*>(p + at(c, 0));
            const float4 a = in ? q[0] : make_float4(0, 0, 0, 0), b = in ? q[1] : make_float4(0, 0, 0, 0);
            o.v8[0] = a.x, o.v8[1] = a.y, o.v8[2] = a.z, o.v8[3] = a.w;
            o.v8[4] = b.x, o.v8[5] = b.y, o.v8[6] = b.z, o.v8[7] = b.w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) o.v8[e] = at(c, e) < n ? p[at(c, e)] : 0.0f;
        }
    }
    // eight values of a vector of either type (`other` where there is none)
    __device__ __forceinline__ void vector(const void* p, int f32, int c, float other, float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = other;
        if (p == nullptr) return;
        if (f32) {
            Eight<float> o;
            load(static_cast<const float*>(p), c, o);
            o.get(v);
        } else {
            Eight<bf16> o;
            load(static_cast<const bf16*>(p), c, o);
            o.get(v);
        }
    }
    __device__ __forceinline__ void store(bf16* p, int c, const float (&v)[8]) const {
        if (WIDE) {
            if (at(c, 0) < n) {
                *reinterpret_cast<uint4*>(p + at(c, 0)) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (at(c, e) < n) p[at(c, e)] = __float2bfloat16_rn(v[e]);
            }
        }
    }
    __device__ __forceinline__ void store(float* p, int c, const float (&v)[8]) const {
        if (WIDE) {
            if (at(c, 0) < n) {
                float4* q = reinterpret_cast<float4*>(p + at(c, 0));
                q[0] = make_float4(v[0], v[1], v[2], v[3]);
                q[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (at(c, e) < n) p[at(c, e)] = v[e];
            }
        }
    }
};

// Sums over the g threads of a row (a power of two, 32 at least); every thread of the block calls it.
__device__ __forceinline__ float2 row_sum(float2 v, int g, float2* shared) {
#pragma unroll
    for (int d = 16; d >= 1; d /= 2) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, d);
    }
    if (g == 32) return v;
    const int warp = threadIdx.x / 32, each = g / 32;
    __syncthreads();                       // the last sums have been read
    if (threadIdx.x % 32 == 0) shared[warp] = v;
    __syncthreads();
    const float2* from = shared + warp / each * each;
    v = from[0];
    for (int i = 1; i < each; ++i) {
        v.x += from[i].x;
        v.y += from[i].y;
    }
    return v;
}

struct Norm {
    int64_t m, n;
    const void* x;
    int64_t x_ld;
    const void *w, *b;
    int w_f32, b_f32;
    float eps;
    void* y;
    int64_t y_ld;
    float* stats;                          // [2][m]
    int g;                                 // threads a row
};

// A row's CHUNKS x 8 values a thread stay in registers between the two sums of the variance.
template <class X, class Y, bool WIDE, int CHUNKS>
__global__ void __launch_bounds__(1024) norm_kernel(const __grid_constant__ Norm a) {
    __shared__ float2 sums[32];
    tc::let_next_start();
    tc::wait_for_previous();
    const int per = blockDim.x / a.g;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * per + threadIdx.x / a.g;
    const bool live = row < a.m;
    const Columns<WIDE> cols{live ? a.n : 0, static_cast<int>(threadIdx.x) & (a.g - 1), a.g};
    const X* x = static_cast<const X*>(a.x) + row * a.x_ld;
    Eight<X> held[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) cols.load(x, c, held[c]);
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        float v[8];
        held[c].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[e];
    }
    const float n = static_cast<float>(a.n), mean = row_sum(make_float2(s, 0.0f), a.g, sums).x / n;
    s = 0.0f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        float v[8];
        held[c].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = v[e] - mean;
            if (cols.at(c, e) < cols.n) s = __fmaf_rn(d, d, s);
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum(make_float2(s, 0.0f), a.g, sums).x / n + a.eps);
    if (!live) return;
    if (cols.t == 0) {
        a.stats[row] = mean;
        a.stats[a.m + row] = rstd;
    }
    Y* y = static_cast<Y*>(a.y) + row * a.y_ld;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        float v[8], w[8], b[8];
        held[c].get(v);
        cols.vector(a.w, a.w_f32, c, 1.0f, w);
        cols.vector(a.b, a.b_f32, c, 0.0f, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmaf_rn((v[e] - mean) * rstd, w[e], b[e]);
        cols.store(y, c, v);
    }
}

// Rows too wide for registers: a block reads its row three times.
template <class X, class Y, bool WIDE>
__global__ void __launch_bounds__(1024) norm_long_kernel(const __grid_constant__ Norm a) {
    __shared__ float2 sums[32];
    tc::let_next_start();
    tc::wait_for_previous();
    const int64_t row = blockIdx.x;
    const Columns<WIDE> cols{a.n, static_cast<int>(threadIdx.x), a.g};
    const X* x = static_cast<const X*>(a.x) + row * a.x_ld;
    const int chunks = static_cast<int>((a.n + a.g * 8 - 1) / (a.g * 8));
    const float n = static_cast<float>(a.n);
    float s = 0.0f;
    for (int c = 0; c < chunks; ++c) {
        Eight<X> o;
        float v[8];
        cols.load(x, c, o);
        o.get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[e];
    }
    const float mean = row_sum(make_float2(s, 0.0f), a.g, sums).x / n;
    s = 0.0f;
    for (int c = 0; c < chunks; ++c) {
        Eight<X> o;
        float v[8];
        cols.load(x, c, o);
        o.get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = v[e] - mean;
            if (cols.at(c, e) < a.n) s = __fmaf_rn(d, d, s);
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum(make_float2(s, 0.0f), a.g, sums).x / n + a.eps);
    if (threadIdx.x == 0) {
        a.stats[row] = mean;
        a.stats[a.m + row] = rstd;
    }
    Y* y = static_cast<Y*>(a.y) + row * a.y_ld;
    for (int c = 0; c < chunks; ++c) {
        Eight<X> o;
        float v[8], w[8], b[8];
        cols.load(x, c, o);
        o.get(v);
        cols.vector(a.w, a.w_f32, c, 1.0f, w);
        cols.vector(a.b, a.b_f32, c, 0.0f, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmaf_rn((v[e] - mean) * rstd, w[e], b[e]);
        cols.store(y, c, v);
    }
}

struct NormBack {
    int64_t m, n;
    const void* dy;
    int64_t dy_ld;
    const void* x;
    int64_t x_ld;
    const void* w;
    int w_f32;
    const float* stats;
    const void* residual;
    int64_t r_ld;
    void* dx;
    int64_t dx_ld;
    float* parts;                          // [blocks][2][n]: each block's share of dw and db; null if neither is wanted
    int g;
};

// A block takes every gridDim.x-th set of rows and keeps its share of dw and db in registers; the rows' sums are added in the
// order of the block's rows, the blocks' in the order of the blocks (norm_sums_kernel): the same result every time.
template <class X, class Y, bool WIDE, int CHUNKS>
__global__ void __launch_bounds__(512) norm_backward_kernel(const __grid_constant__ NormBack a) {
    extern __shared__ float total[];       // [2][n]
    __shared__ float2 sums[32];
    tc::let_next_start();
    tc::wait_for_previous();
    const int per = blockDim.x / a.g, group = threadIdx.x / a.g;
    const Columns<WIDE> all{a.n, static_cast<int>(threadIdx.x) & (a.g - 1), a.g};
    const float n = static_cast<float>(a.n);
    float dw[CHUNKS][8] = {}, db[CHUNKS][8] = {};
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * per; first < a.m; first += static_cast<int64_t>(gridDim.x) * per) {
        const int64_t row = first + group;
        const bool live = row < a.m;
        const Columns<WIDE> cols{live ? a.n : 0, all.t, a.g};
        Eight<X> x[CHUNKS], r[CHUNKS];
        Eight<Y> dy[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            cols.load(static_cast<const X*>(a.x) + row * a.x_ld, c, x[c]);
            cols.load(static_cast<const Y*>(a.dy) + row * a.dy_ld, c, dy[c]);
            if (a.residual != nullptr) cols.load(static_cast<const X*>(a.residual) + row * a.r_ld, c, r[c]);
        }
        const float mean = live ? a.stats[row] : 0.0f, rstd = live ? a.stats[a.m + row] : 0.0f;
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float v[8], d[8], w[8];
            x[c].get(v);
            dy[c].get(d);
            all.vector(a.w, a.w_f32, c, 1.0f, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = cols.at(c, e) < cols.n;
                const float h = in ? (v[e] - mean) * rstd : 0.0f, u = w[e] * d[e];
                dw[c][e] = __fmaf_rn(d[e], h, dw[c][e]);
                db[c][e] += d[e];
                s.x += u;
                s.y = __fmaf_rn(u, h, s.y);
            }
        }
        if (a.dx == nullptr) continue;
        s = row_sum(s, a.g, sums);
        const float along = s.x / n, turn = s.y / n;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float v[8], d[8], w[8], skip[8] = {};
            x[c].get(v);
            dy[c].get(d);
            all.vector(a.w, a.w_f32, c, 1.0f, w);
            if (a.residual != nullptr) r[c].get(skip);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float h = (v[e] - mean) * rstd;
                v[e] = __fmaf_rn(rstd, __fmaf_rn(-h, turn, __fmaf_rn(w[e], d[e], -along)), skip[e]);
            }
            cols.store(static_cast<X*>(a.dx) + row * a.dx_ld, c, v);
        }
    }
    if (a.parts == nullptr) return;
    for (int i = 0; i < per; ++i) {
        if (group == i) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t at = all.at(c, e);
                    if (at >= a.n) continue;
                    total[at] = i == 0 ? dw[c][e] : total[at] + dw[c][e];
                    total[a.n + at] = i == 0 ? db[c][e] : total[a.n + at] + db[c][e];
                }
            }
        }
        __syncthreads();
    }
    float* to = a.parts + static_cast<int64_t>(blockIdx.x) * 2 * a.n;
    for (int64_t i = threadIdx.x; i < 2 * a.n; i += blockDim.x) to[i] = total[i];
}

// Rows too wide for registers: a block a row for dx, which reads the row twice ...
template <class X, class Y, bool WIDE>
__global__ void __launch_bounds__(1024) norm_backward_long_kernel(const __grid_constant__ NormBack a) {
    __shared__ float2 sums[32];
    tc::let_next_start();
    tc::wait_for_previous();
    const int64_t row = blockIdx.x;
    const Columns<WIDE> cols{a.n, static_cast<int>(threadIdx.x), a.g};
    const X* x = static_cast<const X*>(a.x) + row * a.x_ld;
    const Y* dy = static_cast<const Y*>(a.dy) + row * a.dy_ld;
    const int chunks = static_cast<int>((a.n + a.g * 8 - 1) / (a.g * 8));
    const float n = static_cast<float>(a.n), mean = a.stats[row], rstd = a.stats[a.m + row];
    float2 s = make_float2(0.0f, 0.0f);
    float v[8], d[8], w[8], skip[8] = {};
    auto take = [&](int c) {
        Eight<X> ox;
        Eight<Y> oy;
        cols.load(x, c, ox);
        cols.load(dy, c, oy);
        ox.get(v);
        oy.get(d);
        cols.vector(a.w, a.w_f32, c, 1.0f, w);
    };
    for (int c = 0; c < chunks; ++c) {
        take(c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float h = cols.at(c, e) < a.n ? (v[e] - mean) * rstd : 0.0f, u = w[e] * d[e];
            s.x += u;
            s.y = __fmaf_rn(u, h, s.y);
        }
    }
    s = row_sum(s, a.g, sums);
    const float along = s.x / n, turn = s.y / n;
    for (int c = 0; c < chunks; ++c) {
        take(c);
        if (a.residual != nullptr) {
            Eight<X> o;
            cols.load(static_cast<const X*>(a.residual) + row * a.r_ld, c, o);
            o.get(skip);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float h = (v[e] - mean) * rstd;
            v[e] = __fmaf_rn(rstd, __fmaf_rn(-h, turn, __fmaf_rn(w[e], d[e], -along)), skip[e]);
        }
        cols.store(static_cast<X*>(a.dx) + row * a.dx_ld, c, v);
    }
}

// ... and a thread a column for dw and db: blocks of 128 columns by the gridDim.y shares of the rows.
template <class X, class Y>
__global__ void __launch_bounds__(128) norm_columns_kernel(const __grid_constant__ NormBack a) {
    tc::let_next_start();
    tc::wait_for_previous();
    const int64_t col = static_cast<int64_t>(blockIdx.x) * 128 + threadIdx.x;
    if (col >= a.n) return;
    float dw = 0.0f, db = 0.0f;
#pragma unroll 4
    for (int64_t row = blockIdx.y; row < a.m; row += gridDim.y) {
        const float d = static_cast<float>(static_cast<const Y*>(a.dy)[row * a.dy_ld + col]);
        const float h = (static_cast<float>(static_cast<const X*>(a.x)[row * a.x_ld + col]) - a.stats[row]) * a.stats[a.m + row];
        dw = __fmaf_rn(d, h, dw);
        db += d;
    }
    float* to = a.parts + static_cast<int64_t>(blockIdx.y) * 2 * a.n;
    to[col] = dw;
    to[a.n + col] = db;
}

// dw and db out of the blocks' shares: 32 columns a block, 32 threads a column.
struct NormSums {
    const float* parts;
    int64_t n;
    int count, f32;
    void *dw, *db;
};

__global__ void __launch_bounds__(1024) norm_sums_kernel(const __grid_constant__ NormSums a) {
    __shared__ float sum[32][33];
    tc::let_next_start();
    tc::wait_for_previous();
    const int lane = threadIdx.x % 32, line = threadIdx.x / 32;
    void* out = blockIdx.y == 0 ? a.dw : a.db;
    if (out == nullptr) return;
    const int64_t col = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    float s = 0.0f;
    if (col < a.n) {
        const float* p = a.parts + blockIdx.y * a.n + col;
#pragma unroll 8
        for (int i = line; i < a.count; i += 32) s += p[static_cast<int64_t>(i) * 2 * a.n];
    }
    sum[line][lane] = s;
    __syncthreads();
    s = sum[lane][line];                   // now a warp has a column
#pragma unroll
    for (int d = 16; d >= 1; d /= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
    const int64_t mine = static_cast<int64_t>(blockIdx.x) * 32 + line;
    if (lane == 0 && mine < a.n) {
        if (a.f32) {
            static_cast<float*>(out)[mine] = s;
        } else {
            static_cast<bf16*>(out)[mine] = __float2bfloat16_rn(s);
        }
    }
}

// ---------------------------------------------------------------- host
template <class F>
void with_types(int x_type, int y_type, F f) {
    if (x_type == DLION_GRAD_F32) {
        y_type == DLION_GRAD_F32 ? f(float{}, float{}) : f(float{}, bf16{});
    } else {
        y_type == DLION_GRAD_F32 ? f(bf16{}, float{}) : f(bf16{}, bf16{});
    }
}

bool wide(const void* p, int64_t ld, int type, int64_t rows) { return p == nullptr || (aligned16(p) && (rows <= 1 || ld * type_bytes(type) % 16 == 0)); }

// Threads a row, the fewest that hold it with `most` chunks of eight each; 0 if it is too wide for `threads`.
int group_of(int64_t n, int most, int threads) {
    for (int g = 32; g <= threads; g *= 2) {
        if (parts(n, static_cast<int64_t>(g) * 8) <= most) return g;
    }
    return 0;
}

dlion_status check(const dlion_norm_fwd* p) {
    if (p == nullptr || p->m < 0 || p->m > kMost || p->n < 1 || p->n > kMost) return DLION_EINVAL;
    if (!type_ok(p->x_type) || !type_ok(p->y_type) || (p->w != nullptr && !type_ok(p->w_type)) || (p->b != nullptr && !type_ok(p->b_type))) return DLION_EINVAL;
    if (!(p->eps >= 0.0f) || !(p->eps < INFINITY) || !ld_ok(p->x_ld, p->m, p->n) || !ld_ok(p->y_ld, p->m, p->n)) return DLION_EINVAL;
    if (p->m == 0) return DLION_OK;
    if (p->x == nullptr || p->y == nullptr || p->stats == nullptr) return DLION_EINVAL;
    if (!aligned(p->x, type_bytes(p->x_type)) || !aligned(p->y, type_bytes(p->y_type)) || !aligned(p->stats, 4)) return DLION_EALIGN;
    if (p->w != nullptr && !aligned(p->w, type_bytes(p->w_type))) return DLION_EALIGN;
    return p->b == nullptr || aligned(p->b, type_bytes(p->b_type)) ? DLION_OK : DLION_EALIGN;
}

void forward(Call& c, const dlion_norm_fwd& p) {
    if (p.m == 0 || !c.live()) return;
    Norm a{p.m, p.n, p.x, p.x_ld, p.w, p.b, p.w_type == DLION_GRAD_F32, p.b_type == DLION_GRAD_F32, p.eps, p.y, p.y_ld, p.stats, 0};
    const bool grid16 = p.n % 8 == 0 && wide(p.x, p.x_ld, p.x_type, p.m) && wide(p.y, p.y_ld, p.y_type, p.m) && wide(p.w, 0, 0, 1) && wide(p.b, 0, 0, 1);
    a.g = group_of(p.n, 4, 1024);
    with_types(p.x_type, p.y_type, [&](auto x, auto y) {
        using X = decltype(x);
        using Y = decltype(y);
        if (a.g == 0) {
            a.g = 1024;
            start(c, grid16 ? &norm_long_kernel<X, Y, true> : &norm_long_kernel<X, Y, false>, dim3(static_cast<unsigned>(p.m)), dim3(1024), 0, 1, a);
            return;
        }
        const int threads = std::max(a.g, kBlock);
        const dim3 grid(static_cast<unsigned>(parts(p.m, threads / a.g)));
        auto go = [&](auto* kernel) { start(c, kernel, grid, dim3(threads), 0, 1, a); };
        const int chunks = static_cast<int>(parts(p.n, a.g * 8));
        if (!grid16) {
            chunks <= 2 ? go(norm_kernel<X, Y, false, 2>) : go(norm_kernel<X, Y, false, 4>);
        } else if (chunks == 1) {
            go(norm_kernel<X, Y, true, 1>);
        } else if (chunks == 2) {
            go(norm_kernel<X, Y, true, 2>);
        } else {
            chunks == 3 ? go(norm_kernel<X, Y, true, 3>) : go(norm_kernel<X, Y, true, 4>);
        }
    });
}

dlion_status check(const dlion_norm_bwd* p) {
    if (p == nullptr || p->m < 0 || p->m > kMost || p->n < 1 || p->n > kMost) return DLION_EINVAL;
    if (!type_ok(p->x_type) || !type_ok(p->dy_type) || (p->w != nullptr && !type_ok(p->w_type)) || !type_ok(p->grad_type)) return DLION_EINVAL;
    if (!ld_ok(p->x_ld, p->m, p->n) || !ld_ok(p->dy_ld, p->m, p->n)) return DLION_EINVAL;
    if (p->dx != nullptr && (!ld_ok(p->dx_ld, p->m, p->n) || (p->residual != nullptr && !ld_ok(p->r_ld, p->m, p->n)))) return DLION_EINVAL;
    const int bytes = type_bytes(p->grad_type);
    if ((p->dw != nullptr && !aligned(p->dw, bytes)) || (p->db != nullptr && !aligned(p->db, bytes))) return DLION_EALIGN;
    if (p->m == 0) return DLION_OK;
    if (p->x == nullptr || p->dy == nullptr || p->stats == nullptr) return DLION_EINVAL;
    if (!aligned(p->x, type_bytes(p->x_type)) || !aligned(p->dy, type_bytes(p->dy_type)) || !aligned(p->stats, 4)) return DLION_EALIGN;
    if (p->w != nullptr && !aligned(p->w, type_bytes(p->w_type))) return DLION_EALIGN;
    if (p->dx != nullptr && (!aligned(p->dx, type_bytes(p->x_type)) || !aligned(p->residual, type_bytes(p->x_type)))) return DLION_EALIGN;
    return DLION_OK;
}

constexpr int kBackChunks = 3, kBackThreads = 512;

void backward(Call& c, const dlion_norm_bwd& p) {
    const bool sums = p.dw != nullptr || p.db != nullptr;
    if (p.m == 0) {                        // sums over no rows
        if (!c.live()) return;
        const size_t bytes = static_cast<size_t>(p.n) * type_bytes(p.grad_type);
        if (p.dw != nullptr) c.check(cudaMemsetAsync(p.dw, 0, bytes, c.stream));
        if (p.db != nullptr) c.check(cudaMemsetAsync(p.db, 0, bytes, c.stream));
        return;
    }
    if (p.dx == nullptr && !sums) return;
    NormBack a{p.m, p.n, p.dy, p.dy_ld, p.x, p.x_ld, p.w, p.w_type == DLION_GRAD_F32, p.stats, p.dx != nullptr ? p.residual : nullptr, p.r_ld, p.dx, p.dx_ld, nullptr, 0};
    const bool grid16 = p.n % 8 == 0 && wide(p.x, p.x_ld, p.x_type, p.m) && wide(p.dy, p.dy_ld, p.dy_type, p.m) && wide(p.w, 0, 0, 1) &&
                        wide(a.residual, p.r_ld, p.x_type, p.m) && wide(p.dx, p.dx_ld, p.x_type, p.m);
    a.g = group_of(p.n, kBackChunks, kBackThreads);
    const bool whole = a.g != 0;
    const int threads = std::max(a.g, kBlock);
    const int64_t blocks = whole ? std::min<int64_t>(parts(p.m, threads / a.g), 2 * c.sms) : std::min<int64_t>(p.m, 64);
    if (sums) a.parts = c.ws.take<float>(static_cast<uint64_t>(blocks) * 2 * p.n);
    if (!c.live()) return;
    with_types(p.x_type, p.dy_type, [&](auto x, auto y) {
        using X = decltype(x);
        using Y = decltype(y);
        if (!whole) {
            a.g = 1024;
            if (p.dx != nullptr) {
                start(c, grid16 ? &norm_backward_long_kernel<X, Y, true> : &norm_backward_long_kernel<X, Y, false>, dim3(static_cast<unsigned>(p.m)), dim3(1024), 0, 1, a);
            }
            if (sums) start(c, norm_columns_kernel<X, Y>, dim3(static_cast<unsigned>(parts(p.n, 128)), static_cast<unsigned>(blocks)), dim3(128), 0, 1, a);
            return;
        }
        const size_t shared = sums ? static_cast<size_t>(p.n) * 8 : 0;
        auto go = [&](auto* kernel) {
            if (shared > 48 * 1024) raise_shared(c, kernel, kBackChunks * 8 * kBackThreads * 8);
            start(c, kernel, dim3(static_cast<unsigned>(blocks)), dim3(threads), shared, 1, a);
        };
        const int chunks = static_cast<int>(parts(p.n, a.g * 8));
        if (!grid16) {
            chunks <= 2 ? go(&norm_backward_kernel<X, Y, false, 2>) : go(&norm_backward_kernel<X, Y, false, 3>);
        } else if (chunks == 1) {
            go(&norm_backward_kernel<X, Y, true, 1>);
        } else {
            chunks == 2 ? go(&norm_backward_kernel<X, Y, true, 2>) : go(&norm_backward_kernel<X, Y, true, 3>);
        }
    });
    if (!sums) return;
    const NormSums s{a.parts, p.n, static_cast<int>(blocks), p.grad_type == DLION_GRAD_F32, p.dw, p.db};
    start(c, norm_sums_kernel, dim3(static_cast<unsigned>(parts(p.n, 32)), 2), dim3(1024), 0, 1, s);
}

}  // namespace

extern "C" {

dlion_status dlion_norm_forward(const dlion_norm_fwd* p, void* cuda_stream) {
    const dlion_status st = check(p);
    return st != DLION_OK ? st : run(*p, forward, nullptr, 0, cuda_stream);
}

uint64_t dlion_norm_backward_workspace(const dlion_norm_bwd* p) { return check(p) == DLION_OK ? workspace_of(*p, backward) : 0; }

dlion_status dlion_norm_backward(const dlion_norm_bwd* p, void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
    const dlion_status st = check(p);
    return st != DLION_OK ? st : run(*p, backward, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
