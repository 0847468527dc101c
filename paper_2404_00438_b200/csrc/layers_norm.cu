// Layer norm and its gradient (include/dlion_layers.h).
//
//   y = (x - mean) rstd w + b,  rstd = 1 / sqrt(var + eps)
//   with h = (x - mean) rstd and u = w dy:  dx = rstd (u - mean(u) - h mean(u h)) + r,  dw = sum dy h,  db = sum dy
//
// Bound by memory: every value is read once and stays in registers, all arithmetic is binary32.  The exceptions are rows too wide for
// registers: y beyond 32768 columns reads x three times, and beyond 8192 dx reads x, dy and w twice, and dw and db, in a kernel of their
// own, x and dy once more.
#include <climits>

#include "layers_math.cuh"
#include "product_host.h"

namespace {

using namespace dlion;
using namespace dlion::prod;
using bf16 = __nv_bfloat16;

constexpr int64_t kMost = int64_t{1} << 30;
constexpr int kBlock = 256, kWarpColumns = 2048;
constexpr int kRowsThreads = 512, kManyRows = 32, kManyWide = 2;     // rows an SM, and turns of wide rows, from which on blocks stay
constexpr int kBackThreads = 512;          // 128 registers a thread: a row's values and sums for as many columns

bool type_ok(int t) { return t == DLION_GRAD_F32 || t == DLION_GRAD_BF16; }
int type_bytes(int t) { return t == DLION_GRAD_F32 ? 4 : 2; }
bool ld_ok(int64_t ld, int64_t rows, int64_t cols) { return ld >= 0 && ld <= (int64_t{1} << 40) && (rows <= 1 || ld >= cols); }

// Eight values of a row, as a thread holds them until they are used.
template <class T>
struct Eight;
template <>
struct Eight<bf16> {
    uint4 w;
    __device__ __forceinline__ void get(float2 (&v)[4]) const { widen(w, v); }
};
template <>
struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void get(float2 (&v)[4]) const {
        v[0] = make_float2(a.x, a.y);
        v[1] = make_float2(a.z, a.w);
        v[2] = make_float2(b.x, b.y);
        v[3] = make_float2(b.z, b.w);
    }
};

// The columns of thread t of a row's G threads (0: `g`, known at run time).  WIDE: eight adjacent ones at a time, by 16-byte accesses.
// Otherwise (rows off the 16-byte grid) single ones, G apart, so that a warp's accesses are adjacent.
template <bool WIDE, int G>
struct Columns {
    int n, t, g;
    __device__ __forceinline__ int threads() const { return G != 0 ? G : g; }
    __device__ __forceinline__ int at(int c, int e) const { return WIDE ? (c * threads() + t) * 8 + e : (c * 8 + e) * threads() + t; }
    __device__ __forceinline__ bool whole(int c) const { return (c + 1) * 8 * threads() <= n; }    // for every thread of the row
    __device__ __forceinline__ bool has(int c, int e) const { return at(c, e) < n; }

    __device__ __forceinline__ void load(const bf16* p, int c, Eight<bf16>& o) const {
        if (WIDE) {
            o.w = has(c, 0) ? *reinterpret_cast<const uint4*>(p + at(c, 0)) : make_uint4(0, 0, 0, 0);
        } else {
            const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
            uint32_t w[8];
            if (whole(c)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = q[at(c, e)];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = has(c, e) ? q[at(c, e)] : 0u;
            }
            o.w = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
    }
    __device__ __forceinline__ void load(const float* p, int c, Eight<float>& o) const {
        if (WIDE) {
            const bool in = has(c, 0);
            const float4* q = reinterpret_cast<const float4*>(p + at(c, 0));
            o.a = in ? q[0] : make_float4(0, 0, 0, 0);
            o.b = in ? q[1] : make_float4(0, 0, 0, 0);
        } else {
            float v[8];
            if (whole(c)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = p[at(c, e)];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = has(c, e) ? p[at(c, e)] : 0.0f;
            }
            o.a = make_float4(v[0], v[1], v[2], v[3]);
            o.b = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
    // eight values of a vector of either type (`other` where there is none)
    __device__ __forceinline__ void vector(const void* p, int f32, int c, float other, float2 (&v)[4]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = twice(other);
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
    __device__ __forceinline__ void store(bf16* p, int c, const float2 (&v)[4]) const {
        if (WIDE) {
            if (has(c, 0)) {
                *reinterpret_cast<uint4*>(p + at(c, 0)) = make_uint4(pack_bf16(v[0].x, v[0].y), pack_bf16(v[1].x, v[1].y), pack_bf16(v[2].x, v[2].y), pack_bf16(v[3].x, v[3].y));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (has(c, e)) p[at(c, e)] = __float2bfloat16_rn(e % 2 ? v[e / 2].y : v[e / 2].x);
            }
        }
    }
    __device__ __forceinline__ void store(float* p, int c, const float2 (&v)[4]) const {
        if (WIDE) {
            if (has(c, 0)) {
                float4* q = reinterpret_cast<float4*>(p + at(c, 0));
                q[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
                q[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (has(c, e)) p[at(c, e)] = e % 2 ? v[e / 2].y : v[e / 2].x;
            }
        }
    }
    // differences from the mean; 0 in columns that are not there
    __device__ __forceinline__ void centre(int c, float mean, float2 (&v)[4]) const {
        const bool full = WIDE ? has(c, 0) : whole(c);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = add2(v[e], twice(-mean));
            if (!full) v[e] = make_float2(has(c, 2 * e) ? v[e].x : 0.0f, has(c, 2 * e + 1) ? v[e].y : 0.0f);
        }
    }
};

// Sums over the g threads of a row (a power of two, 32 at least), which are neighbours in the block and all call it.  `shared`: 32 values
// a block and turn; two turns, so that one barrier a sum is enough.
__device__ __forceinline__ float2 row_sum(float2 v, int g, float2 (*shared)[32], int turn) {
#pragma unroll
    for (int d = 16; d >= 1; d /= 2) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, d);
    }
    if (g == 32) return v;
    const int warp = threadIdx.x / 32, each = g / 32, first = warp / each * each;
    if (threadIdx.x % 32 == 0) shared[turn & 1][warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / each), "r"(g) : "memory");
    v = shared[turn & 1][first];
    for (int i = 1; i < each; ++i) {
        v.x += shared[turn & 1][first + i].x;
        v.y += shared[turn & 1][first + i].y;
    }
    return v;
}

struct Norm {
    int64_t m;
    int n;
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

// A row's CHUNKS x 8 values a thread, between the two sums of its variance.
template <class X, class Y, bool WIDE, int CHUNKS, int G, class F>
__device__ __forceinline__ void norm_row(const Norm& a, const Columns<WIDE, G>& cols, int g, float2 (*sums)[32], int turn, int64_t row, bool live,
                                         const Eight<X> (&held)[CHUNKS], F weights) {
    float2 v[CHUNKS][4], s = twice(0.0f);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        held[c].get(v[c]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = add2(s, v[c][e]);
    }
    const float n = static_cast<float>(a.n), mean = row_sum(make_float2(s.x + s.y, 0.0f), g, sums, turn).x / n;
    s = twice(0.0f);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        cols.centre(c, mean, v[c]);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fma2(v[c][e], v[c][e], s);
    }
    const float rstd = 1.0f / sqrtf(row_sum(make_float2(s.x + s.y, 0.0f), g, sums, turn + 1).x / n + a.eps);
    if (!live) return;
    if (cols.t == 0) {
        a.stats[row] = mean;
        a.stats[a.m + row] = rstd;
    }
    Y* y = static_cast<Y*>(a.y) + row * a.y_ld;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        float2 w[4], b[4];
        weights(c, w, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[c][e] = fma2(mul2(v[c][e], twice(rstd)), w[e], b[e]);
        cols.store(y, c, v[c]);
    }
}

// Few rows, or wide ones: a set of rows a block.  Up to 2048 columns a warp has a row (G = 32), and no barrier.
template <class X, class Y, bool WIDE, int CHUNKS, int G>
__global__ void __launch_bounds__(G != 0 ? 128 : 1024) norm_kernel(const __grid_constant__ Norm a) {
    __shared__ float2 sums[2][32];
    tc::let_next_start();
    tc::wait_for_previous();
    const int g = G != 0 ? G : a.g;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (blockDim.x / g) + threadIdx.x / g;
    const bool live = row < a.m;
    const Columns<WIDE, G> cols{live ? a.n : 0, static_cast<int>(threadIdx.x) & (g - 1), g};
    Eight<X> held[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) cols.load(static_cast<const X*>(a.x) + row * a.x_ld, c, held[c]);
    norm_row<X, Y, WIDE, CHUNKS, G>(a, cols, g, sums, 0, row, live, held, [&](int c, float2 (&w)[4], float2 (&b)[4]) {
        cols.vector(a.w, a.w_f32, c, 1.0f, w);
        cols.vector(a.b, a.b_f32, c, 0.0f, b);
    });
}

// Many rows of up to 16384 columns: one block an SM, G threads for every so many-th row, their next row on its way while they work on
// this one; weight and bias in shared memory, as binary32 and in the order in which the threads want them.  16384 x 2048 bf16: 27 us
// (134 MB, 5.0 TB/s; with 64 threads a row, two barriers and a block for each set of rows 42 us).  Against a block for each set of rows,
// us: 4000 x 8192 31, 38; off the 16-byte grid 2817 x 4450 28, 41, 700 x 4450 10.2, 13.3.  Binary32 rows of 1025 to 2048 columns
// spill 60 to 280 bytes a thread.
template <class X, class Y, bool WIDE, int CHUNKS, int G>
__global__ void __launch_bounds__(kRowsThreads, 1) norm_rows_kernel(const __grid_constant__ Norm a) {
    extern __shared__ float4 vectors[];    // [CHUNKS][4][G]: w, b of two columns
    __shared__ float2 sums[2][32];
    tc::let_next_start();
    tc::wait_for_previous();
    constexpr int kGroups = kRowsThreads / G;
    const int t = threadIdx.x % G, group = threadIdx.x / G;
    const Columns<WIDE, G> cols{a.n, t, G};
    const int64_t step = static_cast<int64_t>(gridDim.x) * kGroups;
    int64_t row = static_cast<int64_t>(blockIdx.x) * kGroups + group;
    Eight<X> now[CHUNKS], next[CHUNKS];
    auto load = [&](int64_t r, Eight<X> (&to)[CHUNKS]) {
        if (r >= a.m) return;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) cols.load(static_cast<const X*>(a.x) + r * a.x_ld, c, to[c]);
    };
    load(row, now);
    for (int c = group; c < CHUNKS; c += kGroups) {
        float2 w[4], b[4];
        cols.vector(a.w, a.w_f32, c, 1.0f, w);
        cols.vector(a.b, a.b_f32, c, 0.0f, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) vectors[(c * 4 + e) * G + t] = make_float4(w[e].x, w[e].y, b[e].x, b[e].y);
    }
    __syncthreads();
    for (; row < a.m; row += step) {       // (a group's threads leave together: its barriers are its own)
        load(row + step, next);
        norm_row<X, Y, WIDE, CHUNKS, G>(a, cols, G, sums, 0, row, true, now, [&](int c, float2 (&w)[4], float2 (&b)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 x = vectors[(c * 4 + e) * G + t];
                w[e] = make_float2(x.x, x.y);
                b[e] = make_float2(x.z, x.w);
            }
        });
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) now[c] = next[c];
    }
}

// Rows too wide for registers: a block reads its row three times.
template <class X, class Y, bool WIDE>
__global__ void __launch_bounds__(1024) norm_long_kernel(const __grid_constant__ Norm a) {
    __shared__ float2 sums[2][32];
    tc::let_next_start();
    tc::wait_for_previous();
    const int64_t row = blockIdx.x;
    const Columns<WIDE, 1024> cols{a.n, static_cast<int>(threadIdx.x), 1024};
    const X* x = static_cast<const X*>(a.x) + row * a.x_ld;
    const int chunks = (a.n + 8191) / 8192;
    const float n = static_cast<float>(a.n);
    float2 s = twice(0.0f), v[4];
    auto take = [&](int c) {
        Eight<X> o;
        cols.load(x, c, o);
        o.get(v);
    };
    for (int c = 0; c < chunks; ++c) {
        take(c);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = add2(s, v[e]);
    }
    const float mean = row_sum(make_float2(s.x + s.y, 0.0f), 1024, sums, 0).x / n;
    s = twice(0.0f);
    for (int c = 0; c < chunks; ++c) {
        take(c);
        cols.centre(c, mean, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fma2(v[e], v[e], s);
    }
    const float rstd = 1.0f / sqrtf(row_sum(make_float2(s.x + s.y, 0.0f), 1024, sums, 1).x / n + a.eps);
    if (threadIdx.x == 0) {
        a.stats[row] = mean;
        a.stats[a.m + row] = rstd;
    }
    Y* y = static_cast<Y*>(a.y) + row * a.y_ld;
    for (int c = 0; c < chunks; ++c) {
        float2 w[4], b[4];
        take(c);
        cols.vector(a.w, a.w_f32, c, 1.0f, w);
        cols.vector(a.b, a.b_f32, c, 0.0f, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fma2(mul2(add2(v[e], twice(-mean)), twice(rstd)), w[e], b[e]);
        cols.store(y, c, v);
    }
}

struct NormBack {
    int64_t m;
    int n;
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
    float* parts;                          // [blocks][2][n]: each block's share of dw and db; null if neither is wanted, or
    int joined;                            // the blocks, a cluster, that add their shares up themselves
    void *dw, *db;                         // joined: where to
    int grads_f32;
    int g;
};

__device__ __forceinline__ void copy16(void* to, const void* from, bool there) {       // 16 bytes, zero where they are not there
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_addr(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}

// What a thread has of a row, and how its next rows come.  On the 16-byte grid they come through shared memory, DEPTH rows ahead
// (each thread copies and reads only its own 16 bytes, so that it waits for nobody); elsewhere into registers, at once.
template <class X, class Y, bool WIDE, int CHUNKS>
struct NormRow {
    Eight<X> x[CHUNKS], r[CHUNKS];
    Eight<Y> dy[CHUNKS];
    float mean, rstd;
    static constexpr int kUnits = CHUNKS * (4 * sizeof(X) + 2 * sizeof(Y)) / 4;       // of 16 bytes a row
    static constexpr int kFit = 24 / kUnits;                         // rows a thread in some 200 KB
    static constexpr int kDepth = !WIDE ? 1 : kFit > 4 ? 4 : kFit > 2 ? kFit : 2;

    template <class C>
    __device__ __forceinline__ void ask(const NormBack& a, const C& all, int64_t row, uint4* ring, int stage) const {
        if (!WIDE) return;
        const int threads = static_cast<int>(blockDim.x);
        uint4* to = ring + stage * kUnits * threads + threadIdx.x;
        auto copy = [&](const auto* p, int c) {
            constexpr int kParts = sizeof(*p) / 2;
            const bool there = row < a.m && all.has(c, 0);
#pragma unroll
            for (int i = 0; i < kParts; ++i, to += threads) copy16(to, there ? reinterpret_cast<const uint4*>(p + all.at(c, 0)) + i : reinterpret_cast<const uint4*>(a.x), there);
        };
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            copy(static_cast<const X*>(a.x) + row * a.x_ld, c);
            copy(static_cast<const Y*>(a.dy) + row * a.dy_ld, c);
            if (a.residual != nullptr) copy(static_cast<const X*>(a.residual) + row * a.r_ld, c);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }

    template <class C>
    __device__ __forceinline__ void take(const NormBack& a, const C& all, int64_t row, const uint4* ring, int stage) {
        const bool live = row < a.m;
        mean = live ? a.stats[row] : 0.0f;
        rstd = live ? a.stats[a.m + row] : 0.0f;                     // a row that is not there: h = 0, dy = 0
        if (!WIDE) {
            const C cols{live ? all.n : 0, all.t, all.g};
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                cols.load(static_cast<const X*>(a.x) + row * a.x_ld, c, x[c]);
                cols.load(static_cast<const Y*>(a.dy) + row * a.dy_ld, c, dy[c]);
                if (a.residual != nullptr) cols.load(static_cast<const X*>(a.residual) + row * a.r_ld, c, r[c]);
            }
            return;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
        const int threads = static_cast<int>(blockDim.x);
        const uint4* from = ring + stage * kUnits * threads + threadIdx.x;
        auto read = [&](auto& to) {
            uint4* t = reinterpret_cast<uint4*>(&to);
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(to) / 16); ++i, from += threads) t[i] = *from;
        };
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            read(x[c]);
            read(dy[c]);
            if (a.residual != nullptr) read(r[c]);
        }
    }
};

// A block takes every gridDim.x-th set of rows and keeps its share of dw and db in registers; groups' and blocks' shares are added in
// their order, by norm_sums_kernel or, where a cluster has all the rows, by its blocks: the same result every time.  Bound by memory and, with
// one row a group under way, by the latency of a row's sums: 16384 x 2048 bf16 with a residual 56 us (268 MB, 4.8 TB/s); with
// a row ahead in registers and three groups 89 us; 4097 x 1001 binary32, off the 16-byte grid, 18 us (49 MB).  128 registers do not
// suffice for three chunks a thread (513 to 768 columns: 230 to 580 bytes spilled), nor off the grid for two of 256 or 512 threads.
template <class X, class Y, bool WIDE, int CHUNKS, int G>
__global__ void __launch_bounds__(kBackThreads, 1) norm_backward_kernel(const __grid_constant__ NormBack a) {
    extern __shared__ uint4 memory[];      // rows on their way; at the end the groups' dw and db
    __shared__ float2 sums[2][32];
    using Row = NormRow<X, Y, WIDE, CHUNKS>;
    tc::let_next_start();
    tc::wait_for_previous();
    const int g = G != 0 ? G : a.g, per = blockDim.x / g, group = threadIdx.x / g;
    const Columns<WIDE, G> all{a.n, static_cast<int>(threadIdx.x) & (g - 1), g};
    const float n = static_cast<float>(a.n);
    const float share = 1.0f / n;
    float2 dw[CHUNKS][4] = {}, db[CHUNKS][4] = {}, w[CHUNKS][4];
    const int64_t step = static_cast<int64_t>(gridDim.x) * per;
    Row now;
#pragma unroll
    for (int i = 0; i + 1 < Row::kDepth; ++i) now.ask(a, all, static_cast<int64_t>(blockIdx.x) * per + group + i * step, memory, i);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) all.vector(a.w, a.w_f32, c, 1.0f, w[c]);
    int turn = 0, stage = 0;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * per; first < a.m; first += step, ++turn) {
        const int64_t row = first + group;
        const bool live = row < a.m;
        now.ask(a, all, row + (Row::kDepth - 1) * step, memory, stage == 0 ? Row::kDepth - 1 : stage - 1);
        now.take(a, all, row, memory, stage);
        stage = stage + 1 == Row::kDepth ? 0 : stage + 1;
        float2 h[CHUNKS][4], u[CHUNKS][4], sx = twice(0.0f), sy = twice(0.0f);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            now.x[c].get(h[c]);
            now.dy[c].get(u[c]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {  // a column that is not there has dy = 0
                h[c][e] = mul2(add2(h[c][e], twice(-now.mean)), twice(now.rstd));
                dw[c][e] = fma2(u[c][e], h[c][e], dw[c][e]);
                db[c][e] = add2(db[c][e], u[c][e]);
                u[c][e] = mul2(u[c][e], w[c][e]);
                sx = add2(sx, u[c][e]);
                sy = fma2(u[c][e], h[c][e], sy);
            }
        }
        if (a.dx == nullptr) continue;
        const float2 s = row_sum(make_float2(sx.x + sx.y, sy.x + sy.y), g, sums, turn);
        const float2 along = twice(-s.x * share), turned = twice(-s.y * share);
        const Columns<WIDE, G> cols{live ? a.n : 0, all.t, g};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float2 skip[4] = {};
            if (a.residual != nullptr) now.r[c].get(skip);
#pragma unroll
            for (int e = 0; e < 4; ++e) u[c][e] = fma2(twice(now.rstd), fma2(h[c][e], turned, add2(u[c][e], along)), skip[e]);
            cols.store(static_cast<X*>(a.dx) + row * a.dx_ld, c, u[c]);
        }
    }
    if (WIDE) asm volatile("cp.async.wait_all;" ::: "memory");
    if (a.parts == nullptr && a.joined == 0) return;
    float* total = reinterpret_cast<float*>(memory);                 // [per][2][n], then the block's in the first of them
    __syncthreads();
    float* mine = total + group * 2 * a.n;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        if (WIDE) {
            if (!all.has(c, 0)) continue;
            float4 *pw = reinterpret_cast<float4*>(mine + all.at(c, 0)), *pb = reinterpret_cast<float4*>(mine + a.n + all.at(c, 0));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                pw[h] = make_float4(dw[c][2 * h].x, dw[c][2 * h].y, dw[c][2 * h + 1].x, dw[c][2 * h + 1].y);
                pb[h] = make_float4(db[c][2 * h].x, db[c][2 * h].y, db[c][2 * h + 1].x, db[c][2 * h + 1].y);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!all.has(c, e)) continue;
                mine[all.at(c, e)] = e % 2 ? dw[c][e / 2].y : dw[c][e / 2].x;
                mine[a.n + all.at(c, e)] = e % 2 ? db[c][e / 2].y : db[c][e / 2].x;
            }
        }
    }
    __syncthreads();
    float* to = a.parts + static_cast<int64_t>(blockIdx.x) * 2 * a.n;
    for (int i = threadIdx.x; i < 2 * a.n; i += blockDim.x) {
        float s = total[i];
#pragma unroll 4
        for (int r = 1; r < per; ++r) s += total[r * 2 * a.n + i];
        if (a.joined != 0) {
            total[i] = s;
        } else {
            to[i] = s;
        }
    }
    if (a.joined != 0) {
        tc::cluster_sync();
        for (int i = static_cast<int>(blockIdx.x * blockDim.x + threadIdx.x); i < 2 * a.n; i += a.joined * static_cast<int>(blockDim.x)) {
            const uint32_t at = tc::smem_addr(total + i);
            float s = 0.0f;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                if (r < a.joined) s += tc::load_cluster(tc::map_to_rank(at, r));
            }
            void* out = i < a.n ? a.dw : a.db;
            const int col = i < a.n ? i : i - a.n;
            if (out == nullptr) continue;
            if (a.grads_f32) {
                static_cast<float*>(out)[col] = s;
            } else {
                static_cast<bf16*>(out)[col] = __float2bfloat16_rn(s);
            }
        }
        tc::cluster_sync();                // the shares stay until they are read
    }
}

// Rows too wide for registers: a block a row for dx, which reads the row twice (and stores what it has read the second time: dx may lie
// over dy or r) ...
template <class X, class Y, bool WIDE>
__global__ void __launch_bounds__(1024) norm_backward_long_kernel(const __grid_constant__ NormBack a) {
    __shared__ float2 sums[2][32];
    tc::let_next_start();
    tc::wait_for_previous();
    const int64_t row = blockIdx.x;
    const Columns<WIDE, 1024> cols{a.n, static_cast<int>(threadIdx.x), 1024};
    const X* x = static_cast<const X*>(a.x) + row * a.x_ld;
    const Y* dy = static_cast<const Y*>(a.dy) + row * a.dy_ld;
    const int chunks = (a.n + 8191) / 8192;
    const float n = static_cast<float>(a.n), mean = a.stats[row], rstd = a.stats[a.m + row];
    float2 h[4], u[4], sx = twice(0.0f), sy = twice(0.0f);
    auto take = [&](int c) {
        Eight<X> ox;
        Eight<Y> oy;
        float2 w[4];
        cols.load(x, c, ox);
        cols.load(dy, c, oy);
        ox.get(h);
        oy.get(u);
        cols.vector(a.w, a.w_f32, c, 1.0f, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {      // a column that is not there has dy = 0
            h[e] = mul2(add2(h[e], twice(-mean)), twice(rstd));
            u[e] = mul2(u[e], w[e]);
        }
    };
    for (int c = 0; c < chunks; ++c) {
        take(c);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sx = add2(sx, u[e]);
            sy = fma2(u[e], h[e], sy);
        }
    }
    const float2 s = row_sum(make_float2(sx.x + sx.y, sy.x + sy.y), 1024, sums, 0), along = twice(-s.x / n), turned = twice(-s.y / n);
    for (int c = 0; c < chunks; ++c) {
        float2 skip[4] = {};
        take(c);
        if (a.residual != nullptr) {
            Eight<X> o;
            cols.load(static_cast<const X*>(a.residual) + row * a.r_ld, c, o);
            o.get(skip);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = fma2(twice(rstd), fma2(h[e], turned, add2(u[e], along)), skip[e]);
        cols.store(static_cast<X*>(a.dx) + row * a.dx_ld, c, u);
    }
}

// ... and a thread a column for dw and db: blocks of 128 columns by the gridDim.y shares of the rows.
template <class X, class Y>
__global__ void __launch_bounds__(128) norm_columns_kernel(const __grid_constant__ NormBack a) {
    tc::let_next_start();
    tc::wait_for_previous();
    const int col = static_cast<int>(blockIdx.x) * 128 + static_cast<int>(threadIdx.x);
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
    int n, count, f32;
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
        const float* p = a.parts + static_cast<int64_t>(blockIdx.y) * a.n + col;
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
    Norm a{p.m, static_cast<int>(p.n), p.x, p.x_ld, p.w, p.b, p.w_type == DLION_GRAD_F32, p.b_type == DLION_GRAD_F32, p.eps, p.y, p.y_ld, p.stats, 0};
    const bool grid16 = p.n % 8 == 0 && wide(p.x, p.x_ld, p.x_type, p.m) && wide(p.y, p.y_ld, p.y_type, p.m) && wide(p.w, 0, 0, 1) && wide(p.b, 0, 0, 1);
    with_types(p.x_type, p.y_type, [&](auto x, auto y) {
        using X = decltype(x);
        using Y = decltype(y);
        auto rows = [&](auto* kernel, int units) {                   // chunks times threads a row
            const int shared = units * 4 * static_cast<int>(sizeof(float4));
            if (shared > 47 * 1024) raise_shared(c, kernel, shared);
            start(c, kernel, dim3(static_cast<unsigned>(c.sms)), dim3(kRowsThreads), shared, 1, a);
        };
        if (p.n <= kWarpColumns) {         // a warp a row
            auto go = [&](auto* kernel) { start(c, kernel, dim3(static_cast<unsigned>(parts(p.m, 4))), dim3(128), 0, 1, a); };
            const int chunks = static_cast<int>(parts(p.n, 256));
            if (p.m >= kManyRows * c.sms) {
                if (!grid16) {
                    chunks <= 2 ? rows(&norm_rows_kernel<X, Y, false, 2, 32>, 2 * 32) : chunks <= 4 ? rows(&norm_rows_kernel<X, Y, false, 4, 32>, 4 * 32) : rows(&norm_rows_kernel<X, Y, false, 8, 32>, 8 * 32);
                } else if (chunks <= 2) {
                    chunks == 1 ? rows(&norm_rows_kernel<X, Y, true, 1, 32>, 1 * 32) : rows(&norm_rows_kernel<X, Y, true, 2, 32>, 2 * 32);
                } else if (chunks <= 4) {
                    chunks == 3 ? rows(&norm_rows_kernel<X, Y, true, 3, 32>, 3 * 32) : rows(&norm_rows_kernel<X, Y, true, 4, 32>, 4 * 32);
                } else {
                    chunks <= 6 ? rows(&norm_rows_kernel<X, Y, true, 6, 32>, 6 * 32) : rows(&norm_rows_kernel<X, Y, true, 8, 32>, 8 * 32);
                }
                return;
            }
            if (!grid16) {
                chunks <= 2 ? go(&norm_kernel<X, Y, false, 2, 32>) : chunks <= 4 ? go(&norm_kernel<X, Y, false, 4, 32>) : go(&norm_kernel<X, Y, false, 8, 32>);
            } else if (chunks <= 2) {
                chunks == 1 ? go(&norm_kernel<X, Y, true, 1, 32>) : go(&norm_kernel<X, Y, true, 2, 32>);
            } else if (chunks <= 4) {
                chunks == 3 ? go(&norm_kernel<X, Y, true, 3, 32>) : go(&norm_kernel<X, Y, true, 4, 32>);
            } else {
                chunks <= 6 ? go(&norm_kernel<X, Y, true, 6, 32>) : go(&norm_kernel<X, Y, true, 8, 32>);
            }
            return;
        }
        a.g = group_of(p.n, 4, 1024);
        if (a.g == 0) {
            start(c, grid16 ? &norm_long_kernel<X, Y, true> : &norm_long_kernel<X, Y, false>, dim3(static_cast<unsigned>(p.m)), dim3(1024), 0, 1, a);
            return;
        }
        if (a.g <= 512 && p.m >= kManyWide * c.sms * (kRowsThreads / a.g)) {
            if (a.g == 128) {
                grid16 ? rows(&norm_rows_kernel<X, Y, true, 4, 128>, 4 * 128) : rows(&norm_rows_kernel<X, Y, false, 4, 128>, 4 * 128);
            } else if (a.g == 256) {
                grid16 ? rows(&norm_rows_kernel<X, Y, true, 4, 256>, 4 * 256) : rows(&norm_rows_kernel<X, Y, false, 4, 256>, 4 * 256);
            } else {
                grid16 ? rows(&norm_rows_kernel<X, Y, true, 4, 512>, 4 * 512) : rows(&norm_rows_kernel<X, Y, false, 4, 512>, 4 * 512);
            }
            return;
        }
        const int threads = std::max(a.g, kBlock);
        start(c, grid16 ? &norm_kernel<X, Y, true, 4, 0> : &norm_kernel<X, Y, false, 4, 0>, dim3(static_cast<unsigned>(parts(p.m, threads / a.g))), dim3(threads), 0, 1, a);
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

constexpr int kMostShared = 224 * 1024, kMostVectors = 16 * 768 * 8;

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
    NormBack a{p.m, static_cast<int>(p.n), p.dy, p.dy_ld, p.x, p.x_ld, p.w, p.w_type == DLION_GRAD_F32, p.stats, p.dx != nullptr ? p.residual : nullptr, p.r_ld, p.dx, p.dx_ld, nullptr, 0, p.dw, p.db, p.grad_type == DLION_GRAD_F32, 0};
    const bool grid16 = p.n % 8 == 0 && wide(p.x, p.x_ld, p.x_type, p.m) && wide(p.dy, p.dy_ld, p.dy_type, p.m) && wide(p.w, 0, 0, 1) &&
                        wide(a.residual, p.r_ld, p.x_type, p.m) && wide(p.dx, p.dx_ld, p.x_type, p.m);
    a.g = p.n <= 768 ? 32 : group_of(p.n, 2, 512);
    const bool whole = a.g != 0;
    // One block an SM, or smaller ones where the rows are so few that those have no more than one turn; or, where up to eight blocks
    // have no more than two, a cluster, which needs no second kernel and no workspace.
    const int units = (p.x_type == DLION_GRAD_F32 ? 4 : 2) + (p.dy_type == DLION_GRAD_F32 ? 2 : 1);       // of 16 bytes a chunk
    const int small = std::max(a.g, 128), large = a.g == 32 && units * 3 > 13 ? 384 : kBackThreads;          // two rows ahead have to fit
    const int64_t turns = whole ? parts(p.m, large / a.g) : 0;
    if (whole && sums && turns <= 16) {
        for (a.joined = 1; a.joined < 8 && a.joined < turns; a.joined *= 2) {
        }
    }
    const int threads = a.joined != 0 || (whole && parts(p.m, small / a.g) > 2 * c.sms) ? large : small;
    const int64_t blocks = a.joined != 0 ? a.joined
                           : whole       ? std::min<int64_t>(parts(p.m, threads / a.g), threads == 128 ? 2 * c.sms : c.sms)
                                         : std::min<int64_t>(p.m, 64);
    if (sums && a.joined == 0) a.parts = c.ws.take<float>(static_cast<uint64_t>(blocks) * 2 * p.n);
    if (!c.live()) return;
    with_types(p.x_type, p.dy_type, [&](auto x, auto y) {
        using X = decltype(x);
        using Y = decltype(y);
        if (!whole) {                      // the sums first: dx may lie over dy
            if (sums) start(c, norm_columns_kernel<X, Y>, dim3(static_cast<unsigned>(parts(p.n, 128)), static_cast<unsigned>(blocks)), dim3(128), 0, 1, a);
            if (p.dx != nullptr) {
                start(c, grid16 ? &norm_backward_long_kernel<X, Y, true> : &norm_backward_long_kernel<X, Y, false>, dim3(static_cast<unsigned>(p.m)), dim3(1024), 0, 1, a);
            }
            return;
        }
        const size_t vectors = sums ? static_cast<size_t>(p.n) * 8 * (threads / a.g) : 0;
        auto go = [&](auto* kernel, size_t ring, int most) {
            if (std::max(ring, vectors) > 47 * 1024) raise_shared(c, kernel, std::max(most, kMostVectors));
            start(c, kernel, dim3(static_cast<unsigned>(blocks)), dim3(threads), std::max(ring, vectors), std::max(a.joined, 1), a);
        };
        auto with = [&](auto chunk, auto threads_a_row) {
            constexpr int C = decltype(chunk)::value, G = decltype(threads_a_row)::value;
            using Row = NormRow<X, Y, true, C>;
            grid16 ? go(&norm_backward_kernel<X, Y, true, C, G>, static_cast<size_t>(Row::kDepth) * Row::kUnits * threads * 16, std::min(Row::kDepth * Row::kUnits * kBackThreads * 16, kMostShared))
                   : go(&norm_backward_kernel<X, Y, false, C, G>, 0, 0);
        };
        using std::integral_constant;
        const int chunks = static_cast<int>(parts(p.n, a.g * 8));
        if (a.g == 32) {
            if (chunks == 1) {
                with(integral_constant<int, 1>{}, integral_constant<int, 32>{});
            } else {
                chunks == 2 ? with(integral_constant<int, 2>{}, integral_constant<int, 32>{}) : with(integral_constant<int, 3>{}, integral_constant<int, 32>{});
            }
        } else if (a.g == 64) {
            with(integral_constant<int, 2>{}, integral_constant<int, 64>{});
        } else {
            a.g == 128 ? with(integral_constant<int, 2>{}, integral_constant<int, 128>{}) : with(integral_constant<int, 2>{}, integral_constant<int, 0>{});
        }
    });
    if (!sums || a.joined != 0) return;
    const NormSums s{a.parts, static_cast<int>(p.n), static_cast<int>(blocks), p.grad_type == DLION_GRAD_F32, p.dw, p.db};
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
