// Softmax cross entropy over a large vocabulary (include/dlion_layers.h, dlion_lm_loss).
//
// A piece of the rows at a time: one product gives the logits tile by tile, and its epilogue leaves, for
// each row and group of columns (half a tile), the maximum and the sum of exp(l - maximum), and each logit
// as a 16-bit distance below that maximum in steps of 2^-10 octaves (relative error of exp at most 3.4e-4, a
// sixth of the bf16 rounding that d gets anyway; what lies 64 octaves, 5e-20, below its group's maximum counts
// as 0, so that a word masked by a huge negative weight does not bring that weight into dx).  Once the rows' log-sum-exps are known the codes become d / g in bf16, in place, and two
// more products give dx and dw.  6 m h v operations instead of the 8 of computing the logits twice; the codes
// cost 6 bytes of traffic a logit, against the 6 h operations that the products spend on it.
#include <climits>
#include <cmath>

#include "product_host.h"

namespace {

using namespace dlion;
using namespace dlion::prod;

constexpr float kStep = 1024.0f;            // codes per octave
constexpr int64_t kPiece = 4096;
// Without gradients nothing is kept of a piece but its groups' maxima and sums, 8 bytes a row and group (0.1 GB at 50257 words): the
// largest batches alone are divided, whose products fill the GPU by far.
constexpr int64_t kEvalPiece = 32768;
constexpr int64_t kMost = int64_t{1} << 30;

struct LossTile {
    static constexpr bool kSplits = false;
    struct Args {
        int m, n;
        const int64_t* targets;
        unsigned int* blocks_done;          // set to 0 for the kernel that follows
        float2* stats;                      // [group][m]: maximum, sum of exp(l - maximum)
        float* at_target;                   // [m]
        uint16_t* codes;                    // nullable: [m][ld]
        int64_t ld;
    };

    using Ahead = int64_t;                  // this lane's target, asked for before the sums are waited for

    template <int WIDTH>
    static __device__ __forceinline__ Ahead ahead(const Args& p, int row0, int, int lane) {
        return row0 + lane < p.m ? p.targets[row0 + lane] : -1;
    }

    // MASKED: columns from `valid` on do not exist
    template <bool MASKED>
    static __device__ __forceinline__ float greatest(const float (&v)[32], int valid, float top) {
        float t[4] = {top, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (!MASKED || j < valid) t[j % 4] = fmaxf(t[j % 4], v[j]);
        }
        return fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
    }

    template <bool MASKED, bool CODES>
    static __device__ __forceinline__ float exponentials(const float (&v)[32], int valid, float top, uint32_t (&w)[16]) {
        float t[4] = {};
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const float x = v[j] - top;     // exact where it counts, near the maximum
            const float e = exp2_fast(x * kLog2e);
            if (!MASKED || j < valid) t[j % 4] += e;
            if (CODES) {
                // x <= 0: 1.5 * 2^23 + the distance leaves it, rounded, in the low bits
                const uint32_t u = __float_as_uint(fminf(__fmaf_rn(x, -kStep * kLog2e, 12582912.0f), 12582912.0f + 65535.0f));
                w[j / 2] = j % 2 == 0 ? u : __byte_perm(w[j / 2], u, 0x5410);
            }
        }
        return (t[0] + t[1]) + (t[2] + t[3]);
    }

    // Two passes over the accumulator, which is cheaper to read again than to hold: the maximum, then the exponentials.
    static __device__ __forceinline__ void tile(const Args& p, int64_t target, uint32_t acc, int row0, int col0, int width, bool live, uint4* stage, int lane) {
        if (row0 >= p.m || col0 >= p.n) return;
        if (row0 == 0 && col0 == 0 && lane == 0) *p.blocks_done = 0;
        const int row = row0 + lane;
        const int valid = min(width, p.n - col0);
        const int rows = live ? min(32, p.m - row0) : 0;
        const int hit = lane < rows && target >= col0 && target < col0 + valid ? static_cast<int>(target - col0) : -1;
        const bool codes = p.codes != nullptr;
        float top = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < valid; c += 32) {
            float v[32];
            tc::tmem_load32(acc + c, v);
            top = c + 32 <= valid ? greatest<false>(v, 32, top) : greatest<true>(v, valid - c, top);
            if (__any_sync(0xffffffffu, hit >= c && hit < c + 32)) {
                float l = 0.0f;
#pragma unroll
                for (int j = 0; j < 32; ++j) {          // a select each: indexed, the 32 sums would live in memory
                    asm("{\n.reg .pred p;\nsetp.eq.s32 p, %2, 0;\nselp.f32 %0, %1, %0, p;\n}" : "+f"(l) : "f"(v[j]), "r"(hit - c - j));
                }
                if (hit >= c && hit < c + 32) p.at_target[row] = l;
            }
            if (!live) break;
        }
        // The differences need a finite reference: a group masked whole by -infinity has none of its own, and sums to 0 against
        // any.  One masked by a finite value, the type's lowest even, keeps it, and vanishes when the groups are joined, unless
        // all of the row's words have it.  An infinity above makes the row NaN.
        const float zero = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll 1
        for (int c = 0; c < valid; c += 32) {
            float v[32];
            uint32_t w[16];
            tc::tmem_load32(acc + c, v);
            if (c + 32 > valid) {
                sum += exponentials<true, true>(v, valid - c, zero, w);
            } else if (codes) {
                sum += exponentials<false, true>(v, 32, zero, w);
            } else {
                sum += exponentials<false, false>(v, 32, zero, w);
            }
            if (codes) Piece{stage, lane, row0, col0 + c, rows, 32}.put16(w, p.codes, p.ld, true);      // ld covers the last tile
            if (!live) break;
        }
        if (lane < rows) p.stats[static_cast<int64_t>(col0 / width) * p.m + row] = make_float2(top, sum);
    }
};

constexpr int kRowThreads = 256;

__device__ __forceinline__ float block_sum(float v, float* shared) {       // kRowThreads threads, fixed order
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < kRowThreads / 32; ++i) v += shared[i];
    return v;
}

__device__ __forceinline__ int block_count(const int64_t* targets, int64_t m, int64_t ignore, int* shared) {
    int n = 0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < m; i += kRowThreads) n += targets[i] != ignore;
    n = __reduce_add_sync(0xffffffffu, n);
    if (threadIdx.x % 32 == 0) shared[threadIdx.x / 32] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int i = 0; i < kRowThreads / 32; ++i) n += shared[i];
    return n;
}

// factor[0] = scale / (rows with a target), where it is needed before the first piece's rows are done: one block, 8 bytes a row, latency
__global__ void __launch_bounds__(kRowThreads) factor_kernel(const int64_t* targets, int64_t m, int64_t ignore, int mean, float scale, float* factor) {
    __shared__ int counts[kRowThreads / 32];
    tc::let_next_start();
    tc::wait_for_previous();
    const int n = block_count(targets, m, ignore, counts);
    if (threadIdx.x == 0) factor[0] = mean && n > 0 ? scale / static_cast<float>(n) : scale;
}

// What the last block of a piece's rows does: the loss of all rows (after the last piece), in a fixed order, and the factor.
struct Last {
    unsigned int* blocks_done;             // 0 before the piece
    const float* rows;                     // of all pieces
    const int64_t* targets;
    int64_t m;
    int mean;
    float scale;
    float* loss;                           // nullable
    float* factor;                         // nullable
};

// Joins the groups of eight rows a block: thread (i, r) = (thread / 8, thread % 8) takes every 32nd group of row r, eight at a
// time; then each row's maximum, the sum's logarithm in octaves, and the loss.  Latency: 2048 rows of 394 groups 8 us, 6.5 MB.
__global__ void __launch_bounds__(kRowThreads) rows_kernel(const float2* stats, int groups, int64_t m, const int64_t* targets, int64_t ignore,
                                                           int64_t v, const float* at_target, float2* lse, float* rows, const Last end) {
    constexpr int kEvery = kRowThreads / 8, kBatch = 8;
    __shared__ float2 part[kEvery][9];
    tc::let_next_start();
    tc::wait_for_previous();
    const int r = threadIdx.x % 8, i = threadIdx.x / 8;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * 8 + r;
    float top = -INFINITY, sum = 0.0f;
    if (row < m) {
        for (int g = i; g < groups; g += kEvery * kBatch) {
            float2 s[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                s[j] = g + j * kEvery < groups ? stats[static_cast<int64_t>(g + j * kEvery) * m + row] : make_float2(-INFINITY, 0.0f);
            }
            float t = top;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) t = fmaxf(t, s[j].x);
            if (top != -INFINITY) sum *= exp2_fast((top - t) * kLog2e);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                // (-infinity, 0): masked, or no group; (-infinity, NaN): a NaN among what is masked
                if (s[j].x != -INFINITY || s[j].y != 0.0f) sum += s[j].y * exp2_fast((s[j].x - t) * kLog2e);
            }
            top = t;
        }
    }
    part[i][r] = make_float2(top, sum);
    __syncthreads();
    if (threadIdx.x < 8 && row < m) {
#pragma unroll
        for (int j = 0; j < kEvery; ++j) top = fmaxf(top, part[j][r].x);
        sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kEvery; ++j) {
            const float2 s = part[j][r];
            if (s.x != -INFINITY || s.y != 0.0f) sum += s.y * exp2_fast((s.x - top) * kLog2e);
        }
        const float log_sum = logf(sum);
        const int64_t t = targets[row];
        float loss = (top - at_target[row]) + log_sum;
        if (t < 0 || t >= v) loss = NAN;
        if (t == ignore) loss = 0.0f;
        rows[row] = loss;
        lse[row] = make_float2(top, log_sum * kLog2e);
    }
    if (end.loss == nullptr && end.factor == nullptr) return;
    __shared__ unsigned int before;
    __shared__ int counts[kRowThreads / 32];
    __shared__ float sums[kRowThreads / 32];
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) before = atomicAdd(end.blocks_done, 1u);
    __syncthreads();
    if (before != gridDim.x - 1) return;
    __threadfence();
    const int n = block_count(end.targets, end.m, ignore, counts);
    float total = 0.0f;
    if (end.loss != nullptr) {
#pragma unroll 8
        for (int64_t j = threadIdx.x; j < end.m; j += kRowThreads) total += __ldcg(end.rows + j);
        total = block_sum(total, sums);
    }
    if (threadIdx.x != 0) return;
    if (end.loss != nullptr) end.loss[0] = end.mean && n > 0 ? total / static_cast<float>(n) : total;
    if (end.factor != nullptr) end.factor[0] = end.mean && n > 0 ? end.scale / static_cast<float>(n) : end.scale;
}

// (conversions run at an eighth of the rate of additions)
__device__ __forceinline__ float code_value(uint32_t c) { return __uint_as_float(0x4b000000u | c) - 8388608.0f; }

// Codes to softmax - [target] in bf16, in place; a block has 8192 columns of a row, a thread four times eight.  The factor
// g is left to the products' epilogues: rounded into d it would shift the whole gradient by its own rounding,
// since at the target d is close to -g in every row.  Bound by memory, 4 bytes a logit (2048 x 50257:
// 412 MB in 68 us with nothing beside it, 6.0 TB/s); the rows are taken from the last, of which the L2 still has some.
__global__ void __launch_bounds__(256) gradient_kernel(uint16_t* codes, int64_t ld, int n, int width, const float2* stats, int64_t m,
                                                       const int64_t* targets, int64_t ignore, const float2* lse) {
    tc::let_next_start();
    tc::wait_for_previous();
    const int64_t row = m - 1 - (blockIdx.y + static_cast<int64_t>(blockIdx.z) * 65535);
    if (row < 0) return;
    const int col0 = (static_cast<int>(gridDim.x - 1 - blockIdx.x) * 1024 + static_cast<int>(threadIdx.x)) * 8;
    uint4* p = reinterpret_cast<uint4*>(codes + row * ld + col0);
    const int64_t t = targets[row];
    const float2 l = lse[row];
    uint4 u[4];
    float top[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = col0 + i * 2048;
        if (col < n) {
            u[i] = p[i * 256];
            top[i] = stats[static_cast<int64_t>(col / width) * m + row].x;
        }
    }
    const bool ignored = t == ignore, known = t >= 0 && t < n;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = col0 + i * 2048;
        if (col >= n) break;
        if (ignored) {
            p[i * 256] = make_uint4(0, 0, 0, 0);
            continue;
        }
        const float at = known ? __fmaf_rn(top[i] - l.x, kLog2e, -l.y) : NAN;
        const bool none = at == at;            // the last code stands for 0, unless the row is NaN
        const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
        uint32_t o[4];
        const int hit = known ? static_cast<int>(t) - col : -1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t ca = w[j] & 0xffffu, cb = w[j] >> 16;
            float a = ca == 65535u && none ? 0.0f : exp2_fast(__fmaf_rn(code_value(ca), -1.0f / kStep, at));
            float b = cb == 65535u && none ? 0.0f : exp2_fast(__fmaf_rn(code_value(cb), -1.0f / kStep, at));
            if (hit == 2 * j) a -= 1.0f;
            if (hit == 2 * j + 1) b -= 1.0f;
            o[j] = pack_bf16(a, b);
        }
        p[i * 256] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

dlion_status check_loss(const dlion_loss* p) {
    if (p == nullptr || p->m < 0 || p->m > kMost || p->h < 1 || p->h > kMost || p->v < 1 || p->v > kMost) return DLION_EINVAL;
    if (p->x_rs < 0 || p->x_cs < 0 || p->w_rs < 0 || p->w_cs < 0 || p->piece < 0) return DLION_EINVAL;
    if (p->mean != 0 && p->mean != 1) return DLION_EINVAL;
    if (!std::isfinite(p->scale)) return DLION_EINVAL;
    if (p->loss == nullptr || (p->m != 0 && (p->dx == nullptr) != (p->dw == nullptr))) return DLION_EINVAL;
    if (!aligned(p->loss, 4) || !aligned(p->rows, 4)) return DLION_EALIGN;
    if (p->dw != nullptr) {
        if (p->grad_type != DLION_GRAD_F32 && p->grad_type != DLION_GRAD_BF16) return DLION_EINVAL;
        if ((p->m > 1 && p->dx_ld < p->h) || (p->v > 1 && p->dw_ld < p->h)) return DLION_EINVAL;
        if (!aligned(p->dx, 2) || !aligned(p->dw, p->grad_type == DLION_GRAD_F32 ? 4 : 2)) return DLION_EALIGN;
    }
    if (p->m == 0) return DLION_OK;
    if (p->x == nullptr || p->w == nullptr || p->targets == nullptr || p->rows == nullptr) return DLION_EINVAL;
    return aligned(p->x, 2) && aligned(p->w, 2) && aligned(p->targets, 8) ? DLION_OK : DLION_EALIGN;
}

void loss(Call& c, const dlion_loss& p) {
    const bool grads = p.dw != nullptr, f32 = p.grad_type == DLION_GRAD_F32;
    if (p.m == 0) {
        if (!c.live()) return;
        c.check(cudaMemsetAsync(p.loss, 0, sizeof(float), c.stream));
        if (grads) c.check(cudaMemset2DAsync(p.dw, std::max(p.dw_ld, p.h) * (f32 ? 4 : 2), 0, p.h * (f32 ? 4 : 2), p.v, c.stream));
        return;
    }
    const Matrix x = readable(c, Matrix{p.x, p.m, p.h, p.x_rs, p.x_cs});
    const Matrix w = readable(c, Matrix{p.w, p.v, p.h, p.w_rs, p.w_cs});
    const int64_t piece = std::min(p.m, !grads ? std::max(p.piece, kEvalPiece) : p.piece == 0 ? kPiece : p.piece);
    const int64_t ld = round_up(p.v, 256);
    // rows that are neighbours in memory begin a piece on the 16-byte grid
    const int64_t step = x.cs == 1 ? piece : std::min(p.m, round_up(piece, 8));
    const Config cfg = choose(c, step, p.v, p.h, false, true);
    const int width = cfg.bn / 2;
    const int64_t groups = parts(p.v, width);
    float2* stats = c.ws.take<float2>(static_cast<uint64_t>(groups) * step);
    float* at_target = c.ws.take<float>(step);
    float2* lse = c.ws.take<float2>(step);
    float* factor = c.ws.take<float>(1);
    unsigned int* blocks_done = c.ws.take<unsigned int>(1);
    uint16_t* codes = grads ? c.ws.take<uint16_t>(static_cast<uint64_t>(step) * ld) : nullptr;
    float* sums = grads && !f32 && step < p.m ? c.ws.take<float>(static_cast<uint64_t>(p.v) * p.h) : nullptr;
    if (grads && step < p.m && c.live()) {
        start(c, factor_kernel, dim3(1), dim3(kRowThreads), 0, 1, p.targets, p.m, p.ignore_index, p.mean, p.scale, factor);
    }
    for (int64_t r = 0; r < p.m; r += step) {
        const int64_t rows = std::min(step, p.m - r);
        Matrix xp = x;
        xp.p = static_cast<const uint16_t*>(x.p) + r * x.rs;
        xp.rows = rows;
        if (c.live()) {
            Work<LossTile::Args> work{};
            if (!shape_of(cfg, xp, w, &work.s[0])) {
                c.status = DLION_EINVAL;
                return;
            }
            if (!make_map(&work.a[0], xp, &work.s[0].a_mn, 128) || !make_map(&work.b[0], w, &work.s[0].b_mn, cfg.bn / cfg.cg)) {
                c.status = DLION_ECUDA;
                return;
            }
            work.args[0] = LossTile::Args{static_cast<int>(rows), static_cast<int>(p.v), p.targets + r, blocks_done, stats, at_target, codes, ld};
            if (cfg.cg == 1) {
                launch<1, 64, LossTile, kWhole>(c, work);
            } else if (cfg.bn == 128) {
                launch<2, 128, LossTile, kWhole>(c, work);
            } else {
                launch<2, 256, LossTile, kWhole>(c, work);
            }
            if (c.status != DLION_OK) return;
            const Last end{blocks_done, p.rows, p.targets, p.m, p.mean, p.scale, r + rows >= p.m ? p.loss : nullptr,
                           grads && step >= p.m ? factor : nullptr};
            start(c, rows_kernel, dim3(static_cast<unsigned>(parts(rows, 8))), dim3(kRowThreads), 0, 1, stats, groups, rows, p.targets + r,
                  p.ignore_index, p.v, at_target, lse, p.rows + r, end);
            if (grads) {
                const dim3 grid(static_cast<unsigned>(parts(p.v, 8192)), static_cast<unsigned>(std::min<int64_t>(rows, 65535)),
                                static_cast<unsigned>(parts(rows, 65535)));
                start(c, gradient_kernel, grid, dim3(256), 0, 1, codes, ld, p.v, width, stats, rows, p.targets + r, p.ignore_index, lse);
            }
        }
        if (!grads) continue;
        const Matrix d{codes, rows, p.v, ld, 1};
        Finish fx{};
        fx.scale = factor;
        fx.out = static_cast<uint16_t*>(p.dx) + r * p.dx_ld;
        fx.out_ld = p.dx_ld;
        Finish fw{};
        fw.scale = factor;
        const bool last = r + rows >= p.m;
        float* so_far = f32 ? static_cast<float*>(p.dw) : sums;
        const int64_t so_far_ld = f32 ? p.dw_ld : p.h;
        if (r != 0) {
            fw.accumulated = so_far;
            fw.accumulated_ld = so_far_ld;
        }
        fw.out = last ? p.dw : so_far;
        fw.out_ld = last ? p.dw_ld : so_far_ld;
        fw.out_f32 = f32 || !last;
        fw.rough = 1;
        products(c, Part{d, transposed(w), fx, true}, Part{transposed(d), transposed(xp), fw, true}, Beside{});
    }
}

}  // namespace

extern "C" {

uint64_t dlion_lm_loss_workspace(const dlion_loss* p) { return check_loss(p) == DLION_OK ? workspace_of(*p, loss) : 0; }

dlion_status dlion_lm_loss(const dlion_loss* p, void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
    const dlion_status st = check_loss(p);
    return st != DLION_OK ? st : run(*p, loss, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
