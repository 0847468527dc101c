// D[m][n] = sum_k A[m][k] B[n][k] on the fifth-generation tensor cores, with the epilogue as a
// template parameter.  One persistent block (or pair of blocks, CG = 2) per SM:
//   warp 0      copies 64-wide slices of A and B into a ring of shared-memory stages,
//   warp 1      issues the matrix instructions; accumulators are two sets of BN columns of tensor memory,
//   warps 4-11  take the finished set out while the next one fills (rows 32 (w % 4).., half the columns each).
// A kernel's code is not in the instruction cache when it starts, and an epilogue met cold took 3500 clocks for 64
// columns; so while the first slices are on their way the epilogue warps run it once on nothing (`live` false: no rows).
// Three forms of the same kernel: kWhole (above); kJoined, where the blocks of a cluster each take a share of k of
// one 128 x 64 tile and send each other their sums, every block adding a share of the tile, for products with fewer tiles than SMs;
// kLong, for long sums: the tensor core's accumulator drops what does not fit, which shifts a sum of K products of one sign by
// K 2^-30 (K = 1024) to K 2^-28 (65536) of itself, so it only adds kSegment slices of them (8e-7, however long the sum) and
// the epilogue adds the segments in registers, rounding to nearest (192 columns, so that they fit: 96 a thread).  A sum of K random
// products is off by 1e-6 of its deviation in segments.
// A pair computes 256 x BN with each block holding half of A and half of B.  An SM takes in 57 bytes a clock (measured:
// 12 slices of a lone block's 128 x 128 tile, 393 KB, in 6850 clocks), so what a tile reads for its products decides: a pair's 256 x 256
// needs 32 KB a block for 512 clocks of products, its 256 x 128 and a lone block's 128 x 64 24 KB for 256 and 128.  Large shapes
// use the first, middling ones the second, those with few tiles the third.  8192 x 2048 x 8192 takes 177 to 187 us with the power cap (1550 to
// 1470 TFLOP/s, tensor pipe 91 % of the active clocks), 4096 x 768 x 2304 13.5 to 14.2 us (1070 to 1020), 197 x 768 x 768 5.7 us, which is
// latency.  Rows between: 160 x 4096 x 4096 takes 17.6 us, bound by what the SMs take in, 34 MB of weights notwithstanding.
#pragma once

#include "layers_math.cuh"
#include "tensor_core.cuh"

namespace dlion {
namespace prod {

enum Form { kWhole = 0, kJoined = 1, kLong = 2 };

constexpr int kSegment = 16;               // slices
constexpr int kSlice = 64;                 // values of k per stage: one 128-byte swizzled row
constexpr int kRingBytes = 196608;         // six stages of 32 KB or eight of 24 KB
constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr int kStaging = 4096;             // bytes of shared memory per epilogue warp
constexpr int kSmem = kRingBytes + kEpilogueWarps * kStaging + 1024 + 256;

struct Shape {
    int a_mn, b_mn;                        // operand majors (1: adjacent values along m / n)
    int tiles_m, tiles_n;
    int whole;                             // tiles that one worker sums; the rest are split
    int splits, split_slices, slices;      // splits of a tile, slices of k per split and in all
};

// A worker's u-th piece of work: a tile and its slices.  The split tiles come last, the splits of one side by side.
struct Unit {
    int tile, split, k0, k1;
    bool part;
};

__device__ __forceinline__ Unit unit_of(const Shape& s, int u) {
    Unit x;
    x.part = u >= s.whole;
    const int rest = s.tiles_m * s.tiles_n - s.whole;
    x.split = x.part ? (u - s.whole) / rest : 0;
    x.tile = x.part ? s.whole + (u - s.whole) % rest : u;
    x.k0 = x.part ? x.split * s.split_slices : 0;
    x.k1 = x.part ? min(s.slices, x.k0 + s.split_slices) : s.slices;
    return x;
}

enum Todo : unsigned { kScale = 1, kBias = 2, kKeep16 = 4, kKeep8 = 8, kAct = 16, kSlope = 32, kResidual = 64, kAdd = 128 };

// What happens to a sum; every part is optional.  Order: * scale, + bias, keep z, act, * act'(saved), + residual,
// + accumulated, store.
struct Finish {
    int m, n;
    unsigned todo;                         // kScale.. below: one test where nothing is asked for
    int wide;                              // rows of out begin on the 16-byte grid
    const float* scale;                    // on the device
    const void* bias;
    int bias_f32;
    int act;
    int keep;
    void* kept;
    int64_t kept_ld;
    uint8_t* kept_e;
    int64_t kept_e_ld;
    int slope;                             // activation whose slope at `saved` multiplies
    int saved8;
    const void* saved;
    int64_t saved_ld;
    const uint8_t* saved_e;
    int64_t saved_e_ld;
    const __nv_bfloat16* residual;
    int64_t residual_ld;
    const float* accumulated;
    int64_t accumulated_ld;
    void* out;
    int64_t out_ld;
    int out_f32;
    int rough;                             // a binary32 result whose operands are rounded already: segments only where the sum is very long
    float4* parts;                         // sums of split tiles: [tile][block][epilogue warp][split][32 rows x half the columns]
    unsigned int* tickets;                 // [tile][block][epilogue warp][4 pieces], 0 before the call
};

__device__ __forceinline__ bool on_grid(const void* p, int64_t ld, int bytes) {
    return ((reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * bytes)) & 15u) == 0;
}

// A warp's 32 x 32 piece of a row-major array goes through its staging memory, so that global accesses
// run along rows (64 or 128 bytes a row) while each thread owns one row.  16-byte units are exchanged
// within a row so that neither direction meets bank conflicts.
struct Piece {
    uint4* stage;
    int lane;
    int row0, col0;                        // first row and column of the piece
    int rows, cols;                        // valid ones, 1..32

    __device__ __forceinline__ int unit2(int r, int c) const { return r * 4 + (c ^ ((r >> 1) & 3)); }
    __device__ __forceinline__ int unit4(int r, int c) const { return r * 8 + (c ^ (r & 7)); }

    __device__ __forceinline__ void fetch16(const void* base, int64_t ld) const {
        const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(base) + static_cast<int64_t>(row0) * ld + col0;
        __syncwarp();
        if (cols == 32 && on_grid(base, ld, 2)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = lane / 4 + 8 * i, c = lane % 4;
                if (r < rows) stage[unit2(r, c)] = *reinterpret_cast<const uint4*>(p + r * ld + c * 8);
            }
        } else {
            __nv_bfloat16* s = reinterpret_cast<__nv_bfloat16*>(stage);
            __nv_bfloat16 v[32];           // all on their way before the first is used
#pragma unroll
            for (int r = 0; r < 32; ++r) v[r] = lane < cols && r < rows ? p[r * ld + lane] : __nv_bfloat16();
#pragma unroll
            for (int r = 0; r < 32; ++r) s[unit2(r, lane / 8) * 8 + lane % 8] = v[r];
        }
        __syncwarp();
    }

    // f(j, value) for the 32 columns of this thread's row (columns beyond `cols` hold leftovers)
    template <class F>
    __device__ __forceinline__ void each16(F f) const {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint4 u = stage[unit2(lane, c)];
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f(c * 8 + 2 * i, bf16_lo(w[i]));
                f(c * 8 + 2 * i + 1, bf16_hi(w[i]));
            }
        }
    }

    __device__ __forceinline__ void put16(const uint32_t (&w)[16], void* base, int64_t ld, bool wide) const {
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 4; ++c) stage[unit2(lane, c)] = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
        __syncwarp();
        uint16_t* p = static_cast<uint16_t*>(base) + static_cast<int64_t>(row0) * ld + col0;
        if (cols == 32 && wide) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = lane / 4 + 8 * i, c = lane % 4;
                if (r < rows) *reinterpret_cast<uint4*>(p + r * ld + c * 8) = stage[unit2(r, c)];
            }
        } else if (cols == 32 && ((reinterpret_cast<uintptr_t>(p) & 3u) | static_cast<uintptr_t>(ld & 1)) == 0) {
            const uint32_t* s = reinterpret_cast<const uint32_t*>(stage);      // rows of words, two at a time
            const int l = lane % 16;
#pragma unroll 8
            for (int i = 0; i < 16; ++i) {
                const int r = 2 * i + lane / 16;
                if (r < rows) *reinterpret_cast<uint32_t*>(p + r * ld + 2 * l) = s[unit2(r, l / 4) * 4 + l % 4];
            }
        } else if (lane < cols) {
            const uint16_t* s = reinterpret_cast<const uint16_t*>(stage);
            #pragma unroll 8
            for (int r = 0; r < rows; ++r) p[r * ld + lane] = s[unit2(r, lane / 8) * 8 + lane % 8];
        }
    }

    __device__ __forceinline__ void put32(const float (&v)[32], float* base, int64_t ld, bool wide) const {
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            stage[unit4(lane, c)] = make_uint4(__float_as_uint(v[4 * c]), __float_as_uint(v[4 * c + 1]),
                                               __float_as_uint(v[4 * c + 2]), __float_as_uint(v[4 * c + 3]));
        }
        __syncwarp();
        float* p = base + static_cast<int64_t>(row0) * ld + col0;
        if (cols == 32 && wide) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = lane / 8 + 4 * i, c = lane % 8;
                if (r < rows) *reinterpret_cast<uint4*>(p + r * ld + c * 4) = stage[unit4(r, c)];
            }
        } else if (lane < cols) {
            const float* s = reinterpret_cast<const float*>(stage);
            #pragma unroll 8
            for (int r = 0; r < rows; ++r) p[r * ld + lane] = s[unit4(r, lane / 4) * 4 + lane % 4];
        }
    }

    // adds a binary32 array's piece to v
    __device__ __forceinline__ void add32(float (&v)[32], const float* base, int64_t ld) const {
        const float* p = base + static_cast<int64_t>(row0) * ld + col0;
        __syncwarp();
        if (cols == 32 && on_grid(base, ld, 4)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = lane / 8 + 4 * i, c = lane % 8;
                if (r < rows) stage[unit4(r, c)] = *reinterpret_cast<const uint4*>(p + r * ld + c * 4);
            }
        } else {
            float* s = reinterpret_cast<float*>(stage);
#pragma unroll 8
            for (int r = 0; r < 32; ++r) {
                if (lane < cols && r < rows) s[unit4(r, lane / 4) * 4 + lane % 4] = p[r * ld + lane];
            }
        }
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const uint4 u = stage[unit4(lane, c)];
            v[4 * c] += __uint_as_float(u.x);
            v[4 * c + 1] += __uint_as_float(u.y);
            v[4 * c + 2] += __uint_as_float(u.z);
            v[4 * c + 3] += __uint_as_float(u.w);
        }
    }

    // each lane's value to its column
    __device__ __forceinline__ void add_bias(float (&v)[32], float b) const {
        __syncwarp();
        reinterpret_cast<float*>(stage)[lane] = b;
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float4 u = reinterpret_cast<const float4*>(stage)[c];
            v[4 * c] += u.x;
            v[4 * c + 1] += u.y;
            v[4 * c + 2] += u.z;
            v[4 * c + 3] += u.w;
        }
    }
};

template <class T>
__device__ __forceinline__ void to_bf16(const T (&v)[32], uint32_t (&w)[16]) {
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
}

__device__ __forceinline__ void keep8(const Finish& f, const Piece& pc, const float (&v)[32]) {
    const int row = pc.row0 + pc.lane;
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        if (j < pc.cols) top = larger(top, v[j]);
    }
    const uint32_t e = block_exponent(__float_as_uint(top));
    const float inv = block_inverse(e);
    if (pc.lane >= pc.rows) return;
    f.kept_e[static_cast<int64_t>(pc.col0 / 32) * f.kept_e_ld + row] = static_cast<uint8_t>(e);
    uint32_t w[8];
    auto quantise = [&](auto limited) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[j] = bytes4(quantise8(limited(v[4 * j]), inv), quantise8(limited(v[4 * j + 1]), inv), quantise8(limited(v[4 * j + 2]), inv),
                          quantise8(limited(v[4 * j + 3]), inv));
        }
    };
    if (__builtin_expect(e == kTop8, 0)) {
        quantise([](float x) { return within8(x); });
    } else {
        quantise([](float x) { return x; });
    }
    int8_t* q = static_cast<int8_t*>(f.kept) + static_cast<int64_t>(row) * f.kept_ld + pc.col0;
    if (pc.cols == 32 && on_grid(f.kept, f.kept_ld, 1)) {
        reinterpret_cast<uint4*>(q)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(q)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (j < pc.cols) q[j] = static_cast<int8_t>(w[j / 4] >> (8 * (j % 4)));
        }
    }
}

__device__ __forceinline__ void times_slope8(const Finish& f, const Piece& pc, float (&v)[32]) {
    if (pc.lane >= pc.rows) return;
    const int row = pc.row0 + pc.lane;
    const float s = block_scale(f.saved_e[static_cast<int64_t>(pc.col0 / 32) * f.saved_e_ld + row]);
    const int8_t* q = static_cast<const int8_t*>(f.saved) + static_cast<int64_t>(row) * f.saved_ld + pc.col0;
    uint32_t w[8];
    if (pc.cols == 32 && on_grid(f.saved, f.saved_ld, 1)) {
        const uint4 a = reinterpret_cast<const uint4*>(q)[0], b = reinterpret_cast<const uint4*>(q)[1];
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[j] = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (4 * j + i < pc.cols) w[j] |= static_cast<uint32_t>(static_cast<uint8_t>(q[4 * j + i])) << (8 * i);
            }
        }
    }
    with_act(f.slope, [&](auto kind) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float u[4];
            restore4(w[j], s, u);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * j + i] *= act_slope<decltype(kind)::value>(u[i]);
        }
    });
}

// The epilogue of the layer products.  What a call does not ask for is out of the way of what it does (the hints):
// a small product runs this code once, and each jump over unused code costs a fetch of some 500 clocks.
struct General {
    using Args = Finish;
    static constexpr bool kSplits = true;

    // What an epilogue needs of memory is asked for before its sums are waited for: a load met in the middle stops a warp for some
    // 600 clocks, and there are four pieces in a tile.
    struct Ahead {
        float scale;
        uint32_t bias[4];                      // as it is stored, a lane's column of each piece

        __device__ __forceinline__ float bias_of(const Finish& f, int piece) const {
            const uint32_t b = piece == 0 ? bias[0] : piece == 1 ? bias[1] : piece == 2 ? bias[2] : bias[3];
            return __uint_as_float(f.bias_f32 ? b : b << 16);
        }
    };

    template <int WIDTH>
    static __device__ __forceinline__ Ahead ahead(const Finish& f, int row0, int col0, int lane) {
        Ahead x{1.0f, {0, 0, 0, 0}};
        if (__builtin_expect(f.todo == 0, 1)) return x;
        if (f.todo & kScale) x.scale = *f.scale;
        if (f.todo & kBias) {
#pragma unroll
            for (int i = 0; i < WIDTH / 32; ++i) {
                const int col = col0 + i * 32 + lane;
                if (col < f.n) x.bias[i] = f.bias_f32 ? static_cast<const uint32_t*>(f.bias)[col] : static_cast<const unsigned short*>(f.bias)[col];
            }
        }
        if ((f.todo & (kSlope | kResidual)) && row0 + lane < f.m && col0 < f.n) {
            const int last = min(f.n, col0 + WIDTH) - 1;
            const int64_t row = row0 + lane;
            auto touch = [](const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); };
            if (f.todo & kResidual) {
                touch(f.residual + row * f.residual_ld + col0);
                touch(f.residual + row * f.residual_ld + last);
            }
            if (f.todo & kSlope) {
                const uint8_t* p = static_cast<const uint8_t*>(f.saved);
                const int bytes = f.saved8 ? 1 : 2;
                touch(p + (row * f.saved_ld + col0) * bytes);
                touch(p + (row * f.saved_ld + last) * bytes);
            }
        }
        return x;
    }

    static __device__ __forceinline__ void piece(const Finish& f, unsigned todo, const Piece& pc, float scale, float bias, float (&v)[32]) {
        if (__builtin_expect(todo != 0, 0)) {
            if (todo & kScale) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= scale;
            }
            if (todo & kBias) pc.add_bias(v, bias);
            if (todo & kKeep8) keep8(f, pc, v);
            if (todo & kKeep16) {
                uint32_t w[16];
                to_bf16(v, w);
                pc.put16(w, f.kept, f.kept_ld, on_grid(f.kept, f.kept_ld, 2));
            }
            if (todo & kAct) {
                with_act(f.act, [&](auto kind) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = act_value<decltype(kind)::value>(v[j]);
                });
            }
            if (todo & kSlope) {
                if (f.saved8) {
                    times_slope8(f, pc, v);
                } else {
                    pc.fetch16(f.saved, f.saved_ld);
                    with_act(f.slope, [&](auto kind) {
                        pc.each16([&](int j, float u) { v[j] *= act_slope<decltype(kind)::value>(u); });
                    });
                }
            }
            if (todo & kResidual) {
                pc.fetch16(f.residual, f.residual_ld);
                pc.each16([&](int j, float u) { v[j] += u; });
            }
            if (todo & kAdd) pc.add32(v, f.accumulated, f.accumulated_ld);
        }
        if (__builtin_expect(f.out_f32, 0)) {
            pc.put32(v, static_cast<float*>(f.out), f.out_ld, f.wide != 0);
        } else {
            uint32_t w[16];
            to_bf16(v, w);
            pc.put16(w, f.out, f.out_ld, f.wide != 0);
        }
    }

    // The same from registers.
    template <int W>
    static __device__ __forceinline__ void sums(const Finish& f, const Ahead& x, const float (&acc)[W], int row0, int col0, bool live, uint4* stage,
                                                int lane) {
#pragma unroll
        for (int c = 0; c < W; c += 32) {
            if (col0 + c >= f.n || row0 >= f.m) return;
            float v[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = acc[c + j];
            piece(f, f.todo, Piece{stage, lane, row0, col0 + c, live ? min(32, f.m - row0) : 0, min(32, f.n - col0 - c)}, x.scale,
                  x.bias_of(f, c / 32), v);
        }
    }

    // One warp's 32 rows and `width` columns of a finished accumulator.
    static __device__ __forceinline__ void tile(const Finish& f, const Ahead& x, uint32_t acc, int row0, int col0, int width, bool live, uint4* stage,
                                                int lane) {
        const unsigned todo = f.todo;
#pragma unroll 1
        for (int c = 0; c < width; c += 32) {
            float v[32];
            if (col0 + c >= f.n || row0 >= f.m) return;      // the same for the whole warp
            tc::tmem_load32(acc + c, v);
            const Piece pc{stage, lane, row0, col0 + c, live ? min(32, f.m - row0) : 0, min(32, f.n - col0 - c)};
            piece(f, todo, pc, x.scale, x.bias_of(f, c / 32), v);
            if (!live) return;
        }
    }

    // 32 x 32 sums of a split, kept as the threads have them: 512 bytes side by side at a time
    static __device__ __forceinline__ void put_part(float4* to, const float (&v)[32], int lane) {
#pragma unroll
        for (int i = 0; i < 8; ++i) __stcg(to + i * 32 + lane, make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
    }

    // After a warp's part of a split is in place: whoever finds a piece's other splits done adds them all, in their order, so that
    // the sum does not depend on who that is.  Nobody waits.  The splits look at the pieces in different orders, or the
    // last of them would add all four.
    static __device__ __forceinline__ void join(const Finish& f, const Ahead& x, int place, int split, int splits, int row0, int col0, int width,
                                                uint4* stage, int lane) {
        __threadfence();
        __syncwarp();
        const int pieces = width / 32;
#pragma unroll 1
        for (int i = 0; i < pieces; ++i) {
            const int c = (i + split) % pieces * 32;
            unsigned int before = 0;
            if (lane == 0) before = atomicAdd(f.tickets + place * 4 + c / 32, 1u);
            before = __shfl_sync(0xffffffffu, before, 0);
            if (before != static_cast<unsigned int>(splits - 1) || col0 + c >= f.n || row0 >= f.m) continue;
            __threadfence();
            const float4* from = f.parts + static_cast<int64_t>(place) * splits * (width * 8);
            float v[32] = {};
#pragma unroll 2
            for (int r = 0; r < splits; ++r) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float4 w = __ldcg(from + (r * width + c) * 8 + j * 32 + lane);
                    v[4 * j] += w.x;
                    v[4 * j + 1] += w.y;
                    v[4 * j + 2] += w.z;
                    v[4 * j + 3] += w.w;
                }
            }
            piece(f, f.todo, Piece{stage, lane, row0, col0 + c, min(32, f.m - row0), min(32, f.n - col0 - c)}, x.scale, x.bias_of(f, c / 32), v);
        }
    }
};

// Tiles in groups of 8 rows of tiles, columns outermost within a group: the tiles in flight share
// their operands' slices in L2.
__device__ __forceinline__ void tile_of(const Shape& s, int t, int& tm, int& tn) {
    constexpr int kGroup = 8;
    const int per = kGroup * s.tiles_n, g = t / per, in = t - g * per;
    const int rows = min(kGroup, s.tiles_m - g * kGroup);
    tm = g * kGroup + in % rows;
    tn = in / rows;
}

// Sums over the rows of a matrix on the 16-byte grid (a bias' gradient), taken along by the two warps of a block that have nothing
// to do: strips of 8 * lanes columns, a warp each, the rows 32 / lanes at a time.  They read what the products read
// anyway; a kernel of its own takes 25 us for 8192 x 8192 and took 6 us for 4096 x 2304.  A lane adds rows * lanes / 32 values
// one after another in binary32, each addition to 2^-24; the kernel of its own adds rows / 256 so.
struct Beside {
    const __nv_bfloat16* a;
    int64_t rs;
    int rows, cols;
    void* out;                             // nullable
    int f32;
    int lanes;                             // 1, 2 or 4
};

__device__ __forceinline__ void sum_columns(const Beside& s, int warp, int warps, int lane) {
    const int rows_at_once = 32 / s.lanes, r0 = lane / s.lanes, width = 8 * s.lanes;
    for (int64_t c0 = static_cast<int64_t>(warp) * width; c0 < s.cols; c0 += static_cast<int64_t>(warps) * width) {
        const int64_t col = c0 + lane % s.lanes * 8;
        float v[8] = {};
        if (col < s.cols) {
            // a row's last columns may share their 16 bytes with what lies between it and the next row; after the last row may be nothing
            const bool ragged = col + 8 > s.cols;
            const int whole = ragged ? s.rows - 1 : s.rows;
            const uint4* p = reinterpret_cast<const uint4*>(s.a + r0 * s.rs + col);
            const int64_t step = s.rs / 8 * rows_at_once;
            int r = r0;
            for (; r + 7 * rows_at_once < whole; r += 8 * rows_at_once, p += 8 * step) {
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
            for (; r < whole; r += rows_at_once, p += step) {
                float x[8];
                widen(*p, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += x[j];
            }
            if (ragged && r == s.rows - 1) {
#pragma unroll
                for (int j = 0; j < 7; ++j) {
                    if (col + j < s.cols) v[j] += __bfloat162float(s.a[r * s.rs + col + j]);
                }
            }
        }
        __syncwarp();
        for (int o = 16; o >= s.lanes; o >>= 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += __shfl_xor_sync(0xffffffffu, v[j], o);
        }
        if (r0 == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (col + j >= s.cols) break;
                if (s.f32) {
                    static_cast<float*>(s.out)[col + j] = v[j];
                } else {
                    static_cast<__nv_bfloat16*>(s.out)[col + j] = __float2bfloat16_rn(v[j]);
                }
            }
        }
    }
}

// One product, or two that do not depend on each other (a layer's dx and dW), so that the tiles of the second fill the SMs that
// the first leaves idle.
template <class Args>
struct Work {
    CUtensorMap a[2], b[2];
    Shape s[2];
    Args args[2];
    int units[2];                          // pieces of work in each; those of the first take longer
    Beside beside;
    int extra;                             // pieces of the second ahead of time for each worker that has one fewer of the first
};

// A worker's i-th piece of work, or -1: every `workers`-th of the first product, then, where that leaves some a piece
// short, `extra` of the second for those, then every `workers`-th of the rest.
template <bool TWO, class Args>
__device__ __forceinline__ int unit_at(const Work<Args>& w, int worker, int workers, int i) {
    if (!TWO) return worker + i * workers < w.units[0] ? worker + i * workers : -1;
    const int rounds = w.units[0] / workers, over = w.units[0] - rounds * workers;
    const int firsts = rounds + (worker < over ? 1 : 0);
    if (i < firsts) return worker + i * workers;
    int j = i - firsts, u;
    const int extra = over == 0 ? 0 : w.extra, behind = workers - over;
    if (worker >= over && j < extra) {
        u = j * behind + worker - over;
    } else {
        if (worker >= over) j -= extra;
        u = extra * behind + worker + j * workers;
    }
    return u < w.units[1] ? w.units[0] + u : -1;
}

// TWO: with a second product; with one, what describes it is at fixed places.
template <int CG, int BN, class E, int FORM, bool TWO>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ Work<typename E::Args> work, unsigned int* mark) {
    constexpr int kM = 128 * CG;               // rows of the tile; a block has 128 of them
    constexpr int kBRows = BN / CG;            // of B, in this block
    constexpr uint32_t kCols = BN <= 128 ? 2 * BN : 512;               // tensor memory columns, a power of two: two accumulators
    constexpr int kABytes = 16384;
    static_assert(FORM != kJoined || CG == 1, "joined tiles are a block's own");
    constexpr int kBChunks = (kBRows + 63) / 64;                       // of 64 columns where they are adjacent
    constexpr int kStageBytes = kABytes + kBChunks * 8192;

    extern __shared__ uint8_t raw[];
    const uint32_t base = (tc::smem_addr(raw) + 1023u) & ~1023u;
    uint8_t* mem = raw + (base - tc::smem_addr(raw));
    const uint32_t bars = base + kRingBytes + kEpilogueWarps * kStaging;
    constexpr uint32_t kPiece = 4096, kPieces = 4 * (BN / 32);         // kJoined: 32 x 32 sums land behind a shorter ring
    constexpr uint32_t kLanding = FORM == kJoined ? kPieces * kPiece : 0;
    constexpr int kRing = (kRingBytes - kLanding) / kStageBytes;
    static_assert(kRing <= 8 && (FORM != kJoined || kLanding <= 2 * kStageBytes), "barriers; the ring holds what is sent");
    const uint32_t landing = base + kRingBytes - kLanding;
    const uint32_t full = bars, empty = bars + 64, ready = bars + 128, drained = bars + 144, slot = bars + 160, landed = bars + 168;
    volatile uint32_t* slot_mem = reinterpret_cast<volatile uint32_t*>(mem + (slot - base));

    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = CG == 2 ? tc::cluster_rank() : 0;
    // kJoined: the cluster is the worker, a block's place in it the split; one tile each (whole = 0, the second product empty)
    const int share = FORM == kJoined ? static_cast<int>(tc::cluster_rank()) : 0;
    const int workers = FORM == kJoined ? work.units[0] : gridDim.x / CG;
    const int worker = FORM == kJoined ? static_cast<int>(blockIdx.x) / work.s[0].splits + share * (work.units[0] / work.s[0].splits)
                                       : static_cast<int>(blockIdx.x) / CG;

    tc::let_next_start();
    if (threadIdx.x == 0) {
        for (int i = 0; i < kRing; ++i) {
            tc::bar_init(full + 8 * i, 1);
            tc::bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::bar_init(ready + 8 * i, 1);
            tc::bar_init(drained + 8 * i, kEpilogueWarps * CG);
        }
        if (FORM == kJoined) tc::bar_init(landed, 1);
        tc::bar_init_done();
        if (FORM == kJoined) tc::bar_expect(landed, kPieces * kPiece);
        slot_mem[1] = 0;                       // set when a wait ran out
        tc::prefetch_map(&work.a[0]);
        tc::prefetch_map(&work.b[0]);
    }
    if (warp == 1) tc::tmem_alloc<CG>(slot, kCols);
    tc::fence_before();
    __syncthreads();
    if (CG == 2) tc::cluster_sync();
    if (FORM == kJoined) tc::cluster_arrive();
    tc::fence_after();
    const uint32_t tmem = *slot_mem;
    bool fine = true;
    tc::wait_for_previous();

    // The copying and the issuing warp go through their loops whole and elect a lane at the instructions themselves: so
    // what describes the operands stays in uniform registers, where these instructions want it.  With one lane in the
    // loop the issue of four instructions and the wait before them took 640 clocks, more than the 512 of the products.
    if (warp == 0) {
        const uint32_t lead_full = CG == 2 ? tc::map_to_rank(full, 0) : full;
        int st = 0, filled = 0;
        uint32_t phase = 1;
        for (int i = 0; fine; ++i) {
            const int unit = unit_at<TWO>(work, worker, workers, i);
            if (unit < 0) break;
            const int which = TWO && unit >= work.units[0] ? 1 : 0;
            const Shape& s = work.s[which];
            const CUtensorMap *map_a = &work.a[which], *map_b = &work.b[which];
            int tm, tn;
            const Unit x = unit_of(s, unit - which * work.units[0]);
            tile_of(s, x.tile, tm, tn);
            const int row = tm * kM + static_cast<int>(rank) * 128, col = tn * BN + static_cast<int>(rank) * kBRows;
            for (int kb = x.k0; kb < x.k1; ++kb, ++filled) {
                if (!(fine = tc::bar_wait(empty + 8 * st, phase))) break;
                if (tc::elected()) {
                    const uint32_t a = base + st * kStageBytes, b = a + kABytes, bar = lead_full + 8 * st;
                    if (rank == 0) tc::bar_expect(full + 8 * st, CG * (kABytes + (s.b_mn ? kBChunks * 8192 : kBRows * 128)));
                    if (s.a_mn) {
                        tc::load_tile<CG>(a, map_a, row, kb * kSlice, bar);
                        tc::load_tile<CG>(a + 8192, map_a, row + 64, kb * kSlice, bar);
                    } else {
                        tc::load_tile<CG>(a, map_a, kb * kSlice, row, bar);
                    }
                    if (s.b_mn) {
#pragma unroll
                        for (int c = 0; c < kBChunks; ++c) tc::load_tile<CG>(b + 8192 * c, map_b, col + 64 * c, kb * kSlice, bar);
                    } else {
                        tc::load_tile<CG>(b, map_b, kb * kSlice, col, bar);
                    }
                }
                __syncwarp();
                if (++st == kRing) {
                    st = 0;
                    phase ^= 1;
                }
            }
        }
        // Where a wait ran out, what was asked for still lands in this block's memory: it is awaited.
        if (!fine && rank == 0) {
            for (int i = max(0, filled - kRing); i < filled; ++i) tc::bar_wait(full + 8 * (i % kRing), (i / kRing) & 1);
        }
    } else if (warp == 1) {
        if (rank == 0) {
            auto finished = [&](uint32_t bar) {
                if (tc::elected()) tc::commit<CG>(bar);
                __syncwarp();
            };
            int st = 0, n = 0;
            uint32_t phase = 0;
            for (int i = 0; fine; ++i) {
                const int unit = unit_at<TWO>(work, worker, workers, i);
                if (unit < 0) break;
                const int which = TWO && unit >= work.units[0] ? 1 : 0;
                const Shape& s = work.s[which];
                const Unit x = unit_of(s, unit - which * work.units[0]);
                const uint32_t inst = tc::instruction(kM, BN, s.a_mn, s.b_mn);
                const uint32_t a_step = (s.a_mn ? 2048 : 32) >> 4, b_step = (s.b_mn ? 2048 : 32) >> 4;   // 16 values of k
                // (a block's shared addresses have its place in the cluster above bit 23)
                const uint64_t a_desc = tc::operand_base(s.a_mn) | ((base >> 4) & 0x3fff);
                const uint64_t b_desc = tc::operand_base(s.b_mn) | (((base + kABytes) >> 4) & 0x3fff);
                auto multiply = [&](uint32_t acc, int st, bool first) {     // four instructions on stage `st`
                    if (tc::elected()) {
                        const uint32_t at = static_cast<uint32_t>(st * kStageBytes) >> 4;
#pragma unroll
                        for (int j = 0; j < 4; ++j) tc::mma<CG>(acc, a_desc + at + j * a_step, b_desc + at + j * b_step, inst, (j > 0 || !first) ? 1u : 0u);
                    }
                    __syncwarp();
                };
                const int seg = FORM == kLong ? kSegment : x.k1 - x.k0;
                for (int kb = x.k0; kb < x.k1 && fine; ++n) {
                    const int set = n & 1, from = kb, to = min(x.k1, kb + seg);
                    if (!(fine = tc::bar_wait<CG == 2>(drained + 8 * set, ((n >> 1) & 1) ^ 1))) break;
                    tc::fence_after();
                    for (; kb < to; ++kb) {
                        if (!(fine = tc::bar_wait(full + 8 * st, phase))) break;
                        tc::fence_after();
                        multiply(tmem + set * BN, st, kb == from);
                        finished(empty + 8 * st);
                        if (++st == kRing) {
                            st = 0;
                            phase ^= 1;
                        }
                    }
                    if (fine) finished(ready + 8 * set);
                }
            }
        }
    } else if (warp < 4) {
        if (E::kSplits && work.beside.out != nullptr) {
            sum_columns(work.beside, static_cast<int>(blockIdx.x) * 2 + warp - 2, static_cast<int>(gridDim.x) * 2, lane);
        }
    } else {
        const int quarter = warp % 4, half = (warp - 4) / 4;
        uint4* stage = reinterpret_cast<uint4*>(mem + kRingBytes + (warp - 4) * kStaging);
        const uint32_t lead_drained = CG == 2 ? tc::map_to_rank(drained, 0) : drained;
        const uint32_t part = tmem + half * (BN / 2) + (static_cast<uint32_t>(quarter * 32) << 16);
        auto drain = [&](int set) {
            tc::fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 2) {
                    tc::bar_arrive_cluster(lead_drained + 8 * set);
                } else {
                    tc::bar_arrive(drained + 8 * set);
                }
            }
        };
        if (FORM == kJoined) tc::cluster_wait();     // the others' barriers exist
        int n = 0;
        for (int i = -1; fine; ++i) {
            const bool live = i >= 0;
            const int unit = unit_at<TWO>(work, worker, workers, live ? i : 0);
            if (unit < 0) break;
            const int which = TWO && unit >= work.units[0] ? 1 : 0;
            const Shape& s = work.s[which];
            const typename E::Args& args = work.args[which];
            int tm, tn;
            const Unit x = unit_of(s, unit - which * work.units[0]);
            tile_of(s, x.tile, tm, tn);
            const int place = ((x.tile - s.whole) * CG + static_cast<int>(rank)) * kEpilogueWarps + warp - 4;     // of a split tile's part
            const int row0 = tm * kM + static_cast<int>(rank) * 128 + quarter * 32, col0 = tn * BN + half * (BN / 2);
            // (joined, a warp finishes the piece that it adds)
            const int p_own = share + s.splits * (warp - 4);
            const auto needs = FORM == kJoined ? E::template ahead<32>(args, tm * kM + (p_own % 4) * 32, tn * BN + (p_own / 4) * 32, lane)
                                               : E::template ahead<BN / 2>(args, row0, col0, lane);
            if constexpr (FORM == kLong) {
                float sum[BN / 2] = {};
                for (int kb = x.k0; live && kb < x.k1; kb += kSegment, ++n) {
                    const int set = n & 1;
                    if (!(fine = tc::bar_wait(ready + 8 * set, (n >> 1) & 1))) break;
                    tc::fence_after();
#pragma unroll
                    for (int c = 0; c < BN / 2; c += 32) {
                        float v[32];
                        tc::tmem_load32(part + set * BN + c, v);
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum[c + j] += v[j];
                    }
                    drain(set);
                }
                if (!fine) break;
                if (x.part && live) {
                    float4* to = args.parts + (static_cast<int64_t>(place) * s.splits + x.split) * (BN / 2 * 8);
#pragma unroll
                    for (int c = 0; c < BN / 2; c += 32) {
                        float v[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = sum[c + j];
                        E::put_part(to + c * 8, v, lane);
                    }
                    E::join(args, needs, place, x.split, s.splits, row0, col0, BN / 2, stage, lane);
                } else {
                    E::sums(args, needs, sum, row0, col0, live, stage, lane);
                }
            } else if constexpr (FORM == kJoined) {
                if (live) {
                    if (!(fine = tc::bar_wait(ready, 0))) break;
                    tc::fence_after();
                    // into the ring, which has been read: 32 x 32 pieces, units exchanged as in Piece; and off to the
                    // block that adds this piece of all shares
                    const int p0 = half * (BN / 64) * 4 + quarter;
#pragma unroll
                    for (int c = 0; c < BN / 2; c += 32) {
                        float v[32];
                        tc::tmem_load32(part + c, v);
                        float4* to = reinterpret_cast<float4*>(mem + (p0 + c / 8) * kPiece);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            to[lane * 8 + (i ^ (lane & 7))] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                        }
                    }
                    tc::fence_for_copies();
                    __syncwarp();
                    if (lane < BN / 64) {
                        const int p = p0 + lane * 4;
                        const uint32_t owner = static_cast<uint32_t>(p % s.splits);
                        tc::send(tc::map_to_rank(landing + ((p / s.splits) * s.splits + share) * kPiece, owner), base + p * kPiece, kPiece,
                                 tc::map_to_rank(landed, owner));
                    }
                    if (!(fine = tc::bar_wait<true>(landed, 0))) break;
                }
                for (int p = share + s.splits * (warp - 4); p < static_cast<int>(kPieces); p += s.splits * kEpilogueWarps) {
                    const float4* from = reinterpret_cast<const float4*>(mem + kRingBytes - kLanding + (p / s.splits) * s.splits * kPiece);
                    float v[32] = {};
                    for (int r = 0; r < s.splits; ++r, from += kPiece / 16) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float4 w = from[lane * 8 + (i ^ (lane & 7))];
                            v[4 * i] += w.x;
                            v[4 * i + 1] += w.y;
                            v[4 * i + 2] += w.z;
                            v[4 * i + 3] += w.w;
                        }
                    }
                    E::sums(args, needs, v, tm * kM + (p % 4) * 32, tn * BN + (p / 4) * 32, live, stage, lane);
                    if (!live) break;
                }
            } else {
                const int set = n & 1;
                if (live) {
                    if (!(fine = tc::bar_wait(ready + 8 * set, (n >> 1) & 1))) break;
                    tc::fence_after();
                }
                if constexpr (E::kSplits) {
                    if (x.part && live) {
                        float4* to = args.parts + (static_cast<int64_t>(place) * s.splits + x.split) * (BN / 2 * 8);
#pragma unroll 1
                        for (int c = 0; c < BN / 2; c += 32) {
                            float v[32];
                            tc::tmem_load32(part + set * BN + c, v);
                            E::put_part(to + c * 8, v, lane);
                        }
                        drain(set);
                        ++n;
                        E::join(args, needs, place, x.split, s.splits, row0, col0, BN / 2, stage, lane);
                        continue;
                    }
                }
                E::tile(args, needs, part + set * BN, row0, col0, BN / 2, live, stage, lane);
                if (live) {
                    drain(set);
                    ++n;
                }
            }
        }
    }
    if (!fine) {
        slot_mem[1] = 1;
        *mark = 1;
    }
    __syncwarp();
    if (FORM == kJoined && warp < 4) tc::cluster_wait();
    tc::fence_before();
    __syncthreads();
    if (slot_mem[1] != 0) {                    // matrix instructions may still be running: let them end
        const uint64_t t0 = tc::nanoseconds();
        while (tc::nanoseconds() - t0 < 50000000ull) {
        }
    }
    if (CG == 2 || FORM == kJoined) tc::cluster_sync();
    tc::fence_after();
    if (warp == 1) tc::tmem_free<CG>(tmem, kCols);
}

}  // namespace prod
}  // namespace dlion
