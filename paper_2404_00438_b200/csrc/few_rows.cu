// Products of one to 16 rows (a serving step): every weight is read once and used a few times, so the only
// question is how fast the weights stream.  The arithmetic is the warp-level 16 x 8 x 16 matrix instruction with its k (or n)
// indices renamed so that a thread's share of the weights is 16 adjacent bytes.  Each warp has a ring of its own, filled by
// tiled copies of whole 128-byte lines, some 160 KB of which are under way on an SM, through the ends of the columns' sums
// too.  8 rows over 50257 x 2048 with a bias: 35.6 us, 207.5 MB, 5.8 TB/s.  (Shares of 16 bytes loaded by the threads themselves, to registers or to shared memory, cut the lines in half
// between warps: 8 rows over 50257 x 2048 took 41 to 44 us.  One row on fused multiply-adds would do, eight rows would not: 64 of
// them, and 8 conversions, for every 16 bytes against the 23 bytes a clock that an SM streams.)
#include "product_host.h"

namespace dlion {
namespace prod {

namespace {

constexpr int kFewThreads = 256, kFewWarps = 8;

__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint4 shared16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t shared4(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}
// 16-byte unit c of row r of a tile of 128-byte rows, as the copies exchange them
__device__ __forceinline__ uint32_t unit_at(int r, int c) { return static_cast<uint32_t>(r * 128 + ((c ^ (r & 7)) << 4)); }

// A row's 32 columns, a lane each, through the rest of the product (see Finish).
__device__ __forceinline__ void finish_row(const Finish& f, int row, int64_t col, float v, float bias) {
    const bool in = col < f.n;
    if (f.scale != nullptr) v *= *f.scale;
    v += bias;
    if (f.keep == DLION_KEEP_8BIT) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, in ? __float_as_uint(v) & 0x7fffffffu : 0u);
        const uint32_t e = block_exponent(top);
        if (threadIdx.x % 32 == 0 && in) f.kept_e[(col / 32) * f.kept_e_ld + row] = static_cast<uint8_t>(e);
        if (in) static_cast<int8_t*>(f.kept)[row * f.kept_ld + col] = static_cast<int8_t>(quantise8(e == kTop8 ? within8(v) : v, block_inverse(e)));
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

// A warp's step is 64 of k.
// ALONG_K: weights [n][k], k adjacent, T x 8 tokens.  A unit is 32 of the n.  Thread (g, q) = (lane / 4, lane % 4) has 16 bytes, k = 8 q ..
// 8 q + 7 of either half step, of rows g, g + 8, g + 16, g + 24 and of tokens g, g + 8 ..: as fragments these are k pairs q,
// and q + 4, of two instructions, the same pairs on both sides.
// Otherwise: weights [k][n], n adjacent, T x 16 tokens.  A unit is 64 of the n.  Thread (g, q) has n = 8 g .. 8 g + 7 of k = 2 q, 2 q + 1,
// 2 q + 8, 2 q + 9 of either quarter step; column g of the eight instructions' j-th is n = 8 g + j.
// A block's warps, and a cluster's blocks, share the k of a unit.  What does not exist is copied as 0.
template <bool ALONG_K, int T>
struct Few {
    static constexpr int kUnit = ALONG_K ? 32 : 64;
    static constexpr int kRows = ALONG_K ? 8 * T : 16 * T;         // tokens
    static constexpr int kWeights = ALONG_K ? 4096 : 8192;         // bytes of a stage
    static constexpr int kStage = kWeights + kRows * 128;
    static constexpr int kAhead = 163840 / (kFewWarps * kStage);
    static constexpr int kRing = kFewWarps * kAhead * kStage;
    static constexpr int kPitch = kRows + 1;                       // part[warp][column][token]
    static constexpr int kPart = kFewWarps * 32 * kPitch * 4;
    static constexpr int kTotal = kRows * kUnit * 4;
    static constexpr int kShared = kRing + kPart + kTotal + kFewWarps * kAhead * 8 + 1024;
};

template <bool ALONG_K, int T>
__global__ void __launch_bounds__(kFewThreads, 1)
few_rows_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, int k, int units,
                const __grid_constant__ Finish f, unsigned int* mark) {
    using S = Few<ALONG_K, T>;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (tc::smem_addr(raw) + 1023u) & ~1023u;
    uint8_t* mem = raw + (base - tc::smem_addr(raw));
    float* part = reinterpret_cast<float*>(mem + S::kRing);
    float* total = part + S::kPart / 4;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, q = lane % 4;
    const uint32_t ring = base + warp * S::kAhead * S::kStage;
    const uint32_t full = base + S::kRing + S::kPart + S::kTotal + warp * S::kAhead * 8;
    const int rank = static_cast<int>(tc::cluster_rank()), blocks = static_cast<int>(tc::cluster_size());
    const int first = static_cast<int>(blockIdx.x) / blocks, apart = static_cast<int>(gridDim.x) / blocks;
    const int stride = blocks * kFewWarps * 64, from = (rank * kFewWarps + warp) * 64;
    const int steps = from < k ? (k - from + stride - 1) / stride : 0;         // of this warp, a unit
    const int mine = first < units ? (units - first + apart - 1) / apart : 0;
    tc::let_next_start();
    if (lane == 0) {
        for (int i = 0; i < S::kAhead; ++i) tc::bar_init(full + 8 * i, 1);
        tc::bar_init_done();
        tc::prefetch_map(&map_w);
        tc::prefetch_map(&map_x);
    }
    __syncwarp();
    tc::wait_for_previous();

    int ahead_unit = first, ahead_at = from, ahead_left = mine * steps, ahead_stage = 0;
    auto fetch = [&] {
        if (ahead_left == 0) return;
        if (tc::elected()) {
            const uint32_t to = ring + ahead_stage * S::kStage, bar = full + 8 * ahead_stage;
            tc::bar_expect(bar, S::kStage);
            if (ALONG_K) {
                tc::load_tile<1>(to, &map_w, ahead_at, ahead_unit * 32, bar);
            } else {
                tc::load_tile<1>(to, &map_w, ahead_unit * 64, ahead_at, bar);
            }
            tc::load_tile<1>(to + S::kWeights, &map_x, ahead_at, 0, bar);
        }
        __syncwarp();
        if (++ahead_stage == S::kAhead) ahead_stage = 0;
        --ahead_left;
        ahead_at += stride;
        if (ahead_at >= k) {
            ahead_at = from;
            ahead_unit += apart;
        }
    };
#pragma unroll 1
    for (int i = 0; i < S::kAhead; ++i) fetch();

    int stage = 0, left = mine * steps;
    uint32_t phase = 0;
    // A wait that ran out ends the waiting and the copying; the sums that follow are of what is there.  The stages still under
    // way are awaited at the end, so that no copy lands in memory that another block has by then.
    int late = 0, late_stage = 0;
    uint32_t late_phase = 0;
    bool fine = true;
    for (int u = first; u < units; u += apart) {
        float c[T][8][4] = {};                 // along k the first two of eight
        // asked for now and turned into a number at the unit's end, a load from memory is waited for nowhere
        // (8 rows over 50257 x 2048: 43 us when loaded at the end)
        uint32_t bias[S::kUnit / 32] = {};
        if (f.bias != nullptr) {
#pragma unroll
            for (int i = 0; i < S::kUnit / 32; ++i) {
                const int64_t col = static_cast<int64_t>(u) * S::kUnit + i * 32 + lane;
                if (col < f.n) {
                    bias[i] = f.bias_f32 ? static_cast<const uint32_t*>(f.bias)[col] : static_cast<const unsigned short*>(f.bias)[col];
                }
            }
        }
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
            if (fine && !tc::bar_wait(full + 8 * stage, phase)) {
                fine = false;
                late = left - ahead_left;
                late_stage = stage;
                late_phase = phase;
                ahead_left = 0;
            }
            --left;
            const uint32_t w = ring + stage * S::kStage, x = w + S::kWeights;
            if constexpr (ALONG_K) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint4 a[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) a[r] = shared16(w + unit_at(g + 8 * r, 4 * half + q));
#pragma unroll
                    for (int t = 0; t < T; ++t) {
                        const uint4 b = shared16(x + unit_at(g + 8 * t, 4 * half + q));
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            mma_16x8x16(c[t][h], a[2 * h].x, a[2 * h + 1].x, a[2 * h].y, a[2 * h + 1].y, b.x, b.y);
                            mma_16x8x16(c[t][h], a[2 * h].z, a[2 * h + 1].z, a[2 * h].w, a[2 * h + 1].w, b.z, b.w);
                        }
                    }
                }
            } else {
#pragma unroll
                for (int part4 = 0; part4 < 4; ++part4) {
                    uint32_t r[4][4], a[T][4];
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const uint4 v = shared16(w + unit_at(16 * part4 + 2 * q + 8 * (i4 / 2) + i4 % 2, g));
                        r[i4][0] = v.x, r[i4][1] = v.y, r[i4][2] = v.z, r[i4][3] = v.w;
                    }
#pragma unroll
                    for (int t = 0; t < T; ++t) {
#pragma unroll
                        for (int i4 = 0; i4 < 4; ++i4) {      // tokens g, g + 8; k 2 q and 2 q + 8: word q of two units
                            a[t][i4] = shared4(x + unit_at(16 * t + g + 8 * (i4 % 2), 2 * part4 + i4 / 2) + 4 * q);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t e0 = __byte_perm(r[0][j], r[1][j], 0x5410), e1 = __byte_perm(r[2][j], r[3][j], 0x5410);
                        const uint32_t o0 = __byte_perm(r[0][j], r[1][j], 0x7632), o1 = __byte_perm(r[2][j], r[3][j], 0x7632);
#pragma unroll
                        for (int t = 0; t < T; ++t) {
                            mma_16x8x16(c[t][2 * j], a[t][0], a[t][1], a[t][2], a[t][3], e0, e1);
                            mma_16x8x16(c[t][2 * j + 1], a[t][0], a[t][1], a[t][2], a[t][3], o0, o1);
                        }
                    }
                }
            }
            __syncwarp();                      // the stage has been read
            if (++stage == S::kAhead) {
                stage = 0;
                phase ^= 1;
            }
            fetch();
        }
        // the warps' sums, 32 columns at a time, then the blocks'
#pragma unroll
        for (int half = 0; half < S::kUnit / 32; ++half) {
            __syncthreads();                   // what was in `part` has been read
            float* to = part + warp * 32 * S::kPitch;
            if constexpr (ALONG_K) {
#pragma unroll
                for (int t = 0; t < T; ++t) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) to[(h * 16 + g + 8 * (i / 2)) * S::kPitch + 8 * t + 2 * q + i % 2] = c[t][h][i];
                    }
                }
            } else if (q / 2 == half) {
#pragma unroll
                for (int t = 0; t < T; ++t) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) to[(16 * (q % 2) + 8 * (i % 2) + j) * S::kPitch + 16 * t + g + 8 * (i / 2)] = c[t][j][i];
                    }
                }
            }
            __syncthreads();
#pragma unroll 1
            for (int t = warp; t < f.m; t += kFewWarps) {
                float v = 0.0f;
#pragma unroll
                for (int i = 0; i < kFewWarps; ++i) v += part[(i * 32 + lane) * S::kPitch + t];
                total[t * S::kUnit + half * 32 + lane] = v;
            }
        }
        if (blocks > 1) tc::cluster_sync();
#pragma unroll 1
        for (int t = warp; t < f.m; t += kFewWarps) {          // the row's own warp, or after the cluster's barrier
            if (t % blocks != rank) continue;
#pragma unroll
            for (int i = 0; i < S::kUnit / 32; ++i) {
                float v = 0.0f;
                if (blocks == 1) {
                    v = total[t * S::kUnit + i * 32 + lane];
                } else {
                    const uint32_t here = tc::smem_addr(total + t * S::kUnit + i * 32 + lane);
#pragma unroll 4
                    for (int r = 0; r < blocks; ++r) v += tc::load_cluster(tc::map_to_rank(here, static_cast<uint32_t>(r)));
                }
                const int64_t col0 = static_cast<int64_t>(u) * S::kUnit + i * 32;
                if (col0 < f.n) finish_row(f, t, col0 + lane, v, __uint_as_float(f.bias_f32 ? bias[i] : bias[i] << 16));
            }
        }
        if (blocks > 1) tc::cluster_sync();    // the sums stay until they are read
    }
    if (!fine) {
        *mark = 1;
        for (; late > 0; --late) {
            tc::bar_wait(full + 8 * late_stage, late_phase);
            if (++late_stage == S::kAhead) {
                late_stage = 0;
                late_phase ^= 1;
            }
        }
    }
}

template <bool ALONG_K, int T>
void start_few(Call& c, const Matrix& a, const Matrix& b, const Finish& f) {
    using S = Few<ALONG_K, T>;
    auto* kernel = &few_rows_kernel<ALONG_K, T>;
    raise_shared(c, kernel, S::kShared);
    CUtensorMap mx, mw;
    int mn = 0;
    if (!make_map(&mx, a, &mn, S::kRows) || !make_map(&mw, b, &mn, 32)) {
        c.status = DLION_ECUDA;
        return;
    }
    const int k = static_cast<int>(a.cols);
    const int64_t units = parts(b.rows, S::kUnit);
    // Clocks: an SM takes in 60 bytes a clock, all of them 3400; sharing k among the blocks of a cluster costs some 3500.
    int blocks = 1;
    double least = 1e300;
    for (int n = 1; n <= 8; n *= 2) {
        if (n > 1 && k <= (n / 2) * kFewWarps * 64) break;
        const double rounds = static_cast<double>(parts(units, std::max<int64_t>(1, c.sms / n)));
        const double t = std::max(rounds * S::kUnit * 2.0 * k / n / 60.0, 2.0 * k * b.rows / 3400.0) + (n > 1 ? 3500.0 * rounds : 0.0);
        if (t < least) {
            least = t;
            blocks = n;
        }
    }
    const int64_t clusters = std::min<int64_t>(units, std::max<int64_t>(1, c.sms / blocks));
    start(c, kernel, dim3(static_cast<unsigned>(clusters * blocks)), dim3(kFewThreads), S::kShared, blocks, mx, mw, k, units, f, c.mark);
}

}  // namespace

// Rows of k adjacent on both the tokens' side and one of the weights' two orders; nothing accumulated.
bool few_rows(Call& c, const Matrix& a, const Matrix& b, const Finish& f) {
    // (a single column's rows may be neighbours: those are not on the 16-byte grid)
    if (a.rows > kFewRows || a.cs != 1 || (a.rows > 1 && a.rs % 8 != 0) || f.accumulated != nullptr) return false;
    if (!c.live()) return true;
    if (b.cs == 1) {
        a.rows <= 8 ? start_few<true, 1>(c, a, b, f) : start_few<true, 2>(c, a, b, f);
    } else {
        start_few<false, 1>(c, a, b, f);
    }
    return true;
}

}  // namespace prod
}  // namespace dlion
