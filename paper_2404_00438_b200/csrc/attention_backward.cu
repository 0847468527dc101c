// The gradients of attention (include/dlion_layers.h).
//
//   p_ij = exp(s_ij - lse_i),  dp_ij = do_i . v_j,  D_i = do_i . out_i,  ds_ij = p_ij (dp_ij - D_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i
//
// in two kernels, one whose blocks keep a tile of queries and its dq, and one whose blocks keep a tile of keys and its dk and dv.
// Scores and dp are computed in both, seven products instead of five; in return nothing is added up across blocks: no atomics,
// whose order would change the results, and no binary32 dq in memory.
//
// Floors, 128 x 128 x 128 twice 1024 clocks: dq three products (1536 for a tile of 128 keys, heads of 128), dk and dv four (2048); operands
// out of shared memory take 1792 and 2048; exponentials 1024 in each.  Measured at 16384 causal rows, 16 heads of 128: dq 1.47 to 1.56 ms
// (1.06 to 1.12 PFLOP/s), dk and dv 1.8 to 1.9 ms (1.16 to 1.22), tensor pipe 52 and 61 % busy, power at the cap; 8 x 1024 rows, 12
// heads of 64: 112 us together, again and again on warm caches.  Bound by the chain score, weight, product of a tile: tensor memory holds
// two tiles' scores for dq, for dk and dv two with heads of 64 and one with wider ones, and one tile's dp.  dq's kernel for heads of 64
// spills 220 bytes a thread (128 registers, two blocks an SM), the others nothing.
//
// p and ds are rounded to bf16 as operands of the second products, whose other operands are bf16 (the instruction takes both of one
// type): 2^-8 of each at most, gradients 0.0023 to 0.0024 of their norm off, where the results' rounding alone is 0.0017.
#include "attention.cuh"

namespace dlion {
namespace att {

namespace {

struct Backward {
    CUtensorMap q, k, v, dout;
    Plan plan;
    int dim, causal;
    Divisor heads, group;                  // heads: of the tiles' own kind
    float c, scale;                        // scale * log2(e)
    Rows out, dout_rows;                   // read row by row
    const float* lse;
    int64_t lse_ld;
    float* delta;                          // [heads][rows], D
    int64_t delta_ld;
    Rows dq, dk, dv;
};

// Four or eight warps of arithmetic, a copying, an issuing and other warps.  Lanes of tensor memory go by warp % 4; of eight warps two
// have the same rows, each 64 columns.  What a warp leaves there as an operand (64 bf16, 32 columns) goes over the first of the
// columns that it has read itself, which leaves a gap of 32 between the operand's halves.

struct Finish {                            // the end of every kernel: see product_kernel
    template <uint32_t COLUMNS>
    __device__ static void end(bool fine, volatile uint32_t* slot_mem, unsigned int* mark, uint32_t tmem, bool frees) {
        if (!fine) {
            slot_mem[1] = 1;
            *mark = 1;
        }
        __syncwarp();
        tc::fence_before();
        __syncthreads();
        if (slot_mem[1] != 0) {            // matrix instructions may still be running: let them end
            const uint64_t t0 = tc::nanoseconds();
            while (tc::nanoseconds() - t0 < 50000000ull) {
            }
        }
        tc::fence_after();
        if (frees) tc::tmem_free<1>(tmem, COLUMNS);
    }
};

// ---------------------------------------------------------------- dq
// Tensor memory: two sets of scores in turn, dp, dq; ds goes over its scores.
//
// D = do . out is off by out's rounding, which matters where a row has few keys: ds is a difference of dp and D, which then is not
// small beside p.  Such rows (those of a tile that sees at most 128 keys) go over their keys twice, and D = sum_j p_ij dp_ij
// is summed in binary32 the first time; dk's kernel takes it from here.  (Gradients of 64 causal rows: 0.0024 off in place of 0.0026,
// of 16 rows 0.0022 in place of 0.0030, where their own rounding is 0.0017.)
template <int D>
struct QueryShared {
    static constexpr int kRows = kPassing<D>, kWarps = kRows / 16;   // of a tile of keys; warps of arithmetic
    static constexpr uint32_t kBytes = kTile * D * 2, kRowBytes = kRows * D * 2;
    static constexpr int kKeys = 3, kValues = 2;                     // stages
    static constexpr uint32_t kStats = 2 * kBytes + (kKeys + kValues) * kRowBytes;    // lse and D of the tile of queries
    static constexpr uint32_t kBars = kStats + 2 * kTile * 4;
    static constexpr uint32_t kAll = kBars + 256 + kTurnBytes + 1024;
    static constexpr uint32_t kColumns = D == 64 ? 256 : 512;        // of tensor memory
    static constexpr int kThreads = 32 * kWarps + 128;               // a copying and an issuing warp, and two that work out D ahead of time
};

template <int D>
__global__ void __launch_bounds__(QueryShared<D>::kThreads, 512 / QueryShared<D>::kColumns) query_gradient_kernel(const __grid_constant__ Backward w, unsigned int* mark) {
    using S = QueryShared<D>;
    constexpr int kRows = S::kRows, kCopying = S::kWarps, kIssuing = kCopying + 1, kAhead = kCopying + 2;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (tc::smem_addr(raw) + 1023u) & ~1023u;
    uint8_t* mem = raw + (base - tc::smem_addr(raw));
    const uint32_t keys = base + 2 * S::kBytes, values = keys + S::kKeys * S::kRowBytes, bars = base + S::kBars;
    const uint32_t k_full = bars, k_empty = bars + 32, v_full = bars + 64, v_empty = bars + 96, scores = bars + 128, products = bars + 144,
                   taken = bars + 152, slopes = bars + 160, rows_full = bars + 176, done = bars + 184, rows_empty = bars + 192, stats_full = bars + 200,
                   stats_empty = bars + 208, slot = bars + 216, meet = bars + 224;
    const uint32_t turns = bars + 256;
    volatile uint32_t* slot_mem = reinterpret_cast<volatile uint32_t*>(mem + (slot - base));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    if (threadIdx.x == 0) {
        tc::bar_init(stats_full, 2);
        tc::bar_init(meet, S::kWarps);
        tc::bar_init(stats_empty, S::kWarps);
        for (int i = 0; i < S::kKeys; ++i) {
            tc::bar_init(k_full + 8 * i, 1);
            tc::bar_init(k_empty + 8 * i, 1);
        }
        for (int i = 0; i < S::kValues; ++i) {
            tc::bar_init(v_full + 8 * i, 1);
            tc::bar_init(v_empty + 8 * i, 1);
        }
        tc::bar_init(scores, 1);
        tc::bar_init(scores + 8, 1);
        tc::bar_init(products, 1);
        tc::bar_init(taken, S::kWarps);
        tc::bar_init(slopes, S::kWarps);                             // in turn: the next ones may all be there before these have been awaited
        tc::bar_init(slopes + 8, S::kWarps);
        tc::bar_init(rows_full, 1);
        tc::bar_init(rows_empty, 1);
        tc::bar_init(done, 1);
        Pieces::init(turns, blockDim.x / 32);
        tc::bar_init_done();
        slot_mem[1] = 0;
        tc::prefetch_map(&w.q);
        tc::prefetch_map(&w.k);
        tc::prefetch_map(&w.v);
        tc::prefetch_map(&w.dout);
    }
    if (warp == kIssuing) tc::tmem_alloc<1>(slot, S::kColumns);
    tc::fence_before();
    __syncthreads();
    tc::let_next_start();                  // now that this block has its tensor memory
    tc::fence_after();
    const uint32_t tmem = same(*slot_mem), products_at = tmem + 2 * kRows, dq_at = products_at + kRows;
    bool fine = true;
    tc::wait_for_previous();

    Pieces pieces(w.plan, w.heads, turns);
    Piece piece{};
    int head = 0, row0 = 0, n = 0;         // a piece's first row in the sequence, its tiles of keys, from the last to the first,
    int rounds = 0;                        // and how often it meets one: n or 2 n times
    auto divide = [&] {
        row0 = piece.tile * kTile;
        n = (min(piece.length, w.causal ? row0 + kTile : piece.length) + kRows - 1) / kRows;
        rounds = (w.causal ? piece.tile == 0 : piece.length <= kTile) ? 2 * n : n;
    };

    if (warp == kCopying) {
        int i = 0, begun = 0, k_asked = 0, v_asked = 0, asked = 0;           // tiles of keys, and pieces, of all
        while (fine && pieces.take(piece, head, fine)) {
            divide();
            const int kv_head = w.group.quotient(head);
            for (int r = 0; r < rounds && fine; ++r, ++i) {
                if (r == rounds - 1) {
                    asked = pieces.turn;
                    if (!(fine = pieces.ask())) break;
                }
                const int row = piece.start + (n - 1 - (r < n ? r : r - n)) * kRows, ks = i % S::kKeys, vs = i % S::kValues;
                if (!(fine = tc::bar_wait(k_empty + 8 * ks, ((i / S::kKeys) & 1) ^ 1))) break;
                if (tc::elected()) {
                    tc::bar_expect(k_full + 8 * ks, S::kRowBytes);
                    load_head<D>(keys + ks * S::kRowBytes, &w.k, kv_head, row, k_full + 8 * ks);
                }
                __syncwarp();
                ++k_asked;
                if (r == 0) {
                    if (!(fine = tc::bar_wait(rows_empty, (begun & 1) ^ 1))) break;
                    if (tc::elected()) {
                        tc::bar_expect(rows_full, 2 * S::kBytes);
                        load_head<D>(base, &w.q, head, piece.start + row0, rows_full);
                        load_head<D>(base + S::kBytes, &w.dout, head, piece.start + row0, rows_full);
                    }
                    __syncwarp();
                    ++begun;
                }
                if (!(fine = tc::bar_wait(v_empty + 8 * vs, ((i / S::kValues) & 1) ^ 1))) break;
                if (tc::elected()) {
                    tc::bar_expect(v_full + 8 * vs, S::kRowBytes);
                    load_head<D>(values + vs * S::kRowBytes, &w.v, kv_head, row, v_full + 8 * vs);
                }
                __syncwarp();
                ++v_asked;
            }
        }
        if (!fine) {                       // what was asked for still lands in this block's memory: it is awaited
            pieces.settle(asked);
            if (begun > 0) tc::bar_wait(rows_full, (begun - 1) & 1);
            for (int a = max(0, k_asked - S::kKeys); a < k_asked; ++a) tc::bar_wait(k_full + 8 * (a % S::kKeys), (a / S::kKeys) & 1);
            for (int a = max(0, v_asked - S::kValues); a < v_asked; ++a) tc::bar_wait(v_full + 8 * (a % S::kValues), (a / S::kValues) & 1);
        }
    } else if (warp == kIssuing) {
        const int k_steps = (w.dim + 15) / 16;
        const uint32_t wide = tc::instruction(kTile, k_steps * 16, 0, 1);
        auto finished = [&](uint32_t bar) {
            if (tc::elected()) tc::commit<1>(bar);
            __syncwarp();
        };
        // A round: scores of a tile of keys (two sets of columns in turn), its dp once the last one's has been read, then dq of the
        // round before, which may be the last piece's.
        int i = 0, begun = 0, steps = 0;
        bool first = false, last = false, summing = false;
        auto gather = [&] {
            const int b = i - 1;
            if (!(fine = tc::bar_wait(slopes + 8 * (b & 1), (b >> 1) & 1))) return;
            tc::fence_after();
            if (!summing) weights_by_rows<0, kRows / 16, 32>(dq_at, tmem + (b & 1) * kRows, keys + (b % S::kKeys) * S::kRowBytes, wide, steps, !first);
            if (last) finished(done);
            finished(k_empty + 8 * (b % S::kKeys));
        };
        while (fine && pieces.take(piece, head, fine)) {
            divide();
            for (int r = 0; r < rounds && fine; ++r, ++i) {
                if (r == 0 && !(fine = tc::bar_wait(rows_full, begun++ & 1))) break;
                if (!(fine = tc::bar_wait(k_full + 8 * (i % S::kKeys), (i / S::kKeys) & 1))) break;
                tc::fence_after();
                rows_by_rows<D, kRows>(tmem + (i & 1) * kRows, base, keys + (i % S::kKeys) * S::kRowBytes, k_steps);
                finished(scores + 8 * (i & 1));
                if (!(fine = tc::bar_wait(v_full + 8 * (i % S::kValues), (i / S::kValues) & 1))) break;
                if (i > 0 && !(fine = tc::bar_wait(taken, (i - 1) & 1))) break;
                tc::fence_after();
                rows_by_rows<D, kRows>(products_at, base + S::kBytes, values + (i % S::kValues) * S::kRowBytes, k_steps);
                finished(products);
                finished(v_empty + 8 * (i % S::kValues));
                if (r == rounds - 1) finished(rows_empty);
                if (i > 0) gather();
                steps = (min(kRows, piece.length - (n - 1 - (r < n ? r : r - n)) * kRows) + 15) / 16;
                summing = r < rounds - n;
                first = r == rounds - n;
                last = r == rounds - 1;
            }
        }
        if (fine && i > 0) gather();
    } else if (warp >= kAhead) {
        // D = do . out of half the tile's rows, D / 8 lanes a row, while the others work on the piece before
        constexpr int kLanes = D / 8, kEach = 32 / kLanes, kAtOnce = D == 64 ? 4 : 8;
        float* stats = reinterpret_cast<float*>(mem + S::kStats);
        const int unit = lane % kLanes;
        int begun = 0;
        while (fine && pieces.take(piece, head, fine)) {
            divide();
            float lse[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = row0 + (warp - kAhead) * (kTile / 2) + e * 32 + lane;
                lse[e] = row < piece.length ? w.lse[head * w.lse_ld + piece.start + row] * kLog2e : 0.0f;
            }
            if (!(fine = tc::bar_wait(stats_empty, (begun & 1) ^ 1))) break;
            for (int first = (warp - kAhead) * (kTile / 2); rounds == n && first < (warp - kAhead + 1) * (kTile / 2); first += kAtOnce * kEach) {
                uint4 o[kAtOnce], d[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int row = row0 + first + u * kEach + lane / kLanes;
                    const bool live = row < piece.length && unit * 8 < w.dim;
                    const int64_t at = piece.start + row;
                    o[u] = live ? *reinterpret_cast<const uint4*>(w.out.p + at * w.out.rs + head * w.out.hs + unit * 8) : make_uint4(0, 0, 0, 0);
                    d[u] = live ? *reinterpret_cast<const uint4*>(w.dout_rows.p + at * w.dout_rows.rs + head * w.dout_rows.hs + unit * 8) : make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    float2 x[4], y[4], sum = twice(0.0f);
                    widen(o[u], x);
                    widen(d[u], y);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum = fma2(x[e], y[e], sum);
                    float delta = sum.x + sum.y;
#pragma unroll
                    for (int e = kLanes / 2; e >= 1; e /= 2) delta += __shfl_xor_sync(0xffffffffu, delta, e);
                    const int in_tile = first + u * kEach + lane / kLanes;
                    if (unit == 0 && row0 + in_tile < piece.length) {
                        const int64_t at = piece.start + row0 + in_tile;
                        w.delta[head * w.delta_ld + at] = delta;
                        stats[kTile + in_tile] = delta;
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) stats[(warp - kAhead) * (kTile / 2) + e * 32 + lane] = lse[e];
            __syncwarp();
            if (lane == 0) tc::bar_arrive(stats_full);
            ++begun;
        }
    } else {
        const int half = warp / 4, quarter = warp % 4;
        const float* stats = reinterpret_cast<const float*>(mem + S::kStats);
        const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
        const float2 cc = twice(w.c);
        int i = 0, ended = 0, met = 0;
        bool more = pieces.take(piece, head, fine);
        while (fine && more) {
            divide();
            const int row = row0 + quarter * 32 + lane;
            const bool live = row < piece.length;
            if (!(fine = tc::bar_wait(stats_full, ended & 1))) break;
            const float lse2 = live ? stats[quarter * 32 + lane] : 0.0f, delta = live ? stats[kTile + quarter * 32 + lane] : 0.0f;
            __syncwarp();
            if (lane == 0) tc::bar_arrive(stats_empty);
            const float2 minus = twice(-lse2);
            float2 less = twice(-delta), sum = twice(0.0f);
            for (int r = 0; r < rounds; ++r, ++i) {
                const int j = n - 1 - (r < n ? r : r - n), valid = piece.length - j * kRows;
                const uint32_t s_at = tmem + (i & 1) * kRows + half * 64 + lanes;
                if (!(fine = tc::bar_wait(scores + 8 * (i & 1), (i >> 1) & 1))) break;
                tc::fence_after();
                float s[64];
                tmem_load64(s_at, s);
#pragma unroll
                for (int e = 0; e < 64; e += 2) {
                    const float2 x = fma2(make_float2(s[e], s[e + 1]), cc, minus);
                    s[e] = exp2_fast(x.x);
                    s[e + 1] = exp2_fast(x.y);
                }
                if (!(fine = tc::bar_wait(products, i & 1))) break;
                tc::fence_after();
                float dp[64];
                tmem_load64(products_at + half * 64 + lanes, dp);
                tc::fence_before();
                __syncwarp();
                if (lane == 0) tc::bar_arrive(taken);
                const bool masked = valid < kRows || (w.causal && (j + 1) * kRows > row0);
                const int behind = (w.causal ? min(row, piece.length - 1) : piece.length - 1) - j * kRows - half * 64;
                if (r < rounds - n) {      // D alone
#pragma unroll
                    for (int e = 0; e < 64; e += 2) {
                        const float2 x = mul2(make_float2(dp[e], dp[e + 1]), make_float2(s[e], s[e + 1]));
                        sum = add2(sum, masked ? make_float2(e <= behind ? x.x : 0.0f, e < behind ? x.y : 0.0f) : x);
                    }
                    if (r == n - 1) {
                        float d = sum.x + sum.y;
                        if (S::kWarps == 8) {                        // the other half of the row has the rest
                            tmem_store1(s_at, d);
                            tmem_stored();
                            tc::fence_before();
                            __syncwarp();
                            if (lane == 0) tc::bar_arrive(meet);
                            if (!(fine = tc::bar_wait(meet, met++ & 1))) break;
                            tc::fence_after();
                            const float other = tmem_load1(tmem + (i & 1) * kRows + (half ^ 1) * 64 + lanes);
                            d = half == 0 ? d + other : other + d;
                            // (both have read before either's scores are overwritten: each announces it below)
                        }
                        less = twice(-d);
                        if (half == 0 && live) w.delta[head * w.delta_ld + piece.start + row] = d;
                    }
                    tc::fence_before();
                    __syncwarp();
                    if (lane == 0) tc::bar_arrive(slopes + 8 * (i & 1));
                    continue;
                }
#pragma unroll
                for (int e = 0; e < 64; e += 2) {
                    const float2 x = mul2(add2(make_float2(dp[e], dp[e + 1]), less), make_float2(s[e], s[e + 1]));
                    s[e] = x.x;
                    s[e + 1] = x.y;
                }
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 64; ++e) s[e] = e <= behind ? s[e] : 0.0f;
                    if (valid < kRows) {   // the keys' rows behind the sequence
                        if (!(fine = tc::bar_wait(k_full + 8 * (i % S::kKeys), (i / S::kKeys) & 1))) break;
                        clear_rows<D>(mem + (keys - base) + (i % S::kKeys) * S::kRowBytes, valid, threadIdx.x, 32 * S::kWarps);
                    }
                }
                uint32_t p[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) p[e] = pack_bf16(s[2 * e], s[2 * e + 1]);
                tmem_store32(s_at, p);
                tmem_stored();
                tc::fence_before();
                __syncwarp();
                if (lane == 0) tc::bar_arrive(slopes + 8 * (i & 1));
            }
            if (!fine) break;
            constexpr int kColumns = D * 64 / kRows;                 // of dq: all, or half of them a warp
            __nv_bfloat16* to = w.dq.p + static_cast<int64_t>(piece.start + row) * w.dq.rs + head * w.dq.hs + half * kColumns;
            more = pieces.take(piece, head, fine);                   // the next one's whereabouts, while the last product runs
            if (!fine || !(fine = tc::bar_wait(done, ended++ & 1))) break;
            tc::fence_after();
            give_row<kColumns>(dq_at + half * kColumns + lanes, w.scale, to, live, w.dim - half * kColumns);
            tc::fence_before();
        }
    }
    Finish::end<S::kColumns>(fine, slot_mem, mark, tmem, warp == kIssuing);
}

// ---------------------------------------------------------------- dk, dv
// Scores and dp are computed transposed, keys as rows: so p and ds are operands as they lie in tensor memory.  With heads of up to 64
// columns there is room for a second set of scores; that took less time than two blocks an SM with tiles of 64 queries, at every length (8 x
// 1024 rows, 12 heads, forward and backward: 148 us, 152 so; 64 x 197 rows backward 130, 136).
template <int D>
struct KeyShared {
    static constexpr int kRows = kTile, kWarps = kRows / 16;         // of a tile of queries; warps of arithmetic
    static constexpr uint32_t kBytes = kTile * D * 2, kRowBytes = kRows * D * 2;
    static constexpr int kStages = D == 64 ? 3 : 2;                  // of queries and of do
    static constexpr uint32_t kStats = 2 * kBytes + 2 * kStages * kRowBytes;          // lse and D of two tiles of queries
    static constexpr uint32_t kBars = kStats + 2 * 2 * kRows * 4;
    static constexpr uint32_t kAll = kBars + 256 + kTurnBytes + 1024;
    static constexpr uint32_t kColumns = 512;                        // of tensor memory
    static constexpr int kSets = D == 64 ? 2 : 1;                    // of scores: where there is room, the next ones do not wait for dv
    static constexpr int kThreads = 32 * kWarps + 96;                // a copying and an issuing warp, and one that brings lse and D
};

template <int D>
__global__ void __launch_bounds__(KeyShared<D>::kThreads, 1) key_gradient_kernel(const __grid_constant__ Backward w, unsigned int* mark) {
    using S = KeyShared<D>;
    constexpr int kRows = S::kRows, kSets = S::kSets, kStages = S::kStages, kCopying = S::kWarps, kIssuing = kCopying + 1, kAhead = kCopying + 2;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (tc::smem_addr(raw) + 1023u) & ~1023u;
    uint8_t* mem = raw + (base - tc::smem_addr(raw));
    const uint32_t queries = base + 2 * S::kBytes, douts = queries + kStages * S::kRowBytes, bars = base + S::kBars;
    const uint32_t q_full = bars, q_empty = bars + 24, d_full = bars + 48, d_empty = bars + 72, scores = bars + 96, products = bars + 112,
                   weights = bars + 120, slopes = bars + 136, rows_full = bars + 144, done = bars + 152, rows_empty = bars + 160,
                   stats_full = bars + 168, stats_empty = bars + 184, slot = bars + 200;
    const uint32_t turns = bars + 256;
    volatile uint32_t* slot_mem = reinterpret_cast<volatile uint32_t*>(mem + (slot - base));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            tc::bar_init(q_full + 8 * i, 1);
            tc::bar_init(q_empty + 8 * i, 1);
            tc::bar_init(d_full + 8 * i, 1);
            tc::bar_init(d_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::bar_init(stats_full + 8 * i, 1);
            tc::bar_init(stats_empty + 8 * i, S::kWarps);
            tc::bar_init(scores + 8 * i, 1);
            tc::bar_init(weights + 8 * i, S::kWarps);                // in turn: with two sets of scores the next ones may all be there
        }
        tc::bar_init(products, 1);
        tc::bar_init(slopes, S::kWarps);
        tc::bar_init(rows_full, 1);
        tc::bar_init(rows_empty, 1);
        tc::bar_init(done, 1);
        Pieces::init(turns, blockDim.x / 32);
        tc::bar_init_done();
        slot_mem[1] = 0;
        tc::prefetch_map(&w.q);
        tc::prefetch_map(&w.k);
        tc::prefetch_map(&w.v);
        tc::prefetch_map(&w.dout);
    }
    if (warp == kIssuing) tc::tmem_alloc<1>(slot, S::kColumns);
    tc::fence_before();
    __syncthreads();
    tc::let_next_start();                  // now that this block has its tensor memory
    tc::fence_after();
    const uint32_t tmem = same(*slot_mem), products_at = tmem + kSets * kRows, dk_at = products_at + kRows, dv_at = dk_at + D;
    bool fine = true;
    tc::wait_for_previous();

    Pieces pieces(w.plan, w.heads, turns);
    Piece piece{};
    int kv_head = 0, key0 = 0, first = 0, per = 0, n = 0;            // tiles of queries: of a head, the first of them, and in all
    const int group = static_cast<int>(w.group.d);
    auto divide = [&] {
        key0 = piece.tile * kTile;
        first = w.causal ? key0 / kRows : 0;
        per = (piece.length + kRows - 1) / kRows - first;
        n = per * group;
    };
    // The tiles of queries in turn: the query heads that share these keys one after the other.
    int head = 0, tile = 0;
    auto begin = [&] {
        head = kv_head * group;
        tile = first;
    };
    auto advance = [&] {
        if (++tile == first + per) {
            tile = first;
            ++head;
        }
    };

    if (warp == kCopying) {
        int i = 0, begun = 0, q_asked = 0, d_asked = 0, asked = 0;
        while (fine && pieces.take(piece, kv_head, fine)) {
            divide();
            begin();
            for (int r = 0; r < n && fine; ++r, ++i, advance()) {
                if (r == n - 1) {
                    asked = pieces.turn;
                    if (!(fine = pieces.ask())) break;
                }
                const int row = piece.start + tile * kRows, st = i % kStages;
                const uint32_t parity = ((i / kStages) & 1) ^ 1;
                if (!(fine = tc::bar_wait(q_empty + 8 * st, parity))) break;
                if (tc::elected()) {
                    tc::bar_expect(q_full + 8 * st, S::kRowBytes);
                    load_head<D>(queries + st * S::kRowBytes, &w.q, head, row, q_full + 8 * st);
                }
                __syncwarp();
                ++q_asked;
                if (r == 0) {
                    if (!(fine = tc::bar_wait(rows_empty, (begun & 1) ^ 1))) break;
                    if (tc::elected()) {
                        tc::bar_expect(rows_full, 2 * S::kBytes);
                        load_head<D>(base, &w.k, kv_head, piece.start + key0, rows_full);
                        load_head<D>(base + S::kBytes, &w.v, kv_head, piece.start + key0, rows_full);
                    }
                    __syncwarp();
                    ++begun;
                }
                if (!(fine = tc::bar_wait(d_empty + 8 * st, parity))) break;
                if (tc::elected()) {
                    tc::bar_expect(d_full + 8 * st, S::kRowBytes);
                    load_head<D>(douts + st * S::kRowBytes, &w.dout, head, row, d_full + 8 * st);
                }
                __syncwarp();
                ++d_asked;
            }
        }
        if (!fine) {                       // what was asked for still lands in this block's memory: it is awaited
            pieces.settle(asked);
            if (begun > 0) tc::bar_wait(rows_full, (begun - 1) & 1);
            for (int a = max(0, q_asked - kStages); a < q_asked; ++a) tc::bar_wait(q_full + 8 * (a % kStages), (a / kStages) & 1);
            for (int a = max(0, d_asked - kStages); a < d_asked; ++a) tc::bar_wait(d_full + 8 * (a % kStages), (a / kStages) & 1);
        }
    } else if (warp == kAhead) {
        float* stats = reinterpret_cast<float*>(mem + S::kStats);
        int i = 0;
        while (fine && pieces.take(piece, kv_head, fine)) {
            divide();
            begin();
            for (int r = 0; r < n; ++r, ++i, advance()) {
                const int st = i & 1;
                float lse[kRows / 32], delta[kRows / 32];
#pragma unroll
                for (int e = 0; e < kRows / 32; ++e) {
                    const int row = tile * kRows + e * 32 + lane;
                    const bool live = row < piece.length;
                    lse[e] = live ? w.lse[head * w.lse_ld + piece.start + row] * kLog2e : 0.0f;
                    delta[e] = live ? w.delta[head * w.delta_ld + piece.start + row] : 0.0f;
                }
                if (!(fine = tc::bar_wait(stats_empty + 8 * st, ((i >> 1) & 1) ^ 1))) break;
#pragma unroll
                for (int e = 0; e < kRows / 32; ++e) {
                    stats[st * 2 * kRows + e * 32 + lane] = -lse[e];
                    stats[st * 2 * kRows + kRows + e * 32 + lane] = -delta[e];
                }
                __syncwarp();
                if (lane == 0) tc::bar_arrive(stats_full + 8 * st);
            }
        }
    } else if (warp == kIssuing) {
        const int k_steps = (w.dim + 15) / 16;
        const uint32_t wide = tc::instruction(kTile, k_steps * 16, 0, 1);
        auto finished = [&](uint32_t bar) {
            if (tc::elected()) tc::commit<1>(bar);
            __syncwarp();
        };
        int i = 0, begun = 0, steps = 0;
        bool opening = false, last = false;                          // of the round before
        auto score = [&] {
            const int st = i % kStages;
            if (!(fine = tc::bar_wait(q_full + 8 * st, (i / kStages) & 1))) return;
            tc::fence_after();
            rows_by_rows<D, kRows>(tmem + (i % kSets) * kRows, base, queries + st * S::kRowBytes, k_steps);
            finished(scores + 8 * (i % kSets));
        };
        auto product = [&] {
            const int st = i % kStages;
            if (!(fine = tc::bar_wait(d_full + 8 * st, (i / kStages) & 1))) return;
            tc::fence_after();
            rows_by_rows<D, kRows>(products_at, base + S::kBytes, douts + st * S::kRowBytes, k_steps);
            finished(products);
        };
        auto gather_v = [&] {
            const int b = i - 1, sb = b % kStages;
            if (!(fine = tc::bar_wait(weights + 8 * (b & 1), (b >> 1) & 1))) return;
            tc::fence_after();
            weights_by_rows<0, kRows / 16, 32>(dv_at, tmem + (b % kSets) * kRows, douts + sb * S::kRowBytes, wide, steps, !opening);
            finished(d_empty + 8 * sb);
        };
        auto gather_k = [&] {
            const int b = i - 1, sb = b % kStages;
            if (!(fine = tc::bar_wait(slopes, b & 1))) return;
            tc::fence_after();
            weights_by_rows<0, kRows / 16, 32>(dk_at, products_at, queries + sb * S::kRowBytes, wide, steps, !opening);
            finished(q_empty + 8 * sb);
            if (last) finished(done);
        };
        // A round: dv of the round before, the scores (with one set of them, over its weights), dk of the round before, dp over its slopes.
        while (fine && pieces.take(piece, kv_head, fine)) {
            divide();
            begin();
            for (int r = 0; r < n && fine; ++r, ++i, advance()) {
                if (r == 0 && !(fine = tc::bar_wait(rows_full, begun++ & 1))) break;
                if (kSets == 2) score();
                if (fine && i > 0) gather_v();
                if (fine && kSets == 1) score();
                if (fine && i > 0) gather_k();
                if (fine) product();
                if (!fine) break;
                if (r == n - 1) finished(rows_empty);
                steps = (min(kRows, piece.length - tile * kRows) + 15) / 16;
                opening = r == 0;
                last = r == n - 1;
            }
        }
        if (fine && i > 0) gather_v();
        if (fine && i > 0) gather_k();
    } else {
        const int half = warp / 4, quarter = warp % 4;
        const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t d_at = products_at + half * 64 + lanes;
        const float* stats = reinterpret_cast<const float*>(mem + S::kStats);
        const float2 cc = twice(w.c);
        int i = 0, ended = 0;
        bool more = pieces.take(piece, kv_head, fine);
        while (fine && more) {
            divide();
            begin();
            const int key = key0 + quarter * 32 + lane;
            for (int r = 0; r < n; ++r, ++i, advance()) {
                const int st = i & 1, valid = piece.length - tile * kRows;
                const uint32_t s_at = tmem + (i % kSets) * kRows + half * 64 + lanes;
                const float4* lse = reinterpret_cast<const float4*>(stats + st * 2 * kRows + half * 64);
                const float4* delta = lse + kRows / 4;
                const bool masked = valid < kRows || (w.causal && tile * kRows < key0 + kTile);
                const int low = w.causal ? key - tile * kRows - half * 64 : 0, high = valid - half * 64;     // queries [low, high) of this warp's columns
                if (!(fine = tc::bar_wait(stats_full + 8 * st, (i >> 1) & 1))) break;
                if (!(fine = tc::bar_wait(scores + 8 * (i % kSets), (i / kSets) & 1))) break;
                tc::fence_after();
                float s[64];
                tmem_load64(s_at, s);
#pragma unroll
                for (int e = 0; e < 64; e += 4) {
                    const float4 x = lse[e / 4];
                    const float2 a = fma2(make_float2(s[e], s[e + 1]), cc, make_float2(x.x, x.y)), b = fma2(make_float2(s[e + 2], s[e + 3]), cc, make_float2(x.z, x.w));
                    s[e] = exp2_fast(a.x);
                    s[e + 1] = exp2_fast(a.y);
                    s[e + 2] = exp2_fast(b.x);
                    s[e + 3] = exp2_fast(b.y);
                }
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 64; ++e) s[e] = e >= low && e < high ? s[e] : 0.0f;
                    if (valid < kRows) {   // the queries' rows behind the sequence
                        const int at = i % kStages;
                        const uint32_t parity = (i / kStages) & 1;
                        if (!(fine = tc::bar_wait(q_full + 8 * at, parity))) break;
                        if (!(fine = tc::bar_wait(d_full + 8 * at, parity))) break;
                        clear_rows<D>(mem + (queries - base) + at * S::kRowBytes, valid, threadIdx.x, 32 * S::kWarps);
                        clear_rows<D>(mem + (douts - base) + at * S::kRowBytes, valid, threadIdx.x, 32 * S::kWarps);
                    }
                }
                uint32_t p[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) p[e] = pack_bf16(s[2 * e], s[2 * e + 1]);
                tmem_store32(s_at, p);
                tmem_stored();
                tc::fence_before();
                __syncwarp();
                if (lane == 0) tc::bar_arrive(weights + 8 * (i & 1));
                if (!(fine = tc::bar_wait(products, i & 1))) break;
                tc::fence_after();
                float dp[64];
                tmem_load64(d_at, dp);
#pragma unroll
                for (int e = 0; e < 64; e += 4) {
                    const float4 x = delta[e / 4];
                    const float2 a = mul2(add2(make_float2(dp[e], dp[e + 1]), make_float2(x.x, x.y)), make_float2(s[e], s[e + 1]));
                    const float2 b = mul2(add2(make_float2(dp[e + 2], dp[e + 3]), make_float2(x.z, x.w)), make_float2(s[e + 2], s[e + 3]));
                    dp[e] = a.x;
                    dp[e + 1] = a.y;
                    dp[e + 2] = b.x;
                    dp[e + 3] = b.y;
                }
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 64; ++e) dp[e] = e >= low && e < high ? dp[e] : 0.0f;
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) p[e] = pack_bf16(dp[2 * e], dp[2 * e + 1]);
                tmem_store32(d_at, p);
                tmem_stored();
                tc::fence_before();
                __syncwarp();
                if (lane == 0) {
                    tc::bar_arrive(slopes);
                    tc::bar_arrive(stats_empty + 8 * st);
                }
            }
            if (!fine) break;
            constexpr int kHalf = D / 2;                             // columns of a warp
            const bool live = key < piece.length;
            const int64_t at = piece.start + key;
            __nv_bfloat16 *to_k = w.dk.p + at * w.dk.rs + kv_head * w.dk.hs + half * kHalf, *to_v = w.dv.p + at * w.dv.rs + kv_head * w.dv.hs + half * kHalf;
            more = pieces.take(piece, kv_head, fine);                // the next one's whereabouts, while the last products run
            if (!fine || !(fine = tc::bar_wait(done, ended++ & 1))) break;
            tc::fence_after();
            give_row<kHalf>(dk_at + half * kHalf + lanes, w.scale, to_k, live, w.dim - half * kHalf);
            give_row<kHalf>(dv_at + half * kHalf + lanes, 1.0f, to_v, live, w.dim - half * kHalf);
            tc::fence_before();
        }
    }
    Finish::end<S::kColumns>(fine, slot_mem, mark, tmem, warp == kIssuing);
}

Sequences sequences_of(const dlion_attention_bwd& p) { return Sequences{p.rows, p.length, p.sequences, p.offsets, p.offsets_64}; }

dlion_status check(const dlion_attention_bwd* p) {
    if (p == nullptr || p->heads < 1 || p->kv_heads < 1 || p->heads > 65535 || p->heads % p->kv_heads != 0) return DLION_EINVAL;
    if (p->dim < 8 || p->dim > 128 || p->dim % 8 != 0 || p->causal < 0 || p->causal > 1 || !scale_ok(p->scale)) return DLION_EINVAL;
    const dlion_status seq = check_sequences(sequences_of(*p));
    if (seq != DLION_OK) return seq;
    if (p->zero_rest < 0 || p->zero_rest > 1 || p->lse_ld < p->rows) return DLION_EINVAL;
    for (const Operand& a : {Operand{p->q, p->q_rs, p->q_hs, p->heads}, Operand{p->k, p->k_rs, p->k_hs, p->kv_heads},
                             Operand{p->v, p->v_rs, p->v_hs, p->kv_heads}, Operand{p->out, p->out_rs, p->out_hs, p->heads},
                             Operand{p->dout, p->dout_rs, p->dout_hs, p->heads}, Operand{p->dq, p->dq_rs, p->dq_hs, p->heads},
                             Operand{p->dk, p->dk_rs, p->dk_hs, p->kv_heads}, Operand{p->dv, p->dv_rs, p->dv_hs, p->kv_heads}}) {
        const dlion_status st = check_operand(a, p->rows, p->dim);
        if (st != DLION_OK) return st;
    }
    if (p->rows > 0 && p->lse == nullptr) return DLION_EINVAL;
    if (!aligned(p->lse, 4)) return DLION_EALIGN;
    return most_pieces(sequences_of(*p), kTile) * p->heads <= INT_MAX / 2 ? DLION_OK : DLION_EINVAL;
}

template <int D>
void launch(prod::Call& c, Backward& w, const dlion_attention_bwd& p, const Plan* plans, int64_t pieces) {
    prod::raise_shared(c, &query_gradient_kernel<D>, QueryShared<D>::kAll);
    prod::raise_shared(c, &key_gradient_kernel<D>, KeyShared<D>::kAll);
    // the tiles that a block keeps, and those that pass by
    auto maps = [&](int queries, int keys) {
        return map_rows(&w.q, Operand{p.q, p.q_rs, p.q_hs, p.heads}, p.rows, p.dim, queries) &&
               map_rows(&w.dout, Operand{p.dout, p.dout_rs, p.dout_hs, p.heads}, p.rows, p.dim, queries) &&
               map_rows(&w.k, Operand{p.k, p.k_rs, p.k_hs, p.kv_heads}, p.rows, p.dim, keys) &&
               map_rows(&w.v, Operand{p.v, p.v_rs, p.v_hs, p.kv_heads}, p.rows, p.dim, keys);
    };
    if (!maps(kTile, kPassing<D>)) c.status = DLION_ECUDA;
    w.plan = plans[0];
    w.heads = divisor(p.heads);
    prod::start(c, query_gradient_kernel<D>, dim3(static_cast<unsigned>(pieces * p.heads)), dim3(QueryShared<D>::kThreads), QueryShared<D>::kAll, 1, w, c.mark);
    if (!maps(kTile, kTile)) c.status = DLION_ECUDA;
    w.plan = plans[1];
    w.heads = divisor(p.kv_heads);
    prod::start(c, key_gradient_kernel<D>, dim3(static_cast<unsigned>(pieces * p.kv_heads)), dim3(KeyShared<D>::kThreads), KeyShared<D>::kAll, 1, w, c.mark);
}

void backward(prod::Call& c, const dlion_attention_bwd& p) {
    const Sequences seq = sequences_of(p);
    const int64_t pieces = most_pieces(seq, kTile);
    if (p.rows == 0) return;
    int4* tables[2] = {nullptr, nullptr};
    if (p.offsets != nullptr) {
        tables[0] = c.ws.take<int4>(pieces);
        tables[1] = c.ws.take<int4>(pieces);
    }
    float* delta = c.ws.take<float>(static_cast<uint64_t>(p.rows) * p.heads);
    if (!c.live()) return;
    auto rows = [](const void* t, int64_t rs, int64_t hs) { return Rows{static_cast<__nv_bfloat16*>(const_cast<void*>(t)), rs, hs}; };
    Backward w{};
    w.dq = rows(p.dq, p.dq_rs, p.dq_hs);
    w.dk = rows(p.dk, p.dk_rs, p.dk_hs);
    w.dv = rows(p.dv, p.dv_rs, p.dv_hs);
    Clear clear{};
    if (p.zero_rest) {
        clear.t[0] = w.dq;
        clear.t[1] = w.dk;
        clear.t[2] = w.dv;
        clear.heads[0] = static_cast<int>(p.heads);
        clear.heads[1] = clear.heads[2] = static_cast<int>(p.kv_heads);
        clear.count = 3;
        clear.dim = static_cast<int>(p.dim);
    }
    const PlanRequest requests[2] = {{kTile, p.causal, 0}, {kTile, p.causal, 1}};
    Plan plans[2];
    make_plans(c, seq, requests, 2, tables, plans, p.zero_rest ? &clear : nullptr);
    if (pieces == 0) return;
    w.group = divisor(p.heads / p.kv_heads);
    w.dim = static_cast<int>(p.dim);
    w.causal = p.causal;
    w.c = p.scale * kLog2e;
    w.scale = p.scale;
    w.out = rows(p.out, p.out_rs, p.out_hs);
    w.dout_rows = rows(p.dout, p.dout_rs, p.dout_hs);
    w.lse = p.lse;
    w.lse_ld = p.lse_ld;
    w.delta = delta;
    w.delta_ld = p.rows;
    p.dim <= 64 ? launch<64>(c, w, p, plans, pieces) : launch<128>(c, w, p, plans, pieces);
}

}  // namespace
}  // namespace att
}  // namespace dlion

extern "C" {

uint64_t dlion_attention_backward_workspace(const dlion_attention_bwd* p) {
    return dlion::att::check(p) == DLION_OK ? dlion::prod::workspace_of(*p, dlion::att::backward) : 0;
}

dlion_status dlion_attention_backward(const dlion_attention_bwd* p, void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
    const dlion_status st = dlion::att::check(p);
    return st != DLION_OK ? st : dlion::prod::run(*p, dlion::att::backward, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
