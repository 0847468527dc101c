// Attention over whole sequences (include/dlion_layers.h).
//
//   s_ij = scale q_i . k_j,  out_i = sum_j exp(s_ij - lse_i) v_j,  lse_i = log sum_j exp s_ij
//
// in one pass over the keys: with m the running maximum of a row, its sum l and its output o are held relative to exp(m) and
// rescaled when m grows.
//
// The weights are rounded to bf16 as operands of the second product: the matrix instruction takes both of one type, and v is bf16.  l is
// their sum before that.  A weight is off by 2^-8 of itself at most, the output by about as much again as by its own rounding (0.0018 to
// 0.0023 of its norm against 64 bits, where the rounding of the result alone is 0.0017).
//
// Floors: 4 d operations a score on the tensor cores (128 x 128 x 128 twice: 1024 clocks), one exponential a score (16 a clock and SM:
// 1024 clocks for 128 x 128).  What bounds it is neither alone: a row's scores, maximum, exponentials and weights and the two products
// wait for one another, and what runs beside them is another tile's.  16384 causal rows, 16 heads: of 128 0.93 to 1.1 ms (1.0 to 1.18
// PFLOP/s, the lower figure under the power cap; tensor pipe 53 %, special functions 53 % busy), of 64 0.80 ms (690 TFLOP/s; special
// functions 54 % busy).  All warps of a block have the same number of registers, and those of the arithmetic have too few: with heads
// of 64 (96 registers, three blocks an SM) they spill 290 bytes a thread, with wider ones (168) 120 to 160.  Tried in vain, with these
// spills: part of the exponentials as polynomials on the multiply-add pipe (equal within 3 %, more power), half a row a thread (equal),
// turns at the special function units (slower), passing over masked blocks of 32 keys (a second copy of the loop costs more than it
// saves).
#include "attention.cuh"

namespace dlion {
namespace att {

namespace {

constexpr int64_t kLongCausal = 1024, kLongFull = 256;               // rows a sequence

struct Forward {
    CUtensorMap q, k, v;
    Plan plan;
    int dim, causal;
    Divisor heads, group;
    float c;                               // scale * log2(e)
    Rows out;
    float* lse;
    int64_t lse_ld;
};

// SIDES tiles of queries share each tile of keys and values that a block copies.  Every side has a group of four warps, a row a
// thread; one warp copies and one issues the products.  With two sides one's exponentials run while the tensor cores work for the
// other; with one, the blocks of an SM do that for each other.
template <int D, int SIDES>
struct ForwardShared {
    static constexpr int kKeys = kPassing<D>;
    static constexpr uint32_t kBytes = kTile * D * 2, kKeyBytes = kKeys * D * 2;      // of a tile
    static constexpr int kRing = D == 128 && SIDES == 1 ? 2 : 4;     // tiles of keys and values, in turn
    static constexpr uint32_t kStages = SIDES * kBytes + kRing * kKeyBytes;           // results on their way out
    static constexpr uint32_t kBars = kStages + 4 * SIDES * kStage;
    static constexpr uint32_t kAll = kBars + 256 + kTurnBytes + 1024;
    static constexpr int kThreads = 128 * SIDES + 64;
    static constexpr uint32_t kColumns = SIDES * (kKeys + D);        // of tensor memory: scores, over them weights, and outputs
    static constexpr int kBlocks = kColumns == 128 ? 3 : 512 / kColumns;              // an SM: three spill at 96 registers; of four, warps would have 80
    static constexpr int kHalves = kKeys / 64;                       // of the weights, announced one by one
};

template <int D, int SIDES>
__global__ void __launch_bounds__(ForwardShared<D, SIDES>::kThreads, ForwardShared<D, SIDES>::kBlocks) attend_kernel(const __grid_constant__ Forward w, unsigned int* mark) {
    using S = ForwardShared<D, SIDES>;
    constexpr int kRing = S::kRing, kKeys = S::kKeys, kCopying = 4 * SIDES, kIssuing = kCopying + 1;    // warps: SIDES groups of four, and one each
    extern __shared__ uint8_t raw[];
    const uint32_t base = (tc::smem_addr(raw) + 1023u) & ~1023u;
    uint8_t* mem = raw + (base - tc::smem_addr(raw));
    const uint32_t ring = base + SIDES * S::kBytes, bars = base + S::kBars;
    const uint32_t full = bars, empty = bars + 64, q_full = bars + 128, scores = bars + 144, weights = bars + 160, done = bars + 192,
                   q_empty = bars + 216, slot = bars + 240;
    const uint32_t turns = bars + 256;
    volatile uint32_t* slot_mem = reinterpret_cast<volatile uint32_t*>(mem + (slot - base));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kRing; ++i) {
            tc::bar_init(full + 8 * i, 1);
            tc::bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < SIDES; ++i) {
            tc::bar_init(q_full + 8 * i, 1);
            tc::bar_init(q_empty + 8 * i, 1);
            tc::bar_init(scores + 8 * i, 1);
            tc::bar_init(weights + 16 * i, 4);                       // the first half's and the second's
            tc::bar_init(weights + 16 * i + 8, 4);
            tc::bar_init(done + 8 * i, 1);
        }
        Pieces::init(turns, blockDim.x / 32);
        tc::bar_init_done();
        slot_mem[1] = 0;                   // set when a wait ran out
        tc::prefetch_map(&w.q);
        tc::prefetch_map(&w.k);
        tc::prefetch_map(&w.v);
    }
    if (warp == kIssuing) tc::tmem_alloc<1>(slot, S::kColumns);
    tc::fence_before();
    __syncthreads();
    tc::let_next_start();                  // now that this block has its tensor memory
    tc::fence_after();
    const uint32_t tmem = same(*slot_mem);
    bool fine = true;
    tc::wait_for_previous();

    Pieces pieces(w.plan, w.heads, turns);
    Piece piece{};
    int head = 0;
    // What a piece is made of: tiles of queries (sides) and each side's tiles of keys, taken from the last to the first
    int row0 = 0, n0 = 0, n1 = 0, most = 0;
    auto divide = [&] {
        row0 = piece.tile * SIDES * kTile;
        auto keys = [&](int row) { return (min(piece.length, w.causal ? row + kTile : piece.length) + kKeys - 1) / kKeys; };
        n0 = keys(row0);
        n1 = SIDES == 2 && piece.length - row0 > kTile ? keys(row0 + kTile) : 0;
        most = max(n0, n1);
    };

    if (warp == kCopying) {
        int filled = 0, queries = 0, others = 0, asked = 0;                    // tiles asked for: into the ring, of either side
        while (fine && pieces.take(piece, head, fine)) {
            divide();
            const int kv_head = w.group.quotient(head);
            for (int r = 0; r < most && fine; ++r) {
                if (r == most - 1) {
                    asked = pieces.turn;
                    if (!(fine = pieces.ask())) break;
                }
                const int row = piece.start + (most - 1 - r) * kKeys;
                for (int kind = 0; kind < 2; ++kind, ++filled) {
                    const int st = filled % kRing;
                    if (!(fine = tc::bar_wait(empty + 8 * st, ((filled / kRing) & 1) ^ 1))) break;
                    if (tc::elected()) {
                        tc::bar_expect(full + 8 * st, S::kKeyBytes);
                        load_head<D>(ring + st * S::kKeyBytes, kind ? &w.v : &w.k, kv_head, row, full + 8 * st);
                    }
                    __syncwarp();
                    if (r > 0 || kind > 0) continue;
                    for (int side = 0; side < (n1 > 0 ? 2 : 1); ++side) {             // behind the first keys
                        int& count = side ? others : queries;
                        if (!(fine = tc::bar_wait(q_empty + 8 * side, (count & 1) ^ 1))) break;
                        if (tc::elected()) {
                            tc::bar_expect(q_full + 8 * side, S::kBytes);
                            load_head<D>(base + side * S::kBytes, &w.q, head, piece.start + row0 + side * kTile, q_full + 8 * side);
                        }
                        __syncwarp();
                        ++count;
                    }
                    if (!fine) {
                        ++filled;
                        break;
                    }
                }
            }
        }
        if (!fine) {                       // what was asked for still lands in this block's memory: it is awaited
            pieces.settle(asked);
            if (queries > 0) tc::bar_wait(q_full, (queries - 1) & 1);
            if (others > 0) tc::bar_wait(q_full + 8, (others - 1) & 1);
            for (int i = max(0, filled - kRing); i < filled; ++i) tc::bar_wait(full + 8 * (i % kRing), (i / kRing) & 1);
        }
    } else if (warp == kIssuing) {
        const int k_steps = (w.dim + 15) / 16;
        const uint32_t out_inst = tc::instruction(kTile, k_steps * 16, 0, 1);
        auto finished = [&](uint32_t bar) {
            if (tc::elected()) tc::commit<1>(bar);
            __syncwarp();
        };
        auto filled = [&](int i) { return tc::bar_wait(full + 8 * (i % kRing), (i / kRing) & 1); };
        int round = 0;                     // of all pieces: its keys and values are the ring's 2 round and 2 round + 1
        int weighed[2] = {}, begun[2] = {};                          // tiles of each side; pieces
        // What is left of the last round: the weighted values
        bool waiting[2] = {}, first[2] = {};
        int steps = 0;
        bool last = false;
        auto gather = [&](int side) {
            const uint32_t values = ring + ((2 * round - 1) % kRing) * S::kKeyBytes, p_at = tmem + side * kKeys, o_at = tmem + SIDES * kKeys + side * D;
            if (!(fine = tc::bar_wait(weights + 16 * side, weighed[side] & 1))) return;
            tc::fence_after();
            weights_by_rows<0, 4, 0>(o_at, p_at, values, out_inst, steps, !first[side]);
            if (S::kHalves == 2) {
                if (!(fine = tc::bar_wait(weights + 16 * side + 8, weighed[side] & 1))) return;
                tc::fence_after();
                weights_by_rows<4, 8, 0>(o_at, p_at, values, out_inst, steps, true);
            }
            ++weighed[side];
            if (last) finished(done + 8 * side);
        };
        auto score = [&](int side, int r) {
            const int n = side ? n1 : n0;
            if (r == most - n && !(fine = tc::bar_wait(q_full + 8 * side, begun[side] & 1))) return;
            tc::fence_after();
            rows_by_rows<D, kKeys>(tmem + side * kKeys, base + side * S::kBytes, ring + (2 * round % kRing) * S::kKeyBytes, k_steps);
            finished(scores + 8 * side);
            if (r == most - 1) {
                ++begun[side];
                finished(q_empty + 8 * side);
            }
        };
        auto release = [&] {               // the last round's values
            if (round > 0) finished(empty + 8 * ((2 * round - 1) % kRing));
        };
        // A round: the weighted values of the round before it, then, over its weights, the scores of a tile of keys; one side after the
        // other, so that a side's products run while the other's exponentials do (with a warp to issue each side's, both sides' came to
        // run and to wait together: a quarter slower).
        while (fine && pieces.take(piece, head, fine)) {
            divide();
            for (int r = 0; r < most && fine; ++r, ++round) {
                if (round > 0 && !(fine = filled(2 * round - 1))) break;
                if (!(fine = filled(2 * round))) break;
#pragma unroll
                for (int side = 0; side < SIDES; ++side) {
                    if (fine && waiting[side]) gather(side);
                    if (fine && r >= most - (side ? n1 : n0)) score(side, r);
                }
                if (!fine) break;
                release();
                finished(empty + 8 * (2 * round % kRing));
                steps = (min(kKeys, piece.length - (most - 1 - r) * kKeys) + 15) / 16;
                last = r == most - 1;
#pragma unroll
                for (int side = 0; side < SIDES; ++side) {
                    const int n = side ? n1 : n0;
                    waiting[side] = r >= most - n;
                    first[side] = r == most - n;
                }
            }
        }
        if (fine && round > 0 && (fine = filled(2 * round - 1))) {
#pragma unroll
            for (int side = 0; side < SIDES; ++side) {
                if (fine && waiting[side]) gather(side);
            }
        }
    } else {
        const int side = warp / 4, quarter = warp % 4;
        const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t s_at = tmem + side * kKeys + lanes, o_at = tmem + SIDES * kKeys + side * D + lanes;
        const float c = w.c;
        int round = 0, scored = 0, ended = 0;                        // rounds of all pieces; this side's tiles; its pieces
        bool more = pieces.take(piece, head, fine);
        while (fine && more) {
            divide();
            const int n = side ? n1 : n0;
            const int row = row0 + side * kTile + quarter * 32 + lane;                // in the sequence
            float m = -INFINITY, mc = 0.0f;                          // the row's reference, and c times it
            float2 l = make_float2(0.0f, 0.0f);
            for (int r = 0; r < n; ++r, ++scored) {
                const int j = n - 1 - r;
                if (!(fine = tc::bar_wait(scores + 8 * side, scored & 1))) break;
                tc::fence_after();
                float s[kKeys];
                if constexpr (kKeys == 64) {
                    tmem_load64(s_at, s);
                } else {
                    tmem_load128(s_at, s);
                }
                const int valid = piece.length - j * kKeys;          // keys of the tile that are the sequence's
                if (valid < kKeys || (w.causal && (j + 1) * kKeys > row0 + side * kTile)) {
                    const int behind = (w.causal ? min(row, piece.length - 1) : piece.length - 1) - j * kKeys;
#pragma unroll
                    for (int i = 0; i < kKeys; ++i) s[i] = i <= behind ? s[i] : -INFINITY;
                }
                float top4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                for (int i = 4; i < kKeys; i += 8) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (i + 2 * e + 1 < kKeys) top4[e] = max3(top4[e], s[i + 2 * e], s[i + 2 * e + 1]);
                    }
                }
                const float top = max3(max3(top4[0], top4[1], top4[2]), top4[3], top4[3]);
                // The reference follows the maximum only where weights would exceed 2^8: bf16 and binary32 hold them as exactly, and
                // the output is seldom taken out and put back.  It is -infinity as long as all scores are.  A score of +infinity makes
                // c times it, and so all of the row's weights, NaN; one that is NaN (the maximum passes it over) its own weight, and so
                // the sum.
                const bool grows = m > -INFINITY ? !((top - m) * c <= 8.0f) : !(top == -INFINITY);
                if (__any_sync(0xffffffffu, grows)) {
                    const float to = grows ? top : m, to_c = to == -INFINITY ? 0.0f : (to - to) + to * c;
                    if (r > 0) {           // (the last scores came after the weighted values before them: the output is at rest)
                        const float f = grows ? (m == -INFINITY ? 0.0f : exp2_fast(mc - to_c)) : 1.0f;
                        l = mul2(l, make_float2(f, f));
#pragma unroll
                        for (int i = 0; i < D; i += 32) {
                            float o[32];
                            tc::tmem_load32(o_at + i, o);
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] *= f;
                            tmem_store_f32(o_at + i, o);
                        }
                    }
                    m = to;
                    mc = to_c;
                }
                if (valid < kKeys) {       // the values' rows behind the sequence
                    const int at = 2 * (round + most - 1 - j) + 1;
                    if (!(fine = tc::bar_wait(full + 8 * (at % kRing), (at / kRing) & 1))) break;
                    clear_rows<D>(mem + (ring - base) + (at % kRing) * S::kKeyBytes, valid, threadIdx.x % 128, 128);
                }
                const float2 cc = make_float2(c, c), minus = make_float2(-mc, -mc);
#pragma unroll
                for (int h = 0; h < S::kHalves; ++h) {
                    uint32_t p[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float2 e = fma2(make_float2(s[h * 64 + 2 * i], s[h * 64 + 2 * i + 1]), cc, minus);
                        e.x = exp2_fast(e.x);
                        e.y = exp2_fast(e.y);
                        l = add2(l, e);
                        p[i] = pack_bf16(e.x, e.y);
                    }
                    tmem_store32(s_at + 32 * h, p);
                    tmem_stored();
                    tc::fence_before();
                    __syncwarp();
                    if (lane == 0) tc::bar_arrive(weights + 16 * side + 8 * h);
                }
            }
            round += most;
            if (!fine) break;
            const int start = piece.start, mine = head, left = piece.length - row;
            more = pieces.take(piece, head, fine);                   // the next one's whereabouts, while the last values are being weighed
            if (!fine) break;
            if (n == 0) continue;
            if (!(fine = tc::bar_wait(done + 8 * side, ended & 1))) break;
            ++ended;
            tc::fence_after();
            const float sum = l.x + l.y;
            if (left > 0) w.lse[mine * w.lse_ld + start + row] = (mc + log2f(sum)) * kLn2;
            give_rows<D>(o_at, 1.0f / sum, mem + S::kStages + warp * kStage, w.out, start + row - lane, left + lane, mine, w.dim, lane);
            tc::fence_before();
        }
    }
    if (!fine) {
        slot_mem[1] = 1;
        *mark = 1;
    }
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    if (slot_mem[1] != 0) {                // matrix instructions may still be running: let them end
        const uint64_t t0 = tc::nanoseconds();
        while (tc::nanoseconds() - t0 < 50000000ull) {
        }
    }
    tc::fence_after();
    if (warp == kIssuing) tc::tmem_free<1>(tmem, S::kColumns);
}

dlion_status check(const dlion_attention_fwd* p) {
    if (p == nullptr || p->heads < 1 || p->kv_heads < 1 || p->heads > 65535 || p->heads % p->kv_heads != 0) return DLION_EINVAL;
    if (p->dim < 8 || p->dim > 128 || p->dim % 8 != 0 || p->causal < 0 || p->causal > 1 || !scale_ok(p->scale)) return DLION_EINVAL;
    const dlion_status seq = check_sequences(Sequences{p->rows, p->length, p->sequences, p->offsets, p->offsets_64});
    if (seq != DLION_OK) return seq;
    if (p->zero_rest < 0 || p->zero_rest > 1 || p->lse_ld < p->rows) return DLION_EINVAL;
    for (const Operand& a : {Operand{p->q, p->q_rs, p->q_hs, p->heads}, Operand{p->k, p->k_rs, p->k_hs, p->kv_heads},
                             Operand{p->v, p->v_rs, p->v_hs, p->kv_heads}, Operand{p->out, p->out_rs, p->out_hs, p->heads}}) {
        const dlion_status st = check_operand(a, p->rows, p->dim);
        if (st != DLION_OK) return st;
    }
    if (p->rows > 0 && p->lse == nullptr) return DLION_EINVAL;
    if (!aligned(p->lse, 4)) return DLION_EALIGN;
    return most_pieces(Sequences{p->rows, p->length, p->sequences, p->offsets, p->offsets_64}, kTile) * p->heads <= INT_MAX / 2 ? DLION_OK : DLION_EINVAL;
}

// Two tiles of queries to a block where heads are wide and sequences long on average (16384 rows, 8 heads of 128, one tile against two,
// us: causal 512 rows 47.7, 49.3, 1024 rows 69.9, 67.8; full 128 rows 32.9, 41.3, 256 rows 43.1, 41.9, 512 rows 59.8, 56.9).
int sides_of(const dlion_attention_fwd& p) {
    const int64_t count = p.offsets != nullptr ? p.sequences : p.length == 0 ? 1 : p.rows / p.length;
    return p.dim > 64 && p.rows >= count * (p.causal ? kLongCausal : kLongFull) ? 2 : 1;
}

template <int D, int SIDES>
void launch(prod::Call& c, Forward& w, int64_t pieces) {
    using S = ForwardShared<D, SIDES>;
    prod::raise_shared(c, &attend_kernel<D, SIDES>, S::kAll);
    prod::start(c, attend_kernel<D, SIDES>, dim3(static_cast<unsigned>(pieces * w.heads.d)), dim3(S::kThreads), S::kAll, 1, w, c.mark);
}

void forward(prod::Call& c, const dlion_attention_fwd& p) {
    const Sequences seq{p.rows, p.length, p.sequences, p.offsets, p.offsets_64};
    if (p.rows == 0) return;
    const int sides = sides_of(p);
    const int64_t pieces = most_pieces(seq, sides * kTile);
    int4* table = p.offsets != nullptr ? c.ws.take<int4>(pieces) : nullptr;
    if (!c.live()) return;
    Forward w{};
    Clear clear{};
    if (p.zero_rest) {
        clear.t[0] = Rows{static_cast<__nv_bfloat16*>(p.out), p.out_rs, p.out_hs};
        clear.heads[0] = clear.lse_heads = static_cast<int>(p.heads);
        clear.count = 1;
        clear.dim = static_cast<int>(p.dim);
        clear.lse = p.lse;
        clear.lse_ld = p.lse_ld;
    }
    const PlanRequest request{sides * kTile, p.causal, 0};
    make_plans(c, seq, &request, 1, &table, &w.plan, p.zero_rest ? &clear : nullptr);
    if (pieces == 0) return;
    const int passing = p.dim <= 64 ? kPassing<64> : kPassing<128>;
    if (!map_rows(&w.q, Operand{p.q, p.q_rs, p.q_hs, p.heads}, p.rows, p.dim, kTile) || !map_rows(&w.k, Operand{p.k, p.k_rs, p.k_hs, p.kv_heads}, p.rows, p.dim, passing) ||
        !map_rows(&w.v, Operand{p.v, p.v_rs, p.v_hs, p.kv_heads}, p.rows, p.dim, passing)) {
        c.status = DLION_ECUDA;
        return;
    }
    w.heads = divisor(p.heads);
    w.group = divisor(p.heads / p.kv_heads);
    w.dim = static_cast<int>(p.dim);
    w.causal = p.causal;
    w.c = p.scale * kLog2e;
    w.out = Rows{static_cast<__nv_bfloat16*>(p.out), p.out_rs, p.out_hs};
    w.lse = p.lse;
    w.lse_ld = p.lse_ld;
    if (p.dim <= 64) {
        launch<64, 1>(c, w, pieces);
    } else {
        sides == 1 ? launch<128, 1>(c, w, pieces) : launch<128, 2>(c, w, pieces);
    }
}

}  // namespace
}  // namespace att
}  // namespace dlion

extern "C" {

uint64_t dlion_attention_forward_workspace(const dlion_attention_fwd* p) {
    return dlion::att::check(p) == DLION_OK ? dlion::prod::workspace_of(*p, dlion::att::forward) : 0;
}

dlion_status dlion_attention_forward(const dlion_attention_fwd* p, void* workspace, uint64_t workspace_bytes, void* cuda_stream) {
    const dlion_status st = dlion::att::check(p);
    return st != DLION_OK ? st : dlion::prod::run(*p, dlion::att::forward, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
