// Attention over whole sequences (include/dlion_layers.h).
//
//   s_ij = scale q_i . k_j,  out_i = sum_j exp(s_ij - lse_i) v_j,  lse_i = log sum_j exp s_ij
//
// in one pass over the keys: with m the running maximum of a row, its sum l and its output o are held relative to exp(m) and
// rescaled when m grows.
#include "attention.cuh"

namespace dlion {
namespace att {

namespace {

struct Forward {
    CUtensorMap q, k, v;
    Plan plan;
    int heads, group, dim, causal;
    float c;                               // scale * log2(e)
    Rows out;
    float* lse;
    int64_t lse_ld;
};

constexpr int kForwardThreads = 320;       // two groups of four warps with a tile of queries each, a copying and an issuing warp
constexpr int kForwardRows = 2 * kTile;

template <int D>
struct ForwardShared {
    static constexpr uint32_t kBytes = kTile * D * 2;                // of a tile
    static constexpr int kRing = D == 128 ? 4 : 8;                   // tiles of keys and values, in turn
    static constexpr uint32_t kBars = (2 + kRing) * kBytes;
    static constexpr uint32_t kAll = kBars + 256 + 1024;
};

template <int D>
__global__ void __launch_bounds__(kForwardThreads, 1) attend_kernel(const __grid_constant__ Forward w, unsigned int* mark) {
    using S = ForwardShared<D>;
    constexpr int kRing = S::kRing;
    extern __shared__ uint8_t raw[];
    const uint32_t base = (tc::smem_addr(raw) + 1023u) & ~1023u;
    uint8_t* mem = raw + (base - tc::smem_addr(raw));
    const uint32_t ring = base + 2 * S::kBytes, bars = base + S::kBars;
    const uint32_t full = bars, empty = bars + 64, q_full = bars + 128, scores = bars + 144, weights = bars + 160, done = bars + 176, slot = bars + 192;
    volatile uint32_t* slot_mem = reinterpret_cast<volatile uint32_t*>(mem + (slot - base));
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

    tc::let_next_start();
    if (w.plan.table != nullptr) tc::wait_for_previous();            // the table is the kernel's before
    const int head = static_cast<int>(blockIdx.x) % w.heads;
    const Piece piece = piece_of(w.plan, static_cast<int>(blockIdx.x) / w.heads);
    if (piece.length < 0) return;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kRing; ++i) {
            tc::bar_init(full + 8 * i, 1);
            tc::bar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::bar_init(q_full + 8 * i, 1);
            tc::bar_init(scores + 8 * i, 1);
            tc::bar_init(weights + 8 * i, 4);
            tc::bar_init(done + 8 * i, 1);
        }
        tc::bar_init_done();
        slot_mem[1] = 0;                   // set when a wait ran out
        tc::prefetch_map(&w.q);
        tc::prefetch_map(&w.k);
        tc::prefetch_map(&w.v);
    }
    if (warp == 9) tc::tmem_alloc<1>(slot, 512);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = *slot_mem;
    const int row0 = piece.tile * kForwardRows;                      // in the sequence
    const int sides = piece.length - row0 > kTile ? 2 : 1;           // tiles of queries
    const int key_tiles = (piece.length + kTile - 1) / kTile;
    // tiles of keys of each side, taken from the last to the first
    const int n0 = w.causal ? min(key_tiles, 2 * piece.tile + 1) : key_tiles;
    const int n1 = sides == 2 ? (w.causal ? min(key_tiles, 2 * piece.tile + 2) : key_tiles) : 0;
    const int most = max(n0, n1);
    const int kv_head = head / w.group;
    bool fine = true;
    if (w.plan.table == nullptr) tc::wait_for_previous();

    if (warp == 8) {
        if (tc::elected()) {
            for (int i = 0; i < sides; ++i) {
                tc::bar_expect(q_full + 8 * i, S::kBytes);
                load_head<D>(base + i * S::kBytes, &w.q, head, piece.start + row0 + i * kTile, q_full + 8 * i);
            }
        }
        __syncwarp();
        int st = 0, filled = 0;
        uint32_t phase = 1;
        for (int j = most - 1; j >= 0 && fine; --j) {
            for (int kind = 0; kind < 2; ++kind, ++filled) {
                if (!(fine = tc::bar_wait(empty + 8 * st, phase))) break;
                if (tc::elected()) {
                    tc::bar_expect(full + 8 * st, S::kBytes);
                    load_head<D>(ring + st * S::kBytes, kind ? &w.v : &w.k, kv_head, piece.start + j * kTile, full + 8 * st);
                }
                __syncwarp();
                if (++st == kRing) {
                    st = 0;
                    phase ^= 1;
                }
            }
        }
        if (!fine) {                       // what was asked for still lands in this block's memory: it is awaited
            for (int i = 0; i < sides; ++i) tc::bar_wait(q_full + 8 * i, 0);
            for (int i = max(0, filled - kRing); i < filled; ++i) tc::bar_wait(full + 8 * (i % kRing), (i / kRing) & 1);
        }
    } else if (warp == 9) {
        const int k_steps = (w.dim + 15) / 16;
        const uint32_t score_inst = tc::instruction(kTile, kTile, 0, 0), out_inst = tc::instruction(kTile, k_steps * 16, 0, 1);
        auto finished = [&](uint32_t bar) {
            if (tc::elected()) tc::commit<1>(bar);
            __syncwarp();
        };
        auto filled = [&](int i) { return tc::bar_wait(full + 8 * (i % kRing), (i / kRing) & 1); };
        // round r: the weighted values of round r - 1 and the scores of round r, first for one side, then for the other, so that
        // one side's products run while the other's exponentials do
        for (int r = 0; r <= most && fine; ++r) {
            const int j = most - 1 - r;    // tile of keys of this round
            bool have_k = false, have_v = false;
            for (int side = 0; side < sides && fine; ++side) {
                const int n = side ? n1 : n0;
                if (r > 0 && j + 1 < n) {
                    const int before = 2 * (r - 1) + 1;              // the values' place in the ring's order
                    if (!have_v && !(fine = filled(before))) break;
                    have_v = true;
                    if (!(fine = tc::bar_wait(weights + 8 * side, (n - 2 - j) & 1))) break;
                    tc::fence_after();
                    if (tc::elected()) {
                        const uint64_t b = along_column(ring + (before % kRing) * S::kBytes);
                        const uint32_t a = tmem + side * kTile, d = tmem + 2 * kTile + side * D;
                        const int steps = (min(kTile, piece.length - (j + 1) * kTile) + 15) / 16;
                        for (int i = 0; i < steps; ++i) mma_tmem(d, a + 8 * i, b + column_step(i), out_inst, (i > 0 || j + 1 < n - 1) ? 1u : 0u);
                    }
                    __syncwarp();
                    if (j < 0) finished(done + 8 * side);
                }
                if (j >= 0 && j < n) {
                    if (!have_k && !(fine = filled(2 * r))) break;
                    have_k = true;
                    if (r == most - n && !(fine = tc::bar_wait(q_full + 8 * side, 0))) break;
                    tc::fence_after();
                    if (tc::elected()) {
                        const uint64_t a = along_row(base + side * S::kBytes), b = along_row(ring + (2 * r % kRing) * S::kBytes);
                        for (int i = 0; i < k_steps; ++i) tc::mma<1>(tmem + side * kTile, a + row_step(i), b + row_step(i), score_inst, i > 0 ? 1u : 0u);
                    }
                    __syncwarp();
                    finished(scores + 8 * side);
                }
            }
            if (!fine) break;
            if (r > 0) finished(empty + 8 * ((2 * r - 1) % kRing));
            if (j >= 0) finished(empty + 8 * (2 * r % kRing));
        }
    } else {
        const int side = warp / 4, quarter = warp % 4;
        const int n = side ? n1 : n0;
        const int row = row0 + side * kTile + quarter * 32 + lane;                    // in the sequence
        const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t s_at = tmem + side * kTile + lanes, o_at = tmem + 2 * kTile + side * D + lanes;
        const float c = w.c;
        float m = -INFINITY, mc = 0.0f;    // the row's reference, and c times it
        float2 l = make_float2(0.0f, 0.0f);
        for (int r = 0; r < n; ++r) {
            const int j = n - 1 - r;
            if (!(fine = tc::bar_wait(scores + 8 * side, r & 1))) break;
            tc::fence_after();
            float s[kTile];
            tmem_load64(s_at, *reinterpret_cast<float(*)[64]>(s));
            tmem_load64(s_at + 64, *reinterpret_cast<float(*)[64]>(s + 64));
            const int valid = piece.length - j * kTile;              // keys of the tile that are the sequence's
            if (valid < kTile || (w.causal && (j + 1) * kTile > row0 + side * kTile)) {
                const int last = (w.causal ? min(row, piece.length - 1) : piece.length - 1) - j * kTile;
#pragma unroll
                for (int i = 0; i < kTile; ++i) s[i] = i <= last ? s[i] : -INFINITY;
            }
            float top = max3(s[0], s[1], s[2]), top1 = s[3];
#pragma unroll
            for (int i = 4; i < kTile; i += 4) {
                top = max3(top, s[i], s[i + 1]);
                top1 = max3(top1, s[i + 2], s[i + 3]);
            }
            top = fmaxf(top, top1);
            // The reference follows the maximum only where weights would exceed 2^8: bf16 and binary32 hold them as exactly, and
            // the output is seldom taken out and put back.
            const bool grows = r == 0 ? top > -INFINITY : !(m > -INFINITY ? (top - m) * c <= 8.0f : top == -INFINITY);
            if (__any_sync(0xffffffffu, grows)) {
                const float to = grows ? top : m, to_c = to > -INFINITY ? to * c : 0.0f;
                if (r > 0) {
                    const float f = grows ? (m > -INFINITY ? exp2_fast(mc - to_c) : 0.0f) : 1.0f;
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
            const float2 cc = make_float2(c, c), minus = make_float2(-mc, -mc);
#pragma unroll
            for (int h = 0; h < kTile; h += 64) {
                uint32_t p[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    float2 e = fma2(make_float2(s[h + 2 * i], s[h + 2 * i + 1]), cc, minus);
                    e.x = exp2_fast(e.x);
                    e.y = exp2_fast(e.y);
                    l = add2(l, e);
                    p[i] = pack_bf16(e.x, e.y);
                }
                tmem_store32(s_at + h / 2, p);
            }
            if (valid < kTile) {           // the values' rows behind the sequence
                const int at = 2 * (most - 1 - j) + 1;
                if (!(fine = tc::bar_wait(full + 8 * (at % kRing), (at / kRing) & 1))) break;
                clear_rows<D>(mem + (ring - base) + (at % kRing) * S::kBytes, valid, threadIdx.x % 128, 128);
            }
            tmem_stored();
            tc::fence_before();
            __syncwarp();
            if (lane == 0) tc::bar_arrive(weights + 8 * side);
        }
        if (n > 0 && fine) fine = tc::bar_wait(done + 8 * side, 0);
        if (n > 0 && fine) {
            tc::fence_after();
            const float sum = l.x + l.y;
            const int rows = piece.length - row0 - side * kTile - quarter * 32;
            if (lane < rows) w.lse[head * w.lse_ld + piece.start + row] = (mc + log2f(sum)) * kLn2;
            const float inverse = 1.0f / sum;
            // 64 columns at a time, through this side's queries, which have been read
            uint8_t* stage = mem + side * S::kBytes + quarter * (32 * D * 2);
            give_rows<D>(o_at, inverse, stage, w.out, piece.start + row - lane, rows, head, 0, w.dim, lane);
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
    if (warp == 9) tc::tmem_free<1>(tmem, 512);
}

dlion_status check(const dlion_attention_fwd* p) {
    if (p == nullptr || p->heads < 1 || p->kv_heads < 1 || p->heads > 65535 || p->heads % p->kv_heads != 0) return DLION_EINVAL;
    if (p->dim < 8 || p->dim > 128 || p->dim % 8 != 0 || p->causal < 0 || p->causal > 1 || !(p->scale > 0.0f) || !(p->scale < INFINITY)) return DLION_EINVAL;
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
    return most_pieces(Sequences{p->rows, p->length, p->sequences, p->offsets, p->offsets_64}, kForwardRows) * p->heads <= INT_MAX ? DLION_OK : DLION_EINVAL;
}

void forward(prod::Call& c, const dlion_attention_fwd& p) {
    const Sequences seq{p.rows, p.length, p.sequences, p.offsets, p.offsets_64};
    const int64_t pieces = most_pieces(seq, kForwardRows);
    if (p.rows == 0) return;
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
    const PlanRequest request{kForwardRows, p.causal, 0};
    make_plans(c, seq, &request, 1, &table, &w.plan, p.zero_rest ? &clear : nullptr);
    if (pieces == 0) return;
    if (!map_rows(&w.q, Operand{p.q, p.q_rs, p.q_hs, p.heads}, p.rows, p.dim) || !map_rows(&w.k, Operand{p.k, p.k_rs, p.k_hs, p.kv_heads}, p.rows, p.dim) ||
        !map_rows(&w.v, Operand{p.v, p.v_rs, p.v_hs, p.kv_heads}, p.rows, p.dim)) {
        c.status = DLION_ECUDA;
        return;
    }
    w.heads = static_cast<int>(p.heads);
    w.group = static_cast<int>(p.heads / p.kv_heads);
    w.dim = static_cast<int>(p.dim);
    w.causal = p.causal;
    w.c = p.scale * kLog2e;
    w.out = Rows{static_cast<__nv_bfloat16*>(p.out), p.out_rs, p.out_hs};
    w.lse = p.lse;
    w.lse_ld = p.lse_ld;
    const dim3 grid(static_cast<unsigned>(pieces * p.heads)), block(kForwardThreads);
    if (p.dim <= 64) {
        prod::raise_shared(c, &attend_kernel<64>, ForwardShared<64>::kAll);
        prod::start(c, attend_kernel<64>, grid, block, ForwardShared<64>::kAll, 1, w, c.mark);
    } else {
        prod::raise_shared(c, &attend_kernel<128>, ForwardShared<128>::kAll);
        prod::start(c, attend_kernel<128>, grid, block, ForwardShared<128>::kAll, 1, w, c.mark);
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
