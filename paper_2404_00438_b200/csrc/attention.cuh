// What the attention kernels share: the sequences' tiles, copies of rows of one head, products with an
// operand in tensor memory, and the arithmetic on pairs of binary32 values.
#pragma once

#include <climits>

#include "layers_math.cuh"
#include "product_host.h"
#include "tensor_core.cuh"

namespace dlion {
namespace att {

constexpr int kTile = 128;                 // rows of the tile that a block keeps: the lanes of tensor memory

// Rows of the tiles of keys that pass by it.  With heads of up to 64 columns these are short: then two blocks of dq's kernel fit an SM,
// three of the forward one, whose warps wait at different times.  12 heads of 64, tiles of 128 against 64, us: 64 x 197 rows forward 39, 33,
// backward 167, 130; 8 x 1024 both directions 152, 150; only very long sequences lose (16384, 16 heads, backward 2326, 2444).
template <int D>
constexpr int kPassing = D == 64 ? 64 : 128;

// Which sequence and which of its tiles a piece of work is.  Sequences of one length are numbered by arithmetic; others by a
// table in the workspace (plan_kernel), which ends with entries of length -1.  The longest pieces come first, because
// a block's work grows with the tile's place under a causal mask, and the last blocks should be short.
struct Divisor {                           // of numbers below 2^31, by a product: a division takes 100 clocks and more
    uint32_t d, m, shift;
    __device__ __forceinline__ int quotient(int n) const { return static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(n)) * m) >> shift); }
};

inline Divisor divisor(int64_t d) {        // m = floor(2^(31 + l) / d) + 1 with 2^l >= d: exact below 2^31
    int l = 0;
    while ((int64_t{1} << l) < d) ++l;
    return Divisor{static_cast<uint32_t>(d), static_cast<uint32_t>((uint64_t{1} << (31 + l)) / static_cast<uint64_t>(d) + 1), static_cast<uint32_t>(31 + l)};
}

struct Plan {
    const int4* table;                     // {first row, length, tile, 0}
    int length, tiles;                     // without a table
    Divisor sequences;
    int descending;
};

struct Piece {
    int start, length, tile;
};

__device__ __forceinline__ Piece piece_of(const Plan& p, int i) {
    if (p.table != nullptr) {
        const int4 e = p.table[i];
        return Piece{e.x, e.y, e.z};
    }
    const int rank = p.sequences.quotient(i);
    return Piece{(i - rank * static_cast<int>(p.sequences.d)) * p.length, p.length, p.descending ? p.tiles - 1 - rank : rank};
}

// A value that all lanes of a converged warp have, as one that the compiler knows to be the same in all (and may keep in a uniform
// register): what comes out of memory is otherwise one value a lane, and the operands of a matrix instruction are then brought
// over one by one before each.
__device__ __forceinline__ int same(int v) { return static_cast<int>(__reduce_or_sync(0xffffffffu, static_cast<unsigned>(v))); }

// A block's pieces of work, each a tile of a sequence and a head.  The kernels are persistent: a block takes over the work of blocks
// that have not started (the grid has one for each piece), so that while a tile's last rows are weighed and its results leave, the
// next one's first products run, and whoever is free takes the next piece.  (64 images of 197 rows forward: 47 us with a block for
// each tile, 41 so.  With every so many-th piece for each block, 8192 rows of 11 documents: 12 % slower backward.)  The copying warp asks
// for the next piece when it comes to a piece's last tile (at its first, everyone would take two of the longest pieces), in two places of
// shared memory in turn; every warp of the block reads the answer.
constexpr uint32_t kTurnBytes = 64;        // two barriers for answers, two for their readers, the answers

struct Pieces {
    const Plan* plan;
    Divisor heads;
    uint32_t at;                           // shared memory
    int turn;                              // pieces taken

    __device__ __forceinline__ Pieces(const Plan& p, const Divisor& heads_, uint32_t at_) : plan(&p), heads(heads_), at(at_), turn(0) {}

    __device__ static void init(uint32_t at, int warps) {
        for (int i = 0; i < 2; ++i) {
            tc::bar_init(at + 8 * i, 1);
            tc::bar_init(at + 16 + 8 * i, warps);
        }
    }
    __device__ __forceinline__ uint32_t parity(int k) const { return ((k - 1) >> 1) & 1; }

    // False when there are no more (or a wait ran out, and `fine` says so).
    __device__ __forceinline__ bool take(Piece& piece, int& head, bool& fine) {
        int unit = static_cast<int>(blockIdx.x);
        if (turn > 0) {
            const uint32_t place = turn & 1;
            if (!(fine = tc::bar_wait(at + 8 * place, parity(turn)))) return false;
            uint32_t got, first;
            asm volatile(
                "{\n.reg .pred p;\n.reg .b128 r;\nld.shared.b128 r, [%2];\n"
                "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\nselp.u32 %0, 1, 0, p;\nmov.u32 %1, 0;\n"
                "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n}"
                : "=r"(got), "=r"(first)
                : "r"(at + 32 + 16 * place)
                : "memory");
            tc::fence_for_copies();        // read, before the next answer comes to this place
            __syncwarp();
            if (threadIdx.x % 32 == 0) tc::bar_arrive(at + 16 + 8 * place);
            if (same(got) == 0) return false;
            unit = same(first);
        }
        ++turn;
        const int i = heads.quotient(unit);
        const Piece found = piece_of(*plan, i);
        piece = Piece{same(found.start), same(found.length), same(found.tile)};
        head = unit - i * static_cast<int>(heads.d);
        return piece.length >= 0;
    }

    // By the copying warp, in a piece that it has taken: the next one.
    __device__ __forceinline__ bool ask() const {
        const uint32_t place = turn & 1;
        if (!tc::bar_wait(at + 16 + 8 * place, parity(turn) ^ 1)) return false;
        if (tc::elected()) {
            tc::bar_expect(at + 8 * place, 16);
            asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(at + 32 + 16 * place),
                         "r"(at + 8 * place)
                         : "memory");
        }
        __syncwarp();
        return true;
    }
    // An answer that may still be on its way, where a wait ran out.
    __device__ __forceinline__ void settle(int asked) const {
        if (asked >= turn && asked > 0) tc::bar_wait(at + 8 * (asked & 1), parity(asked));
    }
};

// bf16 [rows][heads][dim], strides in elements
struct Rows {
    __nv_bfloat16* p;
    int64_t rs, hs;
};

// ---------------------------------------------------------------- copies
// 64 columns of some rows of one head, 128-byte swizzled; x is 0 or 64.
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* map, int x, int head, int row, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(head), "r"(row), "r"(bar)
        : "memory");
}

constexpr uint32_t kChunk = kTile * 128;   // bytes of 64 columns

template <int D>
__device__ __forceinline__ void load_head(uint32_t dst, const CUtensorMap* map, int head, int row, uint32_t bar) {
#pragma unroll
    for (int c = 0; c < D / 64; ++c) load_rows(dst + c * kChunk, map, 64 * c, head, row, bar);
}

// Rows of a tile from `first` on become zero, up to the end of the sixteen that a matrix instruction takes (by `threads` threads):
// they are other sequences' rows, or no one's, and what they hold, NaN too, must not meet the zeros of a masked product.  The
// caller announces it to the matrix instructions by a barrier.
template <int D>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int first, int thread, int threads) {
    for (int i = first * 8 + thread; i < ((first + 15) & ~15) * 8; i += threads) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c) *reinterpret_cast<uint4*>(tile + c * kChunk + i * 16) = make_uint4(0, 0, 0, 0);
    }
    tc::fence_for_copies();
}

// ---------------------------------------------------------------- products
// Operand whose k runs along a row of the tile (a head's columns): chunks of 64 columns, 32 bytes for 16 of k.
__device__ __forceinline__ uint64_t along_row(uint32_t tile) { return tc::operand_base(0) | ((tile >> 4) & 0x3fff); }
__device__ __forceinline__ uint32_t row_step(int k16) { return ((k16 >> 2) * kChunk + (k16 & 3) * 32) >> 4; }

// Operand whose k is the tile's rows, its other axis the head's columns: 64 of them to a chunk, 2048 bytes for 16 of k.
__device__ __forceinline__ uint64_t along_column(uint32_t tile) {
    return (static_cast<uint64_t>(kChunk >> 4) << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61) |
           ((tile >> 4) & 0x3fff);
}
__device__ __forceinline__ uint32_t column_step(int k16) { return (k16 * 2048) >> 4; }

// The first operand out of tensor memory: 16 of k are 8 columns of bf16 pairs.
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t inst, uint32_t add) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b), "r"(inst), "r"(add)
        : "memory");
}

// The matrix instructions of one product, by a converged warp: what describes the operands is worked out by the whole warp, so
// that it stays in uniform registers, where these instructions want it, and the instructions of a full product stand one behind
// the other.  (Inside a branch that one lane has taken, with a loop, an instruction took 150 clocks to issue, and its product 64.)
//
// d = kTile rows of a times N rows of b, both along a head's columns, 16 * steps of them (the rest of D is not there).
template <int D, int N>
__device__ __forceinline__ void rows_by_rows(uint32_t d, uint32_t a_tile, uint32_t b_tile, int steps) {
    static_assert(D == 64 || N == kTile, "a tile's chunks of 64 columns are kChunk apart");
    const uint64_t a = along_row(a_tile), b = along_row(b_tile);
    const uint32_t inst = tc::instruction(kTile, N, 0, 0);
    if (tc::elected()) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            if (i < steps) tc::mma<1>(d, a + row_step(i), b + row_step(i), inst, i > 0 ? 1u : 0u);
        }
    }
    __syncwarp();
}

// d (+)= the 16-value steps [FROM, TO) of a, in tensor memory 8 columns a step (GAP more between the halves), times the tile's
// rows; `steps` of all eight are there.
template <int FROM, int TO, int GAP>
__device__ __forceinline__ void weights_by_rows(uint32_t d, uint32_t a, uint32_t b_tile, uint32_t inst, int steps, bool add) {
    const uint64_t b = along_column(b_tile);
    const uint32_t onto = add ? 1u : 0u;
    if (tc::elected()) {
#pragma unroll
        for (int i = FROM; i < TO; ++i) {
            if (i < steps) mma_tmem(d, a + 8 * i + (i >= 4 ? GAP : 0), b + column_step(i), inst, i > 0 ? 1u : onto);
        }
    }
    __syncwarp();
}

// ---------------------------------------------------------------- tensor memory
// 64 consecutive columns of this warp's 32 lanes, a row a thread.
__device__ __forceinline__ void tmem_load64(uint32_t addr, float (&v)[64]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, "
        "%8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, "
        "%40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, "
        "%56, %57, %58, %59, %60, %61, %62, %63"
        "}, [%64];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(addr)
        : "memory");
}

// 128 columns: both halves asked for before the first is waited for.
__device__ __forceinline__ void tmem_load128(uint32_t addr, float (&v)[128]) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%0, %1, %2, %3, %4, %5, %6, %7, "
        "%8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, "
        "%40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, "
        "%56, %57, %58, %59, %60, %61, %62, %63"
        "}, [%128];\n"
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%64, %65, %66, %67, %68, %69, %70, %71, "
        "%72, %73, %74, %75, %76, %77, %78, %79, "
        "%80, %81, %82, %83, %84, %85, %86, %87, "
        "%88, %89, %90, %91, %92, %93, %94, %95, "
        "%96, %97, %98, %99, %100, %101, %102, %103, "
        "%104, %105, %106, %107, %108, %109, %110, %111, "
        "%112, %113, %114, %115, %116, %117, %118, %119, "
        "%120, %121, %122, %123, %124, %125, %126, %127"
        "}, [%129];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63]),
          "=r"(r[64]), "=r"(r[65]), "=r"(r[66]), "=r"(r[67]), "=r"(r[68]), "=r"(r[69]), "=r"(r[70]), "=r"(r[71]),
          "=r"(r[72]), "=r"(r[73]), "=r"(r[74]), "=r"(r[75]), "=r"(r[76]), "=r"(r[77]), "=r"(r[78]), "=r"(r[79]),
          "=r"(r[80]), "=r"(r[81]), "=r"(r[82]), "=r"(r[83]), "=r"(r[84]), "=r"(r[85]), "=r"(r[86]), "=r"(r[87]),
          "=r"(r[88]), "=r"(r[89]), "=r"(r[90]), "=r"(r[91]), "=r"(r[92]), "=r"(r[93]), "=r"(r[94]), "=r"(r[95]),
          "=r"(r[96]), "=r"(r[97]), "=r"(r[98]), "=r"(r[99]), "=r"(r[100]), "=r"(r[101]), "=r"(r[102]), "=r"(r[103]),
          "=r"(r[104]), "=r"(r[105]), "=r"(r[106]), "=r"(r[107]), "=r"(r[108]), "=r"(r[109]), "=r"(r[110]), "=r"(r[111]),
          "=r"(r[112]), "=r"(r[113]), "=r"(r[114]), "=r"(r[115]), "=r"(r[116]), "=r"(r[117]), "=r"(r[118]), "=r"(r[119]),
          "=r"(r[120]), "=r"(r[121]), "=r"(r[122]), "=r"(r[123]), "=r"(r[124]), "=r"(r[125]), "=r"(r[126]), "=r"(r[127])
        : "r"(addr), "r"(addr + 64)
        : "memory");
}

// 32 columns of this warp's 32 lanes; there after tmem_stored().
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {"
        "%0, %1, %2, %3, %4, %5, %6, %7, "
        "%8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31"
        "};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
          "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
          "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
          "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]),
          "r"(addr)
        : "memory");
}

// One column, a value a thread.
__device__ __forceinline__ void tmem_store1(uint32_t addr, float v) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(addr), "r"(__float_as_uint(v)) : "memory");
}
__device__ __forceinline__ float tmem_load1(uint32_t addr) {
    uint32_t v;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\ntcgen05.wait::ld.sync.aligned;" : "=r"(v) : "r"(addr) : "memory");
    return __uint_as_float(v);
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_store_f32(uint32_t addr, const float (&v)[32]) {
    tmem_store32(addr, reinterpret_cast<const uint32_t(&)[32]>(v));
}

// a NaN is passed over
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// ---------------------------------------------------------------- results
// COLS columns of a row a thread (binary32, in tensor memory at `addr`), times `factor`, as bf16 rows of a head: through
// shared memory (`stage`, kStage bytes, this warp's own), 32 columns at a time, so that 64 bytes of a row leave together (each thread
// its own row, 16 bytes at a time: 5 % slower where sequences are short).  row0: the warp's first row, of which `rows` are there
// (may be negative).
constexpr uint32_t kStage = 2048;

template <int COLS>
__device__ __forceinline__ void give_rows(uint32_t addr, float factor, uint8_t* stage, const Rows& to, int64_t row0, int rows, int head, int dim, int lane) {
    const int unit = lane % 4;
    __nv_bfloat16* out = to.p + row0 * to.rs + head * to.hs + unit * 8;
    float v[COLS];
    if constexpr (COLS == 128) {
        tmem_load128(addr, v);
    } else {
        tmem_load64(addr, v);
    }
#pragma unroll
    for (int c = 0; c < COLS; c += 32) {
        __syncwarp();                      // what was there has left
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float* x = v + c + 8 * i;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= factor;
            const uint4 w = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
            *reinterpret_cast<uint4*>(stage + lane * 64 + ((i ^ (lane / 2 % 4)) * 16)) = w;
        }
        __syncwarp();
        const bool inside = c + unit * 8 < dim;
        __nv_bfloat16* at = out + (lane / 4) * to.rs + c;
        uint4 got[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) got[r] = *reinterpret_cast<const uint4*>(stage + (lane / 4 + 8 * r) * 64 + ((unit ^ ((lane / 4 + 8 * r) / 2 % 4)) * 16));
#pragma unroll
        for (int r = 0; r < 4; ++r, at += 8 * to.rs) {
            if (inside && lane / 4 + 8 * r < rows) *reinterpret_cast<uint4*>(at) = got[r];
        }
    }
    __syncwarp();
}

// The same to the row at `out` where it is there (`live`), without a place to put rows together: each thread stores its own row, 16
// bytes at a time, and the halves of sectors meet in L2.
template <int COLS>
__device__ __forceinline__ void give_row(uint32_t addr, float factor, __nv_bfloat16* out, bool live, int dim) {
#pragma unroll
    for (int c = 0; c < COLS; c += 32) {
        float v[32];
        tc::tmem_load32(addr + c, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 w = make_uint4(pack_bf16(v[8 * i] * factor, v[8 * i + 1] * factor), pack_bf16(v[8 * i + 2] * factor, v[8 * i + 3] * factor),
                                       pack_bf16(v[8 * i + 4] * factor, v[8 * i + 5] * factor), pack_bf16(v[8 * i + 6] * factor, v[8 * i + 7] * factor));
            if (live && c + 8 * i < dim) *reinterpret_cast<uint4*>(out + c + 8 * i) = w;
        }
    }
}

// ---------------------------------------------------------------- host side (attention_plan.cu)
constexpr int64_t kMostRows = int64_t{1} << 30;

inline bool scale_ok(float scale) { return scale > 0.0f && scale <= 2e38f; }          // log2(e) times it is finite

struct Operand {                           // bf16 [rows][heads][dim] as an argument
    const void* p;
    int64_t rs, hs, heads;
};

// DLION_OK if 16-byte accesses and tiled copies can take it.
dlion_status check_operand(const Operand& a, int64_t rows, int64_t dim);
bool map_rows(CUtensorMap* map, const Operand& a, int64_t rows, int64_t dim, int tile);

struct Sequences {
    int64_t rows, length, count;
    const void* offsets;
    int offsets64;
};
dlion_status check_sequences(const Sequences& s);

// Pieces of `tile` rows that the sequences have at most, and the plan for them; with offsets, tables are filled by one launch
// for all plans (make_plans), which also clears what belongs to no sequence.
struct PlanRequest {
    int tile, causal, keys;                // keys: pieces are tiles of keys, of which the first have most queries
};
int64_t most_pieces(const Sequences& s, int tile);

struct Clear {                             // rows in no sequence
    Rows t[3];
    int heads[3];
    int count, dim;
    float* lse;
    int64_t lse_ld;
    int lse_heads;
};
// tables: n device arrays of most_pieces() entries, from the workspace (nullptr without offsets)
void make_plans(prod::Call& c, const Sequences& s, const PlanRequest* requests, int n, int4* const* tables, Plan* plans, const Clear* clear);

}  // namespace att
}  // namespace dlion
