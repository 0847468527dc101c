// Host side of the attention kernels and the table of pieces of sequences of different lengths.
#include "attention.cuh"

namespace dlion {
namespace att {

namespace {

constexpr int kBuckets = 1024;
constexpr int kClearBlocks = 64;

struct PlanArgs {
    const void* offsets;
    int offsets64, count, rows;
    int4* table[2];
    int most[2];
    PlanRequest request[2];
    int tables;
    Clear clear;
};

__device__ __forceinline__ int offset_at(const PlanArgs& a, int i) {
    const int64_t v = a.offsets64 ? static_cast<const int64_t*>(a.offsets)[i] : static_cast<const int32_t*>(a.offsets)[i];
    return static_cast<int>(v < 0 ? 0 : v > a.rows ? a.rows : v);
}

// How many tiles of the other side a piece meets.
__device__ __forceinline__ int work_of(const PlanRequest& r, int length, int tile) {
    const int last = min((tile + 1) * r.tile, length);                                // one behind the piece's last row
    if (!r.causal) return (length + kTile - 1) / kTile;
    return r.keys ? (length - tile * r.tile + kTile - 1) / kTile : (last + kTile - 1) / kTile;
}

// One block a table: pieces are counted by their work, the counts summed from the longest on, and the pieces put in their
// places; which of two equal pieces comes first is left to chance and changes no result.  Offsets are held to the rows there
// are; if they ascend, the pieces are no more than the table's entries.  Offsets that do not ascend are found while counting (some
// length is negative; a warp that has met more pieces than there can be stops, so that their number bounds the time), and
// then there are no pieces: the counts, which may have passed 32 bits, are not used.
// A few us where there are some hundred sequences; the launch is most of it.
__global__ void __launch_bounds__(1024) plan_kernel(const __grid_constant__ PlanArgs a) {
    __shared__ int place[kBuckets];
    __shared__ int sums[32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    tc::let_next_start();
    tc::wait_for_previous();
    if (static_cast<int>(blockIdx.x) >= a.tables) {            // rows in no sequence: before the first and behind the last
        const Clear& c = a.clear;
        const int first = offset_at(a, 0), last = max(first, offset_at(a, a.count));
        const int64_t rest = first + (a.rows - last), step = static_cast<int64_t>(gridDim.x - a.tables) * 1024;
        const int64_t at = static_cast<int64_t>(blockIdx.x - a.tables) * 1024 + threadIdx.x;
        const int units = c.dim / 8;
        for (int t = 0; t < c.count; ++t) {
            const int64_t per = static_cast<int64_t>(c.heads[t]) * units;
            for (int64_t i = at; i < rest * per; i += step) {
                const int64_t r = i / per, row = r < first ? r : r - first + last;
                const int in = static_cast<int>(i - r * per);
                *reinterpret_cast<uint4*>(c.t[t].p + row * c.t[t].rs + (in / units) * c.t[t].hs + (in % units) * 8) = make_uint4(0, 0, 0, 0);
            }
        }
        for (int64_t i = at; c.lse != nullptr && i < rest * c.lse_heads; i += step) {
            const int64_t h = i / rest, r = i - h * rest;
            c.lse[h * c.lse_ld + (r < first ? r : r - first + last)] = 0.0f;
        }
        return;
    }
    const PlanRequest& request = a.request[blockIdx.x];
    int4* table = a.table[blockIdx.x];
    const int most = a.most[blockIdx.x];
    place[threadIdx.x] = 0;
    __syncthreads();
    // twice over the sequences, a warp for each: counting, then placing; false where the offsets are seen not to ascend
    auto pieces = [&](auto f) {
        int met = 0;                       // by this warp: most + 2^23 at most, below 2^31
        for (int s = warp; s < a.count; s += 32) {
            const int start = offset_at(a, s), length = offset_at(a, s + 1) - start;
            const int tiles = length <= 0 ? 0 : (length + request.tile - 1) / request.tile;
            met += tiles;
            if (length < 0 || met > most) return false;
            for (int t = lane; t < tiles; t += 32) f(start, length, t, kBuckets - 1 - min(work_of(request, length, t), kBuckets - 1));
        }
        return true;
    };
    const bool counted = pieces([&](int, int, int, int bucket) { atomicAdd(&place[bucket], 1); });
    const bool ascend = __syncthreads_and(counted) != 0;
    const int mine = place[threadIdx.x];
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    if (warp == 0) {
        int v = sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int o = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v += o;
        }
        sums[lane] = v;
    }
    __syncthreads();
    place[threadIdx.x] = upto - mine + (warp > 0 ? sums[warp - 1] : 0);
    const int total = ascend ? sums[31] : 0;
    __syncthreads();
    if (ascend) {
        pieces([&](int start, int length, int tile, int bucket) {
            const int at = atomicAdd(&place[bucket], 1);
            if (at < most) table[at] = make_int4(start, length, tile, 0);
        });
    }
    for (int i = total + threadIdx.x; i < most; i += 1024) table[i] = make_int4(0, -1, 0, 0);
}

bool stride_ok(int64_t s, int64_t dim, bool used) { return !used || (s >= dim && s % 8 == 0 && s < (int64_t{1} << 38)); }

}  // namespace

dlion_status check_operand(const Operand& a, int64_t rows, int64_t dim) {
    if (!stride_ok(a.rs, dim, rows > 1) || !stride_ok(a.hs, dim, a.heads > 1)) return DLION_EINVAL;
    if (rows > 0 && a.p == nullptr) return DLION_EINVAL;
    return aligned16(a.p) ? DLION_OK : DLION_EALIGN;
}

bool map_rows(CUtensorMap* map, const Operand& a, int64_t rows, int64_t dim, int tile) {
    const uint64_t sizes[3] = {static_cast<uint64_t>(dim), static_cast<uint64_t>(a.heads), static_cast<uint64_t>(rows)};
    const uint64_t strides[2] = {static_cast<uint64_t>(a.heads > 1 ? a.hs : dim) * 2, static_cast<uint64_t>(rows > 1 ? a.rs : dim) * 2};
    const uint32_t box[3] = {64, 1, static_cast<uint32_t>(tile)};
    return prod::encode_map(map, a.p, 3, sizes, strides, box);
}

dlion_status check_sequences(const Sequences& s) {
    if (s.rows < 0 || s.rows > kMostRows || s.length < 0 || s.count < 0 || s.count > kMostRows) return DLION_EINVAL;
    if (s.offsets != nullptr) return s.length != 0 || s.offsets64 < 0 || s.offsets64 > 1 ? DLION_EINVAL : aligned(s.offsets, s.offsets64 ? 8 : 4) ? DLION_OK : DLION_EALIGN;
    if (s.count != 0) return DLION_EINVAL;
    return s.length == 0 || s.rows % s.length == 0 ? DLION_OK : DLION_EINVAL;
}

int64_t most_pieces(const Sequences& s, int tile) {
    if (s.offsets != nullptr) return s.rows / tile + std::min(s.count, s.rows);
    const int64_t length = s.length == 0 ? s.rows : s.length;
    return s.rows == 0 ? 0 : s.rows / length * prod::parts(length, tile);
}

void make_plans(prod::Call& c, const Sequences& s, const PlanRequest* requests, int n, int4* const* tables, Plan* plans, const Clear* clear) {
    for (int i = 0; i < n; ++i) {
        const int64_t length = s.length == 0 ? s.rows : s.length;
        const int64_t count = s.offsets != nullptr || length == 0 ? 1 : s.rows / length;
        plans[i] = Plan{tables[i], static_cast<int>(length), static_cast<int>(prod::parts(length, requests[i].tile)), divisor(count), !requests[i].keys};
    }
    if (s.offsets == nullptr || !c.live()) return;
    PlanArgs a{};
    a.offsets = s.offsets;
    a.offsets64 = s.offsets64;
    a.count = static_cast<int>(s.count);
    a.rows = static_cast<int>(s.rows);
    a.tables = n;
    for (int i = 0; i < n; ++i) {
        a.table[i] = tables[i];
        a.most[i] = static_cast<int>(most_pieces(s, requests[i].tile));
        a.request[i] = requests[i];
    }
    if (clear != nullptr) a.clear = *clear;
    prod::start(c, plan_kernel, dim3(static_cast<unsigned>(n + (clear != nullptr ? kClearBlocks : 0))), dim3(1024), 0, 1, a);
}

}  // namespace att
}  // namespace dlion
