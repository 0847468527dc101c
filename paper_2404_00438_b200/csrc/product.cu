// Launches of the layer products, the sum of split products, and the packing of operands that tiled
// copies cannot read in place.
#include "product_host.h"

#include <algorithm>

namespace dlion {
namespace prod {

__device__ unsigned int wait_ran_out = 0;

namespace {

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder() {
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess) {
            p = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// Rows of `cols` adjacent values, off the 16-byte grid, to rows on it.  A thread puts eight values together from the two
// 16-byte units that hold them (the second one comes from L1), all of a row shifted alike; units that reach beyond the row are
// read value by value.  Bound by memory: 4 bytes a value (8192 x 8191: 150 us with 2-byte accesses).  The grid's second axis has
// 65535 blocks at most, so longer rows (a column-major operand of more than 67 million rows) take several turns.
constexpr int kPackCols = 1024;

__device__ __forceinline__ uint4 unit_of_row(const uint8_t* unit, const uint8_t* from, const uint8_t* to) {
    if (unit >= from && unit + 16 <= to) return *reinterpret_cast<const uint4*>(unit);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint8_t* p = unit + 2 * i;
        if (p >= from && p < to) w[i / 2] |= static_cast<uint32_t>(*reinterpret_cast<const unsigned short*>(p)) << (16 * (i % 2));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__global__ void __launch_bounds__(256) pack_rows_kernel(const uint16_t* a, int64_t rs, int64_t rows, int64_t cols, uint16_t* out, int64_t ld) {
    tc::let_next_start();
    tc::wait_for_previous();
    for (int64_t col = static_cast<int64_t>(blockIdx.y) * kPackCols + threadIdx.x % 128 * 8; col < cols; col += static_cast<int64_t>(gridDim.y) * kPackCols) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t row = static_cast<int64_t>(blockIdx.x) * 8 + threadIdx.x / 128 + 2 * i;
            if (row >= rows) break;
            const uint8_t* from = reinterpret_cast<const uint8_t*>(a + row * rs);
            const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(from) & 15u);
            const uint8_t* unit = from - off + col * 2;
            const uint4 x = unit_of_row(unit, from, from + cols * 2);
            const uint4 y = off == 0 ? x : unit_of_row(unit + 16, from, from + cols * 2);
            const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {      // the row's offset is the same for the whole warp
                const uint32_t lo = off < 4 ? w[j] : off < 8 ? w[j + 1] : off < 12 ? w[j + 2] : w[j + 3];
                const uint32_t hi = off < 4 ? w[j + 1] : off < 8 ? w[j + 2] : off < 12 ? w[j + 3] : w[j + 4];
                o[j] = (off & 2u) ? __funnelshift_r(lo, hi, 16) : lo;
            }
            *reinterpret_cast<uint4*>(out + row * ld + col) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

// out[r][c] = a[r * rs + c * cs], rows of ld elements; reads run along whichever stride is smaller.
__global__ void __launch_bounds__(256) pack_kernel(const uint16_t* a, int64_t rs, int64_t cs, int64_t rows, int64_t cols,
                                                   uint16_t* out, int64_t ld) {
    __shared__ uint16_t t[32][34];
    tc::let_next_start();
    tc::wait_for_previous();
    const int x = threadIdx.x % 32, y = threadIdx.x / 32;
    const int64_t across = (cols + 31) / 32;
    const int64_t r0 = blockIdx.x / across * 32, c0 = blockIdx.x % across * 32;
    const bool along_rows = rs < cs;
    for (int i = y; i < 32; i += 8) {
        const int64_t r = r0 + (along_rows ? x : i), c = c0 + (along_rows ? i : x);
        if (r < rows && c < cols) t[along_rows ? x : i][along_rows ? i : x] = a[r * rs + c * cs];
    }
    __syncthreads();
    for (int i = y; i < 32; i += 8) {
        if (r0 + i < rows && c0 + x < cols) out[(r0 + i) * ld + c0 + x] = t[i][x];
    }
}

}  // namespace

namespace {

// Clocks of an SM.  A slice takes 580 in a pair's 256 x 256 tile (its 32 KB come at 57 to 64 bytes a clock, its products take
// 512) and 420 (24 KB) in the others; a tile costs 300 beside its slices, the last one its epilogue.
struct Tiles {
    int cg, bn, form;
    double slice, last;
};
constexpr Tiles kPair{2, 256, kWhole, 580.0, 4000.0}, kHalfPair{2, 128, kWhole, 420.0, 2000.0}, kLongPair{2, 192, kLong, 560.0, 3000.0},
    kBlock{1, 64, kWhole, 420.0, 1000.0}, kJoinedBlock{1, 64, kJoined, 420.0, 1000.0};
constexpr double kLaunch = 4000.0;         // from one kernel's end to the next one's first products

int64_t tiles_of(const Tiles& t, int64_t m, int64_t n) { return parts(m, 128 * t.cg) * parts(n, t.bn); }

}  // namespace

// The division of the work with the least estimated time.  Tiles that do not fill a last round of the workers may be split, and
// joined by whoever finishes last, which takes some 12 us (2048 x 2048 x 8192, 256 tiles for 74 pairs: 48 us in four rounds, 55 us in
// three and the halves of 34): it pays where a round is longer than that.  Blocks of a cluster exchange their sums in about
// 4500 (197 x 768 x 768: 6.3 us with four shares of k, 5.7 us without).
Config choose(const Call& c, int64_t m, int64_t n, int64_t k, bool sums, bool alone) {
    const int64_t slices = std::max<int64_t>(1, parts(k, kSlice));
    const bool long_sums = sums && slices > kSegment;
    Config best{2, 256, kWhole, static_cast<int>(tiles_of(kPair, m, n)), 1, static_cast<int>(slices), 1e300};
    auto consider = [&](const Tiles& f, int64_t s) {
        const int64_t per = parts(slices, s);
        if (parts(slices, per) != s) return;
        const int64_t tiles = tiles_of(f, m, n), workers = c.sms / f.cg;
        int64_t whole = 0;
        double t;
        if (f.form == kJoined) {
            if (tiles > (s == 2 ? c.sms / 2 : s == 4 ? c.sms * 33 / 148 : c.sms * 15 / 148)) return;     // clusters that fit at a time
            t = per * f.slice + 4500.0 + f.last;
        } else {
            whole = s == 1 ? tiles : tiles / workers * workers;
            t = static_cast<double>(parts(whole, workers)) * (slices * f.slice + 300.0) + f.last;
            if (s > 1) t += static_cast<double>(parts((tiles - whole) * s, workers)) * (per * f.slice + 300.0) + 20000.0 + 1200.0 * s * (f.bn / 128);
        }
        if (t < best.clocks) best = Config{f.cg, f.bn, f.form, static_cast<int>(whole), static_cast<int>(s), static_cast<int>(per), t};
    };
    const int64_t most = alone ? 1 : std::min<int64_t>(16, std::max<int64_t>(1, slices / 8));
    for (int64_t s = 1; s <= most; ++s) {
        if (long_sums) {
            consider(kLongPair, s);
        } else {
            consider(kPair, s);
            consider(kHalfPair, s);
        }
    }
    if (!long_sums) consider(kBlock, 1);
    for (int64_t s = 2; !alone && s <= 8; s *= 2) {
        if (sums && parts(slices, s) > kSegment) continue;
        consider(kJoinedBlock, s);
    }
    return best;
}

// What a device's properties and the library's symbols say, asked once a device.
struct Device {
    std::atomic<int> sms{0};
    std::atomic<unsigned int*> mark{nullptr};
};
static Device devices[64];

bool device_of(Call& c) {
    if (cudaGetDevice(&c.device) != cudaSuccess || c.device < 0 || c.device >= 64) return false;
    Device& d = devices[c.device];
    int sms = d.sms.load(std::memory_order_acquire);
    if (sms == 0) {
        void* mark = nullptr;
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, c.device) != cudaSuccess) return false;
        if (cudaGetSymbolAddress(&mark, wait_ran_out) != cudaSuccess || encoder() == nullptr) return false;
        d.mark.store(static_cast<unsigned int*>(mark), std::memory_order_relaxed);
        d.sms.store(sms, std::memory_order_release);
    }
    c.sms = sms;
    c.mark = d.mark.load(std::memory_order_relaxed);
    return true;
}

dlion_status begin(Call& c, void* workspace, uint64_t bytes, void* stream) {
    c.ws.base = static_cast<uint8_t*>(workspace);
    c.ws.size = bytes;
    c.ws.dry = false;
    c.stream = static_cast<cudaStream_t>(stream);
    return device_of(c) ? DLION_OK : DLION_ECUDA;
}

static bool rows_in_place(const void* p, int64_t rows, int64_t cols, int64_t rs, int64_t cs) {
    if (cs != 1 && cols != 1) return false;
    if (!aligned16(p)) return false;
    return rows == 1 || (rs % 8 == 0 && rs >= cols);
}

Matrix readable(Call& c, const Matrix& a) {
    Matrix r = a;
    if (rows_in_place(a.p, a.rows, a.cols, a.rs, a.cs)) {
        r.cs = 1;
        if (a.rows == 1) r.rs = round_up(a.cols, 8);
        return r;
    }
    if (rows_in_place(a.p, a.cols, a.rows, a.cs, a.rs)) {
        r.rs = 1;
        if (a.cols == 1) r.cs = round_up(a.rows, 8);
        return r;
    }
    // adjacent columns stay adjacent, adjacent rows too; anything else becomes adjacent columns
    const bool along_rows = a.cs != 1 && a.rs == 1;
    const int64_t rows = along_rows ? a.cols : a.rows, cols = along_rows ? a.rows : a.cols;
    const int64_t ld = round_up(cols, 8);
    r.rs = along_rows ? 1 : ld;
    r.cs = along_rows ? ld : 1;
    uint16_t* out = c.ws.take<uint16_t>(static_cast<uint64_t>(rows) * ld);
    r.p = out;
    if (!c.live()) return r;
    const auto* from = static_cast<const uint16_t*>(a.p);
    if (a.cs == 1 || a.rs == 1) {
        const dim3 grid(static_cast<unsigned>(parts(rows, 8)), static_cast<unsigned>(std::min<int64_t>(parts(cols, kPackCols), 65535)));
        start(c, pack_rows_kernel, grid, dim3(256), 0, 1, from, along_rows ? a.cs : a.rs, rows, cols, out, ld);
    } else {                                   // neither adjacent: a.rows and a.cols as they are
        start(c, pack_kernel, dim3(static_cast<unsigned>(parts(rows, 32) * parts(cols, 32))), dim3(256), 0, 1, from, a.rs, a.cs, rows, cols, out, ld);
    }
    return r;
}

bool make_map(CUtensorMap* map, const Matrix& a, int* mn_major, int box_rows) {
    const bool mn = a.cs != 1;                 // adjacent rows
    *mn_major = mn ? 1 : 0;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(mn ? a.rows : a.cols), static_cast<cuuint64_t>(mn ? a.cols : a.rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(mn ? a.cs : a.rs) * 2};
    const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(mn ? kSlice : box_rows)};
    const cuuint32_t one[2] = {1, 1};
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(a.p), dims, strides, box, one,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool shape_of(const Config& cfg, const Matrix& a, const Matrix& b, Shape* s) {
    s->tiles_m = static_cast<int>(parts(a.rows, 128 * cfg.cg));
    s->tiles_n = static_cast<int>(parts(b.rows, cfg.bn));
    s->slices = static_cast<int>(parts(a.cols, kSlice));
    s->whole = cfg.whole;
    s->splits = cfg.splits;
    s->split_slices = cfg.split_slices;
    return static_cast<int64_t>(s->tiles_m) * s->tiles_n * s->splits < (int64_t{1} << 30);
}

static void complete(Finish& f, const Matrix& a, const Matrix& b) {
    f.m = static_cast<int>(a.rows);
    f.n = static_cast<int>(b.rows);
    f.todo = (f.scale != nullptr ? kScale : 0u) | (f.bias != nullptr ? kBias : 0u) | (f.keep == DLION_KEEP_BF16 ? kKeep16 : 0u) |
             (f.keep == DLION_KEEP_8BIT ? kKeep8 : 0u) | (f.act != DLION_ACT_NONE ? kAct : 0u) | (f.slope != DLION_ACT_NONE ? kSlope : 0u) |
             (f.residual != nullptr ? kResidual : 0u) | (f.accumulated != nullptr ? kAdd : 0u);
    f.wide = aligned16(f.out) && f.out_ld * (f.out_f32 ? 4 : 2) % 16 == 0;
}

static bool place(Call& c, const Config& cfg, const Matrix& a, const Matrix& b, Work<Finish>& w, int i) {
    if (make_map(&w.a[i], a, &w.s[i].a_mn, 128) && make_map(&w.b[i], b, &w.s[i].b_mn, cfg.bn / cfg.cg)) return true;
    c.status = DLION_ECUDA;
    return false;
}

template <bool TWO>
static void launch_as(Call& c, const Config& cfg, Work<Finish>& w) {
    if (cfg.form == kLong) {
        launch<2, 192, General, kLong, TWO>(c, w);
    } else if (cfg.form == kJoined) {
        if constexpr (!TWO) launch<1, 64, General, kJoined>(c, w);
    } else if (cfg.cg == 1) {
        launch<1, 64, General, kWhole, TWO>(c, w);
    } else if (cfg.bn == 128) {
        launch<2, 128, General, kWhole, TWO>(c, w);
    } else {
        launch<2, 256, General, kWhole, TWO>(c, w);
    }
}

// Whether a sum of k products is taken in segments where it is longer than one.  Always for a binary32 result; for one rounded to
// bf16, or whose operands are (rough), not before the tensor core's accumulator may have shifted it by a quarter of that rounding:
// 2^-28 a product where all have one sign.  The segments' tiles take longer (131072 x 2048 x 2048, dx and dW: 1.42 ms without, 1.65 with).
constexpr int64_t kRoughMost = 131072;

static bool long_sums(const Finish& f, int64_t k) { return (f.out_f32 != 0 && f.rough == 0) || k > kRoughMost; }

// Whether `blocks` blocks that are there for `clocks` have the time to sum the columns, and how: a warp has eight loads under way,
// some 1500 clocks, and reads whole sectors where there are columns enough.
static bool fits_beside(Beside& s, int64_t blocks, double clocks) {
    if (s.out == nullptr) return false;
    for (int lanes = 4; lanes >= 1; lanes /= 2) {
        const double strips = static_cast<double>(parts(parts(s.cols, 8 * lanes), 2 * blocks));
        s.lanes = lanes;
        if (strips * parts(s.rows, 8 * (32 / lanes)) * 1500.0 + 1500.0 < 0.7 * clocks) return true;
    }
    return false;
}

static bool product_beside(Call& c, const Matrix& a, const Matrix& b, Finish f, Beside beside) {
    complete(f, a, b);
    if (few_rows(c, a, b, f)) return false;
    const Config cfg = choose(c, a.rows, b.rows, a.cols, long_sums(f, a.cols), false);
    Work<Finish> w{};
    if (!shape_of(cfg, a, b, &w.s[0])) {
        c.status = DLION_EINVAL;
        return false;
    }
    const uint64_t mark = c.ws.used;
    const int64_t split_tiles = cfg.form == kJoined || cfg.splits == 1 ? 0 : static_cast<int64_t>(w.s[0].tiles_m) * w.s[0].tiles_n - cfg.whole;
    uint64_t tickets = 0;
    if (split_tiles != 0) {
        tickets = static_cast<uint64_t>(split_tiles) * cfg.cg * kEpilogueWarps;
        f.parts = c.ws.take<float4>(tickets * cfg.splits * (cfg.bn / 2) * 8);
        tickets *= 4;
        f.tickets = c.ws.take<unsigned int>(tickets);
    }
    const int64_t blocks = std::min<int64_t>(units_of(w.s[0]), c.sms / cfg.cg) * cfg.cg;
    const bool summed = fits_beside(beside, blocks, cfg.clocks);
    if (c.live() && place(c, cfg, a, b, w, 0)) {
        w.args[0] = f;
        if (summed) w.beside = beside;
        if (tickets != 0) c.check(cudaMemsetAsync(f.tickets, 0, tickets * sizeof(unsigned int), c.stream));
        launch_as<false>(c, cfg, w);
    }
    // later products of the call reuse the split sums' place (the stream orders them): the size query keeps the maximum
    if (c.ws.dry) c.ws.size = std::max(c.ws.size, c.ws.used);
    c.ws.used = mark;
    return summed;
}

void product(Call& c, const Matrix& a, const Matrix& b, Finish f) { product_beside(c, a, b, f, Beside{}); }

bool products(Call& c, const Part& first, const Part& second, Beside beside) {
    // both as whole tiles of one kind, the longer sums first, against each for itself; few rows have their own kernel
    const Part* parts_of[2] = {&first, &second};
    if (second.a.cols > first.a.cols) std::swap(parts_of[0], parts_of[1]);
    const Part &p0 = *parts_of[0], &p1 = *parts_of[1];
    const bool few = p0.a.rows <= kFewRows || p1.a.rows <= kFewRows;
    const Config best0 = choose(c, p0.a.rows, p0.b.rows, p0.a.cols, long_sums(p0.f, p0.a.cols), false);
    const Config best1 = choose(c, p1.a.rows, p1.b.rows, p1.a.cols, long_sums(p1.f, p1.a.cols), false);
    const int64_t slices0 = parts(p0.a.cols, kSlice), slices1 = parts(p1.a.cols, kSlice);
    const bool sums = (long_sums(p0.f, p0.a.cols) && slices0 > kSegment) || (long_sums(p1.f, p1.a.cols) && slices1 > kSegment);
    double clocks = best0.clocks + best1.clocks + kLaunch;
    Config cfg{};
    int64_t extra = 0;
    for (const Tiles* f : {&kPair, &kHalfPair, &kBlock, &kLongPair}) {
        if (few || sums != (f->form == kLong)) continue;
        const int64_t t0 = tiles_of(*f, p0.a.rows, p0.b.rows), t1 = tiles_of(*f, p1.a.rows, p1.b.rows), workers = c.sms / f->cg;
        if (t0 + t1 >= (int64_t{1} << 30)) continue;
        const double big = slices0 * f->slice + 300.0, small = slices1 * f->slice + 300.0;
        const int64_t over = t0 % workers, ahead = over == 0 ? 0 : static_cast<int64_t>(big / small + 0.5);
        const int64_t rest = std::max<int64_t>(0, t1 - ahead * (workers - over));
        const double t = parts(t0, workers) * big + parts(rest, workers) * small + f->last;
        if (t < clocks) {
            clocks = t;
            cfg = Config{f->cg, f->bn, f->form, 0, 1, 0, t};
            extra = ahead;
        }
    }
    if (cfg.cg == 0) {
        bool summed = false;
        for (const Part* part : {&first, &second}) {
            if (!part->wanted) continue;
            summed = product_beside(c, part->a, part->b, part->f, beside) || summed;
            if (summed) beside.out = nullptr;
        }
        return summed;
    }
    if (!first.wanted && !second.wanted) return false;
    Work<Finish> w{};
    w.extra = static_cast<int>(extra);
    int n = 0;
    for (const Part* part : parts_of) {
        if (!part->wanted) continue;
        w.args[n] = part->f;
        complete(w.args[n], part->a, part->b);
        cfg.split_slices = static_cast<int>(parts(part->a.cols, kSlice));
        cfg.whole = static_cast<int>(parts(part->a.rows, 128 * cfg.cg) * parts(part->b.rows, cfg.bn));
        if (!shape_of(cfg, part->a, part->b, &w.s[n])) {
            c.status = DLION_EINVAL;
            return false;
        }
        if (c.live() && !place(c, cfg, part->a, part->b, w, n)) return false;
        ++n;
    }
    const int units = units_of(w.s[0]) + (n == 2 ? units_of(w.s[1]) : 0);
    const bool summed = fits_beside(beside, std::min(units, c.sms / cfg.cg) * cfg.cg, n == 2 ? clocks : clocks / 2);
    if (summed) w.beside = beside;
    if (!c.live()) return summed;
    if (n == 2) launch_as<true>(c, cfg, w);
    if (n == 1) launch_as<false>(c, cfg, w);
    return summed;
}

}  // namespace prod
}  // namespace dlion

extern "C" dlion_status dlion_layers_check(void* cuda_stream) {
    if (cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess) return DLION_ECUDA;
    unsigned int mark = 0;
    if (cudaMemcpyFromSymbol(&mark, dlion::prod::wait_ran_out, sizeof mark) != cudaSuccess) return DLION_ECUDA;
    if (mark == 0) return DLION_OK;
    mark = 0;
    if (cudaMemcpyToSymbol(dlion::prod::wait_ran_out, &mark, sizeof mark) != cudaSuccess) return DLION_ECUDA;
    return DLION_ESTATE;
}
