// Host side of the layer products: operands, workspace, launches.
#pragma once

#include <algorithm>
#include <atomic>

#include "host_checks.h"
#include "product.cuh"

namespace dlion {
namespace prod {

// bf16 matrix of any strides (in elements)
struct Matrix {
    const void* p;
    int64_t rows, cols, rs, cs;
};

// Workspace handed out front to back.  With no memory behind it, it only counts: the size queries run
// the same code as the calls.
struct Workspace {
    uint8_t* base = nullptr;
    uint64_t used = 0, size = 0;
    bool dry = true;
    bool enough = true;

    template <class T>
    T* take(uint64_t count) {
        const uint64_t at = used;
        used += (count * sizeof(T) + 255u) & ~uint64_t{255};
        if (dry) return nullptr;
        if (used > size) {
            enough = false;
            return nullptr;
        }
        return reinterpret_cast<T*>(base + at);
    }
};

struct Call {
    Workspace ws;
    cudaStream_t stream = nullptr;
    int device = -1, sms = 148;
    unsigned int* mark = nullptr;
    dlion_status status = DLION_OK;

    bool live() const { return !ws.dry && ws.enough && status == DLION_OK; }
    void check(cudaError_t e) {
        if (e != cudaSuccess && status == DLION_OK) status = DLION_ECUDA;
    }
    dlion_status end() const { return status != DLION_OK ? status : (ws.dry || ws.enough) ? DLION_OK : DLION_EINVAL; }
};

// Device, SM count and the mark's address; the workspace's extent.
bool device_of(Call& c);
dlion_status begin(Call& c, void* workspace, uint64_t bytes, void* stream);

// `a` itself if tiles of it can be copied in place, otherwise a packed copy in the workspace.
Matrix readable(Call& c, const Matrix& a);

// D[rows of a][rows of b] = sum over the columns of both; a.T / b.T by swapping rows and cols, rs and cs.
// Both must be readable.  f.m, f.n are set here.
void product(Call& c, const Matrix& a, const Matrix& b, Finish f);

// Two products that do not depend on each other, in one launch where that is expected to take less time.  One of them alone
// (the other's matrices need only their sizes) is divided as it is beside the other, so that its bits are the same.
struct Part {
    Matrix a, b;
    Finish f;
    bool wanted;
};
// `beside`: column sums that the products' idle warps take along where they have the time for it; false if they do not.
bool products(Call& c, const Part& first, const Part& second, Beside beside);

constexpr int64_t kFewRows = 16;

// The same for at most kFewRows rows of a; false if this is not such a product.  (few_rows.cu)
bool few_rows(Call& c, const Matrix& a, const Matrix& b, const Finish& f);

inline Matrix transposed(const Matrix& a) { return Matrix{a.p, a.cols, a.rows, a.cs, a.rs}; }

// Tensor map of 64 x `box` tiles; `mn` of the operand's rows adjacent (1) or its columns (0).
bool make_map(CUtensorMap* map, const Matrix& a, int* mn_major, int box_rows);

struct Config {
    int cg, bn, form, whole, splits, split_slices;
    double clocks;                         // estimated
};
// `sums`: binary32 results, whose long sums are taken in segments.  `alone`: no splits.
Config choose(const Call& c, int64_t m, int64_t n, int64_t k, bool sums, bool alone);

// Tile counts of a configuration; false if the tiles cannot be numbered.
bool shape_of(const Config& cfg, const Matrix& a, const Matrix& b, Shape* s);

// Every kernel of the library's layer calls goes out like this: it may be set up while its predecessor drains.
template <class... P, class... A>
void start(Call& c, void (*kernel)(P...), dim3 grid, dim3 block, size_t shared, int cluster, const A&... args) {
    if (c.status != DLION_OK) return;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = shared;
    cfg.stream = c.stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = static_cast<unsigned>(cluster);
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    c.check(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
}

// More than 48 KB of shared memory for a kernel, asked for once a device.
template <class K>
void raise_shared(Call& c, K* kernel, int bytes) {
    struct Entry {
        std::atomic<const void*> kernel{nullptr};
        std::atomic<uint64_t> devices{0};
    };
    static Entry entries[16];                  // of kernels of this type
    const uint64_t bit = uint64_t{1} << (c.device & 63);
    for (Entry& e : entries) {
        const void* seen = nullptr;
        if (!e.kernel.compare_exchange_strong(seen, reinterpret_cast<const void*>(kernel)) && seen != reinterpret_cast<const void*>(kernel)) continue;
        if ((e.devices.load(std::memory_order_acquire) & bit) != 0) return;
        c.check(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
        if (c.status == DLION_OK) e.devices.fetch_or(bit, std::memory_order_release);
        return;
    }
    c.check(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
}

inline int units_of(const Shape& s) { return s.whole + (s.tiles_m * s.tiles_n - s.whole) * s.splits; }

// `w` but for its unit counts.
template <int CG, int BN, class E, int FORM, bool TWO = false>
void launch(Call& c, Work<typename E::Args>& w) {
    auto* kernel = &product_kernel<CG, BN, E, FORM, TWO>;
    raise_shared(c, kernel, kSmem);
    w.units[0] = units_of(w.s[0]);
    w.units[1] = TWO ? units_of(w.s[1]) : 0;
    const int units = w.units[0] + w.units[1], blocks = FORM == kJoined ? units : std::min(units, c.sms / CG) * CG;
    start(c, kernel, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), kSmem, FORM == kJoined ? w.s[0].splits : CG, w, c.mark);
}

inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline int64_t parts(int64_t v, int64_t of) { return (v + of - 1) / of; }

template <class P, class F>
uint64_t workspace_of(const P& p, F f) {
    Call c;
    device_of(c);                              // without a GPU the SM count of a B200 stands
    f(c, p);
    return std::max(c.ws.size, c.ws.used);
}

template <class P, class F>
dlion_status run(const P& p, F f, void* workspace, uint64_t bytes, void* stream) {
    if (bytes != 0 && workspace == nullptr) return DLION_EINVAL;
    if (!aligned16(workspace)) return DLION_EALIGN;
    if (bytes < workspace_of(p, f)) return DLION_EINVAL;        // nothing is launched
    Call c;
    const dlion_status st = begin(c, workspace, bytes, stream);
    if (st != DLION_OK) return st;
    f(c, p);
    return c.end();
}

}  // namespace prod
}  // namespace dlion
