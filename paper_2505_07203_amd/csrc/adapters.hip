// Low-rank adapters of many requests at once, beside a shared projection (gfx950).
//
//   C[r] = R[r] + scale_a (x[r] A_a^T) B_a^T,    A_a [rank, K], B_a [N, rank]: the adapter a of the request that row r belongs to
//
// Adapters lie in slots of a pool, A [slots][width][K] and B [slots][N][width].  T = x A^T is a float32 number; so is its product with B.
#include "adapters.h"

#include <string.h>

#include <algorithm>

namespace po {
namespace {

// Requests of one launch, passed by value (a captured launch keeps them, and nothing has to be copied to the device first).  Rows
// of no request and of requests without an adapter are entries of rank 0.
constexpr int MAX_SEGMENTS = 128;
struct Segment {
    int row, n, slot, rank;
    float scale;
    int tile0;                 // its first row tile
};
struct Table {
    int n, tiles;
    Segment seg[MAX_SEGMENTS];
};
struct AdapterParams {
    const void *x, *a, *b, *res;
    void* c;
    float* t;                  // [rows][width]
    int N, K, width;
};

__device__ __forceinline__ int segment_of(const Table& t, int tile) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.seg[mid].tile0 <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

constexpr int ROWS = 8;        // of a tile

// T of a tile's rows: a wavefront per element of T
template <typename T>
__global__ void __launch_bounds__(256) adapter_down_kernel(const AdapterParams p, const Table tab) {
    const Segment& sg = tab.seg[segment_of(tab, blockIdx.x)];
    const int r0 = sg.row + ((int)blockIdx.x - sg.tile0) * ROWS, n = min(ROWS, sg.row + sg.n - r0);
    const int lane = threadIdx.x & 63;
    const T* a = (const T*)p.a + (int64_t)sg.slot * p.width * p.K;
    for (int i = threadIdx.x >> 6; i < n * sg.rank; i += 4) {
        const int r = i / sg.rank, j = i - r * sg.rank;
        const T* x = (const T*)p.x + (int64_t)(r0 + r) * p.K;
        float acc = 0.f;
        for (int k = lane; k < p.K; k += 64) acc = fmaf(to_f32(x[k]), to_f32(a[(int64_t)j * p.K + k]), acc);
        for (int off = 32; off > 0; off >>= 1) acc += __shfl_xor(acc, off);
        if (lane == 0) p.t[(int64_t)(r0 + r) * p.width + j] = acc * sg.scale;
    }
}

// C of a tile's rows and 256 columns
template <typename T>
__global__ void __launch_bounds__(256) adapter_up_kernel(const AdapterParams p, const Table tab) {
    const Segment& sg = tab.seg[segment_of(tab, blockIdx.x)];
    const int r0 = sg.row + ((int)blockIdx.x - sg.tile0) * ROWS, n = min(ROWS, sg.row + sg.n - r0);
    const int col = blockIdx.y * 256 + threadIdx.x;
    if (col >= p.N) return;
    const T* b = (const T*)p.b + ((int64_t)sg.slot * p.N + col) * p.width;
    for (int r = 0; r < n; ++r) {
        const int64_t at = (int64_t)(r0 + r) * p.N + col;
        float acc = 0.f;
        for (int j = 0; j < sg.rank; ++j) acc = fmaf(p.t[(int64_t)(r0 + r) * p.width + j], to_f32(b[j]), acc);
        if (p.res) acc += to_f32(((const T*)p.res)[at]);
        if (sg.rank || p.res != p.c) ((T*)p.c)[at] = from_f32<T>(acc);
    }
}

template <typename T>
void run(const AdapterParams& p, const Table& t, hipStream_t s) {
    hipLaunchKernelGGL((adapter_down_kernel<T>), dim3((unsigned)t.tiles), dim3(256), 0, s, p, t);
    hipLaunchKernelGGL((adapter_up_kernel<T>), dim3((unsigned)t.tiles, (unsigned)((p.N + 255) / 256)), dim3(256), 0, s, p, t);
}

}  // namespace

size_t adapters_scratch(int64_t rows, int width) { return (size_t)rows * (size_t)width * sizeof(float); }

void launch_adapters(int dtype, const void* x, const void* a, const void* b, const int32_t* ranks, const float* scales, int width, const void* res,
                     void* c, int64_t rows, int N, int K, const po_adapter_rows* seg, int n_seg, float* t, hipStream_t s) {
    AdapterParams p = {x, a, b, res, c, t, N, K, width};
    Table tab;
    tab.n = tab.tiles = 0;
    auto flush = [&]() {
        if (tab.n) {
            if (dtype == 0) run<float>(p, tab, s);
            else run<bf16_t>(p, tab, s);
        }
        tab.n = tab.tiles = 0;
    };
    auto add = [&](int64_t row, int64_t n, int slot) {
        const int rank = slot < 0 ? 0 : ranks[slot];
        if (n <= 0 || (rank == 0 && res == c)) return;         // (nothing to do: the rows stay as they are)
        Segment* last = tab.n ? &tab.seg[tab.n - 1] : nullptr;
        if (last && last->row + last->n == row && last->rank == rank && (rank == 0 || last->slot == slot)) {       // one run of rows
            tab.tiles -= (last->n + ROWS - 1) / ROWS;
            last->n += (int)n;
            tab.tiles += (last->n + ROWS - 1) / ROWS;
            return;
        }
        if (tab.n == MAX_SEGMENTS) flush();
        tab.seg[tab.n++] = {(int)row, (int)n, rank ? slot : 0, rank, rank ? scales[slot] : 0.f, tab.tiles};
        tab.tiles += (int)((n + ROWS - 1) / ROWS);
    };
    int64_t at = 0;
    for (int i = 0; i < n_seg; ++i) {
        add(at, seg[i].row - at, -1);
        add(seg[i].row, seg[i].n_rows, (int)seg[i].adapter);
        at = seg[i].row + seg[i].n_rows;
    }
    add(at, rows - at, -1);
    flush();
}

}  // namespace po
