// Low-rank adapters of many requests at once, beside a shared projection (gfx950).
//
//   C[r] = R[r] + scale_a T[r] B_a^T,  T[r] = x[r] A_a^T,    A_a [rank, K], B_a [N, rank]: the adapter a of the request that row r belongs to
//
// Adapters lie in slots of a pool, A [slots][width][K] and B [slots][N][width].  Two launches: T, in as many pieces of K as it takes to fill the
// card, each a plane of float32 sums in scratch; then C, whose workgroups add the planes first.  Rows go in tiles of 16 MR of one
// request; a request's tiles multiply with its slot alone, so a batch costs the bytes of its rows and of the slots that it uses.
// Operands go from memory to registers in the matrix instruction's own order, 16 bytes a lane and load: no element is read twice by a workgroup,
// so there is nothing to stage.
#include "adapters.h"

#include <string.h>

#include <algorithm>

namespace po {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

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
    float* t;                  // [pieces][tiles][16 MR][rp]
    int N, K, width;
    int rp;                    // ranks of a row of t: 16 NR of the launch
    int pieces, per;           // of K, and k-steps of 32 of a wavefront's share of one
    int cols;                  // of a workgroup of the second launch
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

// Eight consecutive elements of K of a row, for lane (row = lane & 15, elements 8 (lane >> 4) .. + 7 of a step of 32).  The float32 instruction
// takes one element of each lane: with e the same in both operands eight of them cover the step.
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { bf16x8 v; };
template <> struct Frag<float> { f32x4 lo, hi; };

__device__ __forceinline__ void load(Frag<bf16_t>& f, const bf16_t* p) { f.v = *(const bf16x8*)p; }
__device__ __forceinline__ void load(Frag<float>& f, const float* p) {
    f.lo = *(const f32x4*)p;
    f.hi = *(const f32x4*)(p + 4);
}
__device__ __forceinline__ void zero(Frag<bf16_t>& f) { f.v = __builtin_bit_cast(bf16x8, make_uint4(0, 0, 0, 0)); }
__device__ __forceinline__ void zero(Frag<float>& f) { f.lo = f.hi = f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ f32x4 mma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(const Frag<float>& a, const Frag<float>& b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.lo[e], b.lo[e], c, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.hi[e], b.hi[e], c, 0, 0, 0);
    return c;
}
// of the first n of eight elements, the others 0 whatever they hold
__device__ __forceinline__ void keep(Frag<bf16_t>& f, int n) {
    uint4 w = __builtin_bit_cast(uint4, f.v);
    uint32_t* p = (uint32_t*)&w;
#pragma unroll
    for (int c = 0; c < 4; ++c) p[c] = 2 * c + 1 < n ? p[c] : 2 * c < n ? p[c] & 0xffffu : 0u;
    f.v = __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ void keep(Frag<float>& f, int n) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        f.lo[c] = c < n ? f.lo[c] : 0.f;
        f.hi[c] = 4 + c < n ? f.hi[c] : 0.f;
    }
}

// T of a tile of 16 MR rows over one piece of K: its four wavefronts take a quarter each and add up in LDS.  A lane of a product of 16 ranks
// and 16 rows holds row lane & 15 and ranks 4 (lane >> 4) .. + 3.
template <typename T, int MR, int NR>
__global__ void __launch_bounds__(256) adapter_down_kernel(const AdapterParams p, const Table tab) {
    __shared__ f32x4 red[4][MR * NR][64];
    const int tile = blockIdx.x;
    const Segment& sg = tab.seg[segment_of(tab, tile)];
    if (sg.rank == 0) return;
    const int r0 = sg.row + (tile - sg.tile0) * (16 * MR), last = sg.row + sg.n - 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, l4 = lane >> 4;
    const int nr = (sg.rank + 15) >> 4, steps = (p.K + 31) >> 5;
    const int s0 = min((int)(blockIdx.y * 4 + wave) * p.per, steps), s1 = min(s0 + p.per, steps);
    const T* xp[MR];                             // (rows behind the request's last one and ranks behind the slot's: that one again)
    const T* ap[NR];
#pragma unroll
    for (int m = 0; m < MR; ++m) xp[m] = (const T*)p.x + (int64_t)min(r0 + m * 16 + l15, last) * p.K + l4 * 8;
#pragma unroll
    for (int j = 0; j < NR; ++j) ap[j] = (const T*)p.a + ((int64_t)sg.slot * p.width + min(j * 16 + l15, sg.rank - 1)) * p.K + l4 * 8;
    f32x4 acc[MR][NR];
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int j = 0; j < NR; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // U steps are multiplied while the next U are on their way
    constexpr int U = MR + NR <= 2 ? 4 : MR + NR <= 8 ? 2 : 1;
    struct Stage {
        Frag<T> x[U][MR], a[U][NR];
    };
    auto fetch = [&](Stage& g, int at) {
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int u = 0; u < U; ++u) load(g.x[u][m], xp[m] + (at + u) * 32);
#pragma unroll
        for (int j = 0; j < NR; ++j)
            if (j < nr) {
#pragma unroll
                for (int u = 0; u < U; ++u) load(g.a[u][j], ap[j] + (at + u) * 32);
            }
    };
    auto multiply = [&](const Stage& g) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < NR; ++j)
                if (j < nr) {
#pragma unroll
                    for (int m = 0; m < MR; ++m) acc[m][j] = mma(g.a[u][j], g.x[u][m], acc[m][j]);
                }
    };
    int s = s0;
    const int whole = min(s1, p.K >> 5);         // (steps without a border of K)
    if (s + U <= whole) {
        Stage g0, g1;
        fetch(g0, s);
        for (; s + 3 * U <= whole; s += 2 * U) {
            fetch(g1, s + U);
            __builtin_amdgcn_sched_barrier(0);
            multiply(g0);
            fetch(g0, s + 2 * U);
            __builtin_amdgcn_sched_barrier(0);
            multiply(g1);
        }
        multiply(g0);
        s += U;
    }
    for (; s < s1; ++s) {
        const bool in = s * 32 + l4 * 8 < p.K;   // (K is a multiple of 8)
        Frag<T> x[MR];
#pragma unroll
        for (int m = 0; m < MR; ++m) {
            zero(x[m]);
            if (in) load(x[m], xp[m] + s * 32);
        }
#pragma unroll
        for (int j = 0; j < NR; ++j)
            if (j < nr) {
                Frag<T> a;
                zero(a);
                if (in) load(a, ap[j] + s * 32);
#pragma unroll
                for (int m = 0; m < MR; ++m) acc[m][j] = mma(a, x[m], acc[m][j]);
            }
    }
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int j = 0; j < NR; ++j) red[wave][m * NR + j][lane] = acc[m][j];
    __syncthreads();
    float* t = p.t + ((int64_t)blockIdx.y * gridDim.x + tile) * (16 * MR) * p.rp;
    for (int f = wave; f < MR * NR; f += 4) {
        const int m = f / NR, j = f - m * NR;
        if (j >= nr) continue;
        const f32x4 v = red[0][f][lane] + red[1][f][lane] + red[2][f][lane] + red[3][f][lane];
        *(f32x4*)(t + (m * 16 + l15) * p.rp + j * 16 + 4 * l4) = v;
    }
}

// the fragments of T in the second product: bf16 in two parts (the rounding of T and that of what it left, 2^-16 of T together),
// float32 whole
template <typename T> struct Parts;
template <> struct Parts<bf16_t> { static constexpr int N = 2; };
template <> struct Parts<float> { static constexpr int N = 1; };
__device__ __forceinline__ void split(const float (&v)[8], Frag<bf16_t> (&f)[2]) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const bf16_t h0 = f2bf(v[2 * c]), h1 = f2bf(v[2 * c + 1]);
        hi[c] = (uint32_t)h0 | ((uint32_t)h1 << 16);
        lo[c] = (uint32_t)f2bf(v[2 * c] - bf2f(h0)) | ((uint32_t)f2bf(v[2 * c + 1] - bf2f(h1)) << 16);
    }
    f[0].v = __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
    f[1].v = __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
}
__device__ __forceinline__ void split(const float (&v)[8], Frag<float> (&f)[1]) {
    f[0].lo = f32x4{v[0], v[1], v[2], v[3]};
    f[0].hi = f32x4{v[4], v[5], v[6], v[7]};
}

__device__ __forceinline__ void load_out(float (&v)[8], const bf16_t* p) {
    const uint4 w = *(const uint4*)p;
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        v[2 * c] = __uint_as_float(u[c] << 16);
        v[2 * c + 1] = __uint_as_float(u[c] & 0xffff0000u);
    }
}
__device__ __forceinline__ void load_out(float (&v)[8], const float* p) {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store_out(bf16_t* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = (uint32_t)f2bf(v[2 * c]) | ((uint32_t)f2bf(v[2 * c + 1]) << 16);
    *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_out(float* p, const float (&v)[8]) {
    *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// C of a tile of 16 MR rows and p.cols columns, a quarter of them a wavefront, 64 at a time (lines of 128 bytes in bf16).  Product h of those takes the
// columns 32 (h / 2) + 8 g + 4 (h & 1) + e (g, e < 4) as its rows 4 g + e, so that a lane ends up with eight consecutive ones, from 8 (lane >> 4) on of
// either half, of row lane & 15.
template <typename T, int MR, int KS>
__global__ void __launch_bounds__(256) adapter_up_kernel(const AdapterParams p, const Table tab) {
    constexpr int NP = Parts<T>::N;
    __shared__ Frag<T> tf[MR][KS][NP][64];
    const int tile = blockIdx.x;
    const Segment& sg = tab.seg[segment_of(tab, tile)];
    const int r0 = sg.row + (tile - sg.tile0) * (16 * MR), end = sg.row + sg.n;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, l4 = lane >> 4;
    const int ks = (sg.rank + 31) >> 5;
    const int64_t plane = (int64_t)gridDim.x * (16 * MR) * p.rp;
    for (int f = wave; f < MR * ks; f += 4) {    // (a wavefront at a time: fragment f / ks, step f % ks)
        const int m = f / ks, k = f - m * ks, j0 = k * 32 + l4 * 8;
        const float* t = p.t + ((int64_t)tile * (16 * MR) + m * 16 + l15) * p.rp + j0;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
        if (j0 < sg.rank)
            for (int i = 0; i < p.pieces; ++i) {
                const f32x4 a = *(const f32x4*)(t + i * plane), b = *(const f32x4*)(t + i * plane + 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] += a[e];
                    v[4 + e] += b[e];
                }
            }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = j0 + e < sg.rank ? v[e] * sg.scale : 0.f;
        Frag<T> part[NP];
        split(v, part);
#pragma unroll
        for (int i = 0; i < NP; ++i) tf[m][k][i][lane] = part[i];
    }
    __syncthreads();
    Frag<T> t[MR][KS][NP];
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (k < ks) t[m][k][i] = tf[m][k][i][lane];
    const T* b = (const T*)p.b + (int64_t)sg.slot * p.N * p.width;
    const int share = p.cols >> 2, first = blockIdx.y * p.cols + wave * share, n1 = min(first + share, p.N);
    for (int c0 = first; c0 < n1; c0 += 64) {
        float out[MR][2][8];
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int col = c0 + q * 32 + l4 * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e) out[m][q][e] = 0.f;
                if (p.res && r0 + m * 16 + l15 < end && col < n1) load_out(out[m][q], (const T*)p.res + (int64_t)(r0 + m * 16 + l15) * p.N + col);
            }
        f32x4 acc[MR][4];
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int h = 0; h < 4; ++h) acc[m][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const T* bp = b + (int64_t)min(c0 + (h >> 1) * 32 + (l15 >> 2) * 8 + (h & 1) * 4 + (l15 & 3), p.N - 1) * p.width + l4 * 8;
#pragma unroll
            for (int k = 0; k < KS; ++k)
                if (k < ks) {
                    const int left = sg.rank - k * 32 - l4 * 8;
                    Frag<T> w;
                    zero(w);
                    if (left > 0) {              // (width is a multiple of 8)
                        load(w, bp + k * 32);
                        if (left < 8) keep(w, left);
                    }
#pragma unroll
                    for (int m = 0; m < MR; ++m)
#pragma unroll
                        for (int i = NP - 1; i >= 0; --i) acc[m][h] = mma(w, t[m][k][i], acc[m][h]);
                }
        }
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int col = c0 + q * 32 + l4 * 8;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    out[m][q][e] += acc[m][2 * q][e];
                    out[m][q][4 + e] += acc[m][2 * q + 1][e];
                }
                if (r0 + m * 16 + l15 < end && col < n1) store_out((T*)p.c + (int64_t)(r0 + m * 16 + l15) * p.N + col, out[m][q]);
            }
    }
}

struct Launch {
    Table tab;
    int rank, mr, nr, pieces, per, cols;
    size_t floats;             // of scratch
};

// tiles, pieces and columns of a launch
void plan(Launch& l, int N, int K) {
    Table& t = l.tab;
    int longest = 0;
    l.rank = 0;
    for (int i = 0; i < t.n; ++i) {
        l.rank = std::max(l.rank, t.seg[i].rank);
        longest = std::max(longest, t.seg[i].n);
    }
    l.nr = l.rank <= 16 ? 1 : l.rank <= 32 ? 2 : l.rank <= 64 ? 4 : 8;
    l.mr = longest <= 16 ? 1 : l.nr == 8 ? 2 : 4;
    t.tiles = 0;
    for (int i = 0; i < t.n; ++i) {
        t.seg[i].tile0 = t.tiles;
        t.tiles += (t.seg[i].n + 16 * l.mr - 1) / (16 * l.mr);
    }
    const int steps = (K + 31) / 32;
    l.pieces = std::max(1, std::min({8, 1024 / t.tiles, steps / 16}));
    l.per = ((steps + l.pieces * 4 - 1) / (l.pieces * 4) + 1) / 2 * 2;         // (whole lines of 128 bytes)
    l.cols = 1024;
    while (l.cols > 256 && (int64_t)t.tiles * ((N + l.cols - 1) / l.cols) < 1024) l.cols /= 2;
    l.floats = l.rank ? (size_t)l.pieces * t.tiles * 16 * l.mr * 16 * l.nr : 0;
}

// calls f(Launch&) for every launch's table of requests, tiles counted
template <typename F>
void for_launches(const int32_t* ranks, const float* scales, bool in_place, int64_t rows, int N, int K, const po_adapter_rows* seg, int n_seg, F f) {
    Launch l;
    Table& tab = l.tab;
    tab.n = 0;
    auto flush = [&]() {
        if (tab.n) {
            plan(l, N, K);
            f(l);
        }
        tab.n = 0;
    };
    auto add = [&](int64_t row, int64_t n, int slot) {
        const int rank = slot < 0 ? 0 : ranks[slot];
        if (n <= 0 || (rank == 0 && in_place)) return;         // (nothing to do: the rows stay as they are)
        Segment* last = tab.n ? &tab.seg[tab.n - 1] : nullptr;
        if (last && last->row + last->n == row && last->rank == rank && (rank == 0 || last->slot == slot)) {       // one run of rows
            last->n += (int)n;
            return;
        }
        if (tab.n == MAX_SEGMENTS) flush();
        tab.seg[tab.n++] = {(int)row, (int)n, rank ? slot : 0, rank, rank && scales ? scales[slot] : 0.f, 0};
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

template <typename T, int MR, int NR>
void run_t(const AdapterParams& p, const Launch& l, hipStream_t s) {
    const unsigned tiles = (unsigned)l.tab.tiles;
    if (l.rank) hipLaunchKernelGGL((adapter_down_kernel<T, MR, NR>), dim3(tiles, (unsigned)l.pieces), dim3(256), 0, s, p, l.tab);
    hipLaunchKernelGGL((adapter_up_kernel<T, MR, (NR + 1) / 2>), dim3(tiles, (unsigned)((p.N + p.cols - 1) / p.cols)), dim3(256), 0, s, p, l.tab);
}

template <typename T>
void run(AdapterParams p, const Launch& l, hipStream_t s) {
    p.rp = 16 * l.nr;
    p.pieces = l.pieces;
    p.per = l.per;
    p.cols = l.cols;
    switch (l.nr * 8 + l.mr) {
        case 8 + 1: run_t<T, 1, 1>(p, l, s); break;
        case 16 + 1: run_t<T, 1, 2>(p, l, s); break;
        case 32 + 1: run_t<T, 1, 4>(p, l, s); break;
        case 64 + 1: run_t<T, 1, 8>(p, l, s); break;
        case 8 + 4: run_t<T, 4, 1>(p, l, s); break;
        case 16 + 4: run_t<T, 4, 2>(p, l, s); break;
        case 32 + 4: run_t<T, 4, 4>(p, l, s); break;
        default: run_t<T, 2, 8>(p, l, s); break;
    }
}

}  // namespace

size_t adapters_scratch(const int32_t* ranks, int64_t rows, int N, int K, const po_adapter_rows* seg, int n_seg) {
    size_t most = 0;
    // (in place or not changes the tables of launches: the larger of both)
    for (const bool in_place : {false, true})
        for_launches(ranks, nullptr, in_place, rows, N, K, seg, n_seg, [&](const Launch& l) { most = std::max(most, l.floats); });
    return most * sizeof(float);
}

void launch_adapters(int dtype, const void* x, const void* a, const void* b, const int32_t* ranks, const float* scales, int width, const void* res,
                     void* c, int64_t rows, int N, int K, const po_adapter_rows* seg, int n_seg, float* t, hipStream_t s) {
    AdapterParams p;
    memset(&p, 0, sizeof(p));
    p.x = x; p.a = a; p.b = b; p.res = res; p.c = c; p.t = t;
    p.N = N; p.K = K; p.width = width;
    for_launches(ranks, scales, res == c, rows, N, K, seg, n_seg, [&](const Launch& l) {
        if (dtype == 0) run<float>(p, l, s);
        else run<bf16_t>(p, l, s);
    });
}

}  // namespace po
