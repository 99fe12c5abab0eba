// Low-rank adapters of many requests at once, beside a shared projection (gfx950).
//
//   C[r] = R[r] + scale_a T[r] B_a^T,  T[r] = x[r] A_a^T,    A_a [rank, K], B_a [N, rank]: the adapter a of the request that row r belongs to
//
// Adapters lie in slots of a pool, A [slots][width][K] and B [slots][N][width].  Two launches: T, in pieces of K, each a plane of float32 sums in
// scratch; then C, whose workgroups add the planes first.  A request's rows multiply with its slot alone, so a batch costs the bytes of its rows and
// of the slots that it uses.  Both launches are bound by memory, operands go from there to registers in the matrix instruction's own
// order, 16 bytes a lane and load.
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
    int row, n;
    int slot_rank;             // slot * 256 + rank
    float scale;
    int group0;                // its first group of 16 rows in t
    __host__ __device__ int slot() const { return slot_rank >> 8; }
    __host__ __device__ int rank() const { return slot_rank & 255; }
};
struct Table {
    int n;
    Segment seg[MAX_SEGMENTS];
    int down0[MAX_SEGMENTS + 1], up0[MAX_SEGMENTS + 1];        // first row tile of each request in either launch, and their number
};
static_assert(sizeof(Table) <= 3840, "with the parameters within 4096 bytes of kernel arguments");
struct AdapterParams {
    const void *x, *a, *b, *res;
    void* c;
    float* t;                  // [pieces][groups of 16 rows][16][rp]
    int64_t plane;             // floats of a piece of t
    int N, K, width;
    int rp;                    // ranks of a row of t: 16 NR of the launch
    int pieces;                // of K
    int groups;                // of 16 rows that a workgroup of the first launch takes
    int cols;                  // of a workgroup of the second launch
};

// the request a tile belongs to: one load a lane instead of a chain of them
__device__ __forceinline__ int segment_of(const int (&tile0)[MAX_SEGMENTS + 1], int n, int tile) {
    const int lane = threadIdx.x & 63;
    int at = 0;
#pragma unroll
    for (int i = 0; i < MAX_SEGMENTS; i += 64) at += __popcll(__ballot(i + lane < n && tile0[i + lane + 1] <= tile));
    return __builtin_amdgcn_readfirstlane(at);
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

// T of a run of rows of one request over one piece of K, 16 rows at a time.  A wavefront takes C steps of 32 of the piece, 512 bytes of a row, and
// holds that part of A in registers for all its rows: A is read once a run, x in visits of 512 bytes, two groups of rows ahead.  The
// wavefronts' sums meet in LDS.  A lane of a product of 16 ranks and 16 rows holds row lane & 15 and ranks 4 (lane >> 4) .. + 3.
constexpr int DOWN_WAVES = 8;
template <typename T, int NR> struct DownSteps { static constexpr int C = (NR == 8 ? 4 : 8) * 2 / (int)sizeof(T); };

template <typename T, int NR>
__global__ void __launch_bounds__(64 * DOWN_WAVES, 2) adapter_down_kernel(const AdapterParams p, const Table tab) {
    constexpr int C = DownSteps<T, NR>::C;
    extern __shared__ f32x4 red[];               // [2][waves][NR][64]
    const int si = segment_of(tab.down0, tab.n, blockIdx.x);
    const Segment& sg = tab.seg[si];
    const int rank = sg.rank();
    if (rank == 0) return;
    const int g0 = ((int)blockIdx.x - tab.down0[si]) * p.groups, g1 = min(g0 + p.groups, (sg.n + 15) >> 4), last = sg.row + sg.n - 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int l15 = lane & 15, l4 = lane >> 4;
    const int nr = (rank + 15) >> 4;
    const int k0 = ((int)blockIdx.y * waves + wave) * (C * 32);
    const bool whole = k0 + C * 32 <= p.K;
    Frag<T> a[NR][C];                            // (ranks behind the slot's last one: that one again)
#pragma unroll
    for (int j = 0; j < NR; ++j)
        if (j < nr) {
            const T* ap = (const T*)p.a + ((int64_t)sg.slot() * p.width + min(j * 16 + l15, rank - 1)) * p.K + k0 + l4 * 8;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (whole || k0 + c * 32 + l4 * 8 < p.K) load(a[j][c], ap + c * 32);       // (K is a multiple of 8)
                else zero(a[j][c]);
            }
        }
    auto fetch = [&](Frag<T> (&x)[C], int g) {   // (rows behind the request's last one: that one again)
        const T* xp = (const T*)p.x + (int64_t)min(sg.row + g * 16 + l15, last) * p.K + k0 + l4 * 8;
        if (whole) {
#pragma unroll
            for (int c = 0; c < C; ++c) load(x[c], xp + c * 32);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (k0 + c * 32 + l4 * 8 < p.K) load(x[c], xp + c * 32);
                else zero(x[c]);
            }
        }
    };
    float* const t = p.t + (int64_t)blockIdx.y * p.plane + (int64_t)sg.group0 * 16 * p.rp;
    auto turn = [&](Frag<T> (&x)[C], int g) {
        f32x4 acc[NR];
#pragma unroll
        for (int j = 0; j < NR; ++j)
            if (j < nr) {
                acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < C; ++c) acc[j] = mma(a[j][c], x[c], acc[j]);
            }
        if (g + 2 < g1) fetch(x, g + 2);
        f32x4* const mine = red + (g & 1) * waves * (NR * 64);     // (two places in turn: one barrier a group)
#pragma unroll
        for (int j = 0; j < NR; ++j)
            if (j < nr) mine[(wave * NR + j) * 64 + lane] = acc[j];
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");         // (not for the loads that are under way)
        for (int j = wave; j < nr; j += waves) {
            f32x4 v = mine[j * 64 + lane];
            for (int w = 1; w < waves; ++w) v += mine[(w * NR + j) * 64 + lane];
            *(f32x4*)(t + (int64_t)(g * 16 + l15) * p.rp + j * 16 + 4 * l4) = v;
        }
    };
    Frag<T> x0[C], x1[C];
    fetch(x0, g0);
    if (g0 + 1 < g1) fetch(x1, g0 + 1);
    for (int g = g0; g < g1; g += 2) {
        turn(x0, g);
        if (g + 1 < g1) turn(x1, g + 1);
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

// eight values as they lie in memory
template <typename T> struct Raw;
template <> struct Raw<bf16_t> { uint4 w; };
template <> struct Raw<float> { float4 a, b; };
__device__ __forceinline__ void unpack(const Raw<bf16_t>& r, float (&v)[8]) {
    const uint32_t u[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        v[2 * c] = __uint_as_float(u[c] << 16);
        v[2 * c + 1] = __uint_as_float(u[c] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const Raw<float>& r, float (&v)[8]) {
    v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
    v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
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
    const int si = segment_of(tab.up0, tab.n, blockIdx.x);
    const Segment& sg = tab.seg[si];
    const int tile = (int)blockIdx.x - tab.up0[si];
    const int rank = sg.rank(), r0 = sg.row + tile * (16 * MR), end = sg.row + sg.n;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l15 = lane & 15, l4 = lane >> 4;
    const int ks = (rank + 31) >> 5;
    for (int f = wave; f < MR * ks; f += 4) {    // (a wavefront at a time: group f / ks, step f % ks)
        const int m = f / ks, k = f - m * ks, j0 = k * 32 + l4 * 8;
        const int group = min(tile * MR + m, (sg.n - 1) >> 4);       // (groups behind the last one: that one again)
        const float* t = p.t + ((int64_t)(sg.group0 + group) * 16 + l15) * p.rp + j0;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
        if (j0 < rank)
            for (int i0 = 0; i0 < p.pieces; i0 += 8) {               // (eight pieces' loads under way together)
                f32x4 a[8], b[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i0 + i < p.pieces) {
                        a[i] = *(const f32x4*)(t + (i0 + i) * p.plane);
                        b[i] = *(const f32x4*)(t + (i0 + i) * p.plane + 4);
                    }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i0 + i < p.pieces) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            v[e] += a[i][e];
                            v[4 + e] += b[i][e];
                        }
                    }
            }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = j0 + e < rank ? v[e] * sg.scale : 0.f;
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
    const T* b = (const T*)p.b + (int64_t)sg.slot() * p.N * p.width;
    const int share = p.cols >> 2, first = blockIdx.y * p.cols + wave * share, n1 = min(first + share, p.N);
    for (int c0 = first; c0 < n1; c0 += 64) {
        Raw<T> out[MR][2];
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int row = r0 + m * 16 + l15, col = c0 + q * 32 + l4 * 8;
                if (p.res && row < end && col < n1) out[m][q] = *(const Raw<T>*)((const T*)p.res + (int64_t)row * p.N + col);
                else out[m][q] = Raw<T>{};
            }
        f32x4 acc[MR][4];
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int h = 0; h < 4; ++h) acc[m][h] = f32x4{0.f, 0.f, 0.f, 0.f};
        Frag<T> w[4][KS];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            const T* bp = b + (int64_t)min(c0 + (h >> 1) * 32 + (l15 >> 2) * 8 + (h & 1) * 4 + (l15 & 3), p.N - 1) * p.width + l4 * 8;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int left = rank - k * 32 - l4 * 8;
                if (left > 0) load(w[h][k], bp + k * 32);            // (width is a multiple of 8)
                else zero(w[h][k]);
            }
        }
        if (rank & 7) {
#pragma unroll
            for (int h = 0; h < 4; ++h)
#pragma unroll
                for (int k = 0; k < KS; ++k) keep(w[h][k], rank - k * 32 - l4 * 8);
        }
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int k = 0; k < KS; ++k)
                if (k < ks) {
#pragma unroll
                    for (int m = 0; m < MR; ++m)
#pragma unroll
                        for (int i = NP - 1; i >= 0; --i) acc[m][h] = mma(w[h][k], t[m][k][i], acc[m][h]);
                }
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int row = r0 + m * 16 + l15, col = c0 + q * 32 + l4 * 8;
                float v[8];
                unpack(out[m][q], v);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] += acc[m][2 * q][e];
                    v[4 + e] += acc[m][2 * q + 1][e];
                }
                if (row < end && col < n1) store_out((T*)p.c + (int64_t)row * p.N + col, v);
            }
    }
}

struct Launch {
    Table tab;
    int rank, mr, nr, groups, cols;
    int total;                 // groups of 16 rows
};

inline int down_steps(int nr, int esz) { return (nr == 8 ? 4 : 8) * 2 / esz; }
inline int k_slices(int nr, int esz, int K) { return (K + 32 * down_steps(nr, esz) - 1) / (32 * down_steps(nr, esz)); }
inline int k_pieces(int nr, int esz, int K) { return (k_slices(nr, esz, K) + DOWN_WAVES - 1) / DOWN_WAVES; }

// tiles and columns of a launch
void plan(Launch& l, int esz, int N, int K) {
    Table& t = l.tab;
    int longest = 0;
    l.rank = l.total = 0;
    for (int i = 0; i < t.n; ++i) {
        l.rank = std::max(l.rank, t.seg[i].rank());
        longest = std::max(longest, t.seg[i].n);
        t.seg[i].group0 = l.total;
        l.total += (t.seg[i].n + 15) / 16;
    }
    l.nr = l.rank <= 16 ? 1 : l.rank <= 32 ? 2 : l.rank <= 64 ? 4 : 8;
    l.mr = longest <= 16 ? 1 : l.nr == 8 ? 2 : 4;
    l.groups = std::max(1, std::min(16, l.total * k_pieces(l.nr, esz, K) / 512));
    t.down0[0] = t.up0[0] = 0;
    for (int i = 0; i < t.n; ++i) {
        const int g = (t.seg[i].n + 15) / 16;
        t.down0[i + 1] = t.down0[i] + (g + l.groups - 1) / l.groups;
        t.up0[i + 1] = t.up0[i] + (g + l.mr - 1) / l.mr;
    }
    l.cols = 1024;
    while (l.cols > 256 && (int64_t)t.up0[t.n] * ((N + l.cols - 1) / l.cols) < 1024) l.cols /= 2;
}
size_t floats_of(const Launch& l, int esz, int K) { return l.rank ? (size_t)k_pieces(l.nr, esz, K) * l.total * 16 * (16 * l.nr) : 0; }

// calls f(Launch&) for every launch's table of requests, tiles counted
template <typename F>
void for_launches(const int32_t* ranks, const float* scales, bool in_place, int esz, int64_t rows, int N, int K, const po_adapter_rows* seg, int n_seg, F f) {
    Launch l;
    Table& tab = l.tab;
    tab.n = 0;
    auto flush = [&]() {
        if (tab.n) {
            plan(l, esz, N, K);
            f(l);
        }
        tab.n = 0;
    };
    auto add = [&](int64_t row, int64_t n, int slot) {
        const int rank = slot < 0 ? 0 : ranks[slot];
        if (n <= 0 || (rank == 0 && in_place)) return;         // (nothing to do: the rows stay as they are)
        Segment* last = tab.n ? &tab.seg[tab.n - 1] : nullptr;
        if (last && last->row + last->n == row && last->rank() == rank && (rank == 0 || last->slot() == slot)) {       // one run of rows
            last->n += (int)n;
            return;
        }
        if (tab.n == MAX_SEGMENTS) flush();
        tab.seg[tab.n++] = {(int)row, (int)n, rank ? slot * 256 + rank : 0, rank && scales ? scales[slot] : 0.f, 0};
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
    if (l.rank) {
        constexpr int LDS = 2 * DOWN_WAVES * NR * 64 * 16;
        static OncePerDevice once;
        if (LDS > 64 * 1024) once.run(current_device(), [] { allow_dynamic_lds((const void*)(adapter_down_kernel<T, NR>), LDS); });
        const int waves = std::min(DOWN_WAVES, k_slices(NR, sizeof(T), p.K));
        hipLaunchKernelGGL((adapter_down_kernel<T, NR>), dim3((unsigned)l.tab.down0[l.tab.n], (unsigned)p.pieces), dim3(64 * waves),
                           2 * waves * NR * 64 * 16, s, p, l.tab);
    }
    hipLaunchKernelGGL((adapter_up_kernel<T, MR, (NR + 1) / 2>), dim3((unsigned)l.tab.up0[l.tab.n], (unsigned)((p.N + p.cols - 1) / p.cols)), dim3(256), 0, s, p, l.tab);
}

template <typename T>
void run(AdapterParams p, const Launch& l, hipStream_t s) {
    p.rp = 16 * l.nr;
    p.pieces = k_pieces(l.nr, sizeof(T), p.K);
    p.plane = (int64_t)l.total * 16 * p.rp;
    p.groups = l.groups;
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

size_t adapters_scratch(int dtype, const int32_t* ranks, int64_t rows, int N, int K, const po_adapter_rows* seg, int n_seg) {
    size_t most = 0;
    const int esz = dtype == 0 ? 4 : 2;
    // (in place or not changes the tables of launches: the larger of both)
    for (const bool in_place : {false, true})
        for_launches(ranks, nullptr, in_place, esz, rows, N, K, seg, n_seg, [&](const Launch& l) { most = std::max(most, floats_of(l, esz, K)); });
    return most * sizeof(float);
}

void launch_adapters(int dtype, const void* x, const void* a, const void* b, const int32_t* ranks, const float* scales, int width, const void* res,
                     void* c, int64_t rows, int N, int K, const po_adapter_rows* seg, int n_seg, float* t, hipStream_t s) {
    AdapterParams p;
    memset(&p, 0, sizeof(p));
    p.x = x; p.a = a; p.b = b; p.res = res; p.c = c; p.t = t;
    p.N = N; p.K = K; p.width = width;
    for_launches(ranks, scales, res == c, dtype == 0 ? 4 : 2, rows, N, K, seg, n_seg, [&](const Launch& l) {
        if (dtype == 0) run<float>(p, l, s);
        else run<bf16_t>(p, l, s);
    });
}

}  // namespace po
