// Low-rank adapters of many requests at once, beside a shared projection (gfx950).
//
//   C[r] = R[r] + scale_a T[r] B_a^T,  T[r] = x[r] A_a^T,    A_a [rank, K], B_a [N, rank]: the adapter a of the request that row r belongs to
//
// Adapters lie in slots of a pool, A [slots][width][K] and B [slots][N][width].  First T, in pieces of K, each a plane of float32 sums in scratch.
// Then C: of requests of up to 16 rows by wavefronts that add the planes themselves; of longer ones from T joined to the matrix instruction's
// fragments by a launch of its own.  A request's rows multiply with its slot alone, so a batch costs the bytes of its rows and of the
// slots that it uses, and memory bounds it.
#include "adapters.h"
#include "slice_window.h"

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
    int down0[MAX_SEGMENTS + 1], up0[MAX_SEGMENTS + 1];        // first run of rows of each request in the first launch and in the last one, and their number
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
    int groups, up_groups;     // of 16 rows that a workgroup of the first launch and of the last one takes
    void* frags;               // T as fragments, of ks steps each
    int ks;
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
// from a row in LDS, whose 16-byte segments are XOR-swizzled with the row
__device__ __forceinline__ void load(Frag<bf16_t>& f, const unsigned char* row, int at, int swizzle) {
    f.v = *(const bf16x8*)(row + ((at ^ swizzle) << 4));
}
__device__ __forceinline__ void load(Frag<float>& f, const unsigned char* row, int at, int swizzle) {
    f.lo = *(const f32x4*)(row + (((2 * at) ^ swizzle) << 4));
    f.hi = *(const f32x4*)(row + (((2 * at + 1) ^ swizzle) << 4));
}
// 16 bytes of a fragment
typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
__device__ __forceinline__ void set(Frag<bf16_t>& f, int, const u32x4& v) { f.v = __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ void set(Frag<float>& f, int q, const u32x4& v) { (q ? f.hi : f.lo) = __builtin_bit_cast(f32x4, v); }
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

// T of a run of rows of one request over one piece of K, 16 rows at a time.  A wavefront takes C steps of 32 of the piece, 512 bytes of a row
// (256 with ranks beyond 64), and holds that part of A in registers for all its rows: A is read once a run.  x goes straight into a ring of D
// groups of rows in LDS, a load covering whole lines of two rows (four); 16-byte segments are XOR-swizzled with the row on the global side, so
// that a fragment's 16 rows meet 16 different banks.  The wavefronts' sums meet in LDS.  A lane of a product of 16 ranks and 16 rows holds row
// lane & 15 and ranks 4 (lane >> 4) .. + 3.
// What bounds it: x from memory.  16584 rows of K 14336, rank 64, 99 us (4.8 TB/s; 120 where x passes through the caches, ONCE false); the
// fragments straight from memory to registers, 64 bytes of a line each, 161 where this took 149 (runs of rows of another length).  7394 rows of K 4096 in 41 requests 26: one round of workgroups, each of which waits for A first.  64 single tokens 7.4.
// (LDS is read as vectors of bf16 or float: as uint4 the compiler, which cannot tell them from what the loads write, waits for all loads.)
constexpr int DOWN_WAVES = 8;
template <typename T, int NR> struct Down {
    static constexpr int ROWB = NR == 8 ? 256 : 512;             // bytes of a row that a wavefront takes
    static constexpr int C = ROWB / 32 / (int)sizeof(T);         // steps
    static constexpr int GROUP = 16 * ROWB, NL = GROUP / 1024;   // bytes of a group, and its loads
    static constexpr int D = NR == 8 ? 3 : 2;
    static constexpr int WAVE = D * GROUP + NR * 1024;           // LDS of a wavefront: the ring, and its sums
    static_assert(DOWN_WAVES * WAVE <= 160 * 1024, "LDS of a compute unit");
};

template <typename T, int NR, bool ONCE>
__global__ void __launch_bounds__(64 * DOWN_WAVES, 2) adapter_down_kernel(const AdapterParams p, const Table tab) {
    typedef Down<T, NR> L;
    constexpr int C = L::C, D = L::D, ROWB = L::ROWB, SEGS = ROWB / 16, RPL = 1024 / ROWB;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int si = segment_of(tab.down0, tab.n, blockIdx.x);
    const Segment& sg = tab.seg[si];
    const int rank = sg.rank();
    if (rank == 0) return;
    const int g0 = ((int)blockIdx.x - tab.down0[si]) * p.groups, g1 = min(g0 + p.groups, (sg.n + 15) >> 4);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int l15 = lane & 15, l4 = lane >> 4;
    const int nr = (rank + 15) >> 4;
    const int k0 = ((int)blockIdx.y * waves + wave) * (C * 32);
    const int ks = min(p.K - k0, C * 32);        // elements of K of this wavefront (none: 0 or less)
    unsigned char* const ring = smem + wave * L::WAVE;
    f32x4* const red = (f32x4*)(ring + D * L::GROUP);

    // loads of a group: rows behind the request's last one read as zero, what lies behind K in a row is dropped with the fragments
    const uint32_t pitch = (uint32_t)p.K * (uint32_t)sizeof(T);
    uint32_t vo[8];                              // (NL entries used)
#pragma unroll
    for (int i = 0; i < L::NL; ++i) {
        const int row = i * RPL + lane / SEGS;
        vo[i] = (uint32_t)row * pitch + (uint32_t)(((lane & (SEGS - 1)) ^ row) << 4);
    }
    const unsigned char* const xbase = (const unsigned char*)p.x + ((int64_t)sg.row * p.K + k0) * (int64_t)sizeof(T);
#define PO_FETCH(g_, pos_)                                                                                             \
    {                                                                                                                  \
        const int at_ = (g_), rows_ = at_ < g1 ? min(16, sg.n - at_ * 16) : 0;                                         \
        const uint32_t bytes_ = rows_ > 0 && ks > 0 ? (uint32_t)(rows_ - 1) * pitch + (uint32_t)ks * (uint32_t)sizeof(T) : 0u; \
        const __amdgpu_buffer_rsrc_t rs_ = __builtin_amdgcn_make_buffer_rsrc(                                          \
            (void*)(xbase + (int64_t)(bytes_ ? at_ : g0) * 16 * pitch), 0, (int)bytes_, 0x00020000);                   \
        _Pragma("unroll") for (int i = 0; i < L::NL; ++i)                                                              \
            __builtin_amdgcn_raw_ptr_buffer_load_lds(                                                                  \
                rs_, (__attribute__((address_space(3))) void*)(ring + (pos_) * L::GROUP + i * 1024), 16, vo[i], 0, 0, ONCE ? LOAD_ONCE : 0); \
    }
#pragma unroll
    for (int d = 0; d < D; ++d) PO_FETCH(g0 + d, d)
    Frag<T> a[NR][C];                            // (ranks behind the slot's last one: that one again)
#pragma unroll
    for (int j = 0; j < NR; ++j)
        if (j < nr) {
            const T* ap = (const T*)p.a + ((int64_t)sg.slot() * p.width + min(j * 16 + l15, rank - 1)) * p.K + k0 + l4 * 8;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (c * 32 + l4 * 8 < ks) load(a[j][c], ap + c * 32);          // (K is a multiple of 8)
                else zero(a[j][c]);
            }
        }
    // (A is here before the loop: from then on the counter of loads counts the ring's alone, and at the end of a turn a store)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    float* const t = p.t + (int64_t)blockIdx.y * p.plane + (int64_t)sg.group0 * 16 * p.rp;
    int pos = 0;
    for (int g = g0; g < g1; ++g) {
        PO_WAIT_LOADS((D - 1) * L::NL);            // the group has landed (loads return in order)
        Frag<T> x[C];
        const unsigned char* const u = ring + pos * L::GROUP + l15 * ROWB;
#pragma unroll
        for (int c = 0; c < C; ++c) load(x[c], u, c * 4 + l4, l15);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                     // (every fragment is in registers: the place is free)
        PO_FETCH(g + D, pos)
        pos = pos + 1 == D ? 0 : pos + 1;
        if (ks < C * 32) {
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (c * 32 + l4 * 8 >= ks) zero(x[c]);
        }
        f32x4 acc[NR];
#pragma unroll
        for (int j = 0; j < NR; ++j)
            if (j < nr) {
                acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < C; ++c) acc[j] = mma(a[j][c], x[c], acc[j]);
            }
        asm volatile("s_barrier" ::: "memory");                                // (the sums of the group before have been read)
#pragma unroll
        for (int j = 0; j < NR; ++j)
            if (j < nr) red[j * 64 + lane] = acc[j];
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");         // (not for the loads that are under way)
        for (int j = wave; j < nr; j += waves) {
            f32x4 v = *(const f32x4*)(smem + D * L::GROUP + (j * 64 + lane) * 16);
            for (int w = 1; w < waves; ++w) v += *(const f32x4*)(smem + w * L::WAVE + D * L::GROUP + (j * 64 + lane) * 16);
            *(f32x4*)(t + (int64_t)(g * 16 + l15) * p.rp + j * 16 + 4 * l4) = v;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
#undef PO_FETCH
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // (nothing is on its way into LDS when the workgroup ends)
}

// The fragments of T in the second product: float32 whole, in bf16 three numbers, whose sum T is (each takes the upper 8 bits of what the ones
// before left, cut, not rounded: T up to the largest number has none above it; what lies below the smallest bf16 number is lost).  Two of them would leave 2^-16 of T out, which shows where the residual takes the rest away, for
// 2 % of the time of the whole call with rank 64 (posts 64 / 66 us) and 5 % with 128 (two prompts of 4000 rows 81 / 85).
template <typename T> struct Parts;
template <> struct Parts<bf16_t> { static constexpr int N = 3; };
template <> struct Parts<float> { static constexpr int N = 1; };
__device__ __forceinline__ void split(const float (&v)[8], Frag<bf16_t> (&f)[3]) {
    float left[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) left[e] = v[e];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t a = __float_as_uint(left[2 * c]) & 0xffff0000u, b = __float_as_uint(left[2 * c + 1]) & 0xffff0000u;
            w[c] = a >> 16 | b;
            left[2 * c] -= __uint_as_float(a);
            left[2 * c + 1] -= __uint_as_float(b);
        }
        f[i].v = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
    }
}
__device__ __forceinline__ void split(const float (&v)[8], Frag<float> (&f)[1]) {
    f[0].lo = f32x4{v[0], v[1], v[2], v[3]};
    f[0].hi = f32x4{v[4], v[5], v[6], v[7]};
}

// 16 bytes of a row of C or R
__device__ __forceinline__ void unpack(const uint4& w, float (&v)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        v[2 * c] = __uint_as_float(u[c] << 16);
        v[2 * c + 1] = __uint_as_float(u[c] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4& w, float (&v)[4]) {
    v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ uint4 pack(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = (uint32_t)f2bf(v[2 * c]) | ((uint32_t)f2bf(v[2 * c + 1]) << 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}

// What both kernels of the second launch do with 16 rows x 64 columns: the products of 16 columns each leave a lane with four of them of row lane & 15;
// they pass through 4 KiB of LDS of the wavefront's own (16-byte groups XOR-swizzled with the row), so that R is read and C written in whole lines.
// R and C go by the rows' own bounds, B by its slot's: what lies behind their ends reads as zero and is not written, and so does what a lane's offset
// is moved out of bounds for.  Whole offsets are the lane's (a scalar offset may not count in the check of bounds).
template <typename T> struct Out {
    static constexpr int E = (int)sizeof(T), V = 16 / E, LPR = 64 / V, RPP = 64 / LPR, PASSES = 16 / RPP;      // of 16 bytes; lanes of a row; rows of a pass
};
constexpr uint32_t NONE = 0x80000000u;

// what the sums onto R start with: for rows without an adapter the zero that leaves R's sign alone
__device__ __forceinline__ f32x4 nothing(int rank) {
    const float z = rank ? 0.f : -0.f;
    return f32x4{z, z, z, z};
}

template <typename T>
__device__ __forceinline__ void add_out(const f32x4 (&acc)[4], const u32x4 (&r)[Out<T>::PASSES], unsigned char* stg, __amdgpu_buffer_rsrc_t rc, uint32_t vo,
                                        uint32_t pitch, int lane) {
    typedef Out<T> O;
    const int l15 = lane & 15, l4 = lane >> 4;
#pragma unroll
    for (int h = 0; h < 4; ++h) *(f32x4*)(stg + l15 * 256 + (((h * 4 + l4) ^ l15) << 4)) = acc[h];
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < O::PASSES; ++i) {
        const int rl = i * O::RPP + lane / O::LPR;
        float v[O::V];
        unpack(__builtin_bit_cast(uint4, r[i]), v);
#pragma unroll
        for (int q = 0; q < O::V / 4; ++q) {
            const f32x4 d = *(const f32x4*)(stg + rl * 256 + ((((lane & (O::LPR - 1)) * (O::V / 4) + q) ^ rl) << 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[q * 4 + e] += d[e];
        }
        // (no scalar offset: with one the compiler takes a store's registers as free at once, and the next instruction overwrote
        // the first of them before the last lanes were read)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, pack(v)), rc, vo + (uint32_t)(i * O::RPP) * pitch, 0, 0);
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

// the sum of the planes of T at a lane's eight ranks, times the scale; 0 behind the rank
__device__ __forceinline__ void sum_planes(const AdapterParams& p, const float* t, int j0, int rank, float scale, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    if (j0 < rank)
        for (int i0 = 0; i0 < p.pieces; i0 += 8) {         // (eight pieces' loads under way together)
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
    for (int e = 0; e < 8; ++e) v[e] = j0 + e < rank ? v[e] * scale : 0.f;
}

// C of up to 16 rows of a request and 64 columns a wavefront, for batches of requests of up to 16 rows: every wavefront adds the planes of T itself.
// Its loads are all under way together: this is what a single token waits for (64 of them, N 4096, rank 16: 5.5 us; by the two kernels below
// 3.2 + 6.2).
template <typename T, int KS>
__global__ void __launch_bounds__(256) adapter_up_few_kernel(const AdapterParams p, const Table tab) {
    typedef Out<T> O;
    constexpr int NP = Parts<T>::N, E = O::E;
    __shared__ __attribute__((aligned(16))) unsigned char stage[4][4096];
    const int chunks = (p.N + 255) / 256, si = (int)(blockIdx.x / (unsigned)chunks);       // (a tile is a request)
    const Segment& sg = tab.seg[si];
    const int rank = sg.rank(), lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15, l4 = lane >> 4;
    const int c0 = ((int)blockIdx.x - si * chunks) * 256 + wave * 64;
    if (c0 >= p.N) return;
    const uint32_t pitch = (uint32_t)p.N * E, bytes = (uint32_t)sg.n * pitch;
    const int64_t at = (int64_t)sg.row * p.N * E;
    const __amdgpu_buffer_rsrc_t rr = __builtin_amdgcn_make_buffer_rsrc((void*)((const unsigned char*)(p.res ? p.res : p.c) + at), 0, p.res ? (int)bytes : 0, 0x00020000);
    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc((void*)((unsigned char*)p.c + at), 0, (int)bytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(
        (void*)((const unsigned char*)p.b + (int64_t)sg.slot() * p.N * p.width * E), 0, (int)((uint32_t)p.N * (uint32_t)p.width * E), 0x00020000);
    Frag<T> w[4][KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        const uint32_t vb = rank - k * 32 - l4 * 8 > 0 ? (uint32_t)(l15 * p.width + k * 32 + l4 * 8) * E : NONE;
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int q = 0; q < E / 2; ++q)
                set(w[h][k], q, __builtin_amdgcn_raw_buffer_load_b128(rb, vb + (uint32_t)(c0 + h * 16) * (uint32_t)p.width * E + q * 16, 0, 0));
    }
    const uint32_t vo = c0 + (lane & (O::LPR - 1)) * O::V < p.N ? (uint32_t)(lane / O::LPR) * pitch + (uint32_t)(lane & (O::LPR - 1)) * 16u + (uint32_t)c0 * E : NONE;
    u32x4 r[O::PASSES];
#pragma unroll
    for (int i = 0; i < O::PASSES; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b128(rr, vo + (uint32_t)(i * O::RPP) * pitch, 0, 0);
    f32x4 acc[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) acc[h] = nothing(rank);
#pragma unroll
    for (int k = 0; k < KS; ++k)
        if (k * 32 < rank) {
            const int j0 = k * 32 + l4 * 8;
            float v[8];
            sum_planes(p, p.t + ((int64_t)sg.group0 * 16 + l15) * p.rp + j0, j0, rank, sg.scale, v);
            Frag<T> t[NP];
            split(v, t);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                if (rank & 7) keep(w[h][k], rank - j0);
#pragma unroll
                for (int i = NP - 1; i >= 0; --i) acc[h] = mma(w[h][k], t[i], acc[h]);
            }
        }
    add_out<T>(acc, r, stage[wave], rc, vo, pitch, lane);
}

// Longer requests: first T as the second product's fragments, in the order of its lanes: [group][step][part][lane] (in scratch behind the planes;
// 16584 rows, rank 64, seven planes: 10 us) ...
template <typename T>
__global__ void __launch_bounds__(256) adapter_join_kernel(const AdapterParams p, const Table tab) {
    constexpr int NP = Parts<T>::N;
    const int si = segment_of(tab.up0, tab.n, blockIdx.x);
    const Segment& sg = tab.seg[si];
    const int rank = sg.rank(), ks = (rank + 31) >> 5, lane = threadIdx.x & 63, l15 = lane & 15, l4 = lane >> 4;
    const int g0 = ((int)blockIdx.x - tab.up0[si]) * p.up_groups, g1 = min(g0 + p.up_groups, (sg.n + 15) >> 4);
    const int f = (int)blockIdx.y * 4 + (threadIdx.x >> 6);        // (a wavefront per group and step)
    if (f >= (g1 - g0) * ks) return;
    const int g = g0 + f / ks, k = f % ks, j0 = k * 32 + l4 * 8;
    float v[8];
    sum_planes(p, p.t + ((int64_t)(sg.group0 + g) * 16 + l15) * p.rp + j0, j0, rank, sg.scale, v);
    Frag<T> part[NP];
    split(v, part);
    Frag<T>* o = (Frag<T>*)p.frags + (((int64_t)(sg.group0 + g) * p.ks + k) * NP) * 64 + lane;
#pragma unroll
    for (int i = 0; i < NP; ++i) o[i * 64] = part[i];
}

// ... then C of a run of rows of one request and 4 x 16 H columns, a quarter a wavefront, which holds its part of B in registers for all of
// them: B is read once a run.  16 rows at a time, the next ones' R and T on their way; wavefronts wait for nobody.  What bounds it: R and C,
// 16584 x 4096 with rank 64 65 us (4.2 TB/s; a copy of as many bytes 46).  Tiles of 64 rows x 1024 columns that read B and the planes of T
// anew took 89: what a compute unit can have under way towards it is the limit there, and reads that caches answer take their places in it.
template <typename T, int KS> struct UpCols {
    static constexpr int H = 32 / (int)sizeof(T) / (KS == 1 ? 1 : KS / 2);              // 128 registers of B (64 with one step)
};
template <typename T, int KS>
__global__ void __launch_bounds__(256, 2) adapter_up_kernel(const AdapterParams p, const Table tab) {
    typedef Out<T> O;
    constexpr int NP = Parts<T>::N, E = O::E, H = UpCols<T, KS>::H, SUB = H / 4;          // SUB: 64 columns each
    __shared__ __attribute__((aligned(16))) unsigned char stage[4][4096];
    // (a run's workgroups side by side: those that run together cover whole rows)
    const int chunks = (p.N + 64 * H - 1) / (64 * H), at = (int)(blockIdx.x / (unsigned)chunks);
    const int si = segment_of(tab.up0, tab.n, at);
    const Segment& sg = tab.seg[si];
    const int rank = sg.rank(), ks = (rank + 31) >> 5;
    const int g0 = (at - tab.up0[si]) * p.up_groups, g1 = min(g0 + p.up_groups, (sg.n + 15) >> 4);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l15 = lane & 15, l4 = lane >> 4;
    const int c0 = ((int)blockIdx.x - at * chunks) * (64 * H) + wave * (16 * H);
    if (c0 >= p.N) return;
    const uint32_t pitch = (uint32_t)p.N * E;
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(
        (void*)((const unsigned char*)p.b + (int64_t)sg.slot() * p.N * p.width * E), 0, (int)((uint32_t)p.N * (uint32_t)p.width * E), 0x00020000);
    Frag<T> w[H][KS];
#pragma unroll
    for (int k = 0; k < KS; ++k) {
        const uint32_t vb = rank - k * 32 - l4 * 8 > 0 ? (uint32_t)(l15 * p.width + k * 32 + l4 * 8) * E : NONE;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int q = 0; q < E / 2; ++q)
                set(w[h][k], q, __builtin_amdgcn_raw_buffer_load_b128(rb, vb + (uint32_t)(c0 + h * 16) * (uint32_t)p.width * E + q * 16, 0, 0));
    }
    if (rank & 7) {
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int k = 0; k < KS; ++k) keep(w[h][k], rank - k * 32 - l4 * 8);
    }
    const uint32_t vr = (uint32_t)(lane / O::LPR) * pitch + (uint32_t)(lane & (O::LPR - 1)) * 16u + (uint32_t)c0 * E;
    uint32_t vo[SUB];
#pragma unroll
    for (int b = 0; b < SUB; ++b) vo[b] = c0 + b * 64 + (lane & (O::LPR - 1)) * O::V < p.N ? vr + b * 64 * E : NONE;
    const Frag<T>* const frags = (const Frag<T>*)p.frags + (int64_t)sg.group0 * p.ks * NP * 64 + lane;
    u32x4 r[SUB][O::PASSES];
    auto fetch_t = [&](Frag<T> (&t)[KS][NP], int g) {
#pragma unroll
        for (int k = 0; k < KS; ++k)
            if (k < ks) {
#pragma unroll
                for (int i = 0; i < NP; ++i) t[k][i] = frags[(((int64_t)g * p.ks + k) * NP + i) * 64];
            }
    };
    auto fetch_r = [&](int b, int g) {
        const __amdgpu_buffer_rsrc_t rr = __builtin_amdgcn_make_buffer_rsrc((void*)((const unsigned char*)(p.res ? p.res : p.c) + (int64_t)(sg.row + g * 16) * pitch), 0,
                                                                            p.res ? (int)((uint32_t)min(16, sg.n - g * 16) * pitch) : 0, 0x00020000);
#pragma unroll
        for (int i = 0; i < O::PASSES; ++i) r[b][i] = __builtin_amdgcn_raw_buffer_load_b128(rr, vo[b] + (uint32_t)(i * O::RPP) * pitch, 0, 0);
    };
    // (the next rows' R go where this one's are no longer needed: B, two of these and of T do not fit the registers; nor does another T of twelve
    // fragments, with which two prompts of 4000 rows and rank 128 took 121 us instead of 85)
    constexpr bool AHEAD = NP * KS < 12;
    auto turn = [&](Frag<T> (&t)[KS][NP], Frag<T> (&next)[KS][NP], int g) {
        const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc((void*)((unsigned char*)p.c + (int64_t)(sg.row + g * 16) * pitch), 0,
                                                                            (int)((uint32_t)min(16, sg.n - g * 16) * pitch), 0x00020000);
        const bool more = g + 1 < g1;
        if (AHEAD && more) fetch_t(next, g + 1);
#pragma unroll
        for (int b = 0; b < SUB; ++b) {
            f32x4 acc[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) acc[h] = nothing(rank);
#pragma unroll
            for (int k = 0; k < KS; ++k)
                if (k < ks) {
#pragma unroll
                    for (int i = NP - 1; i >= 0; --i)
#pragma unroll
                        for (int h = 0; h < 4; ++h) acc[h] = mma(w[b * 4 + h][k], t[k][i], acc[h]);
                }
            if (!AHEAD && b == SUB - 1 && more) fetch_t(t, g + 1);
            add_out<T>(acc, r[b], stage[wave], rc, vo[b], pitch, lane);
            if (more) fetch_r(b, g + 1);
        }
    };
    Frag<T> t0[KS][NP], t1[KS][NP];
    fetch_t(t0, g0);
#pragma unroll
    for (int b = 0; b < SUB; ++b) fetch_r(b, g0);
    for (int g = g0; g < g1; g += 2) {
        turn(t0, t1, g);
        if (g + 1 < g1) turn(AHEAD ? t1 : t0, t0, g + 1);
    }
}

struct Launch {
    Table tab;
    int rank, nr, groups, up_groups;
    bool few;                  // requests of up to 16 rows
    int total;                 // groups of 16 rows
};

inline int k_slices(int nr, int esz, int K) {                    // of a wavefront each
    const int k = (nr == 8 ? 256 : 512) / esz;
    return (K + k - 1) / k;
}
inline int k_pieces(int nr, int esz, int K) { return (k_slices(nr, esz, K) + DOWN_WAVES - 1) / DOWN_WAVES; }

inline int nr_of(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8; }

constexpr int ks_of(int nr) { return (nr + 1) / 2; }
inline int up_h(int nr, int esz) { return 32 / esz / (nr <= 2 ? 1 : ks_of(nr) / 2); }

// runs of rows of a launch
void plan(Launch& l, int esz, int N, int K) {
    Table& t = l.tab;
    int longest = 0;
    l.rank = l.total = 0;
    for (int i = 0; i < t.n; ++i) {
        l.rank = std::max(l.rank, t.seg[i].rank());
        longest = std::max(longest, t.seg[i].n);
        t.seg[i].group0 = l.total;
        if (t.seg[i].rank()) l.total += (t.seg[i].n + 15) / 16;
    }
    l.nr = nr_of(l.rank);
    l.few = longest <= 16;
    // Rows of a workgroup: rounds of workgroups, one a compute unit in the first launch and two in the last, each with the time of its groups
    // and of two more for A, or one for B.  On eight batches, every number of groups from 1 to 64 timed for either launch, the whole
    // call is within 8 % of the fastest (two prompts of 8000 rows, K 14336, rank 64: 32 groups 200 us, 28 246, 8 219, 1 409).
    const int pieces = k_pieces(l.nr, esz, K), most = (longest + 15) / 16, chunks = (N + 64 * up_h(l.nr, esz) - 1) / (64 * up_h(l.nr, esz));
    auto run = [&](bool down, int wide, int slots, int more) {
        int64_t best = INT64_MAX;
        int pick = 1;
        for (int g : {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32, 40, 48, 56, 64}) {
            int64_t wgs = 0;
            for (int i = 0; i < t.n; ++i)
                if (!down || t.seg[i].rank()) wgs += ((t.seg[i].n + 15) / 16 + g - 1) / g;
            const int64_t time = (wgs * wide + slots - 1) / slots * (std::min(g, most) + more);
            if (time < best) {
                best = time;
                pick = g;
            }
            if (g >= most) break;
        }
        return pick;
    };
    l.groups = l.few ? 1 : run(true, pieces, 256, 2);
    l.up_groups = l.few ? 1 : run(false, chunks, 512, 1);
    t.down0[0] = t.up0[0] = 0;
    for (int i = 0; i < t.n; ++i) {
        const int g = (t.seg[i].n + 15) / 16;
        t.down0[i + 1] = t.down0[i] + (g + l.groups - 1) / l.groups;
        t.up0[i + 1] = t.up0[i] + (g + l.up_groups - 1) / l.up_groups;
    }
}

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

template <typename T, int NR, bool ONCE>
void run_down(const AdapterParams& p, const Launch& l, hipStream_t s) {
    constexpr int WAVE = Down<T, NR>::WAVE;
    static OncePerDevice once;
    once.run(current_device(), [] { allow_dynamic_lds((const void*)(adapter_down_kernel<T, NR, ONCE>), DOWN_WAVES * WAVE); });
    const int waves = std::min(DOWN_WAVES, k_slices(NR, sizeof(T), p.K));
    hipLaunchKernelGGL((adapter_down_kernel<T, NR, ONCE>), dim3((unsigned)l.tab.down0[l.tab.n], (unsigned)p.pieces), dim3(64 * waves), waves * WAVE, s, p, l.tab);
}

template <typename T, int NR>
void run_t(const AdapterParams& p, const Launch& l, hipStream_t s) {
    constexpr int KS = ks_of(NR), H = UpCols<T, KS>::H;
    if (l.rank) {
        // (x past the caches / not, us.  K 14336, N 4096, rank 64, the whole call: 2000 rows 42 / 41, 8000 86 / 104, 16000 157 / 178.  Of far more columns
        // than K, x just written by the norm, whose time is in it, K 4096, N 28672, rank 64: 2300 rows 88 / 91, 4000 138 / 137, 9000 272 / 276)
        if ((int64_t)l.total * 16 * ((int64_t)p.K + 2 * p.N) * (int64_t)sizeof(T) >= READ_ONCE_BYTES) run_down<T, NR, true>(p, l, s);
        else run_down<T, NR, false>(p, l, s);
    }
    if (l.few) {
        hipLaunchKernelGGL((adapter_up_few_kernel<T, KS>), dim3((unsigned)l.tab.n * (unsigned)((p.N + 255) / 256)), dim3(256), 0, s, p, l.tab);
        return;
    }
    const unsigned runs = (unsigned)l.tab.up0[l.tab.n];
    if (l.rank) hipLaunchKernelGGL((adapter_join_kernel<T>), dim3(runs, (unsigned)((l.up_groups * KS + 3) / 4)), dim3(256), 0, s, p, l.tab);
    hipLaunchKernelGGL((adapter_up_kernel<T, KS>), dim3(runs * (unsigned)((p.N + 64 * H - 1) / (64 * H))), dim3(256), 0, s, p, l.tab);
}

template <typename T>
void run(AdapterParams p, const Launch& l, hipStream_t s) {
    p.rp = 16 * l.nr;
    p.pieces = k_pieces(l.nr, sizeof(T), p.K);
    p.plane = (int64_t)l.total * 16 * p.rp;
    p.groups = l.groups;
    p.up_groups = l.up_groups;
    p.ks = ks_of(l.nr);
    p.frags = p.t + p.pieces * p.plane;
    switch (l.nr) {
        case 1: run_t<T, 1>(p, l, s); break;
        case 2: run_t<T, 2>(p, l, s); break;
        case 4: run_t<T, 4>(p, l, s); break;
        default: run_t<T, 8>(p, l, s); break;
    }
}

}  // namespace

// (of all requests in one launch: each of several takes less)
size_t adapters_scratch(int dtype, const int32_t* ranks, int K, const po_adapter_rows* seg, int n_seg) {
    int rank = 0;
    int64_t groups = 0;
    for (int i = 0; i < n_seg; ++i) {
        const int r = seg[i].adapter < 0 ? 0 : ranks[seg[i].adapter];
        if (r) groups += (seg[i].n_rows + 15) / 16;
        rank = std::max(rank, r);
    }
    const int nr = nr_of(rank);
    // planes of T, and T as fragments (32 ranks a step: of float32, or of three bf16 numbers)
    return rank ? (size_t)groups * 16 * ((size_t)k_pieces(nr, dtype == 0 ? 4 : 2, K) * (16 * nr) * sizeof(float) + 32 * ks_of(nr) * (dtype == 0 ? sizeof(float) : 3 * sizeof(bf16_t))) : 0;
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
