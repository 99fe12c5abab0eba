// Attention of a batch of requests behind one shared prefix, bf16 MFMA (gfx950).
//
// Row i of a request sees all n2 keys of the prefix and its own keys 0 .. kv_len - q_len + i:
//   o = sum over those keys of p v / sum of p,  p = exp(score - maximum)
// All query heads of a KV head are rows of one tile (a request of q_len positions has q_len * group of them), since they share
// their keys.  A lane owns one row: S^T = K Q^T leaves it 16 of a block's 32 keys (its partner lane ^ 32 the others), the
// softmax is per lane, and the probabilities are at once the operand of O^T += V^T P^T (K rows are read in an order that makes
// the eight keys a lane feeds to an MFMA contiguous in V^T, as in attn_mfma.hip).
#include "attn_shared.h"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace po {

typedef shared_bf16x8 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;

namespace {

__device__ __forceinline__ float other_half_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ int swz8(int row) { return (row & 7) ^ ((row >> 3) & 1); }

// 32 rows of a wavefront, a lane's column, and what has been summed for it
template <int HD>
struct Rows {
    static constexpr int KS = HD / 16, HT = HD / 32;
    bf16x8 qf[KS];
    f32x16 acc[HT];            // O^T: row 32 ht + 8 (r / 4) + 4 (lane / 32) + r % 4
    float m, l;                // maximum so far (score units, -inf: none), this lane's half of the sum

    __device__ __forceinline__ void start(const bf16_t* q, bool valid) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint4 t = make_uint4(0, 0, 0, 0);
            if (valid) t = *(const uint4*)(q + ks * 16);
            qf[ks] = __builtin_bit_cast(bf16x8, t);
        }
#pragma unroll
        for (int ht = 0; ht < HT; ++ht)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[ht][r] = 0.f;
        m = -INFINITY;
        l = 0.f;
    }

    // scores of N blocks of 32 keys -> their probabilities, as the operand of O^T += V^T P^T; see: how many of the keys this
    // lane's row sees (all of them unless `masked`)
    template <int N>
    __device__ __forceinline__ void softmax(f32x16 (&s)[N], bf16x8 (&pf)[2 * N], bool masked, int see, int lhi, float sc) {
        if (masked) {
#pragma unroll
            for (int a = 0; a < N; ++a)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (a * 32 + (r & 7) + 8 * lhi + 16 * (r >> 3) >= see) s[a][r] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int a = 0; a < N; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[a][r]);
        top = fmaxf(m, other_half_max(top));
        const float ref = top == -INFINITY ? 0.f : top * sc;      // (nothing seen yet: all probabilities come out 0)
        if (__any(top > m)) {                                     // (else every factor is 1)
            const float f = __builtin_amdgcn_exp2f(fmaf(m, sc, -ref));
            l *= f;
#pragma unroll
            for (int ht = 0; ht < HT; ++ht)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[ht][r] *= f;
            m = top;
        }
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int a = 0; a < N; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float e = __builtin_amdgcn_exp2f(fmaf(s[a][r], sc, -ref));
                sum[r & 1] += e;
                pf[2 * a + (r >> 3)][r & 7] = (__bf16)e;      // (the one rounding of a probability: the matrix instruction's operand)
            }
        l += sum[0] + sum[1];
    }
};

// o = y / l in bf16, 4 values; a row that sees nothing: 0
__device__ __forceinline__ void store4(bf16_t* o, float a, float b, float c, float d, float inv) {
    uint2 w;
    w.x = (uint32_t)f2bf(a * inv) | ((uint32_t)f2bf(b * inv) << 16);
    w.y = (uint32_t)f2bf(c * inv) | ((uint32_t)f2bf(d * inv) << 16);
    *(uint2*)o = w;
}

// 64 keys of K (rows as they are) or V^T (128 bytes of each row) of one KV head in LDS, 16-byte segments swizzled with the row; the
// loads (1 KB each) by whole cache lines past the registers, the swizzle on the global side.  Loads j0 .. j0 + N.
// n: keys of it that there are (<= 0: nothing is read, though as many loads are on their way).  K rows from n on read as 0; V^T
// columns from there on hold anything, the last row's up to the eight that hold the last key.
template <int HD, int N>
__device__ __forceinline__ void dma_k_tile(unsigned char* lds, const bf16_t* k, int64_t krs, int n, int lane, int j0) {
    constexpr int LPR = HD / 8;                                 // lanes (16 bytes each) of a row
    n = min(n, 64);
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc((void*)k, 0, n > 0 ? (int)((uint32_t)(n - 1) * (uint32_t)(krs * 2) + HD * 2) : 0, 0x00020000);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int row = (j0 + j) * (64 / LPR) + lane / LPR, seg = lane % LPR;
        const int sw = LPR == 16 ? seg ^ (row & 15) : seg ^ swz8(row);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (j0 + j) * 1024), 16,
                                                 (uint32_t)row * (uint32_t)(krs * 2) + (uint32_t)(sw << 4), 0, 0, 0);
    }
}
template <int HD, int N>
__device__ __forceinline__ void dma_vt_tile(unsigned char* lds, const bf16_t* v, int64_t ld, int n, int lane, int j0) {
    const uint32_t ld2 = (uint32_t)(ld * 2);
    const uint32_t bytes = n > 0 ? (HD - 1) * ld2 + (uint32_t)min(64, (n + 7) & ~7) * 2 : 0u;
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)v, 0, (int)bytes, 0x00020000);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int row = (j0 + j) * 8 + (lane >> 3);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (j0 + j) * 1024), 16,
                                                 (uint32_t)row * ld2 + (uint32_t)(((lane & 7) ^ swz8(row)) << 4), 0, 0, 0);
    }
}
// columns from n on (of the eight keys 16 j + 8 lhi ..) as 0, whatever they hold: a probability of 0 times a NaN would be one
__device__ __forceinline__ void clear_columns(uint4& v, int n) {
    v.x &= n >= 2 ? 0xffffffffu : n == 1 ? 0xffffu : 0u;
    v.y &= n >= 4 ? 0xffffffffu : n == 3 ? 0xffffu : 0u;
    v.z &= n >= 6 ? 0xffffffffu : n == 5 ? 0xffffu : 0u;
    v.w &= n >= 8 ? 0xffffffffu : n == 7 ? 0xffffu : 0u;
}

// One workgroup: 128 rows of one request and KV head, 32 a wavefront, all their keys, 64 at a time in LDS for all four; the next 64
// are on their way while these are worked on, and one barrier a step says both that they are there and that the last ones are
// out of use.
// What bounds it: with two workgroups a compute unit 0.85 to 1.1 us for 128 rows and 64 keys, where the matrix instructions take 0.45;
// without the copies a sixth less, without the softmax a sixth less: two wavefronts a SIMD wait for one another's LDS reads and
// vector instructions.  (64 rows a wavefront halve the LDS reads, but one wavefront a SIMD then has nobody to hide behind: 2.7 us.)
// Measured (us, 32 heads on 8 KV heads): 20 requests of 500 rows alone 84, 60 of 500 behind 1000 keys 770 (0.8 PFLOP/s), 27 of 161
// behind 45 37; head dimension 64, 20 of 150 behind 4000 87.
template <int HD>
__global__ void __launch_bounds__(256, 2) attn_shared_rows_kernel(const SharedParams p, const SharedTable tab) {
    constexpr int KS = HD / 16, HT = HD / 32;
    constexpr int UNIT = 64 * HD * 2, N_DMA = UNIT / 1024 / 4;  // bytes of 64 keys of K or V^T; loads of a wavefront
    __shared__ __attribute__((aligned(16))) unsigned char smem[2][2][UNIT];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l31 = lane & 31, lhi = lane >> 5;
    const int kvh = (int)(blockIdx.x % (unsigned)p.Hkv), item = (int)(blockIdx.x / (unsigned)p.Hkv), group = p.Hq / p.Hkv;
    const int req = __builtin_amdgcn_readfirstlane(shared_request(tab, item));
    const SharedSeq sq = tab.seq[req];
    const int n_rows = sq.q_len * group, wg0 = (item - tab.item0[req]) * 128, row0 = wg0 + wave * 32;      // (position, head) order
    const int vr = min(row0 + l31, n_rows - 1), pos = vr / group, head = kvh * group + vr - pos * group;
    const bool valid = row0 + l31 < n_rows;
    const int64_t orow = ((int64_t)(sq.q_row + pos) * p.Hq + head) * HD;
    const int hidden = sq.kv_len - sq.q_len + 1;               // position i of the request sees i + hidden own keys (may be below 0)
    const int see_max = row0 < n_rows ? max(0, hidden + min(row0 + 31, n_rows - 1) / group) : 0, see_min = hidden + min(row0, n_rows - 1) / group;
    const int wg_max = max(0, hidden + min(wg0 + 127, n_rows - 1) / group);

    Rows<HD> st;
    st.start((const bf16_t*)p.q + orow + lhi * 8, valid);
    const int64_t krs = (int64_t)p.Hkv * HD;
    const bf16_t* const ko = (const bf16_t*)p.k + (int64_t)sq.kv_row * krs + kvh * HD;
    const bf16_t* const kp = (const bf16_t*)p.k2 + kvh * HD;
    const bf16_t* const vo = (const bf16_t*)p.v + (int64_t)kvh * HD * p.ldv + sq.kv_row;
    const bf16_t* const vp = (const bf16_t*)p.v2 + (int64_t)kvh * HD * p.ldv2;
    const int nb2 = (p.n2 + 63) / 64, nb = nb2 + (wg_max + 63) / 64;
    auto dma = [&](int b) {
        if (b >= nb) return;
        const bool own = b >= nb2;
        const int key0 = (own ? b - nb2 : b) * 64, n = (own ? sq.kv_len : p.n2) - key0;
        dma_k_tile<HD, N_DMA>(smem[b & 1][0], (own ? ko : kp) + key0 * krs, krs, n, lane, wave * N_DMA);
        dma_vt_tile<HD, N_DMA>(smem[b & 1][1], (own ? vo : vp) + key0, own ? p.ldv : p.ldv2, n, lane, wave * N_DMA);
    };
    const int pk = (l31 & 0x13) | ((l31 & 4) << 1) | ((l31 & 8) >> 1);       // MFMA row i holds key pi(i): bits 2, 3 swapped
    const int k_sw = HD == 128 ? (pk & 15) : swz8(pk), v_sw = swz8(l31);
    dma(0);
#pragma unroll 1
    for (int b = 0; b < nb; ++b) {
        const bool own = b >= nb2;
        const int key0 = (own ? b - nb2 : b) * 64;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        dma(b + 1);
        if (key0 >= (own ? see_max : row0 < n_rows ? p.n2 : 0)) continue;      // (wavefront-uniform)
        const unsigned char *const sk = smem[b & 1][0], *const sv = smem[b & 1][1];
        const int n_v = (own ? sq.kv_len : p.n2) - key0;       // V^T columns that are keys
        f32x16 s[2];
        bf16x8 pf[4];
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[a][r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const bf16x8 kf = *(const bf16x8*)(sk + (a * 32 + pk) * (HD * 2) + (((ks * 2 + lhi) ^ k_sw) << 4));
                s[a] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, st.qf[ks], s[a], 0, 0, 0);
            }
        uint4 v[2][HT];
        const auto read_v = [&](int j0) {                       // V^T of 32 keys
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int ht = 0; ht < HT; ++ht) v[j][ht] = *(const uint4*)(sv + (ht * 32 + l31) * 128 + ((((j0 + j) * 2 + lhi) ^ v_sw) << 4));
            if (n_v < 64) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int ht = 0; ht < HT; ++ht) clear_columns(v[j][ht], n_v - (16 * (j0 + j) + 8 * lhi));
            }
        };
        read_v(0);
        st.template softmax<2>(s, pf, key0 + 64 > (own ? see_min : p.n2), (own ? pos + hidden : p.n2) - key0, lhi, p.sc);
#pragma unroll
        for (int j0 = 0; j0 < 4; j0 += 2) {
            if (j0) read_v(j0);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int ht = 0; ht < HT; ++ht)
                    st.acc[ht] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[j][ht]), pf[j0 + j], st.acc[ht], 0, 0, 0);
        }
    }
    // through LDS, so that whole rows are written side by side (16 bytes of 32 rows at a time took 6.5 us for 16 MB more)
    constexpr int PITCH = HD * 2 + 16, LPR = HD / 8;           // lanes (16 bytes each) of a row
    const float l = other_half_sum(st.l), inv = l > 0.f ? 1.0f / l : 0.f;
    __syncthreads();
    unsigned char* const so = &smem[0][0][0] + wave * 32 * PITCH;
#pragma unroll
    for (int ht = 0; ht < HT; ++ht)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            store4((bf16_t*)(so + l31 * PITCH) + ht * 32 + 8 * g + 4 * lhi, st.acc[ht][4 * g], st.acc[ht][4 * g + 1], st.acc[ht][4 * g + 2],
                   st.acc[ht][4 * g + 3], inv);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (a wavefront's own rows: no barrier)
#pragma unroll
    for (int i = 0; i < 32 * LPR / 64; ++i) {
        const int row = i * (64 / LPR) + lane / LPR;
        const uint4 x = *(const uint4*)(so + row * PITCH + lane % LPR * 16);
        const int64_t at = __shfl(orow, row);
        if (row0 + row < n_rows) *(uint4*)((bf16_t*)p.o + at + lane % LPR * 8) = x;
    }
}

// How a launch of few rows is divided.  Partial results: opart [piece][row of the table][head][HD], mlpart [..][2] (maximum in
// powers of 2, sum), the prefix's np pieces first, then those of a request's own keys.
struct Parts {
    float *opart, *mlpart;
    int np, per;               // the prefix: pieces of `per` keys
    int own_per;               // own keys: pieces of that many (0: their part is not among the pieces)
    int prefix_items;          // workgroups of the prefix per KV head
};

// Few rows (one token a request): what counts is how many keys are on their way at once.  Every wavefront has 64 keys of its own in LDS
// at a time, loaded by whole cache lines past the registers (K rows as they are, 128 bytes of each V^T row), no two wavefronts wait
// for each other, and they meet at the end.  K of its next block is on its way as soon as the scores are there, V^T as soon as
// the products are.  RT: tiles of 32 rows that go through the same keys.
// What bounds it: reading the keys, 4.2 to 4.8 TB/s where there are many (128 tokens with 3000 keys each: 1.6 GB in 307 us), else the
// chain of a launch, a first block, the meeting in LDS and the join: one token behind 14000 keys 22 us, two behind 500 10.
// WHOLE: a workgroup is 32 rows of one request, all keys they see; result in o.
// PARTS: a workgroup is a piece of the prefix, which all requests share, with 32 RT rows of any requests; or a piece of a request's own keys
// with 32 of its rows.  Partial results.
// FINISH: a workgroup is 32 rows of one request, the own keys they see, joined with the prefix's np pieces of these rows; result in o.
enum { WHOLE, PARTS, FINISH };
template <int HD, int NW, int RT, int MODE>
__global__ void __launch_bounds__(NW * 64, 1) attn_shared_tokens_kernel(const SharedParams p, const Parts parts, const SharedTable tab) {
    constexpr int KS = HD / 16, HT = HD / 32;
    constexpr int UNIT = 64 * HD * 2, N_DMA = UNIT / 1024;      // bytes of 64 keys of K or V^T; loads of a wavefront
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l31 = lane & 31, lhi = lane >> 5;
    const int kvh = (int)(blockIdx.x % (unsigned)p.Hkv), group = p.Hq / p.Hkv;
    int item = (int)(blockIdx.x / (unsigned)p.Hkv);
    const bool of_prefix = MODE == PARTS && item < parts.prefix_items;
    if (MODE == PARTS && !of_prefix) item -= parts.prefix_items;
    // rows in (position, head) order: of one request, or (a piece of the prefix) of the table
    int req = 0, row0, n_rows, piece = 0;
    SharedSeq sq = {0, 0, 0, 0};
    if (of_prefix) {
        piece = item % parts.np;
        row0 = item / parts.np * (32 * RT);
        n_rows = tab.row0[tab.n] * group;
    } else {
        req = __builtin_amdgcn_readfirstlane(shared_request(tab, item));
        sq = tab.seq[req];
        int tile = item - tab.item0[req];
        if (MODE == PARTS) {
            const int pieces = (sq.kv_len + parts.own_per - 1) / parts.own_per;
            piece = tile % pieces;
            tile /= pieces;
        }
        row0 = tile * 32;
        n_rows = sq.q_len * group;
    }
    const int n_rt = of_prefix ? min(RT, (n_rows - row0 + 31) / 32) : 1;
    const int hidden = sq.kv_len - sq.q_len + 1;               // position i of the request sees i + hidden own keys (may be below 0)
    const int see = min(row0 + l31, n_rows - 1) / group + hidden;
    const int see_max = max(0, hidden + min(row0 + 31, n_rows - 1) / group), see_min = hidden + row0 / group;
    // prefix keys [a0, a1), then own keys [b0, b1)
    const int a0 = of_prefix ? piece * parts.per : 0;
    const int a1 = MODE == WHOLE ? p.n2 : of_prefix ? min(a0 + parts.per, p.n2) : 0;
    const int b0 = MODE == PARTS && !of_prefix ? piece * parts.own_per : 0;
    const int b1 = MODE != PARTS ? see_max : of_prefix ? 0 : min(b0 + parts.own_per, see_max);
    const int nb2 = max(a1 - a0 + 63, 0) / 64, nb = nb2 + max(b1 - b0 + 63, 0) / 64;

    Rows<HD> st[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int vr = min(row0 + rt * 32 + l31, n_rows - 1), pos = vr / group;
        int q_row = sq.q_row + pos;
        if (of_prefix) {
            const int r = shared_request_of_row(tab, pos);
            q_row = tab.seq[r].q_row + pos - tab.row0[r];
        }
        st[rt].start((const bf16_t*)p.q + ((int64_t)q_row * p.Hq + kvh * group + vr - pos * group) * HD + lhi * 8, row0 + rt * 32 + l31 < n_rows);
    }
    const int64_t krs = (int64_t)p.Hkv * HD;
    const bf16_t* const ko = (const bf16_t*)p.k + (int64_t)sq.kv_row * krs + kvh * HD;
    const bf16_t* const kp = (const bf16_t*)p.k2 + kvh * HD;
    const bf16_t* const vo = (const bf16_t*)p.v + (int64_t)kvh * HD * p.ldv + sq.kv_row;
    const bf16_t* const vp = (const bf16_t*)p.v2 + (int64_t)kvh * HD * p.ldv2;
    unsigned char* const sk = smem + wave * (2 * UNIT);
    unsigned char* const sv = sk + UNIT;
    auto first_key = [&](int b) { return b < nb2 ? a0 + b * 64 : b0 + (b - nb2) * 64; };
    // Block b's K, and V^T, into this wavefront's LDS; from block nb on nothing (the number of loads in flight stays known).
    auto dma_k = [&](int b) {
        const int key0 = first_key(b), end = b < nb2 ? p.n2 : sq.kv_len;
        dma_k_tile<HD, N_DMA>(sk, (b < nb2 ? kp : ko) + (b < nb ? key0 * krs : 0), krs, b < nb ? end - key0 : 0, lane, 0);
    };
    auto dma_v = [&](int b) {
        const int key0 = first_key(b), end = b < nb2 ? p.n2 : sq.kv_len;
        dma_vt_tile<HD, N_DMA>(sv, (b < nb2 ? vp : vo) + (b < nb ? key0 : 0), b < nb2 ? p.ldv2 : p.ldv, b < nb ? end - key0 : 0, lane, 0);
    };
    // fragments: K row pi(i) of a 32-key half (bits 2, 3 swapped: the eight keys a lane feeds to an MFMA are then side by side in
    // V^T), V^T row i of a 32-row tile
    const int pk = (l31 & 0x13) | ((l31 & 4) << 1) | ((l31 & 8) >> 1);
    const int k_sw = HD == 128 ? (pk & 15) : swz8(pk), v_sw = swz8(l31);
    int b = wave;
    dma_k(b);
    dma_v(b);
#pragma unroll 1
    for (; b < nb; b += NW) {
        const bool own = b >= nb2;
        const int key0 = first_key(b), end = own ? sq.kv_len : p.n2;
        const bool masked = key0 + 64 > (own ? see_min : a1);
        const int n_v = end - key0;                            // V^T columns that are keys
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (rt >= n_rt) break;
            if (rt == 0) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N_DMA) : "memory");        // K is there, V^T may be on its way
            f32x16 s[2];
            bf16x8 pf[4];
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[a][r] = 0.f;
            bf16x8 kf[KS][2];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int a = 0; a < 2; ++a) kf[ks][a] = *(const bf16x8*)(sk + (a * 32 + pk) * (HD * 2) + (((ks * 2 + lhi) ^ k_sw) << 4));
            if (rt == n_rt - 1) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                // (the fragments are in registers)
                dma_k(b + NW);
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int a = 0; a < 2; ++a) s[a] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks][a], st[rt].qf[ks], s[a], 0, 0, 0);
            st[rt].template softmax<2>(s, pf, masked, (own ? see : a1) - key0, lhi, p.sc);
            if (rt == 0) {                                                        // V^T is there (K of the next block may be on its way)
                if (n_rt == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N_DMA) : "memory");
                else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int ht = 0; ht < HT; ++ht) {
                    uint4 v = *(const uint4*)(sv + (ht * 32 + l31) * 128 + (((j * 2 + lhi) ^ v_sw) << 4));
                    if (n_v < 64) clear_columns(v, n_v - (16 * j + 8 * lhi));
                    st[rt].acc[ht] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), pf[j], st[rt].acc[ht], 0, 0, 0);
                }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        dma_v(b + NW);
    }
    // ---- the wavefronts' parts, a row tile at a time: [wave][row][HD + 4] sums, then [wave][row] maxima and sums of p, joined in
    // wavefront order (what the loads still on their way write is out of use)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    constexpr int LD = HD + 4, DV = HD / 4;                    // 4 values a thread and turn
    float* const lds = (float*)smem;
    float* const sm = lds + NW * 32 * LD;
    float* const sl = sm + NW * 32;
    const int64_t plane = (int64_t)tab.row0[tab.n] * p.Hq;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        if (rt >= n_rt) break;
        const float l = other_half_sum(st[rt].l);
        __syncthreads();
        // (maxima in powers of 2 from here on)
        if (lhi == 0) { sm[wave * 32 + l31] = st[rt].m == -INFINITY ? -1.0e30f : st[rt].m * p.sc; sl[wave * 32 + l31] = l; }
#pragma unroll
        for (int ht = 0; ht < HT; ++ht)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(float4*)(lds + (wave * 32 + l31) * LD + ht * 32 + 8 * g + 4 * lhi) =
                    make_float4(st[rt].acc[ht][4 * g], st[rt].acc[ht][4 * g + 1], st[rt].acc[ht][4 * g + 2], st[rt].acc[ht][4 * g + 3]);
        __syncthreads();
        const int rows_here = min(32, n_rows - row0 - rt * 32);
        for (int i = tid; i < rows_here * DV; i += NW * 64) {
            const int jr = i / DV, d = i % DV * 4, jv = row0 + rt * 32 + jr, jp = jv / group, jh = kvh * group + jv - jp * group;
            const int64_t rh = (of_prefix ? jp : tab.row0[req] + jp) * (int64_t)p.Hq + jh;
            float top = sm[jr];
#pragma unroll
            for (int w = 1; w < NW; ++w) top = fmaxf(top, sm[w * 32 + jr]);
            float lt = 0.f;
            float4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = __builtin_amdgcn_exp2f(sm[w * 32 + jr] - top);
                const float4 v = *(const float4*)(lds + (w * 32 + jr) * LD + d);
                lt += f * sl[w * 32 + jr];
                y.x += f * v.x; y.y += f * v.y; y.z += f * v.z; y.w += f * v.w;
            }
            if (MODE == PARTS) {
                const int64_t slot = (of_prefix ? piece : parts.np + piece) * plane + rh;
                *(float4*)(parts.opart + slot * HD + d) = y;
                if (d == 0) *(float2*)(parts.mlpart + slot * 2) = make_float2(top, lt);
                continue;
            }
            if (MODE == FINISH) {
                const float* const ml = parts.mlpart + rh * 2;
                float all = top;
#pragma unroll 8
                for (int e = 0; e < parts.np; ++e) all = fmaxf(all, ml[e * plane * 2]);
                const float f = __builtin_amdgcn_exp2f(top - all);
                lt *= f;
                y.x *= f; y.y *= f; y.z *= f; y.w *= f;
#pragma unroll 8
                for (int e = 0; e < parts.np; ++e) {
                    const float2 m2 = *(const float2*)(ml + e * plane * 2);
                    const float4 v = *(const float4*)(parts.opart + (e * plane + rh) * HD + d);
                    const float w = __builtin_amdgcn_exp2f(m2.x - all);
                    lt += w * m2.y;
                    y.x += w * v.x; y.y += w * v.y; y.z += w * v.z; y.w += w * v.w;
                }
            }
            store4((bf16_t*)p.o + ((int64_t)(sq.q_row + jp) * p.Hq + jh) * HD + d, y.x, y.y, y.z, y.w, lt > 0.f ? 1.0f / lt : 0.f);
        }
    }
}

// The pieces of every row, in their order: o = sum of 2^(m - top) O / sum of 2^(m - top) l; HD / 4 threads a row and head.
template <int HD>
__global__ void __launch_bounds__(256) attn_shared_join_kernel(const SharedParams p, const Parts parts, const SharedTable tab) {
    constexpr int PER = HD / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int rows = tab.row0[tab.n];
    const int64_t plane = (int64_t)rows * p.Hq;
    if (i >= plane * PER) return;
    const int64_t rh = i / PER;
    const int c = (int)(rh / p.Hq), head = (int)(rh - (int64_t)c * p.Hq), f = (int)(i - rh * PER) * 4;
    const int req = shared_request_of_row(tab, c);
    const SharedSeq sq = tab.seq[req];
    const int n = parts.np + (parts.own_per ? (sq.kv_len + parts.own_per - 1) / parts.own_per : 0);
    const int lane = threadIdx.x & (PER - 1);
    float top = -1.0e30f;
    for (int s = lane; s < n; s += PER) top = fmaxf(top, parts.mlpart[(s * plane + rh) * 2]);
#pragma unroll
    for (int off = PER / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, PER));
    float4 acc = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int s0 = 0; s0 < n; s0 += PER) {
        const float2 ml = *(const float2*)(parts.mlpart + (min(s0 + lane, n - 1) * plane + rh) * 2);
        const float wl = s0 + lane < n ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
        for (int e0 = 0; e0 < min(PER, n - s0); e0 += 4) {              // (pieces past the last one: the last one, weight 0)
            float4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = *(const float4*)(parts.opart + (min(s0 + e0 + u, n - 1) * plane + rh) * HD + f);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float w = __shfl(wl, e0 + u, PER);
                acc.x += w * v[u].x; acc.y += w * v[u].y; acc.z += w * v[u].z; acc.w += w * v[u].w;
                l += w * __shfl(ml.y, e0 + u, PER);
            }
        }
    }
    const float inv = l > 0.f ? 1.0f / l : 0.f;
    uint2 w2;
    w2.x = (uint32_t)f2bf(acc.x * inv) | ((uint32_t)f2bf(acc.y * inv) << 16);
    w2.y = (uint32_t)f2bf(acc.z * inv) | ((uint32_t)f2bf(acc.w * inv) << 16);
    *(uint2*)((bf16_t*)p.o + ((int64_t)(sq.q_row + c - tab.row0[req]) * p.Hq + head) * HD + f) = w2;
}

// How the requests of a table run.
//   TOKENS       one launch, 32 rows of a request and all their keys a workgroup
//   ROWS         one launch, 128 rows of a request and all their keys a workgroup
//   TILES        256 rows of any requests a workgroup of attn_mfma.hip's tile kernel, the prefix in np pieces; joined when np > 1
//   SPLIT        the prefix in np pieces with 32 rt rows of any requests, own keys in pieces of own_per, joined
//   TILES_SPLIT  the prefix by the tile kernel, own keys in pieces, joined
//   TILES_FINISH the prefix by the tile kernel, own keys whole, which joins both
enum Mode { TOKENS = PO_SHARED_TOKENS, ROWS = PO_SHARED_ROWS, TILES = PO_SHARED_TILES, SPLIT = PO_SHARED_SPLIT, TILES_SPLIT = PO_SHARED_TILES_SPLIT, TILES_FINISH = PO_SHARED_TILES_FINISH };
struct Plan {
    Mode mode;
    int np, per, own_per, rt, slots;     // slots: partial results of a row at most
};

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// The one expected to take the least time (microseconds) with the scratch there is.  Every form's time is what one workgroup takes
// times how often the card is filled with them, and no less than its bytes at what memory gives.  Measured (us, 32 heads on 8 KV heads
// of 128; requests x rows / prefix):        TOKENS  ROWS  TILES  SPLIT  TILES_SPLIT  TILES_FINISH
//   3 x 161 / 45                                13    12      -     41            -             -
//   20 x 500 / 0                               200    83      -      -            -             -
//   20 x 20 / 2000                              52    49     41     67           50            52
//   4 x 150 / 14000                            447   288    148    355          160           172
//   60 x 500 / 1000                           1608   768    823      -         1605          1633
//   1 x 1, 300 own keys / 14000                110   278     26     22           34            29
//   1 x 40, 3000 own / 14000                   153   355    165     50           45            69
//   64 x 1, 300 own / 14000                    275   304    341     70           62            57
//   20 x 1, 9000 own / 14000                   309   740   7120    170          198           229
//   128 x 1, 3000 own / 2000                   378   435   4097    309          327           341
Plan plan(const SharedTable& t, int Hq, int Hkv, int hd, int n2, size_t scratch_bytes) {
    const int group = Hq / Hkv, rows = t.row0[t.n], tiles2 = n2 / 64;
    const int64_t vr = (int64_t)rows * group;
    const double row_bytes = (double)rows * Hq * (hd + 2) * 4.0, slot_us = row_bytes * 2.0 / 6.0e6;      // a slot of every row, written and read
    const double narrow = hd / 128.0, key_bytes = Hkv * hd * 4.0;
    int own_max = 0;
    int64_t own_sum = 0, tiles32 = 0, tiles128 = 0;
    double seen = 0.0;                                        // own keys of all rows
    for (int i = 0; i < t.n; ++i) {
        const SharedSeq& q = t.seq[i];
        own_max = std::max(own_max, q.kv_len);
        own_sum += q.kv_len;
        seen += q.q_len * std::max(0.0, q.kv_len - 0.5 * q.q_len);
        tiles32 += ceil_div((int64_t)q.q_len * group, 32);
        tiles128 += ceil_div((int64_t)q.q_len * group, 128);
    }
    seen /= rows;
    Plan best{TOKENS, 0, 0, 0, 1, 0};
    // 32 rows a workgroup; two wavefronts, and two workgroups a compute unit, where there are more than 256.  A wavefront's block of
    // 64 keys: 1.9 us alone on its compute unit, 2.2 to 2.4 with another workgroup beside it
    const auto tokens_us = [&](double wgs, double most, double mean, double keys_read) {
        const double us = wgs <= 256 ? 1.9 * (std::ceil(most / 256) + 1.0)
                                     : std::max(2.4 * (std::ceil(most / 128) + 1.0), 2.2 * wgs / 512.0 * (mean / 128 + 2.0));
        return std::max(us * narrow, keys_read * key_bytes / 4.2e6);
    };
    double t_best = 5.0 + tokens_us((double)tiles32 * Hkv, n2 + own_max, n2 + seen, (double)n2 + own_sum);
    // (pieces that one launch can join: hd / 4 threads a row and head)
    const bool joined = ((int64_t)rows * Hq * (hd / 4) + 255) / 256 <= MAX_WORKGROUPS_256;
    const auto take = [&](const Plan& p, double us) {
        if (us < t_best && (p.slots == 0 || joined) && p.slots * row_bytes <= (double)scratch_bytes) { best = p; t_best = us; }
    };
    // 128 rows a workgroup: 64 keys 1.3 us alone, 0.85 a workgroup with two on a compute unit, 6 more for its beginning and end
    const double wg128 = (double)tiles128 * Hkv, c1 = hd == 128 ? 1.3 : 0.9, c2 = hd == 128 ? 0.85 : 0.65;
    take({ROWS, 0, 0, 0, 1, 0}, 5.0 + std::max((wg128 <= 256 ? c1 : 2.0 * c2) * (std::ceil((n2 + own_max) / 64.0) + 2.0),
                                              std::max(wg128 / 256.0 * c2 * ((n2 + seen) / 64.0 + 6.0), ((double)n2 + own_sum) * key_bytes / 3.6e6)));
    if (n2 == 0 && own_max == 0) return best;
    constexpr int64_t MOST = MAX_WORKGROUPS_256;              // workgroups of a launch of pieces
    // own keys by pieces, and the join
    const int own_per = (int)std::min<int64_t>(2048, std::max<int64_t>(512, (own_sum * Hkv / 256 + 255) / 256 * 256));
    const int own_slots = ceil_div(own_max, own_per);
    int64_t own_wgs = 0;
    for (int i = 0; i < t.n; ++i) own_wgs += (int64_t)ceil_div((int64_t)t.seq[i].q_len * group, 32) * ceil_div(t.seq[i].kv_len, own_per) * Hkv;
    // the prefix by the tile kernel: a tile of 64 keys 1.35 us, 5 of them for its beginning and end
    if (hd == 128 && tiles2 > 0) {
        const int64_t wgs = (vr + 255) / 256 * Hkv;
        // own keys in the tile: a wavefront goes through those of all requests that its 64 rows meet, 32 keys in 3 us
        const double meets = std::min<double>(t.n, std::ceil(64.0 / group / ((double)rows / t.n)) + 0.5);
        const double in_tile = own_sum ? 3.0 * meets * std::ceil(seen / 32) : 0.0;
        const double finish_rows = std::ceil((double)vr / (double)tiles32 / 4.0);        // (128 threads: four rows at once)
        for (int np = 1; np <= std::min(tiles2, 64); ++np) {
            const int per = ceil_div(tiles2, np);
            if (ceil_div(tiles2, per) != np || (uint64_t)per * 64 * (uint64_t)Hkv * 256 >= (1ull << 32) || wgs * np > MOST) continue;
            const double us = 6.0 + ceil_div(wgs * np, 256) * (per + 5) * 1.35;
            take({TILES, np, 0, 0, 1, np > 1 ? np : 0}, us + ceil_div(wgs, 256) * in_tile + (np > 1 ? 4.0 + np * slot_us : 0.0));
            if (!own_wgs || own_wgs > MOST) continue;
            take({TILES_SPLIT, np, 0, own_per, 1, np + own_slots},
                 us + 3.0 + tokens_us((double)own_wgs, std::min(own_per, own_max), seen / own_slots, (double)own_sum) + 7.0 + (np + own_slots) * slot_us);
            take({TILES_FINISH, np, 0, 0, 1, np}, us + 1.0 + tokens_us((double)tiles32 * Hkv, own_max, seen, (double)own_sum) +
                                                      (1.5 + 0.1 * np) * finish_rows * std::max(1.0, tiles32 * Hkv / 512.0) + np * slot_us);
        }
    }
    // the prefix like the own keys, with 32 or 64 rows of any requests: 256 keys of a workgroup 1.9 or 5 us, 3 or 10 for its beginning and end
    // (the 4.0 of it, at near ties: with 3.0, 43 single tokens of 40 heads with 370 keys alone took 29 us by pieces instead of 17, and 39 x 8
    // rows with 652 keys 41 instead of 27; 79 x 1 with 92 keys behind 1082 lose most by it, 44 instead of 35)
    const int rt = vr <= 32 ? 1 : 2;
    const int64_t groups = (vr + 32 * rt - 1) / (32 * rt) * Hkv;
    const double own_us = own_wgs ? (3.0 + 1.9 * std::ceil(std::min<double>(own_per, seen) / 256)) * narrow : 0.0;
    const double own_most = own_wgs ? (3.0 + 1.9 * std::ceil(std::min(own_per, own_max) / 256.0)) * narrow : 0.0;
    const double read_us = ((double)n2 + own_sum) * key_bytes / 4.8e6;
    for (int np = n2 > 0 ? 1 : 0; np <= 64; ++np) {
        const int per = np ? std::max(256, ceil_div(ceil_div(n2, np), 64) * 64) : 0;
        if (np && ceil_div(n2, per) != np) continue;
        const double pre = np ? (rt == 1 ? 3.0 + 1.9 * std::ceil(per / 256.0) : 10.0 + 5.0 * std::ceil(per / 256.0)) * narrow : 0.0;
        const int64_t wgs = groups * np;
        if (wgs + own_wgs > MOST) break;
        take({SPLIT, np, per, own_per, rt, np + own_slots},
             4.0 + std::max({wgs > 256 && wgs <= 512 ? 2.0 * pre : pre, own_most, (wgs * pre + own_wgs * own_us) / 256.0, read_us}) + 3.0 + (np + own_slots) * slot_us);
        if (np == 0) break;
    }
    return best;
}

template <int HD, int NW, int RT, int MODE>
void launch_tokens(const SharedParams& p, const Parts& parts, const SharedTable& tab, unsigned items, hipStream_t s) {
    constexpr int RING = NW * 2 * 64 * HD * 2, JOIN = (NW * 32 * (HD + 4) + 2 * NW * 32) * 4, LDS = RING > JOIN ? RING : JOIN;
    static OncePerDevice lds;
    lds.run(current_device(), [] { allow_dynamic_lds((const void*)(attn_shared_tokens_kernel<HD, NW, RT, MODE>), LDS); });
    hipLaunchKernelGGL((attn_shared_tokens_kernel<HD, NW, RT, MODE>), dim3(items * p.Hkv), dim3(NW * 64), LDS, s, p, parts, tab);
}

// (two wavefronts, two workgroups a compute unit, where there are enough of them)
template <int HD, int MODE>
void launch_tokens(const SharedParams& p, const Parts& parts, const SharedTable& tab, unsigned items, hipStream_t s) {
    if (items * p.Hkv > 256) launch_tokens<HD, 2, 1, MODE>(p, parts, tab, items, s);
    else launch_tokens<HD, 4, 1, MODE>(p, parts, tab, items, s);
}

template <int HD>
void launch_t(const SharedParams& p, const po_request_rows* seq, int n, float* scratch, size_t scratch_bytes, hipStream_t s) {
    const int group = p.Hq / p.Hkv;
    for (int i = 0; i < n;) {
        SharedTable tab;
        const int i0 = i;
        i = fill_table(tab, seq, i0, n, [](const SharedSeq&) { return 0; });
        if (tab.n == 0) continue;
        const Plan t = plan(tab, p.Hq, p.Hkv, HD, p.n2, scratch ? scratch_bytes : 0);
        const int rows = tab.row0[tab.n];
        Parts parts{};
        parts.np = t.np;
        parts.per = t.per;
        parts.own_per = t.own_per;
        parts.opart = scratch;
        parts.mlpart = scratch + (size_t)t.slots * rows * p.Hq * HD;
        const auto items = [&](int tile) {
            fill_table(tab, seq, i0, n, [&](const SharedSeq& q) {
                return ceil_div((int64_t)q.q_len * group, tile) * (t.own_per ? ceil_div(q.kv_len, t.own_per) : 1);
            });
            return (unsigned)tab.item0[tab.n];
        };
        unsigned n_items;
        switch (t.mode) {
            case TOKENS:
                launch_tokens<HD, WHOLE>(p, parts, tab, items(32), s);
                break;
            case ROWS:
                n_items = items(128);
                hipLaunchKernelGGL(attn_shared_rows_kernel<HD>, dim3(n_items * p.Hkv), dim3(256), 0, s, p, tab);
                break;
            case TILES:
                launch_attention_shared_tiles(p, tab, t.np, true, parts.opart, parts.mlpart, s);
                break;
            case TILES_SPLIT:
                launch_attention_shared_tiles(p, tab, t.np, false, parts.opart, parts.mlpart, s);
                n_items = items(32);
                if (n_items) launch_tokens<HD, PARTS>(p, parts, tab, n_items, s);
                break;
            case TILES_FINISH:
                launch_attention_shared_tiles(p, tab, t.np, false, parts.opart, parts.mlpart, s);
                launch_tokens<HD, FINISH>(p, parts, tab, items(32), s);
                break;
            case SPLIT:
                parts.prefix_items = ceil_div((int64_t)rows * group, 32 * t.rt) * t.np;
                n_items = items(32) + parts.prefix_items;
                if (t.rt == 1) launch_tokens<HD, 4, 1, PARTS>(p, parts, tab, n_items, s);
                else launch_tokens<HD, 4, 2, PARTS>(p, parts, tab, n_items, s);
                break;
        }
        if (t.slots > 0 && t.mode != TILES_FINISH)
            hipLaunchKernelGGL(attn_shared_join_kernel<HD>, dim3((unsigned)(((int64_t)rows * p.Hq * (HD / 4) + 255) / 256)), dim3(256), 0, s, p,
                               parts, tab);
    }
}

}  // namespace

size_t attention_shared_scratch(const po_request_rows* seq, int n, int Hq, int Hkv, int hd, int64_t n2) {
    size_t most = 0;
    for (int i = 0; i < n;) {
        SharedTable tab;
        i = fill_table(tab, seq, i, n, [](const SharedSeq&) { return 0; });
        if (tab.n) most = std::max(most, (size_t)plan(tab, Hq, Hkv, hd, (int)n2, SIZE_MAX).slots * tab.row0[tab.n] * Hq * (hd + 2) * sizeof(float));
    }
    return most;
}

void attention_shared_form(const po_request_rows* seq, int n, int Hq, int Hkv, int hd, int64_t n2, size_t scratch_bytes, int* form, int* pieces) {
    SharedTable tab;
    fill_table(tab, seq, 0, n, [](const SharedSeq&) { return 0; });
    const Plan p = tab.n ? plan(tab, Hq, Hkv, hd, (int)n2, scratch_bytes) : Plan{TOKENS, 0, 0, 0, 1, 0};
    *form = p.mode;
    *pieces = p.np;
}

void launch_attention_shared_bf16(const SharedParams& p, const po_request_rows* seq, int n, int hd, float* scratch, size_t scratch_bytes,
                                  hipStream_t s) {
    if (hd == 128) launch_t<128>(p, seq, n, scratch, scratch_bytes, s);
    else launch_t<64>(p, seq, n, scratch, scratch_bytes, s);
}

}  // namespace po
