// Log-probabilities of given tokens, the entropy and the most likely tokens of rows of logits (gfx950).
//
//   m = max_i l_i,  S = sum_i exp(l_i - m),  T = sum_i (l_i - m) exp(l_i - m)
//   log p(t) = (l_t - m) - log S,   entropy = log S - T / S
//
// A row is read once, in pieces by a wavefront each: (m, S, T) of a piece, and the largest logit of each of its chunks of 512.  Then a workgroup per
// row joins the pieces and finds the first tokens of the order (logit descending, index ascending): a number that at least as many
// disjoint groups of logits reach as tokens are wanted is a floor under them, and the chunks that reach it are read again for the few elements that
// do.  Where those are more than a list holds: the tokens lie in the chunks whose largest logits come first in that order, as many chunks as
// tokens (an element of any other chunk has the largest elements of all of those before it), and the same holds for the runs of 8
// within those chunks, so that at most 8 elements a token are ordered in the end, whatever the row holds.
// What bounds it: many rows, reading them (1024 float32 rows of 128256 in one launch 97 us, 5.4 TB/s; pieces of 256 bf16 rows of 152064 17, 4.6: five
// operations and an exponential a logit), then the answers, 7.2 us for 256 rows' five tokens and 16 for 64, a chain of loads, exchanges and
// rankings; one row, that chain (4.7 + 7.1 us for twenty tokens).
// NaN counts as -infinity; -infinity has no weight; with +infinity among the logits only those have, the same each.
#include "po_internal.h"

#include <algorithm>

namespace po {
namespace {

constexpr int CHUNK = 512;                       // logits; 8 a lane
constexpr int PER_WAVE = 4;                      // chunks of a piece
constexpr int PIECE = CHUNK * PER_WAVE;
constexpr int MAX_TOP = 64;

struct Stats { float m, s, t, pad; };            // of a piece

// A logit as it is read: the sum quiets a signalling NaN.  (Of a number and a quiet NaN the larger is the number; of a signalling one it is NaN, and
// of that and the next number the next one: what came before it would be lost.)
__device__ __forceinline__ float quiet(float v) { return v + 0.0f; }
// the logits of a lane: 8 from i on; they exist, and lie on 16 bytes
__device__ __forceinline__ void load8_whole(const float* p, float (&v)[8]) {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    v[0] = quiet(a.x); v[1] = quiet(a.y); v[2] = quiet(a.z); v[3] = quiet(a.w);
    v[4] = quiet(b.x); v[5] = quiet(b.y); v[6] = quiet(b.z); v[7] = quiet(b.w);
}
__device__ __forceinline__ void load8_whole(const bf16_t* p, float (&v)[8]) {
    const uint4 a = *(const uint4*)p;
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        v[2 * c] = quiet(__uint_as_float(w[c] << 16));
        v[2 * c + 1] = quiet(__uint_as_float(w[c] & 0xffff0000u));
    }
}
// -infinity beyond V
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int i, int V, float (&v)[8]) {
    if (VEC && i + 8 <= V) {
        load8_whole(row + i, v);
        return;
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = i + c < V ? quiet(to_f32(row[i + c])) : -INFINITY;
}

// Over a wavefront, all lanes get it, on the vector ALU: within rows of 16 lanes, then the four rows (the same by way of LDS, six exchanges for
// each of seven reductions a piece, took 11 us of LDS in 256 rows of 152064).
template <int CTRL>
__device__ __forceinline__ float moved_lanes(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true)); }
constexpr int ROR8 = 0x128, HALF_MIRROR = 0x141, QUAD_1032 = 0xb1, QUAD_2301 = 0x4e;       // lane ^ 8; 7 - lane in each 8; lane ^ 1; lane ^ 2
__device__ __forceinline__ float max_quads(float v) {
    v = fmaxf(v, moved_lanes<QUAD_1032>(v));
    return fmaxf(v, moved_lanes<QUAD_2301>(v));
}
__device__ __forceinline__ float sum_quads(float v) {
    v += moved_lanes<QUAD_1032>(v);
    return v + moved_lanes<QUAD_2301>(v);
}
template <typename F>
__device__ __forceinline__ float over_rows(float v, F f) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);       // (a row beside the next one)
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float added(float a, float b) { return a + b; }
__device__ __forceinline__ float first_lane(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, moved_lanes<ROR8>(v));
    v = fmaxf(v, moved_lanes<HALF_MIRROR>(v));
    return first_lane(over_rows(max_quads(v), larger));
}
// Four maxima together: each exchange halves how many values a lane still holds.  Lane 4 q gets number (q & 1) * 2 + (q >> 1 & 1).
__device__ __forceinline__ float wave_max4(const float (&v)[4]) {
    const bool b3 = threadIdx.x & 8, b2 = threadIdx.x & 4;
    const float p = fmaxf(b3 ? v[1] : v[0], moved_lanes<ROR8>(b3 ? v[0] : v[1])), q = fmaxf(b3 ? v[3] : v[2], moved_lanes<ROR8>(b3 ? v[2] : v[3]));
    return over_rows(max_quads(fmaxf(b2 ? q : p, moved_lanes<HALF_MIRROR>(b2 ? p : q))), larger);
}
// ... and two sums
__device__ __forceinline__ void wave_sum2(float& s, float& t) {
    const bool b3 = threadIdx.x & 8;
    float p = (b3 ? t : s) + moved_lanes<ROR8>(b3 ? s : t);
    p += moved_lanes<HALF_MIRROR>(p);
    p = over_rows(sum_quads(p), added);
    s = first_lane(p);
    t = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(p), 8));
}

// S and T of the wavefront's values with maximum m, in powers of 2 (T log2(e)).  A distance is one fma, v log2(e) - c with c = m log2(e) rounded: what
// that rounding adds to all of them, delta, is taken out of the sums.  -infinity, NaN and a product beyond float32 leave T no finite number; then,
// and where m is so large that delta is not small, every distance held to where a term is 0 in float32 (fmaxf turns NaN into its other operand).
__device__ __forceinline__ Stats wave_stats(const float (&x)[PER_WAVE][8], float m) {
    constexpr int N = PER_WAVE * 8;
    const float(&v)[N] = *(const float(*)[N])&x;
    constexpr float LOG2E = 1.44269504f, LN2 = 0.693147181f;
    Stats r = {m, 0.f, 0.f, 0.f};
    if (m == INFINITY) {
#pragma unroll
        for (int i = 0; i < N; ++i) r.s += v[i] == INFINITY ? 1.f : 0.f;
        wave_sum2(r.s, r.t);
    } else if (m > -INFINITY) {
        bool done = fabsf(m) < 0x1p20f;          // (delta is below 0.1)
        if (done) {
            const float c = m * LOG2E, delta = fmaf(m, LOG2E, -c), back = __builtin_amdgcn_exp2f(-delta);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = fmaf(v[i], LOG2E, -c), e = __builtin_amdgcn_exp2f(d);
                r.s += e;
                r.t = fmaf(d, e, r.t);
            }
            wave_sum2(r.s, r.t);
            done = fabsf(r.t) < INFINITY;
            r.t = fmaf(-delta, r.s, r.t) * back;
            r.s *= back;
        }
        if (!done) {
            r.s = r.t = 0.f;
            asm volatile("" : "+v"(m));          // (else the compiler keeps the first pass's 32 distances for this one)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float d = fmaxf((v[i] - m) * LOG2E, -250.0f), e = __builtin_amdgcn_exp2f(d);
                r.s += e;
                r.t = fmaf(d, e, r.t);
            }
            wave_sum2(r.s, r.t);
        }
        r.t *= LN2;
    }
    return r;
}

// the logits of a wavefront's piece p
template <typename T, bool VEC>
__device__ __forceinline__ void load_piece(const T* row, int p, int V, float (&v)[PER_WAVE][8]) {
    const int lane = threadIdx.x & 63, i0 = p * PIECE;
    if (VEC && i0 + PIECE <= V) {
#pragma unroll
        for (int c = 0; c < PER_WAVE; ++c) load8_whole(row + i0 + c * CHUNK + lane * 8, v[c]);
        return;
    }
#pragma unroll 1
    for (int c = 0; c < PER_WAVE; ++c) {
        float x[8];
        load8<T, VEC>(row, i0 + c * CHUNK + lane * 8, V, x);
#pragma unroll
        for (int u = 0; u < PER_WAVE; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = u == c ? x[e] : v[u][e];
    }
}
// ... its sums, and the largest logits of its chunks where they are asked for (chunk_max: of the row)
__device__ __forceinline__ Stats piece_stats(const float (&v)[PER_WAVE][8], int p, float* chunk_max, int chunks) {
    float cm[PER_WAVE];
#pragma unroll
    for (int c = 0; c < PER_WAVE; ++c) {
        cm[c] = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) cm[c] = fmaxf(cm[c], v[c][e]);
    }
    float m = -INFINITY;
    if (chunk_max) {
        const float one = wave_max4(cm);
        const int lane = threadIdx.x & 63, c = (lane >> 2 & 1) * 2 + (lane >> 3 & 1);
        if (lane < 16 && (lane & 3) == 0 && p * PER_WAVE + c < chunks) chunk_max[p * PER_WAVE + c] = one;
        m = fmaxf(one, moved_lanes<ROR8>(one));
        m = first_lane(fmaxf(m, moved_lanes<HALF_MIRROR>(m)));
    } else {
#pragma unroll
        for (int c = 0; c < PER_WAVE; ++c) m = fmaxf(m, cm[c]);
        m = wave_max(m);
    }
    return wave_stats(v, m);
}

// Pieces of rows: a wavefront each.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256, 6) logprob_pieces_kernel(const T* __restrict__ logits, int64_t ld, int V, int pieces, int64_t total,
                                                                Stats* __restrict__ stats, float* __restrict__ chunk_max, int chunks) {
    const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (w >= total) return;
    const int64_t r = w / pieces;
    const int p = (int)(w - r * pieces);
    float v[PER_WAVE][8];
    load_piece<T, VEC>(logits + r * ld, p, V, v);
    const Stats st = piece_stats(v, p, chunk_max ? chunk_max + r * chunks : nullptr, chunks);
    if ((threadIdx.x & 63) == 0) stats[w] = st;
}

// what joins pieces: their m, S, T relative to a common maximum
struct Sums { double s, t; };
__device__ __forceinline__ void join(const Stats& x, float m, Sums& r) {
    if (x.m == m) {                              // (also where both are infinite)
        r.s += x.s;
        r.t += x.t;
    } else if (x.m > -INFINITY && m < INFINITY) {
        const double d = (double)x.m - (double)m, e = (double)__expf((float)d);
        r.s += x.s * e;
        r.t += ((double)x.t + d * x.s) * e;
    }
}
// the sums relative to another maximum, at least as large
__device__ __forceinline__ Sums moved(const Sums& r, float from, float to) {
    if (from == to || !(from > -INFINITY)) return r;
    const double d = (double)from - (double)to, e = (double)__expf((float)d);
    return {r.s * e, (r.t + d * r.s) * e};
}
__device__ __forceinline__ float logprob_of(float l, float m, double log_s) {
    if (!(l > -INFINITY)) return -INFINITY;      // (NaN too)
    if (m == INFINITY) return l == INFINITY ? (float)-log_s : -INFINITY;
    return (float)((double)l - (double)m - log_s);
}

// Orders logits: the larger key first.  0: a logit without weight.
__device__ __forceinline__ unsigned long long order_key(float l, uint32_t index) {
    if (!(l > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(l + 0.0f), u = b & 0x80000000u ? ~b : b | 0x80000000u;       // (-0 is 0)
    return ((unsigned long long)u << 32) | (uint32_t)~index;
}
__device__ __forceinline__ float key_logit(unsigned long long k) {
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

constexpr int RUNS = MAX_TOP * (CHUNK / 8);      // of the chunks that are read again
constexpr int ROW_THREADS = 512;                 // (256: 64 tokens of 256 rows 23 us instead of 16, twenty of one 8.8 instead of 7.1)
constexpr int LIST = 512;                        // elements that are ordered at once; 8 of each of MAX_TOP runs

// Leaves in out[0 .. min(n, top)) the largest of keys[0 .. n), in order; keys[n .. n + 32) are overwritten.  All different, but for
// zeros, which are left out.  256 keys at a time are ranked, a thread holding four of them: each wavefront compares all of them with every
// fourth eight of the list (read as a broadcast, which a thread per key would read four times as often), and ranks[256] adds up.  (The
// callers' barriers stand around it; threads from 256 on only wait.)
__device__ __forceinline__ void largest(unsigned long long* keys, int n, int top, unsigned long long* out, int* ranks) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid < 32) keys[n + tid] = 0;
    for (int i0 = 0; i0 < n; i0 += 256) {
        if (tid < 256) ranks[tid] = 0;
        __syncthreads();
        unsigned long long k[4];
        int rank[4] = {0, 0, 0, 0};
        const int mine = min(n - i0, 256);
#pragma unroll
        for (int u = 0; u < 4; ++u) k[u] = u * 64 + lane < mine ? keys[i0 + u * 64 + lane] : ~0ull;
        for (int j = wave < 4 ? wave * 8 : n; j < n; j += 32) {
            unsigned long long o[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) o[c] = keys[j + c];
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (u * 64 < mine) rank[u] += o[c] > k[u];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (wave < 4 && u * 64 + lane < mine) atomicAdd(&ranks[u * 64 + lane], rank[u]);
        __syncthreads();
        if (tid < mine && keys[i0 + tid] && ranks[tid] < top) out[ranks[tid]] = keys[i0 + tid];
    }
}

// What a workgroup that answers for a row needs of LDS, beside the list of keys
struct RowShared {
    double red_s[4], red_t[4];
    unsigned long long best[MAX_TOP];
    float red_m[4], group_max[256];
    int chunk_count, count, ranks[256];
};
struct RowAnswer {
    const int32_t* tokens;
    int n_tokens;
    float *logprobs, *entropy;
    int top;
    int32_t* top_tokens;
    float* top_logprobs;
};

// A number that at least `top` of 256 (64) disjoint groups of logits reach, from their largest, as large as 16 bits of it allow; 0: fewer groups have
// weight.  As an order key's upper half.
__device__ __forceinline__ uint32_t reached(const float (&largest_of)[256], int top) {
    uint32_t u[4], t = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = (uint32_t)(order_key(largest_of[i * 64 + (threadIdx.x & 63)], 0) >> 32);
    const bool few = top <= 32;                  // (then of 64 groups: four in one)
    if (few) u[0] = max(max(u[0], u[1]), max(u[2], u[3]));
#pragma unroll
    for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
        int n = __popcll(__ballot(u[0] >= (t | bit)));
        if (!few) {
#pragma unroll
            for (int i = 1; i < 4; ++i) n += __popcll(__ballot(u[i] >= (t | bit)));
        }
        if (n >= top) t |= bit;
    }
    return t;
}
// ... as a logit, at least `lowest`.  (Cut to 16 bits it may lie below -infinity, where no logit is.)
__device__ __forceinline__ float reached_logit(uint32_t t, float lowest) {
    return t > 0x007fffffu ? fmaxf(key_logit((unsigned long long)t << 32), lowest) : lowest;
}

// A row's answer, by a workgroup of which 256 threads work, all where elements are read, from its pieces' sums and its chunks' largest logits.  What bounds it is a chain: the
// loads of pieces and chunks' maxima; a floor under the answer from those; the loads of the chunks that reach it, and beside them the sums; the
// order of the few elements that do.  Only rows with more than LIST of those go through the exact way by keys.  keys: RUNS + 32, only where top > 0.
template <typename T, bool VEC>
__device__ __forceinline__ void answer_row(const T* row, int64_t r, int V, int pieces, int chunks, const Stats* st, const float* cm, const RowAnswer& a,
                                           unsigned long long* keys, RowShared& sh) {
    double(&red_s)[4] = sh.red_s, (&red_t)[4] = sh.red_t;
    float(&red_m)[4] = sh.red_m;
    unsigned long long(&best)[MAX_TOP] = sh.best;
    int &count = sh.count, (&ranks)[256] = sh.ranks;
    int* const near = (int*)(keys + 2 * LIST);                         // chunks that reach the floor
    const int n_tokens = a.n_tokens, top = a.top, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tid = threadIdx.x < 256 ? (int)threadIdx.x : MAX_GIVEN_TOKENS;      // (the others only wait: behind the end of every list)
    // (first turn of each list and the first token: asked for together)
    const Stats none = {-INFINITY, 0.f, 0.f, 0.f};
    const Stats first = tid < pieces ? st[tid] : none;
    float cm0[2] = {-INFINITY, -INFINITY};
    if (top) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (tid < 256 && tid + i * 256 < chunks) cm0[i] = cm[tid + i * 256];
    }
    float given = -INFINITY;
    if (tid < n_tokens) {
        const int32_t t = a.tokens[r * n_tokens + tid];
        if (t >= 0 && t < V) given = to_f32(row[t]);
    }
    float m = first.m;
    for (int i = tid + 256; i < pieces; i += 256) m = fmaxf(m, st[i].m);
    m = wave_max(m);
    if (lane == 0 && wave < 4) red_m[wave] = m;
    if (top && wave < 4) {
        float own = fmaxf(cm0[0], cm0[1]);
        for (int i = tid + 512; i < chunks; i += 256) own = fmaxf(own, cm[i]);
        sh.group_max[tid] = own;
    }
    if (tid < MAX_TOP) best[tid] = 0;
    if (tid == 0) sh.chunk_count = count = 0;
    __syncthreads();
    m = fmaxf(fmaxf(red_m[0], red_m[1]), fmaxf(red_m[2], red_m[3]));
    const float lowest = m == INFINITY ? INFINITY : -INFINITY;         // of a logit with weight
    float floor_logit = lowest;
    bool few_groups = false;
    if (top) {
        const uint32_t t = reached(sh.group_max, top);
        few_groups = t == 0;
        floor_logit = reached_logit(t, lowest);
        for (int i = tid; i < chunks; i += 256) {
            const float c = i < 256 ? cm0[0] : i < 512 ? cm0[1] : cm[i];
            if (c >= floor_logit && c > -INFINITY) {
                const int slot = atomicAdd(&sh.chunk_count, 1);
                if (slot < LIST) near[slot] = i;
            }
        }
        __syncthreads();
    }
    const int n_near = sh.chunk_count;
    // f(logits, index of the first) of every run of 8 of n_chunks chunks, four at a time a thread (number t of nt); between: what is done while the
    // first ones come
    auto runs_of = [&](int t, int nt, int n_chunks, auto chunk_of, auto between, auto f) {
        const int n = n_chunks * (CHUNK / 8);
        bool once = true;
        for (int i0 = t; once || i0 < n; i0 += 4 * nt) {
            float v[4][8];
            int at[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * nt;
                at[u] = V;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] = -INFINITY;
                if (i < n) {
                    at[u] = chunk_of(i / (CHUNK / 8)) * CHUNK + (i % (CHUNK / 8)) * 8;
                    load8<T, VEC>(row, at[u], V, v[u]);
                }
            }
            if (once) between();
            once = false;
#pragma unroll
            for (int u = 0; u < 4; ++u) f(v[u], at[u]);
        }
    };
    auto runs = [&](int n_chunks, auto chunk_of, auto between, auto f) { runs_of((int)threadIdx.x, (int)blockDim.x, n_chunks, chunk_of, between, f); };
    auto push = [&](const float (&v)[8], int at) {
        int n = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) n += v[e] >= floor_logit && v[e] > -INFINITY;
        if (n) {
            int slot = atomicAdd(&count, n);                   // (their order in the list changes nothing: the keys are ranked)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (v[e] >= floor_logit && v[e] > -INFINITY) {
                    if (slot < LIST) keys[slot] = order_key(v[e], at + e);
                    ++slot;
                }
        }
    };
    auto nothing = [] {};
    auto sums = [&] {
        Sums sum = {0.0, 0.0};
        join(first, m, sum);
        for (int i = tid + 256; i < pieces; i += 256) join(st[i], m, sum);
        for (int off = 32; off > 0; off >>= 1) {
            sum.s += __shfl_xor(sum.s, off);
            sum.t += __shfl_xor(sum.t, off);
        }
        if (lane == 0 && wave < 4) { red_s[wave] = sum.s; red_t[wave] = sum.t; }
    };
    const bool listed = n_near <= LIST;
    auto near_chunk = [&](int i) { return near[i]; };
    if (few_groups && listed && n_near == chunks && n_near * CHUNK > LIST) {       // (short rows: a floor from their elements)
        float own = -INFINITY;
        runs_of(tid, 256, n_near, near_chunk, nothing, [&](const float (&v)[8], int) {
#pragma unroll
            for (int e = 0; e < 8; ++e) own = fmaxf(own, v[e]);
        });
        if (wave < 4) sh.group_max[tid] = own;
        __syncthreads();
        floor_logit = reached_logit(reached(sh.group_max, top), lowest);
    }
    runs(listed ? n_near : 0, near_chunk, sums, push);
    __syncthreads();
    const Sums sum = {red_s[0] + red_s[1] + red_s[2] + red_s[3], red_t[0] + red_t[1] + red_t[2] + red_t[3]};
    const double log_s = log(sum.s);
    if (tid < n_tokens) a.logprobs[r * n_tokens + tid] = logprob_of(given, m, log_s);
    for (int i = tid + 256; i < n_tokens; i += 256) {
        const int32_t t = a.tokens[r * n_tokens + i];
        a.logprobs[r * n_tokens + i] = t >= 0 && t < V ? logprob_of(to_f32(row[t]), m, log_s) : -INFINITY;
    }
    if (tid == 0 && a.entropy) a.entropy[r] = m > -INFINITY ? (float)fmax(0.0, log_s - sum.t / sum.s) : 0.f;
    if (top == 0) return;

    int n = count;
    if (!listed || n > LIST) {
        // exactly: the chunks that hold the first tokens, as keys of (largest logit, chunk).  (More than a list holds: in turns, the best so far among
        // them.)
        for (int c0 = 0; c0 < chunks; c0 += RUNS - MAX_TOP) {
            const int in = min(chunks - c0, RUNS - MAX_TOP), more = c0 ? MAX_TOP : 0;
            __syncthreads();
            for (int i = tid; i < in; i += 256) {
                const float c = cm[c0 + i];
                keys[i] = c >= lowest ? order_key(c, c0 + i) : 0;
            }
            if (tid < more) keys[in + tid] = best[tid];
            __syncthreads();
            if (tid < more) best[tid] = 0;
            largest(keys, in + more, top, best, ranks);
        }
        __syncthreads();
        if (tid == 0) count = 0;
        const int n_chunks = __popcll(__ballot(lane < top && best[lane] != 0));
        // (as many elements as tokens are wanted are as large as this)
        floor_logit = n_chunks == top ? key_logit(best[top - 1]) : lowest;
        auto best_chunk = [&](int i) { return (int)(uint32_t)~best[i]; };
        __syncthreads();
        runs(n_chunks, best_chunk, nothing, push);
        __syncthreads();
        n = count;
        if (n > LIST) {
            // many as large as that: first the runs of 8 that hold the answer, by their first and largest element
            __syncthreads();
            if (tid == 0) count = 0;
            __syncthreads();
            runs(n_chunks, best_chunk, nothing, [&](const float (&v)[8], int at) {
                unsigned long long k = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned long long ke = v[e] >= floor_logit ? order_key(v[e], at + e) : 0;
                    k = ke > k ? ke : k;
                }
                if (k) keys[atomicAdd(&count, 1)] = k;
            });
            __syncthreads();
            const int n_runs = count;
            if (tid < MAX_TOP) best[tid] = 0;
            largest(keys, n_runs, top, best, ranks);
            __syncthreads();
            if (tid == 0) count = 0;
            __syncthreads();
            for (int i = tid; i < top * 8; i += 256) {
                if (!best[i >> 3]) continue;
                const int at = (int)((uint32_t)~best[i >> 3] & ~7u) + (i & 7);
                const float l = at < V ? to_f32(row[at]) : -INFINITY;
                const unsigned long long k = l >= floor_logit ? order_key(l, at) : 0;
                if (k) keys[atomicAdd(&count, 1)] = k;
            }
            __syncthreads();
            n = count;
        }
        if (tid < MAX_TOP) best[tid] = 0;
    }
    largest(keys, n, top, best, ranks);
    __syncthreads();
    if (tid < top) {
        const unsigned long long k = best[tid];
        a.top_tokens[r * top + tid] = k ? (int32_t)(uint32_t)~k : -1;
        a.top_logprobs[r * top + tid] = k ? logprob_of(key_logit(k), m, log_s) : -INFINITY;
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(ROW_THREADS) logprob_rows_kernel(const T* __restrict__ logits, int64_t ld, int V, int pieces, int chunks,
                                                           const Stats* __restrict__ stats, const float* __restrict__ chunk_max, const RowAnswer a) {
    extern __shared__ unsigned long long keys[];
    __shared__ RowShared sh;
    const int64_t r = blockIdx.x;
    answer_row<T, VEC>(logits + r * ld, r, V, pieces, chunks, stats + r * pieces, chunk_max + r * chunks, a, keys, sh);
}

// Pieces and answer of a row by one workgroup, sums and largest logits in LDS, one launch; the same arithmetic in the same order as by the two
// kernels.  For rows of up to 2^16 logits that all run at once, two a compute unit: a launch less; and for so many long rows of float32 that the next
// row's logits are read while one is answered.  Five alternatives, us against the two kernels, calls from a graph: one row of 1000 9.8 / 11.1, of 8000
// 8.5 / 9.8, of 32000 9.9 / 10.1, of 65536 11.3 / 8.8 (there the launch saved is no longer what the row's eight wavefronts take longer); bf16 rows: 64 of
// 32000 10.4 / 10.6, of 65536 12.4 / 9.8, 256 of 32000 11.9 / 13.5, of 65536 14.3 / 15.2, 512 of 32000 16.0 / 17.2, of 65536 20.8 / 20.8; 512 float32
// rows of 1000 11.4 / 13.8, of 65536 31.3 / 31.8.  By calls: 700 rows of 1000 19.5 / 15.6 (half of the wavefronts only wait during the answer), 64 of
// 128256 20.2 / 15.8; float32 rows of 128256: 512 54 / 54, 768 75.7 / 77.6, 2048 181 / 198; of 65536: 1024 55.5 / 53.8, 1536 76 / 83; 2048 bf16 rows of 152064 128 / 125.
constexpr int WHOLE_WAVES = 8, WHOLE_CHUNKS = 1024;            // (rows of up to 2^19 logits)
template <typename T>
inline bool whole_rows(int64_t rows, int pieces, int chunks) {
    return (pieces <= 32 && rows <= 512) || (sizeof(T) == 4 && pieces >= 32 && rows * pieces >= 48000 && chunks <= WHOLE_CHUNKS);
}
template <typename T, bool VEC>
__global__ void __launch_bounds__(64 * WHOLE_WAVES, 4) logprob_whole_kernel(const T* __restrict__ logits, int64_t ld, int V, int pieces, int chunks, const RowAnswer a) {
    extern __shared__ unsigned long long keys[];
    __shared__ RowShared sh;
    __shared__ Stats st[WHOLE_CHUNKS / PER_WAVE];
    __shared__ float cm[WHOLE_CHUNKS];
    const int64_t r = blockIdx.x;
    const T* row = logits + r * ld;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float v[PER_WAVE][8], next[PER_WAVE][8];
    if (wave < pieces) load_piece<T, VEC>(row, wave, V, v);
    for (int p = wave; p < pieces; p += 2 * WHOLE_WAVES) {     // (the next piece on its way)
        if (p + WHOLE_WAVES < pieces) load_piece<T, VEC>(row, p + WHOLE_WAVES, V, next);
        const Stats x = piece_stats(v, p, a.top ? cm : nullptr, chunks);
        if ((threadIdx.x & 63) == 0) st[p] = x;
        if (p + WHOLE_WAVES >= pieces) break;
        if (p + 2 * WHOLE_WAVES < pieces) load_piece<T, VEC>(row, p + 2 * WHOLE_WAVES, V, v);
        const Stats y = piece_stats(next, p + WHOLE_WAVES, a.top ? cm : nullptr, chunks);
        if ((threadIdx.x & 63) == 0) st[p + WHOLE_WAVES] = y;
    }
    __syncthreads();
    answer_row<T, VEC>(row, r, V, pieces, chunks, st, cm, a, keys, sh);
}

inline int pieces_of(int V) { return (V + PIECE - 1) / PIECE; }
inline int chunks_of(int V) { return (V + CHUNK - 1) / CHUNK; }

template <typename T, bool VEC>
void run(const T* logits, int64_t ld, int64_t rows, int V, const RowAnswer& a, void* scratch, hipStream_t s) {
    const int pieces = pieces_of(V), chunks = chunks_of(V), lds = a.top ? (RUNS + 32) * 8 : 0;
    if (whole_rows<T>(rows, pieces, chunks)) {
        hipLaunchKernelGGL((logprob_whole_kernel<T, VEC>), dim3((unsigned)rows), dim3(64 * WHOLE_WAVES), lds, s, logits, ld, V, pieces, chunks, a);
        return;
    }
    Stats* stats = (Stats*)scratch;
    float* cm = a.top ? (float*)(stats + rows * pieces) : nullptr;
    const int64_t total = rows * pieces;
    hipLaunchKernelGGL((logprob_pieces_kernel<T, VEC>), dim3((unsigned)((total + 3) / 4)), dim3(256), 0, s, logits, ld, V, pieces, total, stats,
                       cm, chunks);
    hipLaunchKernelGGL((logprob_rows_kernel<T, VEC>), dim3((unsigned)rows), dim3(ROW_THREADS), lds, s, logits, ld, V, pieces, chunks, stats, cm, a);
}

}  // namespace

bool token_logprobs_fits(int64_t rows, int V) { return (rows * pieces_of(V) + 3) / 4 <= MAX_WORKGROUPS_256; }

size_t token_logprobs_scratch(int64_t rows, int V, int top) {
    return (size_t)rows * ((size_t)pieces_of(V) * sizeof(Stats) + (top ? (size_t)chunks_of(V) * 4 : 0));
}

void launch_token_logprobs(int dtype, const void* logits, int64_t ld, int64_t rows, int V, const int32_t* tokens, int n_tokens, int top,
                           float* logprobs, float* entropy, int32_t* top_tokens, float* top_logprobs, void* scratch, hipStream_t s) {
    const int esz = dtype == 0 ? 4 : 2;
    const bool vec = (uintptr_t)logits % 16 == 0 && (rows == 1 || ld * esz % 16 == 0);
    const RowAnswer a = {tokens, n_tokens, logprobs, entropy, top, top_tokens, top_logprobs};
#define PO_RUN(T, VEC) run<T, VEC>((const T*)logits, ld, rows, V, a, scratch, s)
    if (dtype == 0) { if (vec) PO_RUN(float, true); else PO_RUN(float, false); }
    else { if (vec) PO_RUN(bf16_t, true); else PO_RUN(bf16_t, false); }
#undef PO_RUN
}

// ------------------------------------------------------------------ through the LM head
// The product leaves (m, S, T) of blocks of 256 or 128 columns (launch_gemm_logprob, launch_head_logprob_f32).
namespace {

__device__ __forceinline__ void head_answer(const Sums& sum, float m, float at, const int32_t* tokens, int V, int64_t r, float* logprobs, float* entropy) {
    const double log_s = log(sum.s);
    if (entropy) entropy[r] = m > -INFINITY ? (float)fmax(0.0, log_s - sum.t / sum.s) : 0.f;
    if (logprobs) {
        const int32_t t = tokens[r];
        logprobs[r] = t >= 0 && t < V ? logprob_of(at, m, log_s) : -INFINITY;
    }
}

// a row's answer from its blocks' planes [blocks][rows]: R rows (a power of two) side by side in a workgroup, 256 / R threads a row (one row of 1002 blocks 5 us,
// 150 of 1188 10, 4001 of 501 20)
__global__ void __launch_bounds__(256) head_blocks_kernel(const float* __restrict__ stats, int64_t plane, int blocks, int R, const float* __restrict__ at,
                                                          const int32_t* __restrict__ tokens, int V, int64_t rows, float* __restrict__ logprobs,
                                                          float* __restrict__ entropy) {
    constexpr float LN2 = 0.693147181f;
    __shared__ float ms[4][16];
    __shared__ double ss[4][16], ts[4][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, parts = 256 / R, at_r = tid % R;
    const int64_t r = (int64_t)blockIdx.x * R + at_r, rr = r < rows ? r : rows - 1;
    // a thread's blocks, four loads under way together
    float m = -INFINITY;
    Sums sum = {0.0, 0.0};
    for (int i0 = tid / R; i0 < blocks; i0 += 4 * parts) {
        Stats q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * parts;
            q[u] = Stats{-INFINITY, 0.f, 0.f, 0.f};
            if (i < blocks) {
                const float* g = stats + i * rows + rr;
                q[u] = Stats{g[0], g[plane], g[2 * plane], 0.f};
            }
        }
        const float more = fmaxf(fmaxf(fmaxf(q[0].m, q[1].m), fmaxf(q[2].m, q[3].m)), m);
        sum = moved(sum, m, more);
        m = more;
#pragma unroll
        for (int u = 0; u < 4; ++u) join(Stats{q[u].m, q[u].s, q[u].t * LN2, 0.f}, m, sum);
    }
    // over the lanes of a row, then over the wavefronts
    float top = m;
    for (int off = 32; off >= R; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    if (lane < R) ms[wave][lane] = top;
    __syncthreads();
    top = fmaxf(fmaxf(ms[0][at_r], ms[1][at_r]), fmaxf(ms[2][at_r], ms[3][at_r]));
    sum = moved(sum, m, top);
    for (int off = 32; off >= R; off >>= 1) {
        sum.s += __shfl_xor(sum.s, off);
        sum.t += __shfl_xor(sum.t, off);
    }
    if (lane < R) { ss[wave][lane] = sum.s; ts[wave][lane] = sum.t; }
    __syncthreads();
    if (tid < R && r < rows) {
        sum = {ss[0][tid] + ss[1][tid] + ss[2][tid] + ss[3][tid], ts[0][tid] + ts[1][tid] + ts[2][tid] + ts[3][tid]};
        head_answer(sum, top, logprobs ? at[r] : 0.f, tokens, V, r, logprobs, entropy);
    }
}

}  // namespace

static int head_blocks(int dtype, int64_t rows, int V, int d) { return dtype == 0 ? head_logprob_f32_blocks(rows, V) : gemm_logprob_blocks(rows, V, d); }

size_t head_logprobs_scratch(int dtype, int64_t rows, int V, int d) { return (size_t)rows * ((size_t)head_blocks(dtype, rows, V, d) * 12 + 4); }

void launch_head_logprobs(int dtype, const void* x, const void* w, int64_t rows, int V, int d, const int32_t* tokens, float* logprobs,
                          float* entropy, void* scratch, hipStream_t s) {
    const int blocks = head_blocks(dtype, rows, V, d);
    const int64_t plane = (int64_t)blocks * rows;
    float* stats = (float*)scratch;
    float* at = stats + 3 * plane;
    if (dtype == 0) launch_head_logprob_f32((const float*)x, (const float*)w, stats, tokens, at, rows, V, d, s);
    else launch_gemm_logprob((const bf16_t*)x, d, (const bf16_t*)w, d, stats, tokens, at, rows, V, d, s);
    // (as many workgroups as fill the card, before whole lines of a plane; us with R 1 / 16: 1 row 5.3 / 26, 150 rows 10 / 38, 4001 rows 39 / 20)
    int R = 1;
    while (R < 16 && rows >= 800 * R) R *= 2;
    hipLaunchKernelGGL(head_blocks_kernel, dim3((unsigned)((rows + R - 1) / R)), dim3(256), 0, s, stats, plane, blocks, R, at, tokens, V, rows, logprobs, entropy);
}

}  // namespace po
