// Drawing one token per row of float32 logits, with temperature, top-k, top-p and min-p, from one given random number a row
// (gfx950).
//
// With m the row's largest logit, w_i = exp((l_i - m) / T).  Tokens are ordered by l descending, equal ones by index; what may
// be drawn is a beginning of that order: the first top_k; of those the shortest beginning whose sum of w is at least top_p times
// the sum of the top_k; of those the ones with w >= min_p; the first one always.  The token is the first kept one, by index, at
// which the running sum of kept w exceeds u times their whole sum.
//
// Whole numbers come out, so sums and comparisons are float64 throughout: an error of 1e-7 in a running sum over 10^5 tokens
// would move a draw to its neighbour once in a hundred.  (Bins, which many threads add to in any order, count whole numbers of 44
// binary digits a weight, 38 with 2^24 logits.)  The exponential is the only costly part (a float64 operation takes a compute unit
// a cycle per wavefront): 2^y by a table of 256 values of 2^(j / 256) in LDS and a polynomial of degree 4, about 16 operations.  Its
// relative error at exp(-x) is below 4e-16 + x 2^-52 (against 64-bit mantissas, 2 10^7 random x up to 70): the exponent's own
// rounding is most of it.
//
// A row is cut into parts, a workgroup each, so that few rows use many compute units, and goes through up to four launches:
//   1  parts: nothing but a temperature: every tile's weight (SUB logits), its own largest logit for reference.  top_k up to
//      K_MAX: the part's own first top_k, found by counting leading bits of keys; the row's are among the parts'.  Otherwise
//      the part's extremes.
//   2  parts, where top_p (or a larger top_k) decides: tokens and weight in 4096 equal steps of the logit below the row's largest.
//   3  rows: the head of the order that holds everything kept, gathered and sorted in LDS, and the draw; or, where that is longer
//      than a list, the last kept token.
//   4  parts, for those rows: every tile's kept weight; the last workgroup of a row to finish draws.
// What bounds it: many rows, the float64 arithmetic of the weights (8 cycles an operation and wavefront: 256 rows of 152064 without
// filters 64 us, of which reading takes 25; 112 with min_p, 217 with top_p, whose rows are weighed three times; 48 greedy); few rows,
// four launches and the steps within them, each a wait for memory or a barrier: one row of 128256 with top_k and top_p 32 us, with
// top_p alone 56, with min_p 25, greedy 9.  64 rows of mixed settings 99.  A row a workgroup (no parts) took 60, 176 and 178 us where
// these take 32, 99 and 64.
#include "po_internal.h"

#include <float.h>

#include <algorithm>
#include <type_traits>

namespace po {
namespace {

constexpr int NT = 1024;            // threads of a workgroup: one part of a row
constexpr int NWAVE = NT / 64;
constexpr int BINS = 4096;
constexpr int PER = BINS / NT;      // bins of a thread
constexpr int CAP = 4096;           // entries that are ordered in LDS
constexpr int MAX_TILES = 1024;
constexpr int SUB = 1024;           // logits that a wavefront reads at once, 16 a lane
constexpr int K_MAX = 1024;         // top_k up to which parts list their own first
constexpr int PART_CAP = 2048;      // tokens that a part may list
constexpr int MAX_PARTS = 16;

struct Shared {
    double table[256];
    double part[NWAVE];
    int ipart[NWAVE];
    unsigned long long wave_best[NWAVE];
    double scan_w[NT];
    int scan_n[NT];
    unsigned long long weight[BINS];        // of a bin, as a multiple of 2^(its reference exponent - fix)
    alignas(16) int count[BINS];
    unsigned long long list[CAP];           // key << 32 | ~index: descending order is the order of the tokens
    double tile[MAX_TILES];
    short ref[2048];                        // reference exponents of a digit's bins
    int n_list;
    int part_end[16];
    // answers of a search, written by the one thread that finds them
    int found;
    int above_n;
    double above_w, total_w;
    unsigned long long cut;
    double cut_sum;
};

// order-preserving integer of a logit (-0 as +0), 0 for what is never drawn: -inf and NaN
__device__ __forceinline__ uint32_t key_of(float l) {
    const uint32_t b = __float_as_uint(l + 0.0f);
    return l > -INFINITY ? (b & 0x80000000u ? ~b : b | 0x80000000u) : 0u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

struct Row {
    const float* z;
    int V, ts, tiles;               // a tile: ts consecutive logits, a wavefront's
    float top;                      // the largest logit
    double rate;                    // 256 log2(e) / T

    // exp((l - top) / T) of a logit that may be drawn
    __device__ __forceinline__ double weight(float l, const double* table) const {
        if (top == INFINITY) return l == top ? 1.0 : 0.0;                     // (wavefront-uniform)
        // 256 log2 of it; what is left below 2^-1090 is 0 (also where the product is no number)
        const double y = fmax(((double)l - (double)top) * rate, -280000.0);
        const double n = rint(y), f = y - n;                                  // 2^(f / 256), |f| <= 1/2: c = ln 2 / 256
        constexpr double c = 0.69314718055994530942 / 256.0;
        double q = fma(f, c * c * c * c / 24.0, c * c * c / 6.0);
        q = fma(q, f, c * c / 2.0);
        q = fma(q, f, c);
        const int i = (int)n;
        const double t = table[i & 255];
        return ldexp(fma(t * f, q, t), i >> 8);
    }
};

// the SUB logits from i0 on, lane l the ones at i0 + l, + 64, ..; -inf past the end.  (The sum quiets a signalling NaN, which the larger of
// it and a number would otherwise be; of a quiet one and a number it is the number.)
__device__ __forceinline__ void read_sub(const Row& r, int i0, float (&v)[16]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const int i = i0 + j * 64 + lane;
        const float x = r.z[min(i, r.V - 1)] + 0.0f;
        v[j] = i < r.V ? x : -INFINITY;
    }
}
// f(first index, the 16 logits of this lane) for every SUB of the logits [i0, i1) of the row (i0 a multiple of SUB), one after the other by
// each wavefront, AHEAD: the next one's logits on their way
template <bool AHEAD = true, typename F>
__device__ __forceinline__ void for_each_sub(const Row& r, int i0, int i1, F f) {
    i0 += (threadIdx.x >> 6) * SUB;
    float v[16], next[16];
    if (AHEAD && i0 < i1) read_sub(r, i0, next);
    for (; i0 < i1; i0 += NWAVE * SUB) {
        if (AHEAD) {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = next[j];
            if (i0 + NWAVE * SUB < i1) read_sub(r, i0 + NWAVE * SUB, next);
        } else {
            read_sub(r, i0, v);
        }
        f(i0, v);
    }
}
// f(logit, its index)
template <bool AHEAD = true, typename F>
__device__ __forceinline__ void for_each(const Row& r, int i0, int i1, F f) {
    for_each_sub<AHEAD>(r, i0, i1, [&](int i, const float (&v)[16]) {
#pragma unroll
        for (int j = 0; j < 16; ++j) f(v[j], i + j * 64 + (int)(threadIdx.x & 63));
    });
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// inclusive sums of (n, w) over the workgroup's threads, in sh.scan_n / scan_w
__device__ void block_scan(Shared& sh, int n, double w) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int a = __shfl_up(n, off);
        const double b = __shfl_up(w, off);
        if (lane >= off) { n += a; w += b; }
    }
    if (lane == 63) { sh.ipart[wave] = n; sh.part[wave] = w; }
    __syncthreads();
    int n0 = 0;
    double w0 = 0.0;
    for (int i = 0; i < wave; ++i) { n0 += sh.ipart[i]; w0 += sh.part[i]; }
    sh.scan_n[threadIdx.x] = n + n0;
    sh.scan_w[threadIdx.x] = w + w0;
    __syncthreads();
}

// What a search is after: the k-th token of an order (k > 0), or the first at which the running sum reaches `sum`, which is above 0
// so that no sum of nothing reaches it.
struct Goal {
    int k;
    double sum;
    __device__ __forceinline__ static Goal share(double p, double all) { return {0, fmax(p * all, DBL_MIN)}; }
    __device__ __forceinline__ bool reached(int n, double w) const { return k > 0 ? n >= k : w >= sum; }
};

// The first thread for which `yes` holds (it holds for some), `before` being its value for the thread in front.
__device__ __forceinline__ int first_thread(Shared& sh, bool yes, bool before) {
    if (threadIdx.x == 0) sh.found = NT;
    __syncthreads();
    if (yes && !before) atomicMin(&sh.found, (int)threadIdx.x);
    __syncthreads();
    const int f = sh.found;
    __syncthreads();
    return f;
}

// The bin of sh.count / sh.weight (bin 0 first, base_n / base_w in front of it) in which the goal is reached, the last one with
// a token where rounding leaves it a little out of reach; sh.above_n / above_w: what is in front of it; sh.total_w: all of it.
// goal(sum of the bins): a Goal; ref(b): a bin's reference exponent.
template <bool weights, typename G, typename Ref>
__device__ int find_bin(Shared& sh, G goal_of, int base_n, double base_w, int fix, Ref ref) {
    const int t = threadIdx.x;
    int n[PER], sum_n = 0;
    double w[PER], sum_w = 0.0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        n[j] = sh.count[t * PER + j];
        w[j] = weights ? ldexp((double)sh.weight[t * PER + j], ref(t * PER + j) - fix) : 0.0;
        sum_n += n[j];
        sum_w += w[j];
    }
    block_scan(sh, sum_n, sum_w);
    const int all = sh.scan_n[NT - 1];
    const Goal goal = goal_of(sh.scan_w[NT - 1]);
    int bn = t ? sh.scan_n[t - 1] : 0;
    double bw = base_w + (t ? sh.scan_w[t - 1] : 0.0);
    const bool yes = sh.scan_n[t] == all || goal.reached(base_n + sh.scan_n[t], base_w + sh.scan_w[t]);
    const bool before = t && (bn == all || goal.reached(base_n + bn, bw));
    if (t == first_thread(sh, yes, before)) {
        int j = 0, at = -1;
        int at_n = 0;
        double at_w = 0.0;
#pragma unroll
        for (j = 0; j < PER; ++j) {                   // the first of its bins that reaches it, else its last one with a token
            if (n[j] && (at < 0 || !goal.reached(base_n + bn, bw))) { at = j; at_n = bn; at_w = bw; }
            bn += n[j];
            bw += w[j];
        }
        sh.found = t * PER + max(at, 0);
        sh.above_n = base_n + at_n;
        sh.above_w = at < 0 ? bw : at_w;
        sh.total_w = sh.scan_w[NT - 1];
    }
    __syncthreads();
    const int b = sh.found;
    __syncthreads();
    return b;
}

// (behind a barrier: wavefronts still on their way from find_bin read the bin that it found)
__device__ void clear_bins(Shared& sh) {
    __syncthreads();
    for (int b = threadIdx.x; b < BINS; b += NT) { sh.count[b] = 0; sh.weight[b] = 0; }
    __syncthreads();
}

__device__ __forceinline__ void add_to_bin(Shared& sh, int b, double w, int digits) {
    atomicAdd(&sh.count[b], 1);                               // whole numbers: the order of the additions does not show
    const unsigned long long f = (unsigned long long)(ldexp(w, digits) + 0.5);      // (to the nearest: sums of many keep no bias)
    if (f) atomicAdd(&sh.weight[b], f);
}

// sh.list[0 .. n) in descending order, n <= E * NT (entries that are not 0 differ).  A bitonic order of m entries, a power of two: E
// in a thread's registers, entry e * NT + t the e-th of thread t, so that steps within a wavefront are shuffles, steps of NT and more
// need no exchange, and only those between wavefronts (10 of 55 at 1024 entries) go through LDS.
template <int E>
__device__ void sort_registers(Shared& sh, int n, int m) {
    const int t = threadIdx.x;
    unsigned long long x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = e * NT + t < n ? sh.list[e * NT + t] : 0;
    __syncthreads();
    const auto settle = [&](int e, unsigned long long o, int size, int half) {
        const int i = e * NT + t;
        const bool larger = ((i & half) == 0) == ((i & size) == 0);
        if ((o > x[e]) == larger) x[e] = o;
    };
    for (int size = 2; size <= m; size <<= 1) {
        if constexpr (E > 1) {
#pragma unroll
            for (int step = E / 2; step > 0; step >>= 1)
                if (step * NT < size) {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (!(e & step)) {
                            const unsigned long long lo = x[e], hi = x[e | step];
                            settle(e, hi, size, step * NT);
                            settle(e | step, lo, size, step * NT);
                        }
                }
        }
        for (int half = min(size, NT) >> 1; half >= 64; half >>= 1) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (t < m) sh.list[e * NT + t] = x[e];
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (t < m) settle(e, sh.list[e * NT + (t ^ half)], size, half);
            __syncthreads();
        }
        if (t < m) {
#pragma unroll
            for (int half = 32; half > 0; half >>= 1)
                if (half < size) {
#pragma unroll
                    for (int e = 0; e < E; ++e) settle(e, __shfl_xor(x[e], half), size, half);
                }
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e * NT + t < n) sh.list[e * NT + t] = x[e];
    __syncthreads();
}
__device__ void sort_list(Shared& sh, int n) {
    int m = 64;
    while (m < n) m <<= 1;
    if (m <= NT) sort_registers<1>(sh, n, m);
    else if (m == 2 * NT) sort_registers<2>(sh, n, m);
    else sort_registers<4>(sh, n, m);
}
static_assert(CAP == 4 * NT, "what sort_list orders");

// The token of the sorted sh.list[0 .. n) at which the goal is reached (base_n / base_w in front of the first; the last one where
// rounding leaves it out of reach): sh.cut, and sh.cut_sum, the running sum up to it.
__device__ void find_in_list(Shared& sh, const Row& r, const Goal& goal, int n, int base_n, double base_w) {
    const int t = threadIdx.x, per = (n + NT - 1) / NT, i0 = t * per, i1 = min(i0 + per, n);
    double w = 0.0;
    for (int i = i0; i < i1; ++i) w += r.weight(value_of((uint32_t)(sh.list[i] >> 32)), sh.table);
    block_scan(sh, max(i1 - i0, 0), w);
    int bn = t ? sh.scan_n[t - 1] : 0;
    double bw = base_w + (t ? sh.scan_w[t - 1] : 0.0);
    const bool yes = sh.scan_n[t] == n || goal.reached(base_n + sh.scan_n[t], base_w + sh.scan_w[t]);
    const bool before = t && (bn == n || goal.reached(base_n + bn, bw));
    if (t == first_thread(sh, yes, before)) {
        int i = i0;
        for (;; ++i) {
            bw += r.weight(value_of((uint32_t)(sh.list[i] >> 32)), sh.table);
            ++bn;
            if (i == i1 - 1 || goal.reached(base_n + bn, bw)) break;
        }
        sh.cut = sh.list[i];
        sh.cut_sum = bw;
    }
    __syncthreads();
}

// Float64 sums, in one order, of the weights of the tokens above a key and of all, and the number of tokens with that key.
struct Sums {
    double above, all;
    int equal;
};
__device__ Sums sums_at(Shared& sh, const Row& r, uint32_t key) {
    double above = 0.0, all = 0.0;
    int equal = 0;
    for_each<false>(r, 0, r.V, [&](float l, int) {
        const uint32_t x = key_of(l);
        const double w = x ? r.weight(l, sh.table) : 0.0;
        all += w;
        above += x > key ? w : 0.0;
        equal += x == key;
    });
    Sums s;
    block_scan(sh, 0, all);
    s.all = sh.scan_w[NT - 1];
    block_scan(sh, equal, above);
    s.above = sh.scan_w[NT - 1];
    s.equal = sh.scan_n[NT - 1];
    return s;
}

// The same over the whole row with nothing known, for bins that hold more tokens than a list: the key digit by digit (11, 11, 10
// bits), then the right one of the tokens with that key by a count of tiles.  p_of_all > 0: the goal is that share of all weights,
// and goal.sum near it.  sum_too: whether sh.cut_sum is wanted.
// Where the goal is a sum, bins count weights in whole numbers with their highest key for reference.  Keys with the same leading bits
// can be many powers of 2 apart, and what rounding takes from millions of weights can be worth a few others; so the key that this
// leads to is held against float64 sums, and where it is not the one (seen for two million logits) the keys 16, 256, .. on and then
// the middle of what is left are, at most 40 more.  One look at the sums is a pass without atomics: 35 of the 390 us of 128256 logits of
// the bf16 grid under top_p.
__device__ void find_in_row(Shared& sh, const Row& r, Goal goal, double p_of_all, bool sum_too, int fix) {
    const bool by_count = goal.k > 0;
    const uint32_t top = key_of(r.top);
    uint32_t key = 0;
    int base_n = 0;
    double base_w = 0.0;
    for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift == 10 ? 0 : -1) {
        const int bits = shift == 0 ? 10 : 11, last = (1 << bits) - 1;
        const uint32_t upper = shift == 21 ? 0u : 0xffffffffu << (shift + bits);
        clear_bins(sh);
        if (!by_count) {
            for (int b = threadIdx.x; b <= last; b += NT) {
                const double high = r.weight(value_of(min(key | (uint32_t)(last - b) << shift | ((1u << shift) - 1), top)), sh.table);
                sh.ref[b] = (short)(high > 0.0 ? ilogb(high) + 1 : -1000);
            }
            __syncthreads();
        }
        for_each<false>(r, 0, r.V, [&](float l, int) {
            const uint32_t x = key_of(l);
            if (!x || (x & upper) != key) return;
            const int b = last - (int)((x >> shift) & (uint32_t)last);
            if (by_count) atomicAdd(&sh.count[b], 1);
            else add_to_bin(sh, b, r.weight(l, sh.table), fix - sh.ref[b]);
        });
        __syncthreads();
        const auto same = [&](double) { return goal; };
        const int b = by_count ? find_bin<false>(sh, same, base_n, 0.0, 0, [](int) { return 0; })
                               : find_bin<true>(sh, same, base_n, base_w, fix, [&](int i) { return (int)sh.ref[i & 2047]; });
        key |= (uint32_t)(last - b) << shift;
        base_n = sh.above_n;
        base_w = sh.above_w;
        __syncthreads();
    }
    // tokens of this key: all of one weight; how many of them
    int ties = sh.count[1023 - (int)(key & 1023u)], want = goal.k - base_n;
    double w = 0.0;
    if (!by_count || sum_too) {
        uint32_t low = 1, high = top, step = 16;                 // keys between which it is, and how far to go from the last one
        bool reached = true;
        for (;;) {
            const Sums s = sums_at(sh, r, key);
            ties = s.equal;
            base_w = s.above;
            w = r.weight(value_of(key), sh.table);
            if (by_count || !reached) break;
            if (p_of_all > 0.0) goal = Goal::share(p_of_all, s.all);
            const bool enough = base_w + ties * w >= goal.sum;
            if (base_w < goal.sum && enough) break;
            if (base_w < goal.sum) high = key - 1;
            else low = key + 1;
            // (sums of these and of those above them, rounded each for itself: the goal between the two, reached by the last of them)
            reached = low <= high;
            const uint32_t middle = reached ? low + (high - low) / 2 : low;
            key = middle < key ? key - min(key - middle, step) : key + min(middle - key, step);
            step = min(step, 1u << 24) * 16;
        }
        if (!by_count) want = reached ? (int)fmin(ceil((goal.sum - base_w) / w), (double)ties) : ties;
    }
    want = max(1, min(want, ties));
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int a = wave; a < NT; a += NWAVE) {
        int n = 0;
        if (a < r.tiles)
            for (int i = a * r.ts + lane; i < min(r.V, (a + 1) * r.ts); i += 64) n += key_of(r.z[i]) == key;
        for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off);
        if (lane == 0) sh.count[a] = n;
    }
    __syncthreads();
    block_scan(sh, sh.count[threadIdx.x], 0.0);
    const int t = first_thread(sh, sh.scan_n[threadIdx.x] >= want, threadIdx.x && sh.scan_n[threadIdx.x - 1] >= want);
    if (wave == 0) {
        int seen = t ? sh.scan_n[t - 1] : 0;
        for (int i = t * r.ts; i < min(r.V, (t + 1) * r.ts) && seen < want; i += 64) {
            const bool tie = i + lane < min(r.V, (t + 1) * r.ts) && key_of(r.z[i + lane]) == key;
            const unsigned long long b = __ballot(tie);
            const int upto = seen + __popcll(b & (0xffffffffffffffffull >> (63 - lane)));
            if (tie && upto == want) {
                sh.cut = (unsigned long long)key << 32 | (uint32_t)~(i + lane);
                sh.cut_sum = base_w + want * w;
            }
            seen += __popcll(b);
        }
    }
    __syncthreads();
}

struct Answer {
    int* token;
    float* logprob;
    __device__ __forceinline__ void give(int t, double lp) const {
        *token = t;
        if (logprob) *logprob = (float)lp;
    }
};

__device__ __forceinline__ double target_of(float u, double all) {
    return (double)(u > 0.0f ? fminf(u, 1.0f - 0x1p-24f) : 0.0f) * all;      // (NaN: 0)
}

// The rest of the way when the n tokens at the head of the order are in sh.list: by_k: the first k of them, otherwise `total` is
// what top_p is a part of.
__device__ void finish_list(Shared& sh, const Row& r, int n, bool by_k, int k, bool by_p, double p, double total, double floor_w, float u,
                            const Answer& answer) {
    const int t = threadIdx.x;
    const auto weight = [&](uint32_t key) { return r.weight(value_of(key), sh.table); };
    sort_list(sh, n);
    const int nk = by_k ? min(k, n) : n, per = (nk + NT - 1) / NT, i0 = t * per, i1 = min(i0 + per, nk);
    int keep = nk;
    if (by_p) {
        double w = 0.0;
        for (int i = i0; i < i1; ++i) w += weight((uint32_t)(sh.list[i] >> 32));
        block_scan(sh, max(i1 - i0, 0), w);
        const double goal = fmax(p * (by_k ? sh.scan_w[NT - 1] : total), DBL_MIN);       // (above 0: no sum of nothing reaches it)
        const bool yes = sh.scan_n[t] == nk || sh.scan_w[t] >= goal;
        const bool before = t && (sh.scan_n[t - 1] == nk || sh.scan_w[t - 1] >= goal);
        if (t == first_thread(sh, yes, before)) {
            double c = t ? sh.scan_w[t - 1] : 0.0;
            int i = i0;
            for (;; ++i) {
                c += weight((uint32_t)(sh.list[i] >> 32));
                if (i == i1 - 1 || c >= goal) break;
            }
            sh.above_n = i + 1;
        }
        __syncthreads();
        keep = sh.above_n;
    }
    // by index: ~index << 32 | key, what is not kept at the end
    for (int i = t; i < n; i += NT) {
        const unsigned long long e = sh.list[i];
        const uint32_t key = (uint32_t)(e >> 32);
        const bool kept = i < keep && (i == 0 || floor_w <= 0.0 || weight(key) >= floor_w);
        sh.list[i] = kept ? (unsigned long long)(uint32_t)e << 32 | key : 0;
    }
    __syncthreads();
    sort_list(sh, keep);
    const int per2 = (keep + NT - 1) / NT, j0 = t * per2, j1 = min(j0 + per2, keep);
    double w = 0.0;
    int some = 0;
    for (int i = j0; i < j1; ++i)
        if (sh.list[i]) { w += weight((uint32_t)sh.list[i]); ++some; }
    block_scan(sh, some, w);
    const int kept = sh.scan_n[NT - 1];
    const double all = sh.scan_w[NT - 1], target = target_of(u, all);
    const bool yes = sh.scan_n[t] == kept || sh.scan_w[t] > target;
    const bool before = t && (sh.scan_n[t - 1] == kept || sh.scan_w[t - 1] > target);
    if (t == first_thread(sh, yes, before)) {
        double c = t ? sh.scan_w[t - 1] : 0.0, wi = 0.0;
        int i = j0;
        for (;; ++i) {
            wi = weight((uint32_t)sh.list[i]);
            c += wi;
            if (i == j0 + some - 1 || (wi > 0.0 && c > target)) break;
        }
        answer.give((int)~(uint32_t)(sh.list[i] >> 32), log(wi / all));
    }
}

// Of the threads with a weight (w > 0, at least one), scanned by block_scan(sh, w > 0, w), the first at which the sum, `run` in
// front of it, exceeds target, or the last where none does (*past).  (Sums of neighbours are added up in different orders: one
// without a weight may seem to be past the target a rounding early.)
__device__ __forceinline__ int first_past(Shared& sh, bool has, double run, double target, bool* past) {
    const int t = threadIdx.x, some = sh.scan_n[NT - 1];
    const bool yes = sh.scan_n[t] == some || run + sh.scan_w[t] > target;
    const bool before = t && (sh.scan_n[t - 1] == some || run + sh.scan_w[t - 1] > target);
    const int f = first_thread(sh, yes, before);
    *past = run + sh.scan_w[f] > target;
    const int in_front = f ? sh.scan_n[f - 1] : 0;
    return first_thread(sh, t >= f && has, t > f && sh.scan_n[t - 1] > in_front);
}

// The token once sh.tile holds the kept weight of every tile (not all of them 0).  kept(logit, index): its weight, or 0.
template <typename F>
__device__ void finish_tiles(Shared& sh, const Row& r, float u, const Answer& answer, F kept) {
    const int t = threadIdx.x;
    const double mine = t < r.tiles ? sh.tile[t] : 0.0;
    block_scan(sh, mine > 0.0, mine);
    const double all = sh.scan_w[NT - 1], target = target_of(u, all);
    bool past;
    const int a = first_past(sh, mine > 0.0, 0.0, target, &past);
    double run = a ? sh.scan_w[a - 1] : 0.0, w_last = 1.0;
    int token = -1;                                      // (the last kept one so far stands in where rounding leaves the target out of reach)
    __syncthreads();
    for (int i0 = a * r.ts; i0 < min(r.V, (a + 1) * r.ts); i0 += NT) {
        const int i = i0 + t;
        const double w = i < r.V ? kept(r.z[i], i) : 0.0;
        block_scan(sh, w > 0.0, w);
        const double end = sh.scan_w[NT - 1];
        if (sh.scan_n[NT - 1]) {
            const int f = first_past(sh, w > 0.0, run, target, &past);
            if (t == f) { sh.above_n = i; sh.above_w = w; }
            __syncthreads();
            token = sh.above_n;
            w_last = sh.above_w;
            __syncthreads();
            if (past) break;
        }
        run += end;
    }
    if (t == 0) answer.give(token, log(w_last / all));
}

// What the launches hand on, in the caller's scratch; arrays of a row one behind the other.
struct Handover {
    unsigned long long* best;        // [row][part] the part's first token (an entry of a list; 0: none)
    uint32_t* least;                 // [row][part] lowest key of what may be drawn
    int* listed;                     // [row][part] tokens of list, PART_CAP + 1: more than it holds
    unsigned long long* list;        // [row][part][PART_CAP]
    double* tile;                    // [row][MAX_TILES] weight of a tile
    float* tile_top;                 // [row][MAX_TILES]
    int* count;                      // [row][part][BINS]
    unsigned long long* weight;      // [row][part][BINS]
    unsigned long long* first;       // [row] the row's first token where the fourth launch has to see to it, else 0
    unsigned long long* cut;         // [row] ... and the last kept one (0: all)
    int* finished;                   // [row][2] parts that have finished the third, and the fourth, launch
};
struct Call {
    const float* logits;
    int64_t ld;
    int V, ts, fix, parts, part_len;
    const float *u, *temperature;
    const int* top_k;
    const float *top_p, *min_p;
    int* tokens;
    float* logprobs;
    Handover h;
};

enum How { GREEDY, FREE, COUNT, WEIGH, KEEP };      // KEEP: min_p alone
struct Settings {
    float T, p, u;
    int k;
    double floor_w;
    bool by_k, by_p;
    How how;
    __device__ Settings(const Call& c, int row) {
        T = c.temperature ? c.temperature[row] : 1.0f;
        k = c.top_k ? c.top_k[row] : 0;
        p = c.top_p ? c.top_p[row] : 1.0f;
        u = c.u[row];
        floor_w = c.min_p && c.min_p[row] > 0.0f ? (double)c.min_p[row] : 0.0;      // (NaN: off)
        by_k = k > 0 && k < c.V;
        by_p = p < 1.0f;
        how = !(T > 0.0f) ? GREEDY : by_k && k <= K_MAX ? COUNT : by_k || by_p ? WEIGH : floor_w > 0.0 ? KEEP : FREE;
    }
};

__device__ __forceinline__ Row row_of(const Call& c, int row, const Settings& s) {
    Row r;
    r.z = c.logits + (int64_t)row * c.ld;
    r.V = c.V;
    r.ts = c.ts;
    r.tiles = (c.V + c.ts - 1) / c.ts;
    r.top = 0.f;
    r.rate = fmin(256.0 * 1.4426950408889634074 / (double)s.T, 1e300);        // (0 * infinity would be none)
    return r;
}

__device__ __forceinline__ Answer answer_of(const Call& c, int row) { return {c.tokens + row, c.logprobs ? c.logprobs + row : nullptr}; }

__device__ __forceinline__ void fill_table(Shared& sh) {
    if (threadIdx.x < 256) sh.table[threadIdx.x] = exp2((double)threadIdx.x / 256.0);
    __syncthreads();
}

// the largest of a workgroup's values
__device__ __forceinline__ unsigned long long block_max(Shared& sh, unsigned long long v) {
    for (int off = 32; off > 0; off >>= 1) {
        const unsigned long long o = __shfl_xor(v, off);
        v = o > v ? o : v;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.wave_best[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int i = 0; i < NWAVE; ++i) v = sh.wave_best[i] > v ? sh.wave_best[i] : v;
    return v;
}

// Between the workgroups of a row within a launch: what one writes for another goes past the caches (hand / handed), each wavefront
// waits until its own has arrived, and one thread counts the workgroup in.  -> whether it is the last, which then finds everything.
__device__ __forceinline__ void hand(unsigned long long* p, unsigned long long v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void hand(int* p, int v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void hand(double* p, double v) { hand((unsigned long long*)p, (unsigned long long)__double_as_longlong(v)); }
template <typename V>
__device__ __forceinline__ V handed(V* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ bool last_to_finish(Shared& sh, int* counter, int parts) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) sh.found = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const bool last = sh.found == parts - 1;
    __syncthreads();
    return last;
}

// ---- launch 1
__global__ void __launch_bounds__(NT) sample_parts_kernel(const Call c) {
    __shared__ Shared sh;
    const int row = blockIdx.x / c.parts, part = blockIdx.x - row * c.parts, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const Settings s(c, row);
    const Row r = row_of(c, row, s);
    const int c0 = part * c.part_len, c1 = min(c.V, c0 + c.part_len);
    const int64_t at = (int64_t)row * c.parts + part;
    if (part == 0 && t < 2) c.h.finished[row * 2 + t] = 0;
    if (part == 0 && t == 0) c.h.first[row] = 0;             // (until it is known that the fourth launch has to see to this row)
    if (s.how == FREE) {
        fill_table(sh);
        // a SUB's weight with its own largest logit for reference, added to its tile's (of one SUB, up to 2^20 logits)
        const auto weigh = [&](const float (&v)[16], Row& q, double& w) {
            float m = -INFINITY;
#pragma unroll
            for (int j = 0; j < 16; ++j) m = fmaxf(m, v[j]);                       // (of a NaN and a number the number)
            for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
            if (m == -INFINITY) return;
            if (m > q.top) {
                const float old = q.top;
                q.top = m;
                w *= old == -INFINITY ? 0.0 : q.weight(old, sh.table);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) w += v[j] > -INFINITY ? q.weight(v[j], sh.table) : 0.0;
        };
        const auto put = [&](int a, const Row& q, double w) {
            w = wave_sum(w);
            if (lane == 0) { c.h.tile[(int64_t)row * MAX_TILES + a] = w; c.h.tile_top[(int64_t)row * MAX_TILES + a] = q.top; }
        };
        Row q = r;
        if (c.ts == SUB) {
            for_each_sub(r, c0, c1, [&](int i0, const float (&v)[16]) {
                q.top = -INFINITY;
                double w = 0.0;
                weigh(v, q, w);
                put(i0 / SUB, q, w);
            });
            return;
        }
        for (int a = c0 / c.ts + wave; a * c.ts < c1; a += NWAVE) {
            q.top = -INFINITY;
            double w = 0.0;
            for (int i0 = a * c.ts; i0 < min(c.V, (a + 1) * c.ts); i0 += SUB) {
                float v[16];
                read_sub(r, i0, v);
                weigh(v, q, w);
            }
            put(a, q, w);
        }
        return;
    }
    // the largest logit of a thread, and the SUB it is in; the lowest that may be drawn
    float m = -INFINITY, low = INFINITY;
    int where = 0;
    float kept[16];                                          // the logits of a part that its wavefronts read at once
    const bool once = c1 - c0 <= NWAVE * SUB;
    if (s.how == COUNT) clear_bins(sh);
    for_each_sub(r, c0, c1, [&](int i0, const float (&v)[16]) {
#pragma unroll
        for (int j = 0; j < 16; ++j) kept[j] = v[j];
        float mi = -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; ++j) mi = fmaxf(mi, v[j]);
        if (mi > m) { m = mi; where = i0; }
        if (s.how == WEIGH) {
#pragma unroll
            for (int j = 0; j < 16; ++j) low = fminf(low, v[j] > -INFINITY ? v[j] : INFINITY);
        } else if (s.how == COUNT) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const uint32_t key = key_of(v[j]);
                if (key) atomicAdd(&sh.count[BINS - 1 - (key >> 20)], 1);
            }
        }
    });
    unsigned long long best = 0;
    if (m > -INFINITY) {
        if (!once) read_sub(r, where, kept);
        int i = where + lane;                                    // (one of the 16 of this thread in that SUB)
#pragma unroll
        for (int j = 15; j >= 0; --j) i = kept[j] == m ? where + lane + j * 64 : i;
        best = (unsigned long long)key_of(m) << 32 | (uint32_t)~i;
    }
    best = block_max(sh, best);
    if (t == 0) c.h.best[at] = best;
    if (s.how == WEIGH) {
        // (all of a thread's may be +inf: m; or none be there)
        const unsigned long long l = block_max(sh, m > -INFINITY ? (unsigned long long)~key_of(low == INFINITY ? m : low) : 0ull);
        if (t == 0) c.h.least[at] = best ? ~(uint32_t)l : 0xffffffffu;
    }
    if (s.how != COUNT) return;
    // the bin of the part's k-th token, and, where the part's first up to that bin are too many for its list (all but a few logits
    // close together), the same by the next 12 bits of the key
    const auto kth = [&](int in_front) {
        return find_bin<false>(sh, [&](double) { return Goal{s.k, 0.0}; }, in_front, 0.0, 0, [](int) { return 0; });
    };
    const uint32_t high = BINS - 1 - kth(0);
    uint32_t lowest = high << 20;
    int in_front = sh.above_n, n = in_front + sh.count[BINS - 1 - high];
    __syncthreads();
    if (n > PART_CAP) {
        clear_bins(sh);
        for_each(r, c0, c1, [&](float l, int) {
            const uint32_t key = key_of(l);
            if (key && key >> 20 == high) atomicAdd(&sh.count[BINS - 1 - (key >> 8 & (BINS - 1))], 1);
        });
        __syncthreads();
        const int b = kth(in_front);
        lowest |= (uint32_t)(BINS - 1 - b) << 8;
        n = sh.above_n + sh.count[b];
        __syncthreads();
    }
    if (n <= PART_CAP && best) {
        if (t == 0) sh.n_list = 0;
        __syncthreads();
        const auto put = [&](float l, int i) {
            const uint32_t key = key_of(l);
            if (key && key >= lowest) c.h.list[at * PART_CAP + atomicAdd(&sh.n_list, 1)] = (unsigned long long)key << 32 | (uint32_t)~i;
        };
        if (!once) {
            for_each(r, c0, c1, put);
        } else if (c0 + wave * SUB < c1) {
#pragma unroll
            for (int j = 0; j < 16; ++j) put(kept[j], c0 + wave * SUB + j * 64 + lane);
        }
    }
    if (t == 0) c.h.listed[at] = best == 0 ? 0 : n <= PART_CAP ? n : PART_CAP + 1;
}

// ---- the row's first token, and the steps of logits that its weights are counted in
static_assert(MAX_PARTS <= 16, "a lane each");
__device__ __forceinline__ unsigned long long first_of(const Call& c, int row) {
    const int lane = threadIdx.x & 15;
    unsigned long long best = lane < c.parts ? c.h.best[(int64_t)row * c.parts + lane] : 0;
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) {
        const unsigned long long o = __shfl_xor(best, off, 16);
        best = o > best ? o : best;
    }
    return best;
}
// Over all logits, or down to where no weight counts any more (the last bin takes the rest).
struct Steps {
    float top, scale;
    double step;
    __device__ Steps(const Call& c, int row, const Row& r, float T) {
        const int lane = threadIdx.x & 15;
        uint32_t least = lane < c.parts ? c.h.least[(int64_t)row * c.parts + lane] : 0xffffffffu;
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) least = min(least, (uint32_t)__shfl_xor((int)least, off, 16));
        top = r.top;
        const double span = fmin((double)top - (double)value_of(least), 64.0 * fmax((double)T, 1.0));
        scale = span > 0.0 && top < INFINITY ? (float)(BINS / span) : 0.0f;
        step = scale > 0.0f ? r.rate / 256.0 / (double)scale : 0.0;
    }
    __device__ __forceinline__ int bin(float l) const {
        const float x = (top - l) * scale;
        return x < (float)(BINS - 1) ? (int)x : BINS - 1;
    }
    // no weight in a bin is above that of its upper edge; 1 for what the steps' own rounding moves across edges
    __device__ __forceinline__ int ref(int b) const { return (int)fmax(ceil(-(double)b * step), -1000.0) + 1; }
};

template <bool AHEAD>
__device__ void fill_bins(Shared& sh, const Row& r, const Steps& st, int c0, int c1, int fix) {
    clear_bins(sh);
    for_each<AHEAD>(r, c0, c1, [&](float l, int) {
        if (l > -INFINITY) {
            const int b = st.bin(l);
            add_to_bin(sh, b, r.weight(l, sh.table), fix - st.ref(b));
        }
    });
    __syncthreads();
}

// ---- launch 2
__global__ void __launch_bounds__(NT) sample_weigh_kernel(const Call c) {
    __shared__ Shared sh;
    const int row = blockIdx.x / c.parts, part = blockIdx.x - row * c.parts;
    const Settings s(c, row);
    if (s.how != WEIGH) return;
    Row r = row_of(c, row, s);
    const unsigned long long best = first_of(c, row);
    if (best == 0) return;
    r.top = value_of((uint32_t)(best >> 32));
    fill_table(sh);
    const Steps st(c, row, r, s.T);
    const int c0 = part * c.part_len;
    fill_bins<true>(sh, r, st, c0, min(c.V, c0 + c.part_len), c.fix);
    const int64_t at = ((int64_t)row * c.parts + part) * BINS;
    for (int b = threadIdx.x; b < BINS; b += NT) { c.h.count[at + b] = sh.count[b]; c.h.weight[at + b] = sh.weight[b]; }
}

// ---- launch 3
__global__ void __launch_bounds__(NT) sample_pick_kernel(const Call c) {
    __shared__ Shared sh;
    const int row = blockIdx.x / c.parts, part = blockIdx.x - row * c.parts, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const Settings s(c, row);
    if (part != 0 && !(s.how == WEIGH && !s.by_k)) return;   // (only top_p alone has work for more than one)
    Row r = row_of(c, row, s);
    const Answer answer = answer_of(c, row);
    fill_table(sh);
    if (s.how == FREE) {
        const float mine = t < r.tiles ? c.h.tile_top[(int64_t)row * MAX_TILES + t] : -INFINITY;
        float m = mine;
        for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
        if (lane == 0) sh.part[wave] = m;
        __syncthreads();
        for (int i = 0; i < NWAVE; ++i) m = fmaxf(m, (float)sh.part[i]);
        __syncthreads();
        if (m == -INFINITY) {
            if (t == 0) answer.give(-1, -INFINITY);
            return;
        }
        r.top = m;
        if (t < r.tiles) sh.tile[t] = mine == -INFINITY ? 0.0 : c.h.tile[(int64_t)row * MAX_TILES + t] * r.weight(mine, sh.table);
        __syncthreads();
        finish_tiles(sh, r, s.u, answer, [&](float l, int) { return l > -INFINITY ? r.weight(l, sh.table) : 0.0; });
        return;
    }
    const unsigned long long best = first_of(c, row);
    if (best == 0 || s.how == GREEDY) {                      // nothing to draw; or the most likely token
        if (part == 0 && t == 0) answer.give(best ? (int)~(uint32_t)best : -1, best ? 0.0 : -INFINITY);
        return;
    }
    r.top = value_of((uint32_t)(best >> 32));
    const auto leave = [&](unsigned long long cut) {         // to the fourth launch
        if (t == 0) { hand(c.h.cut + row, cut); hand(c.h.first + row, best); }
    };
    if (s.how == KEEP) {
        leave(0);
        return;
    }
    // what the whole row has to be searched for, where lists are too short; the last kept token so far
    Goal goal{0, 0.0};
    double p_of_all = 0.0;
    unsigned long long cut = 0;
    if (s.how == COUNT) {
        // the parts' lists, one behind the other: entry e of all
        int n_part = (lane & 15) < c.parts ? c.h.listed[(int64_t)row * c.parts + (lane & 15)] : 0;
        const bool whole = !__any(n_part > PART_CAP);
        if (wave == 0 && lane < 16) sh.part_end[lane] = n_part;
        __syncthreads();
        int total = 0;
        for (int i = 0; i < c.parts; ++i) total += sh.part_end[i];
        const auto entry = [&](int e) {
            int i = 0;
            while (e >= sh.part_end[i]) e -= sh.part_end[i++];
            return c.h.list[((int64_t)row * c.parts + i) * PART_CAP + e];
        };
        const unsigned long long mine = whole && t < total ? entry(t) : 0;           // (a part that holds too many has none)
        const auto listed = [&](auto f) {
            if (t < total) f(mine);
            for (int e = t + NT; e < total; e += NT) f(entry(e));
        };
        if (whole) {
            // what can be among the first k of them, by equal steps of keys between the lowest and the highest
            const uint32_t top = (uint32_t)(best >> 32);
            unsigned long long low = 0;
            listed([&](unsigned long long x) { low = max(low, (unsigned long long)~(uint32_t)(x >> 32)); });
            low = block_max(sh, low);
            const uint32_t lowest = ~(uint32_t)low;
            int shift = 0;
            while ((top - lowest) >> shift >= BINS) ++shift;
            clear_bins(sh);
            listed([&](unsigned long long x) { atomicAdd(&sh.count[(top - (uint32_t)(x >> 32)) >> shift], 1); });
            __syncthreads();
            const int b = find_bin<false>(sh, [&](double) { return Goal{s.k, 0.0}; }, 0, 0.0, 0, [](int) { return 0; }), n = sh.above_n + sh.count[b];
            if (n <= CAP) {
                if (t == 0) sh.n_list = 0;
                __syncthreads();
                listed([&](unsigned long long x) {
                    if ((int)((top - (uint32_t)(x >> 32)) >> shift) <= b) sh.list[atomicAdd(&sh.n_list, 1)] = x;
                });
                __syncthreads();
                finish_list(sh, r, n, true, s.k, s.by_p, s.p, 0.0, s.floor_w, s.u, answer);
                return;
            }
        }
        // (thousands of keys with the same leading bits)
        goal.k = s.k;
    } else {
        // ---- WEIGH: the parts' bins added up
        const Steps st(c, row, r, s.T);
        const auto ref = [&](int b) { return st.ref(b); };
        {
            static_assert(PER == 4, "a thread's bins are one and two 16-byte loads");
            int4 n = {0, 0, 0, 0};
            unsigned long long w[4] = {0, 0, 0, 0};
#pragma unroll 4
            for (int i = 0; i < c.parts; ++i) {
                const int64_t at = ((int64_t)row * c.parts + i) * BINS + t * 4;
                const int4 x = *(const int4*)(c.h.count + at);
                const ulonglong2 a = *(const ulonglong2*)(c.h.weight + at), b = *(const ulonglong2*)(c.h.weight + at + 2);
                n.x += x.x; n.y += x.y; n.z += x.z; n.w += x.w;
                w[0] += a.x; w[1] += a.y; w[2] += b.x; w[3] += b.y;
            }
            *(int4*)(sh.count + t * 4) = n;
#pragma unroll
            for (int j = 0; j < 4; ++j) sh.weight[t * 4 + j] = w[j];
        }
        __syncthreads();
        if (s.by_k) {
            // (more than K_MAX tokens) one workgroup
            const auto in_list = [&](const Goal& g) {
                const int b = find_bin<true>(sh, [&](double) { return g; }, 0, 0.0, c.fix, ref), n = sh.count[b], base_n = sh.above_n;
                const double base_w = sh.above_w;
                if (n > CAP) return false;
                if (t == 0) sh.n_list = 0;
                __syncthreads();
                for_each<false>(r, 0, c.V, [&](float l, int i) {
                    if (l > -INFINITY && st.bin(l) == b) sh.list[atomicAdd(&sh.n_list, 1)] = (unsigned long long)key_of(l) << 32 | (uint32_t)~i;
                });
                __syncthreads();
                sort_list(sh, n);
                find_in_list(sh, r, g, n, base_n, base_w);
                return true;
            };
            goal.k = s.k;
            if (in_list(goal)) {
                cut = sh.cut;
                if (!s.by_p) {
                    leave(cut);
                    return;
                }
                goal = Goal::share(s.p, sh.cut_sum);
                __syncthreads();
                if (in_list(goal)) {
                    leave(sh.cut > cut ? sh.cut : cut);
                    return;
                }
            }
        } else {
            // top_p alone: every part's workgroup finds the bin in which it ends and lists its part's tokens of that bin, or, if they are
            // few, of all up to it; the last one takes them together
            const int b = find_bin<true>(sh, [&](double all) { return Goal::share(s.p, all); }, 0, 0.0, c.fix, ref);
            const int n_bin = sh.count[b], above_n = sh.above_n;
            const double above_w = sh.above_w, sum = sh.total_w;
            goal = Goal::share(s.p, sum);
            __syncthreads();
            if (n_bin <= PART_CAP) {
                const bool all = above_n + n_bin <= NT;
                const int64_t at = (int64_t)row * c.parts + part;
                const int c0 = part * c.part_len;
                if (t == 0) sh.n_list = 0;
                __syncthreads();
                for_each(r, c0, min(c.V, c0 + c.part_len), [&](float l, int i) {
                    if (!(l > -INFINITY)) return;
                    const int x = st.bin(l);
                    if (x == b || (all && x < b)) hand(c.h.list + at * PART_CAP + atomicAdd(&sh.n_list, 1), (unsigned long long)key_of(l) << 32 | (uint32_t)~i);
                });
                __syncthreads();
                if (t == 0) hand(c.h.listed + at, sh.n_list);
                if (!last_to_finish(sh, c.h.finished + row * 2, c.parts)) return;
                int n = 0;
                for (int i = 0; i < c.parts; ++i) {
                    const int64_t from = (int64_t)row * c.parts + i;
                    const int ni = handed(c.h.listed + from);
                    for (int e = t; e < ni; e += NT) sh.list[n + e] = handed(c.h.list + from * PART_CAP + e);
                    n += ni;
                }
                __syncthreads();
                if (all) {
                    finish_list(sh, r, n, false, 0, true, s.p, sum, s.floor_w, s.u, answer);
                    return;
                }
                sort_list(sh, n);
                find_in_list(sh, r, goal, n, above_n, above_w);
                leave(sh.cut);
                return;
            }
            if (part != 0) return;
            p_of_all = s.p;
        }
    }
    // the whole row: the k-th and, in its place, the last one that top_p leaves
    for (;;) {
        find_in_row(sh, r, goal, p_of_all, s.by_p, c.fix);
        cut = sh.cut > cut ? sh.cut : cut;
        if (goal.k <= 0 || !s.by_p) break;
        goal = Goal::share(s.p, sh.cut_sum);
        __syncthreads();
    }
    leave(cut);
}

// ---- launch 4
__global__ void __launch_bounds__(NT) sample_keep_kernel(const Call c) {
    __shared__ Shared sh;
    const int row = blockIdx.x / c.parts, part = blockIdx.x - row * c.parts, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const unsigned long long best = c.h.first[row];
    if (best == 0) return;
    const Settings s(c, row);
    Row r = row_of(c, row, s);
    r.top = value_of((uint32_t)(best >> 32));
    fill_table(sh);
    const unsigned long long cut = c.h.cut[row];
    const float lowest = cut ? value_of((uint32_t)(cut >> 32)) : -INFINITY;
    const auto kept = [&](float l, int i) {
        if (!(l > -INFINITY) || l < lowest) return 0.0;
        const unsigned long long e = (unsigned long long)key_of(l) << 32 | (uint32_t)~i;
        if (e < cut) return 0.0;
        const double w = r.weight(l, sh.table);
        return w >= s.floor_w || e == best ? w : 0.0;
    };
    const int c0 = part * c.part_len, c1 = min(c.V, c0 + c.part_len);
    double* const tile = c.h.tile + (int64_t)row * MAX_TILES;
    const auto weigh = [&](int i0, const float (&v)[16]) {
        double w = 0.0;
#pragma unroll
        for (int j = 0; j < 16; ++j) w += kept(v[j], i0 + j * 64 + lane);
        return w;
    };
    const auto put = [&](int a, double w) {
        w = wave_sum(w);
        if (lane == 0) hand(tile + a, w);
    };
    if (c.ts == SUB) {
        for_each_sub(r, c0, c1, [&](int i0, const float (&v)[16]) { put(i0 / SUB, weigh(i0, v)); });
    } else {
        for (int a = c0 / c.ts + wave; a * c.ts < c1; a += NWAVE) {
            double w = 0.0;
            for (int i0 = a * c.ts; i0 < min(c.V, (a + 1) * c.ts); i0 += SUB) {
                float v[16];
                read_sub(r, i0, v);
                w += weigh(i0, v);
            }
            put(a, w);
        }
    }
    if (!last_to_finish(sh, c.h.finished + row * 2 + 1, c.parts)) return;
    if (t < r.tiles) sh.tile[t] = handed(tile + t);
    __syncthreads();
    finish_tiles(sh, r, s.u, answer_of(c, row), kept);
}

// parts of a row: as many as fill the card with all rows, of whole tiles, not so short that a thread has less than a SUB's 16 logits
int parts_of(int64_t rows, int V, int ts, int* part_len) {
    const int64_t most = std::min<int64_t>(MAX_PARTS, std::max<int64_t>(1, 256 / rows));
    const int64_t unit = std::max<int64_t>(ts, NWAVE * SUB) / ts * ts;
    *part_len = (int)round_up64(std::max<int64_t>((V + most - 1) / most, 1), unit);
    return (V + *part_len - 1) / *part_len;
}
int tile_of(int V) { return (int)round_up64((V + MAX_TILES - 1) / MAX_TILES, SUB); }

// the arrays of a Handover, in `base` if there is one; -> bytes
size_t lay_out(Handover* h, unsigned char* base, int64_t rows, int parts, bool filtered) {
    size_t at = 0;
    const auto place = [&](auto*& p, size_t n) {
        p = (std::remove_reference_t<decltype(p)>)(base + at);
        at += (n * sizeof(*p) + 255) / 256 * 256;
    };
    const size_t rp = (size_t)rows * parts;
    place(h->best, rp);
    place(h->least, rp);
    place(h->listed, rp);
    place(h->cut, rows);
    place(h->first, rows);
    place(h->finished, 2 * rows);
    place(h->tile, (size_t)rows * MAX_TILES);
    place(h->tile_top, (size_t)rows * MAX_TILES);
    place(h->list, filtered ? rp * PART_CAP : 0);
    place(h->count, filtered ? rp * BINS : 0);
    place(h->weight, filtered ? rp * BINS : 0);
    return at;
}

}  // namespace

size_t sample_scratch(int64_t rows, int V, bool top_k, bool top_p) {
    Handover h;
    int part_len;
    const int parts = parts_of(rows, V, tile_of(V), &part_len);
    return lay_out(&h, nullptr, rows, parts, top_k || top_p);
}

void launch_sample(const float* logits, int64_t ld, int rows, int V, const float* u, const float* temperature, const int* top_k,
                   const float* top_p, const float* min_p, int* tokens, float* logprobs, void* scratch, hipStream_t s) {
    if (rows <= 0) return;
    Call c;
    c.logits = logits; c.ld = ld; c.V = V;
    c.u = u; c.temperature = temperature; c.top_k = top_k; c.top_p = top_p; c.min_p = min_p;
    c.tokens = tokens; c.logprobs = logprobs;
    // at most MAX_TILES tiles of whole SUBs; histogram weights of as many digits as V of them may add up
    c.ts = tile_of(V);
    c.fix = 62;
    while (V > (int64_t)1 << (62 - c.fix)) --c.fix;
    c.fix = std::min(c.fix, 44);
    c.parts = parts_of(rows, V, c.ts, &c.part_len);
    lay_out(&c.h, (unsigned char*)scratch, rows, c.parts, top_k || top_p);
    const dim3 parts((unsigned)((int64_t)rows * c.parts)), block(NT);
    hipLaunchKernelGGL(sample_parts_kernel, parts, block, 0, s, c);
    if (top_k || top_p) hipLaunchKernelGGL(sample_weigh_kernel, parts, block, 0, s, c);
    hipLaunchKernelGGL(sample_pick_kernel, parts, block, 0, s, c);
    if (top_k || top_p || min_p) hipLaunchKernelGGL(sample_keep_kernel, parts, block, 0, s, c);
}

}  // namespace po
