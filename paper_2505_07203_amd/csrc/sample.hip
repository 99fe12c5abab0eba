// Drawing one token per row of float32 logits, with temperature, top-k, top-p and min-p, from one given random number a row
// (gfx950).
//
// With m the row's largest logit, w_i = exp((l_i - m) / T).  Tokens are ordered by l descending, equal ones by index; what may
// be drawn is a beginning of that order: the first top_k; of those the shortest beginning whose sum of w is at least top_p times
// the sum of the top_k; of those the ones with w >= min_p; the first one always.  The token is the first kept one, by index, at
// which the running sum of kept w exceeds u times their whole sum.
//
// Whole numbers come out, so sums and comparisons are float64 throughout: an error of 1e-7 in a running sum over 10^5 tokens
// would move a draw to its neighbour once in a hundred.  The exponential is the only costly part (a float64 operation takes a
// compute unit a cycle per wavefront): 2^y by a table of 64 values of 2^(j / 64) in LDS and a polynomial of degree 5, relative
// error below 1e-15, about 12 operations.
#include "po_internal.h"

#include <float.h>

namespace po {
namespace {

constexpr int NT = 1024;            // threads of a workgroup: one row
constexpr int NWAVE = NT / 64;
constexpr int BINS = 4096;
constexpr int PER = BINS / NT;      // bins of a thread
constexpr int CAP = 4096;           // entries that are ordered in LDS
constexpr int MAX_TILES = 1024;
constexpr int SUB = 1024;           // logits that a wavefront reads at once, 16 a lane

struct Shared {
    double table[64];
    double part[NWAVE];
    int ipart[NWAVE];
    unsigned long long wave_best[NWAVE];
    double scan_w[NT];
    int scan_n[NT];
    unsigned long long weight[BINS];        // of a bin, as a multiple of 2^(its reference exponent - fix)
    int count[BINS];
    unsigned long long list[CAP];           // key << 32 | ~index: descending order is the order of the tokens
    double tile[MAX_TILES];
    float tile_top[MAX_TILES];
    int n_list;
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
    double rate;                    // log2(e) / T

    // 2^((l - top) rate) of a logit that may be drawn
    __device__ __forceinline__ double weight(float l, const double* table) const {
        if (l == top) return 1.0;
        const double y = ((double)l - (double)top) * rate;
        if (!(y > -1000.0)) return 0.0;              // (what is left of it no sum holds; -inf, and -inf * 0)
        const double n = rint(y * 64.0);
        const double r = fma(n, -1.0 / 64.0, y) * 0.69314718055994530942;
        double p = fma(r, 1.0 / 120.0, 1.0 / 24.0);
        p = fma(p, r, 1.0 / 6.0);
        p = fma(p, r, 0.5);
        p = fma(p, r, 1.0);
        const int i = (int)n;
        const double t = table[i & 63];
        return ldexp(fma(t * r, p, t), i >> 6);
    }
};

// the SUB logits from i0 on, lane l the ones at i0 + l, + 64, ..; -inf past the end
__device__ __forceinline__ void read_sub(const Row& r, int i0, float (&v)[16]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const int i = i0 + j * 64 + lane;
        const float x = r.z[min(i, r.V - 1)];
        v[j] = i < r.V ? x : -INFINITY;
    }
}
// f(logit, its index) for all logits of the row, a wavefront SUB of them at a time
template <typename F>
__device__ __forceinline__ void for_each(const Row& r, F f) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float v[16], next[16];
    if (wave * SUB < r.V) read_sub(r, wave * SUB, next);
    for (int i0 = wave * SUB; i0 < r.V; i0 += NWAVE * SUB) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = next[j];
        if (i0 + NWAVE * SUB < r.V) read_sub(r, i0 + NWAVE * SUB, next);
#pragma unroll
        for (int j = 0; j < 16; ++j) f(v[j], i0 + j * 64 + lane);
    }
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

// What a search is after: the k-th token of an order (k > 0), or the first at which the running sum reaches `sum`.
struct Goal {
    int k;
    double sum;
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
// ref(b): a bin's reference exponent.
template <bool weights, typename Ref>
__device__ int find_bin(Shared& sh, const Goal& goal, int base_n, double base_w, int fix, Ref ref) {
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

__device__ void clear_bins(Shared& sh) {
    for (int b = threadIdx.x; b < BINS; b += NT) { sh.count[b] = 0; sh.weight[b] = 0; }
    __syncthreads();
}

__device__ __forceinline__ void add_to_bin(Shared& sh, int b, double w, int digits) {
    atomicAdd(&sh.count[b], 1);                               // whole numbers: the order of the additions does not show
    const unsigned long long f = (unsigned long long)ldexp(w, digits);
    if (f) atomicAdd(&sh.weight[b], f);
}

// sh.list[0 .. n) in descending order (n <= CAP)
__device__ void sort_list(Shared& sh, int n) {
    int m = 2;
    while (m < n) m <<= 1;
    for (int i = n + threadIdx.x; i < m; i += NT) sh.list[i] = 0;
    __syncthreads();
    for (int size = 2; size <= m; size <<= 1)
        for (int half = size >> 1; half > 0; half >>= 1) {
            for (int i = threadIdx.x; i < m / 2; i += NT) {
                const int lo = 2 * i - (i & (half - 1)), hi = lo + half;
                const bool down = (lo & size) == 0;
                const unsigned long long a = sh.list[lo], b = sh.list[hi];
                if ((a < b) == down) { sh.list[lo] = b; sh.list[hi] = a; }
            }
            __syncthreads();
        }
}

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

// The same over the whole row with nothing known, for bins that hold more than CAP tokens: the key digit by digit (11, 11, 10
// bits), then the right one of the tokens with that key by a count of tiles.
__device__ void find_in_row(Shared& sh, const Row& r, const Goal& goal, int fix) {
    uint32_t prefix = 0;
    int base_n = 0;
    double base_w = 0.0;
    for (int shift = 21; shift >= 0; shift = shift == 21 ? 10 : shift == 10 ? 0 : -1) {
        const int bits = shift == 0 ? 10 : 11;
        const uint32_t upper = shift == 21 ? 0u : 0xffffffffu << (shift + bits);
        // no token of this group weighs more than its highest key
        const uint32_t high = shift == 21 ? key_of(r.top) : min(prefix | ~upper, key_of(r.top));
        const double wh = r.weight(value_of(high), sh.table);
        const int ref = wh > 0.0 ? ilogb(wh) + 1 : -1000;
        clear_bins(sh);
        for_each(r, [&](float l, int) {
            const uint32_t key = key_of(l);
            if (key && (key & upper) == prefix)
                add_to_bin(sh, (1 << bits) - 1 - (int)((key >> shift) & ((1u << bits) - 1)), r.weight(l, sh.table), fix - ref);
        });
        __syncthreads();
        const int b = find_bin<true>(sh, goal, base_n, base_w, fix, [&](int) { return ref; });
        prefix |= (uint32_t)((1 << bits) - 1 - b) << shift;
        base_n = sh.above_n;
        base_w = sh.above_w;
        __syncthreads();
    }
    // tokens of this key: all of one weight; how many of them
    const int ties = sh.count[1023 - (int)(prefix & 1023u)];
    const double w = r.weight(value_of(prefix), sh.table);
    int want = goal.k > 0 ? goal.k - base_n : ties;
    if (goal.k <= 0 && w > 0.0) want = (int)fmin(fmax(ceil((goal.sum - base_w) / w), 1.0), (double)ties);
    want = max(1, min(want, ties));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    __syncthreads();
    for (int a = wave; a < NT; a += NWAVE) {
        int n = 0;
        if (a < r.tiles)
            for (int i = a * r.ts + lane; i < min(r.V, (a + 1) * r.ts); i += 64) n += key_of(r.z[i]) == prefix;
        for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off);
        if (lane == 0) sh.count[a] = n;
    }
    __syncthreads();
    block_scan(sh, sh.count[threadIdx.x], 0.0);
    const int t = first_thread(sh, sh.scan_n[threadIdx.x] >= want, threadIdx.x && sh.scan_n[threadIdx.x - 1] >= want);
    if (wave == 0) {
        int seen = t ? sh.scan_n[t - 1] : 0;
        for (int i = t * r.ts; i < min(r.V, (t + 1) * r.ts) && seen < want; i += 64) {
            const bool tie = i + lane < min(r.V, (t + 1) * r.ts) && key_of(r.z[i + lane]) == prefix;
            const unsigned long long b = __ballot(tie);
            const int upto = seen + __popcll(b & (0xffffffffffffffffull >> (63 - lane)));
            if (tie && upto == want) {
                sh.cut = (unsigned long long)prefix << 32 | (uint32_t)~(i + lane);
                sh.cut_sum = base_w + want * w;
            }
            seen += __popcll(b);
        }
    }
    __syncthreads();
}

// The first of the largest logits, as an entry of a list (0: there is none), and the lowest key of what may be drawn.
struct Extremes {
    unsigned long long best;
    uint32_t least;
    __device__ __forceinline__ void see(float l, int i) {
        const uint32_t key = key_of(l);
        const unsigned long long e = (unsigned long long)key << 32 | (uint32_t)~i;
        if (key) { best = e > best ? e : best; least = min(least, key); }
    }
    __device__ void join(Shared& sh) {
        for (int off = 32; off > 0; off >>= 1) {
            const unsigned long long o = __shfl_xor(best, off);
            best = o > best ? o : best;
            least = min(least, (uint32_t)__shfl_xor((int)least, off));
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 0) { sh.wave_best[threadIdx.x >> 6] = best; sh.ipart[threadIdx.x >> 6] = (int)least; }
        __syncthreads();
        for (int i = 0; i < NWAVE; ++i) {
            best = sh.wave_best[i] > best ? sh.wave_best[i] : best;
            least = min(least, (uint32_t)sh.ipart[i]);
        }
        __syncthreads();
    }
};

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

// The token once sh.tile holds the kept weight of every tile.  kept(logit, index): its weight, or 0.
template <typename F>
__device__ void finish_tiles(Shared& sh, const Row& r, float u, int best, const Answer& answer, F kept) {
    const int t = threadIdx.x, lane = t & 63;
    block_scan(sh, 0, t < r.tiles ? sh.tile[t] : 0.0);
    const double all = sh.scan_w[r.tiles - 1], target = target_of(u, all);
    const int a = first_thread(sh, t == r.tiles - 1 || sh.scan_w[t] > target, t && (t - 1 == r.tiles - 1 || sh.scan_w[t - 1] > target));
    if (t >= 64) return;
    double run = a ? sh.scan_w[a - 1] : 0.0, w_last = 1.0;
    int token = best;
    for (int i0 = a * r.ts; i0 < min(r.V, (a + 1) * r.ts); i0 += 64) {
        const int i = i0 + lane;
        const double w = i < min(r.V, (a + 1) * r.ts) ? kept(r.z[i], i) : 0.0;
        double c = w;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const double o = __shfl_up(c, off);
            if (lane >= off) c += o;
        }
        // (the last kept token so far stands in where rounding leaves the target out of reach at the very end)
        const unsigned long long some = __ballot(w > 0.0), past = __ballot(w > 0.0 && run + c > target);
        if (some) {
            const int pick = past ? __ffsll(past) - 1 : 63 - __clzll(some);
            token = i0 + pick;
            w_last = __shfl(w, pick);
        }
        if (past) break;
        run += __shfl(c, 63);
    }
    if (lane == 0) answer.give(token, log(w_last / all));
}

// A row, a workgroup.  What it takes by settings: nothing but a temperature, one pass over the logits; top_k (up to half a list), one
// pass that counts keys by their leading bits and one that gathers the head of the order; top_p alone, a pass for the extremes, one
// that adds weights by steps of the logit, one that gathers; where the head is longer than a list holds, passes that find
// the last kept token and one that adds up what is kept.
__global__ void __launch_bounds__(NT) sample_kernel(const float* __restrict__ logits, int64_t ld, int V, int ts, int fix,
                                                    const float* __restrict__ u, const float* __restrict__ temperature,
                                                    const int* __restrict__ top_k, const float* __restrict__ top_p,
                                                    const float* __restrict__ min_p, int* __restrict__ tokens,
                                                    float* __restrict__ logprobs) {
    __shared__ Shared sh;
    const int row = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    Row r;
    r.z = logits + (int64_t)row * ld;
    r.V = V;
    r.ts = ts;
    r.tiles = (V + ts - 1) / ts;
    r.top = 0.f;
    if (t < 64) sh.table[t] = exp2((double)t / 64.0);
    const Answer answer = {tokens + row, logprobs ? logprobs + row : nullptr};
    const float T = temperature ? temperature[row] : 1.0f, uu = u[row];
    const int k = top_k ? top_k[row] : 0;
    const float p = top_p ? top_p[row] : 1.0f;
    const double floor_w = min_p && min_p[row] > 0.0f ? (double)min_p[row] : 0.0;      // (NaN: off)
    const bool greedy = !(T > 0.0f), by_k = k > 0 && k < V, by_p = p < 1.0f;
    r.rate = 1.4426950408889634074 / (double)T;
    Extremes ext = {0ull, 0xffffffffu};

    if (!greedy && !by_k && !by_p && floor_w == 0.0) {
        // ---- nothing is left out: each tile's weight with the tile's own largest logit for reference
        __syncthreads();
        for (int a = wave; a < r.tiles; a += NWAVE) {
            Row q = r;
            q.top = -INFINITY;
            double w = 0.0;
            for (int i0 = a * ts; i0 < min(V, (a + 1) * ts); i0 += SUB) {
                float v[16], m = -INFINITY;
                read_sub(r, i0, v);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    if (!key_of(v[j])) v[j] = -INFINITY;
                    m = fmaxf(m, v[j]);
                }
                for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
                if (m == -INFINITY) continue;
                if (m > q.top) {
                    const float old = q.top;
                    q.top = m;
                    w *= old == -INFINITY ? 0.0 : q.weight(old, sh.table);
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) w += v[j] == -INFINITY ? 0.0 : q.weight(v[j], sh.table);
            }
            w = wave_sum(w);
            if (lane == 0) { sh.tile[a] = w; sh.tile_top[a] = q.top; }
        }
        __syncthreads();
        float m = t < r.tiles ? sh.tile_top[t] : -INFINITY;
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
        if (t < r.tiles) sh.tile[t] *= sh.tile_top[t] == -INFINITY ? 0.0 : r.weight(sh.tile_top[t], sh.table);
        finish_tiles(sh, r, uu, 0, answer, [&](float l, int) { return key_of(l) ? r.weight(l, sh.table) : 0.0; });
        return;
    }
    const bool counts = !greedy && by_k && k <= CAP / 2;
    if (counts) {
        // ---- tokens by the leading 12 bits of their key; once 16 K logits have been seen only what can be among the first k
        clear_bins(sh);
        uint32_t low = 1;
        bool first = true;
        float v[16];
        for (int i0 = wave * SUB; i0 - wave * SUB < V; i0 += NWAVE * SUB) {
            if (i0 < V) {
                read_sub(r, i0, v);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    ext.see(v[j], i0 + j * 64 + lane);
                    const uint32_t key = key_of(v[j]);
                    if (key >= low) atomicAdd(&sh.count[BINS - 1 - (key >> 20)], 1);
                }
            }
            if (first && V > 2 * NWAVE * SUB) {
                __syncthreads();
                const int b = find_bin<false>(sh, Goal{k, 0.0}, 0, 0.0, 0, [](int) { return 0; });
                if (sh.scan_n[NT - 1] >= k) low = (uint32_t)(BINS - 1 - b) << 20;
                low = max(low, 1u);
                __syncthreads();
            }
            first = false;
        }
    } else {
        for_each(r, [&](float l, int i) { ext.see(l, i); });
    }
    ext.join(sh);
    if (ext.best == 0 || greedy) {                            // nothing to draw; or the most likely token
        if (t == 0) answer.give(ext.best ? (int)~(uint32_t)ext.best : -1, ext.best ? 0.0 : -INFINITY);
        return;
    }
    r.top = value_of((uint32_t)(ext.best >> 32));
    const auto gather = [&](auto take) {
        if (t == 0) sh.n_list = 0;
        __syncthreads();
        for_each(r, [&](float l, int i) {
            const uint32_t key = key_of(l);
            if (key && take(l, key)) sh.list[atomicAdd(&sh.n_list, 1)] = (unsigned long long)key << 32 | (uint32_t)~i;
        });
        __syncthreads();
    };
    if (counts) {
        const int b = find_bin<false>(sh, Goal{k, 0.0}, 0, 0.0, 0, [](int) { return 0; }), n = sh.above_n + sh.count[b];
        if (n <= CAP) {
            const uint32_t low = (uint32_t)(BINS - 1 - b) << 20;
            gather([&](float, uint32_t key) { return key >= low; });
            finish_list(sh, r, n, true, k, by_p, p, 0.0, floor_w, uu, answer);
            return;
        }
    }
    unsigned long long cut = 0;                               // the last token of the kept beginning (0: all)
    if (by_k || by_p) {
        // ---- tokens and weight in equal steps of the logit below the largest: over all logits, or down to where no weight
        // counts any more (the last bin takes the rest)
        const double span = fmin((double)r.top - (double)value_of(ext.least), 64.0 * fmax((double)T, 1.0));
        const float scale = span > 0.0 && r.top < INFINITY ? (float)(BINS / span) : 0.0f;
        const double step = scale > 0.0f ? r.rate / (double)scale : 0.0;
        // no weight in a bin is above that of its upper edge; 1 for what the steps' own rounding moves across edges
        const auto ref = [&](int b) { return (int)fmax(ceil(-(double)b * step), -1000.0) + 1; };
        const auto bin = [&](float l) {
            const float x = (r.top - l) * scale;
            return x < (float)(BINS - 1) ? (int)x : BINS - 1;
        };
        const auto fill = [&] {
            clear_bins(sh);
            for_each(r, [&](float l, int) {
                if (key_of(l)) {
                    const int b = bin(l);
                    add_to_bin(sh, b, r.weight(l, sh.table), fix - ref(b));
                }
            });
            __syncthreads();
        };
        // -> whether the bins still are what fill made
        const auto search = [&](const Goal& goal) {
            const int b = find_bin<true>(sh, goal, 0, 0.0, fix, ref), n = sh.count[b], base_n = sh.above_n;
            const double base_w = sh.above_w;
            if (n > CAP) {
                find_in_row(sh, r, goal, fix);
                return false;
            }
            gather([&](float l, uint32_t) { return bin(l) == b; });
            sort_list(sh, n);
            find_in_list(sh, r, goal, n, base_n, base_w);
            return true;
        };
        fill();
        double sum;
        if (by_k) {
            const bool whole = search(Goal{k, 0.0});
            cut = sh.cut;
            sum = sh.cut_sum;
            __syncthreads();
            if (by_p && !whole) fill();
        } else {
            find_bin<true>(sh, Goal{1, 0.0}, 0, 0.0, fix, ref);
            sum = sh.total_w;
            __syncthreads();
            const int b = find_bin<true>(sh, Goal{0, fmax((double)p * sum, DBL_MIN)}, 0, 0.0, fix, ref), n = sh.above_n + sh.count[b];
            if (n <= CAP) {
                gather([&](float l, uint32_t) { return bin(l) <= b; });
                finish_list(sh, r, n, false, 0, true, p, sum, floor_w, uu, answer);
                return;
            }
        }
        if (by_p) {           // (above 0, so that no sum of nothing reaches it)
            search(Goal{0, fmax((double)p * sum, DBL_MIN)});
            cut = sh.cut > cut ? sh.cut : cut;
            __syncthreads();
        }
    }
    // ---- the kept weight of every tile, a wavefront each
    const auto kept = [&](float l, int i) {
        const uint32_t key = key_of(l);
        const unsigned long long e = (unsigned long long)key << 32 | (uint32_t)~i;
        if (!key || e < cut) return 0.0;
        const double w = r.weight(l, sh.table);
        return w >= floor_w || e == ext.best ? w : 0.0;
    };
    for (int a = wave; a < r.tiles; a += NWAVE) {
        double w = 0.0;
        for (int i0 = a * ts; i0 < min(V, (a + 1) * ts); i0 += SUB) {
            float v[16];
            read_sub(r, i0, v);
#pragma unroll
            for (int j = 0; j < 16; ++j) w += kept(v[j], i0 + j * 64 + lane);
        }
        w = wave_sum(w);
        if (lane == 0) sh.tile[a] = w;
    }
    __syncthreads();
    finish_tiles(sh, r, uu, (int)~(uint32_t)ext.best, answer, kept);
}

}  // namespace

void launch_sample(const float* logits, int64_t ld, int rows, int V, const float* u, const float* temperature, const int* top_k,
                   const float* top_p, const float* min_p, int* tokens, float* logprobs, hipStream_t s) {
    if (rows <= 0) return;
    // at most MAX_TILES tiles of whole SUBs; histogram weights of as many digits as V of them may add up
    const int ts = (int)round_up64((V + MAX_TILES - 1) / MAX_TILES, SUB);
    int fix = 62;
    while (fix > 0 && ((int64_t)V << fix) > ((int64_t)1 << 62)) --fix;
    fix = fix < 44 ? fix : 44;
    hipLaunchKernelGGL(sample_kernel, dim3((unsigned)rows), dim3(NT), 0, s, logits, ld, V, ts, fix, u, temperature, top_k, top_p, min_p,
                       tokens, logprobs);
}

}  // namespace po
