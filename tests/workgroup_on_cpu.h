// Runs the workgroups of a HIP source on the CPU, one after the other: every thread a context of its own, switched at barriers and at
// operations of a wavefront.  Between two barriers whole wavefronts run one after the other, in an order that the caller names, so
// that a wavefront is as far ahead of another as the barriers allow; all threads that meet at a barrier must have come to the same one.
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <string.h>
#include <ucontext.h>

#include <algorithm>
#include <vector>

#define __device__
#define __global__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static

struct dim3 {
    unsigned x;
    dim3(unsigned n = 1) : x(n) {}
};
struct int4 { int x, y, z, w; };
struct ulonglong2 { unsigned long long x, y; };
typedef void* hipStream_t;
static struct { unsigned x; } threadIdx, blockIdx;

using std::max;
using std::min;

static inline uint32_t __float_as_uint(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }
static inline float __uint_as_float(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
static inline long long __double_as_longlong(double d) { long long u; memcpy(&u, &d, 8); return u; }
static inline int __popcll(unsigned long long x) { return __builtin_popcountll(x); }
template <typename T> static inline T atomicAdd(T* p, T v) { const T old = *p; *p = old + v; return old; }
static inline int atomicMin(int* p, int v) { const int old = *p; *p = min(old, v); return old; }
#define __HIP_MEMORY_SCOPE_AGENT 0
#define __hip_atomic_store(p, v, order, scope) (void)(*(p) = (v))
#define __hip_atomic_load(p, order, scope) (*(p))
#define __hip_atomic_fetch_add(p, v, order, scope) atomicAdd((p), (v))

namespace on_cpu {

constexpr int WAVE = 64, MAX_THREADS = 1024, STACK = 128 * 1024;
enum State { RUNS, AT_WAVE, AT_BARRIER, ENDED };

struct Thread {
    ucontext_t context;
    State state;
    int line;                                        // of the barrier
    unsigned ops;                                    // operations of the wavefront so far
};
static std::vector<char> stacks;
static Thread threads[MAX_THREADS];
static unsigned long long lanes[MAX_THREADS / WAVE][2][WAVE];
static ucontext_t scheduler;
static int current, fault;                           // fault: a line at which threads met others at another one, or that had ended
static std::vector<int> wave_order;
static void (*body)(void*);
static void* body_arg;

static void stop(State s, int line) {
    const int me = current;
    threads[me].state = s;
    threads[me].line = line;
    swapcontext(&threads[me].context, &scheduler);
    threadIdx.x = (unsigned)me;
}
static void entry() {
    body(body_arg);
    threads[current].state = ENDED;
    swapcontext(&threads[current].context, &scheduler);
}

static void run_workgroup(int n) {
    const int waves = n / WAVE;
    for (int t = 0; t < n; ++t) {
        getcontext(&threads[t].context);
        threads[t].context.uc_stack.ss_sp = &stacks[(size_t)t * STACK];
        threads[t].context.uc_stack.ss_size = STACK;
        threads[t].context.uc_link = nullptr;
        makecontext(&threads[t].context, entry, 0);
        threads[t].state = RUNS;
        threads[t].ops = 0;
    }
    for (;;) {
        int waiting = 0, line = 0;
        for (int o = 0; o < waves; ++o) {
            const int w = wave_order.empty() ? o : wave_order[o] % waves;
            for (bool again = true; again;) {
                int at_wave = 0;
                for (int t = w * WAVE; t < (w + 1) * WAVE; ++t) {
                    if (threads[t].state == RUNS) {
                        current = t;
                        threadIdx.x = (unsigned)t;
                        swapcontext(&scheduler, &threads[t].context);
                    }
                    at_wave += threads[t].state == AT_WAVE;
                }
                again = at_wave > 0;
                if (again && at_wave != WAVE) { fault = -1; return; }        // (a wavefront's operation without all of its lanes)
                for (int t = w * WAVE; again && t < (w + 1) * WAVE; ++t) threads[t].state = RUNS;
            }
        }
        for (int t = 0; t < n; ++t)
            if (threads[t].state == AT_BARRIER) {
                if (waiting && threads[t].line != line) { fault = line; return; }
                line = threads[t].line;
                ++waiting;
            }
        if (waiting == 0) return;
        if (waiting != n) { fault = line; return; }
        for (int t = 0; t < n; ++t) threads[t].state = RUNS;
    }
}

template <typename F>
void launch(unsigned grid, unsigned n, F f) {
    if (stacks.empty()) stacks.resize((size_t)MAX_THREADS * STACK);
    body = [](void* p) { (*(F*)p)(); };
    body_arg = &f;
    for (unsigned b = 0; b < grid && !fault; ++b) {
        blockIdx.x = b;
        run_workgroup((int)n);
    }
}

// what lane `from` of this wavefront put there (each lane puts one value)
template <typename T>
T exchange(T v, int from) {
    const int wave = current / WAVE, me = current % WAVE;
    const unsigned side = threads[current].ops++ & 1;
    unsigned long long x = 0;
    memcpy(&x, &v, sizeof(T));
    lanes[wave][side][me] = x;
    stop(AT_WAVE, 0);
    memcpy(&v, &lanes[wave][side][from], sizeof(T));
    return v;
}
static unsigned long long ballot(bool yes) {
    const int wave = current / WAVE;
    const unsigned side = threads[current].ops & 1;
    exchange((int)yes, 0);
    unsigned long long all = 0;
    for (int i = 0; i < WAVE; ++i) all |= (unsigned long long)(lanes[wave][side][i] & 1) << i;
    return all;
}
static inline int lane() { return current % WAVE; }

}  // namespace on_cpu

#define __syncthreads() on_cpu::stop(on_cpu::AT_BARRIER, __LINE__)
#define __ballot(x) on_cpu::ballot(x)
#define __any(x) (on_cpu::ballot(x) != 0)
template <typename T> T __shfl_xor(T v, int off, int width = 64) { (void)width; return on_cpu::exchange(v, on_cpu::lane() ^ off); }
template <typename T> T __shfl_up(T v, int off) { return on_cpu::exchange(v, max(on_cpu::lane() - off, 0)); }
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, arg) on_cpu::launch((grid).x, (block).x, [&] { kernel(arg); })

namespace po {
static inline int64_t round_up64(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
}  // namespace po
