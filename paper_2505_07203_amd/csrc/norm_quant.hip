// The residual's addition, RMS norm and 8-bit codes in one pass (gfx950).
//
//   h = bf16(x + delta),  y = h * rsqrt(mean(h^2) + eps) * g,  codes = e4m3(y * (448 / amax)), scale = amax / 448
//
// amax = max |y| over a row or over each block of 128 of it.  y is a float32 number throughout: it is rounded once, to the code (and once to bf16
// where the rows are wanted too), not to bf16 first and then to the code.
//
// Bound by memory; a row is read once and stays in the registers of its workgroup.  16384 x 4096 in blocks 78 us, calls of 1 to 12 batches in turn (6.0 TB/s read and
// written; addition, norm and quantisation in three calls 161), 1931 x 5120 in blocks with the bf16 rows 17 (5.2: one round of
// workgroups, which read together and write together), one row of 4096 3.7, a launch and two exchanges.
#include "po_internal.h"

#include <math.h>

namespace po {
namespace {

constexpr float E4M3_MAX = 448.0f;
constexpr float AMAX_MIN = 448.0f * 0x1p-126f;    // below it both quotients would not be normal numbers

struct NormQuant {
    const uint4 *x, *delta, *g;
    uint4 *h, *y;
    uint2* codes;
    float* scales;
    int64_t rows;
    int vecs;                     // of 8 values in a row
    float eps, inv_d;
};

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4;
template <bool ONCE>
__device__ __forceinline__ uint4 load16(const uint4* p) {
    return ONCE ? __builtin_bit_cast(uint4, __builtin_nontemporal_load((const u32x4*)p)) : *p;
}
__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        f[2 * c] = __uint_as_float(w[c] << 16);
        f[2 * c + 1] = __uint_as_float(w[c] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = (uint32_t)f2bf(f[2 * c]) | ((uint32_t)f2bf(f[2 * c + 1]) << 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// What a code is a multiple of.  The row's 1 / rms cancels in y * (448 / amax): with p = h * g (exact, a product of two bf16 numbers) and
// pm = max |p| the code is that of p * 448 / pm, which inv + inv_lo (448 / pm to 2^-46) gives with one rounding, so that codes are those of exact
// arithmetic but for values within 2^-24 of a border.  Where p or 448 / pm leaves the range of normal numbers, or amax is raised, y itself is taken.
struct Code {
    float inv, inv_lo, scale;
    bool of_p;
};
__device__ __forceinline__ Code code_of(float pm, float r) {
    const float ym = pm * r;
    Code c;
    c.of_p = pm >= 0x1p-100f && pm < 0x1p120f && ym >= AMAX_MIN && ym < 0x1p120f;
    if (c.of_p) {
        c.inv = __fdiv_rn(E4M3_MAX, pm);
        c.inv_lo = __fdiv_rn(fmaf(-c.inv, pm, E4M3_MAX), pm);
        c.scale = __fdiv_rn(ym, E4M3_MAX);
    }
    return c;
}
__device__ __forceinline__ Code code_of_y(float ym) {
    const float amax = ym > 0.f ? fmaxf(ym, AMAX_MIN) : E4M3_MAX;
    return {__fdiv_rn(E4M3_MAX, amax), 0.f, __fdiv_rn(amax, E4M3_MAX), false};
}
__device__ __forceinline__ uint2 encode8(const float (&h)[8], const float (&g)[8], float r, const Code& c) {
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float p = h[e] * g[e];
        f[e] = c.of_p ? fmaf(p, c.inv, p * c.inv_lo) : h[e] * r * g[e] * c.inv;
    }
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], lo, true);
    int hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], hi, true);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// A workgroup per row, whose values stay in registers: QV vectors of 8 a thread.  BLOCK: a scale per 128 values, which 16 lanes hold.
// ONCE: x and delta go past the caches.
template <int QV, bool BLOCK, bool ONCE>
__global__ void __launch_bounds__(256) norm_quant_kernel(const NormQuant p) {
    __shared__ float part[4], partm[4], party[4];
    const int64_t row = blockIdx.x, at = row * p.vecs;
    float h[QV][8];
    uint4 gv[QV];
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < QV; ++j) {
        const int i = threadIdx.x + j * 256;
        if (i < p.vecs) {
            gv[j] = p.g[i];
            unpack8(load16<ONCE>(p.x + at + i), h[j]);
            if (p.delta) {
                float a[8];
                unpack8(load16<ONCE>(p.delta + at + i), a);
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] += h[j][e];
                const uint4 v = pack8(a);
                unpack8(v, h[j]);
                if (p.h) p.h[at + i] = v;
            } else if (p.h) {
                p.h[at + i] = pack8(h[j]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(h[j][e], h[j][e], ss);
        }
    }
    for (int off = 32; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = ss;
    __syncthreads();
    float mean = (part[0] + part[1] + part[2] + part[3]) * p.inv_d + p.eps;
    if (mean < 0x1p-100f) {                      // (the workgroup together)
        // Squares below the normal numbers count (each of 16384 may be off by 2^-150): the row times 2^100, exactly, is normed in its place.  Its
        // values are below 2^57, as mean * d is below 2^-86.
        ss = 0.f;
#pragma unroll
        for (int j = 0; j < QV; ++j)
            if ((int)threadIdx.x + j * 256 < p.vecs) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    h[j][e] *= 0x1p100f;
                    ss = fmaf(h[j][e], h[j][e], ss);
                }
            }
        for (int off = 32; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = ss;
        __syncthreads();
        mean = (part[0] + part[1] + part[2] + part[3]) * p.inv_d + p.eps * 0x1p100f * 0x1p100f;
    }
    const float r = mean > 0.f ? 1.0f / sqrtf(mean) : 0.f;               // (a row of zeros with eps 0: zeros)
    float pm = 0.f, ym = 0.f;                    // (ym: for the rare case alone, but a pass over registers)
#pragma unroll
    for (int j = 0; j < QV; ++j) {
        const int i = threadIdx.x + j * 256;
        if (i < p.vecs) {
            float g[8], y[8];
            unpack8(gv[j], g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = h[j][e] * r * g[e];
                pm = fmaxf(pm, fabsf(h[j][e] * g[e]));
                ym = fmaxf(ym, fabsf(y[e]));
            }
            if (p.y) p.y[at + i] = pack8(y);
            if (BLOCK && p.codes) {              // (vecs is a multiple of 16: the 16 lanes of a block are here together)
                for (int off = 8; off > 0; off >>= 1) pm = fmaxf(pm, __shfl_xor(pm, off));
                Code c = code_of(pm, r);
                if (!c.of_p) {
                    for (int off = 8; off > 0; off >>= 1) ym = fmaxf(ym, __shfl_xor(ym, off));
                    c = code_of_y(ym);
                }
                p.codes[at + i] = encode8(h[j], g, r, c);
                if ((threadIdx.x & 15) == 0) p.scales[(int64_t)(i >> 4) * p.rows + row] = c.scale;
                pm = ym = 0.f;
            }
        }
    }
    if (BLOCK || !p.codes) return;
    for (int off = 32; off > 0; off >>= 1) {
        pm = fmaxf(pm, __shfl_xor(pm, off));
        ym = fmaxf(ym, __shfl_xor(ym, off));
    }
    if ((threadIdx.x & 63) == 0) { partm[threadIdx.x >> 6] = pm; party[threadIdx.x >> 6] = ym; }
    __syncthreads();
    Code c = code_of(fmaxf(fmaxf(partm[0], partm[1]), fmaxf(partm[2], partm[3])), r);
    if (!c.of_p) c = code_of_y(fmaxf(fmaxf(party[0], party[1]), fmaxf(party[2], party[3])));
    if (threadIdx.x == 0) p.scales[row] = c.scale;
#pragma unroll
    for (int j = 0; j < QV; ++j) {
        const int i = threadIdx.x + j * 256;
        if (i >= p.vecs) continue;
        float g[8];
        unpack8(gv[j], g);
        p.codes[at + i] = encode8(h[j], g, r, c);
    }
}

template <bool BLOCK, bool ONCE>
void run(const NormQuant& p, hipStream_t s) {
    const dim3 grid((unsigned)p.rows), wg(256);
    if (p.vecs <= 256) hipLaunchKernelGGL((norm_quant_kernel<1, BLOCK, ONCE>), grid, wg, 0, s, p);
    else if (p.vecs <= 512) hipLaunchKernelGGL((norm_quant_kernel<2, BLOCK, ONCE>), grid, wg, 0, s, p);
    else if (p.vecs <= 768) hipLaunchKernelGGL((norm_quant_kernel<3, BLOCK, ONCE>), grid, wg, 0, s, p);
    else if (p.vecs <= 1024) hipLaunchKernelGGL((norm_quant_kernel<4, BLOCK, ONCE>), grid, wg, 0, s, p);
    else hipLaunchKernelGGL((norm_quant_kernel<8, BLOCK, ONCE>), grid, wg, 0, s, p);
}

}  // namespace

void launch_add_rmsnorm_quantize(const bf16_t* x, const bf16_t* delta, const bf16_t* g, bf16_t* h, bf16_t* y, unsigned char* codes, float* scales,
                                 int64_t rows, int d, bool blocks, float eps, hipStream_t s) {
    const NormQuant p = {(const uint4*)x, (const uint4*)delta, (const uint4*)g, (uint4*)h, (uint4*)y, (uint2*)codes, scales, rows, d / 8, eps,
                         1.0f / (float)d};
    // (x and delta past the caches / not, rows of 4096 in blocks: 8192 43.6 / 42.4 us, 12288 61 / 67, 16384 78 / 87)
    const bool once = rows * d * (2 + (delta ? 2 : 0) + (h ? 2 : 0) + (y ? 2 : 0) + (codes ? 1 : 0)) >= READ_ONCE_BYTES;
    if (blocks) { if (once) run<true, true>(p, s); else run<true, false>(p, s); }
    else { if (once) run<false, true>(p, s); else run<false, false>(p, s); }
}

}  // namespace po
