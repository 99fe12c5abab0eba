// Attention of a batch of requests behind one shared prefix, bf16 MFMA (gfx950).
//
// Row i of a request sees all n2 keys of the prefix and its own keys 0 .. kv_len - q_len + i:
//   o = sum over those keys of p v / sum of p,  p = exp(score - maximum)
// All query heads of a KV head are rows of one tile (a request of q_len positions has q_len * group of them), since they share
// their keys.  A lane owns one row: S^T = K Q^T leaves it 16 of a block's 32 keys (its partner lane ^ 32 the others), the
// softmax is per lane, and the probabilities are at once the operand of O^T += V^T P^T (K rows are read in an order that makes
// the eight keys a lane feeds to an MFMA contiguous in V^T, as in attn_mfma.hip).  K and V^T go from memory to
// registers: a wavefront's fragments are whole 16-byte pieces, and what several wavefronts read they find in the caches.
#include "attn_shared.h"

#include <algorithm>

namespace po {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
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

    // 32 keys; see: how many of them this lane's row sees (all of them unless `masked`)
    __device__ __forceinline__ void block(const bf16x8 (&kf)[KS], const bf16x8 (&vf)[2][HT], bool masked, int see, int lhi, float sc) {
        f32x16 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], s, 0, 0, 0);
        if (masked) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if ((r & 7) + 8 * lhi + 16 * (r >> 3) >= see) s[r] = -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
        top = fmaxf(m, other_half_max(top));
        const float ref = top == -INFINITY ? 0.f : top * sc;      // (nothing seen yet: all probabilities come out 0)
        if (__any(top > m)) {                                     // (else every factor is 1)
            const float a = __builtin_amdgcn_exp2f(fmaf(m, sc, -ref));
            l *= a;
#pragma unroll
            for (int ht = 0; ht < HT; ++ht)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[ht][r] *= a;
            m = top;
        }
        bf16x8 pf[2];
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float e = __builtin_amdgcn_exp2f(fmaf(s[r], sc, -ref));
            sum += e;
            pf[r >> 3][r & 7] = (__bf16)e;        // (the one rounding of a probability: the matrix instruction's operand)
        }
        l += sum;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int ht = 0; ht < HT; ++ht) acc[ht] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[j][ht], pf[j], acc[ht], 0, 0, 0);
    }
};

// One workgroup: a tile of rows of one request and KV head, all its keys.
// SPLIT: the tile is 32 rows and the wavefronts take every NW-th block of keys each, meeting in LDS at the end (few rows, one
// token of a request: what counts is how many keys are on their way at once); otherwise each wavefront has 32 rows of its own.
template <int HD, int NW, bool SPLIT>
__global__ void __launch_bounds__(NW * 64) attn_shared_kernel(const SharedParams p, const SharedTable tab) {
    constexpr int KS = HD / 16, HT = HD / 32, ROWS = SPLIT ? 32 : 32 * NW;
    extern __shared__ __attribute__((aligned(16))) float lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l31 = lane & 31, lhi = lane >> 5;
    const int kvh = (int)(blockIdx.x % (unsigned)p.Hkv), item = (int)(blockIdx.x / (unsigned)p.Hkv);
    const int req = __builtin_amdgcn_readfirstlane(shared_request(tab, item));
    const SharedSeq sq = tab.seq[req];
    const int group = p.Hq / p.Hkv;
    const int row0 = (item - tab.item0[req]) * ROWS + (SPLIT ? 0 : wave * 32);      // of this wavefront, in (position, head) order
    const int n_rows = sq.q_len * group;
    if (!SPLIT && row0 >= n_rows) return;
    const int vr = min(row0 + l31, n_rows - 1);
    const int pos = vr / group, head = kvh * group + vr - pos * group;
    const bool valid = row0 + l31 < n_rows;
    const int64_t orow = ((int64_t)(sq.q_row + pos) * p.Hq + head) * HD;
    const int see = sq.kv_len - sq.q_len + pos + 1;            // own keys this row sees (may be below 0)
    // own keys that any, and that every, row of the wavefront sees
    const int see_max = max(0, sq.kv_len - sq.q_len + min(row0 + 31, n_rows - 1) / group + 1);
    const int see_min = sq.kv_len - sq.q_len + row0 / group + 1;

    Rows<HD> st;
    st.start((const bf16_t*)p.q + orow + lhi * 8, valid);
    const int pk = (l31 & 0x13) | ((l31 & 4) << 1) | ((l31 & 8) >> 1);       // MFMA row i holds key pi(i): bits 2, 3 swapped
    const int64_t krs = (int64_t)p.Hkv * HD;
    const bf16_t* const ko = (const bf16_t*)p.k + (int64_t)sq.kv_row * krs + kvh * HD + lhi * 8;
    const bf16_t* const kp = (const bf16_t*)p.k2 + kvh * HD + lhi * 8;
    const bf16_t* const vo = (const bf16_t*)p.v + ((int64_t)kvh * HD + l31) * p.ldv + sq.kv_row;
    const bf16_t* const vp = (const bf16_t*)p.v2 + ((int64_t)kvh * HD + l31) * p.ldv2;
    const int nb2 = (p.n2 + 31) / 32, nb = nb2 + (see_max + 31) / 32;
    // K rows of block b; past the last key the last one (those scores are masked)
    auto load_k = [&](int b, bf16x8 (&kf)[KS]) {
        const bool own = b >= nb2;
        const int key = (own ? b - nb2 : b) * 32 + pk;
        const bf16_t* const r = (own ? ko : kp) + (int64_t)min(key, (own ? sq.kv_len : p.n2) - 1) * krs;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks] = __builtin_bit_cast(bf16x8, *(const uint4*)(r + ks * 16));
    };
    // V^T of block b; columns past the last key count as 0, whatever they hold
    auto load_v = [&](int b, bf16x8 (&vf)[2][HT]) {
        const bool own = b >= nb2;
        const int key0 = (own ? b - nb2 : b) * 32, end = own ? sq.kv_len : p.n2;
        const bf16_t* const r = own ? vo : vp;
        const int64_t ld = own ? p.ldv : p.ldv2;
        if (key0 + 32 <= end) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int ht = 0; ht < HT; ++ht)
                    vf[j][ht] = __builtin_bit_cast(bf16x8, *(const uint4*)(r + ht * 32 * ld + key0 + 16 * j + 8 * lhi));
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int key = key0 + 16 * j + 8 * lhi, n = end - key;        // n of the eight are keys
                uint32_t mask[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) mask[w] = n >= 2 * w + 2 ? 0xffffffffu : n == 2 * w + 1 ? 0xffffu : 0u;
#pragma unroll
                for (int ht = 0; ht < HT; ++ht) {
                    uint4 t = make_uint4(0, 0, 0, 0);
                    if (n > 0) t = *(const uint4*)(r + ht * 32 * ld + key);
                    t.x &= mask[0]; t.y &= mask[1]; t.z &= mask[2]; t.w &= mask[3];
                    vf[j][ht] = __builtin_bit_cast(bf16x8, t);
                }
            }
        }
    };
    const int step = SPLIT ? NW : 1;
    bf16x8 kf[KS], kn[KS], vf[2][HT];
    int b = SPLIT ? wave : 0;
    if (b < nb) load_k(b, kf);
    for (; b < nb; b += step) {
        load_v(b, vf);
        if (b + step < nb) load_k(b + step, kn);
        const bool own = b >= nb2;
        const int key0 = (own ? b - nb2 : b) * 32;
        st.block(kf, vf, key0 + 32 > (own ? see_min : p.n2), (own ? see : p.n2) - key0, lhi, p.sc);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks] = kn[ks];
    }
    bf16_t* const o = (bf16_t*)p.o;
    const float l = other_half_sum(st.l);
    if (!SPLIT) {
        if (!valid) return;
        const float inv = l > 0.f ? 1.0f / l : 0.f;             // (a row that sees nothing: 0)
#pragma unroll
        for (int ht = 0; ht < HT; ++ht)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                uint2 w;
                w.x = (uint32_t)f2bf(st.acc[ht][4 * g] * inv) | ((uint32_t)f2bf(st.acc[ht][4 * g + 1] * inv) << 16);
                w.y = (uint32_t)f2bf(st.acc[ht][4 * g + 2] * inv) | ((uint32_t)f2bf(st.acc[ht][4 * g + 3] * inv) << 16);
                *(uint2*)(o + orow + ht * 32 + 8 * g + 4 * lhi) = w;
            }
        return;
    }
    // SPLIT: [wave][row][HD + 4] accumulators, then [wave][row] maxima and sums, joined in wavefront order
    constexpr int LD = HD + 4;
    float* const sm = lds + NW * 32 * LD;
    float* const sl = sm + NW * 32;
    if (lhi == 0) { sm[wave * 32 + l31] = st.m; sl[wave * 32 + l31] = l; }
#pragma unroll
    for (int ht = 0; ht < HT; ++ht)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *(float4*)(lds + (wave * 32 + l31) * LD + ht * 32 + 8 * g + 4 * lhi) =
                make_float4(st.acc[ht][4 * g], st.acc[ht][4 * g + 1], st.acc[ht][4 * g + 2], st.acc[ht][4 * g + 3]);
    __syncthreads();
    constexpr int PER = NW * 64 / 32, DV = HD / PER;            // threads of a row, values of a thread
    const int jr = tid / PER, d0 = tid % PER * DV;
    const int jv = row0 + jr;
    if (jv >= n_rows) return;
    float top = sm[jr];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, sm[w * 32 + jr]);
    float lt = 0.f, y[DV];
#pragma unroll
    for (int e = 0; e < DV; ++e) y[e] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const float mw = sm[w * 32 + jr];
        const float f = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - top) * p.sc);
        lt += f * sl[w * 32 + jr];
#pragma unroll
        for (int e = 0; e < DV; ++e) y[e] += f * lds[(w * 32 + jr) * LD + d0 + e];
    }
    const float inv = lt > 0.f ? 1.0f / lt : 0.f;
    const int jp = jv / group;
    bf16_t* const op = o + ((int64_t)(sq.q_row + jp) * p.Hq + kvh * group + jv - jp * group) * HD + d0;
#pragma unroll
    for (int e = 0; e < DV; e += 4) {
        uint2 w;
        w.x = (uint32_t)f2bf(y[e] * inv) | ((uint32_t)f2bf(y[e + 1] * inv) << 16);
        w.y = (uint32_t)f2bf(y[e + 2] * inv) | ((uint32_t)f2bf(y[e + 3] * inv) << 16);
        *(uint2*)(op + e) = w;
    }
}

template <int HD>
void launch_t(const SharedParams& p, const po_request_rows* seq, int n, hipStream_t s) {
    constexpr int SPLIT_LDS = (8 * 32 * (HD + 4) + 2 * 8 * 32) * 4;
    static OncePerDevice lds;
    lds.run(current_device(), [] { allow_dynamic_lds((const void*)(attn_shared_kernel<HD, 8, true>), SPLIT_LDS); });
    const int group = p.Hq / p.Hkv;
    int64_t longest = 0;
    for (int i = 0; i < n; ++i) longest = std::max<int64_t>(longest, seq[i].q_len);
    if (longest * group <= 32)
        for_tables(seq, n, group, 32, [&](const SharedTable& tab, int items) {
            hipLaunchKernelGGL((attn_shared_kernel<HD, 8, true>), dim3((unsigned)items * p.Hkv), dim3(512), SPLIT_LDS, s, p, tab);
        });
    else
        for_tables(seq, n, group, 128, [&](const SharedTable& tab, int items) {
            hipLaunchKernelGGL((attn_shared_kernel<HD, 4, false>), dim3((unsigned)items * p.Hkv), dim3(256), 0, s, p, tab);
        });
}

}  // namespace

void launch_attention_shared_bf16(const SharedParams& p, const po_request_rows* seq, int n, int hd, hipStream_t s) {
    if (hd == 128) launch_t<128>(p, seq, n, s);
    else launch_t<64>(p, seq, n, s);
}

}  // namespace po
