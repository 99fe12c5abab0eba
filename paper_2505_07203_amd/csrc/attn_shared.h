// Attention of a batch of requests behind one shared prefix: what its kernels share.
#pragma once
#include "../../include/po.h"
#include "po_internal.h"

#include <string.h>

namespace po {

// Requests of one launch, passed by value (a captured launch keeps them, and nothing has to be copied to the device first).
constexpr int SHARED_MAX = 128;
struct SharedSeq {
    int q_row, q_len;      // rows of q and o
    int kv_row, kv_len;    // rows of k (columns of V^T); query i of the request sees own keys 0 .. kv_len - q_len + i
};
struct SharedTable {
    int n;
    SharedSeq seq[SHARED_MAX];
    int item0[SHARED_MAX + 1];      // first work item of each request, and their number
    int row0[SHARED_MAX + 1];       // first row of each request when all of them are counted through, and their number
};
struct SharedParams {
    const void *q, *k, *v, *k2, *v2;
    void* o;
    int64_t ldv, ldv2;     // pitches of V^T (bf16)
    int n2;                // keys of the prefix
    int Hq, Hkv;
    float sc;              // scores times this are exponents of 2 (bf16) or e (float32)
};

// the request a row tile belongs to (item0 ascends); every lane of a wavefront gets the answer
__device__ __forceinline__ int shared_request(const SharedTable& t, int item) {
    const int lane = threadIdx.x & 63;
    int n = 0;
#pragma unroll
    for (int i = 0; i < SHARED_MAX; i += 64) n += __popcll(__ballot(i + lane < t.n && t.item0[i + lane + 1] <= item));
    return n;
}

// the request of row c of the table
__device__ __forceinline__ int shared_request_of_row(const SharedTable& t, int c) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.row0[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 shared_bf16x8;
// Eight keys (key on; a multiple of 8) of V^T rows r, r + 32, .. of pitch ld.  Keys from `end` on count as 0, whatever the columns hold:
// a probability of 0 times a NaN would be one.
template <int HT>
__device__ __forceinline__ void load_vt_eight(const bf16_t* r, int64_t ld, int key, int end, shared_bf16x8 (&v)[HT]) {
    const int n = end - key;
    if (n >= 8) {
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) v[ht] = __builtin_bit_cast(shared_bf16x8, *(const uint4*)(r + ht * 32 * ld + key));
        return;
    }
    uint32_t mask[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) mask[w] = n >= 2 * w + 2 ? 0xffffffffu : n == 2 * w + 1 ? 0xffffu : 0u;
#pragma unroll
    for (int ht = 0; ht < HT; ++ht) {
        uint4 t = make_uint4(0, 0, 0, 0);
        if (n > 0) t = *(const uint4*)(r + ht * 32 * ld + key);
        t.x &= mask[0]; t.y &= mask[1]; t.z &= mask[2]; t.w &= mask[3];
        v[ht] = __builtin_bit_cast(shared_bf16x8, t);
    }
}

// Requests [i, n) into a table until it is full (those without a row are left out); items(request): how many work items it has.
// -> the first request that is not in it
template <typename F>
int fill_table(SharedTable& tab, const po_request_rows* seq, int i, int n, F items) {
    memset(&tab, 0, sizeof(tab));
    for (; i < n && tab.n < SHARED_MAX; ++i) {
        if (seq[i].q_len == 0) continue;
        const SharedSeq q = {(int)seq[i].q_row, (int)seq[i].q_len, (int)seq[i].kv_row, (int)seq[i].kv_len};
        tab.seq[tab.n] = q;
        tab.item0[tab.n + 1] = tab.item0[tab.n] + items(q);
        tab.row0[tab.n + 1] = tab.row0[tab.n] + q.q_len;
        ++tab.n;
    }
    return i;
}

// (attn_mfma.hip) the prefix in `pieces` pieces and, own, the requests' own keys; head dimension 128, at least one whole tile of 64
// keys, pieces <= tiles.  More than one piece or without the own keys: partial results of every row of the table in opart, mlpart.
// -> the number of pieces that it came to
int launch_attention_shared_tiles(const SharedParams& p, const SharedTable& tab, int pieces, bool own, float* opart, float* mlpart, hipStream_t s);
// scratch (may be null): for partial results; attention_shared_scratch: how much of it the requests can use
size_t attention_shared_scratch(const po_request_rows* seq, int n, int Hq, int Hkv, int hd, int64_t n2);
// how the first table of them runs with that much, as the public enumeration has it
void attention_shared_form(const po_request_rows* seq, int n, int Hq, int Hkv, int hd, int64_t n2, size_t scratch_bytes, int* form, int* pieces);
void launch_attention_shared_bf16(const SharedParams& p, const po_request_rows* seq, int n, int hd, float* scratch, size_t scratch_bytes,
                                  hipStream_t s);
void launch_attention_shared_f32(const SharedParams& p, const po_request_rows* seq, int n, int hd, hipStream_t s);

}  // namespace po
