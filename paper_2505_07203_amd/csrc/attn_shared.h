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
    int item0[SHARED_MAX + 1];      // first row tile of each request, and their number
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

// requests in tables of SHARED_MAX, with their row tiles
template <typename F>
void for_tables(const po_request_rows* seq, int n, int group, int rows, F launch) {
    SharedTable tab;
    memset(&tab, 0, sizeof(tab));
    for (int i = 0; i < n;) {
        tab.n = 0;
        int items = 0;
        for (; i < n && tab.n < SHARED_MAX; ++i) {
            if (seq[i].q_len == 0) continue;
            tab.seq[tab.n] = {(int)seq[i].q_row, (int)seq[i].q_len, (int)seq[i].kv_row, (int)seq[i].kv_len};
            tab.item0[tab.n++] = items;
            items += (int)((seq[i].q_len * group + rows - 1) / rows);
        }
        tab.item0[tab.n] = items;
        if (items) launch(tab, items);
    }
}

void launch_attention_shared_bf16(const SharedParams& p, const po_request_rows* seq, int n, int hd, hipStream_t s);
void launch_attention_shared_f32(const SharedParams& p, const po_request_rows* seq, int n, int hd, hipStream_t s);

}  // namespace po
