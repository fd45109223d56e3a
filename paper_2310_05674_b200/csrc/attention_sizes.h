// What attention works out from a call's sizes, on the host and in kernels.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define SAMA_HD __host__ __device__
#else
#define SAMA_HD
#endif

namespace sama {

struct AttnText {
    int q0, lq, k0, lk, prefix;   // first row and number of queries and keys; prefix: keys that every query sees
};
// The position of query i of a text, a tile's rows behind its last among them.  (i + lk might pass 31 bits.)
SAMA_HD inline int attn_position(const AttnText& x, int i) { return i - (x.lq - x.lk); }
// Query i sees keys 0 .. result - 1: more of them, never fewer, as i grows.
SAMA_HD inline int attn_seen(int causal, const AttnText& x, int i) {
    if (!causal) return x.lk;
    const int past = attn_position(x, i) + 1, seen = past > x.prefix ? past : x.prefix;
    return seen < 0 ? 0 : seen < x.lk ? seen : x.lk;
}
// Key j is seen by queries result .. lq - 1.
SAMA_HD inline int attn_first_query(int causal, const AttnText& x, int j) {
    if (!causal || j < x.prefix) return 0;
    const int i = j - (x.lk - x.lq);
    return i > 0 ? i : 0;
}

// A sequence's keys are counted in 31 bits, and worked on in steps of 64: the last step has to be countable, too.
constexpr int kPagedStep = 64;
constexpr int64_t kPagedMostKeys = 0x7fffffff / kPagedStep * kPagedStep;
SAMA_HD inline int64_t paged_most_keys(int64_t max_pages, int64_t page_size) {
    const int64_t table = max_pages * page_size;
    return table < kPagedMostKeys ? table : kPagedMostKeys;
}
// The length as it is used: the nearest that the table holds.
SAMA_HD inline int paged_keys(int length, int64_t max_pages, int64_t page_size) {
    const int64_t most = paged_most_keys(max_pages, page_size);
    return length < 0 ? 0 : length > most ? (int)most : length;
}
SAMA_HD inline int paged_steps(int keys) { return (keys + (kPagedStep - 1)) / kPagedStep; }

}  // namespace sama
