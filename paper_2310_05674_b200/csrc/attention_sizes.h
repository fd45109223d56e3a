// What attention works out from a call's sizes, on the host and in kernels.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define SAMA_HD __host__ __device__
#else
#define SAMA_HD
#endif

namespace sama {

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
