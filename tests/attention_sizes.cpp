// Prints, for each line of the standard input, what attention's kernels work out from a call's sizes.  Built so that a result
// that 32 bits do not hold ends the program.
//   paged LENGTH MAX_PAGES PAGE_SIZE  ->  keys that are used, steps, the position of the last step's last key
#include <cstdio>
#include <cstring>

#include "attention_sizes.h"

int main() {
    char what[16];
    while (std::scanf("%15s", what) == 1) {
        int length;
        long long pages, page;
        if (std::strcmp(what, "paged") == 0 && std::scanf("%d %lld %lld", &length, &pages, &page) == 3) {
            const int keys = sama::paged_keys(length, pages, page), steps = sama::paged_steps(keys);
            std::printf("%d %d %d\n", keys, steps, steps > 0 ? (steps - 1) * sama::kPagedStep + (sama::kPagedStep - 1) : -1);
        } else {
            return 1;
        }
    }
    return 0;
}
