// Prints, for each line of the standard input, what attention's kernels work out from a call's sizes.  Built so that a result
// that 32 bits do not hold ends the program.
//   query CAUSAL LQ LK PREFIX ROW     ->  position of a row of the queries, keys that it sees
//   key CAUSAL LQ LK PREFIX ROW       ->  the first query that sees a key
//   paged LENGTH MAX_PAGES PAGE_SIZE  ->  keys that are used, steps, the position of the last step's last key
#include <cstdio>
#include <cstring>

#include "attention_sizes.h"

int main() {
    char what[16];
    sama::AttnText x = {};
    while (std::scanf("%15s", what) == 1) {
        int length, causal, row;
        long long pages, page;
        if (std::strcmp(what, "paged") == 0 && std::scanf("%d %lld %lld", &length, &pages, &page) == 3) {
            const int keys = sama::paged_keys(length, pages, page), steps = sama::paged_steps(keys);
            std::printf("%d %d %d\n", keys, steps, steps > 0 ? (steps - 1) * sama::kPagedStep + (sama::kPagedStep - 1) : -1);
        } else if (std::scanf("%d %d %d %d %d", &causal, &x.lq, &x.lk, &x.prefix, &row) != 5) {
            return 1;
        } else if (std::strcmp(what, "query") == 0) {
            std::printf("%d %d\n", sama::attn_position(x, row), sama::attn_seen(causal, x, row));
        } else if (std::strcmp(what, "key") == 0) {
            std::printf("%d\n", sama::attn_first_query(causal, x, row));
        } else {
            return 1;
        }
    }
    return 0;
}
