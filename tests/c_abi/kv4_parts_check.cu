/* The merge of a 4-bit decode finds a unit's partial results from two notes in the workspace.  True notes give the slots from the first
 * worker's to the last one's; whatever else stands there, nothing but the slots of workers is named. */
#include <climits>
#include <cstdio>
#include <random>

#include "kv4.cuh"

int main() {
    std::mt19937 rng(1);
    auto any = [&](int workers) -> int {
        switch (rng() % 5) {
            case 0: return (int)rng();
            case 1: return (int)(rng() % (unsigned)workers);
            case 2: return workers - 1 + (int)(rng() % 3);
            case 3: return rng() % 2 ? INT_MAX : INT_MIN;
            default: return (int)(rng() % 5) - 2;
        }
    };
    for (int i = 0; i < 2000000; ++i) {
        const int workers = 2 + (int)(rng() % 2400), first = any(workers), last = any(workers);
        int begin = -1;
        const int n = loma::kv4_parts(first, last, workers, &begin);
        const bool inside = n >= 0 && begin >= 0 && begin < workers && n <= workers - begin;
        const bool truly = first >= 0 && first <= last && last < workers;
        if (!inside || (truly && (begin != first || n != last - first + 1)) || (first == 1 && last == 0 && n != 0)) {
            std::printf("workers %d, notes %d and %d: %d from %d\n", workers, first, last, n, begin);
            return 1;
        }
    }
    std::printf("kv4 parts ok\n");
    return 0;
}
