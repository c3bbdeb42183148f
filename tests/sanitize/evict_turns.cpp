// The turns of the eviction's search for the digits of a rank, on the CPU: which array of bins each turn counts into, reads and clears (kv8.hpp), against
// what its one barrier orders.  Wavefronts run between barriers in any order, so what one writes there no other may touch.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "kv8.hpp"

using namespace slora;

struct Access {
    int array;
    bool clears, adds; // else it reads; additions are atomic and go together
};

int main()
{
    for (int turns = 1; turns <= 8; ++turns) {
        std::vector<std::vector<Access>> between(turns + 2); // of one wavefront, between barrier i - 1 and barrier i
        std::vector<int> count_of(turns);
        int array = 0;
        between[0].push_back({array, true, false}); // the first array is cleared, then a barrier
        for (int t = 0; t < turns; ++t, array = kv_next_bins(array)) {
            count_of[t] = array;
            between[t + 1].push_back({array, false, true});
            if (t + 1 < turns) between[t + 1].push_back({kv_next_bins(array), true, false});
            between[t + 2].push_back({array, false, false}); // behind the turn's barrier
        }
        for (size_t i = 0; i < between.size(); ++i)
            for (const Access &a : between[i])
                for (const Access &b : between[i]) // of another wavefront
                    if (a.array == b.array && a.clears != b.clears) {
                        std::printf("turns %d: array %d is cleared by one wavefront and %s by another between barriers %zu and %zu\n", turns, a.array,
                                    (a.clears ? b : a).adds ? "counted into" : "read", i, i + 1);
                        return 1;
                    } else if (a.array == b.array && a.adds != b.adds && !a.clears && !b.clears) {
                        std::printf("turns %d: array %d is counted into and read between barriers %zu and %zu\n", turns, a.array, i, i + 1);
                        return 1;
                    }
        // every turn's array has been cleared since it was last counted into
        for (int t = 1; t < turns; ++t)
            if (kv_next_bins(count_of[t - 1]) != count_of[t]) return 1;
    }
    std::puts("evict_turns OK");
    return 0;
}
