// Sizes that the operators without a model work out on the host and in their kernels, checked on the CPU.
#include <cstdio>

#include "ops.h"

using namespace rnnlm;

#define CHECK(c) do { if (!(c)) { printf("%s:%d: %s\n", __FILE__, __LINE__, #c); return 1; } } while (0)

// What is copied to LDS is in the list: nothing behind it is read, however many words were counted.
static int list_of_a_long_row() {
    const int sizes[] = {65537, 70000, 100000, 131072, 131073, 140000, 196607, 196608, 196609, 200000, 1000000, 1 << 30};
    for (int V : sizes)
        for (int listed = 0; listed < 80000; ++listed)
            if (list_in_lds(listed, V)) CHECK(listed <= long_list(V) && listed <= kLongHeld);
    CHECK(list_in_lds(8192, 70000) && !list_in_lds(8193, 70000) && list_in_lds(12288, 200000) && !list_in_lds(12289, 200000));
    return 0;
}

// The gradient alone: a grid of fewer than 2^32 threads for every number of rows and words that is taken, and segments that cover a row.
static int segments_of_the_gradient() {
    const int rows[] = {1, 3, 509, 65536, 1000003, (1 << 21) - 1, 1 << 21}, words[] = {1, 7, 8192, 8193, 20011, 57344, 57345, 65536, 70001, 1000000, (1 << 30) - 1, 1 << 30};
    for (int N : rows)
        for (int V : words)
            for (int E = 4; E <= 8; E += 4) {
                const Cut c = cut_for_backward(N, V, E);
                CHECK(c.segments >= 1 && c.len % E == 0 && (long long)c.segments * N * kDistillThreads < (1ll << 32));
                CHECK((long long)c.segments * c.len >= V && (long long)(c.segments - 1) * c.len < V);
                CHECK(N > 65536 || V > 1000000 || c.len <= 8192);
            }
    return 0;
}

int main() {
    if (list_of_a_long_row() || segments_of_the_gradient()) return 1;
    puts("ok");
    return 0;
}
