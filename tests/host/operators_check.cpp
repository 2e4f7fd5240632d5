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

int main() {
    if (list_of_a_long_row()) return 1;
    puts("ok");
    return 0;
}
