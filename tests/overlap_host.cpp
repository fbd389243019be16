// bs_overlap.cuh on the host.  stdin: at st sh T H d element of two arrays a line; stdout: 1 where they share a byte, else 0.
#include <stdio.h>

#include "bs_overlap.cuh"

int main() {
    long long v[14];
    for (;;) {
        for (auto& x : v)
            if (scanf("%lld", &x) != 1) return 0;
        auto of = [&](const long long* w) { return bs::rows_of((const void*)(uintptr_t)w[0], w[1], w[2], w[3], w[4], w[5], w[6]); };
        printf("%d\n", bs::rows_overlap(of(v), of(v + 7)) ? 1 : 0);
    }
}
