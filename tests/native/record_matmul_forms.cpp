// Prints the form the library would run a matrix product in.  Reads lines "n_cu M N K ldx shift workspace": shift in elements
// from an aligned address, workspace in bytes.  Prints "form split pack".  No device is touched; the pointers are made up.
#include <cstdio>

#include "gpulet_internal.h"

int main() {
    using namespace gpulet;
    int n_cu, M, N, K, ldx, shift;
    unsigned long long ws;
    while (std::scanf("%d %d %d %d %d %d %llu", &n_cu, &M, &N, &K, &ldx, &shift, &ws) == 7) {
        gpulet_matmul_desc d{};
        d.x = reinterpret_cast<void *>((1ull << 50) + 2ull * static_cast<unsigned>(shift));
        d.w = reinterpret_cast<void *>(1ull << 51);
        d.y = reinterpret_cast<void *>(1ull << 52);
        d.M = M; d.N = N; d.K = K; d.ldx = ldx;
        MatmulArgs a;
        if (check_matmul(&d, a) != GPULET_OK) return 1;
        a.ws = ws ? reinterpret_cast<void *>(1ull << 53) : nullptr;
        a.ws_bytes = ws;
        const MatmulChoice c = choose_matmul(a, n_cu);
        std::printf("%d %d %d\n", static_cast<int>(c.form), c.split, c.pack);
    }
    return 0;
}
