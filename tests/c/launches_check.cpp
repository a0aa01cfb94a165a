// Work cut into launches (fc_launches.h): every unit is in exactly one part, in
// order, and no part reaches 2^32 threads, at the operators' documented limits.
#include <cstdio>

#include "fc_launches.h"

static int fails = 0;

static void check(const char* what, int64_t units, int64_t threads) {
    int64_t next = 0, parts = 0;
    fc::by_launches(units, threads, [&](int64_t first, int64_t count) {
        const int64_t blocks = (count * threads + 255) / 256;
        if (first != next || count < 1 || blocks * 256 >= (int64_t)1 << 32) ++fails;
        next = first + count;
        ++parts;
    });
    if (next != (units > 0 ? units : 0) || (units > 0 && units * threads <= fc::LAUNCH_THREADS && parts != 1)) {
        std::printf("%s: %lld of %lld units in %lld launches\n", what, (long long)next, (long long)units, (long long)parts);
        ++fails;
    }
}

int main() {
    for (int64_t threads = 1; threads <= 256; threads *= 2) {
        check("looked-up rows", ((int64_t)1 << 31) - 1, threads);
        check("looked-up rows", ((int64_t)1 << 24) + 3, threads);
        check("looked-up rows", 1, threads);
    }
    check("chunks of a gradient", (int64_t)1 << 25, 256);
    check("joins of one chunk", 0, 256);
    check("no chunks", -1, 256);
    for (int64_t rows : {(int64_t)1, (int64_t)1 << 20, (int64_t)1 << 21})
        for (int64_t len : {1, 8, 4096, 513, (1 << 21) - 1, 1 << 21}) check("rows of elements or vectors", rows, len);
    std::printf("%s\n", fails ? "failed" : "ok");
    return fails != 0;
}
