// Prints how the operators' products are computed (fc_choice.h), a line for each line read:
//   ckpt MAX_TOKENS MAX_OUTS DIM TOKENS OUTS     a weight's gradient
//   product ROWS DIM MAX_TOKENS TOKENS           of two packed matrices
//   linear ROWS DIM MAX_TOKENS TOKENS            with its inputs packed on the way
// "NAME SPLITS", of the launch of at most 2^18 tokens that comes first.
#include <cstdio>
#include <cstring>

#include "fc_choice.h"

int main() {
    static const char* const dw[] = {"LARGE", "BROAD", "MIDDLE", "TINY"};
    static const char* const four[] = {"WIDE4", "HALF4", "SMALL4"};
    char op[16];
    while (std::scanf("%15s", op) == 1) {
        long long a, b, c, n, outs = 0;
        if (std::scanf("%lld %lld %lld %lld", &a, &b, &c, &n) != 4) return 1;
        if (!std::strcmp(op, "ckpt")) {
            if (std::scanf("%lld", &outs) != 1) return 1;
            const Choice q = ckpt_choice(n, outs, c, ckpt_sums(b, c));
            if (ckpt_small(q, n, outs, c)) std::printf("FEW 1\n");
            else std::printf("%s %d\n", dw[q.kind], q.splits);
            continue;
        }
        if (!std::strcmp(op, "linear") && mxfp_few(n, a, b)) {
            std::printf("FEW 1\n");
        } else if (!std::strcmp(op, "linear") && mxfp_small(n, a, b)) {
            std::printf("SMALL 1\n");
        } else {
            const Choice q = mxfp_choice(std::min<int64_t>(n, MXFP_CHUNK), a, b, mxfp_sums(c, a));
            std::printf("%s %d\n", four[q.kind], q.splits);
        }
    }
    return 0;
}
