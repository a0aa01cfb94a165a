// Prints how the operators' products are computed (fc_choice.h), a line for each line read:
//   ckpt MAX_TOKENS MAX_OUTS DIM TOKENS OUTS     a weight's gradient
//   product ROWS DIM MAX_TOKENS TOKENS           of two packed matrices
//   linear ROWS DIM MAX_TOKENS TOKENS            with its inputs packed on the way
// "NAME SPLITS FLOATS ROOM", of the launch of at most 2^18 tokens that comes first: the
// partial sums that it writes and those that the plan has.
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
            const Choice q = ckpt_choice(n, outs, c, ckpt_limit(b, c));
            const bool few = ckpt_small(q, n, outs, c);
            const int splits = few ? 1 : q.splits;
            std::printf("%s %d %lld %lld\n", few ? "FEW" : dw[q.kind], splits, splits > 1 ? splits * outs * c : 0, (long long)ckpt_room(a, b, c));
            continue;
        }
        n = std::min<long long>(n, MXFP_CHUNK);
        const long long room = mxfp_room(c, a, b);
        if (!std::strcmp(op, "linear") && mxfp_few(n, a, b)) {
            std::printf("FEW 1 0 %lld\n", room);
        } else if (!std::strcmp(op, "linear") && mxfp_small(n, a, b)) {
            std::printf("SMALL 1 0 %lld\n", room);
        } else {
            const Choice q = mxfp_choice(n, a, b, mxfp_limit(c, a));
            std::printf("%s %d %lld %lld\n", four[q.kind], q.splits, q.splits > 1 ? q.splits * n * a : 0, room);
        }
    }
    return 0;
}
