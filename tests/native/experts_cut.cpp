// Host-only (experts_cut.h): how calls of products grouped by expert are cut.  Reads, a line each, a product (0 linear, 1 input gradient, 2 weight
// gradient), a type, whether memory can fill tiles directly, and rows, experts, outs and ins; prints the cut, the splits and, of tiles of
// 256, how `tiles` of them, the line's last number, end: 0 in whole rounds, 1 in tiles, 2 in quarters, 3 in small tiles, plus 4 where whole rounds
// go before.
#include <cstdio>

#include "experts_cut.h"

using namespace dear_ops;

int main()
{
    int kind, direct;
    unsigned tiles;
    long long rows;
    dear_experts_t x = {};
    while (std::scanf("%d %d %d %lld %d %d %d %u", &kind, &x.dtype, &direct, &rows, &x.experts, &x.outs, &x.ins, &tiles) == 8) {
        x.rows = rows;
        const choice c = kind == LINEAR ? choose_cut<LINEAR>(x, direct) : kind == INPUT_GRAD ? choose_cut<INPUT_GRAD>(x, direct) : choose_cut<WEIGHT_GRAD>(x, direct);
        const int over = tiles % CUS;
        const int end = over == 0 ? 0 : over > MOST_IN_QUARTERS ? 1 : kind == WEIGHT_GRAD || over > MOST_SMALL ? 2 : 3;
        std::printf("%d %d %d\n", (int)c.how, c.splits, c.how == WIDE ? end + (tiles / CUS ? 4 : 0) : 0);
    }
    return 0;
}
