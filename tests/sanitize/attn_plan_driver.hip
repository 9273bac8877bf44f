// Host driver for how attention calls are cut up (test infrastructure, no kernel and no GPU call): reads calls from stdin, a line each (format tree dtype T n_seq Hq Hkv max_q max_kv total_kv sink
// window beside), and prints the rows of a workgroup, the tokens of a tile, the number of ranges, the tiles of a range, and at the end how many microseconds a plan took.
//
// With arguments "fill" it reads pairs of numbers (tokens, rows read back) and prints how many wavefronts a token has and how many rows a lane.
#include <stdio.h>
#include <string.h>

#include <chrono>

#include "ilre_internal.h"

using namespace ilre;

int main(int argc, char **argv)
{
    if (argc > 1 && !strcmp(argv[1], "fill")) {
        int tokens;
        long rows;
        while (scanf("%d %ld", &tokens, &rows) == 2) printf("%d %d\n", fill_wavefronts(tokens), read_rows(rows));
        return 0;
    }
    int format, tree, dtype, T, n, Hq, Hkv, max_q, max_kv, sink, window, beside;
    long total, plans = 0;
    double seconds = 0;
    while (scanf("%d %d %d %d %d %d %d %d %d %ld %d %d %d", &format, &tree, &dtype, &T, &n, &Hq, &Hkv, &max_q, &max_kv, &total, &sink, &window, &beside) == 13) {
        const auto start = std::chrono::steady_clock::now();
        const AttnPlan p = make_attn_plan(dtype, format, tree != 0, T, n, Hq, Hkv, max_q, max_kv, total, sink, window, (size_t)1 << 62, beside != 0);
        seconds += std::chrono::duration<double>(std::chrono::steady_clock::now() - start).count();
        ++plans;
        printf("%d %d %d %d\n", p.rows, p.tile, p.nsplit, p.split_tiles);
    }
    printf("%.3f\n", plans ? seconds / plans * 1e6 : 0.0);
    return 0;
}
