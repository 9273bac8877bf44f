// Host driver for the numbering of the attention kernels' units (test infrastructure, no kernel and no GPU call): calls of several sequences, cut up as the library
// cuts them; every number of the grid is taken as a workgroup takes it, and every range that the merge adds up has to have been taken, once.  And no lookup of a page reads
// an entry past its sequence's length.
//
// With arguments "plan" it reads calls from stdin, a line each (dtype T n_seq Hq Hkv max_q max_kv total_kv sink window), and prints the rows of a workgroup and
// the number of ranges.
#include <stdio.h>
#include <string.h>

#include <algorithm>
#include <vector>

#include "attn_blocks.h"
#include "ilre_internal.h"

using namespace ilre;

struct Call {
    int dtype, Hq, Hkv;
    Mask m;
    std::vector<int> q, kv;
    int T() const { return sum(q); }
    static int sum(const std::vector<int> &x)
    {
        int n = 0;
        for (int y : x) n += y;
        return n;
    }
};

static void print(const Call &c, const AttnPlan &p)
{
    printf("dtype %d heads %d/%d causal %d sink %d window %d rows %d tile %d ranges %d of %d:", c.dtype, c.Hq, c.Hkv, c.m.causal, c.m.sink, c.m.window, p.rows, p.tile,
           p.nsplit, p.split_tiles);
    for (size_t s = 0; s < c.q.size(); ++s) printf(" %d of %d", c.q[s], c.kv[s]);
    printf("\n");
}

// Ranges that nobody takes, that two take, and numbers beyond the grid.
static int faults(const Call &c, const AttnPlan &p)
{
    const int G = c.Hq / c.Hkv, n = (int)c.q.size();
    std::vector<Block> seq(n);
    std::vector<std::vector<int>> taken(n);  // [block * nsplit + range]
    std::vector<long> first(n + 1, 0);
    int bad = 0;
    for (int s = 0; s < n; ++s) {
        Block b{};
        b.seq = s, b.q_len = c.q[s], b.kv = c.kv[s], b.nrows = c.q[s] * G;
        seq[s] = b;
        taken[s].assign((size_t)blocks_of(b, p.rows) * p.nsplit, 0);
        first[s + 1] = first[s] + units_of(b, c.m, G, p.rows, p.tile, p.split_tiles, p.nsplit);
    }
    const long grid = (long)p.nsplit * p.nblocks;
    if (n > 1 && first[n] > grid) ++bad;
    for (long w = 0; w < grid; ++w) {
        const int s = n == 1 ? 0 : (int)(std::upper_bound(first.begin(), first.end(), w) - first.begin()) - 1;
        if (s >= n) break;
        Block b = seq[s];
        int split = -1;
        if (!take_unit(b, (int)(w - (n == 1 ? 0 : first[s])), c.m, G, p.rows, p.tile, p.split_tiles, p.nsplit, split)) continue;
        if (split < 0 || split >= p.nsplit || b.rows0 < 0 || b.rows0 >= b.nrows)
            ++bad;
        else
            ++taken[s][(size_t)(b.rows0 / p.rows) * p.nsplit + split];
    }
    for (int s = 0; s < n; ++s)
        for (int i = 0; i < blocks_of(seq[s], p.rows); ++i) {
            Block b = seq[s];
            b.rows0 = i * p.rows;
            tiles_of(b, c.m, G, p.rows, p.tile);
            const int ranges = ranges_of(b.nt, p.split_tiles, p.nsplit);
            // whatever token of its tiles, or behind them, a workgroup looks up: the entry is one of the sequence's
            const int shift = 4 + i % 3, width = ((b.kv + 9000) >> shift) + 1;
            for (int k = 0; k < b.nt; k += 1 + b.nt / 4)
                for (int t = tile_token(b, b.nt - 1 - k, p.tile), e = t + p.tile + 64; t < e; t += 16) {
                    const int at = page_column(b, t, shift, width);
                    if (at < 0 || at > (b.kv - 1) >> shift || (t < b.hi && at != t >> shift)) ++bad;
                }
            for (int k = 0; k < p.nsplit; ++k)
                if (taken[s][(size_t)i * p.nsplit + k] != (k < ranges)) ++bad;
        }
    return bad;
}

static AttnPlan plan_of(const Call &c, int max_q, int max_kv, int64_t total_kv, double share)
{
    // the workspace that a caller asks for, or a share of it
    const size_t bytes = make_attn_plan(c.dtype, c.T(), (int)c.q.size(), c.Hq, c.Hkv, max_q, max_kv, total_kv, 0, 0, (size_t)1 << 62).bytes;
    return make_attn_plan(c.dtype, c.T(), (int)c.q.size(), c.Hq, c.Hkv, max_q, max_kv, total_kv, c.m.sink, c.m.window, (size_t)(bytes * share));
}

int main(int argc, char **argv)
{
    if (argc > 1 && !strcmp(argv[1], "plan")) {
        int dtype, T, n, Hq, Hkv, max_q, max_kv, sink, window;
        long total;
        while (scanf("%d %d %d %d %d %d %d %ld %d %d", &dtype, &T, &n, &Hq, &Hkv, &max_q, &max_kv, &total, &sink, &window) == 10) {
            const size_t bytes = make_attn_plan(dtype, T, n, Hq, Hkv, max_q, max_kv, total, 0, 0, (size_t)1 << 62).bytes;
            const AttnPlan p = make_attn_plan(dtype, T, n, Hq, Hkv, max_q, max_kv, total, sink, window, bytes);
            printf("%d %d\n", p.rows, p.nsplit);
        }
        return 0;
    }
    int failures = 0;
    long calls = 0, cut = 0;
    auto check = [&](const Call &c, const AttnPlan &p) {
        ++calls;
        cut += p.nsplit > 1;
        if (faults(c, p) && ++failures <= 10) print(c, p);
    };
    // calls whose last block sees fewer tiles than the others, in lists that are cut right there
    const Call known[] = {
        {ILRE_BF16, 4, 4, {1, 4, 320}, {129, 129}, {600, 600}},
        {ILRE_BF16, 2, 2, {1, 4, 320}, {129, 129}, {1000, 1000}},
        {ILRE_F32, 8, 8, {1, 4, 512}, {150, 150}, {900, 900}},
        {ILRE_F32, 4, 4, {1, 4, 100}, {129, 129}, {600, 600}},
        {ILRE_BF16, 28, 4, {1, 4, 1024}, {940, 335, 659, 261}, {8132, 2261, 5504, 5724}},
        {ILRE_BF16, 32, 32, {1, 4, 1024}, {341, 513, 433, 520}, {3740, 4241, 3178, 1297}},
        {ILRE_BF16, 4, 4, {1, 4, 64}, {388, 79}, {2725, 2332}},
        {ILRE_F32, 12, 4, {1, 4, 512}, {392, 444}, {2019, 1118}},
    };
    for (const Call &c : known)
        check(c, plan_of(c, *std::max_element(c.q.begin(), c.q.end()), *std::max_element(c.kv.begin(), c.kv.end()), Call::sum(c.kv), 1.0));
    uint32_t x = 4711;
    auto below = [&](uint32_t n) {
        x = x * 1664525u + 1013904223u;
        return (int)((x >> 8) % n);
    };
    const int groups[10] = {1, 1, 2, 2, 3, 4, 5, 7, 8, 40}, heads[5] = {1, 2, 4, 8, 32};
    for (int round = 0; round < 60000; ++round) {
        Call c;
        c.dtype = below(2) ? ILRE_BF16 : ILRE_F32;
        c.Hkv = heads[below(5)], c.Hq = c.Hkv * groups[below(10)];
        c.m = Mask{1, 0, 0};
        if (below(4)) {
            c.m.window = below(3) ? 1 + below(1200) : 64 * (1 + below(16));
            c.m.sink = below(3) ? 4 : below(200);
        } else if (below(3) == 0) {
            c.m.causal = 0;
        }
        const int n = 1 + below(below(8) ? 5 : 40), most = below(3) ? 1100 : 90;
        const bool prompts = below(4) == 0;
        for (int s = 0; s < n; ++s) {
            const int q = below(12) ? 1 + below(most) : 0;
            c.q.push_back(q);
            c.kv.push_back(prompts ? q : below(20) ? q + below(below(3) ? 9000 : 400) : below(q + 1));
        }
        if (c.T() == 0) continue;
        const int max_q = *std::max_element(c.q.begin(), c.q.end()), max_kv = *std::max_element(c.kv.begin(), c.kv.end());
        if (below(5))
            check(c, plan_of(c, max_q, max_kv, Call::sum(c.kv), below(4) ? 1.0 : below(100) * 0.01));
        else  // promised lengths only decide how the work is cut up
            check(c, plan_of(c, below(2000), below(12000), below(30000), 1.0));
    }
    printf("%ld calls, %ld of them cut into ranges, %d failures\n", calls, cut, failures);
    return failures != 0;
}
