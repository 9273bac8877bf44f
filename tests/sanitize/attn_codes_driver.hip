// Host driver for the numbering of the attention kernels' units over quantised caches and under trees of drafted tokens (test infrastructure, no kernel and no GPU call): calls are cut up as the
// library cuts them, and every range that the merge adds up has to have been taken, once.
//
// With arguments "plan" it reads calls from stdin, a line each (format tree dtype T n_seq Hq Hkv max_q max_kv total_kv sink window beside), and prints the rows of a
// workgroup, the number of ranges and the kv heads of a workgroup.
#define main attn_units_main
#include "attn_units_driver.hip"
#undef main

static AttnPlan plan_of_format(const Call &c, int format, bool tree, bool beside, int max_q, int max_kv, int64_t total_kv, double share)
{
    // the workspace that a caller asks for: the largest that any kind of cache can make use of
    size_t bytes = 0;
    for (int f : {kPlain, (int)ILRE_KV_FP8, (int)ILRE_KV_FP4})
        for (bool b : {false, true})
            bytes = std::max(bytes, make_attn_plan(c.dtype, f, false, c.T(), (int)c.q.size(), c.Hq, c.Hkv, max_q, max_kv, total_kv, 0, 0, (size_t)1 << 62, b).bytes);
    return make_attn_plan(c.dtype, format, tree, c.T(), (int)c.q.size(), c.Hq, c.Hkv, max_q, max_kv, total_kv, c.m.sink, c.m.window, (size_t)(bytes * share), beside);
}

int main(int argc, char **argv)
{
    if (argc > 1 && !strcmp(argv[1], "plan")) {
        int format, tree, dtype, T, n, Hq, Hkv, max_q, max_kv, sink, window, beside;
        long total;
        while (scanf("%d %d %d %d %d %d %d %d %d %ld %d %d %d", &format, &tree, &dtype, &T, &n, &Hq, &Hkv, &max_q, &max_kv, &total, &sink, &window, &beside) == 13) {
            const AttnPlan p = make_attn_plan(dtype, format, tree != 0, T, n, Hq, Hkv, max_q, max_kv, total, sink, window, (size_t)1 << 62, beside != 0);
            printf("%d %d %d\n", p.rows, p.nsplit, p.heads);
        }
        return 0;
    }
    int failures = 0;
    long calls = 0, cut = 0, sixteen = 0, several = 0;
    uint32_t x = 815;
    auto below = [&](uint32_t n) {
        x = x * 1664525u + 1013904223u;
        return (int)((x >> 8) % n);
    };
    const int groups[10] = {1, 1, 2, 2, 3, 4, 5, 7, 8, 40}, heads[5] = {1, 2, 4, 8, 32};
    for (int round = 0; round < 40000; ++round) {
        Call c;
        c.dtype = below(4) ? ILRE_BF16 : ILRE_F32;
        c.Hkv = heads[below(5)], c.Hq = c.Hkv * groups[below(10)];
        const bool tree = below(3) == 0;
        const int format = below(3);  // the states' own type, 8 bits, 4 bits
        c.m = Mask{tree ? 0 : 1, 0, 0};
        if (!tree && below(2)) {
            c.m.window = below(3) ? 1 + below(1200) : 64 * (1 + below(16));
            c.m.sink = below(3) ? 4 : below(200);
        }
        const int n = 1 + below(below(8) ? 6 : 100), most = below(3) ? 4 : below(2) ? 40 : 1100;
        for (int s = 0; s < n; ++s) {
            const int q = below(12) ? 1 + below(most) : 0;
            c.q.push_back(q);
            c.kv.push_back(below(20) ? q + below(below(3) ? 20000 : 400) : below(q + 1));
        }
        if (c.T() == 0) continue;
        const int max_q = *std::max_element(c.q.begin(), c.q.end()), max_kv = *std::max_element(c.kv.begin(), c.kv.end());
        const double share = below(4) ? 1.0 : below(100) / 100.0;
        // what the caller says, or something else
        const bool honest = below(5) != 0, beside = format != kPlain && below(2);
        const AttnPlan p = plan_of_format(c, format, tree, beside, honest ? max_q : 1 + below(2 * max_q), honest ? max_kv : below(2 * max_kv + 1), below(3) ? Call::sum(c.kv) : 0, share);
        ++calls;
        cut += p.nsplit > 1;
        sixteen += p.rows == 16;
        several += p.heads > 1;
        if (c.Hkv % p.heads || p.tile * p.heads > 128 || (p.heads > 1 && (p.rows != 16 || tree || !beside || c.dtype != ILRE_BF16))) ++failures;
        if (faults(c, p) && ++failures <= 10) printf("format %d tree %d ", format, tree), print(c, p);
    }
    printf("%ld calls, %ld cut, %ld in blocks of 16 rows, %ld with several heads a workgroup, %d failures\n", calls, cut, sixteen, several, failures);
    if (several < 100) return 1;
    return failures != 0;
}
