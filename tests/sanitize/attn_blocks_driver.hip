// Host driver for the attention kernels' arithmetic on rows, tokens, tiles and ranges (test infrastructure, no kernel and no GPU call): against the mask
// written out token by token, and what the kernels index the page table with.
#include <stdio.h>

#include "attn_blocks.h"

int main()
{
    using namespace ilre;
    int failures = 0;
    long cases = 0;
    uint32_t x = 12345;
    auto below = [&](uint32_t n) {
        x = x * 1664525u + 1013904223u;
        return (int)((x >> 8) % n);
    };
    const int tiles[3] = {32, 64, 128}, sizes[3] = {32, 128, 256}, groups[6] = {1, 2, 4, 5, 7, 8}, pages[4] = {4, 5, 6, 8};
    for (int round = 0; round < 6000; ++round) {
        const int G = groups[below(6)], rows = sizes[below(3)], tile = tiles[below(3)], shift = pages[below(4)];
        const int q_len = 1 + below(below(4) ? 40 : 400), kv = below(5) ? q_len + below(below(3) ? 300 : 2500) : below(q_len + 1);
        Mask m{below(4) ? 1 : 0, 0, 0};
        if (m.causal && below(2)) {
            m.window = 1 + below(below(2) ? 20 : 600);
            m.sink = below(2) ? below(200) : 0;
        }
        const int width = kv ? ((kv - 1) >> shift) + 1 : 1;
        for (int rows0 = 0; rows0 < q_len * G; rows0 += rows) {
            Block b{};
            b.rows0 = rows0, b.nrows = q_len * G, b.q_len = q_len, b.kv = kv;
            tiles_of(b, m, G, rows, tile);
            ++cases;
            bool bad = b.nt < 0 || b.hi < 0 || b.hi > kv || b.lo < 0 || b.lo > b.hi;
            // tiles ascend, none twice, all within the sequence
            int before = -1;
            for (int i = 0; i < b.nt; ++i) {
                const int t = tile_token(b, i, tile);
                bad = bad || t <= before || t % tile || t >= b.hi;
                before = t;
            }
            auto listed = [&](int t) {
                for (int i = 0; i < b.nt; ++i)
                    if (tile_token(b, i, tile) == t / tile * tile) return true;
                return false;
            };
            const int last_row = (rows0 + rows < b.nrows ? rows0 + rows : b.nrows) - 1;
            for (int t = 0; t < kv; t += 1 + below(3)) {
                bool some = false, all = true;
                for (int r = rows0; r <= last_row; r += G - r % G) {
                    const bool sees = row_sees(m, (int64_t)kv - q_len + r / G, kv, t);
                    some = some || sees;
                    all = all && sees;
                }
                const bool copied = t < b.hi && (t >= b.lo || t < b.sink);
                if (some && !(copied && listed(t))) bad = true;              // what a row sees is read
                if (t >= b.all_lo && t < b.all_hi && !all) bad = true;       // what is taken as seen by all is
                if (copied && !some && m.window == 0) bad = true;
            }
            // ranges of tiles: none empty, together the list, whatever their size
            for (int per = 1; per <= b.nt + 1; per += 1 + below(4)) {
                const int nsplit = 1 + below(40), n = ranges_of(b.nt, per, nsplit);
                int at = 0;
                for (int s = 0; s < n; ++s) {
                    const int first = s * per, count = (s == n - 1 ? b.nt : first + per) - first;
                    if (first != at || (count < 1 && b.nt)) bad = true;
                    at += count;
                }
                if (n < 1 || n > nsplit || at != b.nt) bad = true;
            }
            // what the wavefronts look up: the tokens of a tile and of the places behind the list, clamped to the block's last token
            for (int i = 0; i < b.nt + 5 && b.nt; ++i)
                for (int w = 0; w < tile + 16; w += 8) {
                    const int tok = i < b.nt ? tile_token(b, i, tile) + w : b.hi, t = tok < b.hi - 1 ? tok : b.hi - 1;
                    const int at = page_column(t, shift, width), loose = page_column(tok, shift, width);
                    if (at < 0 || at >= width || loose < 0 || loose >= width) bad = true;
                }
            if (bad && ++failures < 10)
                printf("G %d rows %d tile %d q %d kv %d causal %d sink %d window %d rows0 %d\n", G, rows, tile, q_len, kv, m.causal, m.sink, m.window, rows0);
        }
    }
    printf("%ld blocks, %d failures\n", cases, failures);
    return failures != 0;
}
