// Attention over caches of the states' own element type and over packed prompts, and how a call of any kind is cut up.
#include "attend.h"

namespace ilre {

// Which kernel, and how the tokens are cut up.
//   - Up to 32 rows: attend_tokens.  More: 256 rows a workgroup, unless that leaves compute units without one and the lists are short, or there are 128 rows
//     at most: then 128 (1024 tokens of 32/8 heads, window 512: 128 workgroups of 256 rows, cut in two, 54 us with the merge; 256 of 128 rows 24 us; over
//     66560 tokens 256 rows cut in two take 1.02 ms, 128 rows 1.24 ms).
//   - A list is cut so that the ranges of all sequences together are one for each place that LDS has room for (twice as many: 48 requests 75 -> 78 us).
//     Up to three tiles of 128 tokens stay whole, as a merge costs more (four requests of 300 tokens 11.9 -> 9.3 us); more are cut down to single tiles while those
//     are one for each compute unit at most (four requests of 1000 tokens: 1 11.0 us, 2 12.8; one of 2000: 10.5 and 10.9), else into two at least (one of 4097: 12.1 and
//     11.7; 30000 tokens, 8/2 heads: 17.7 and 15.7).  More rows: 12 tiles of 64 tokens at least, and 4 while the merge has little to do (32/8 heads, 4096 tokens: 16
//     new ones 18.4 us with 4, 25.2 with 12, 64 29.7 and 35.7, 200 51.9 and 40.3), 2 of 32 in fp32 (prompts of 77 to 900 tokens, 8/2 heads: 2 55.7 us, 4 58.6,
//     6 74).
//   - fp32 states over a quantised cache: 16 rows a workgroup however many there are, as only that kernel splits them into parts for the bf16 matrix instructions (32/8 heads, 8 bits: one token over 131072
//     234 us with the fp32 instructions, 53 so; 8 over 30000 69 and 28, 100 over 9000 247 and 75, 1024 over 33000 5150 and 1740).
//   - Trees, and more than 16 rows over a quantised cache: a range leaves 32 rows behind for the merge, a quarter to half of what a tile of 128 tokens is. A range a compute unit, two from twelve tiles each
//     on, and whole where that is a merge's worth longer at most (8 drafted tokens, 32/8 heads: contexts of 4105, 9009, 7 and 300 26.1 -> 20.8 us, eight of 3000 28.3 -> 26.9, one of 30000 33.9 -> 31.7,
//     sixteen of 900 22.0 -> 19.8; in 8 bits 24.3 -> 18.8, 22.1 -> 20.4, 23.3 -> 21.7, 20.2 -> 16.8).
//   - Up to 16 rows over a quantised cache (tiles of 128 tokens): a workgroup a compute unit reads nearly as fast as HBM gives (32 requests of 1500 tokens, 8 kv heads 24.9 us whole, 25.5 in two),
//     so that lists stay whole where the longest has no more tiles than a compute unit's share of all and what a merge costs, four, or five at most (128 requests of 1000 tokens: whole 56 us, in two
//     63; one of 640: whole 9.4, single tiles 10.5; four of 1000: single tiles 10.7, whole 13.6). What is cut makes two ranges a compute unit (48 requests of 1 to 16384 tokens, 4 kv heads:
//     ranges of 12 tiles 47.0 us, 10 53.0, 7 50.3; 65536 tokens, 8 kv heads: 8 33.7, 6 36.3; 262144: 32 102.7, 22 106.8). No range is longer than what would stay whole: many lists make two ranges a
//     compute unit before the longest is cut, and one workgroup would walk it (32/8 heads, 8 bits: 128 requests of 1000 tokens but one of 1000003, in one range 11.0 ms, so 0.46; but one of 131072 1450
//     and 144 us; 28/4 heads, 512 of 30 to 30000 tokens 754 us either way, with half of that 503, which the former calls take for 494 and 166).
AttnPlan make_attn_plan(int dtype, int format, bool tree, int T, int n_seq, int Hq, int Hkv, int max_q, int max_kv, int64_t total_kv, int sink, int window, size_t workspace,
                        bool beside)
{
    AttnPlan p{};
    p.dtype = dtype;
    p.heads = 1;
    const int64_t G = Hq / Hkv, rows = (int64_t)max_q * G;
    if (total_kv <= 0) total_kv = (int64_t)n_seq * max_kv;
    auto cut = [&](int block, int tile) {
        p.rows = block;
        p.tile = tile;
        // at most so many blocks, whatever the sequences' lengths
        p.nblocks = (int)std::min(((int64_t)T * G + (int64_t)n_seq * (block - 1)) / block, (int64_t)T * G);
    };
    auto tiles = [&](int64_t kv) {
        const int64_t all = (kv + p.tile - 1) / p.tile;
        if (window <= 0) return all;
        return std::min(all, (std::min((int64_t)sink, kv) + p.tile - 1) / p.tile + (window + (p.rows + G - 1) / G) / p.tile + 2);
    };
    if (format != kPlain && (rows <= 16 || dtype == ILRE_F32)) {
        cut(16, 128);
        // Heads that lie side by side: a workgroup takes two or four of them, as 128 bytes here and there are read more slowly than what follows each other (one token, 8 kv heads, 8 bits: 131072
        // tokens 67 us with one, 61 with two, 60 with four, 524288 231, 203 and 190; 4 bits 524288 142, 137 and 128, 131072 44, 44 and 44).  Only there: not for 17 to 32 rows, trees and fp32 states, where nothing was measured.  It cuts sequences into more ranges: not where a
        // workgroup's share is short (8 bits, 16384 tokens 17.3, 18.0 and 20.9) or few lists are cut into very many ranges (131072 tokens of 4 kv heads 35.9, 37.5 and 38.3).
        const int64_t lists = std::min<int64_t>(p.nblocks, std::max<int64_t>((int64_t)T * G / p.rows, n_seq)) * Hkv, share = lists * tiles(total_kv / n_seq) / (2 * kNumCU);
        if (beside && dtype == ILRE_BF16 && !tree) p.heads = share >= 32 && Hkv % 4 == 0 && lists >= 8 ? 4 : format == ILRE_KV_FP8 && share >= 8 && Hkv % 2 == 0 && lists >= 8 ? 2 : 1;
        cut(16, 128 / p.heads);
    } else if (rows <= 32) {
        cut(32, 128);
    } else if (dtype == ILRE_F32) {
        cut(128, 32);
    } else {
        cut(256, 64);
        if (rows <= 128 || ((int64_t)p.nblocks * Hkv < kNumCU && tiles(max_kv) <= 24)) cut(128, 64);
    }
    p.one_block = rows <= p.rows;
    const int64_t most = std::max<int64_t>(tiles(max_kv), 1);
    const int64_t blocks = std::min<int64_t>(p.nblocks, std::max<int64_t>((int64_t)T * G / p.rows, n_seq));
    const int64_t work = std::max<int64_t>(blocks * (Hkv / p.heads) * tiles(total_kv / n_seq), 1);
    p.many_tiles = work >= 16 * kNumCU;
    const int64_t places = (p.rows == 32) == (dtype == ILRE_BF16) ? 2 * kNumCU : kNumCU;  // what LDS has room for
    const int64_t least = p.rows == 32 ? (most <= 3 ? 3 : work <= kNumCU ? 1 : 2) : dtype == ILRE_F32 ? 2 : (int64_t)T * Hq <= 2048 ? 4 : 12;
    int64_t per = std::max<int64_t>((work + places - 1) / places, least);
    if (p.rows == 32 && dtype == ILRE_BF16 && (format != kPlain || tree)) {
        per = work / (2 * kNumCU) >= 12 ? per : std::max<int64_t>((work + kNumCU - 1) / kNumCU, work <= kNumCU ? 1 : 2);
        if (most <= (work < kNumCU ? 3 : work / kNumCU + 4)) per = most;
    } else if (p.rows == 16) {
        const int64_t lists = blocks * (Hkv / p.heads), mean = tiles(total_kv / n_seq), whole = std::max<int64_t>(5, work / kNumCU + 4);
        per = most <= whole ? most : std::max<int64_t>(work <= kNumCU ? 1 : 2, work / (2 * kNumCU));
        if (per < most) {
            // the least that makes two ranges a compute unit at most: of lists of one length 2 kNumCU / lists each, of unlike ones lists (2 mean + per) / (2 per) together, as they end with half a range each
            int64_t enough = most;
            if (most == mean && lists <= 2 * kNumCU) enough = (most + 2 * kNumCU / lists - 1) / (2 * kNumCU / lists);
            if (most != mean && lists < 4 * kNumCU + 2) enough = 2 * mean * lists / (4 * kNumCU + 2 - lists) + 1;
            per = std::min({std::max(per, enough), most, whole});
        }
    }
    int64_t n = (most + per - 1) / per;
    const int64_t row_bytes = (int64_t)T * Hq * (kHeadDim + 1) * (int64_t)sizeof(float);
    n = std::max<int64_t>(1, std::min({n, (int64_t)256, (int64_t)(workspace / (size_t)row_bytes), kMaxUnits / std::max<int64_t>(p.nblocks * (int64_t)Hkv, 1)}));
    if ((int64_t)T * Hq > kMaxUnits) n = 1;  // (more rows than a merge is launched for)
    p.nsplit = (int)n;
    p.split_tiles = (int)(n == 1 ? most : std::max(per, (most + n - 1) / n));
    p.bytes = n == 1 ? 0 : (size_t)(n * row_bytes);
    return p;
}

hipError_t launch_attention(const AttnPlan &p, AttnArgs a, int format, void *workspace, hipStream_t s)
{
    a.nsplit = p.nsplit;
    a.split_tiles = p.split_tiles;
    a.nblocks = p.nblocks;
    a.rows = p.rows;
    a.tile = p.tile;
    a.part_o = (float *)workspace;
    a.part_e = a.part_o + (int64_t)p.nsplit * a.T * a.Hq * kHeadDim;
    if (format == ILRE_KV_FP8) return a.tree ? launch_attention_tree_fp8(p, a, s) : launch_attention_fp8(p, a, s);
    if (format == ILRE_KV_FP4) return a.tree ? launch_attention_tree_fp4(p, a, s) : launch_attention_fp4(p, a, s);
    if (a.tree) return launch_attention_tree(p, a, s);
    return a.table ? launch_kernels<true>(p, a, s) : launch_kernels<false>(p, a, s);
}

}  // namespace ilre
