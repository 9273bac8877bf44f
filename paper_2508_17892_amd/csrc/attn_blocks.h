// Which tokens the rows of an attention workgroup see, and the tiles they lie in: integers only, on their own so that they also run on the host.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ilre {

__host__ __device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// New token i of a sequence stands at p = kv - q_len + i and sees t < kv with t <= p (causal) and, with a window, t > p - window or t < sink.  A row is a new
// token and one of the G query heads of a kv head: row = i * G + head.
struct Mask {
    int causal, sink, window;
};

// The rows of one workgroup, and the tokens they see.
struct Block {
    int seq, rows0, nrows;  // rows0: first row within the sequence; nrows: rows of the sequence
    int q0, q_len;          // first new token in the packed order
    int kv, kv0;            // tokens in the sequence; first one in the packed order (contiguous keys)
    int lo, hi;             // tokens that some row of the block may see: [0, sink) and [lo, hi)
    int sink;               // of the sink part, what lies before lo
    int ns, w0, nt;         // tiles [0, ns) and [w0, w0 + nt - ns)
    int all_lo, all_hi;     // [all_lo, all_hi) is seen by every row of the block
};

// Fills in the tokens and tiles of `tile` tokens for rows rows0 .. rows0 + rows - 1 (as many as there are).  kv < 2^31 - 65536.
__host__ __device__ __forceinline__ void tiles_of(Block &b, const Mask &m, int G, int rows, int tile)
{
    auto lower = [](int64_t x, int64_t y) { return x < y ? x : y; };
    auto upper = [](int64_t x, int64_t y) { return x < y ? y : x; };
    const int first = b.rows0 / G, last = (int)(lower((int64_t)b.rows0 + rows, b.nrows) - 1) / G;
    const int64_t p0 = (int64_t)b.kv - b.q_len + first, p1 = (int64_t)b.kv - b.q_len + last;
    b.hi = m.causal ? (int)lower(upper(p1 + 1, 0), b.kv) : b.kv;
    b.all_hi = m.causal ? (int)lower(upper(p0 + 1, 0), b.kv) : b.kv;
    b.lo = b.all_lo = b.sink = 0;
    if (m.window > 0) {
        b.lo = (int)lower(upper(p0 - m.window + 1, 0), b.hi);
        b.all_lo = (int)upper(p1 - m.window + 1, 0);
        b.sink = (int)lower(m.sink, b.lo);
    }
    const int end = (b.hi + tile - 1) / tile;
    b.ns = (int)lower((b.sink + tile - 1) / tile, end);
    b.w0 = (int)upper(b.lo / tile, b.ns);
    b.nt = b.hi > 0 ? b.ns + (int)upper(end - b.w0, 0) : 0;
}

// First token of place i of a block's list of tiles.
__host__ __device__ __forceinline__ int tile_token(const Block &b, int i, int tile) { return (i < b.ns ? i : i - b.ns + b.w0) * tile; }

// Into how many ranges of per tiles a list of nt is cut, nsplit at most (the last one takes what is left): the same for the workgroups and the merge.
__host__ __device__ __forceinline__ int ranges_of(int nt, int per, int nsplit)
{
    const int n = nsplit == 1 || nt <= per ? 1 : (nt + per - 1) / per;
    return n < nsplit ? n : nsplit;
}

// A unit is a block of `rows` rows and one range of its tiles.  A sequence's units have consecutive numbers: its first ranges before its second ones and, within
// them, the last block first (with a causal mask it has most to do).
__host__ __device__ __forceinline__ int blocks_of(const Block &b, int rows) { return (b.nrows + rows - 1) / rows; }

// How many numbers a sequence (q_len, kv, nrows) has: at least one for each range of each block.  Without a window no block has more tiles than the last one.  With
// one, a block whose first and last rows are `apart` tokens apart sees window + apart tokens in a row, the last block window at the least (where a sequence is shorter
// than that it sees everything), and the two may lie otherwise over the tiles: (apart - 1) / tile, rounded up, + 1 tiles more.  Numbers that no range needs end at once.
__host__ __device__ __forceinline__ int units_of(Block b, const Mask &m, int G, int rows, int tile, int per, int nsplit)
{
    const int n = blocks_of(b, rows);
    if (nsplit == 1 || n == 0) return n;
    b.rows0 = (n - 1) * rows;
    tiles_of(b, m, G, rows, tile);
    const int apart = (rows + G - 2) / G;
    return n * ranges_of(m.window > 0 ? b.nt + (apart + tile - 2) / tile + 1 : b.nt, per, nsplit);
}

// The sequence's unit number `at`: fills in the block and its tiles, and says which range.  False where the block has no such range.
__host__ __device__ __forceinline__ bool take_unit(Block &b, int at, const Mask &m, int G, int rows, int tile, int per, int nsplit, int &split)
{
    const int n = blocks_of(b, rows);
    if (n == 0 || at < 0) return false;
    split = at / n;
    b.rows0 = (n - 1 - (at - split * n)) * rows;
    tiles_of(b, m, G, rows, tile);
    return split < ranges_of(b.nt, per, nsplit);
}

// The page table's column for token t: within the table whatever t >= 0 is.
__host__ __device__ __forceinline__ int page_column(int t, int page_shift, int table_width)
{
    const int at = t >> page_shift;
    return at < table_width ? at : table_width - 1;
}

// The same for a workgroup: tokens behind the last one that its rows see are looked up as that one, so that entries past a sequence's length are not read.
__host__ __device__ __forceinline__ int page_column(const Block &b, int t, int page_shift, int table_width)
{
    return page_column(t < b.hi ? t : b.hi - 1, page_shift, table_width);
}

// Whether a row at position p sees token t.
__host__ __device__ __forceinline__ bool row_sees(const Mask &m, int64_t p, int kv, int t)
{
    return t < kv && (!m.causal || t <= p) && (m.window == 0 || t > p - m.window || t < m.sink);
}

}  // namespace ilre
