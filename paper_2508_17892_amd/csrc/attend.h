// The kernels of attention over a cache of pages and over whole packed prompts, for gfx950, as templates: each file that includes this makes the ones it launches.
//
//   out[r] = sum_t p_rt V_t / sum_t p_rt,   p_rt = exp(q_r . K_t * scale - m_r),   log sum_t exp(q_r . K_t * scale)
//
// over the tokens t that row r sees: t < kv_len, t <= p (causal; p is the row's position in its sequence) and, with a window,
// t > p - window or t < sink.  A row is a new token and a query head; the rows of a kv head's G query heads are taken together
// (row = token * G + head of the group), so that a K tile that is in LDS serves all of them.
//
// Both products run with the tokens of the tile as matrix rows: S^T = K Q^T leaves lane l with the logits of query l % 32 and
// tokens 8 (i / 4) + 4 (l / 32) + i % 4, i = 0..15, so that the softmax of a row is that lane's (and its partner's, l ^ 32) own
// business, and the same registers, rounded to bf16 in pairs, are the right operand of O^T += V^T P^T: which token stands at
// which place of the contraction is free as long as both operands agree, and V^T is read from LDS with the transposing
// read (four tokens of one channel a lane) in that very order.  P never goes through LDS.
//
// Weights are taken relative to a reference m per row.  attend_rows takes it from the tiles before those that all of a workgroup's rows see whole, or from the
// first 32 tokens of these, and then keeps it: any m gives the same quotient as long as the exponentials stay in range, and the maximum, the rescaling and the branch in
// front of it are a fifth of the vector work.  A row whose later logits exceed its reference by more than 2^60 shows in its
// sum, and the workgroup walks its tiles again, following the maximum all the way.
//
// Measured (32/8 heads): a causal prompt of 16384 tokens 1.92 - 2.05 ms, 1.07 - 1.15 PFLOP/s (a large bf16 product of the library: 1.19 - 1.28), the matrix pipe
// busy for 57 % of the cycles and LDS without conflicts; without the kept references and the three-stage steps 2.85 ms.  One token over a million 0.68 ms,
// 6.0 TB/s of keys and values.
#pragma once

#include "attn_blocks.h"
#include "ilre_internal.h"
#include "kv_codes.h"

#include <math.h>

#include <algorithm>
#include <mutex>
#include <type_traits>

namespace ilre {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

namespace {

constexpr float kFloor = -1.0e30f;            // reference of a row that has seen nothing, in base-2 units
constexpr float kSumLimit = 1.152921504606847e18f;  // 2^60: a sum against a kept reference beyond this is made again
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }
// The larger of a lane's and its partner's, 32 lanes on (a swap of registers' halves, where __shfl_xor goes by way of LDS).
__device__ __forceinline__ float larger_of_halves(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ u32x4 lds_read16(unsigned at) { return *(const __attribute__((address_space(3))) u32x4 *)(size_t)at; }
__device__ __forceinline__ float lds_read4(unsigned at) { return *(const __attribute__((address_space(3))) float *)(size_t)at; }
// Four tokens of the lane's channel: the 16 lanes of a group point at 4 rows x 16 channels (8 bytes each), and each gets a column.
__device__ __forceinline__ u32x2 lds_read_tr(unsigned at)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(size_t)at));
}
// Table entries and lengths: not written while the kernel runs.  Where the address is the same for the whole wavefront they come through the scalar cache,
// outside the count of vector loads that the tile copies are waited for by.
__device__ __forceinline__ int read_i32(const int32_t *p) { return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p; }

__device__ __forceinline__ unsigned pack_bf16(float a, float b)  // nearest even
{
    return __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// ------------------------------------------------------------------------------------------------ which rows, which tiles

// All of a Block is the same for the whole wavefront.
__device__ __forceinline__ Mask mask_of(const AttnArgs &a) { return Mask{a.causal, a.sink, a.window}; }

template <bool PAGED>
__device__ __forceinline__ void sequence_of(const AttnArgs &a, int seq, Block &b)
{
    b.seq = seq;
    b.q0 = clamp_to(read_i32(a.cu_q + seq), 0, a.T);
    b.q_len = clamp_to(read_i32(a.cu_q + seq + 1), b.q0, a.T) - b.q0;
    if (PAGED) {
        b.kv0 = 0;
        b.kv = (int)min((int64_t)max(read_i32(a.kv_len + seq), 0), a.kv_limit);
    } else {
        b.kv0 = clamp_to(read_i32(a.cu_k + seq), 0, a.Tk);
        b.kv = clamp_to(read_i32(a.cu_k + seq + 1), b.kv0, a.Tk) - b.kv0;
    }
    b.nrows = b.q_len * a.G;
}

// Unit w of the call.  The units of all sequences come one after the other; what is left of the grid has none and ends at once, behind all that work (between
// them, 48 requests with contexts of 1 to 16384 tokens, it cost 10 of 85 us).  64 sequences a step: 256 requests of 512 tokens 47 us (5.7 TB/s), 1024 210 us (5.1),
// 4096 1.6 ms (2.7).  False where there is none.
template <bool PAGED>
__device__ __forceinline__ bool find_unit(const AttnArgs &a, int w, int rows, int tile, Block &b, int &split)
{
    int before = 0;
    if (a.n_seq == 1) {
        sequence_of<PAGED>(a, 0, b);
    } else {
        const int lane = threadIdx.x & 63;
        bool found = false;
        for (int base = 0; base < a.n_seq && !found; base += 64) {
            const int s = base + lane;
            Block x{};
            int n = 0;
            if (s < a.n_seq) {
                sequence_of<PAGED>(a, s, x);
                n = units_of(x, mask_of(a), a.G, rows, tile, a.split_tiles, a.nsplit);
            }
            int sum = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int y = __shfl_up(sum, o);
                if (lane >= o) sum += y;
            }
            const unsigned long long past = __ballot(before + sum > w);
            if (past) {
                const int at = __builtin_ctzll(past);
                auto of = [&](int y) { return __builtin_amdgcn_readlane(y, at); };
                b.seq = base + at;
                b.q0 = of(x.q0), b.q_len = of(x.q_len), b.kv = of(x.kv), b.kv0 = of(x.kv0), b.nrows = of(x.nrows);
                before += of(sum - n);
                found = true;
            } else {
                before += __builtin_amdgcn_readlane(sum, 63);
            }
        }
        if (!found) return false;
    }
    const int at = __builtin_amdgcn_readfirstlane(w - before);  // (negative where boundaries do not ascend)
    return take_unit(b, at, mask_of(a), a.G, rows, tile, a.split_tiles, a.nsplit, split);
}

// ------------------------------------------------------------------------------------------------ tile copies

// Where a kv head's keys (or values) lie, and the part of a tile that one wavefront copies: `rows` consecutive tokens, 16 at most and
// aligned, so that they are on one page.
struct Source {
    uint64_t base;
    int64_t page, token;  // bytes
};

// The number of a token's page (blk.hi > 0); -1 where the entry names no page (its tokens count as absent).
__device__ __forceinline__ int page_of(const AttnArgs &a, const Block &b, int tok)
{
    const int id = read_i32(a.table + (int64_t)b.seq * a.table_stride + page_column(b, tok, a.page_shift, a.table_width));
    return (unsigned)id < (unsigned)a.num_pages ? id : -1;
}

// One wavefront's share of a tile, from its first token `tok` on: ROWS rows of ROWB bytes to LDS address `to`, 16-byte chunk c of a row at place
// c ^ swizzle(row).  Rows that no row of the block sees (past hi, between sink and lo, on no page) are written as zeros: what lies there may
// be anything, and 0 * NaN is no 0.  Always the same number of copies, so that they can be waited for by count.
template <int ROWS, int ROWB, bool VALUES, bool PAGED, bool ONCE = false>
__device__ __forceinline__ void copy_rows(const AttnArgs &a, const Block &b, const Source &src, int tok, int page, unsigned to, const int (&voff)[ROWS * ROWB / 1024],
                                          int lane)
{
    constexpr int N = ROWS * ROWB / 1024, PER = 1024 / ROWB;
    uint64_t at;
    int n = clamp_to(b.hi - tok, 0, ROWS);
    if (PAGED) {
        at = src.base + (uint64_t)((int64_t)max(page, 0) * src.page + (int64_t)(tok & ((1 << a.page_shift) - 1)) * src.token);
        if (page < 0) n = 0;
    } else {
        at = src.base + (uint64_t)((int64_t)(n > 0 ? tok : 0) * src.token);
    }
    i32x4 rsrc;
    rsrc[0] = __builtin_amdgcn_readfirstlane((int)(unsigned)at);
    rsrc[1] = __builtin_amdgcn_readfirstlane((int)((unsigned)(at >> 32) & 0xFFFFu));
    rsrc[2] = __builtin_amdgcn_readfirstlane(n > 0 ? (int)((n - 1) * src.token) + ROWB : 0);
    rsrc[3] = 0x00020000;
    const bool gap = __builtin_amdgcn_readfirstlane(tok < b.lo && tok + ROWS > b.sink);
    if (!gap) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if constexpr (ONCE)
                lds_dma16_past(rsrc, __builtin_amdgcn_readfirstlane(to + j * 1024), voff[j]);
            else
                lds_dma16(rsrc, __builtin_amdgcn_readfirstlane(to + j * 1024), voff[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int t = tok + j * PER + lane / (64 / PER);
            lds_dma16(rsrc, __builtin_amdgcn_readfirstlane(to + j * 1024), t < b.lo && t >= b.sink ? -1 : voff[j]);
        }
    }
}

// Byte offsets, within the copied rows, of the chunks that this lane moves.
template <int ROWS, int ROWB, bool VALUES>
__device__ __forceinline__ void copy_offsets(int (&voff)[ROWS * ROWB / 1024], int first_row, int64_t token_bytes, int lane)
{
    constexpr int N = ROWS * ROWB / 1024, CPR = ROWB / 16, PER = 1024 / ROWB;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int row = j * PER + lane / CPR, place = lane % CPR, r = first_row + row;
        voff[j] = (int)(row * token_bytes) + (place ^ (VALUES ? (r & 3) << 2 : r & 15)) * 16;
    }
}

// ------------------------------------------------------------------------------------------------ tiles of a quantised cache

// Eight tokens of a kv head at a time: lane l has channels 16 (l % 8) .. + 15 of token l / 8, as codes in registers until they are written to LDS as bf16,
// where copy_rows would have put them.  Tokens that no row of the block sees are zeros here too (codes and scales past the end of a buffer read as zero).
template <int FMT>
struct Codes {
    static constexpr int W = FMT == ILRE_KV_FP8 ? 4 : 2;  // words of 16 channels
    unsigned w[W];
    unsigned char scale;
};

// Where a kv head's codes and scales of keys and values lie, and a lane's place in eight tokens of them.
template <int FMT>
struct QuantSource {
    const unsigned char *codes[2], *scales[2];
    unsigned token_bytes, token_scales, from, scale_from;
    __device__ __forceinline__ void init(const AttnArgs &a, int head, int lane)
    {
        const int64_t at = head * a.k_head;
        codes[0] = a.k + code_bytes<FMT>(at), codes[1] = a.v + code_bytes<FMT>(at);
        scales[0] = a.k_scales + at / ILRE_KV_BLOCK, scales[1] = a.v_scales + at / ILRE_KV_BLOCK;
        token_bytes = (unsigned)code_bytes<FMT>(a.k_token);
        token_scales = (unsigned)(a.k_token / ILRE_KV_BLOCK);
        from = (lane >> 3) * token_bytes + (lane & 7) * (unsigned)code_bytes<FMT>(16);
        scale_from = (lane >> 3) * token_scales + (lane & 7) / 2;
    }
};

// Keys and values of tokens tok .. tok + 7, which are on one page.
template <int FMT>
__device__ __forceinline__ void fetch_codes(const AttnArgs &a, const Block &b, const QuantSource<FMT> &src, int tok, int page, Codes<FMT> (&c)[2], int lane)
{
    const int n = page < 0 ? 0 : clamp_to(b.hi - tok, 0, 8);
    const int64_t at = (int64_t)max(page, 0) * a.k_page + (int64_t)(tok & ((1 << a.page_shift) - 1)) * a.k_token;
    const int codes_end = n > 0 ? (int)((n - 1) * src.token_bytes + code_bytes<FMT>(ILRE_HEAD_DIM)) : 0;
    const int scales_end = n > 0 ? (int)((n - 1) * src.token_scales + ILRE_HEAD_DIM / ILRE_KV_BLOCK) : 0;
    auto buffer = [](const unsigned char *p, int end) {
        const uint64_t u = (uint64_t)p;
        const uint64_t base = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)u);
        return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, __builtin_amdgcn_readfirstlane(end), 0x00020000);
    };
    unsigned from = src.from, scale_from = src.scale_from;
    if (__builtin_amdgcn_readfirstlane(tok < b.lo && tok + 8 > b.sink)) {
        const int t = tok + (lane >> 3);
        if (t < b.lo && t >= b.sink) from = scale_from = ~0u;
    }
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const __amdgpu_buffer_rsrc_t codes = buffer(src.codes[v] + code_bytes<FMT>(at), codes_end), scales = buffer(src.scales[v] + at / ILRE_KV_BLOCK, scales_end);
        if constexpr (FMT == ILRE_KV_FP8) {
            const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(codes, (int)from, 0, 0));
            c[v].w[0] = x[0], c[v].w[1] = x[1], c[v].w[2] = x[2], c[v].w[3] = x[3];
        } else {
            const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(codes, (int)from, 0, 0));
            c[v].w[0] = x[0], c[v].w[1] = x[1];
        }
        c[v].scale = __builtin_amdgcn_raw_buffer_load_b8(scales, (int)scale_from, 0, 0);
    }
}

__device__ __forceinline__ void lds_write16(unsigned at, const u32x4 &x) { *(__attribute__((address_space(3))) u32x4 *)(size_t)at = x; }

// Eight tokens to rows first_row .. of a tile in LDS (first_row a multiple of 8).  Eight lanes, the pieces of one row, write together: so that they reach all banks, a lane's 16-byte
// pieces go out in an order of its own, piece k ^ turn.
template <bool VALUES>
struct CodeRows {
    unsigned to[2];
    static __device__ __forceinline__ int turn(int lane) { return (lane & 7) >> 2; }
    __device__ __forceinline__ void init(unsigned tile, int first_row, int lane)
    {
        const int r = first_row + (lane >> 3), u = lane & 7, swap = VALUES ? (r & 3) << 2 : r & 15;
#pragma unroll
        for (int k = 0; k < 2; ++k) to[k] = tile + r * 256 + (((2 * u + (k ^ turn(lane))) ^ swap) * 16);
    }
};

// `slot`: the tile's distance from the one that CodeRows was made for.
template <int FMT, bool VALUES>
__device__ __forceinline__ void write_codes(const Codes<FMT> &c, const CodeRows<VALUES> &rows, unsigned slot, int lane)
{
    const float scale = scale_of(c.scale);
    const bool turn = rows.turn(lane);
    unsigned x[8];
    if constexpr (FMT == ILRE_KV_FP8) {
        const unsigned w[4] = {turn ? c.w[2] : c.w[0], turn ? c.w[3] : c.w[1], turn ? c.w[0] : c.w[2], turn ? c.w[1] : c.w[3]};
#pragma unroll
        for (int k = 0; k < 4; ++k) x[2 * k] = bf16_pair<FMT, 0>(w[k], scale), x[2 * k + 1] = bf16_pair<FMT, 1>(w[k], scale);
    } else {
        const unsigned w[2] = {turn ? c.w[1] : c.w[0], turn ? c.w[0] : c.w[1]};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            x[4 * k] = bf16_pair<FMT, 0>(w[k], scale), x[4 * k + 1] = bf16_pair<FMT, 1>(w[k], scale);
            x[4 * k + 2] = bf16_pair<FMT, 2>(w[k], scale), x[4 * k + 3] = bf16_pair<FMT, 3>(w[k], scale);
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) lds_write16(rows.to[k] + slot, u32x4{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]});
}

// ------------------------------------------------------------------------------------------------ products

// Two 16-bit halves, each kept where its bit (0, 1) is set.
__device__ __forceinline__ unsigned keep_halves(unsigned x, unsigned bits)
{
    return x & ((bits & 1 ? 0xFFFFu : 0u) | (bits & 2 ? 0xFFFF0000u : 0u));
}

template <int DT>
struct Elem;

template <>
struct Elem<ILRE_BF16> {
    static constexpr int ROWB = 256, QREGS = 8, RING = 4;  // QREGS: 16-byte pieces a lane holds of its query row
    struct Weights {
        u32x4 p[2];
    };
    static __device__ __forceinline__ void mma(f32x16 &acc, const u32x4 &x, const u32x4 &y)
    {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
    }
    // lane-dependent parts of the LDS addresses: chunk 2 st + half of key row l32; the value rows' column block
    struct Addr {
        unsigned k[8], v[4];
        __device__ __forceinline__ void init(int lane)
        {
            const int l32 = lane & 31, half = lane >> 5, l16 = lane & 15;
#pragma unroll
            for (int st = 0; st < 8; ++st) k[st] = l32 * ROWB + (((2 * st + half) ^ (l32 & 15)) * 16);
#pragma unroll
            for (int db = 0; db < 4; ++db)
                v[db] = (4 * half + (l16 >> 2)) * ROWB + ((db ^ (l16 >> 2)) * 64) + ((lane >> 4) & 1) * 32 + (l16 & 3) * 8;
        }
    };
    static __device__ __forceinline__ void logits(f32x16 &s, const u32x4 (&q)[QREGS], const Addr &ad, unsigned kat)
    {
        s = f32x16{};
#pragma unroll
        for (int st = 0; st < 8; ++st) mma(s, lds_read16(ad.k[st] + kat), q[st]);
    }
    // The weights are rounded to bf16 for the product with V, as the matrix instruction has one type for both operands; their sum is taken before.  Of the 2-norm that is 0.6e-3 to
    // 1.3e-3, beside 1.7e-3 from rounding the result; weights in two parts, upper and lower, would be half as many matrix instructions again.
    static __device__ __forceinline__ void pack(Weights &w, const float (&p)[16])
    {
        unsigned u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
        w.p[0] = u32x4{u[0], u[1], u[2], u[3]};
        w.p[1] = u32x4{u[4], u[5], u[6], u[7]};
    }
    static __device__ __forceinline__ void values(f32x16 (&o)[4], const Weights &w, const Addr &ad, unsigned vat)
    {
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const u32x2 x = lds_read_tr(ad.v[db] + vat + ks * 16 * ROWB), y = lds_read_tr(ad.v[db] + vat + (ks * 16 + 8) * ROWB);
                mma(o[db], u32x4{x[0], x[1], y[0], y[1]}, w.p[ks]);
            }
    }
    // The same with zeros for the values of tokens whose bit in `keep` is not set.
    static __device__ __forceinline__ void values(f32x16 (&o)[4], const Weights &w, const Addr &ad, unsigned vat, unsigned keep, int half)
    {
        keep >>= 4 * half;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const u32x2 x = lds_read_tr(ad.v[db] + vat + ks * 16 * ROWB), y = lds_read_tr(ad.v[db] + vat + (ks * 16 + 8) * ROWB);
                const unsigned b = keep >> (16 * ks);
                mma(o[db], u32x4{keep_halves(x[0], b), keep_halves(x[1], b >> 2), keep_halves(y[0], b >> 8), keep_halves(y[1], b >> 10)}, w.p[ks]);
            }
    }
};

// fp32 states: the fp32 matrix instructions (a sixteenth of the bf16 rate), nothing is rounded on the way.
template <>
struct Elem<ILRE_F32> {
    static constexpr int ROWB = 512, QREGS = 16, RING = 2;
    struct Weights {
        float p[16];
    };
    struct Addr {
        unsigned k[16], v[4];
        __device__ __forceinline__ void init(int lane)
        {
            const int l32 = lane & 31, half = lane >> 5;
#pragma unroll
            for (int st = 0; st < 16; ++st) k[st] = l32 * ROWB + (((2 * st + half) ^ (l32 & 15)) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = 4 * half * ROWB + j * ROWB + (((l32 >> 2) ^ ((j & 1) << 2)) * 16) + (l32 & 3) * 4;
        }
    };
    static __device__ __forceinline__ void logits(f32x16 &s, const u32x4 (&q)[QREGS], const Addr &ad, unsigned kat)
    {
        s = f32x16{};
#pragma unroll
        for (int st = 0; st < 16; ++st) {
            const u32x4 k = lds_read16(ad.k[st] + kat), x = q[st];
#pragma unroll
            for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[e]), __uint_as_float(x[e]), s, 0, 0, 0);
        }
    }
    static __device__ __forceinline__ void pack(Weights &w, const float (&p)[16])
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) w.p[i] = p[i];
    }
    static __device__ __forceinline__ void values(f32x16 (&o)[4], const Weights &w, const Addr &ad, unsigned vat)
    {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                // chunk (8 db + l32 / 4) ^ (i % 4 << 2): the upper bit of the XOR picks another channel block
                const float v = lds_read4(ad.v[i & 3] + vat + (i >> 2) * 8 * ROWB + (db ^ ((i & 3) >> 1)) * 128);
                o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, w.p[i], o[db], 0, 0, 0);
            }
    }
    static __device__ __forceinline__ void values(f32x16 (&o)[4], const Weights &w, const Addr &ad, unsigned vat, unsigned keep, int half)
    {
        keep >>= 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const float v = lds_read4(ad.v[i & 3] + vat + (i >> 2) * 8 * ROWB + (db ^ ((i & 3) >> 1)) * 128);
                o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(keep >> (8 * (i >> 2) + (i & 3)) & 1 ? v : 0.f, w.p[i], o[db], 0, 0, 0);
            }
    }
};

// A word with the lowest n bits set, all for n >= 32, none for n <= 0.
__device__ __forceinline__ unsigned first_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1; }

// A wavefront's running state for 32 rows; a lane and its partner 32 lanes on have row l32, the tokens of each 32 between them.
template <int DT>
struct State {
    using E = Elem<DT>;
    u32x4 q[E::QREGS];
    f32x16 o[4];
    float m, z[4];
    int lo, hi;  // the row sees [0, sink) and [lo, hi)
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int db = 0; db < 4; ++db) o[db] = f32x16{};
        m = kFloor;
        z[0] = z[1] = z[2] = z[3] = 0.f;
    }
    // Query row row0 + l32 of the sequence; past the last one zeros, which see what the last one sees and are written nowhere.
    // HALVES: a lane has the row's first or second 64 channels; otherwise every second 16 bytes.
    template <bool HALVES = false>
    __device__ __forceinline__ void load(const AttnArgs &a, const Block &blk, int head_kv, int row0, int l32, int half)
    {
        const int want = row0 + l32, r = min(want, blk.nrows - 1);
        const int i = r / a.G, g = r - i * a.G;
        const unsigned char *src = a.q + (int64_t)(blk.q0 + i) * a.q_token + (int64_t)(head_kv * a.G + g) * a.q_head + half * (HALVES ? E::QREGS * 16 : 16);
#pragma unroll
        for (int st = 0; st < E::QREGS; ++st) q[st] = *(const u32x4 *)(src + st * (HALVES ? 16 : 32));
        // waited for here, not in the loop over tiles, where that would be a wait for the tile copies as well
#pragma unroll
        for (int st = 0; st < E::QREGS; ++st) asm volatile("" : "+v"(q[st]));
        if (want != r) {
#pragma unroll
            for (int st = 0; st < E::QREGS; ++st) q[st] = u32x4{};
        }
        const int p = max(blk.kv - blk.q_len + i, -1);  // a row in front of its sequence sees nothing
        hi = a.causal ? min(p + 1, blk.kv) : blk.kv;
        lo = a.window > 0 ? max(p - a.window + 1, 0) : 0;
    }
    // Logits of tokens that the row does not see become -inf: 32 tokens from `at` on; bit 0 / 1 of `absent`: the first / last 16 are on no page.  What the row
    // sees is a word of bits, a few instructions a logit: nearly every tile that comes here has an edge in it.
    __device__ __forceinline__ void hide(f32x16 &s, int at, int sink, int half, int absent, unsigned drafted = ~0u) const
    {
        unsigned bits = first_bits(hi - at) & (~first_bits(lo - at) | first_bits(sink - at)) & drafted;
        bits &= ~((absent & 1 ? 0xFFFFu : 0u) | (absent & 2 ? 0xFFFF0000u : 0u));
        bits >>= 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int seen = (int)(bits << (31 - (8 * (i >> 2) + (i & 3)))) >> 31;
            s[i] = __int_as_float((__float_as_int(s[i]) & seen) | (__float_as_int(-INFINITY) & ~seen));
        }
    }
    __device__ __forceinline__ float largest(const f32x16 &s) const
    {
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        return top;
    }
    // A reference for the rows that have none, from the logits of 32 tokens that all rows see.  (What they have summed up so far is zero.)
    __device__ __forceinline__ void refer(const f32x16 &s, float c)
    {
        if (!__ballot(m == kFloor)) return;
        float top = largest(s);
        top = fmaxf(fmaxf(top, other_half(top)) * c, kFloor);
        m = m == kFloor ? top : m;
    }
    // The logits of SUB x 32 tokens become weights; the running maximum is followed.
    template <int SUB, bool SWAP = false>
    __device__ __forceinline__ void weigh(const f32x16 (&s)[SUB], typename E::Weights (&w)[SUB], float c)
    {
        float top = largest(s[0]);
#pragma unroll
        for (int u = 1; u < SUB; ++u) top = fmaxf(top, largest(s[u]));
        top = SWAP ? larger_of_halves(top) : fmaxf(top, other_half(top));
        const float mnew = fmaxf(m, top * c);
        if (__ballot(mnew != m)) {
            const float f = exp2_fast(m - mnew);
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[db][i] *= f;
#pragma unroll
            for (int k = 0; k < 4; ++k) z[k] *= f;
            m = mnew;
        }
#pragma unroll
        for (int u = 0; u < SUB; ++u) weigh_kept(s[u], w[u], c);
    }
    // The same against the reference as it is.
    __device__ __forceinline__ void weigh_kept(const f32x16 &s, typename E::Weights &w, float c)
    {
        float p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = exp2_fast(fmaf(s[i], c, -m));
            z[i & 3] += p[i];
        }
        E::pack(w, p);
    }
    __device__ __forceinline__ float sum() const
    {
        const float x = (z[0] + z[1]) + (z[2] + z[3]);
        return x + other_half(x);
    }
};

// The bits that some lane has.
__device__ __forceinline__ unsigned of_any_lane(unsigned x)
{
    auto from = [](auto ctrl, unsigned y) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)y, ctrl.value, 0xF, 0xF, true); };
    x |= from(std::integral_constant<int, 0xB1>{}, x);   // quad permutation 1 0 3 2
    x |= from(std::integral_constant<int, 0x4E>{}, x);   // 2 3 0 1
    x |= from(std::integral_constant<int, 0x141>{}, x);  // half rows mirrored
    x |= from(std::integral_constant<int, 0x140>{}, x);  // rows of 16 mirrored
    return (unsigned)(__builtin_amdgcn_readlane((int)x, 0) | __builtin_amdgcn_readlane((int)x, 16) | __builtin_amdgcn_readlane((int)x, 32) | __builtin_amdgcn_readlane((int)x, 48));
}

// What a row sees of a tree of drafted tokens, which are the tokens from `base` on (it may lie in front of the sequence).  A drafted token that no row of the wavefront sees may hold
// anything, and stands in the middle of others that are seen: its values are made zeros, as a weight of zero times a NaN is a NaN (attend_rows, whose wavefronts share tiles: on the way from LDS to the
// matrix instruction; the others: in LDS).
struct Drafted {
    const uint32_t *words;
    int base, n;
    __device__ __forceinline__ void init(const AttnArgs &a, const Block &blk, int want)
    {
        base = blk.kv - blk.q_len;
        n = a.tree_words;
        words = a.tree + (int64_t)(blk.q0 + min(want, blk.nrows - 1) / a.G) * a.tree_stride;
    }
    // The bits of 32 tokens from `at` on, all set in front of the drafted ones.
    __device__ __forceinline__ unsigned bits(int at) const
    {
        const int j = at - base;
        if (j <= -32) return ~0u;
        if (j < 0) return first_bits(-j) | words[0] << -j;
        const int w = j >> 5;
        const unsigned lo = w < n ? words[w] : 0, hi = w + 1 < n ? words[w + 1] : 0;
        return (unsigned)(((unsigned long long)hi << 32 | lo) >> (j & 31));
    }
};

// Zeros for those of a wavefront's 32 rows of values in LDS whose bit is not set.
template <int ROWB>
__device__ __forceinline__ void keep_rows(unsigned tile, unsigned keep, int lane)
{
    for (unsigned gone = ~keep; gone; gone &= gone - 1) {
        const unsigned row = tile + (unsigned)__builtin_ctz(gone) * ROWB;
#pragma unroll
        for (int at = 0; at < ROWB; at += 256) *(__attribute__((address_space(3))) unsigned *)(size_t)(row + at + lane * 4) = 0;
    }
    __builtin_amdgcn_wave_barrier();
}

// Where a row's results go: where all of its tokens were in this workgroup's range, out and the logarithm of the sum; otherwise the quotient in
// fp32 and the base-2 logarithm for the merge.
struct Target {
    bool real, direct;
    int64_t row;          // token * Hq + head (in the range's part of the partial results)
    unsigned char *out;
    float f, e;           // 1 / sum, log2 of the sum of 2^logit
};

__device__ __forceinline__ Target target_of(const AttnArgs &a, const Block &blk, int head_kv, int want, bool direct, int split, float m, float sum)
{
    Target t;
    t.real = want < blk.nrows;
    t.direct = direct;
    const int r = t.real ? want : 0, i = r / a.G, g = r - i * a.G;
    const int token = blk.q0 + i, head = head_kv * a.G + g;
    t.row = ((int64_t)(direct ? 0 : split) * a.T + token) * a.Hq + head;
    t.out = a.out + (int64_t)token * a.out_token + (int64_t)head * a.out_head;
    t.f = sum == 0.f ? 0.f : 1.f / sum;
    t.e = sum == 0.f ? -INFINITY : m + __log2f(sum);
    return t;
}

// x holds channels 32 db + 8 (i / 4) + 4 half + i % 4.
template <int DT>
__device__ __forceinline__ void store_channels(const AttnArgs &a, const Target &t, int db, const f32x16 &x, int half)
{
    float y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = x[i] * t.f;
    if (!t.direct || DT == ILRE_F32) {
        float *to = t.direct ? (float *)t.out : a.part_o + t.row * kHeadDim;
        if (t.real) {
#pragma unroll
            for (int k = 0; k < 4; ++k) *(float4 *)(to + db * 32 + 8 * k + 4 * half) = make_float4(y[4 * k], y[4 * k + 1], y[4 * k + 2], y[4 * k + 3]);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 16; k += 8) {
        // the halves hold 4 channels each of two groups of 8: after the swap each has one group whole
        const u32x2 u = __builtin_amdgcn_permlane32_swap(pack_bf16(y[k], y[k + 1]), pack_bf16(y[k + 4], y[k + 5]), false, false);
        const u32x2 v = __builtin_amdgcn_permlane32_swap(pack_bf16(y[k + 2], y[k + 3]), pack_bf16(y[k + 6], y[k + 7]), false, false);
        if (t.real) *(uint4 *)(t.out + (db * 32 + 2 * k + 8 * half) * 2) = make_uint4(u[0], v[0], u[1], v[1]);
    }
}

__device__ __forceinline__ void store_sum(const AttnArgs &a, const Target &t, int half)
{
    if (!t.real || half != 0) return;
    if (!t.direct)
        a.part_e[t.row] = t.e;
    else if (a.lse)
        a.lse[t.row] = t.e * kLn2;
}

// ------------------------------------------------------------------------------------------------ many rows

// WAVES / TS groups of 32 rows share the tiles of TN tokens; with TS = 2 two wavefronts have the same rows and a half of each tile's tokens, and add up what
// they have at the end.  Keys and values have four tile buffers each; while tile i is worked on, its values, the keys of tile i + 1 and (in the pipelined
// loop) the values of tile i - 1 are in use, and the copies of keys i + 2, i + 3 and values i + 1, i + 2 under way.  fp32 tiles have two buffers
// each, so that two workgroups of four wavefronts fit a compute unit: with one wavefront a SIMD every wait for LDS is a hole between matrix instructions.
//
// Of a quantised cache (FMT) the codes of tile i + 2 are on their way to registers while tile i is worked on; before, those of tile i + 1 have been converted and written to LDS.  Bound as without:
// 1024 tokens over 66560 (32/8 heads) 1.00 - 1.06 ms in 8 bits, 0.98 - 1.00 in 4, 0.99 - 1.06 in 16.
template <int DT, int WAVES, int TS, int TN, bool PAGED, int FMT = kPlain, bool TREE = false>
__global__ __launch_bounds__(WAVES * 64, 2) void attend_rows(const AttnArgs a)
{
    using E = Elem<DT>;
    constexpr int ROWB = E::ROWB, SLOT = TN * ROWB, GROUPS = WAVES / TS, ROWS = GROUPS * 32, SUB = TN / 32 / TS, RING = E::RING;
    constexpr int CROWS = TN / WAVES, COPIES = CROWS * ROWB / 1024;  // a wavefront's rows and copies of a tile
    static_assert(CROWS <= 16 && CROWS * ROWB % 1024 == 0 && TN % 32 == 0, "a wavefront's rows lie on one page");
    static_assert(FMT == kPlain || (PAGED && DT == ILRE_BF16 && CROWS == 8), "a wavefront has eight rows of codes of a tile");
    extern __shared__ __align__(16) unsigned char smem[];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    // kv heads run fastest: workgroups that share keys and values are a multiple of Hkv apart, on one XCD where Hkv is a multiple of 8
    const int head = blockIdx.x % a.Hkv;
    Block blk;
    int split;
    if (!find_unit<PAGED>(a, blockIdx.x / a.Hkv, ROWS, TN, blk, split)) return;
    if (TREE) blk.all_hi = max(blk.kv - blk.q_len, 0);
    const int nsp = ranges_of(blk.nt, a.split_tiles, a.nsplit);
    const int first = split * a.split_tiles, count = (split == nsp - 1 ? blk.nt : first + a.split_tiles) - first;
    auto token_of = [&](int i) { return tile_token(blk, first + i, TN); };

    State<DT> st;
    const int row0 = blk.rows0 + wave % GROUPS * 32, part = wave / GROUPS * SUB * 32;  // its rows, and where its part of a tile begins
    const bool idle = row0 >= blk.nrows;
    Drafted drafted;
    if (TREE) drafted.init(a, blk, row0 + l32);

    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)smem;
    typename E::Addr ad;
    ad.init(lane);
    // Set where a kept reference turns out too low, or an entry of the table names no page: then the tiles are walked again, with care.
    int *flag = (int *)(smem + 2 * RING * SLOT);
    if (tid == 0) *flag = 0;
    __syncthreads();

    Source ks, vs;
    ks.base = (uint64_t)a.k + (uint64_t)((int64_t)head * a.k_head + (int64_t)blk.kv0 * a.k_token);
    vs.base = (uint64_t)a.v + (uint64_t)((int64_t)head * a.v_head + (int64_t)blk.kv0 * a.v_token);
    ks.page = a.k_page, vs.page = a.v_page, ks.token = a.k_token, vs.token = a.v_token;
    int kvoff[COPIES], vvoff[COPIES];
    copy_offsets<CROWS, ROWB, false>(kvoff, wave * CROWS, a.k_token, lane);
    copy_offsets<CROWS, ROWB, true>(vvoff, wave * CROWS, a.v_token, lane);
    auto own_token = [&](int i) { return i < count ? token_of(i) + wave * CROWS : blk.hi; };
    // of a quantised cache: where the head lies, and the codes that are on their way
    constexpr int QF = FMT == kPlain ? ILRE_KV_FP8 : FMT;
    QuantSource<QF> quant;
    CodeRows<false> key_rows;
    CodeRows<true> value_rows;
    if (FMT != kPlain) {
        quant.init(a, head, lane);
        key_rows.init(lds0, wave * CROWS, lane);
        value_rows.init(lds0 + RING * SLOT, wave * CROWS, lane);
    }
    Codes<QF> codes[2];  // of keys and values
    auto fetch = [&](int i, int page) { fetch_codes<QF>(a, blk, quant, own_token(i), page, codes, lane); };
    auto write = [&](int i) {
        write_codes<QF, false>(codes[0], key_rows, i % RING * SLOT, lane);
        write_codes<QF, true>(codes[1], value_rows, i % RING * SLOT, lane);
    };
    int pages[2];  // of this wavefront's rows: of the last tile whose keys were asked for, and the next one
    auto lookup = [&](int i) {
        if (!PAGED) return 0;
        const int t = min(own_token(i), blk.hi - 1), page = page_of(a, blk, t);
        if (page < 0 && (t + CROWS > blk.lo || t < blk.sink)) *flag = 1;
        return page;
    };
    auto copy_keys = [&](int i, int page) {
        copy_rows<CROWS, ROWB, false, PAGED>(a, blk, ks, own_token(i), page, lds0 + i % RING * SLOT + wave * CROWS * ROWB, kvoff, lane);
    };
    auto copy_values = [&](int i, int page) {
        copy_rows<CROWS, ROWB, true, PAGED>(a, blk, vs, own_token(i), page, lds0 + (RING + i % RING) * SLOT + wave * CROWS * ROWB, vvoff, lane);
    };
    auto begin = [&]() {
        if constexpr (FMT != kPlain) {
            const int p0 = lookup(0), p1 = lookup(1);
            fetch(0, p0);
            write(0);
            fetch(1, p1);
            pages[0] = lookup(2);
            return;
        }
        if (RING == 2) {
            const int p = lookup(0);
            copy_keys(0, p);
            copy_values(0, p);
            pages[0] = lookup(1);
            return;
        }
        const int p0 = lookup(0), p1 = lookup(1), p2 = lookup(2);
        copy_keys(0, p0);
        copy_keys(1, p1);
        copy_values(0, p0);
        copy_keys(2, p2);
        copy_values(1, p1);
        pages[0] = p2;
        pages[1] = lookup(3);
    };
    // Tile i's values and tile i + 1's keys (two buffers: tile i's) are there, everybody is done with tile i - 1, and the next copies are on their way.
    auto advance = [&](int i) {
        if constexpr (FMT != kPlain) {
            write(i + 1);
            fetch(i + 2, pages[0]);
            pages[0] = lookup(i + 3);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            return;
        }
        if (RING == 2) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            copy_keys(i + 1, pages[0]);
            copy_values(i + 1, pages[0]);
            pages[0] = lookup(i + 2);
            return;
        }
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * COPIES) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        copy_keys(i + 3, pages[1]);
        copy_values(i + 2, pages[0]);
        pages[0] = pages[1];
        pages[1] = lookup(i + 4);
    };
    auto keys_at = [&](int i, int sub) { return lds0 + i % RING * SLOT + (part + sub * 32) * ROWB; };
    auto values_at = [&](int i, int sub) { return lds0 + (RING + i % RING) * SLOT + (part + sub * 32) * ROWB; };
    // A tile that some rows see a part of, following the maximum or (kept) against the references as they are.
    auto edge_tile = [&](int i, bool careful, auto kept) {
        advance(i);
        if (idle) return;
        const int tok = token_of(i) + part;
        f32x16 s[SUB];
        typename E::Weights w[SUB];
        unsigned seen[SUB];
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) E::logits(s[sub], st.q, ad, keys_at(i, sub));
        int absent = 0;
        if (PAGED && careful) {
            for (int k = 0; k < SUB * 2; ++k) absent |= (page_of(a, blk, tok + 16 * k) < 0 ? 1 : 0) << k;
        }
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
            seen[sub] = TREE ? drafted.bits(tok + 32 * sub) : ~0u;
            st.hide(s[sub], tok + 32 * sub, a.sink, half, absent >> (2 * sub), seen[sub]);
        }
        if (kept.value) {
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) st.weigh_kept(s[sub], w[sub], a.c);
        } else {
            st.template weigh<SUB>(s, w, a.c);
        }
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) {
            if constexpr (TREE)
                E::values(st.o, w[sub], ad, values_at(i, sub), of_any_lane(seen[sub]), half);
            else
                E::values(st.o, w[sub], ad, values_at(i, sub));
        }
    };

    // Tiles g1 .. g2 - 1, which all rows see whole, against the references that the tiles before have left.  32 tokens are a step, and a step holds three
    // stages that do not wait for each other: the logits of the next 32 tokens, these ones' weights, the product of the weights before with their values.
    auto kept_step = [&](f32x16 &now, f32x16 &next, typename E::Weights &w, unsigned kat, unsigned vat) {
        typename E::Weights wn;
        E::logits(next, st.q, ad, kat);
        E::values(st.o, w, ad, vat);
        st.weigh_kept(now, wn, a.c);
        w = wn;
        if (DT == ILRE_BF16) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction, two LDS reads, an exponential, three other vector instructions
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
            }
        }
    };
    auto kept_tiles = [&](int g1, int g2) {
        if (idle) {
            for (int i = g1; i < g2; ++i) advance(i);
            return;
        }
        f32x16 s[2];
        typename E::Weights w;
        E::logits(s[0], st.q, ad, keys_at(g1, 0));
        st.refer(s[0], a.c);
        advance(g1);
        // the first step has no weights before it
        if (SUB == 2) {
            E::logits(s[1], st.q, ad, keys_at(g1, 1));
            st.weigh_kept(s[0], w, a.c);
            kept_step(s[1], s[0], w, keys_at(g1 + 1, 0), values_at(g1, 0));
            for (int i = g1 + 1; i < g2; ++i) {
                advance(i);
                kept_step(s[0], s[1], w, keys_at(i, 1), values_at(i - 1, 1));
                kept_step(s[1], s[0], w, keys_at(i + 1, 0), values_at(i, 0));
            }
        } else {
            E::logits(s[1], st.q, ad, keys_at(g1 + 1, 0));
            st.weigh_kept(s[0], w, a.c);
            int i = g1 + 1;
            for (; i + 1 < g2; i += 2) {
                advance(i);
                kept_step(s[1], s[0], w, keys_at(i + 1, 0), values_at(i - 1, 0));
                advance(i + 1);
                kept_step(s[0], s[1], w, keys_at(i + 2, 0), values_at(i, 0));
            }
            if (i < g2) {
                advance(i);
                kept_step(s[1], s[0], w, keys_at(i + 1, 0), values_at(i - 1, 0));
            }
        }
        E::values(st.o, w, ad, values_at(g2 - 1, SUB - 1));
    };

    // g1 .. g2 - 1: the tiles that all rows see whole and whose weights are taken against references that stay.  A row has its reference from the tiles before: the
    // sink part or one such tile that is followed; where they hold nothing that it sees (the range begins here, or its wavefront has the half of the sink tile
    // behind the sink part and the window begins with this tile), from the first 32 tokens here.  Without that last one every second workgroup of 1024 new tokens
    // over 9216 (32/8 heads, window 512) walked its tiles twice: 39 us, over 9220 24.
    int g1 = count, g2 = count;
    if (DT == ILRE_BF16) {
        const int from = a.window > 0 ? max((blk.all_lo + TN - 1) / TN, blk.w0) - blk.w0 + blk.ns : 0;
        const int to = a.window > 0 ? blk.all_hi / TN - blk.w0 + blk.ns : blk.all_hi / TN;
        g1 = max(from - first, 0);
        if (g1 > 0 && (first > 0 || blk.ns == 0)) ++g1;
        g2 = min(to - first, count);
        if (g2 <= g1) g1 = g2 = count;
    }
    if (count > 0) begin();
    st.load(a, blk, head, row0, l32, half);  // behind the copies: they are on their way together
    st.clear();
    if (count > 0) {
        for (int i = 0; i < g1; ++i) edge_tile(i, false, std::false_type{});
        if (g1 < g2) {
            if (g1 == 0) {  // nobody has waited for the first keys yet (other than along with the queries)
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
            }
            kept_tiles(g1, g2);
        }
        for (int i = g2; i < count; ++i) edge_tile(i, false, std::true_type{});
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (PAGED || g1 < g2) {
            bool far = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) far = far || !(st.z[k] <= kSumLimit);
            if (!idle && far && g1 < g2) *flag = 1;
            __syncthreads();
            if (__builtin_amdgcn_readfirstlane(*flag)) {
                st.clear();
                begin();
                for (int i = 0; i < count; ++i) edge_tile(i, PAGED, std::false_type{});
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
        }
    }
    float m = st.m, sum = st.sum();
    if (TS == 2) {
        // Each of the two keeps two of the four channel blocks and hands the other two to its partner, 16-byte pieces of row l32 at place piece ^ l32 % 16.
        static_assert(TS == 1 || WAVES * 32 * 256 <= 2 * RING * SLOT, "half the sums of every wavefront fit where the tiles were");
        __syncthreads();  // everybody is done with the tiles
        const int mine = wave / GROUPS;
        auto piece = [&](int w, int at) { return (f32x4 *)(smem + w * 32 * 256 + l32 * 256 + (at ^ (l32 & 15)) * 16); };
        float2 *stats = (float2 *)(smem + 2 * RING * SLOT + 16);  // [WAVES][32]
        const int other = wave < GROUPS ? wave + GROUPS : wave - GROUPS;
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x16 &x = mine == 0 ? st.o[2 + d] : st.o[d];
                *piece(wave, d * 8 + 2 * k + half) = f32x4{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]};
            }
        if (half == 0) stats[wave * 32 + l32] = make_float2(m, sum);
        __syncthreads();
        if (idle) return;
        const float2 theirs = stats[other * 32 + l32];
        const float top = fmaxf(m, theirs.x), f = exp2_fast(m - top), g = exp2_fast(theirs.x - top);
        // the same order on both sides: the first half's sum and then the second's
        sum = mine == 0 ? fmaf(theirs.y, g, sum * f) : fmaf(sum, f, theirs.y * g);
        m = top;
        const Target t = target_of(a, blk, head, row0 + l32, nsp == 1, split, m, sum);
#pragma unroll
        for (int d = 0; d < 2; ++d) {
            f32x16 x = mine == 0 ? st.o[d] : st.o[2 + d];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x4 y = *piece(other, d * 8 + 2 * k + half);
                x[4 * k] = fmaf(x[4 * k], f, y.x * g);
                x[4 * k + 1] = fmaf(x[4 * k + 1], f, y.y * g);
                x[4 * k + 2] = fmaf(x[4 * k + 2], f, y.z * g);
                x[4 * k + 3] = fmaf(x[4 * k + 3], f, y.w * g);
            }
            store_channels<DT>(a, t, 2 * mine + d, x, half);
        }
        if (mine == 0) store_sum(a, t, half);
        return;
    }
    if (idle) return;
    const Target t = target_of(a, blk, head, row0 + l32, nsp == 1, split, m, sum);
#pragma unroll
    for (int db = 0; db < 4; ++db) store_channels<DT>(a, t, db, st.o[db], half);
    store_sum(a, t, half);
}

// ------------------------------------------------------------------------------------------------ few rows

// What the wavefronts of a few-row kernel have, added up: sums in LDS where their tiles were (`pitch` bytes a wavefront), the 16-byte pieces of row l32 at place piece ^ l32 % 16,
// references and sums of weights behind all of them.
template <int DT, int WAVES, int PITCH>
__device__ __forceinline__ void join_waves(const AttnArgs &a, const Block &blk, const State<DT> &st, unsigned char *smem, int head, int wave, int l32, int half, bool direct, int split)
{
    static_assert(32 * kHeadDim * 4 <= PITCH, "a wavefront's sums fit where its tiles were");
    auto piece = [&](int w, int at) { return (f32x4 *)(smem + w * PITCH + l32 * kHeadDim * 4 + (at ^ (l32 & 15)) * 16); };
    float2 *stats = (float2 *)(smem + WAVES * PITCH);  // [WAVES][32]
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            *piece(wave, db * 8 + 2 * k + half) = f32x4{st.o[db][4 * k], st.o[db][4 * k + 1], st.o[db][4 * k + 2], st.o[db][4 * k + 3]};
    const float z = st.sum();
    if (half == 0) stats[wave * 32 + l32] = make_float2(st.m, z);
    __syncthreads();
    float2 ms[WAVES];
    float top = kFloor, sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        ms[w] = stats[w * 32 + l32];
        top = fmaxf(top, ms[w].x);
    }
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        ms[w].x = exp2_fast(ms[w].x - top);
        sum = fmaf(ms[w].y, ms[w].x, sum);
    }
    const Target t = target_of(a, blk, head, blk.rows0 + l32, direct, split, top, sum);
    static_assert(4 % WAVES == 0, "a wavefront's share of the four channel blocks");
#pragma unroll
    for (int db = wave; db < 4; db += WAVES) {
        f32x16 x = f32x16{};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x4 y = *piece(w, db * 8 + 2 * k + half);
                x[4 * k] = fmaf(y.x, ms[w].x, x[4 * k]);
                x[4 * k + 1] = fmaf(y.y, ms[w].x, x[4 * k + 1]);
                x[4 * k + 2] = fmaf(y.z, ms[w].x, x[4 * k + 2]);
                x[4 * k + 3] = fmaf(y.w, ms[w].x, x[4 * k + 3]);
            }
        }
        store_channels<DT>(a, t, db, x, half);
    }
    if (wave == 0) store_sum(a, t, half);
}

// Bound by reading the cache, and by latency where that is short.  Up to 32 rows: each of WAVES wavefronts takes 32 of a tile's 32 * WAVES tokens, with
// tile buffers of its own and no barrier on the way; what they have is added up at the end.  One buffer each for keys and values (the next keys are asked for
// when these have become logits) and two workgroups a compute unit: a workgroup's start is 3 us of dependent loads, and the other one reads meanwhile.
// Two buffers each and one workgroup, 48 requests with 1 to 16384 tokens 96 -> 86 us, one token of 4097 15.4 -> 13.0 us, of a million 695 either way.
template <int DT, int WAVES, bool PAGED, bool TREE = false, bool ONCE = false>
__global__ __launch_bounds__(WAVES * 64, DT == ILRE_BF16 ? 2 : 1) void attend_tokens(const AttnArgs a)
{
    using E = Elem<DT>;
    constexpr int ROWB = E::ROWB, SLOT = 32 * ROWB, TN = 32 * WAVES;
    constexpr int HALF = 16 * ROWB / 1024, COPIES = 2 * HALF;  // copies of 16 rows, of 32
    extern __shared__ __align__(16) unsigned char smem[];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    const int head = blockIdx.x % a.Hkv;
    Block blk;
    int split;
    if (!find_unit<PAGED>(a, blockIdx.x / a.Hkv, 32, TN, blk, split)) return;
    Drafted drafted;
    if (TREE) drafted.init(a, blk, blk.rows0 + l32);
    const int nsp = ranges_of(blk.nt, a.split_tiles, a.nsplit);
    const int first = split * a.split_tiles, count = (split == nsp - 1 ? blk.nt : first + a.split_tiles) - first;
    auto token_of = [&](int i) { return tile_token(blk, first + i, TN) + wave * 32; };

    State<DT> st;
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)smem + wave * 2 * SLOT;
    typename E::Addr ad;
    ad.init(lane);

    Source ks, vs;
    ks.base = (uint64_t)a.k + (uint64_t)((int64_t)head * a.k_head + (int64_t)blk.kv0 * a.k_token);
    vs.base = (uint64_t)a.v + (uint64_t)((int64_t)head * a.v_head + (int64_t)blk.kv0 * a.v_token);
    ks.page = a.k_page, vs.page = a.v_page, ks.token = a.k_token, vs.token = a.v_token;
    int kvoff[HALF], vvoff[HALF];
    copy_offsets<16, ROWB, false>(kvoff, 0, a.k_token, lane);
    copy_offsets<16, ROWB, true>(vvoff, 0, a.v_token, lane);
    struct Pages {
        int id[2];
    };
    auto lookup = [&](int i) {
        Pages p{};
        if (PAGED) {
            const int t = token_of(i);
            p.id[0] = page_of(a, blk, t);
            p.id[1] = page_of(a, blk, t + 16);
        }
        return p;
    };
    auto copy_keys = [&](int i, const Pages &p) {
        copy_rows<16, ROWB, false, PAGED, ONCE>(a, blk, ks, token_of(i), p.id[0], lds0, kvoff, lane);
        copy_rows<16, ROWB, false, PAGED, ONCE>(a, blk, ks, token_of(i) + 16, p.id[1], lds0 + 16 * ROWB, kvoff, lane);
    };
    auto copy_values = [&](int i, const Pages &p) {
        copy_rows<16, ROWB, true, PAGED, ONCE>(a, blk, vs, token_of(i), p.id[0], lds0 + SLOT, vvoff, lane);
        copy_rows<16, ROWB, true, PAGED, ONCE>(a, blk, vs, token_of(i) + 16, p.id[1], lds0 + SLOT + 16 * ROWB, vvoff, lane);
    };

    Pages now, next;
    if (count > 0) {
        now = lookup(0);
        next = lookup(min(1, count - 1));
        copy_keys(0, now);
        copy_values(0, now);
    }
    st.load(a, blk, head, blk.rows0, l32, half);  // behind the copies: they are on their way together
    st.clear();
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
        const bool more = i + 1 < count;
        const int absent = PAGED ? (now.id[0] < 0 ? 1 : 0) | (now.id[1] < 0 ? 2 : 0) : 0;
        f32x16 s[1];
        typename E::Weights w[1];
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");  // this step's values may still be on their way
        E::logits(s[0], st.q, ad, lds0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the reads are done before the buffer is written again
        if (more) copy_keys(i + 1, next);
        const unsigned seen = TREE ? drafted.bits(token_of(i)) : ~0u;
        st.hide(s[0], token_of(i), a.sink, half, absent, seen);
        st.template weigh<1>(s, w, a.c);
        if (more)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (TREE && __builtin_amdgcn_readfirstlane(token_of(i) + 32 > drafted.base)) keep_rows<E::ROWB>(lds0 + SLOT, of_any_lane(seen), lane);
        E::values(st.o, w[0], ad, lds0 + SLOT);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) {
            copy_values(i + 1, next);
            now = next;
            next = lookup(min(i + 2, count - 1));
        }
    }
    join_waves<DT, WAVES, 2 * SLOT>(a, blk, st, smem, head, wave, l32, half, nsp == 1, split);
}

// ------------------------------------------------------------------------------------------------ few rows over a quantised cache

// The same for a quantised cache: 132 or 68 bytes a token and head instead of 256, so that instructions and LDS count as much as bytes do.  Each wavefront takes 32 of a tile's tokens.
//   - Keys never go through LDS: lane l has half of token l % 32's codes (channels 64 (l / 32) ..), which is the left operand of the matrix instruction once they are converted, two
//     channels an instruction, scale included.  Which channel stands at which place of the contraction is free; the queries are loaded in the same order.
//   - Values are converted, 16 or 32 channels of a token a lane, and written to LDS as numbers, from where the transposing read takes them.
//   - The next tile's codes are asked for when this one's have been converted.
// Bound: HBM; 8 new tokens (32/8 heads) over a million in 8 bits 330 us, 6.4 TB/s, over 131072 61 us in 8 bits and 42 in 4.
// Rows that a wavefront does not see: a key's logit is masked whatever it is (the codes come from a page of the pool in any case); values are read through a buffer that ends with the
// last token, and are zeros past it.
template <int FMT>
struct KeyCodes {
    static constexpr int N = FMT == ILRE_KV_FP8 ? 4 : 2;  // 16-byte pieces of half a token
    u32x4 w[N];
    unsigned scales;  // of the whole token
};
template <int FMT>
struct ValueCodes {
    static constexpr int N = FMT == ILRE_KV_FP8 ? 4 : 2, ROWS = 32 / N;  // pieces a lane, rows that a piece of all lanes holds
    u32x4 w[N];
    unsigned char scale[N];
};

// A piece as bf16, 16 bytes at a time.
template <int FMT>
__device__ __forceinline__ void piece_to_numbers(const u32x4 &w, float scale, u32x4 (&x)[FMT == ILRE_KV_FP8 ? 2 : 4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (FMT == ILRE_KV_FP8)
            x[i / 2][i % 2 * 2] = bf16_pair<FMT, 0>(w[i], scale), x[i / 2][i % 2 * 2 + 1] = bf16_pair<FMT, 1>(w[i], scale);
        else
            x[i] = u32x4{bf16_pair<FMT, 0>(w[i], scale), bf16_pair<FMT, 1>(w[i], scale), bf16_pair<FMT, 2>(w[i], scale), bf16_pair<FMT, 3>(w[i], scale)};
    }
}

// 16 bytes of codes.  LAST: nobody reads their cache line again (the instruction's lanes take it whole, or what is left of it), so that it need not stay in L2.
template <bool LAST>
__device__ __forceinline__ u32x4 load_codes(const unsigned char *p)
{
    return LAST ? __builtin_nontemporal_load((const u32x4 *)p) : *(const u32x4 *)p;
}
template <bool LAST>
__device__ __forceinline__ u32x4 load_codes(__amdgpu_buffer_rsrc_t from, unsigned at)
{
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (int)at, 0, LAST ? 2 : 0));
}

// Workgroups go to the XCDs in turn.  With 4 bits the kv heads of a unit go to the same one: where a token's heads lie side by side, two heads' codes share a cache line, which then comes to one
// L2 and not to two (a million tokens in that layout 369 -> 261 us, 48 requests 38.5 -> 31.2; with a layout by heads 197 either way).  8-bit codes fill their lines, and a kv head an XCD is
// as good (428 us, together 432).  `heads`: of which a workgroup is counted to have one.
template <int FMT>
__device__ __forceinline__ int head_of_block(int heads)
{
    return FMT == ILRE_KV_FP4 ? blockIdx.x / kNumXCD % heads : blockIdx.x % heads;
}
template <int FMT>
__device__ __forceinline__ int unit_of_block(int heads)
{
    return FMT == ILRE_KV_FP4 ? blockIdx.x / kNumXCD / heads * kNumXCD + blockIdx.x % kNumXCD : blockIdx.x / heads;
}

// ONCE: one workgroup reads a cache line of codes, and no other does: there is one block of rows, and no line holds codes of two heads.  Without a place in L2 for each of them, one token over a million in 8 bits
// 359 -> 323 us, in 4 198 -> 186; 48 requests, heads side by side, 48.4 -> 43.8 in 8 bits.  In 4 bits such heads share lines, which then have to stay: 261 us, with ONCE 283.
template <int FMT, int WAVES, bool TREE, bool ONCE>
__global__ __launch_bounds__(WAVES * 64, 2) void attend_codes(const AttnArgs a)
{
    using E = Elem<ILRE_BF16>;
    using K = KeyCodes<FMT>;
    using V = ValueCodes<FMT>;
    constexpr int ROWB = E::ROWB, PITCH = 32 * kHeadDim * 4, TN = 32 * WAVES, ROW = (int)code_bytes<FMT>(ILRE_HEAD_DIM), LANES = ROW / 16;  // lanes a row of values
    static_assert(32 * ROWB <= PITCH, "the values of a tile fit where the sums go");
    extern __shared__ __align__(16) unsigned char smem[];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    const int head = head_of_block<FMT>(a.Hkv);
    Block blk;
    int split;
    if (!find_unit<true>(a, unit_of_block<FMT>(a.Hkv), 32, TN, blk, split)) return;
    Drafted drafted;
    if (TREE) {
        drafted.init(a, blk, blk.rows0 + l32);
        blk.all_hi = max(drafted.base, 0);
    }
    const int nsp = ranges_of(blk.nt, a.split_tiles, a.nsplit);
    const int first = split * a.split_tiles, count = (split == nsp - 1 ? blk.nt : first + a.split_tiles) - first;
    auto token_of = [&](int i) { return tile_token(blk, first + i, TN) + wave * 32; };

    State<ILRE_BF16> st;
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)smem + wave * PITCH;
    typename E::Addr ad;
    ad.init(lane);

    // the kv head's codes and scales, and the lane's places in 32 tokens of them that follow each other
    const int64_t head_at = head * a.k_head;
    const unsigned char *k_codes = a.k + code_bytes<FMT>(head_at), *k_scales = a.k_scales + head_at / ILRE_KV_BLOCK;
    const unsigned char *v_codes = a.v + code_bytes<FMT>(head_at), *v_scales = a.v_scales + head_at / ILRE_KV_BLOCK;
    const unsigned token_bytes = (unsigned)code_bytes<FMT>(a.k_token), token_scales = (unsigned)(a.k_token / ILRE_KV_BLOCK);
    // Pages of 32 tokens and more: a wavefront's tokens are on one.  Otherwise 16 at a time are.  (Offsets within 32 tokens fit 32 bits.)
    const bool wide = a.page_shift >= 5;
    const unsigned k_lane = l32 * token_bytes + half * (ROW / 2), k_lane_scales = l32 * token_scales;
    const int v_row = lane / LANES, v_piece = lane % LANES;  // of a piece of values: its row and place in it
    unsigned v_lane[V::N], v_lane_scales[V::N];
#pragma unroll
    for (int j = 0; j < V::N; ++j) {
        const unsigned row = j * V::ROWS + v_row;
        v_lane[j] = row * token_bytes + v_piece * 16;
        v_lane_scales[j] = row * token_scales + v_piece * 4 / LANES;
    }
    const int page_mask = (1 << a.page_shift) - 1;
    struct Pages {
        int id[2];
    };
    auto lookup = [&](int i) {
        const int t = token_of(i), p = page_of(a, blk, t);
        return Pages{{p, wide ? p : page_of(a, blk, t + 16)}};
    };
    // Where token `tok` lies, in channels from the kv head's first page on.
    auto place = [&](int tok, int page) { return (int64_t)max(page, 0) * a.k_page + (int64_t)(tok & page_mask) * a.k_token; };
    auto fetch_keys = [&](int i, const Pages &p, K &c) {
        const int tok = token_of(i);
        const int64_t at = place(tok, p.id[0]);
        const unsigned char *codes = k_codes + code_bytes<FMT>(at), *scales = k_scales + at / ILRE_KV_BLOCK;
        if (!wide && l32 >= 16) {
            const int64_t skip = place(tok + 16, p.id[1]) - 16 * a.k_token;
            codes = k_codes + code_bytes<FMT>(skip);
            scales = k_scales + skip / ILRE_KV_BLOCK;
        }
#pragma unroll
        for (int j = 0; j < K::N; ++j) c.w[j] = j < K::N - 1 ? load_codes<false>(codes + k_lane + 16 * j) : load_codes<ONCE>(codes + k_lane + 16 * j);
        c.scales = *(const unsigned *)(scales + k_lane_scales);
    };
    // Rows first .. of the tile, N of them at most, which follow each other in memory from `at` (of row 0) on.
    auto fetch_rows = [&](int i, int page, int64_t at, auto begin, auto end, V &c) {
        const int tok = token_of(i), n = page < 0 ? 0 : clamp_to(blk.hi - tok, 0, end.value * V::ROWS);
        auto buffer = [&](const unsigned char *from, unsigned step, unsigned row) {
            const uint64_t u = (uint64_t)from;
            const uint64_t base = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)u);
            return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, __builtin_amdgcn_readfirstlane(n > 0 ? (int)((n - 1) * step + row) : 0), 0x00020000);
        };
        const __amdgpu_buffer_rsrc_t codes = buffer(v_codes + code_bytes<FMT>(at), token_bytes, ROW), scales = buffer(v_scales + at / ILRE_KV_BLOCK, token_scales, 4);
        const bool gap = __builtin_amdgcn_readfirstlane(tok < blk.lo && tok + 32 > blk.sink);
#pragma unroll
        for (int j = begin.value; j < end.value; ++j) {
            unsigned from = v_lane[j], scale_from = v_lane_scales[j];
            if (gap) {
                const int t = tok + j * V::ROWS + v_row;
                if (t < blk.lo && t >= blk.sink) from = scale_from = ~0u;
            }
            c.w[j] = load_codes<ONCE>(codes, from);
            c.scale[j] = __builtin_amdgcn_raw_buffer_load_b8(scales, (int)scale_from, 0, 0);
        }
    };
    auto fetch_values = [&](int i, const Pages &p, V &c) {
        constexpr std::integral_constant<int, 0> none{};
        constexpr std::integral_constant<int, V::N / 2> middle{};
        constexpr std::integral_constant<int, V::N> all{};
        const int tok = token_of(i);
        if (wide) {
            fetch_rows(i, p.id[0], place(tok, p.id[0]), none, all, c);
        } else {
            fetch_rows(i, p.id[0], place(tok, p.id[0]), none, middle, c);
            fetch_rows(i, p.id[1], place(tok + 16, p.id[1]) - 16 * a.k_token, middle, all, c);
        }
    };
    constexpr int NX = FMT == ILRE_KV_FP8 ? 2 : 4;  // 16-byte pieces of numbers in one of codes
    // Eight lanes write together; so that they reach all banks, a lane's pieces go out in an order of its own: piece k ^ turn.
    const int turn = NX == 2 ? v_piece >> 2 : v_piece >> 1 | (v_row & 1) << 1;
    unsigned v_to[NX];
#pragma unroll
    for (int k = 0; k < NX; ++k) v_to[k] = lds0 + v_row * ROWB + (((NX * v_piece + (k ^ turn)) ^ (v_row & 3) << 2) * 16);
    auto write_values = [&](const V &c) {
#pragma unroll
        for (int j = 0; j < V::N; ++j) {
            u32x4 w = c.w[j], x[NX];
            if (NX == 2) {
                w = turn ? u32x4{w[2], w[3], w[0], w[1]} : w;
            } else {
                w = turn & 1 ? u32x4{w[1], w[0], w[3], w[2]} : w;
                w = turn & 2 ? u32x4{w[2], w[3], w[0], w[1]} : w;
            }
            piece_to_numbers<FMT>(w, scale_of(c.scale[j]), x);
#pragma unroll
            for (int k = 0; k < NX; ++k) lds_write16(v_to[k] + j * V::ROWS * ROWB, x[k]);
        }
    };
    // Logits of the tile's 32 tokens: piece j of a lane holds channels 64 half + ROW / 2 / N j .. of its token.
    auto logits = [&](f32x16 &s, const K &c) {
        s = f32x16{};
        const unsigned mine = c.scales >> (16 * half);
        const float scale[2] = {scale_of(mine & 255), scale_of(mine >> 8 & 255)};
#pragma unroll
        for (int j = 0; j < K::N; ++j) {
            u32x4 x[NX];
            piece_to_numbers<FMT>(c.w[j], scale[j * 2 / K::N], x);
#pragma unroll
            for (int k = 0; k < NX; ++k) E::mma(s, x[k], st.q[j * NX + k]);
        }
    };

    K keys;
    V values;
    Pages now, next;
    if (count > 0) {
        now = lookup(0);
        next = lookup(min(1, count - 1));
        fetch_keys(0, now, keys);
        fetch_values(0, now, values);
    }
    st.template load<true>(a, blk, head, blk.rows0, l32, half);  // behind the codes: they are on their way together
    st.clear();
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
        const bool more = i + 1 < count;
        const int tok = token_of(i), absent = (now.id[0] < 0 ? 1 : 0) | (now.id[1] < 0 ? 2 : 0);
        f32x16 s[1];
        typename E::Weights w[1];
        logits(s[0], keys);
        write_values(values);
        if (more) {
            fetch_keys(i + 1, next, keys);
            fetch_values(i + 1, next, values);
        }
        if (tok < blk.all_lo || tok + 32 > blk.all_hi || absent) {  // an edge: what a row does not see is hidden
            const unsigned seen = TREE ? drafted.bits(tok) : ~0u;
            if (TREE) keep_rows<ROWB>(lds0, of_any_lane(seen), lane);
            st.hide(s[0], tok, a.sink, half, absent, seen);
        }
        st.template weigh<1, true>(s, w, a.c);
        E::values(st.o, w[0], ad, lds0);
        if (more) {
            now = next;
            next = lookup(min(i + 2, count - 1));
        }
    }
    join_waves<ILRE_BF16, WAVES, PITCH>(a, blk, st, smem, head, wave, l32, half, nsp == 1, split);
}

// Up to 16 rows: the matrix instructions of 16 rows, as half of the logits, exponentials and sums above would be nobody's.  Lane l has query l % 16; tokens 16 b + 4 (l / 16) + i of
// logits, i = 0..3, b = 0, 1; channels 16 db + 4 (l / 16) + i of sums.  Of keys it has a quarter of the codes, one block of a scale, of tokens l % 16 and 16 + l % 16.  With fewer
// registers and half the LDS three or four workgroups fit a compute unit.  HEADS: kv heads a workgroup, whose wavefronts then share out the tokens of WAVES / HEADS x 32 between those of a head.
//
// Bound: HBM.  One token over a million (32/8 heads) 323 us in 8 bits, 6.5 TB/s, and 187 in 4, 5.8 (with the merge, 6); heads side by side 349 and 228; over 4097, 8 bits, 6.8 us and 3.6 for the merge.
//
// Keys and values are exact in bf16, so that fp32 states take the bf16 matrix instructions too: queries and weights go in as three parts, each the upper 16 bits of what is left, which hold 24 bits
// (the fp32 matrix instructions are a sixteenth as fast; the nearest bf16 of a number beyond 2^128 - 2^119 would be an infinity).
__device__ __forceinline__ void split_parts(const float (&x)[8], u32x4 (&part)[3])
{
    float rest[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) rest[k] = x[k];
#pragma unroll
    for (int n = 0; n < 3; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned lo = __float_as_uint(rest[2 * k]), hi = __float_as_uint(rest[2 * k + 1]);
            part[n][k] = __builtin_amdgcn_perm(hi, lo, 0x07060302);
            rest[2 * k] -= __uint_as_float(lo & 0xFFFF0000u);
            rest[2 * k + 1] -= __uint_as_float(hi & 0xFFFF0000u);
        }
}

template <int DT, int FMT, int WAVES, bool TREE, bool ONCE, int HEADS>
__global__ __launch_bounds__(WAVES * 64, DT == ILRE_F32 ? 2 : FMT == ILRE_KV_FP4 && !TREE ? 4 : 3) void attend_codes16(const AttnArgs a)
{
    constexpr int PARTS = DT == ILRE_F32 ? 3 : 1;  // of queries and weights
    using V = ValueCodes<FMT>;
    constexpr int ROWB = 256, PITCH = 32 * ROWB, SHARE = WAVES / HEADS, TN = 32 * SHARE, ROW = (int)code_bytes<FMT>(ILRE_HEAD_DIM), LANES = ROW / 16, KN = ROW / 64;  // KN: 16-byte pieces of a quarter of a token
    extern __shared__ __align__(16) unsigned char smem[];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int head0 = head_of_block<FMT>(a.Hkv / HEADS) * HEADS, head = head0 + wave / SHARE;
    Block blk;
    int split;
    if (!find_unit<true>(a, unit_of_block<FMT>(a.Hkv / HEADS), 16, TN, blk, split)) return;
    Drafted drafted;
    if (TREE) {
        drafted.init(a, blk, blk.rows0 + l16);
        blk.all_hi = max(drafted.base, 0);
    }
    const int nsp = ranges_of(blk.nt, a.split_tiles, a.nsplit);
    const int first = split * a.split_tiles, count = (split == nsp - 1 ? blk.nt : first + a.split_tiles) - first;
    auto token_of = [&](int i) { return tile_token(blk, first + i, TN) + wave % SHARE * 32; };

    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)smem + wave * PITCH;
    // the kv head's codes and scales, and the lane's places in 16 or 32 tokens of them that follow each other
    const int64_t head_at = head * a.k_head;
    const unsigned char *k_codes = a.k + code_bytes<FMT>(head_at), *k_scales = a.k_scales + head_at / ILRE_KV_BLOCK;
    const unsigned char *v_codes = a.v + code_bytes<FMT>(head_at), *v_scales = a.v_scales + head_at / ILRE_KV_BLOCK;
    const unsigned token_bytes = (unsigned)code_bytes<FMT>(a.k_token), token_scales = (unsigned)(a.k_token / ILRE_KV_BLOCK);
    const bool wide = a.page_shift >= 5;  // a wavefront's 32 tokens are on one page
    const unsigned k_lane = l16 * token_bytes + g * (ROW / 4), k_lane_scales = l16 * token_scales + g;
    const int v_row = lane / LANES, v_piece = lane % LANES;
    const unsigned v_lane = v_row * token_bytes + v_piece * 16, v_lane_scales = v_row * token_scales + v_piece * 4 / LANES;
    const int page_mask = (1 << a.page_shift) - 1;
    struct Pages {
        int id[2];
    };
    auto lookup = [&](int i) {
        const int t = token_of(i), p = page_of(a, blk, t);
        return Pages{{p, wide ? p : page_of(a, blk, t + 16)}};
    };
    auto place = [&](int tok, int page) { return (int64_t)max(page, 0) * a.k_page + (int64_t)(tok & page_mask) * a.k_token; };
    struct K {
        u32x4 w[2][KN];
        unsigned char scale[2];
    };
    auto fetch_keys = [&](int i, const Pages &p, K &c) {
        const int tok = token_of(i);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int64_t at = place(tok + 16 * b, p.id[b]);
            const unsigned char *codes = k_codes + code_bytes<FMT>(at), *scales = k_scales + at / ILRE_KV_BLOCK;
#pragma unroll
            for (int j = 0; j < KN; ++j) c.w[b][j] = j < KN - 1 ? load_codes<false>(codes + k_lane + 16 * j) : load_codes<ONCE>(codes + k_lane + 16 * j);
            c.scale[b] = scales[k_lane_scales];
        }
    };
    auto fetch_values = [&](int i, const Pages &p, V &c) {
        const int tok = token_of(i);
        const bool gap = __builtin_amdgcn_readfirstlane(tok < blk.lo && tok + 32 > blk.sink);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int t0 = tok + 16 * b, n = p.id[b] < 0 ? 0 : clamp_to(blk.hi - t0, 0, 16);
            const int64_t at = place(t0, p.id[b]);
            auto buffer = [&](const unsigned char *from, unsigned step, unsigned row) {
                const uint64_t u = (uint64_t)from;
                const uint64_t base = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)u);
                return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, __builtin_amdgcn_readfirstlane(n > 0 ? (int)((n - 1) * step + row) : 0), 0x00020000);
            };
            const __amdgpu_buffer_rsrc_t codes = buffer(v_codes + code_bytes<FMT>(at), token_bytes, ROW), scales = buffer(v_scales + at / ILRE_KV_BLOCK, token_scales, 4);
#pragma unroll
            for (int j = 0; j < V::N / 2; ++j) {
                unsigned from = v_lane + j * V::ROWS * token_bytes, scale_from = v_lane_scales + j * V::ROWS * token_scales;
                if (gap) {
                    const int t = t0 + j * V::ROWS + v_row;
                    if (t < blk.lo && t >= blk.sink) from = scale_from = ~0u;
                }
                c.w[b * (V::N / 2) + j] = load_codes<ONCE>(codes, from);
                c.scale[b * (V::N / 2) + j] = __builtin_amdgcn_raw_buffer_load_b8(scales, (int)scale_from, 0, 0);
            }
        }
    };
    // Values in LDS: 16-byte chunk c of row r at place c ^ 2 (r % 4), for the transposing read of 4 rows and 16 channels by 16 lanes; a lane's chunks are written in an order of its own, k ^ turn,
    // so that eight lanes reach all banks.
    constexpr int NX = FMT == ILRE_KV_FP8 ? 2 : 4;
    const int turn = FMT == ILRE_KV_FP8 ? v_piece >> 2 : v_piece >> 1;
    unsigned v_to[NX], v_from[4];
#pragma unroll
    for (int k = 0; k < NX; ++k) v_to[k] = lds0 + v_row * ROWB + (((NX * v_piece + (k ^ turn)) ^ (v_row & 3) << 1) * 16);
#pragma unroll
    for (int d = 0; d < 4; ++d) v_from[d] = lds0 + (4 * g + (l16 >> 2)) * ROWB + (d ^ (l16 >> 2)) * 32 + (l16 & 3) * 8;
    auto write_values = [&](const V &c) {
#pragma unroll
        for (int j = 0; j < V::N; ++j) {
            u32x4 w = c.w[j], x[NX];
            w = turn ? (NX == 2 ? u32x4{w[2], w[3], w[0], w[1]} : u32x4{w[1], w[0], w[3], w[2]}) : w;
            piece_to_numbers<FMT>(w, scale_of(c.scale[j]), x);
#pragma unroll
            for (int k = 0; k < NX; ++k) lds_write16(v_to[k] + j * V::ROWS * ROWB, x[k]);
        }
    };
    auto mma = [](f32x4 &acc, const u32x4 &x, const u32x4 &y) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), acc, 0, 0, 0);
    };

    K keys;
    V values;
    Pages now, next;
    if (count > 0) {
        now = lookup(0);
        next = lookup(min(1, count - 1));
        fetch_keys(0, now, keys);
        fetch_values(0, now, values);
    }
    // the lane's query: channels 32 g + 8 st .. of row rows0 + l16; past the last row zeros, which see what the last one sees and are written nowhere
    u32x4 q[4][PARTS];
    int lo, hi;
    {
        const int want = blk.rows0 + l16, r = min(want, blk.nrows - 1), i = r / a.G;
        const unsigned char *src = a.q + (int64_t)(blk.q0 + i) * a.q_token + (int64_t)(head * a.G + r - i * a.G) * a.q_head + g * (DT == ILRE_F32 ? 128 : 64);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (DT == ILRE_F32) {
                const f32x4 x = ((const f32x4 *)src)[2 * k], y = ((const f32x4 *)src)[2 * k + 1];
                const bool real = want == r;
                const float f[8] = {real ? x[0] : 0.f, real ? x[1] : 0.f, real ? x[2] : 0.f, real ? x[3] : 0.f, real ? y[0] : 0.f, real ? y[1] : 0.f, real ? y[2] : 0.f, real ? y[3] : 0.f};
                split_parts(f, q[k]);
            } else {
                q[k][0] = want == r ? *(const u32x4 *)(src + k * 16) : u32x4{};
            }
        }
        const int p = max(blk.kv - blk.q_len + i, -1);
        hi = a.causal ? min(p + 1, blk.kv) : blk.kv;
        lo = a.window > 0 ? max(p - a.window + 1, 0) : 0;
    }
    f32x4 o[8];
#pragma unroll
    for (int db = 0; db < 8; ++db) o[db] = f32x4{};
    float m = kFloor, z = 0.f;
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
        const bool more = i + 1 < count;
        const int tok = token_of(i), absent = (now.id[0] < 0 ? 1 : 0) | (now.id[1] < 0 ? 2 : 0);
        f32x4 s[2] = {f32x4{}, f32x4{}};
#pragma unroll
        for (int j = 0; j < KN; ++j) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                u32x4 x[NX];
                piece_to_numbers<FMT>(keys.w[b][j], scale_of(keys.scale[b]), x);
#pragma unroll
                for (int k = 0; k < NX; ++k)
#pragma unroll
                    for (int n = PARTS - 1; n >= 0; --n) mma(s[b], x[k], q[j * NX + k][n]);
            }
        }
        write_values(values);
        if (more) {
            fetch_keys(i + 1, next, keys);
            fetch_values(i + 1, next, values);
        }
        if (tok < blk.all_lo || tok + 32 > blk.all_hi || absent) {  // an edge: what a row does not see is hidden
            const unsigned seen = TREE ? drafted.bits(tok) : ~0u;
            if (TREE) keep_rows<ROWB>(lds0, of_any_lane(seen), lane);
            unsigned bits = first_bits(hi - tok) & (~first_bits(lo - tok) | first_bits(a.sink - tok)) & seen;
            bits &= ~((absent & 1 ? 0xFFFFu : 0u) | (absent & 2 ? 0xFFFF0000u : 0u));
            bits >>= 4 * g;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int k = 0; k < 4; ++k) s[b][k] = bits >> (16 * b + k) & 1 ? s[b][k] : -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int k = 1; k < 8; ++k) top = fmaxf(top, s[k / 4][k % 4]);
        top = larger_of_halves(top);
        {
            const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
        }
        const float mnew = fmaxf(m, top * a.c);
        if (__ballot(mnew != m)) {
            const float f = exp2_fast(m - mnew);
#pragma unroll
            for (int db = 0; db < 8; ++db) o[db] *= f;
            z *= f;
            m = mnew;
        }
        float p[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) p[k] = exp2_fast(fmaf(s[k / 4][k % 4], a.c, -m));
        z += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        u32x4 w[PARTS];
        if constexpr (DT == ILRE_F32)
            split_parts(p, w);
        else
            w[0] = u32x4{pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7])};
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            const u32x2 x = lds_read_tr(v_from[db & 3] + (db >> 2) * 128), y = lds_read_tr(v_from[db & 3] + (db >> 2) * 128 + 16 * ROWB);
#pragma unroll
            for (int n = PARTS - 1; n >= 0; --n) mma(o[db], u32x4{x[0], x[1], y[0], y[1]}, w[n]);
        }
        if (more) {
            now = next;
            next = lookup(min(i + 2, count - 1));
        }
    }
    // What the wavefronts have, added up: sums where the values were, 16-byte piece of row l16 at place piece ^ l16 % 8, references and sums of weights behind all of them; then a thread
    // has eight channels of a row.
    static_assert(16 * kHeadDim * 4 <= PITCH && WAVES * 64 == 256, "sums of 16 rows; 16 threads a row");
    z += __shfl_xor(z, 16);
    z += __shfl_xor(z, 32);
    float2 *stats = (float2 *)(smem + WAVES * PITCH);  // [WAVES][16]
    auto piece = [&](int w, int row, int at) { return (f32x4 *)(smem + w * PITCH + row * kHeadDim * 4 + (at ^ (row & 7)) * 16); };
#pragma unroll
    for (int db = 0; db < 8; ++db) *piece(wave, l16, db * 4 + g) = o[db];
    if (g == 0) stats[wave * 16 + l16] = make_float2(m, z);
    __syncthreads();
    const int row = tid >> 4, part = tid & 15;
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        float2 ms[SHARE];
        float top = kFloor, sum = 0.f;
#pragma unroll
        for (int w = 0; w < SHARE; ++w) {
            ms[w] = stats[(h * SHARE + w) * 16 + row];
            top = fmaxf(top, ms[w].x);
        }
        f32x4 x[2] = {f32x4{}, f32x4{}};
#pragma unroll
        for (int w = 0; w < SHARE; ++w) {
            const float f = exp2_fast(ms[w].x - top);
            sum = fmaf(ms[w].y, f, sum);
#pragma unroll
            for (int k = 0; k < 2; ++k) x[k] += *piece(h * SHARE + w, row, 2 * part + k) * f;
        }
        const Target t = target_of(a, blk, head0 + h, blk.rows0 + row, nsp == 1, split, top, sum);
        if (!t.real) return;
        x[0] *= t.f;
        x[1] *= t.f;
        if (t.direct && DT == ILRE_BF16) {
            *(uint4 *)(t.out + part * 16) = make_uint4(pack_bf16(x[0][0], x[0][1]), pack_bf16(x[0][2], x[0][3]), pack_bf16(x[1][0], x[1][1]), pack_bf16(x[1][2], x[1][3]));
        } else {
            f32x4 *to = (f32x4 *)(t.direct ? (float *)t.out : a.part_o + t.row * kHeadDim) + part * 2;
            to[0] = x[0];
            to[1] = x[1];
        }
        store_sum(a, t, part);
    }
}

// ------------------------------------------------------------------------------------------------ merge of the ranges

// What is read here has just been written: latency.  16 lanes a row (token, head), 8 channels each: out = sum_s 2^(e_s - E) o_s / sum_s 2^(e_s - E), E the largest e_s.  WIDE: a workgroup a row, its 16 groups
// of 16 lanes take every 16th range and are added up in their order: with few rows there is nothing else to have loads under way from.  Logarithms and
// results are asked for before it is known how many ranges there are (all of them lie in the workspace), so that one latency passes, not three.  32 rows
// of 64 ranges 5.4 us (16 lanes a row: 15), 32768 rows of two 11 us (a wavefront a row: 22).
template <int DT, bool PAGED, bool WIDE>
__global__ __launch_bounds__(256) void merge_ranges(const AttnArgs a)
{
    constexpr int STEP = WIDE ? 16 : 1, EARLY = 2;
    __shared__ float4 parts[WIDE ? 16 : 1][16][2];
    __shared__ float sums[16];
    const int lane = threadIdx.x & 63, l16 = threadIdx.x & 15, group = threadIdx.x >> 4, mine = WIDE ? group : 0;
    const int64_t rows = (int64_t)a.T * a.Hq, row = WIDE ? blockIdx.x : (int64_t)blockIdx.x * 16 + group;
    // the row's sequence: the wavefront looks for the one of its first row's token, the others follow it
    const int64_t first_row = WIDE ? row : (int64_t)blockIdx.x * 16 + (threadIdx.x >> 6) * 4;
    if (first_row >= rows) return;
    const float *e = a.part_e + min(row, rows - 1), *o = a.part_o + min(row, rows - 1) * kHeadDim + 8 * l16;
    float ee = l16 < a.nsplit ? e[l16 * rows] : 0.f;
    float4 y[EARLY], z[EARLY];
#pragma unroll
    for (int k = 0; k < EARLY; ++k) {
        const int64_t s = min(mine + k * STEP, a.nsplit - 1);
        y[k] = *(const float4 *)(o + s * rows * kHeadDim);
        z[k] = *(const float4 *)(o + s * rows * kHeadDim + 4);
    }
    const int token = (int)(row / a.Hq), head = (int)(row - (int64_t)token * a.Hq), first = (int)(first_row / a.Hq);
    int seq = 0;
    if (a.n_seq > 1) {
        for (int base = 0; base < a.n_seq; base += 64) {
            const int s = base + lane;
            const unsigned long long past = __ballot(s < a.n_seq && clamp_to(a.cu_q[s + 1], 0, a.T) > first);
            if (past) {
                seq = base + __builtin_ctzll(past);
                break;
            }
        }
    }
    if (row >= rows) return;
    while (seq < a.n_seq - 1 && clamp_to(a.cu_q[seq + 1], 0, a.T) <= token) ++seq;
    Block blk;
    sequence_of<PAGED>(a, seq, blk);
    if (token < blk.q0 || token >= blk.q0 + blk.q_len) return;  // a token of no sequence
    const int r = (token - blk.q0) * a.G + head % a.G;
    blk.rows0 = r / a.rows * a.rows;
    tiles_of(blk, mask_of(a), a.G, a.rows, a.tile);
    const int nsp = ranges_of(blk.nt, a.split_tiles, a.nsplit);
    if (nsp == 1) return;  // written already
    float top = l16 < nsp ? ee : -INFINITY;
    for (int s = l16 + 16; s < nsp; s += 16) top = fmaxf(top, e[s * rows]);
#pragma unroll
    for (int k = 1; k < 16; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
    const float ref = top == -INFINITY ? 0.f : top;  // no range has a token that the row sees
    float sum = 0.f, x[8] = {};
    auto take = [&](int s, const float4 &u, const float4 &v) {
        const float w = exp2_fast(e[s * rows] - ref);
        sum += w;
        x[0] = fmaf(w, u.x, x[0]), x[1] = fmaf(w, u.y, x[1]), x[2] = fmaf(w, u.z, x[2]), x[3] = fmaf(w, u.w, x[3]);
        x[4] = fmaf(w, v.x, x[4]), x[5] = fmaf(w, v.y, x[5]), x[6] = fmaf(w, v.z, x[6]), x[7] = fmaf(w, v.w, x[7]);
    };
#pragma unroll
    for (int k = 0; k < EARLY; ++k)
        if (mine + k * STEP < nsp) take(mine + k * STEP, y[k], z[k]);
#pragma unroll 4
    for (int s = mine + EARLY * STEP; s < nsp; s += STEP)
        take(s, *(const float4 *)(o + s * rows * kHeadDim), *(const float4 *)(o + s * rows * kHeadDim + 4));
    if (WIDE) {
        parts[group][l16][0] = make_float4(x[0], x[1], x[2], x[3]);
        parts[group][l16][1] = make_float4(x[4], x[5], x[6], x[7]);
        if (l16 == 0) sums[group] = sum;
        __syncthreads();
        if (group != 0) return;
        const int n = min(nsp, 16);
        for (int g = 1; g < n; ++g) {
            const float4 u = parts[g][l16][0], v = parts[g][l16][1];
            x[0] += u.x, x[1] += u.y, x[2] += u.z, x[3] += u.w;
            x[4] += v.x, x[5] += v.y, x[6] += v.z, x[7] += v.w;
            sum += sums[g];
        }
    }
    const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] *= f;
    unsigned char *to = a.out + (int64_t)token * a.out_token + (int64_t)head * a.out_head;
    if (DT == ILRE_F32) {
        *(float4 *)(to + 32 * l16) = make_float4(x[0], x[1], x[2], x[3]);
        *(float4 *)(to + 32 * l16 + 16) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        *(uint4 *)(to + 16 * l16) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
    if (l16 == 0 && a.lse) a.lse[row] = sum == 0.f ? -INFINITY : (ref + __log2f(sum)) * kLn2;
}

template <int DT, bool PAGED>
hipError_t launch_merge(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    const int64_t rows = (int64_t)a.T * a.Hq;
    if (rows <= 512 && p.nsplit > 4)
        hipLaunchKernelGGL((merge_ranges<DT, PAGED, true>), dim3((unsigned)rows), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((merge_ranges<DT, PAGED, false>), dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, s, a);
    return hipGetLastError();
}

constexpr int kMaxLds = 136 * 1024;
hipError_t raise_lds_limit_once(const void *kernel)
{
    static std::mutex mutex;
    static const void *done[32];
    static int ndone = 0;
    std::lock_guard<std::mutex> lock(mutex);
    for (int i = 0; i < ndone; ++i)
        if (done[i] == kernel) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kMaxLds);
    if (e == hipSuccess && ndone < 32) done[ndone++] = kernel;
    return e;
}

// units_step: the number of units is rounded up to a multiple of it.
template <typename K>
hipError_t launch(K kernel, const AttnPlan &p, int threads, size_t lds, const AttnArgs &a, hipStream_t s, unsigned units_step = 1, int heads = 1)
{
    const hipError_t e = raise_lds_limit_once((const void *)kernel);
    if (e != hipSuccess) return e;
    const unsigned units = ((unsigned)p.nsplit * p.nblocks + units_step - 1) / units_step * units_step;
    hipLaunchKernelGGL(kernel, dim3(units * (a.Hkv / heads)), dim3(threads), lds, s, a);
    return hipGetLastError();
}

template <int DT, int WAVES, int TS, int TN, bool PAGED, int FMT, bool TREE>
hipError_t launch_rows(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    return launch(attend_rows<DT, WAVES, TS, TN, PAGED, FMT, TREE>, p, WAVES * 64, 2 * Elem<DT>::RING * TN * Elem<DT>::ROWB + 16 + (TS == 2 ? WAVES * 32 * sizeof(float2) : 0), a, s);
}

// Whether a workgroup is the only reader of the cache lines that it reads codes from.  (bf16 states come to the kernels for few rows with one block of rows a sequence.)
template <int DT, int FMT>
bool read_once(const AttnPlan &p, const AttnArgs &a)
{
    return (DT == ILRE_BF16 || p.one_block) && (FMT == ILRE_KV_FP8 || a.k_token == ILRE_HEAD_DIM);
}

template <int DT, int WAVES, bool PAGED, int FMT, bool TREE>
hipError_t launch_tokens(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    if constexpr (FMT != kPlain)
        return launch(read_once<DT, FMT>(p, a) ? attend_codes<FMT, WAVES, TREE, true> : attend_codes<FMT, WAVES, TREE, FMT == ILRE_KV_FP8>, p, WAVES * 64,
                      WAVES * (32 * kHeadDim * 4 + 32 * sizeof(float2)), a, s, FMT == ILRE_KV_FP4 ? kNumXCD : 1);
    else
        // Under a tree, tiles that are many take no place in L2 (8 drafted tokens over a million 687 -> 621 us, four drafts over 32768 each 106 -> 95; where a workgroup has a few tiles 20.9 -> 21.3).
        return launch(TREE && p.many_tiles ? attend_tokens<DT, WAVES, PAGED, TREE, TREE> : attend_tokens<DT, WAVES, PAGED, TREE>, p, WAVES * 64,
                      WAVES * (2 * 32 * Elem<DT>::ROWB + 32 * sizeof(float2)), a, s);
}

template <int DT, int FMT, bool TREE>
hipError_t launch_codes16(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    auto go = [&](auto kernel, int heads) { return launch(kernel, p, 256, 4 * (32 * 256 + 16 * sizeof(float2)), a, s, FMT == ILRE_KV_FP4 ? kNumXCD : 1, heads); };
    if constexpr (DT == ILRE_BF16 && !TREE) {
        if (p.heads == 4) return go(attend_codes16<DT, FMT, 4, TREE, FMT == ILRE_KV_FP8, 4>, 4);
        if constexpr (FMT == ILRE_KV_FP8) {
            if (p.heads == 2) return go(attend_codes16<DT, FMT, 4, TREE, true, 2>, 2);
        }
    }
    return read_once<DT, FMT>(p, a) ? go(attend_codes16<DT, FMT, 4, TREE, true, 1>, 1) : go(attend_codes16<DT, FMT, 4, TREE, DT == ILRE_BF16 && FMT == ILRE_KV_FP8, 1>, 1);
}

template <bool PAGED, int FMT = kPlain, bool TREE = false>
hipError_t launch_kernels(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    hipError_t e;
    if constexpr (FMT != kPlain) {
        if (p.rows == 16) {
            e = p.dtype == ILRE_BF16 ? launch_codes16<ILRE_BF16, FMT, TREE>(p, a, s) : launch_codes16<ILRE_F32, FMT, TREE>(p, a, s);
            if (e != hipSuccess || p.nsplit == 1) return e;
            return p.dtype == ILRE_BF16 ? launch_merge<ILRE_BF16, PAGED>(p, a, s) : launch_merge<ILRE_F32, PAGED>(p, a, s);
        }
    }
    if (p.dtype == ILRE_BF16) {
        if (p.rows == 32)
            e = launch_tokens<ILRE_BF16, 4, PAGED, FMT, TREE>(p, a, s);
        else if (p.rows == 128)
            e = launch_rows<ILRE_BF16, 8, 2, 64, PAGED, FMT, TREE>(p, a, s);
        else
            e = launch_rows<ILRE_BF16, 8, 1, 64, PAGED, FMT, TREE>(p, a, s);
    } else if constexpr (FMT == kPlain) {
        if (p.rows == 32)
            e = launch_tokens<ILRE_F32, 4, PAGED, FMT, TREE>(p, a, s);
        else
            e = launch_rows<ILRE_F32, 4, 1, 32, PAGED, FMT, TREE>(p, a, s);
    } else {
        e = hipErrorInvalidValue;  // (fp32 states over a quantised cache are cut into 16 rows)
    }
    if (e != hipSuccess || p.nsplit == 1) return e;
    return p.dtype == ILRE_BF16 ? launch_merge<ILRE_BF16, PAGED>(p, a, s) : launch_merge<ILRE_F32, PAGED>(p, a, s);
}

}  // namespace
}  // namespace ilre
