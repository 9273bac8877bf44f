// Attention of new tokens over a cache of pages, and over whole packed prompts, for gfx950.
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
#include "attn_blocks.h"
#include "ilre_internal.h"

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
template <int ROWS, int ROWB, bool VALUES, bool PAGED>
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
        for (int j = 0; j < N; ++j) lds_dma16(rsrc, __builtin_amdgcn_readfirstlane(to + j * 1024), voff[j]);
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

// ------------------------------------------------------------------------------------------------ products

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
    __device__ __forceinline__ void load(const AttnArgs &a, const Block &blk, int head_kv, int row0, int l32, int half)
    {
        const int want = row0 + l32, r = min(want, blk.nrows - 1);
        const int i = r / a.G, g = r - i * a.G;
        const unsigned char *src = a.q + (int64_t)(blk.q0 + i) * a.q_token + (int64_t)(head_kv * a.G + g) * a.q_head + half * 16;
#pragma unroll
        for (int st = 0; st < E::QREGS; ++st) q[st] = *(const u32x4 *)(src + st * 32);
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
    __device__ __forceinline__ void hide(f32x16 &s, int at, int sink, int half, int absent) const
    {
        unsigned bits = first_bits(hi - at) & (~first_bits(lo - at) | first_bits(sink - at));
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
    template <int SUB>
    __device__ __forceinline__ void weigh(const f32x16 (&s)[SUB], typename E::Weights (&w)[SUB], float c)
    {
        float top = largest(s[0]);
#pragma unroll
        for (int u = 1; u < SUB; ++u) top = fmaxf(top, largest(s[u]));
        top = fmaxf(top, other_half(top));
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
template <int DT, int WAVES, int TS, int TN, bool PAGED>
__global__ __launch_bounds__(WAVES * 64, 2) void attend_rows(const AttnArgs a)
{
    using E = Elem<DT>;
    constexpr int ROWB = E::ROWB, SLOT = TN * ROWB, GROUPS = WAVES / TS, ROWS = GROUPS * 32, SUB = TN / 32 / TS, RING = E::RING;
    constexpr int CROWS = TN / WAVES, COPIES = CROWS * ROWB / 1024;  // a wavefront's rows and copies of a tile
    static_assert(CROWS <= 16 && CROWS * ROWB % 1024 == 0 && TN % 32 == 0, "a wavefront's rows lie on one page");
    extern __shared__ __align__(16) unsigned char smem[];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    // kv heads run fastest: workgroups that share keys and values are a multiple of Hkv apart, on one XCD where Hkv is a multiple of 8
    const int head = blockIdx.x % a.Hkv;
    Block blk;
    int split;
    if (!find_unit<PAGED>(a, blockIdx.x / a.Hkv, ROWS, TN, blk, split)) return;
    const int nsp = ranges_of(blk.nt, a.split_tiles, a.nsplit);
    const int first = split * a.split_tiles, count = (split == nsp - 1 ? blk.nt : first + a.split_tiles) - first;
    auto token_of = [&](int i) { return tile_token(blk, first + i, TN); };

    State<DT> st;
    const int row0 = blk.rows0 + wave % GROUPS * 32, part = wave / GROUPS * SUB * 32;  // its rows, and where its part of a tile begins
    const bool idle = row0 >= blk.nrows;

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
    int pages[2];  // of this wavefront's rows: of the last tile whose keys were asked for, and the next one
    auto own_token = [&](int i) { return i < count ? token_of(i) + wave * CROWS : blk.hi; };
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
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) E::logits(s[sub], st.q, ad, keys_at(i, sub));
        int absent = 0;
        if (PAGED && careful) {
            for (int k = 0; k < SUB * 2; ++k) absent |= (page_of(a, blk, tok + 16 * k) < 0 ? 1 : 0) << k;
        }
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) st.hide(s[sub], tok + 32 * sub, a.sink, half, absent >> (2 * sub));
        if (kept.value) {
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) st.weigh_kept(s[sub], w[sub], a.c);
        } else {
            st.template weigh<SUB>(s, w, a.c);
        }
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub) E::values(st.o, w[sub], ad, values_at(i, sub));
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

// Bound by reading the cache, and by latency where that is short.  Up to 32 rows: each of WAVES wavefronts takes 32 of a tile's 32 * WAVES tokens, with
// tile buffers of its own and no barrier on the way; what they have is added up at the end.  One buffer each for keys and values (the next keys are asked for
// when these have become logits) and two workgroups a compute unit: a workgroup's start is 3 us of dependent loads, and the other one reads meanwhile.
// Two buffers each and one workgroup, 48 requests with 1 to 16384 tokens 96 -> 86 us, one token of 4097 15.4 -> 13.0 us, of a million 695 either way.
template <int DT, int WAVES, bool PAGED>
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
        copy_rows<16, ROWB, false, PAGED>(a, blk, ks, token_of(i), p.id[0], lds0, kvoff, lane);
        copy_rows<16, ROWB, false, PAGED>(a, blk, ks, token_of(i) + 16, p.id[1], lds0 + 16 * ROWB, kvoff, lane);
    };
    auto copy_values = [&](int i, const Pages &p) {
        copy_rows<16, ROWB, true, PAGED>(a, blk, vs, token_of(i), p.id[0], lds0 + SLOT, vvoff, lane);
        copy_rows<16, ROWB, true, PAGED>(a, blk, vs, token_of(i) + 16, p.id[1], lds0 + SLOT + 16 * ROWB, vvoff, lane);
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
        st.hide(s[0], token_of(i), a.sink, half, absent);
        st.template weigh<1>(s, w, a.c);
        if (more)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        E::values(st.o, w[0], ad, lds0 + SLOT);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) {
            copy_values(i + 1, next);
            now = next;
            next = lookup(min(i + 2, count - 1));
        }
    }
    // What the wavefronts have: sums where their tiles were, the 16-byte pieces of row l32 at place piece ^ l32 % 16, references and sums of weights
    // behind all of them.
    static_assert(32 * kHeadDim * 4 <= 2 * SLOT, "a wavefront's sums fit where its tiles were");
    auto piece = [&](int w, int at) { return (f32x4 *)(smem + w * 2 * SLOT + l32 * kHeadDim * 4 + (at ^ (l32 & 15)) * 16); };
    float2 *stats = (float2 *)(smem + WAVES * 2 * SLOT);  // [WAVES][32]
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
    const Target t = target_of(a, blk, head, blk.rows0 + l32, nsp == 1, split, top, sum);
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

template <typename K>
hipError_t launch(K kernel, const AttnPlan &p, int threads, size_t lds, const AttnArgs &a, hipStream_t s)
{
    const hipError_t e = raise_lds_limit_once((const void *)kernel);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.nsplit * p.nblocks * a.Hkv), dim3(threads), lds, s, a);
    return hipGetLastError();
}

template <int DT, int WAVES, int TS, int TN, bool PAGED>
hipError_t launch_rows(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    return launch(attend_rows<DT, WAVES, TS, TN, PAGED>, p, WAVES * 64, 2 * Elem<DT>::RING * TN * Elem<DT>::ROWB + 16 + (TS == 2 ? WAVES * 32 * sizeof(float2) : 0), a, s);
}

template <int DT, int WAVES, bool PAGED>
hipError_t launch_tokens(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    return launch(attend_tokens<DT, WAVES, PAGED>, p, WAVES * 64, WAVES * (2 * 32 * Elem<DT>::ROWB + 32 * sizeof(float2)), a, s);
}

template <bool PAGED>
hipError_t launch_kernels(const AttnPlan &p, const AttnArgs &a, hipStream_t s)
{
    hipError_t e;
    if (p.dtype == ILRE_BF16) {
        if (p.rows == 32)
            e = launch_tokens<ILRE_BF16, 4, PAGED>(p, a, s);
        else if (p.rows == 128)
            e = launch_rows<ILRE_BF16, 8, 2, 64, PAGED>(p, a, s);
        else
            e = launch_rows<ILRE_BF16, 8, 1, 64, PAGED>(p, a, s);
    } else {
        if (p.rows == 32)
            e = launch_tokens<ILRE_F32, 4, PAGED>(p, a, s);
        else
            e = launch_rows<ILRE_F32, 4, 1, 32, PAGED>(p, a, s);
    }
    if (e != hipSuccess || p.nsplit == 1) return e;
    return p.dtype == ILRE_BF16 ? launch_merge<ILRE_BF16, PAGED>(p, a, s) : launch_merge<ILRE_F32, PAGED>(p, a, s);
}

}  // namespace

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
AttnPlan make_attn_plan(int dtype, int T, int n_seq, int Hq, int Hkv, int max_q, int max_kv, int64_t total_kv, int sink, int window, size_t workspace)
{
    AttnPlan p{};
    p.dtype = dtype;
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
    if (rows <= 32) {
        cut(32, 128);
    } else if (dtype == ILRE_F32) {
        cut(128, 32);
    } else {
        cut(256, 64);
        if (rows <= 128 || ((int64_t)p.nblocks * Hkv < kNumCU && tiles(max_kv) <= 24)) cut(128, 64);
    }
    const int64_t most = std::max<int64_t>(tiles(max_kv), 1);
    const int64_t blocks = std::min<int64_t>(p.nblocks, std::max<int64_t>((int64_t)T * G / p.rows, n_seq));
    const int64_t work = std::max<int64_t>(blocks * Hkv * tiles(total_kv / n_seq), 1);
    const int64_t places = (p.rows == 32) == (dtype == ILRE_BF16) ? 2 * kNumCU : kNumCU;  // what LDS has room for
    const int64_t least = p.rows == 32 ? (most <= 3 ? 3 : work <= kNumCU ? 1 : 2) : dtype == ILRE_F32 ? 2 : (int64_t)T * Hq <= 2048 ? 4 : 12;
    const int64_t per = std::max<int64_t>((work + places - 1) / places, least);
    int64_t n = (most + per - 1) / per;
    const int64_t row_bytes = (int64_t)T * Hq * (kHeadDim + 1) * (int64_t)sizeof(float);
    n = std::max<int64_t>(1, std::min({n, (int64_t)256, (int64_t)(workspace / (size_t)row_bytes), kMaxUnits / std::max<int64_t>(p.nblocks * (int64_t)Hkv, 1)}));
    if ((int64_t)T * Hq > kMaxUnits) n = 1;  // (more rows than a merge is launched for)
    p.nsplit = (int)n;
    p.split_tiles = (int)(n == 1 ? most : std::max(per, (most + n - 1) / n));
    p.bytes = n == 1 ? 0 : (size_t)(n * row_bytes);
    return p;
}

hipError_t launch_attention(const AttnPlan &p, AttnArgs a, void *workspace, hipStream_t s)
{
    a.nsplit = p.nsplit;
    a.split_tiles = p.split_tiles;
    a.nblocks = p.nblocks;
    a.rows = p.rows;
    a.tile = p.tile;
    a.part_o = (float *)workspace;
    a.part_e = a.part_o + (int64_t)p.nsplit * a.T * a.Hq * kHeadDim;
    return a.table ? launch_kernels<true>(p, a, s) : launch_kernels<false>(p, a, s);
}

}  // namespace ilre
