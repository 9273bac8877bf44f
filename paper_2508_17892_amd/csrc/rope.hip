// Rotary positions of new tokens, with the fill of a paged cache, for gfx950.
//
//   (x, y) -> m (x cos a - y sin a, y cos a + x sin a),  a = position * inv_freq[j] for pair j of the first `rotary` channels
//
// One pass: every element is read once and written once, 16 bytes an access.  A head is eight units of two 16-byte chunks (fp32: sixteen), a thread has one unit of
// a token's heads, one head after the other, so that its few sines and cosines are made once.  A unit holds whole pairs: chunks u and u + rotary / 16 of the
// half-split pairing, chunks 2u and 2u + 1 of the interleaved one; the channels behind `rotary` are units that are copied.
//
// The angle is reduced in turns in fp64 (position * inv_freq / 2 pi reaches 10^5 turns at a million positions, and its fraction is all that counts), then
// sine and cosine of the fraction are fp32: of its upper 24 bits, and the rest of it, 2^-26 of a turn at most, by the first term of the addition theorem, so that small sines
// and cosines keep their bits too.
#include "ilre_internal.h"

namespace ilre {
namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kThreads = 256;

template <int DT>
struct Chunk;  // 16 bytes as floats
template <>
struct Chunk<ILRE_BF16> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void get(const uint4 &v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ uint4 put(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{f[2 * i], f[2 * i + 1]}), bf16x2));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Chunk<ILRE_F32> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void get(const uint4 &v, float (&f)[4])
    {
        f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 put(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

// A wavefront has one token.  WPT wavefronts share a token's heads.
template <int DT, int PAIRING, int WPT>
__global__ __launch_bounds__(kThreads) void turn_kernel(const TurnArgs a)
{
    using C = Chunk<DT>;
    constexpr int E = C::E, UNITS = ILRE_HEAD_DIM / (2 * E), AT_ONCE = 64 / UNITS * WPT;  // heads at a time
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int token = (int)blockIdx.x * (kThreads / 64 / WPT) + wave / WPT;
    if (token >= a.T) return;
    const int u = lane % UNITS, first = lane / UNITS + wave % WPT * (64 / UNITS);

    const int turned = a.rotary / (2 * E);  // units
    const bool turn = u < turned;
    // byte offsets of the unit's two chunks
    int c0, c1;
    if (PAIRING == ILRE_ROPE_HALF && turn) {
        c0 = u * 16;
        c1 = (u + turned) * 16;
    } else {
        c0 = 2 * u * 16;
        c1 = c0 + 16;
    }
    // queries, keys and values as one list of heads
    const int nq = a.q ? a.Hq : 0, nk = a.k ? a.Hkv : 0, nv = a.v ? a.Hkv : 0, n = nq + nk + nv;
    auto from = [&](int h) -> const unsigned char * {
        return h < nq ? a.q + token * a.q_token + h * a.q_head : h < nq + nk ? a.k + token * a.k_token + (h - nq) * a.k_head : a.v + token * a.v_token + (h - nq - nk) * a.v_head;
    };
    constexpr int AHEAD = 4;
    uint4 x[AHEAD], y[AHEAD];
    auto fetch = [&](int h0) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int h = h0 + i * AT_ONCE;
            if (h < n) {
                const unsigned char *p = from(h);
                x[i] = *(const uint4 *)(p + c0);
                y[i] = *(const uint4 *)(p + c1);
            }
        }
    };
    if (WPT > 1) fetch(first);  // on their way while the token's place and angles are worked out

    // the token's place in its sequence, and where that is in the cache
    double place = (double)a.first_position + token;  // (their sum may not fit 32 bits)
    int64_t cell = -1;
    if (a.cu_q) {
        int seq = -1;
        for (int base = 0; base < a.n_seq; base += 64) {
            const int s = base + lane;
            const unsigned long long past = __ballot(s < a.n_seq && a.cu_q[s + 1] > token);
            if (past) {
                seq = __builtin_amdgcn_readfirstlane(base + __builtin_ctzll(past));
                break;
            }
        }
        if (seq < 0) return;  // a token of no sequence
        const int q0 = max(a.cu_q[seq], 0), q1 = min(a.cu_q[seq + 1], a.T);
        if (token < q0) return;
        const int64_t at = (int64_t)a.kv_len[seq] - (q1 - q0) + (token - q0);
        place = (double)at;
        if (at >= 0 && at < a.kv_limit) {
            const int page = a.table[seq * a.table_stride + (at >> a.page_shift)];
            if ((unsigned)page < (unsigned)a.num_pages) cell = page * a.page_bytes + (at & (((int64_t)1 << a.page_shift) - 1)) * a.token_bytes;
        }
    }
    if (a.positions) place = a.positions[token];

    float co[E], si[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const double n = place * a.turns[turn ? u * E + e : 0];
        const double part = n - rint(n);
        const float upper = (float)part, lower = (float)(part - upper) * 6.283185307f;
        float s, c;
        sincospif(2.0f * upper, &s, &c);
        si[e] = fmaf(c, lower, s) * a.magnitude;
        co[e] = fmaf(-s, lower, c) * a.magnitude;
    }
    auto turned_unit = [&](uint4 &x, uint4 &y) {
        float f[E], g[E];
        C::get(x, f);
        C::get(y, g);
        if (PAIRING == ILRE_ROPE_HALF) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float t = f[e] * co[e] - g[e] * si[e];
                g[e] = g[e] * co[e] + f[e] * si[e];
                f[e] = t;
            }
        } else {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                const float t = f[2 * e] * co[e] - f[2 * e + 1] * si[e], r = g[2 * e] * co[E / 2 + e] - g[2 * e + 1] * si[E / 2 + e];
                f[2 * e + 1] = f[2 * e + 1] * co[e] + f[2 * e] * si[e];
                g[2 * e + 1] = g[2 * e + 1] * co[E / 2 + e] + g[2 * e] * si[E / 2 + e];
                f[2 * e] = t;
                g[2 * e] = r;
            }
        }
        x = C::put(f);
        y = C::put(g);
    };
    auto to = [&](int h) -> unsigned char * {
        return h < nq ? a.q_out + token * a.out_token + h * a.out_head
                      : h < nq + nk ? a.k_pages + cell + (h - nq) * a.head_bytes : a.v_pages + cell + (h - nq - nk) * a.head_bytes;
    };
    for (int h0 = first; h0 < n; h0 += AT_ONCE * AHEAD) {
        if (WPT == 1 || h0 != first) fetch(h0);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int h = h0 + i * AT_ONCE;
            if (h < nq || (h < n && cell >= 0)) {
                if (turn && h < nq + nk) turned_unit(x[i], y[i]);
                unsigned char *p = to(h);
                *(uint4 *)(p + c0) = x[i];
                *(uint4 *)(p + c1) = y[i];
            }
        }
    }
}

template <int DT, int PAIRING>
hipError_t launch(const TurnArgs &a, hipStream_t s)
{
    // Up to a few thousand tokens four wavefronts share a token, for the latency (1028 tokens, 32/8 heads 9.5 -> 8.8 us); many tokens have one each, so that
    // the angles are worked out once (65539 tokens, 28/4 heads 333 -> 223 us).
    if (a.T < 4096)
        hipLaunchKernelGGL((turn_kernel<DT, PAIRING, 4>), dim3((unsigned)a.T), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((turn_kernel<DT, PAIRING, 1>), dim3((unsigned)((a.T + 3) / 4)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_turn(const TurnArgs &a, int dtype, int pairing, hipStream_t s)
{
    if (dtype == ILRE_BF16)
        return pairing == ILRE_ROPE_HALF ? launch<ILRE_BF16, ILRE_ROPE_HALF>(a, s) : launch<ILRE_BF16, ILRE_ROPE_INTERLEAVED>(a, s);
    return pairing == ILRE_ROPE_HALF ? launch<ILRE_F32, ILRE_ROPE_HALF>(a, s) : launch<ILRE_F32, ILRE_ROPE_INTERLEAVED>(a, s);
}

}  // namespace ilre
