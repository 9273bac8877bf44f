// Norms of queries and keys, their rotation to positions along one axis or several, and the fill of a cache of pages held in 16 (32), 8 or 4 bits, in one pass, for gfx950.
//
//   y = x w / sqrt(mean(x^2) + eps),   (y_1, y_2) -> m (y_1 cos a - y_2 sin a, y_2 cos a + y_1 sin a),   a = position[axis of pair j] * inv_freq[j]
//
// A wavefront has one token.  Lane j makes sine and cosine of pair j, once for all heads of the token, and leaves them in LDS; eight lanes then share a head, each with channels 8u .. 8u + 7
// and 64 + 8u .. 64 + 8u + 7, so that a head's loads and stores are whole, and the 32 channels that share a scale lie with four neighbouring lanes.  A channel is
// r (x A + p B): p the other channel of its pair, A and B its cosine and signed sine times the weights of the two, r the norm.
//
// Queries and caches of the states' own type: fp32 (the angle's fraction of a turn in fp64).  Keys of a quantised cache: fp64 throughout, fp64 sines and cosines too (of angles whose whole turns are
// taken off before any rounding, so that far positions are as good as near ones), and one rounding, to the code.  A
// code's border is met by one key in 2^19 or so if the key itself is off by 2^-24, and then what a cache holds depends on the order of operations of whoever fills it.
//
// Bound: HBM where tokens are many (65539 of 28/4 heads into 8 bits 220 us, 5.2 TB/s), otherwise the chain of loads from cu_q to the page, sines and stores (8 tokens 5.7 us, 1028 of 32/8 heads 9.5).
#include "kv_codes.h"

#include <type_traits>

namespace ilre {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned words4;

constexpr int kThreads = 256;
// Where the other channel of a pair is: with the same lane (half-split pairing over all 128 channels), anywhere (half-split over fewer), next to it.
enum { kSameLane, kElsewhere, kNeighbour };

template <int DT>
struct Eight {  // channels, as they lie in memory
    static constexpr int N = DT == ILRE_BF16 ? 1 : 2;
    uint4 v[N];
    __device__ __forceinline__ void load(const unsigned char *p)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = ((const uint4 *)p)[i];
    }
    __device__ __forceinline__ void store(unsigned char *p) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) ((uint4 *)p)[i] = v[i];
    }
    // What is written is more than the L2s hold: it takes no place there.
    __device__ __forceinline__ void store_past(unsigned char *p) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) __builtin_nontemporal_store(__builtin_bit_cast(words4, v[i]), (words4 *)p + i);
    }
    __device__ __forceinline__ void choose(bool mine, const Eight &o)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = make_uint4(mine ? v[i].x : o.v[i].x, mine ? v[i].y : o.v[i].y, mine ? v[i].z : o.v[i].z, mine ? v[i].w : o.v[i].w);
    }
    // What has been worked out from the channels so far is worked out again, not kept in registers.
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i].x), "+v"(v[i].y), "+v"(v[i].z), "+v"(v[i].w));
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (DT == ILRE_BF16) {
                    f[2 * k] = __uint_as_float(w[k] << 16);
                    f[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
                } else {
                    f[4 * i + k] = __uint_as_float(w[k]);
                }
            }
        }
    }
    __device__ __forceinline__ void put(const float (&f)[8])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = DT == ILRE_BF16 ? __builtin_bit_cast(uint32_t, __builtin_convertvector((kv_f32x2{f[2 * k], f[2 * k + 1]}), kv_bf16x2)) : __float_as_uint(f[4 * i + k]);
            v[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

// What lane l ^ 1, l ^ 2 and (where every four lanes hold the same already) l ^ 4 has.
template <int CTRL>
__device__ __forceinline__ unsigned from_lane(unsigned x)
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kXor4 = 0x141;  // quad permutations 1 0 3 2 and 2 3 0 1; a mirrored half row
template <int CTRL>
__device__ __forceinline__ float from_lane(float x) { return __uint_as_float(from_lane<CTRL>(__float_as_uint(x))); }
template <int CTRL>
__device__ __forceinline__ double from_lane(double x)
{
    const unsigned long long u = (unsigned long long)__double_as_longlong(x);
    const unsigned lo = from_lane<CTRL>((unsigned)u), hi = from_lane<CTRL>((unsigned)(u >> 32));
    return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
// Over a head's eight lanes.
template <typename T>
__device__ __forceinline__ T sum_of_eight(T x)
{
    x += from_lane<kXor1>(x);
    x += from_lane<kXor2>(x);
    return x + from_lane<kXor4>(x);
}

// Sine and cosine of `part` turns, |part| <= 1/2 (or 2^-20 more): to the nearest quarter turn, then the series of both up to x^15 and x^16, whose rests are below 2^-54 for |x| <= pi / 4.
__device__ __forceinline__ void sine_and_cosine(double part, double &s, double &c)
{
    const double quarter = rint(4.0 * part), x = fma(quarter, -0.25, part) * 6.283185307179586476925, y = x * x;
    double p = -1.0 / 1307674368000.0, q = 1.0 / 20922789888000.0;
    p = fma(p, y, 1.0 / 6227020800.0);
    p = fma(p, y, -1.0 / 39916800.0);
    p = fma(p, y, 1.0 / 362880.0);
    p = fma(p, y, -1.0 / 5040.0);
    p = fma(p, y, 1.0 / 120.0);
    p = fma(p, y, -1.0 / 6.0);
    p = fma(p * y, x, x);
    q = fma(q, y, -1.0 / 87178291200.0);
    q = fma(q, y, 1.0 / 479001600.0);
    q = fma(q, y, -1.0 / 3628800.0);
    q = fma(q, y, 1.0 / 40320.0);
    q = fma(q, y, -1.0 / 720.0);
    q = fma(q, y, 1.0 / 24.0);
    q = fma(q, y, -0.5);
    q = fma(q, y, 1.0);
    const int k = (int)quarter;  // -2 .. 2
    s = k & 1 ? q : p;
    c = k & 1 ? p : q;
    if (k & 2) s = -s;
    if ((k + 1) & 2) c = -c;
}

// Where pair j's sine and cosine lie: eight lanes read every eighth pair (every fourth) at a time, from different banks.
__device__ __forceinline__ int spread(int j) { return j + (j >> 3); }

template <int DT, int FMT, int PAIR, int WPT>
__global__ __launch_bounds__(WPT > 4 ? WPT * 64 : kThreads) void fill_kernel(const FillArgs a)
{
    constexpr int WAVES = WPT > 4 ? WPT : kThreads / 64;
    using Real = std::conditional_t<FMT == kPlain, float, double>;  // of keys
    struct Turn {
        float c, s;  // cosine and sine, times the magnitude
    };
    struct KeyTurn {
        Real c, s;
    };
    constexpr int ES = DT == ILRE_BF16 ? 2 : 4;
    __shared__ Turn wheels[WAVES][ILRE_HEAD_DIM / 2 + 8];
    __shared__ KeyTurn key_wheels[FMT == kPlain ? 1 : WAVES][FMT == kPlain ? 1 : ILRE_HEAD_DIM / 2 + 8];
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int token = (int)blockIdx.x * (WAVES / WPT) + wave / WPT;
    if (token >= a.T) return;
    const int u = lane & 7, slot = lane >> 3;
    Turn *wheel = wheels[wave];
    KeyTurn *key_wheel = key_wheels[FMT == kPlain ? 0 : wave];

    // of the lane's two runs of eight channels: where they begin, whether they are turned, their pairs, and where the others of these begin
    const int half = a.rotary / 2;
    int from[2], pair[2], other[2];
    bool turned[2], first[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        from[s] = 64 * s + 8 * u;
        turned[s] = PAIR == kSameLane || from[s] < a.rotary;
        first[s] = PAIR == kSameLane ? s == 0 : from[s] < half;
        pair[s] = PAIR == kNeighbour ? from[s] / 2 : first[s] ? from[s] : from[s] - half;
        other[s] = !turned[s] ? from[s] : first[s] ? from[s] + half : from[s] - half;
    }
    // A head's channels, and the others of their pairs; likewise their weights.
    struct Head {
        Eight<DT> x[2], p[2];
    };
    auto fetch = [&](Head &h, const unsigned char *at) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            h.x[s].load(at + from[s] * ES);
            if (PAIR == kElsewhere) h.p[s].load(at + other[s] * ES);
        }
    };
    // Queries eight heads at a time, then keys and values as one list of heads; WPT wavefronts take turns.  What the first of a wavefront's steps needs is asked for at once, before it is
    // known where the token stands, and each step's heads a step ahead.
    const int nq = a.q ? a.Hq : 0, nk = a.k ? a.Hkv : 0, nv = a.v ? a.Hkv : 0;
    const int steps_q = (nq + 7) / 8, steps = steps_q + (nk + nv + 7) / 8;
    auto fetch_step = [&](Head &h, int step) {
        if (step >= steps) return;
        if (step < steps_q) {
            fetch(h, a.q + (int64_t)token * a.q_token + min(step * 8 + slot, nq - 1) * a.q_head);
        } else {
            const int at = min((step - steps_q) * 8 + slot, nk + nv - 1);
            fetch(h, at < nk ? a.k + (int64_t)token * a.k_token + at * a.k_head : a.v + (int64_t)token * a.v_token + (at - nk) * a.v_head);
        }
    };
    int step = wave % WPT;
    Head head, weight;
    fetch_step(head, step);
    auto fetch_weights = [&](bool norm, const unsigned char *w) {
        if (norm && w) fetch(weight, w);
    };
    const bool queries = step < steps_q;
    fetch_weights(queries ? a.q_norm : a.k_norm, queries ? a.q_weight : a.k_weight);
    const double turns = lane < half ? a.turns[lane] : 0.0, turns_rest = lane < half ? a.turns_rest[lane] : 0.0;
    const int position = a.positions && lane < half ? a.positions[(int64_t)a.axes[lane] * a.T + token] : 0;

    // the token's place in its sequence, and where that is in the cache
    double place = (double)a.first_position + token;
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
            if ((unsigned)page < (unsigned)a.num_pages) cell = page * a.page + (at & (((int64_t)1 << a.page_shift) - 1)) * a.token;
        }
    }
    if (a.positions) place = position;
    if (lane < half) {
        const double part = fma(place, turns, -rint(place * turns)) + place * turns_rest;
        if (FMT == kPlain) {
            const float upper = (float)part, lower = (float)(part - upper) * 6.283185307f, m = (float)a.magnitude;
            float s, c;
            sincospif(2.0f * upper, &s, &c);
            wheel[spread(lane)].s = fmaf(c, lower, s) * m;
            wheel[spread(lane)].c = fmaf(-s, lower, c) * m;
        } else {
            double s, c;
            sine_and_cosine(part, s, c);
            s *= a.magnitude;
            c *= a.magnitude;
            key_wheel[spread(lane)] = KeyTurn{(Real)c, (Real)s};
            wheel[spread(lane)] = Turn{(float)c, (float)s};
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();

    // Channel e of run s: its pair's cosine and sine (with the sign that its part takes); what is not turned is multiplied with one and added to minus zero, which changes nothing.
    auto turn_of = [&](auto *wheels, int s, int e) {
        const int j = (pair[s] + (PAIR == kNeighbour ? e / 2 : e)) & 63;
        auto t = wheels[spread(j)];
        if (PAIR == kNeighbour ? !(e & 1) : first[s]) t.s = -t.s;
        if (!turned[s]) t.c = 1, t.s = -(t.c * 0);
        return t;
    };
    // The other channels of the pairs of run s (where it is turned), of states or weights.
    auto other_channels = [&](const Head &h, int s, float (&p)[8]) {
        if (PAIR == kSameLane) {
            h.x[1 - s].get(p);
        } else if (PAIR == kElsewhere) {
            h.p[s].get(p);
        } else {
            float x[8];
            h.x[s].get(x);
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = x[e ^ 1];
        }
    };
    // 1 / sqrt(mean + eps) of a head, the same for its eight lanes
    auto norm32 = [&](const float (&x)[2][8]) {
        float sum = 0.f;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[s][e], x[s][e], sum);
        return rsqrtf(sum_of_eight(sum) * (1.f / ILRE_HEAD_DIM) + (float)a.eps);
    };
    auto norm64 = [&](const float (&x)[2][8]) {
        double sum = 0.0;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fma((double)x[s][e], (double)x[s][e], sum);
        return 1.0 / sqrt(sum_of_eight(sum) * (1.0 / ILRE_HEAD_DIM) + a.eps);
    };
    // fp32: coefficients of the token's heads, and a head turned
    float A[2][8], B[2][8];
    auto coefficients = [&](bool norm, const unsigned char *w) {
        const bool there = norm && w;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            float own[8], others[8];
            weight.x[s].get(own);
            other_channels(weight, s, others);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const Turn t = turn_of(wheel, s, e);
                A[s][e] = (there ? own[e] + a.offset : 1.f) * t.c;
                B[s][e] = turned[s] ? (there ? others[e] + a.offset : 1.f) * t.s : -0.f;
            }
        }
    };
    auto turn32 = [&](Head &h, bool norm) {
        float x[2][8], p[2][8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            h.x[s].get(x[s]);
            other_channels(h, s, p[s]);
        }
        const float r = norm ? norm32(x) : 1.f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float q = turned[s] ? p[s][e] : 0.f;  // (an infinity where nothing is turned would not stay out)
                x[s][e] = fmaf(x[s][e], A[s][e], q * B[s][e]) * r;
            }
            h.x[s].put(x[s]);
        }
    };

    if (queries) coefficients(a.q_norm, a.q_weight);
    for (; step < steps_q; step += WPT) {
        Head x = head;
        fetch_step(head, step + WPT);
        turn32(x, a.q_norm);
        const int h = step * 8 + slot;
        if (h < nq) {
            unsigned char *to = a.q_out + (int64_t)token * a.out_token + h * a.out_head;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (WPT == 1)
                    x.x[s].store_past(to + from[s] * ES);
                else
                    x.x[s].store(to + from[s] * ES);
            }
        }
    }
    if (step >= steps || cell < 0) return;
    if (queries) fetch_weights(a.k_norm, a.k_weight);
    if (FMT == kPlain) coefficients(a.k_norm, a.k_weight);
    for (; step < steps; step += WPT) {
        const int h = (step - steps_q) * 8 + slot;
        const bool key = h < nk;
        Head x = head;
        fetch_step(head, step + WPT);
        const int64_t to = cell + (key ? h : h - nk) * a.head;
        if (FMT == kPlain) {
            Head y = x;
            turn32(y, a.k_norm);
            if (h < nk + nv) {
                unsigned char *p = (key ? a.k_pages : a.v_pages) + to * ES;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    y.x[s].choose(key, x.x[s]);
                    y.x[s].store(p + from[s] * ES);
                }
            }
            continue;
        }
        const bool keys = __ballot(key);
        double r = 1.0;
        if (keys && a.k_norm) {
            float f[2][8];
#pragma unroll
            for (int s = 0; s < 2; ++s) x.x[s].get(f[s]);
            r = norm64(f);
        }
        const bool weighted = a.k_norm && a.k_weight;
        auto weight64 = [&](float w) { return weighted ? (double)w + a.offset : 1.0; };
        float y[2][8];
        if (PAIR == kSameLane && keys) {  // both channels of a pair at once
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float f[2][8], w[2][8];
#pragma unroll
                for (int s = 0; s < 2; ++s) x.x[s].get(f[s]), weight.x[s].get(w[s]);
                const KeyTurn t = turn_of(key_wheel, 1, e);
                const double m = f[0][e] * weight64(w[0][e]) * r, n = f[1][e] * weight64(w[1][e]) * r;
                y[0][e] = cut_off(m * t.c - n * t.s);
                y[1][e] = cut_off(n * t.c + m * t.s);
                if (e == 3) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int s = 0; s < 2; ++s) x.x[s].forget(), weight.x[s].forget();
                }
            }
        }
        auto run = [&](auto number) {  // eight channels
            constexpr int s = number.value;
            float f[8];
            x.x[s].get(f);
            if (PAIR == kSameLane) {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = key ? y[s][e] : f[e];
            } else if (keys) {
                float p[8], own[8], others[8];
                other_channels(x, s, p);
                weight.x[s].get(own);
                other_channels(weight, s, others);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const KeyTurn t = turn_of(key_wheel, s, e);
                    const float q = turned[s] ? p[e] : 0.f;
                    const float z = cut_off((f[e] * weight64(own[e]) * t.c + q * weight64(others[e]) * t.s) * r);
                    f[e] = key ? z : f[e];
                }
            }
            unsigned top = 0;  // the largest magnitude, as bits: a NaN's are larger than any number's
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7FFFFFFFu);
            top = max(top, from_lane<kXor1>(top));
            top = max(top, from_lane<kXor2>(top));
            const unsigned byte = scale_byte<FMT == kPlain ? ILRE_KV_FP8 : FMT>(__uint_as_float(top));
            const float inv = inverse_scale(byte);
            const int64_t channel = to + from[s];
            if (h >= nk + nv) return;
            unsigned char *codes = (key ? a.k_pages : a.v_pages) + (FMT == ILRE_KV_FP8 ? channel : channel / 2);
            if (FMT == ILRE_KV_FP8)
                *(uint2 *)codes = byte == 255 ? make_uint2(0, 0) : to_fp8(f, inv);
            else
                *(unsigned *)codes = byte == 255 ? 0 : to_fp4(f, inv);
            if ((u & 3) == 0) (key ? a.k_scales : a.v_scales)[channel / ILRE_KV_BLOCK] = (unsigned char)byte;
        };
        // (both at once, or numbers in fp64 and sines and cosines kept from one for the other, would take registers that a fourth wavefront can have)
        auto forget = [&]() {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                x.x[s].forget();
                weight.x[s].forget();
                if (PAIR == kElsewhere) x.p[s].forget(), weight.p[s].forget();
            }
            asm volatile("" : "+v"(pair[1]));
        };
        forget();
        run(std::integral_constant<int, 0>{});
        forget();
        run(std::integral_constant<int, 1>{});
    }
}

template <int DT, int FMT, int PAIR>
hipError_t launch(const FillArgs &a, hipStream_t s)
{
    // A token's heads go to several wavefronts while there are not tokens for all of them: eight up to 512 tokens (32/8 heads, 8 bits; a step of 8 heads each: 8 tokens 6.4 -> 5.4 us, 512 8.5 -> 7.9,
    // but 1028 12.2 -> 15.8), four up to a few thousand; many tokens have one each, so that sines and weights are worked out once.  Their queries, and what is read back of
    // many, are written past the L2s (65539 tokens of 28/4 heads stored in 8 bits and read back 271 -> 256 us, a million keys read back 607 -> 568).
    const int wavefronts = fill_wavefronts(a.T);
    if (wavefronts == 8)
        hipLaunchKernelGGL((fill_kernel<DT, FMT, PAIR, 8>), dim3((unsigned)a.T), dim3(512), 0, s, a);
    else if (wavefronts == 4)
        hipLaunchKernelGGL((fill_kernel<DT, FMT, PAIR, 4>), dim3((unsigned)a.T), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((fill_kernel<DT, FMT, PAIR, 1>), dim3((unsigned)((a.T + 3) / 4)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <int DT, int FMT>
hipError_t launch_pairing(const FillArgs &a, int pairing, hipStream_t s)
{
    if (pairing == ILRE_ROPE_INTERLEAVED) return launch<DT, FMT, kNeighbour>(a, s);
    return a.rotary == ILRE_HEAD_DIM ? launch<DT, FMT, kSameLane>(a, s) : launch<DT, FMT, kElsewhere>(a, s);
}

template <int DT>
hipError_t launch_format(const FillArgs &a, int format, int pairing, hipStream_t s)
{
    return format == ILRE_KV_FP8   ? launch_pairing<DT, ILRE_KV_FP8>(a, pairing, s)
           : format == ILRE_KV_FP4 ? launch_pairing<DT, ILRE_KV_FP4>(a, pairing, s)
                                   : launch_pairing<DT, kPlain>(a, pairing, s);
}

// ------------------------------------------------------------------------------------------------ reading a cache back

// Rows (token, head) with eight lanes each, which have the channels that they have above; ITEMS rows a lane, whose loads are under way together.  One pass, HBM: a million keys of 8 kv heads
// out of 8 bits 568 us, 5.5 TB/s.
template <int DT, int FMT, int ITEMS>
__global__ __launch_bounds__(kThreads) void read_kernel(const ReadArgs a, int rows_first)
{
    constexpr int ES = DT == ILRE_BF16 ? 2 : 4;
    const int lane = threadIdx.x & 63, u = lane & 7;
    const unsigned items = (unsigned)a.T * a.Hkv, first = blockIdx.x * (kThreads / 8 * ITEMS) + (threadIdx.x >> 6) * (8 * ITEMS) + (lane >> 3);  // (2^30 at most)
    int row[ITEMS], head[ITEMS];
    bool real[ITEMS];
    int64_t cell[ITEMS];  // -1: zeros
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {  // rows or heads running fastest
        const unsigned item = min(first + 8 * k, items - 1), by = rows_first ? a.T : a.Hkv, quotient = item / by, rest = item - quotient * by;
        real[k] = first + 8 * k < items;
        row[k] = (int)(rows_first ? rest : quotient);
        head[k] = (int)(rows_first ? quotient : rest);
    }
    int token[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) token[k] = a.tokens ? a.tokens[row[k]] : 0;
    // The rows' sequences: the wavefront looks for its first row's; the others look on from there, or from the beginning where the next head's rows begin.
    const int lowest = __builtin_amdgcn_readfirstlane(row[0]);
    int begin = a.n_seq;
    for (int base = 0; base < a.n_seq; base += 64) {
        const int s = base + lane;
        const unsigned long long past = __ballot(s < a.n_seq && a.cu_q[s + 1] > lowest);
        if (past) {
            begin = base + __builtin_ctzll(past);
            break;
        }
    }
    int seq = begin, seen = lowest;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        if (row[k] < seen) seq = 0;
        seen = row[k];
        while (seq < a.n_seq && a.cu_q[seq + 1] <= row[k]) ++seq;
        cell[k] = -1;
        const int r0 = seq < a.n_seq ? max(a.cu_q[seq], 0) : 0x7FFFFFFF;
        real[k] = real[k] && row[k] >= r0;  // otherwise a row of no sequence
        if (!real[k]) continue;
        const int r1 = min(a.cu_q[seq + 1], a.T), len = a.kv_len[seq];
        const int64_t at = a.tokens ? (int64_t)token[k] : (int64_t)len - (r1 - r0) + (row[k] - r0);
        if (at < 0 || at >= min((int64_t)len, a.kv_limit)) continue;
        const int page = a.table[seq * a.table_stride + (at >> a.page_shift)];
        if ((unsigned)page < (unsigned)a.num_pages) cell[k] = page * a.page + (at & (((int64_t)1 << a.page_shift) - 1)) * a.token + head[k] * a.head;
    }
    // Codes and scales of a run of eight channels, all zeros where there is nothing to read.
    struct Run {
        Eight<DT> x;
        uint2 codes;
        unsigned byte;
    };
    auto fetch = [&](Run &r, const unsigned char *pages, const unsigned char *scales, int64_t at) {
        r.x.zero();
        r.codes = make_uint2(0, 0);
        r.byte = 0;
        if (at < 0) return;
        if (FMT == kPlain) {
            r.x.load(pages + at * ES);
            return;
        }
        r.byte = scales[at / ILRE_KV_BLOCK];
        if (FMT == ILRE_KV_FP8)
            r.codes = *(const uint2 *)(pages + at);
        else
            r.codes.x = *(const unsigned *)(pages + at / 2);
    };
    auto store = [&](Run &r, unsigned char *to) {
        if constexpr (FMT != kPlain) {
            const float scale = r.byte == 255 ? __uint_as_float(0x7FC00000u) : scale_of(r.byte);
            float f[8];
            if constexpr (FMT == ILRE_KV_FP8) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const unsigned c = k ? r.codes.y : r.codes.x;
                    const float2 x = f32_pair<FMT, 0>(c, 1.f), z = f32_pair<FMT, 1>(c, 1.f);
                    f[4 * k] = x.x * scale, f[4 * k + 1] = x.y * scale, f[4 * k + 2] = z.x * scale, f[4 * k + 3] = z.y * scale;
                }
            } else {
                const unsigned c = r.codes.x;
                const float2 x[4] = {f32_pair<FMT, 0>(c, 1.f), f32_pair<FMT, 1>(c, 1.f), f32_pair<FMT, 2>(c, 1.f), f32_pair<FMT, 3>(c, 1.f)};
#pragma unroll
                for (int k = 0; k < 4; ++k) f[2 * k] = x[k].x * scale, f[2 * k + 1] = x[k].y * scale;
            }
            r.x.put(f);
        }
        if (ITEMS > 1)
            r.x.store_past(to);
        else
            r.x.store(to);
    };
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        unsigned char *out = t ? a.v_out : a.k_out;
        if (!out) continue;
        const unsigned char *pages = t ? a.v_pages : a.k_pages, *scales = t ? a.v_scales : a.k_scales;
        const int64_t out_token = t ? a.v_token : a.k_token, out_head = t ? a.v_head : a.k_head;
        Run r[ITEMS][2];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int s = 0; s < 2; ++s) fetch(r[k][s], pages, scales, cell[k] < 0 ? -1 : cell[k] + 64 * s + 8 * u);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (real[k]) store(r[k][s], out + row[k] * out_token + head[k] * out_head + (64 * s + 8 * u) * ES);
    }
}

template <int DT, int FMT>
hipError_t launch_read_items(const ReadArgs &a, hipStream_t s)
{
    const int64_t items = (int64_t)a.T * a.Hkv;
    const int rows_first = a.k_out ? a.k_token < a.k_head : a.v_token < a.v_head;
    const int64_t each = kThreads / 8;
    // Four rows a lane where there are many, one where what counts is how soon the first arrive (8 kv heads: 4100 tokens 10.4 -> 8.0 us with one, 16000 25.0 -> 24.4, 131072 158 -> 162, a
    // million's keys 568, with one row 854).
    if (read_rows(items) == 1)
        hipLaunchKernelGGL((read_kernel<DT, FMT, 1>), dim3((unsigned)((items + each - 1) / each)), dim3(kThreads), 0, s, a, rows_first);
    else
        hipLaunchKernelGGL((read_kernel<DT, FMT, 4>), dim3((unsigned)((items + 4 * each - 1) / (4 * each))), dim3(kThreads), 0, s, a, rows_first);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_read_format(const ReadArgs &a, int format, hipStream_t s)
{
    return format == ILRE_KV_FP8   ? launch_read_items<DT, ILRE_KV_FP8>(a, s)
           : format == ILRE_KV_FP4 ? launch_read_items<DT, ILRE_KV_FP4>(a, s)
                                   : launch_read_items<DT, kPlain>(a, s);
}

}  // namespace

hipError_t launch_fill(const FillArgs &a, int dtype, int format, int pairing, hipStream_t s)
{
    return dtype == ILRE_BF16 ? launch_format<ILRE_BF16>(a, format, pairing, s) : launch_format<ILRE_F32>(a, format, pairing, s);
}

hipError_t launch_read(const ReadArgs &a, int dtype, int format, hipStream_t s)
{
    return dtype == ILRE_BF16 ? launch_read_format<ILRE_BF16>(a, format, s) : launch_read_format<ILRE_F32>(a, format, s);
}

}  // namespace ilre
