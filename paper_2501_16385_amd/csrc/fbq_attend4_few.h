// Attention of a few query rows against a long row of a cache in 4 bits: the work of fbq_attend_few.h (its items, pieces and join) over codes.
//
// Codes go into the matrix cores as they are, fp16 numbers below the normal ones (fbq_cache4.h), and are multiplied exactly; scales come in afterwards, in 32 bits.
//   scores   k = m + s c of a key's group:  q . k = sum over groups of  s (q . c) + m sum(q).  Queries are fp16 here, times a power of two for the row (which goes into its scale): the row's
//            largest feature is near 2^15, and those of codes at high bits are divided by 16, so that only what is 2^-24 of the largest and less loses any.  Scores of
//            bf16 are summed as 2^-24 of them: no number of the type takes such a sum beyond fp32.
//   results  sum p v = sum (p s) (c - 8) + sum p (m + 8 s):  p s is operand B of the second product, a rounding to fp16 where fbq_attend_few.h rounds p; the 8 is a product of its own with the
//            rounded numbers, and the second sum stays in 32 bits, in the lane.  (Without the 8 the rounding is that of numbers three times as large, which add up to the same: relative L2
//            against 64 bits 5.4e-4 instead of 3e-4 for 1000 keys in fp16.)  p s has to be in fp16's range whatever the scales: p is relative to 2^e too, e the exponent of the largest 2^10 s
//            so far, less 5, and follows when it is passed by 2^7.  Of bf16, where that could be an exponent that p itself has no room for, e stays within -24 .. 34 - at 34 no sum of p m or
//            p s over 2^24 tokens passes fp32's range - and what is beyond, x, is taken from the scales while they are spread.
//   scales   A key's scale is wanted in all 16 lanes that have its row of a product.  The matrix cores, which have time, put it there: the scale words as operand A, [key][group] with m and s as
//            neighbours, times constants as operand B are s, m + 8 s, and, with the sums of q in three parts of 16 bits each, m sum(q) - in 32 bits, exactly but for the last addition.
//            (Vector instructions instead, neighbours' words by quad_perm: 350 a step, 100 of them for this, and 5.2 TB/s where it is now 5.9.)
// Bound by HBM in long rows: 16 rows of 16000 tokens, 32 heads of 128, 1.18 GB, 200 us (5.9 TB/s), 64 of 4096 with 64 heads to 8 62; in short ones by the time that begins and ends a piece, 8.5 us with one
// step of 32 keys and nothing to join: 16 rows of about 1000 (74 MB) 25 us, one of 65537 with 8 heads (75 MB) 25.
// A value that a row does not see has weight zero there and finite scales, so nothing of it is added.  But rows share e, and what some of them see and others do not may take bits of the others' p s:
// where such scales are more than 2^4 times what all see, the wave does its work again, slowly, with an e and x for each row by the scales that it sees.  (4 tokens of 32 heads to 8 behind
// 4000, the last one's values 10^4 times the others': 22 us, else 16.)
#ifndef FBQ_ATTEND4_FEW_H
#define FBQ_ATTEND4_FEW_H

#include <algorithm>
#include <type_traits>

#include "fbq_attend_codes.h"
#include "fbq_attend_few.h"
#include "fbq_cache4.h"

namespace fbq {

constexpr int kFew4Parts = kFewTile / 16;                     // of a step, 16 keys each

template <int NW>
struct Step4 {
    static constexpr int kParts = kFew4Parts;
    uint32_t k[kParts][NW], v[kParts][NW];
    uint32_t ks[kParts], vs[kParts];                          // scale word of key l % 16 and group l / 16
};

template <int NW>
struct Piece4 {
    int b, h, step, steps, limit, n, key0, t, sees;           // as in Piece
    word4_t q[NW];
    int pages[kFew4Parts];                                    // of its first step
};

// The queries of a wave's 16 rows: operands for codes, of a group those at low bits and those at high bits; for scale words, what makes s of a group and m sum(q) of all, 2^10 and 2^-14 of them,
// or 1 and 2^-24; and what scores are to be multiplied by.
template <class TY, class NT, int NW>
struct Queries4 {
    static constexpr int G = groups4(32 * NW);
    word4_t at[G][2], sums;
    word2_t pick[G];
    float unit;

    // q: the words of features 32 w + 8 (lane / 16) .., of the lane's row
    __device__ __forceinline__ void of(const word4_t (&q)[NW], float scale)
    {
        float most = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
            for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(fabsf(NT::of(q[w][e] & 0xffff)), fabsf(NT::of_upper(q[w][e]))));
        const int up = __builtin_amdgcn_frexp_expf(larger_of_32(larger_of_16(most))) - 15;
        const int less = NT::kWide && up <= 96 ? 10 : 0;      // (above, with features of 2^110 and more, the unit itself would be beyond fp32)
        unit = ldexpf(scale * 0x1p14f, up + less);
        word4_t h[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int by = e < 2 ? -up : -up - 4;
                h[w][e] = TypeF16::pack(ldexpf(NT::of(q[w][e] & 0xffff), by), ldexpf(NT::of_upper(q[w][e]), by));
            }
        const word4_t one{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u}, sixteen{0x4c004c00u, 0x4c004c00u, 0x4c004c00u, 0x4c004c00u};
        const int grp = (threadIdx.x & 63) >> 4;
        float sum = 0;                                        // of group l / 16
#pragma unroll
        for (int y = 0; y < G; ++y) {
            const word4_t a = h[2 * y], b = 2 * y + 1 < NW ? h[std::min(2 * y + 1, NW - 1)] : word4_t{0, 0, 0, 0};
            at[y][0] = word4_t{a[0], a[1], b[0], b[1]};
            at[y][1] = word4_t{a[2], a[3], b[2], b[3]};
            const float4_t s = TypeF16::mfma(sixteen, at[y][1], TypeF16::mfma(one, at[y][0], float4_t{0, 0, 0, 0}));
            sum = grp == y ? s[0] * 0x1p-14f : sum;
            pick[y] = word2_t{grp == y ? NT::bits(less ? 1.0f : 1024.0f) << 16 : 0u, 0u};
        }
        sum = ldexpf(sum, -less);
        const uint32_t high = NT::bits(sum);
        const float rest = sum - NT::of(high);
        const uint32_t middle = NT::bits(rest);
        sums = word4_t{high, middle, NT::bits(rest - NT::of(middle)), 0u};
    }
};

// Of 16 keys, a lane's four (4 (l / 16) + i): of their scale words in a group what `pick` makes.
template <class TY>
__device__ __forceinline__ float4_t scales_of(uint32_t words, word2_t pick) { return TY::mfma(word2_t{words, 0u}, pick, float4_t{0, 0, 0, 0}); }

// Scores of 16 keys, 1 / unit of them: keys 4 (l / 16) + i in z[i], the lane's query row.
template <class TY, class NT, int NW>
__device__ __forceinline__ float4_t scores4(const uint32_t (&k)[NW], uint32_t ks, const Queries4<TY, NT, NW> &q)
{
    constexpr int G = groups4(32 * NW);
    float4_t z = TY::mfma(word4_t{ks, ks, ks, 0u}, q.sums, float4_t{0, 0, 0, 0});
#pragma unroll
    for (int y = 0; y < G; ++y) {
        const uint32_t a = k[2 * y], b = 2 * y + 1 < NW ? k[std::min(2 * y + 1, NW - 1)] : 0;
        const float4_t low = TypeF16::mfma(word4_t{a & kLowCodes, a >> 8 & kLowCodes, b & kLowCodes, b >> 8 & kLowCodes}, q.at[y][0], float4_t{0, 0, 0, 0});
        const float4_t all = TypeF16::mfma(word4_t{a & kHighCodes, a >> 8 & kHighCodes, b & kHighCodes, b >> 8 & kHighCodes}, q.at[y][1], low);
        const float4_t s = scales_of<TY>(ks, q.pick[y]);
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = __builtin_fmaf(s[i], all[i], z[i]);
    }
    return z;
}

// Bytes of LDS (aligned to 16) of a block of it: parts of waves 1 .., and a word a wave.
template <int NW>
constexpr int kFew4PartsRoom = (kFewWaves - 1) * (2 * 4 * NW + 2) * 256;
template <int NW>
constexpr int kFew4Room = kFew4PartsRoom<NW> + 4 * kFewWaves;

// The work of the block's wave (see attend4_few), its results written; AGAIN: with exponents for each row.  Whether it has to be done so (for all waves of a block that join theirs the same answer).
// TY: the type of queries and results; NT: its numbers.
template <class TY, class NT, int NW, bool AGAIN>
__device__ __forceinline__ bool attend4_few_wave(const AttendArgs &a, int block, unsigned char *room)
{
    constexpr int DS = 32 * NW, G = groups4(DS), J = 2 * NW;   // products of the results
    constexpr int kParts = kFew4Parts;
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const int worker = uniform(block * kFewWaves + (threadIdx.x >> 6));
    const int D = a.D, ps1 = (1 << a.log_ps) - 1;
    const int member = col % a.group;
    const long head_bytes = (a.page_bytes >> 1) / a.kv_heads;

    Piece4<NW> cur, behind;
    FewLine line;
    if (!line.first(a, block, worker, cur)) return false;
    const bool together = line.together;
    auto prepare = [&](Piece4<NW> &x) __attribute__((always_inline)) {
        few_sight(a, x, col);
#pragma unroll
        for (int part = 0; part < kParts; ++part) x.pages[part] = page_of(few_pages(a, x), (x.key0 + 16 * part) >> a.log_ps, few_page_count(a, x));
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int d = 32 * w + 8 * grp;
            x.q[w] = word4_t{0, 0, 0, 0};
            if (x.t >= 0 && d < D) x.q[w] = (*reinterpret_cast<const word4_t *>(a.q + x.t * a.q_stride + (x.h * a.group + member) * D + d) & a.q_and) ^ a.q_xor;
        }
    };
    // The step that is asked for next: its first key (behind the last of the piece: none), pages, where the piece's keys end, the head; and the list that the pages come from.
    int ask_key = 0, ask_end = 0, ask_h = 0, ask_pages[kParts], ask_count = 1;
    const int32_t *ask_list = a.table;
    auto aim = [&](const Piece4<NW> &x, bool there) __attribute__((always_inline)) {
        ask_key = x.key0;
        ask_end = there ? min(x.limit, x.key0 + x.n * kFewTile) : 0;
        ask_h = x.h;
        ask_list = few_pages(a, x);
        ask_count = few_page_count(a, x);
#pragma unroll
        for (int part = 0; part < kParts; ++part) ask_pages[part] = x.pages[part];
    };
    const int scale_off = grp < G ? (col * G + grp) * 4 : kNowhere;
    // Always as many loads, of nothing where there is nothing: then the waits for a step's know how many came behind it.
    auto load = [&](Step4<NW> &to) __attribute__((always_inline)) {
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            const int key = ask_key + 16 * part, id = ask_pages[part];
            const int valid = (unsigned)id < (unsigned)a.pages ? min(max(ask_end - key, 0), 16) : 0;
            const unsigned char *const keys = a.kv + (valid ? id : 0) * a.page_bytes + ask_h * head_bytes, *const values = keys + (a.page_bytes >> 1);
            const long codes = codes_at4(key & ps1, DS), scales = scales_at4(a.log_ps, key & ps1, DS);
            const int all = valid ? 8 * DS : 0;               // (codes of places without a token do no harm: their scales are zeros)
            load_words<NW, kOnce>(to.k[part], buffer_of(keys + codes, all), (col * 4 + grp) * NW * 4);
            to.ks[part] = __builtin_amdgcn_raw_buffer_load_b32(buffer_of(keys + scales, valid * 4 * G), scale_off, 0, 0);
            load_words<NW, kOnce>(to.v[part], buffer_of(values + codes, all), lane * NW * 4);
            to.vs[part] = __builtin_amdgcn_raw_buffer_load_b32(buffer_of(values + scales, valid * 4 * G), scale_off, 0, 0);
        }
        ask_key += kFewTile;                                  // (the pages of the one behind it, needed a step from now)
#pragma unroll
        for (int part = 0; part < kParts; ++part) ask_pages[part] = page_of(ask_list, (ask_key + 16 * part) >> a.log_ps, ask_count);
    };

    Queries4<TY, NT, NW> q;
    word2_t eighths[G], spread[G];                            // what makes (m + 8 s) / 2 (8 s may be beyond fp32), and 2^(10 - x) s, of a group's scale words
#pragma unroll
    for (int y = 0; y < G; ++y) eighths[y] = word2_t{grp == y ? NT::bits(4.0f) << 16 | NT::bits(0.5f) : 0u, 0u};
    float4_t o[J], eights[G];                                 // eights: sums of 8 p s as it is rounded, times 2^(-14 - x) like those of p s c in o
    float m, l, lows[G];                                      // lows: sum p (m + 8 s) / 2, of the lane's keys
    int least, e, x_of;                                       // what every row of the piece sees; the exponent that p is relative to, and x (AGAIN: of the lane's row; else the same in all lanes)
    uint32_t most;                                            // the largest scale word that goes with them
    bool again = false;
    int beside;                                               // what e goes with of the scales that all rows see
    auto begin = [&]() __attribute__((always_inline)) {
        q.of(cur.q, a.scale);
#pragma unroll
        for (int j = 0; j < J; ++j) o[j] = float4_t{0, 0, 0, 0};
#pragma unroll
        for (int y = 0; y < G; ++y) {
            lows[y] = 0;
            eights[y] = float4_t{0, 0, 0, 0};
            spread[y] = word2_t{grp == y ? NT::bits(1024.0f) << 16 : 0u, 0u};
        }
        m = kNoScore;
        l = 0;
        e = 0;
        x_of = 0;
        most = 0;
        beside = 1 << 20;
        least = cur.t >= 0 ? cur.sees : cur.limit;
#pragma unroll
        for (int x = 8; x; x >>= 1) least = min(least, __shfl_xor(least, x));
        least = uniform(least);
    };
    auto compute = [&](const Step4<NW> &x, int s) __attribute__((always_inline)) {
        float4_t z[kParts];
        float top = -INFINITY;
        const int key = cur.key0 + s * kFewTile;
#pragma unroll
        for (int part = 0; part < kParts; ++part) z[part] = scores4<TY, NT, NW>(x.k[part], x.ks[part], q);
        if (key + kFewTile > least) {
            const int sees = cur.sees - key - 4 * grp;
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (16 * part + i >= sees) z[part][i] = -INFINITY;
        }
        uint32_t largest = 0;                                 // scale word: scales are in its upper half, and not negative
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            top = fmaxf(top, fmaxf(fmaxf(z[part][0], z[part][1]), fmaxf(z[part][2], z[part][3])));
            largest = max(largest, x.vs[part]);
        }
        top = larger_of_16(top);
        top = larger_of_32(top) * q.unit;
        const auto same = [](int v) { return AGAIN ? v : uniform(v); };
        const bool apart = least < min(cur.limit, key + kFewTile);            // (rows see different tokens of the step)
        if (AGAIN && apart) {                                 // of the lane's row
            largest = 0;
#pragma unroll 1
            for (int k = 0; k < kFewTile; ++k)
#pragma unroll
                for (int y = 0; y < G; ++y) {
                    const uint32_t word = __builtin_amdgcn_readlane((int)(k < 16 ? x.vs[0] : x.vs[1]), (k & 15) + 16 * y);
                    if (k < cur.sees - key) largest = max(largest, word);
                }
        }
        if (__ballot(top > m - (float)e + kSlack || largest > most)) {
            const int before = e, x_before = x_of;
            if (!AGAIN || !apart) {
#pragma unroll
                for (int w = 32; w; w >>= 1) largest = max(largest, (uint32_t)__shfl_xor((int)largest, w));
                largest = uniform(largest);
            }
            // (AGAIN: a row's maximum follows as it did the first time, or with the row's own exponent)
            const bool passed = AGAIN && __ballot(top > m - (float)e + kSlack) != 0, follows = !AGAIN || !apart || passed || largest > most;
            if (largest > most) {
                const int all = same(__builtin_amdgcn_frexp_expf(NT::of_upper(largest)) + 5);
                if (!AGAIN && apart) {                        // beside the largest that all see (who sees any of the piece sees its first key)
                    const int seen = max(least - key, key == cur.key0 ? 1 : 0);
                    uint32_t known = max(col < seen ? x.vs[0] : 0, 16 + col < seen ? x.vs[1] : 0);
#pragma unroll 1
                    for (int w = 32; w; w >>= 1) known = max(known, (uint32_t)__shfl_xor((int)known, w));
                    beside = min(beside, uniform(max(known >> 16 ? __builtin_amdgcn_frexp_expf(NT::of_upper(known)) + 5 : -1000, most ? e + x_of : -1000)));
                    again |= all > beside + 4;
                }
                e = all;
                if (NT::kWide) {
                    e = min(max(all, -24), 34);
                    x_of = max(all, -110) - e;                // (so that the factor is a number of the type)
#pragma unroll
                    for (int y = 0; y < G; ++y) spread[y][0] = grp == y ? NT::bits(ldexpf(1024.0f, -x_of)) << 16 : 0u;
                }
                const uint32_t beyond = NT::bits(ldexpf(1.0f, all - 3));                  // (an infinity: no scale is)
                most = same((beyond << 16) - 1);
            }
            const float to = follows ? fmaxf(top, m - (float)before) + (float)e : m, by = __builtin_amdgcn_exp2f(m - to);
            const float by_scaled = NT::kWide ? ldexpf(by, x_before - x_of) : by;
            l *= by;
#pragma unroll
            for (int j = 0; j < J; ++j) o[j] *= by_scaled;
#pragma unroll
            for (int y = 0; y < G; ++y) {
                lows[y] *= by;
                eights[y] *= by_scaled;
            }
            m = to;
        }
        uint32_t ps[G][2 * kParts];
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[part][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[part][i], q.unit, -m));
                l += z[part][i];
            }
#pragma unroll
            for (int y = 0; y < G; ++y) {
                const float4_t s = scales_of<TY>(x.vs[part], spread[y]), low = scales_of<TY>(x.vs[part], eighths[y]);
                float of[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    lows[y] = __builtin_fmaf(low[i], z[part][i], lows[y]);
                    of[i] = (AGAIN && NT::kWide ? fminf(s[i], 0x1p127f) : s[i]) * z[part][i];        // (beyond fp32 it may be where the row does not see it, and p is 0)
                }
                ps[y][2 * part] = TypeF16::pack(of[0], of[1]);
                ps[y][2 * part + 1] = TypeF16::pack(of[2], of[3]);
            }
        }
        const word4_t eight{0x00080008u, 0x00080008u, 0x00080008u, 0x00080008u};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const uint32_t a = x.v[0][w], b = x.v[1][w];
            const word4_t p{ps[w / 2][0], ps[w / 2][1], ps[w / 2][2], ps[w / 2][3]};
            o[2 * w] = TypeF16::mfma(word4_t{a & kLowCodes, a >> 8 & kLowCodes, b & kLowCodes, b >> 8 & kLowCodes}, p, o[2 * w]);
            o[2 * w + 1] = TypeF16::mfma(word4_t{a & kHighCodes, a >> 8 & kHighCodes, b & kHighCodes, b >> 8 & kHighCodes}, p, o[2 * w + 1]);
            if (w % 2 == 0) eights[w / 2] = TypeF16::mfma(eight, p, eights[w / 2]);
        }
    };
    bool first = true;
    auto finish = [&]() __attribute__((always_inline)) {
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
#pragma unroll
        for (int y = 0; y < G; ++y) {
            lows[y] += __shfl_xor(lows[y], 16);
            lows[y] += __shfl_xor(lows[y], 32);
            lows[y] *= 2;
        }
        const float back = NT::kWide ? ldexpf(0x1p14f, x_of) : 0x1p14f;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[j][i] = __builtin_fmaf(j & 1 ? __builtin_fmaf(o[j][i], 0.0625f, -eights[j / 4][i]) : o[j][i] - eights[j / 4][i], back, lows[j / 4]);
        if (together) {                                       // the first wave joins the block's, as in attend_few_wave
            float *const at = reinterpret_cast<float *>(room) + lane;
            int *const flags = reinterpret_cast<int *>(room + kFew4PartsRoom<NW>);
            const int wave = uniform(threadIdx.x >> 6);
            if (AGAIN) __syncthreads();                       // (the first one may still read what was joined before)
            else if (lane == 0) flags[wave] = again;
            if (wave) {
                float *const to = at + (wave - 1) * (4 * J + 2) * 64;
                to[0] = m;
                to[64] = l;
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) to[(2 + 4 * j + i) * 64] = o[j][i];
            }
            __syncthreads();
            if (!AGAIN) {
#pragma unroll
                for (int w = 0; w < kFewWaves; ++w) again |= uniform(flags[w]) != 0;
            }
            if (wave) return;
            float to = m;
#pragma unroll
            for (int w = 0; w < kFewWaves - 1; ++w) to = fmaxf(to, at[w * (4 * J + 2) * 64]);
            const float by = __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= by;
#pragma unroll
            for (int j = 0; j < J; ++j) o[j] *= by;
#pragma unroll
            for (int w = 0; w < kFewWaves - 1; ++w) {
                const float *const from = at + w * (4 * J + 2) * 64;
                const float times = __builtin_amdgcn_exp2f(from[0] - m);
                l += from[64] * times;
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[j][i] += from[(2 + 4 * j + i) * 64] * times;
            }
        }
        if (cur.t < 0) return;
        const bool whole = a.direct || cur.n == cur.steps;
        const Partials to = whole ? (cur.b < 0 ? a.whole_shared : a.whole) : a.piece;
        const int head = cur.h * a.group + member;
        const bool last = whole && !to.o;
        const float by = l == 0 ? 0.0f : 1.0f / l;
        const long r = whole ? (long)cur.t * a.heads + head : ((long)worker * 2 + (first ? 0 : 1)) * a.slot_rows + col;
#pragma unroll
        for (int y = 0; y < G; ++y) {
            const int z = lane_features4(DS, y), d0 = 64 * y + 4 * z * grp;               // 4 z features in a row: feature z i + j in o[4 y + j][i]
#pragma unroll
            for (int c = 0; c < z; ++c) {
                float4_t four;
#pragma unroll
                for (int x = 0; x < 4; ++x) four[x] = o[4 * y + (4 * c + x) % z][(4 * c + x) / z];
                if (d0 + 4 * c >= D) continue;
                if (last) *reinterpret_cast<word2_t *>(a.out + cur.t * a.out_stride + head * D + d0 + 4 * c) = word2_t{TY::pack(four[0] * by, four[1] * by), TY::pack(four[2] * by, four[3] * by)};
                else *reinterpret_cast<float4_t *>(to.o + r * D + d0 + 4 * c) = four;
            }
        }
        if (grp) return;
        if (!last) to.ml[r] = make_float2(m, l);
        else if (a.lse) a.lse[(long)cur.t * a.heads + head] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    };

    if constexpr (AGAIN) {                                    // (few registers before speed)
        while (true) {
            prepare(cur);
            begin();
            aim(cur, cur.n > 0);
            for (int s = 0; s < cur.n; ++s) {
                Step4<NW> x;
                load(x);
                compute(x, s);
            }
            finish();
            if (!line.follow(a, cur, behind)) return false;
            first = false;
            cur = behind;
        }
    }
    // One copy of `finish` and of all that a new piece takes: the kernel is long, and where there is little to do it waits for its instructions.
    prepare(cur);
    behind = cur;                                             // (where there is none, something that is one)
    bool more = line.follow(a, cur, behind);
    if (more) prepare(behind);
    Step4<NW> x0, x1;
    aim(cur, cur.n > 0);
    load(x0);
    while (true) {
        begin();
        for (int s = 0; s < cur.n; s += 2) {                  // (a piece without steps: no tokens in the item, or in this worker's part)
            if (s + 1 >= cur.n) aim(behind, more);
            load(x1);
            compute(x0, s);
            if (s + 1 < cur.n) {
                if (s + 2 >= cur.n) aim(behind, more);
                load(x0);
                compute(x1, s + 1);
            } else {
                x0 = x1;
            }
        }
        finish();
        if (!more) return again;
        first = false;
        cur = behind;
        more = line.follow(a, cur, behind);
        if (more) prepare(behind);
    }
}

// Block `block` of the few-row work, kFewWaves waves.
template <class TY, class NT, int NW>
__device__ __forceinline__ void attend4_few(const AttendArgs &a, int block, unsigned char *room)
{
    if (!attend4_few_wave<TY, NT, NW, false>(a, block, room)) return;
    // What follows from the block and the arguments takes no registers until the second time: the arguments, each such kernel's first parameter, are read again (see fbq_attend4_many.h).
    asm volatile("" : "+s"(block) : : "memory");
    typedef const __attribute__((address_space(4))) AttendArgs *Kept;
    Kept again = (Kept)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(again));
    attend4_few_wave<TY, NT, NW, true>(*(const AttendArgs *)again, block, room);
}

}  // namespace fbq

#endif
