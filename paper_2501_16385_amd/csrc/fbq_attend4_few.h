// Attention of a few query rows against a long row of a cache in 4 bits: the work of fbq_attend_few.h (its items, pieces and join) over codes.
//
// Codes go into the matrix cores as they are, fp16 numbers below the normal ones (fbq_cache4.h), and are multiplied exactly; scales come in afterwards, in 32 bits.
//   scores   k = m + s c of a key's group:  q . k = sum over groups of  s (q . c) + m sum(q):  16 keys' q . c is two products a group, of the codes at low and at high bits, and the
//            sums of q over a group are made once a piece.  Queries of bf16 are fp16 here, times a power of two for the row (which goes into its scale): bf16 has fewer digits, so
//            only what is 2^-28 of the row's largest feature and less loses any.
//   results  sum p v = sum (p s) c + sum p m:  p s is operand B of the second product, a rounding to fp16 where fbq_attend_few.h rounds p; the second sum stays in 32 bits, in the lane.
//            p s has to be in fp16's range whatever the scales: p is relative to 2^e too, e the exponent of the largest scale so far, less 5, and follows when it is passed by 2^7.
// A value that nobody sees has weight zero and finite scales, so nothing of it is added, whatever it is: no second look is needed.
//
// Bound by HBM in long rows: D / 2 + 4 G bytes a key and a value, a third to a fourth of 16 bits' - and close behind by the vector instructions, about 250 for 32 keys of 128 features.
#ifndef FBQ_ATTEND4_FEW_H
#define FBQ_ATTEND4_FEW_H

#include <algorithm>
#include <type_traits>

#include "fbq_attend_few.h"
#include "fbq_cache4.h"

namespace fbq {

template <int NW>
struct Step4 {
    static constexpr int G = groups4(32 * NW);
    uint32_t k[2][NW], v[2][NW];                              // of 16 keys each
    word4_t ks[2][G], vs[2][G];                               // scales of this lane's four of them: [key][group]
};

template <int NW>
__device__ __forceinline__ void load_words(uint32_t (&to)[NW], __amdgpu_buffer_rsrc_t from, int off)
{
    typedef uint32_t word3_t __attribute__((ext_vector_type(3)));
#pragma unroll
    for (int i = 0; i < NW / 4; ++i) {
        const word4_t w = __builtin_amdgcn_raw_buffer_load_b128(from, off + 16 * i, 0, kOnce);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[4 * i + e] = w[e];
    }
    if constexpr (NW % 4 == 2) {
        const word2_t w = __builtin_amdgcn_raw_buffer_load_b64(from, off + 4 * (NW - 2), 0, kOnce);
        to[NW - 2] = w[0];
        to[NW - 1] = w[1];
    }
    if constexpr (NW == 3) {
        const word3_t w = __builtin_amdgcn_raw_buffer_load_b96(from, off, 0, kOnce);
        to[0] = w[0];
        to[1] = w[1];
        to[2] = w[2];
    }
}

// The queries of a wave's 16 rows as operands for codes: of a group, those at low bits and those at high bits; the group's sums of them, times 2^-24; what scores are to be multiplied by.
template <class NT, int NW>
struct Queries4 {
    static constexpr int G = groups4(32 * NW);
    word4_t at[G][2];
    float sum[G];
    float unit;

    // q: the words of features 32 w + 8 (lane / 16) .., of the lane's row
    __device__ __forceinline__ void of(const word4_t (&q)[NW], float scale)
    {
        word4_t h[NW];
        unit = scale * 0x1p24f;
        if constexpr (std::is_same<NT, NumberF16>::value) {
#pragma unroll
            for (int w = 0; w < NW; ++w) h[w] = q[w];
        } else {
            float most = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaxf(fabsf(NT::of(q[w][e] & 0xffff)), fabsf(NT::of_upper(q[w][e]))));
            const int up = __builtin_amdgcn_frexp_expf(larger_of_32(larger_of_16(most))) - 15;
            unit = ldexpf(unit, up);
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e) h[w][e] = TypeF16::pack(ldexpf(NT::of(q[w][e] & 0xffff), -up), ldexpf(NT::of_upper(q[w][e]), -up));
        }
        const word4_t one{0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};
#pragma unroll
        for (int y = 0; y < G; ++y) {
            const word4_t a = h[2 * y], b = 2 * y + 1 < NW ? h[std::min(2 * y + 1, NW - 1)] : word4_t{0, 0, 0, 0};
            at[y][0] = word4_t{a[0], a[1], b[0], b[1]};
            at[y][1] = word4_t{a[2], a[3], b[2], b[3]};
            const float4_t s = TypeF16::mfma(one, at[y][1], TypeF16::mfma(one, at[y][0], float4_t{0, 0, 0, 0}));
            sum[y] = s[0] * 0x1p-24f;
        }
    }
};

// Scores of 16 keys, 2^24 / unit of them: keys 4 (l / 16) + i in z[i], the lane's query row.
template <class NT, int NW>
__device__ __forceinline__ float4_t scores4(const uint32_t (&k)[NW], const word4_t (&ks)[groups4(32 * NW)], const Queries4<NT, NW> &q)
{
    constexpr int G = groups4(32 * NW);
    float4_t z{0, 0, 0, 0};
#pragma unroll
    for (int y = 0; y < G; ++y) {
        const uint32_t a = k[2 * y], b = 2 * y + 1 < NW ? k[std::min(2 * y + 1, NW - 1)] : 0;
        const float4_t low = TypeF16::mfma(word4_t{a & kLowCodes, a >> 8 & kLowCodes, b & kLowCodes, b >> 8 & kLowCodes}, q.at[y][0], float4_t{0, 0, 0, 0});
        const float4_t high = TypeF16::mfma(word4_t{a & kHighCodes, a >> 8 & kHighCodes, b & kHighCodes, b >> 8 & kHighCodes}, q.at[y][1], float4_t{0, 0, 0, 0});
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t word = ks[(i * G + y) / 4][(i * G + y) % 4];
            z[i] = __builtin_fmaf(NT::of(word & 0xffff), q.sum[y], y ? z[i] : 0.0f);
            z[i] = __builtin_fmaf(NT::of_upper(word), __builtin_fmaf(high[i], 0.0625f, low[i]), z[i]);
        }
    }
    return z;
}

template <int NW>
constexpr int kFew4Room = (kFewWaves - 1) * (2 * 4 * NW + 2) * 256;

// TY: the type of queries and results; NT: its numbers.
template <class TY, class NT, int NW>
__device__ __forceinline__ void attend4_few(const AttendArgs &a, int block, unsigned char *room)
{
    constexpr int DS = 32 * NW, G = groups4(DS), J = 2 * NW;   // products of the results
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const int worker = uniform(block * kFewWaves + (threadIdx.x >> 6));
    const int D = a.D, ps1 = (1 << a.log_ps) - 1;
    const int member = col % a.group;
    const long head_bytes = (a.page_bytes >> 1) / a.kv_heads;

    Piece<DS> cur, behind;
    FewLine line;
    if (!line.first(a, block, worker, cur)) return;
    const bool together = line.together;
    auto prepare = [&](Piece<DS> &x) __attribute__((always_inline)) {
        few_sight(a, x, col);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int d = 32 * w + 8 * grp;
            x.q[w] = word4_t{0, 0, 0, 0};
            if (x.t >= 0 && d < D) x.q[w] = (*reinterpret_cast<const word4_t *>(a.q + x.t * a.q_stride + (x.h * a.group + member) * D + d) & a.q_and) ^ a.q_xor;
        }
    };
    auto load = [&](Step4<NW> &to, Piece<DS> &x, int s) __attribute__((always_inline)) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int key = x.key0 + s * kFewTile + 16 * half;
            int valid = min(max(x.limit - key, 0), 16);
            const int id = valid ? x.pages.at(key >> a.log_ps) : 0;
            if ((unsigned)id >= (unsigned)a.pages) valid = 0;
            const unsigned char *const keys = a.kv + (valid ? id : 0) * a.page_bytes + x.h * head_bytes, *const values = keys + (a.page_bytes >> 1);
            const long codes = codes_at4(key & ps1, DS), scales = scales_at4(a.log_ps, key & ps1, DS);
            const int all = valid ? 8 * DS : 0;               // (codes of places without a token do no harm: their scales are zeros)
            load_words<NW>(to.k[half], buffer_of(keys + codes, all), (col * 4 + grp) * NW * 4);
            load_words<NW>(to.v[half], buffer_of(values + codes, all), lane * NW * 4);
            const __amdgpu_buffer_rsrc_t kb = buffer_of(keys + scales, valid * 4 * G), vb = buffer_of(values + scales, valid * 4 * G);
#pragma unroll
            for (int y = 0; y < G; ++y) {
                to.ks[half][y] = __builtin_amdgcn_raw_buffer_load_b128(kb, grp * 16 * G + 16 * y, 0, 0);
                to.vs[half][y] = __builtin_amdgcn_raw_buffer_load_b128(vb, grp * 16 * G + 16 * y, 0, 0);
            }
        }
    };

    Queries4<NT, NW> q;
    float4_t o[J];
    float m, l, lows[G];                                      // lows: sum p m, of the lane's keys
    int least, e;                                             // what every row of the piece sees; the exponent that p is relative to
    uint32_t most;                                            // the largest scale word that goes with e
    auto begin = [&]() __attribute__((always_inline)) {
        q.of(cur.q, a.scale);
#pragma unroll
        for (int j = 0; j < J; ++j) o[j] = float4_t{0, 0, 0, 0};
#pragma unroll
        for (int y = 0; y < G; ++y) lows[y] = 0;
        m = kNoScore;
        l = 0;
        e = 0;
        most = 0;
        least = cur.t >= 0 ? cur.sees : cur.limit;
#pragma unroll
        for (int x = 8; x; x >>= 1) least = min(least, __shfl_xor(least, x));
        least = uniform(least);
    };
    auto compute = [&](const Step4<NW> &x, int s) __attribute__((always_inline)) {
        float4_t z[2];
        float top = -INFINITY;
        const int key = cur.key0 + s * kFewTile;
#pragma unroll
        for (int half = 0; half < 2; ++half) z[half] = scores4<NT, NW>(x.k[half], x.ks[half], q);
        if (key + kFewTile > least) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    if (key + 16 * half + 4 * grp + y >= cur.sees) z[half][y] = -INFINITY;
        }
        uint32_t largest = 0;                                 // scale word: scales are in its upper half, and not negative
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            top = fmaxf(top, fmaxf(fmaxf(z[half][0], z[half][1]), fmaxf(z[half][2], z[half][3])));
#pragma unroll
            for (int y = 0; y < G; ++y)
#pragma unroll
                for (int i = 0; i < 4; ++i) largest = max(largest, x.vs[half][y][i]);
        }
        top = larger_of_16(top);
        top = larger_of_32(top) * q.unit;
        if (__ballot(top > m - (float)e + kSlack || largest > most)) {
            const int before = e;
#pragma unroll
            for (int w = 32; w; w >>= 1) largest = max(largest, (uint32_t)__shfl_xor((int)largest, w));
            largest = uniform(largest);
            if (largest > most) {
                e = uniform(max(__builtin_amdgcn_frexp_expf(NT::of_upper(largest)) - 5, -100));
                const uint32_t beyond = NT::bits(ldexpf(1.0f, e + 7));                    // (an infinity: no scale is)
                most = uniform((beyond << 16) - 1);
            }
            const float to = fmaxf(top, m - (float)before) + (float)e, by = __builtin_amdgcn_exp2f(m - to);
            l *= by;
#pragma unroll
            for (int j = 0; j < J; ++j) o[j] *= by;
#pragma unroll
            for (int y = 0; y < G; ++y) lows[y] *= by;
            m = to;
        }
        uint32_t ps[G][4];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[half][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[half][i], q.unit, -m));
                l += z[half][i];
            }
#pragma unroll
            for (int y = 0; y < G; ++y) {
                float of[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t word = x.vs[half][(i * G + y) / 4][(i * G + y) % 4];
                    lows[y] = __builtin_fmaf(z[half][i], NT::of(word & 0xffff), lows[y]);
                    of[i] = z[half][i] * NT::of_upper(word);
                }
                ps[y][2 * half] = TypeF16::pack(of[0], of[1]);
                ps[y][2 * half + 1] = TypeF16::pack(of[2], of[3]);
            }
        }
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const uint32_t a = x.v[0][w], b = x.v[1][w];
            const word4_t p{ps[w / 2][0], ps[w / 2][1], ps[w / 2][2], ps[w / 2][3]};
            o[2 * w] = TypeF16::mfma(word4_t{a & kLowCodes, a >> 8 & kLowCodes, b & kLowCodes, b >> 8 & kLowCodes}, p, o[2 * w]);
            o[2 * w + 1] = TypeF16::mfma(word4_t{a & kHighCodes, a >> 8 & kHighCodes, b & kHighCodes, b >> 8 & kHighCodes}, p, o[2 * w + 1]);
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
        }
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[j][i] = __builtin_fmaf(o[j][i], j & 1 ? 0x1p20f : 0x1p24f, lows[j / 4]);
        if (together) {                                       // the first wave joins the block's, as in attend_few_wave
            float *const at = reinterpret_cast<float *>(room) + lane;
            const int wave = uniform(threadIdx.x >> 6);
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

    prepare(cur);
    if (cur.n == 0) {                                         // (no tokens in the item, or in this worker's part)
        begin();
        finish();
        return;
    }
    bool more = line.follow(a, cur, behind);
    if (more) prepare(behind);
    Step4<NW> x0, x1;
    load(x0, cur, 0);
    begin();
    int s = 0;
    auto turn = [&](const Step4<NW> &now, Step4<NW> &next) __attribute__((always_inline)) {
        if (s + 1 < cur.n) load(next, cur, s + 1);
        else if (more) load(next, behind, 0);
        compute(now, s);
        if (++s < cur.n) return false;
        finish();
        if (!more) return true;
        first = false;
        cur = behind;
        s = 0;
        more = line.follow(a, cur, behind);
        if (more) prepare(behind);
        begin();
        return false;
    };
    while (!turn(x0, x1) && !turn(x1, x0)) {}
}

}  // namespace fbq

#endif
