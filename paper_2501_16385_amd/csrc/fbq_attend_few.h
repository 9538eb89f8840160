// Attention of a few query rows against a long row of the cache: decode steps, and short prefixes of a shared prompt.
//
// An item is one key/value head of one table row: up to 16 query rows (its query tokens times the heads that share it) against the row's keys and values, which
// are read once.  Bound by HBM: 2 x 2 D bytes a key, for 4 D flops a query row and key.  A step is 32 keys; all steps of all items form one line, which the waves
// of the grid cut into equal pieces - lengths lie on the device, the line is laid out from them by a scan in each wave - so that one long row among short ones
// occupies the whole GPU and no host value decides the cut.  (Where rows are short an item goes to a wave or a block whole: few_direct in fbq_attention.hip.)  A piece of an item leaves partial results for the join kernel; an item that lies
// within one piece is written at once.
//
// Keys and values go from memory to registers to the matrix cores, nothing through LDS, and waves wait for nobody until a block's pieces of one item are joined.  S^T = K Q^T puts a key's scores in rows and a
// query row in a column: v_mfma_f32_16x16x32, operand A lane l key l % 16, features 8 (l / 16) and up of 32, which is how keys lie in memory.  The result has
// column l % 16, keys 4 (l / 16) + i: a lane's eight probabilities of a step are keys 4 g .. 4 g + 3 and 16 + 4 g .. of group g = l / 16.  O^T = V^T P^T
// takes them as operand B where they are, since the order of a contraction is free: V^T's lanes take the same eight keys.  A lane loads DP / 16
// features (l % 16 being the piece) of its eight keys and turns them by byte permutes; row l % 16 of the j-th product is then feature (DP / 16) (l % 16) + j, and
// a lane's results are DP / 4 features in a row of one query row.  The scale by exp(m_old - m_new) is the lane's own.
//
// Measured, 128 features, the join included: 64 rows of 4096 tokens, 64 heads of 8, 169 us (6.35 TB/s; a kernel that only reads 6.31); 16 rows of about 1000, 32 heads, 54 (263 MB; reading alone
// 43.5); one row of 65537, 64 heads of 8, 55.  Two steps of 16 KB are under way in each of eight waves a CU; a wave alone on its SIMD takes 1.65 us a step.
#ifndef FBQ_ATTEND_FEW_H
#define FBQ_ATTEND_FEW_H

#include "fbq_attend.h"
#include "fbq_lds_copy.h"

namespace fbq {

// Cache policy of a load, nt: what is read once takes no room from what is read again (16 rows of about 1000 tokens, 32 heads: 55 us, 62 without it).
constexpr int kOnce = 2;

template <int DP>
struct Step {
    static constexpr int kV = DP == 256 ? 2 : 1;              // 16-byte loads of a lane's features of one value row (DP 64: one of 8 bytes)
    static constexpr int kHalves = DP == 256 ? 1 : 2;         // of its 32 keys that a turn loads and works on (256 features: two turns a step, or registers run out)
    word4_t k[kHalves][DP / 32];
    word4_t v[kHalves][4][kV];
};

// A piece of an item: what its loads and its rows need, both for the piece worked on and the one behind it.
template <int DP>
struct Piece {
    int b, h, step, steps, limit;                             // table row (-1: the shared tokens), head, its first step of the item's `steps`, tokens of the item
    int n, key0;                                              // steps of its own, its first key
    PageList pages;
    int t, sees;                                              // this lane's query row: token (-1: none), how many tokens it sees
    word4_t q[DP / 32];
};

// Bytes of LDS (aligned to 16) of a block of it: parts of waves 1 .., and a word a wave.
template <int DP>
constexpr int kFewParts = (kFewWaves - 1) * (DP / 4 + 2) * 256;
template <int DP>
constexpr int kFewRoom = kFewParts<DP> + 4 * kFewWaves;

// The work of the block's wave (see attend_few), its results written.  AGAIN: slowly, but so that a value reaches the rows that see it and no others, whatever it is.  Without it a
// value that is no number reaches all of the item's rows: zero times it is none either.  Whether that has happened (for all waves of a block that join theirs the same answer).
// Four tokens behind 4000, a NaN among the last one's values: 38 us, else 22.
template <class TY, int DP, bool AGAIN>
__device__ __forceinline__ bool attend_few_wave(const AttendArgs &a, int block, unsigned char *room)
{
    constexpr int J = DP / 16;                                // features of a lane's value pieces, and products O^T of a turn
    constexpr int kHalves = Step<DP>::kHalves, kTurn = 16 * kHalves, kTurns = kFewTile / kTurn;   // keys a turn, turns a step
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const int worker = uniform(block * kFewWaves + (threadIdx.x >> 6));
    const int D = a.D, ps1 = (1 << a.log_ps) - 1;
    const int member = col % a.group;                         // of the heads that share a key/value head: this lane's

    Piece<DP> cur, behind;
    int u = 0, end = 0;
    bool together = false;                                    // the block's waves have a piece each of one item
    if (a.direct) {                                           // an item a worker, or a part of it each for the block's workers
        const int item = a.direct == 1 ? worker : block;
        cur.b = item / a.kv_heads;
        if (cur.b >= a.rows) return false;
        cur.h = item - cur.b * a.kv_heads;
        cur.limit = uniform(row_tokens(a, cur.b));
        cur.steps = uniform(few_steps(a, cur.b, cur.limit));
        together = a.direct == 2;
        const int share = together ? (cur.steps + kFewWaves - 1) / kFewWaves : cur.steps;
        cur.step = together ? min((worker & (kFewWaves - 1)) * share, cur.steps) : 0;
        cur.n = min(share, cur.steps - cur.step);
    } else {
        int own = 0;
        for (int b = lane; b < a.rows; b += 64) own += few_steps(a, b);
        own = __builtin_amdgcn_readlane(wave_scan(own), 63);
        const int shared_steps = a.shared_here ? (a.n_shared + kFewTile - 1) / kFewTile : 0;
        const int total = (own + shared_steps) * a.kv_heads;
        const int share = few_share(a, total);
        u = min(worker, total) * share;                       // (worker * share within an int)
        end = min(total, u + share);
        if (u >= end) return false;
        if (u < shared_steps * a.kv_heads) {
            cur.b = -1;
            cur.limit = a.n_shared;
            cur.steps = shared_steps;
            cur.h = u / cur.steps;
            cur.step = u - cur.h * cur.steps;
        } else {
            int rest = u - shared_steps * a.kv_heads, before = 0, base = 0, tokens, mine, sum;
            while (true) {
                tokens = base + lane < a.rows ? row_tokens(a, base + lane) : 0;
                mine = base + lane < a.rows ? few_steps(a, base + lane, tokens) : 0;
                sum = wave_scan(mine);
                const int some = __builtin_amdgcn_readlane(sum, 63);
                if ((long)rest < (long)(before + some) * a.kv_heads) break;
                before += some;
                base += 64;
                if (base >= a.rows) return false;             // (not unless lengths change under the call)
            }
            const int at = __builtin_ctzll(__ballot((long)(before + sum) * a.kv_heads > rest));
            cur.b = base + at;
            cur.steps = __builtin_amdgcn_readlane(mine, at);
            cur.limit = __builtin_amdgcn_readlane(tokens, at);
            rest -= (before + __builtin_amdgcn_readlane(sum, at) - cur.steps) * a.kv_heads;
            cur.h = rest / cur.steps;
            cur.step = rest - cur.h * cur.steps;
        }
        cur.n = min(end - u, cur.steps - cur.step);
        together = few_together(worker / kFewWaves, share, u - cur.step, u - cur.step + cur.steps);
        u += cur.n;
    }

    // the item behind `x`, which ends with it; false: there is none
    auto follow = [&](const Piece<DP> &x, Piece<DP> &to) __attribute__((always_inline)) {
        if (u >= end) return false;
        to.b = x.b; to.h = x.h + 1; to.steps = x.steps; to.limit = x.limit; to.step = 0;
        if (to.h == a.kv_heads) {
            to.h = 0;
            do {
                if (++to.b >= a.rows) return false;           // (not unless lengths change under the call)
                to.limit = uniform(row_tokens(a, to.b));
                to.steps = uniform(few_steps(a, to.b, to.limit));
            } while (to.steps == 0);
        }
        to.n = min(end - u, to.steps);
        u += to.n;
        return true;
    };
    auto prepare = [&](Piece<DP> &x) __attribute__((always_inline)) {
        const bool is_shared = x.b < 0;
        x.key0 = (is_shared ? 0 : a.n_shared) + x.step * kFewTile;
        x.pages.begin(is_shared ? a.shared : a.table + (long)x.b * a.max_pages, is_shared ? a.n_shared >> a.log_ps : a.max_pages, x.key0 >> a.log_ps);
        const int i = col / a.group;
        x.t = -1;
        x.sees = 0;
        if (is_shared) {
            if (i < a.T) {
                const int row = a.q_start ? row_of_token(a.q_start, a.rows, i) : i;
                if (row >= 0) {
                    const int2 q = queries_of(a, row);
                    if (i - q.x < q.y) {
                        x.t = i;
                        x.sees = min(row_tokens(a, row) - q.y + i - q.x + 1, x.limit);
                    }
                }
            }
        } else {
            const int2 q = queries_of(a, x.b);
            if (i < q.y) {
                x.t = q.x + i;
                x.sees = x.limit - q.y + i + 1;
            }
        }
#pragma unroll
        for (int s = 0; s < DP / 32; ++s) {
            const int d = 32 * s + 8 * grp;
            x.q[s] = word4_t{0, 0, 0, 0};
            if (x.t >= 0 && d < D) x.q[s] = (*reinterpret_cast<const word4_t *>(a.q + x.t * a.q_stride + (x.h * a.group + member) * D + d) & a.q_and) ^ a.q_xor;
        }
    };

    // offsets of this lane's loads from a half step's first key, or value
    int k_off[DP / 32], v_off[4];
#pragma unroll
    for (int s = 0; s < DP / 32; ++s) k_off[s] = 32 * s + 8 * grp < D ? (col * D + 32 * s + 8 * grp) * 2 : kNowhere;
#pragma unroll
    for (int e = 0; e < 4; ++e) v_off[e] = J * col < D ? ((4 * grp + e) * D + J * col) * 2 : kNowhere;
    auto load = [&](Step<DP> &to, Piece<DP> &x, int s) __attribute__((always_inline)) {
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
            const int key = x.key0 + s * kTurn + 16 * half;
            int valid = min(max(x.limit - key, 0), 16);
            const int id = valid ? x.pages.at(key >> a.log_ps) : 0;
            if ((unsigned)id >= (unsigned)a.pages) valid = 0;
            const unsigned char *const at = a.kv + (valid ? id : 0) * a.page_bytes + (((long)x.h << a.log_ps) + (key & ps1)) * D * 2;
            const __amdgpu_buffer_rsrc_t kb = buffer_of(at, valid * D * 2), vb = buffer_of(at + (a.page_bytes >> 1), valid * D * 2);
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) to.k[half][c] = __builtin_amdgcn_raw_buffer_load_b128(kb, k_off[c], 0, kOnce);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (DP == 64) {
                    const word2_t w = __builtin_amdgcn_raw_buffer_load_b64(vb, v_off[e], 0, kOnce);
                    to.v[half][e][0] = word4_t{w[0], w[1], 0, 0};
                } else {
#pragma unroll
                    for (int c = 0; c < Step<DP>::kV; ++c) to.v[half][e][c] = __builtin_amdgcn_raw_buffer_load_b128(vb, v_off[e] + 16 * c, 0, kOnce);
                }
            }
        }
    };

    float4_t o[J];
    float m, l;
    int least;                                                // what every row of the piece sees
    auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < J; ++j) o[j] = float4_t{0, 0, 0, 0};
        m = kNoScore;
        l = 0;
        least = cur.t >= 0 ? cur.sees : cur.limit;
#pragma unroll
        for (int x = 8; x; x >>= 1) least = min(least, __shfl_xor(least, x));
        least = uniform(least);
    };
    auto hide = [&](float4_t (&z)[kHalves], int key) __attribute__((always_inline)) {
#pragma unroll
        for (int half = 0; half < kHalves; ++half)
#pragma unroll
            for (int y = 0; y < 4; ++y)
                if (key + 16 * half + 4 * grp + y >= cur.sees) z[half][y] = -INFINITY;
    };
    // scores of a turn into weights, the operands of the second product; maximum, sum and what was summed before go along
    auto weigh = [&](float4_t (&z)[kHalves], uint32_t (&p)[2 * kHalves]) __attribute__((always_inline)) {
        float top = -INFINITY;
#pragma unroll
        for (int half = 0; half < kHalves; ++half) top = fmaxf(top, fmaxf(fmaxf(z[half][0], z[half][1]), fmaxf(z[half][2], z[half][3])));
        top = larger_of_16(top);
        top = larger_of_32(top) * a.scale;
        if (__ballot(top > m + kSlack)) {
            const float to = fmaxf(top, m), by = __builtin_amdgcn_exp2f(m - to);
            l *= by;
#pragma unroll
            for (int j = 0; j < J; ++j) o[j] *= by;
            m = to;
        }
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                z[half][y] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[half][y], a.scale, -m));
                l += z[half][y];
            }
            p[2 * half] = TY::pack(z[half][0], z[half][1]);
            p[2 * half + 1] = TY::pack(z[half][2], z[half][3]);
        }
    };
    auto turned = [&](uint32_t lo, uint32_t hi, int j) __attribute__((always_inline)) { return __builtin_amdgcn_perm(hi, lo, j & 1 ? 0x07060302u : 0x05040100u); };   // two keys of feature j
    auto add = [&](const uint32_t (&vt)[2 * kHalves], const uint32_t (&p)[2 * kHalves], float4_t to) __attribute__((always_inline)) {
        if constexpr (kHalves == 2) return TY::mfma(word4_t{vt[0], vt[1], vt[2], vt[3]}, word4_t{p[0], p[1], p[2], p[3]}, to);
        else return TY::mfma(word2_t{vt[0], vt[1]}, word2_t{p[0], p[1]}, to);
    };
    auto compute = [&](const Step<DP> &x, int s) __attribute__((always_inline)) {
        float4_t z[kHalves];
        float top = -INFINITY;
        const int key = cur.key0 + s * kTurn;
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
            z[half] = float4_t{0, 0, 0, 0};
#pragma unroll
            for (int y = 0; y < DP / 32; ++y) z[half] = TY::mfma(x.k[half][y], cur.q[y], z[half]);
        }
        if (key + kTurn > least) {
#pragma unroll
            for (int half = 0; half < kHalves; ++half)
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    if (key + 16 * half + 4 * grp + y >= cur.sees) z[half][y] = -INFINITY;
        }
#pragma unroll
        for (int half = 0; half < kHalves; ++half) top = fmaxf(top, fmaxf(fmaxf(z[half][0], z[half][1]), fmaxf(z[half][2], z[half][3])));
        top = larger_of_16(top);
        top = larger_of_32(top) * a.scale;
        if (__ballot(top > m + kSlack)) {
            const float to = fmaxf(top, m), by = __builtin_amdgcn_exp2f(m - to);
            l *= by;
#pragma unroll
            for (int j = 0; j < J; ++j) o[j] *= by;
            m = to;
        }
        uint32_t p[2 * kHalves];
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                z[half][y] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[half][y], a.scale, -m));
                l += z[half][y];
            }
            p[2 * half] = TY::pack(z[half][0], z[half][1]);
            p[2 * half + 1] = TY::pack(z[half][2], z[half][3]);
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            uint32_t vt[2 * kHalves];
#pragma unroll
            for (int y = 0; y < 2 * kHalves; ++y) {           // two keys of feature j
                const uint32_t lo = x.v[y >> 1][2 * (y & 1)][j >> 3][(j & 7) >> 1], hi = x.v[y >> 1][2 * (y & 1) + 1][j >> 3][(j & 7) >> 1];
                vt[y] = __builtin_amdgcn_perm(hi, lo, j & 1 ? 0x07060302u : 0x05040100u);
            }
            if constexpr (kHalves == 2) o[j] = TY::mfma(word4_t{vt[0], vt[1], vt[2], vt[3]}, word4_t{p[0], p[1], p[2], p[3]}, o[j]);
            else o[j] = TY::mfma(word2_t{vt[0], vt[1]}, word2_t{p[0], p[1]}, o[j]);
        }
    };
    // AGAIN: a turn, all of it from memory.  Rows that see equally many of its keys together, the values that they do not see as zeros, the sums of the others left as they are.
    auto compute_again = [&](int s) __attribute__((always_inline)) {
        const int key = cur.key0 + s * kTurn;
        // keys (or values) key + 16 half .. of which the first `end - 16 half` count
        auto sixteen = [&](int half, int end, bool values) __attribute__((always_inline)) {
            const int k = key + 16 * half;
            int valid = min(max(min(cur.limit - key, end) - 16 * half, 0), 16);
            const int id = valid ? uniform(cur.pages.list[k >> a.log_ps]) : 0;
            if ((unsigned)id >= (unsigned)a.pages) valid = 0;
            return buffer_of(a.kv + (valid ? id : 0) * a.page_bytes + (values ? a.page_bytes >> 1 : 0) + (((long)cur.h << a.log_ps) + (k & ps1)) * D * 2, valid * D * 2);
        };
        float4_t z[kHalves];
#pragma unroll
        for (int half = 0; half < kHalves; ++half) {
            const __amdgpu_buffer_rsrc_t from = sixteen(half, kTurn, false);
            z[half] = float4_t{0, 0, 0, 0};
#pragma unroll
            for (int y = 0; y < DP / 32; ++y) z[half] = TY::mfma(__builtin_amdgcn_raw_buffer_load_b128(from, k_off[y], 0, 0), cur.q[y], z[half]);
        }
        hide(z, key);
        uint32_t p[2 * kHalves];
        weigh(z, p);
        const int mine = min(max(cur.sees - key, 0), kTurn);
        for (unsigned long long left = __ballot(mine > 0); left;) {
            const int seen = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
            left &= ~__ballot(mine == seen);
#pragma unroll
            for (int j = 0; j < J; j += 2) {                  // two features at a time: a word of a value's row
                uint32_t lo[2 * kHalves], hi[2 * kHalves];
#pragma unroll
                for (int y = 0; y < 2 * kHalves; ++y) {
                    const __amdgpu_buffer_rsrc_t from = sixteen(y >> 1, seen, true);
                    lo[y] = __builtin_amdgcn_raw_buffer_load_b32(from, v_off[2 * (y & 1)] + 2 * j, 0, 0);
                    hi[y] = __builtin_amdgcn_raw_buffer_load_b32(from, v_off[2 * (y & 1) + 1] + 2 * j, 0, 0);
                }
#pragma unroll
                for (int k = j; k < j + 2; ++k) {
                    uint32_t vt[2 * kHalves];
#pragma unroll
                    for (int y = 0; y < 2 * kHalves; ++y) vt[y] = turned(lo[y], hi[y], k);
                    const float4_t sum = add(vt, p, o[k]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[k][i] = mine == seen ? sum[i] : o[k][i];
                }
                __builtin_amdgcn_sched_barrier(0);            // (few registers before speed)
            }
        }
    };
    bool again = false;
    bool first = true;
    auto finish = [&]() __attribute__((always_inline)) {
        if (!AGAIN && least < min(cur.limit, cur.key0 + cur.n * kFewTile)) {  // (else every row sees all that the piece has)
            float odd = 0;
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) odd = __builtin_fmaf(o[j][i], 0.0f, odd);
            again |= __ballot(cur.t >= 0 && odd != 0) != 0;
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (together) {                                       // then the first one joins them: a fourth of the parts to write and read again
            float *const at = reinterpret_cast<float *>(room) + lane;
            int *const flags = reinterpret_cast<int *>(room + kFewParts<DP>);
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
        const int d0 = 4 * J * grp, head = cur.h * a.group + member;
        if (whole && !to.o) {
            const float by = l == 0 ? 0.0f : 1.0f / l;
            uint16_t *const at = a.out + cur.t * a.out_stride + head * D + d0;
#pragma unroll
            for (int c = 0; c < J / 2; ++c) {                 // eight features: elements 8 c .. of o[j][i] in the order J i + j
                word4_t w;
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int e = 8 * c + 2 * y;
                    w[y] = TY::pack(o[e % J][e / J] * by, o[(e + 1) % J][(e + 1) / J] * by);
                }
                if (d0 + 8 * c < D) *reinterpret_cast<word4_t *>(at + 8 * c) = w;
            }
            if (a.lse && grp == 0) a.lse[(long)cur.t * a.heads + head] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
        } else {
            const long r = whole ? (long)cur.t * a.heads + head : ((long)worker * 2 + (first ? 0 : 1)) * a.slot_rows + col;
            float *const at = to.o + r * D + d0;
#pragma unroll
            for (int c = 0; c < J; ++c) {
                float4_t w;
#pragma unroll
                for (int y = 0; y < 4; ++y) w[y] = o[(4 * c + y) % J][(4 * c + y) / J];
                if (d0 + 4 * c < D) *reinterpret_cast<float4_t *>(at + 4 * c) = w;
            }
            if (grp == 0) to.ml[r] = make_float2(m, l);
        }
    };

    prepare(cur);
    if (cur.n == 0) {                                         // (no tokens in the item, or in this worker's part)
        begin();
        finish();
        return again;
    }
    bool more = follow(cur, behind);
    if constexpr (AGAIN) {
        while (true) {
            begin();
            for (int s = 0; s < cur.n * kTurns; ++s) compute_again(s);
            finish();
            if (!more) return false;
            first = false;
            cur = behind;
            prepare(cur);
            more = follow(cur, behind);
        }
    }
    // A step's loads go out before the step before it is worked on, those of a piece's first step too: page list and queries of the piece behind come while the one
    // before runs.
    if (more) prepare(behind);
    Step<DP> x0, x1;
    load(x0, cur, 0);
    begin();
    int s = 0;
    auto turn = [&](const Step<DP> &now, Step<DP> &next) __attribute__((always_inline)) {
        if (s + 1 < cur.n * kTurns) load(next, cur, s + 1);
        else if (more) load(next, behind, 0);
        compute(now, s);
        if (++s < cur.n * kTurns) return false;
        finish();
        if (!more) return true;
        first = false;
        cur = behind;
        s = 0;
        more = follow(cur, behind);
        if (more) prepare(behind);
        begin();
        return false;
    };
    while (!turn(x0, x1) && !turn(x1, x0)) {}
    return again;
}

// Block `block` of the few-row work, kFewWaves waves.
template <class TY, int DP>
__device__ __forceinline__ void attend_few(const AttendArgs &a, int block, unsigned char *room)
{
    if (!attend_few_wave<TY, DP, false>(a, block, room)) return;
    asm volatile("" : "+s"(block) : : "memory");              // (what was worked out from it, or read, the first time takes no registers until the second)
    attend_few_wave<TY, DP, true>(a, block, room);
}

}  // namespace fbq

#endif
