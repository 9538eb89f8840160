// Attention of a few query rows against a long row of the cache: decode steps, and short prefixes of a shared prompt.
//
// An item is one key/value head of one table row: up to 16 query rows (its query tokens times the heads that share it) against the row's keys and values, which
// are read once.  Bound by HBM: 2 x 2 D bytes a key, for 4 D flops a query row and key.  A step is 32 keys; all steps of all items form one line, which the waves
// of the grid cut into equal pieces - lengths lie on the device, the line is laid out from them by a scan in each wave - so that one long row among short ones
// occupies the whole GPU and no host value decides the cut.  A piece of an item leaves partial results for the join kernel; an item that lies
// within one piece is written at once.
//
// Keys and values go from memory to registers to the matrix cores, nothing through LDS, and waves wait for nobody.  S^T = K Q^T puts a key's scores in rows and a
// query row in a column: v_mfma_f32_16x16x32, operand A lane l key l % 16, features 8 (l / 16) and up of 32, which is how keys lie in memory.  The result has
// column l % 16, keys 4 (l / 16) + i: a lane's eight probabilities of a step are keys 4 g .. 4 g + 3 and 16 + 4 g .. of group g = l / 16.  O^T = V^T P^T
// takes them as operand B where they are, since the order of a contraction is free: V^T's lanes take the same eight keys.  A lane loads DP / 16
// features (l % 16 being the piece) of its eight keys and turns them by byte permutes; row l % 16 of the j-th product is then feature (DP / 16) (l % 16) + j, and
// a lane's results are DP / 4 features in a row of one query row.  The scale by exp(m_old - m_new) is the lane's own.
#include "fbq_attend.h"
#include "fbq_lds_copy.h"

namespace fbq {

constexpr int kNowhere = 1 << 30;             // an offset behind every descriptor's end: loads answer zero

// Cache policy of a load, nt: what is read once takes no room from what is read again (16 rows of about 1000 tokens, 32 heads: 55 us, 62 without it).
constexpr int kOnce = 2;

template <int DP>
struct Step {
    static constexpr int kV = DP == 256 ? 2 : 1;              // 16-byte loads of a lane's features of one value row (DP 64: one of 8 bytes)
    word4_t k[2][DP / 32];
    word4_t v[2][4][kV];
};

template <class TY, int DP>
__global__ __launch_bounds__(64 * kFewWaves, DP == 256 ? 1 : 2) void fbq_attend_few_kernel(const AttendArgs a)
{
    constexpr int J = DP / 16;                                // features of a lane's value pieces, and products O^T of a step
    const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const int worker = uniform(blockIdx.x * kFewWaves + (threadIdx.x >> 6));
    const int D = a.D, ps1 = (1 << a.log_ps) - 1;

    int own = 0;
    for (int b = lane; b < a.rows; b += 64) own += few_steps(a, b);
#pragma unroll
    for (int o = 32; o; o >>= 1) own += __shfl_xor(own, o);
    const int shared_steps = a.shared_here ? (a.n_shared + kFewTile - 1) / kFewTile : 0;
    const int total = uniform(own + shared_steps) * a.kv_heads;
    const int share = few_share(a, total);
    int u = min(worker, total) * share;                       // (worker * share within an int)
    const int end = min(total, u + share);
    if (u >= end) return;

    int b = -1, h, step, steps, limit = a.n_shared;           // the item that u lies in, its tokens; b -1: the shared ones
    if (u < shared_steps * a.kv_heads) {
        steps = shared_steps;
        h = u / steps;
        step = u - h * steps;
    } else {
        int rest = u - shared_steps * a.kv_heads, before = 0, base = 0, tokens, mine, sum;
        while (true) {
            tokens = base + lane < a.rows ? row_tokens(a, base + lane) : 0;
            mine = base + lane < a.rows ? few_steps(a, base + lane, tokens) : 0;
            sum = mine;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int x = __shfl_up(sum, o);
                if (lane >= o) sum += x;
            }
            if ((long)rest < (long)(before + uniform(__shfl(sum, 63))) * a.kv_heads) break;
            before += uniform(__shfl(sum, 63));
            base += 64;
            if (base >= a.rows) return;                       // (not unless lengths change under the call)
        }
        const int at = __builtin_ctzll(__ballot((long)(before + sum) * a.kv_heads > rest));
        b = base + at;
        steps = __builtin_amdgcn_readlane(mine, at);
        limit = __builtin_amdgcn_readlane(tokens, at);
        rest -= (before + __builtin_amdgcn_readlane(sum, at) - steps) * a.kv_heads;
        h = rest / steps;
        step = rest - h * steps;
    }

    // offsets of this lane's loads from a half step's first key, or value
    int k_off[DP / 32], v_off[4];
#pragma unroll
    for (int s = 0; s < DP / 32; ++s) k_off[s] = 32 * s + 8 * grp < D ? (col * D + 32 * s + 8 * grp) * 2 : kNowhere;
#pragma unroll
    for (int e = 0; e < 4; ++e) v_off[e] = J * col < D ? ((4 * grp + e) * D + J * col) * 2 : kNowhere;

    bool first = true;
    while (u < end) {
        const int n = min(end - u, steps - step);
        const bool is_shared = b < 0;

        const int key0 = (is_shared ? 0 : a.n_shared) + step * kFewTile;
        PageList pages;
        pages.begin(is_shared ? a.shared : a.table + (long)b * a.max_pages, is_shared ? a.n_shared >> a.log_ps : a.max_pages, key0 >> a.log_ps);

        // this lane's query row (column `col`): token, head, how many tokens it sees
        int t = -1, sees = 0;
        const int i = col / a.group, head = h * a.group + col - i * a.group;
        if (is_shared) {
            if (i < a.T) {
                const int row = a.q_start ? row_of_token(a.q_start, a.rows, i) : i;
                if (row >= 0) {
                    const int2 q = queries_of(a, row);
                    if (i - q.x < q.y) {
                        t = i;
                        sees = min(row_tokens(a, row) - q.y + i - q.x + 1, limit);
                    }
                }
            }
        } else {
            const int2 q = queries_of(a, b);
            if (i < q.y) {
                t = q.x + i;
                sees = limit - q.y + i + 1;
            }
        }
        word4_t qf[DP / 32];
#pragma unroll
        for (int s = 0; s < DP / 32; ++s) {
            const int d = 32 * s + 8 * grp;
            qf[s] = word4_t{0, 0, 0, 0};
            if (t >= 0 && d < D) qf[s] = (*reinterpret_cast<const word4_t *>(a.q + t * a.q_stride + head * D + d) & a.q_and) ^ a.q_xor;
        }

        auto load = [&](Step<DP> &to, int s) __attribute__((always_inline)) {   // step s of the piece; none past its end
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int key = key0 + s * kFewTile + 16 * half;
                int valid = s < n ? min(max(limit - key, 0), 16) : 0;
                const int id = valid ? pages.at(key >> a.log_ps) : 0;
                if ((unsigned)id >= (unsigned)a.pages) valid = 0;
                const unsigned char *const at = a.kv + (valid ? id : 0) * a.page_bytes + (((long)h << a.log_ps) + (key & ps1)) * D * 2;
                const __amdgpu_buffer_rsrc_t kb = buffer_of(at, valid * D * 2), vb = buffer_of(at + (a.page_bytes >> 1), valid * D * 2);
#pragma unroll
                for (int x = 0; x < DP / 32; ++x) to.k[half][x] = __builtin_amdgcn_raw_buffer_load_b128(kb, k_off[x], 0, kOnce);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (DP == 64) {
                        const word2_t w = __builtin_amdgcn_raw_buffer_load_b64(vb, v_off[e], 0, kOnce);
                        to.v[half][e][0] = word4_t{w[0], w[1], 0, 0};
                    } else {
#pragma unroll
                        for (int x = 0; x < Step<DP>::kV; ++x) to.v[half][e][x] = __builtin_amdgcn_raw_buffer_load_b128(vb, v_off[e] + 16 * x, 0, kOnce);
                    }
                }
            }
        };

        float4_t o[J];
#pragma unroll
        for (int j = 0; j < J; ++j) o[j] = float4_t{0, 0, 0, 0};
        float m = kNoScore, l = 0;
        int least;                                            // what every row sees
        auto compute = [&](const Step<DP> &x, int s) __attribute__((always_inline)) {
            float4_t z[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                z[half] = float4_t{0, 0, 0, 0};
#pragma unroll
                for (int y = 0; y < DP / 32; ++y) z[half] = TY::mfma(x.k[half][y], qf[y], z[half]);
            }
            const int key = key0 + s * kFewTile;
            if (key + kFewTile > least) {
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (key + 16 * half + 4 * grp + y >= sees) z[half][y] = -INFINITY;
            }
            float top = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])));
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            top *= a.scale;
            if (__ballot(top > m + kSlack)) {
                const float to = fmaxf(top, m), by = __builtin_amdgcn_exp2f(m - to);
                l *= by;
#pragma unroll
                for (int j = 0; j < J; ++j) o[j] *= by;
                m = to;
            }
            word4_t p;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
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
                word4_t vt;
#pragma unroll
                for (int y = 0; y < 4; ++y) {                 // two keys of feature j
                    const uint32_t lo = x.v[y >> 1][2 * (y & 1)][j >> 3][(j & 7) >> 1], hi = x.v[y >> 1][2 * (y & 1) + 1][j >> 3][(j & 7) >> 1];
                    vt[y] = __builtin_amdgcn_perm(hi, lo, j & 1 ? 0x07060302u : 0x05040100u);
                }
                o[j] = TY::mfma(vt, p, o[j]);
            }
        };

        Step<DP> x0, x1;
        load(x0, 0);
        least = t >= 0 ? sees : limit;
#pragma unroll
        for (int o = 8; o; o >>= 1) least = min(least, __shfl_xor(least, o));
        least = uniform(least);
        for (int s = 0; s < n; s += 2) {
            load(x1, s + 1);
            compute(x0, s);
            if (s + 1 < n) {
                load(x0, s + 2);
                compute(x1, s + 1);
            }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);

        if (t >= 0) {
            const bool whole = n == steps;
            const Partials to = whole ? (is_shared ? a.whole_shared : a.whole) : a.piece;
            const int d0 = 4 * J * grp;
            if (whole && !to.o) {
                const float by = l == 0 ? 0.0f : 1.0f / l;
                uint16_t *const at = a.out + t * a.out_stride + head * D + d0;
#pragma unroll
                for (int c = 0; c < J / 2; ++c) {             // eight features: elements 8 c .. of o[j][i] in the order J i + j
                    word4_t w;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int e = 8 * c + 2 * y;
                        w[y] = TY::pack(o[e % J][e / J] * by, o[(e + 1) % J][(e + 1) / J] * by);
                    }
                    if (d0 + 8 * c < D) *reinterpret_cast<word4_t *>(at + 8 * c) = w;
                }
                if (a.lse && grp == 0) a.lse[(long)t * a.heads + head] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
            } else {
                const long r = whole ? (long)t * a.heads + head : ((long)worker * 2 + (first ? 0 : 1)) * a.slot_rows + col;
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
        }

        first = false;
        u += n;
        step += n;
        if (u < end && step == steps) {                       // (u < end: some item with steps follows)
            step = 0;
            if (++h == a.kv_heads) {
                h = 0;
                do {
                    if (++b >= a.rows) return;
                    limit = uniform(row_tokens(a, b));
                    steps = uniform(few_steps(a, b, limit));
                } while (steps == 0);
            }
        }
    }
}

template <class TY>
static hipError_t launch_few(const AttendArgs &a, hipStream_t stream)
{
    const dim3 grid(a.workers / kFewWaves), block(64 * kFewWaves);
    if (a.D <= 64) hipLaunchKernelGGL((fbq_attend_few_kernel<TY, 64>), grid, block, 0, stream, a);
    else if (a.D <= 128) hipLaunchKernelGGL((fbq_attend_few_kernel<TY, 128>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((fbq_attend_few_kernel<TY, 256>), grid, block, 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_attend_few(const AttendArgs &a, int type, hipStream_t stream)
{
    return type == FBQ_F16 ? launch_few<TypeF16>(a, stream) : launch_few<TypeBf16>(a, stream);
}

}  // namespace fbq
