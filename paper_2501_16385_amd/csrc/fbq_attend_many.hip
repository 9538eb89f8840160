// Attention of many query rows: prompts, pieces of prompts, and a shared prefix against the rows of a whole batch.
//
// A block has 128 rows (query tokens times the heads that share a key/value head, so grouped heads share what is read) of one key/value head, 32 a wave, and
// goes through the keys 64 at a time: copies of the next 64 keys and values go straight to LDS while these are worked on.  Bound by the matrix cores and, nearly
// as much, by the exponentials: 4 D flops and one exponential a pair.  S^T = K Q^T and O^T = V^T P^T in v_mfma_f32_32x32x16: a lane's column is its query
// row throughout, so the running maximum and sum, the rescaling and P stay in the lane (two lanes share a row), and the probabilities of a step
// are operand B of the second product where the first one left them: keys 16 x + 4 g + (0 .. 3) and 16 x + 8 + 4 g + (0 .. 3) of lane group g = l / 32; the transposed
// reads of V from LDS take their keys in that order.  Rows of a tile end where their last query token's sight ends; later tiles, which see
// more, come first.  Where rows x heads leave the GPU empty the keys are cut into `splits` and the join kernel adds up.
#include "fbq_attend.h"
#include "fbq_lds_copy.h"

namespace fbq {

constexpr int kNowhere = 1 << 30;

// Piece (16 bytes) p of a key's row lies at p ^ key_swap: 16 (or 8) consecutive rows' equal pieces fall on different banks.  A value's row at p ^ value_swap: the four rows
// of a transposed read, 32 bytes each for 16 lanes, do.
__device__ __forceinline__ int key_swap(int row, int pieces) { return pieces == 8 ? piece_key(row) : row & 15; }
__device__ __forceinline__ int value_swap(int row, int pieces) { return pieces == 8 ? 2 * (row & 3) : (4 * (row & 3)) ^ (row & 2); }

__device__ __forceinline__ word2_t read_turned4(const unsigned char *at)
{
    typedef short four_t __attribute__((vector_size(8)));
    typedef __attribute__((address_space(3))) four_t lds_four_t;
    return __builtin_bit_cast(word2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_four_t *)(__attribute__((address_space(3))) const void *)at));
}

template <class TY, int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void fbq_attend_many_kernel(const AttendArgs a, const bool shared)
{
    constexpr int kPieces = DP / 8, kRowBytes = DP * 2, kTileBytes = kManyTile * kRowBytes;
    constexpr int kRowsACopy = 64 / kPieces, kCopies = 16 / kRowsACopy;       // a wave copies 16 keys and 16 values a step
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2][2][kTileBytes];

    const int lane = threadIdx.x & 63, col = lane & 31, grp = lane >> 5, wave = uniform(threadIdx.x >> 6);
    const int D = a.D, ps1 = (1 << a.log_ps) - 1;
    const int h = blockIdx.x, split = blockIdx.z, splits = shared ? a.shared_splits : a.splits;

    // the row of the table and the tile of its query rows (for the shared tokens all query tokens are one row's)
    int b = 0, q0 = 0, nq = a.T, limit = a.n_shared, tile = blockIdx.y;
    if (!shared) {
        if (!a.q_start) {
            const int per = (a.group + kManyRows - 1) / kManyRows;
            b = tile / per;
            tile -= b * per;
            q0 = b;
            nq = 1;
        } else {
            int before = 0, base = 0, mine, sum;
            while (true) {
                mine = base + lane < a.rows ? (queries_of(a, base + lane).y * a.group + kManyRows - 1) / kManyRows : 0;
                sum = mine;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const int x = __shfl_up(sum, o);
                    if (lane >= o) sum += x;
                }
                const int all = uniform(__shfl(sum, 63));
                if (tile < before + all) break;
                before += all;
                base += 64;
                if (base >= a.rows) return;                   // the grid has a block for the most tiles there could be
            }
            const int at = __builtin_ctzll(__ballot(before + sum > tile));
            b = base + at;
            const int tiles = __builtin_amdgcn_readlane(mine, at);
            tile = tiles - 1 - (tile - (before + __builtin_amdgcn_readlane(sum, at) - tiles));
            const int2 q = queries_of(a, b);
            q0 = uniform(q.x);
            nq = uniform(q.y);
        }
        limit = uniform(row_tokens(a, b));
    }

    // this lane's query row: token, head, how many tokens it sees
    const int r = tile * kManyRows + wave * 32 + col, i = r / a.group, head = h * a.group + r - i * a.group;
    int t = -1, sees = 0;
    if (i < nq) {
        if (shared) {
            const int row = a.q_start ? row_of_token(a.q_start, a.rows, i) : i;
            if (row >= 0) {
                const int2 q = queries_of(a, row);
                if (i - q.x < q.y) {
                    t = i;
                    sees = min(row_tokens(a, row) - q.y + i - q.x + 1, limit);
                }
            }
        } else {
            t = q0 + i;
            sees = limit - nq + i + 1;
        }
    }
    int least = t >= 0 ? sees : limit, most = t >= 0 ? sees : 0;              // of the wave's rows
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        least = min(least, __shfl_xor(least, o));
        most = max(most, __shfl_xor(most, o));
    }
    least = uniform(least);
    most = uniform(most);
    if (!shared) limit = max(0, min(limit, limit - nq + min(nq - 1, ((tile + 1) * kManyRows - 1) / a.group) + 1));   // what the block's last row sees

    const int key0 = shared ? 0 : a.n_shared, all_steps = (max(limit - key0, 0) + kManyTile - 1) / kManyTile, per = (all_steps + splits - 1) / splits;
    const int s0 = min(split * per, all_steps), s1 = min(s0 + per, all_steps);

    word4_t qf[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
        const int d = 16 * s + 8 * grp;
        qf[s] = word4_t{0, 0, 0, 0};
        if (t >= 0 && d < D) qf[s] = *reinterpret_cast<const word4_t *>(a.q + t * a.q_stride + head * D + d);
    }

    // where this lane's pieces of a copy come from: rows 16 wave .. of a step
    int k_off[kCopies], v_off[kCopies];
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
        const int row = c * kRowsACopy + lane / kPieces, at = lane % kPieces, kp = at ^ key_swap(row, kPieces), vp = at ^ value_swap(row, kPieces);
        k_off[c] = 8 * kp < D ? row * D * 2 + kp * 16 : kNowhere;
        v_off[c] = 8 * vp < D ? row * D * 2 + vp * 16 : kNowhere;
    }
    const int32_t *const list = shared ? a.shared : a.table + (long)b * a.max_pages;
    const int entries = shared ? a.n_shared >> a.log_ps : a.max_pages;
    auto copy = [&](int step, int buf) __attribute__((always_inline)) {
        const int key = key0 + step * kManyTile + 16 * wave;
        int valid = min(max(limit - key, 0), 16);
        const int id = uniform(list[min(key >> a.log_ps, entries - 1)]);
        if ((unsigned)id >= (unsigned)a.pages) valid = 0;
        const unsigned char *const at = a.kv + (valid ? id : 0) * a.page_bytes + (((long)h << a.log_ps) + (key & ps1)) * D * 2;
        const __amdgpu_buffer_rsrc_t kb = buffer_of(at, valid * D * 2), vb = buffer_of(at + (a.page_bytes >> 1), valid * D * 2);
        const uint32_t to = lds_offset(&lds[buf][0][16 * wave * kRowBytes]);
#pragma unroll
        for (int c = 0; c < kCopies; ++c) copy16_to_lds(kb, k_off[c], 0, to + c * 1024);
#pragma unroll
        for (int c = 0; c < kCopies; ++c) copy16_to_lds(vb, v_off[c], 0, to + kTileBytes + c * 1024);
    };

    // reads: a key's piece s of DP / 16 pairs, and a value's column block dblk of 32
    const int k_at = col * kRowBytes, k_piece = grp ^ key_swap(col, kPieces);
    const int v_row = 4 * grp + ((lane & 15) >> 2), v_at = v_row * kRowBytes + 8 * (lane & 1);
    const int v_piece = (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ value_swap(v_row, kPieces);

    float16_t o[DP / 32];
#pragma unroll
    for (int x = 0; x < DP / 32; ++x)
#pragma unroll
        for (int y = 0; y < 16; ++y) o[x][y] = 0;
    float m = kNoScore, l = 0;

    if (s0 < s1) copy(s0, 0);
    for (int s = s0; s < s1; ++s) {
        const int buf = (s - s0) & 1;
        if (s + 1 < s1) {
            copy(s + 1, buf ^ 1);
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * kCopies) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
        const int key = key0 + s * kManyTile;
        if (key < most) {
            const unsigned char *const kt = lds[buf][0], *const vt = lds[buf][1];
            float16_t z[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int y = 0; y < 16; ++y) z[half][y] = 0;
#pragma unroll
                for (int x = 0; x < DP / 16; ++x) {
                    const word4_t kf = *reinterpret_cast<const word4_t *>(kt + k_at + ((k_piece ^ (2 * x)) << 4) + 32 * half * kRowBytes);
                    z[half] = TY::mfma(kf, qf[x], z[half]);
                }
                z[half] *= a.scale;
            }
            if (key + kManyTile > least) {
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int y = 0; y < 16; ++y)
                        if (key + 32 * half + 8 * (y >> 2) + 4 * grp + (y & 3) >= sees) z[half][y] = -INFINITY;
            }
            float top = fmaxf(z[0][0], z[1][0]);
#pragma unroll
            for (int y = 1; y < 16; ++y) top = fmaxf(top, fmaxf(z[0][y], z[1][y]));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__ballot(top > m)) {
                const float to = fmaxf(top, m), by = __builtin_amdgcn_exp2f(m - to);
                l *= by;
#pragma unroll
                for (int x = 0; x < DP / 32; ++x) o[x] *= by;
                m = to;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    word4_t p;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const float p0 = __builtin_amdgcn_exp2f(z[half][8 * x + 2 * y] - m), p1 = __builtin_amdgcn_exp2f(z[half][8 * x + 2 * y + 1] - m);
                        l += p0 + p1;
                        p[y] = TY::pack(p0, p1);
                    }
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) {
                        const unsigned char *const at = vt + v_at + ((v_piece ^ (4 * d)) << 4) + (32 * half + 16 * x) * kRowBytes;
                        const word2_t lo = read_turned4(at), hi = read_turned4(at + 8 * kRowBytes);
                        o[d] = TY::mfma(word4_t{lo[0], lo[1], hi[0], hi[1]}, p, o[d]);
                    }
                }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");       // all have read: the other buffer's successor may be copied over this one
    }
    l += __shfl_xor(l, 32);

    if (t < 0) return;
    const Partials to = shared ? a.part_shared : a.part;
    const long row = (long)t * a.heads + head;
    if (!to.o) {
        const float by = l == 0 ? 0.0f : 1.0f / l;
        uint16_t *const at = a.out + t * a.out_stride + head * D;
#pragma unroll
        for (int x = 0; x < DP / 32; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int d = 32 * x + 8 * y + 4 * grp;
                if (d < D) *reinterpret_cast<word2_t *>(at + d) = word2_t{TY::pack(o[x][4 * y] * by, o[x][4 * y + 1] * by), TY::pack(o[x][4 * y + 2] * by, o[x][4 * y + 3] * by)};
            }
        if (a.lse && grp == 0) a.lse[row] = l == 0 ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
        return;
    }
    const long at = (long)split * a.T * a.heads + row;
    if (grp == 0) to.ml[at] = make_float2(m, l);
    if (l == 0) return;                                       // (the join does not look at its sums)
#pragma unroll
    for (int x = 0; x < DP / 32; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int d = 32 * x + 8 * y + 4 * grp;
            if (d < D) *reinterpret_cast<float4_t *>(to.o + at * D + d) = float4_t{o[x][4 * y], o[x][4 * y + 1], o[x][4 * y + 2], o[x][4 * y + 3]};
        }
}

template <class TY>
static hipError_t launch_many(const AttendArgs &a, bool shared, hipStream_t stream)
{
    const long rows = (long)a.T * a.group;
    long tiles = (rows + kManyRows - 1) / kManyRows;          // ragged rows: each may have one more, begun
    if (!shared) tiles = a.q_start ? std::min((long)a.T * ((a.group + kManyRows - 1) / kManyRows), tiles + a.rows) : (long)a.rows * ((a.group + kManyRows - 1) / kManyRows);
    const dim3 grid(a.kv_heads, (unsigned)tiles, shared ? a.shared_splits : a.splits), block(256);
    if (a.D <= 64) hipLaunchKernelGGL((fbq_attend_many_kernel<TY, 64>), grid, block, 0, stream, a, shared);
    else if (a.D <= 128) hipLaunchKernelGGL((fbq_attend_many_kernel<TY, 128>), grid, block, 0, stream, a, shared);
    else hipLaunchKernelGGL((fbq_attend_many_kernel<TY, 256>), grid, block, 0, stream, a, shared);
    return hipGetLastError();
}

hipError_t launch_attend_many(const AttendArgs &a, int type, bool shared, hipStream_t stream)
{
    return type == FBQ_F16 ? launch_many<TypeF16>(a, shared, stream) : launch_many<TypeBf16>(a, shared, stream);
}

}  // namespace fbq
