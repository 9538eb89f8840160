// Attention of many query rows: prompts, pieces of prompts, and a shared prefix against the rows of a whole batch.
//
// A block has 128 rows (query tokens times the heads that share a key/value head, so grouped heads share what is read) of one key/value head, 32 a wave, and
// goes through the keys 64 at a time: copies of the next 64 keys and values go straight to LDS while these are worked on.  Bound by the matrix cores and, nearly
// as much, by the exponentials: 4 D flops and one exponential a pair.  S^T = K Q^T and O^T = V^T P^T in v_mfma_f32_32x32x16: a lane's column is its query
// row throughout, so the running maximum and sum, the rescaling and P stay in the lane (two lanes share a row), and the probabilities of a step
// are operand B of the second product where the first one left them: keys 16 x + 4 g + (0 .. 3) and 16 x + 8 + 4 g + (0 .. 3) of lane group g = l / 32; the transposed
// reads of V from LDS take their keys in that order.  Rows of a tile end where their last query token's sight ends; later tiles, which see
// more, come first.  Where rows x heads leave the GPU empty the keys are cut into pieces and the join kernel adds up.
// Measured, 32 heads of 128, fp16: prompt of 8192 tokens 537 to 575 us from card to card (0.96 to 1.02 PFLOP/s; 435 with zeros for data: the matrix cores' power bounds it), 4096 160,
// 2048 50 to 54 (0.63 and more: 512 blocks of unequal length, all at once; eight waves a block instead, two teams on alternating steps, 61.5).  Heads of 64 0.76 to 0.80 PFLOP/s,
// of 80 0.78, of 256 0.76 to 0.80.
#ifndef FBQ_ATTEND_MANY_H
#define FBQ_ATTEND_MANY_H

#include <type_traits>

#include "fbq_attend.h"
#include "fbq_attend_codes.h"
#include "fbq_lds_copy.h"

namespace fbq {

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

// f(0), f(1) .. f(N - 1), each with its number as a constant
template <int N, class F>
__device__ __forceinline__ void each(F f)
{
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(std::integral_constant<int, N - 1>());
    }
}

// A grid has 65535 blocks in y: more tiles than that go on in z, so many at a time.  (That is where a call of shared tokens has their pieces, but not then: it has blocks enough.)
constexpr int kGridTiles = 32768;
inline dim3 many_grid(const AttendArgs &a, bool shared)
{
    const long rows = (long)a.T * a.group, per = (a.group + kManyRows - 1) / kManyRows;
    long tiles = (rows + kManyRows - 1) / kManyRows;          // ragged rows: each may have one more, begun
    if (!shared) tiles = (a.q_start ? std::min(a.T * per, tiles + a.rows) : a.rows * per) * a.splits;
    const bool fits = tiles <= 65535;
    return dim3(a.kv_heads, fits ? (unsigned)tiles : kGridTiles, fits ? (shared ? a.shared_splits : 1) : (unsigned)((tiles + kGridTiles - 1) / kGridTiles));
}

// Bytes of LDS (aligned to 1024) of a block of it.
template <int DP>
constexpr int kManyRoom = 4 * kManyTile * (DP == 96 ? 256 : DP * 2);
template <int DP>
constexpr int kMany4Room = kManyRoom<DP> + 1024;              // (scale words, see Codes)

template <class CODES, class TY>
struct OperandOf { typedef typename CODES::Make::Operand type; };
template <class TY>
struct OperandOf<NoCodes, TY> { typedef TY type; };

// Block (h, y, z) of the many-row work, four waves: head, tile (of the rows' own tokens: tile and piece), piece of the shared tokens.  FOUR: a Codes (fbq_attend_codes.h), where the cache is
// in 4 bits and keys and values are made on their way to LDS; void: it is not.
// `odd`: set where the operands that it makes are not made for what it has met, and its results mean nothing (for the whole block).
template <class TY, int DP, class FOUR = void>
__device__ __forceinline__ void attend_many(const AttendArgs &a, const bool shared, const int h, const int y, const int z, unsigned char *room, bool *odd = nullptr)
{
    constexpr bool kFour = !std::is_void<FOUR>::value;
    typedef typename std::conditional<kFour, FOUR, NoCodes>::type CODES;
    typedef typename OperandOf<CODES, TY>::type OT;           // of the products
    constexpr int kPieces = DP == 96 ? 16 : DP / 8, kRowBytes = kPieces * 16, kTileBytes = kManyTile * kRowBytes;   // (96: rows as long as 128's, so that they fold over the banks)
    constexpr int kRowsACopy = 64 / kPieces, kCopies = 16 / kRowsACopy;       // a wave copies 16 keys and 16 values a step
    unsigned char (*const lds)[2][kTileBytes] = reinterpret_cast<unsigned char (*)[2][kTileBytes]>(room);   // keys, values; two steps each

    int thread = threadIdx.x;
    if constexpr (kFour) asm volatile("" : "+v"(thread));     // (nothing that follows from it is kept in registers for a second time, or another branch of a kernel)
    const int lane = thread & 63, col = lane & 31, grp = lane >> 5, wave = uniform(thread >> 6);
    const int D = a.D, ps1 = (1 << a.log_ps) - 1;

    // the row of the table, the tile of its query rows and the piece of the tile's keys (for the shared tokens all query tokens are one row's)
    int b = 0, q0 = 0, nq = a.T, limit = a.n_shared, tile = y, split = z, splits = a.shared_splits, tokens_of_row = 0;
    if (!shared && !a.q_start && a.rows > 64 && a.splits == 1) {             // many rows of one token: no need to look at all of them in every block
        const int per = many_tiles(a, 1);
        b = y / per;
        if (b >= a.rows) return;                              // (grids of many tiles are rounded up)
        tile = per - 1 - (y - b * per);
        q0 = b;
        nq = 1;
        tokens_of_row = uniform(row_tokens(a, b));
        limit = many_limit(a, tokens_of_row, nq, tile);
        split = 0;
        splits = 1;
    } else if (!shared) {
        const int share = a.splits == 1 ? 1 << 30 : many_share(a);
        int queries, query0, tokens, tiles, pieces, count, longest;   // of the table row that is this lane's
        const auto look = [&](int row) {
            const int2 q = row < a.rows ? queries_of(a, row) : make_int2(0, 0);
            queries = q.y;
            query0 = q.x;
            tokens = row < a.rows ? row_tokens(a, row) : 0;
            tiles = many_tiles(a, queries);
            pieces = many_pieces(a, many_steps(a, tokens), share);
            count = tiles * pieces;
            longest = (many_steps(a, tokens) + pieces - 1) / pieces;
        };
        int all = 0;
        for (int base = (a.rows - 1) & ~63; base >= 0; base -= 64) {          // (the first ones last: they stay in the registers)
            look(base + lane);
            all += __builtin_amdgcn_readlane(wave_scan(count), 63);
        }
        int index = y;
        if (index >= all) return;                             // the grid has a block for the most there could be
        // Long pieces first: the rows by their longest piece where a wave knows them all, the tiles of a row from its last to its first.  Blocks that are all on the GPU at once
        // share CUs two by two, the first with the one half the grid on: then the second half goes from short to long.
        const int half = (all + 1) / 2;
        if (index >= half && (long)all * a.kv_heads <= many_blocks(D)) index = all - 1 - (index - half);
        int offset = 0, base = 0;
        if (a.rows <= 64) {
            for (int x = 0; x < a.rows; ++x) {
                const int other = __builtin_amdgcn_readlane(longest, x);
                if (other > longest || (other == longest && x < lane)) offset += __builtin_amdgcn_readlane(count, x);
            }
        } else {
            int before = 0;
            while (true) {
                look(base + lane);
                const int sum = wave_scan(count), some = __builtin_amdgcn_readlane(sum, 63);
                offset = before + sum - count;
                if (index < before + some) break;
                before += some;
                base += 64;
                if (base >= a.rows) return;                   // (not unless the rows change under the call)
            }
        }
        const int at = __builtin_ctzll(__ballot(count > 0 && offset <= index && index < offset + count));
        b = base + at;
        const int rest = index - __builtin_amdgcn_readlane(offset, at), row_pieces = __builtin_amdgcn_readlane(pieces, at);
        tile = __builtin_amdgcn_readlane(tiles, at) - 1 - rest / row_pieces;
        split = rest % row_pieces;
        nq = __builtin_amdgcn_readlane(queries, at);
        q0 = __builtin_amdgcn_readlane(query0, at);
        tokens_of_row = __builtin_amdgcn_readlane(tokens, at);
        limit = many_limit(a, tokens_of_row, nq, tile);
        splits = many_pieces(a, many_steps(a, limit), share);
        if (split >= splits) return;
    } else if ((long)y * kManyRows >= (long)a.T * a.group) {
        return;
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
            sees = tokens_of_row - nq + i + 1;
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
    const int key0 = shared ? 0 : a.n_shared, all_steps = shared ? (limit + kManyTile - 1) / kManyTile : many_steps(a, limit);
    const int per = (all_steps + splits - 1) / splits;
    const int s0 = min(split * per, all_steps), s1 = min(s0 + per, all_steps);

    const auto query = [&](int t, int grp, int s) __attribute__((always_inline)) {
        const int d = 16 * s + 8 * grp;
        return t >= 0 && d < D ? (*reinterpret_cast<const word4_t *>(a.q + t * a.q_stride + head * D + d) & a.q_and) ^ a.q_xor : word4_t{0, 0, 0, 0};
    };
    word4_t qf[DP / 16];
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) qf[s] = query(t, grp, s);
    float unit = a.scale;                                     // what scores are multiplied by
    if constexpr (kFour) {
        if constexpr (CODES::Make::kScaled) {
            float most = 0;
            const auto each_of = [](uint32_t word, auto f) { return TypeF16::pack(f(CODES::Make::Number::of(word & 0xffff)), f(CODES::Make::Number::of_upper(word))); };
#pragma unroll
            for (int s = 0; s < DP / 16; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) each_of(qf[s][e], [&](float x) { most = fmaxf(most, fabsf(x)); return x; });
            const int up = __builtin_amdgcn_frexp_expf(larger_of_32(most)) - 15;
            unit = ldexpf(unit, up);
#pragma unroll
            for (int s = 0; s < DP / 16; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) qf[s][e] = each_of(qf[s][e], [&](float x) { return ldexpf(x, -up); });
        }
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
    // 16 keys, or values, a wave
    PageList pages;
    CODES codes;
    if constexpr (kFour) {
#pragma unroll
        for (int i = 0; i < 2; ++i) codes.template begin<kPieces>(a, lds[0][i], lds[1][i], room + 4 * kTileBytes, wave, lane);
    }
    auto next_page = [&](int step) __attribute__((always_inline)) { return pages.at((key0 + step * kManyTile + 16 * wave) >> a.log_ps); };
    auto copy = [&](int step, int page, bool values) __attribute__((always_inline)) {
        const int key = key0 + step * kManyTile + 16 * wave;
        const int valid = (unsigned)page < (unsigned)a.pages ? min(max(limit - key, 0), 16) : 0;
        const unsigned char *const at = a.kv + (valid ? page : 0) * a.page_bytes + (values ? a.page_bytes >> 1 : 0) + (((long)h << a.log_ps) + (key & ps1)) * D * 2;
        const __amdgpu_buffer_rsrc_t from = buffer_of(at, valid * D * 2);
        const uint32_t to = lds_offset(&lds[values][step & 1][16 * wave * kRowBytes]);
#pragma unroll
        for (int c = 0; c < kCopies; ++c) copy16_to_lds(from, values ? v_off[c] : k_off[c], 0, to + c * 1024);
    };

    // In 4 bits codes are asked for, and made and put down a step later; behind the last step there are none, and nobody looks at what is put down for it.
    auto ask = [&](int step, int page, bool values) __attribute__((always_inline)) {
        if constexpr (kFour) codes.ask(a, h, page, key0 + step * kManyTile + 16 * wave, step < s1 ? limit : 0, values);
    };
    auto scalar_page = [&](int step) __attribute__((always_inline)) { return page_of(list, (key0 + step * kManyTile + 16 * wave) >> a.log_ps, entries); };
    auto put = [&](int share, int step) __attribute__((always_inline)) {      // of the values of `step` and the keys of the one behind it
        if constexpr (kFour) {
            if (share % codes.kWords == 0) codes.spread(share == 0);
            if (share < codes.kWords) codes.put_values(share, lds[1][step & 1]);
            else codes.put_keys(share - codes.kWords, lds[0][(step + 1) & 1]);
        }
    };
    // reads: a key's piece s of DP / 16 pairs, and a value's column block dblk of 32
    int k_at = col * kRowBytes, k_piece = grp ^ key_swap(col, kPieces);
    const int v_row = 4 * grp + ((lane & 15) >> 2);
    int v_at = v_row * kRowBytes + 8 * (lane & 1);
    int v_piece = (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ value_swap(v_row, kPieces);

    float16_t o[DP / 32];
#pragma unroll
    for (int x = 0; x < DP / 32; ++x)
#pragma unroll
        for (int y = 0; y < 16; ++y) o[x][y] = 0;
    float m = kNoScore, l = 0;

    // A step is a row of slots with one matrix product each, first the next step's scores (kScores products, the two halves of its keys in turn), then this step's P V (kValues,
    // 16 keys at a time).  Every slot asks LDS for the operand of the one kAhead slots on, and carries a share of the step's other work, which the compiler is kept from
    // moving: exponentials of pair k of probabilities (in time for its product), and towards the end the maximum of the next step's scores.
    constexpr int kScores = DP / 8, kValues = DP / 8, kAhead = kFour ? 2 : 4 /* (4 bits: registers for more run out) */, kLate = 12;
    word4_t ring[kAhead];
    auto fetch = [&](int i, int step) __attribute__((always_inline)) {        // operand of slot i of the step `step`
        if (i < kScores) {
            const int half = i & 1, x = i >> 1;
            ring[i % kAhead] = *reinterpret_cast<const word4_t *>(lds[0][(step + 1) & 1] + k_at + ((k_piece ^ (2 * x)) << 4) + 32 * half * kRowBytes);
        } else if (i < kScores + kValues) {
            const int j = (i - kScores) / (DP / 32), d = (i - kScores) % (DP / 32);
            if constexpr (kFour) {
                ring[i % kAhead] = *reinterpret_cast<const word4_t *>(lds[1][step & 1] + turned_at(32 * d + col, 2 * j + grp));
                return;
            }
            const unsigned char *const at = lds[1][step & 1] + v_at + ((v_piece ^ (4 * d)) << 4) + 16 * j * kRowBytes;
            const word2_t lo = read_turned4(at), hi = read_turned4(at + 8 * kRowBytes);
            ring[i % kAhead] = word4_t{lo[0], lo[1], hi[0], hi[1]};
        }
    };
    int page = 0;                                             // of the keys copied last
    float top = -INFINITY;                                    // of this lane's scores of the step that is next
    auto work = [&](float16_t (&z)[2], float16_t (&ahead)[2], int s) __attribute__((always_inline)) {
        if constexpr (kFour) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // what was asked for a step ago is there, what a step ago was read is free
        if constexpr (!kFour) {
            if (s + 1 < s1) copy(s + 1, page, true);
            if (s + 2 < s1) {
                page = next_page(s + 2);
                copy(s + 2, page, false);
            }
        }
        int next = 0, behind = 0;                             // 4 bits: pages of the values and keys that are asked for at this step's end
        if constexpr (kFour) {
            next = scalar_page(s + 2);
            behind = scalar_page(s + 3);
        }
        const int key = key0 + s * kManyTile;
        if (key >= most) {
            if constexpr (kFour) {
#pragma unroll
                for (int x = 0; x < 2 * codes.kWords; ++x) put(x, s + 1);
                ask(s + 2, next, true);
                ask(s + 3, behind, false);
            }
            return;
        }
        // 256 features: all addresses of a step in registers across steps would push others out to memory, whose loads wait for the copies under way
        if constexpr (DP == 256) asm volatile("" : "+v"(k_at), "+v"(k_piece), "+v"(v_at), "+v"(v_piece));
        if constexpr (kFour) codes.step();
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(i, s);         // (past the last step: of whatever lies there, its scores are not used)
        if (key + kManyTile > least) {
            top = -INFINITY;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int y = 0; y < 16; ++y) {
                    if (key + 32 * half + 8 * (y >> 2) + 4 * grp + (y & 3) >= sees) z[half][y] = -INFINITY;
                    top = fmaxf(top, z[half][y]);
                }
        }
        const float high = larger_of_32(top) * unit;
        if (__ballot(high > m + kSlack)) {
            const float to = fmaxf(high, m), by = __builtin_amdgcn_exp2f(m - to);
            l *= by;
#pragma unroll
            for (int x = 0; x < DP / 32; ++x) o[x] *= by;
            m = to;
        }
        word4_t p[4];
        auto pair = [&](int k) __attribute__((always_inline)) {
            const int half = k >> 3, y = 2 * (k & 7);
            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[half][y], unit, -m)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[half][y + 1], unit, -m));
            l += p0 + p1;
            p[k >> 2][k & 3] = OT::pack(p0, p1);
        };
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int y = 0; y < 16; ++y) ahead[half][y] = 0;
        each<kScores + kValues>([&](auto slot) __attribute__((always_inline)) {
            constexpr int i = decltype(slot)::value;
            __builtin_amdgcn_sched_barrier(0);
            const word4_t f = ring[i % kAhead];
            if constexpr (i < kScores) {
                ahead[i & 1] = OT::mfma(f, qf[i >> 1], ahead[i & 1]);
#pragma unroll
                for (int k = 0; k < kLate; ++k)
                    if (k * kScores / kLate == i) pair(k);
            } else {
                constexpr int x = i - kScores, j = x / (DP / 32), d = x % (DP / 32);
                o[d] = OT::mfma(f, p[j], o[d]);
#pragma unroll
                for (int k = kLate; k < 16; ++k)
                    if ((k - kLate) * (kValues / 2) / (16 - kLate) == x) pair(k);
#pragma unroll
                for (int y = 0; y < 16; ++y)
                    if (kValues / 2 + y * (kValues / 2) / 16 == x) top = y == 0 ? fmaxf(ahead[0][0], ahead[1][0]) : fmaxf(fmaxf(top, ahead[0][y]), ahead[1][y]);
            }
            fetch(i + kAhead, s);
            // shares of codes in the second half of the step: what was asked for in the one before has had three quarters of one to come
            if constexpr (kFour) {
                constexpr int kShares = 2 * FOUR::kWords, kHalf = (kScores + kValues) / 2;
#pragma unroll
                for (int k = 0; k < kShares; ++k)
                    if (kHalf + k * kHalf / kShares == i) {
                        put(k, s + 1);
                        if (k == FOUR::kWords - 1) ask(s + 2, next, true);
                    }
            }
        });
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (kFour) ask(s + 3, behind, false);
    };
    // Keys are a step ahead of values: while step s is worked on, keys s + 1 and values s are read, keys s + 2 and values s + 1 copied.
    float16_t z0[2], z1[2];
    if (s0 < s1) {
        if constexpr (kFour) {
            const int page0 = scalar_page(s0), page1 = scalar_page(s0 + 1);
            ask(s0, page0, false);
#pragma unroll
            for (int x = 0; x < codes.kWords; ++x) put(codes.kWords + x, s0 - 1);
            ask(s0, page0, true);
            ask(s0 + 1, page1, false);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
            for (int x = 0; x < 2 * codes.kWords; ++x) put(x, s0);
            ask(s0 + 1, page1, true);
            ask(s0 + 2, scalar_page(s0 + 2), false);
        } else {
            pages.begin(list, entries, (key0 + s0 * kManyTile + 16 * wave) >> a.log_ps);
            page = next_page(s0);
            copy(s0, page, false);
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            copy(s0, page, true);
            if (s0 + 1 < s1) {
                page = next_page(s0 + 1);
                copy(s0 + 1, page, false);
            }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int y = 0; y < 16; ++y) z0[half][y] = 0;
#pragma unroll
        for (int i = 0; i < kScores; ++i) {
            fetch(i, s0 - 1);
            z0[i & 1] = OT::mfma(ring[i % kAhead], qf[i >> 1], z0[i & 1]);
        }
#pragma unroll
        for (int y = 0; y < 16; ++y) top = fmaxf(fmaxf(top, z0[0][y]), z0[1][y]);
    }
    for (int s = s0; s < s1; s += 2) {
        work(z0, z1, s);
        if (s + 1 < s1) work(z1, z0, s + 1);
    }
    const auto write = [&](float16_t (&o)[DP / 32], float m, float l) __attribute__((always_inline)) {
        l += __shfl_xor(l, 32);
        if (t < 0) return;
        const Partials to = shared ? a.part_shared : a.part;
        const long row = (long)t * a.heads + head;
        if (!shared && splits == 1 && !a.part_shared.o) {
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
        if (l == 0) return;                                   // (the join does not look at its sums)
#pragma unroll
        for (int x = 0; x < DP / 32; ++x)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int d = 32 * x + 8 * y + 4 * grp;
                if (d < D) *reinterpret_cast<float4_t *>(to.o + at * D + d) = float4_t{o[x][4 * y], o[x][4 * y + 1], o[x][4 * y + 2], o[x][4 * y + 3]};
            }
    };
    // A value that is no number times the zero of a row that does not see it is none either, and stays in that row's sums.  Where such a sum is found and some row does not see all
    // keys, the wave does its piece again, by itself and from memory: rows that see equally many of a step's keys together, other values as zeros, the others' sums left as they are.
    // Slow (a prompt of 2048 with a NaN among its values 430 us, else 52), but only then: otherwise the look at the sums is all.  (Results are written before, and once more: so the
    // loop's registers are as they would be without.  256 features, a prompt of 8192: 1448 us, 1428 without.)
    if constexpr (kFour) {
        if (CODES::Make::kChecked) {
            int *const flags = reinterpret_cast<int *>(room);
            __syncthreads();                                  // (tiles are read no more)
            if (lane == 0) flags[wave] = codes.met != 0;
            __syncthreads();
            *odd = uniform(flags[0] | flags[1] | flags[2] | flags[3]) != 0;
            __syncthreads();
        }
    }
    bool again = false;
    if (!kFour && least < min(limit, key0 + s1 * kManyTile)) {
        float odd = 0;                                        // then not zero
#pragma unroll
        for (int x = 0; x < DP / 32; ++x)
#pragma unroll
            for (int y = 0; y < 16; ++y) odd = __builtin_fmaf(o[x][y], 0.0f, odd);
        again = __ballot(t >= 0 && odd != 0) != 0;
    }
    write(o, m, l);
    if (!again || kFour) return;         // (a cache in 4 bits has no such values)
    float16_t sums[DP / 32];
#pragma unroll
    for (int x = 0; x < DP / 32; ++x)
#pragma unroll
        for (int y = 0; y < 16; ++y) sums[x][y] = 0;
    m = kNoScore;
    l = 0;
    for (int s = s0; s < s1; ++s) {
        const int key = key0 + s * kManyTile;
        if (key >= most) break;
        int asked = t, at_col = col, at_grp = grp;
        asm volatile("" : "+v"(asked), "+v"(at_col), "+v"(at_grp));   // (queries from memory and offsets anew every step: few registers before speed, here and below)
        // keys (or values) key + 16 c .. of which the first `end - 16 c` count
        auto sixteen = [&](int c, int end, bool values) __attribute__((always_inline)) {
            int valid = min(max(min(limit - key, end) - 16 * c, 0), 16);
            const int page = valid ? uniform(list[(key + 16 * c) >> a.log_ps]) : 0;
            if ((unsigned)page >= (unsigned)a.pages) valid = 0;
            return buffer_of(a.kv + (valid ? page : 0) * a.page_bytes + (values ? a.page_bytes >> 1 : 0) + (((long)h << a.log_ps) + ((key + 16 * c) & ps1)) * D * 2, valid * D * 2);
        };
        float16_t z[2];
        float high = -INFINITY;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const __amdgpu_buffer_rsrc_t lower = sixteen(2 * half, kManyTile, false), upper = sixteen(2 * half + 1, kManyTile, false);
#pragma unroll
            for (int y = 0; y < 16; ++y) z[half][y] = 0;
#pragma unroll
            for (int x = 0; x < DP / 16; ++x) {
                const int d = 16 * x + 8 * at_grp, off = d < D ? ((at_col & 15) * D + d) * 2 : kNowhere;
                const word4_t f = __builtin_amdgcn_raw_buffer_load_b128(lower, at_col < 16 ? off : kNowhere, 0, 0) |
                                  __builtin_amdgcn_raw_buffer_load_b128(upper, at_col < 16 ? kNowhere : off, 0, 0);
                z[half] = TY::mfma(f, query(asked, at_grp, x), z[half]);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int y = 0; y < 16; ++y) {
                if (key + 32 * half + 8 * (y >> 2) + 4 * grp + (y & 3) >= sees) z[half][y] = -INFINITY;
                high = fmaxf(high, z[half][y]);
            }
        }
        high = larger_of_32(high) * a.scale;
        if (__ballot(high > m + kSlack)) {
            const float to = fmaxf(high, m), by = __builtin_amdgcn_exp2f(m - to);
            l *= by;
#pragma unroll
            for (int x = 0; x < DP / 32; ++x) sums[x] *= by;
            m = to;
        }
        word4_t p[4];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int half = k >> 3, y = 2 * (k & 7);
            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[half][y], a.scale, -m)), p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(z[half][y + 1], a.scale, -m));
            l += p0 + p1;
            p[k >> 2][k & 3] = TY::pack(p0, p1);
        }
        const int mine = min(max(sees - key, 0), kManyTile);
        for (unsigned long long left = __ballot(mine > 0); left;) {
            const int seen = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
            left &= ~__ballot(mine == seen);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
                float16_t sum = sums[d];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const __amdgpu_buffer_rsrc_t from = sixteen(j, seen, true);
                    word4_t f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {         // keys 8 (w / 2) + 4 grp + 2 (w % 2) and the next of the sixteen, feature 32 d + col
                        const int off = ((8 * (w >> 1) + 4 * at_grp + 2 * (w & 1)) * D + 32 * d + at_col) * 2;
                        f[w] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(from, off, 0, 0) | (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(from, off + D * 2, 0, 0) << 16;
                    }
                    sum = TY::mfma(f, p[j], sum);
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int y = 0; y < 16; ++y) sums[d][y] = mine == seen ? sum[y] : sums[d][y];
            }
        }
    }
    write(sums, m, l);
}

}  // namespace fbq

#endif
