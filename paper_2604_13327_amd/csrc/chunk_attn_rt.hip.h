// What the chunk attentions share (over pools of bf16 and of 8 bits): how a call is cut into pieces, softmax and second product,
// values that are no numbers, page ids, partial results and their join.
#pragma once
#include <type_traits>

#include "serving_rt.hip.h"

namespace etc {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) short s16x2;

constexpr int kCaWaves = 8, kCaThreads = kCaWaves * 64;
static_assert(kCaRows == 32 * kCaWaves, "32 rows to a wavefront");
// Items of no more than kCaWholeTiles are not cut, nor is a cut estimated.  Whole and as the estimate has it, in us, calls back to back:
//   tiles of the longest                          5           6           7           9          10          12          14
//   3 single tokens, 4 heads of 64 on 2        9.9  11.4   9.9  11.5  10.8  11.4  11.6  12.4  11.8  12.0  12.7  12.4  13.6  12.8
//   3 single tokens, 32 heads of 128 on 8     12.7  14.0  12.7  14.0  14.4  14.1  15.8  15.2  15.9  15.1  17.5  15.3  19.1  16.5
//   1 single token, 64 heads of 128 on 8      12.6  14.0  12.0  13.4  14.2  14.1  15.7  15.1  15.1  14.4  16.6  15.3  18.3  16.2
// With caches turned over between calls: at 6 tiles 13.0 14.5, 17.2 17.8, 16.6 17.0, at 7 tiles 13.9 15.1, 18.9 17.7, 18.9 17.4.  Eight
// prompts of 20 to 40 tokens, which are estimated and then not cut, lose 1.2 us by the estimate.
constexpr int kCaNarrowRows = 64, kCaNarrowKeys = 128;
constexpr float kCaNoReference = -3e38f;     // of a row that has seen no key yet

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float partner_max(float x)      // with lane + 32
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float partner_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A bf16 that is no number, as a count (bf16): +inf 1, -inf 2^8, NaN 2^16; 0 for a number.
__device__ __forceinline__ uint32_t odd_kind(uint32_t e)
{
    return (e & 0x7FFFu) > 0x7F80u ? 0x4780u : e == 0x7F80u ? 0x3F80u : e == 0xFF80u ? 0x4380u : 0u;
}

__device__ __forceinline__ int last_not_above(ETC_AS_LDS const int *indptr, int n, int x)      // the last b with indptr[b] <= x
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (indptr[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// ---- how a call is cut into pieces ---------------------------------------------------------------------------------------
// An item is (sequence, block of rows, KV head).  Its keys are cut into pieces of at most L tiles, about equal ones, with the L out of
// kCaTries that is estimated to end first; every workgroup computes this by itself from the lengths, one sequence to a thread.  A
// sequence's long blocks come first, and workgroups take pieces forwards and backwards in turn, so that their sums come out about
// equal: a chunk of 4096 (32 heads of 128 on 8, 512 pieces of 1 to 64 tiles) takes 145 us, 188 where every workgroup takes piece w + 256
// after piece w, 164 from a queue of pieces.  Where there are more pieces than workgroups, sequences of at most kCaNarrowRows rows (narrow ones) go by
// length, and their pieces are spread among the others': the former are bound by memory, the latter by LDS and matrix units, and those
// at the same time are faster than one after the other.  (64 single tokens take 7 % less than as they come, 32 of them with a prompt of
// 1000 9 %, 30 with two prompts 2 %, and those 25 % more with all narrow ones in front.)  KV heads are the fastest index of a piece:
// neighbouring workgroups, on different dies, take different heads, and a die's L2 sees the keys of one or two.
constexpr int kCaTries = kCaWaves;          // a wavefront estimates one
constexpr int kCaClasses = 8;               // of sequences: narrow ones by length, then the others

struct Seq { int q0, n, kv; };             // first row, new tokens, cached ones

struct CaLds {
    int q0[kServingMaxSeqs], n[kServingMaxSeqs], kv[kServingMaxSeqs];      // n == 0: nothing to do
    int split[kServingMaxSeqs];             // pieces of the longest item
    uint16_t order[kServingMaxSeqs];        // the sequences in the order of their pieces
    int first[kServingMaxSeqs + 1];         // prefix sum, in that order: pieces of the sequences
    int slot[kServingMaxSeqs + 1];          // prefix sum: those that leave a partial result
    float wave_f[kCaWaves];
    int wave_i[kCaClasses / 2][kCaWaves];
    int limit, narrow_limit;                // tiles of a piece; of one of a narrow sequence, where those have a price of their own
    int narrow;                             // pieces of narrow sequences, which are in front (0: in any order)
    int odd, last;
    float try_f[kCaWaves];                  // candidates of a cut with prices of its own
    int try_i[2][kCaWaves];
};

__device__ __forceinline__ int div_up(int a, int b) { return (a + b - 1) / b; }
__device__ __forceinline__ int blocks_of(int n, int grp) { return div_up(n * grp, kCaRows); }                    // n * grp <= 2^26
__device__ __forceinline__ int tiles_of(int kv, int n) { return n > 0 ? (kv + n - 1) / kCaKeys + 1 : 0; }        // of the last block
__device__ __forceinline__ int wave_max_i(int v)
{
    v = max(v, dpp_i32<0xB1>(v));
    v = max(v, dpp_i32<0x4E>(v));
    v = max(v, dpp_i32<0x141>(v));
    v = max(v, dpp_i32<0x140>(v));
    return max(max(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)), max(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

// What a cut is estimated with: candidates of a piece's length, in workgroups' shares, and (OWN) prices of what narrow and wide sequences ask for,
// in wide tiles; without OWN those are as cut() has them.
struct CutPrices {
    static constexpr bool OWN = false;
    static constexpr int WHOLE = kCaWholeTiles;          // tiles of an item up to which none is cut
    static __device__ __forceinline__ float factor(int w) { return w == 1 ? 4.f : w == 2 ? 3.f : w == 3 ? 2.f : w == 4 ? 1.5f : w == 5 ? 1.25f : w == 6 ? 1.1f : 1.f; }
};

// Fills L and returns the number of pieces.
template <int OP, class Prices = CutPrices>
__device__ __forceinline__ int cut(const ServingDev &S, const etc_serving_attention_io &io, ETC_AS_LDS CaLds &L)
{
    const int tid = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), grp = S.nq / S.nkv, grid = (int)gridDim.x;
    float work = 0.f;                                    // tiles, all items
    int tokens = 0, most = 0;                            // at most 2^30; tiles of an item
    for (int b = tid; b < io.n_seqs; b += kCaThreads) {
        const int q0 = gld_i32(io.q_indptr + b), q1 = gld_i32(io.q_indptr + b + 1), kv = gld_i32(io.kv_len + b);
        int n = q1 - q0;
        if (q0 < 0 || q1 < q0 || q1 > io.n_tokens || kv < 0 || kv > S.max_kv_len || n > S.max_kv_len - kv ||
            (int)(((unsigned)(kv + n) + (1u << S.page_shift) - 1) >> S.page_shift) > io.table_cols) {
            if (blockIdx.x == 0) refuse(S.error, SRV_BAD_LENGTH, OP, b, kv);
            n = 0;
        }
        L.q0[b] = q0;
        L.n[b] = n;
        L.kv[b] = kv;
        tokens += n;
        most = max(most, tiles_of(kv, n));
        if (n > 0) {
            float tiles = (float)S.nkv * blocks_of(n, grp) * 0.5f * (float)(tiles_of(kv, n) + tiles_of(kv, min(n, kCaRows / grp)));
            if constexpr (Prices::OWN) tiles *= Prices::tile(n * grp <= kCaNarrowRows);
            work += tiles;
        }
    }
    work = wave_sum(work);
    tokens = wave_sum_i(tokens);
    most = wave_max_i(most);
    if (lane == 0) { L.wave_f[wave] = work; L.wave_i[0][wave] = tokens; L.wave_i[1][wave] = most; }
    __syncthreads();
    work = 0.f;
    tokens = 0;
#pragma unroll
    for (int w = 0; w < kCaWaves; ++w) { work += L.wave_f[w]; tokens += L.wave_i[0][w]; most = max(most, L.wave_i[1][w]); }
    if (tokens > io.n_tokens) {                          // ranges that overlap: no call's lengths
        if (blockIdx.x == 0 && tid == 0) refuse(S.error, SRV_BAD_LENGTH, OP, io.n_seqs, tokens);
        return 0;
    }
    // Candidate of wavefront w: no cut, or pieces of 4, 3, 2, 1.5, 1.25, 1.1, 1 times a workgroup's share, kCaMinTiles at least.  In tiles
    // (1.8 us): a piece costs its tiles and 1 more; a call ends with its longest piece or, where some workgroup takes several, after as
    // many of them; the last join then reads half a tile's time a part, and 9 more where a whole block is joined.  Fitted to the times of
    // all candidates in 17 calls (1 to 64 sequences, chunks of 1 to 8192, caches to 32768): what it chooses is 0.8 % behind the fastest
    // in the mean, 3 % at worst.  The shortest pieces are the fastest for 30 sequences with two prompts (66 us, 81 without a cut), the
    // longest for one token of one sequence (18 and 58), 1.1 for a chunk of 512 behind 8000 keys (89 and 242).
    const float share = work / (float)grid;
    auto limit_of = [&](int w) {
        return w == 0 ? 1 << 30 : max(kCaMinTiles, (int)fminf(ceilf(share * Prices::factor(w)), 1e9f));
    };
    auto narrow_limit_of = [&](int w) {
        if constexpr (Prices::OWN) return w == 0 ? 1 << 30 : max(kCaMinTiles, (int)fminf(ceilf(share * Prices::factor(w) * (1.f / Prices::tile(true))), 1e9f));
        else return limit_of(w);
    };
    int best = 0, longest_piece = most;
    int longest_narrow = 0;                              // (OWN; longest_piece is that of wide sequences then)
    if (most > Prices::WHOLE) {
        float pieces = 0.f, slots = 0.f;
        int longest = 0, parts = 1;
        bool whole = false;
        float ends;
        const int per = limit_of(wave);
        if constexpr (!Prices::OWN) {
            for (int b = lane; b < io.n_seqs; b += 64) {
                const int n = L.n[b], tiles = tiles_of(L.kv[b], n);
                if (n == 0) continue;
                const int blocks = blocks_of(n, grp), s = div_up(tiles, per);
                const float k = (float)S.nkv * blocks, some = 0.5f * (float)(s + div_up(tiles_of(L.kv[b], min(n, div_up(kCaRows, grp))), per));
                pieces += k * some;
                if (s > 1) { slots += k * s; whole |= n * grp > kCaNarrowRows; }
                parts = max(parts, s);
                longest = max(longest, div_up(tiles, s));
            }
            pieces = wave_sum(pieces);
            slots = wave_sum(slots);
            longest = wave_max_i(longest);
            parts = wave_max_i(parts);
            ends = fmaxf((float)longest + 1.f, ceilf(pieces / (float)grid) * ((work + pieces) / fmaxf(pieces, 1.f))) + 0.5f * (float)parts + (__any(whole) ? 9.f : 0.f);
        } else {
            const int narrow_per = narrow_limit_of(wave);
            int narrow_parts = 1;
            float over = 0.f, longest_cost = 0.f;
            for (int b = lane; b < io.n_seqs; b += 64) {
                const int n = L.n[b], tiles = tiles_of(L.kv[b], n);
                if (n == 0) continue;
                const bool narrow = n * grp <= kCaNarrowRows;
                const int blocks = blocks_of(n, grp), p = narrow ? narrow_per : per, s = div_up(tiles, p), len = div_up(tiles, s);
                const float k = (float)S.nkv * blocks, some = k * 0.5f * (float)(s + div_up(tiles_of(L.kv[b], min(n, div_up(kCaRows, grp))), p));
                const float each = Prices::piece(narrow) + (s > 1 ? Prices::part(narrow) : 0.f);
                pieces += some;
                over += some * each;
                if (s > 1) slots += k * s;
                if (narrow) { narrow_parts = max(narrow_parts, s); longest_narrow = max(longest_narrow, len); }
                else { parts = max(parts, s); longest = max(longest, len); }
                longest_cost = fmaxf(longest_cost, (float)len * Prices::alone(narrow) + each);
            }
            pieces = wave_sum(pieces);
            slots = wave_sum(slots);
            longest = wave_max_i(longest);
            longest_narrow = wave_max_i(longest_narrow);
            parts = wave_max_i(parts);
            narrow_parts = wave_max_i(narrow_parts);
            over = wave_sum(over);
            longest_cost = wave_max_f(longest_cost);
            const float all = work + over;
            ends = fmaxf(longest_cost, pieces > (float)grid ? all * (1.f / (float)grid) + Prices::left(all / pieces) : 0.f) +
                   fmaxf(parts > 1 ? Prices::join(false, parts) : 0.f, narrow_parts > 1 ? Prices::join(true, narrow_parts) : 0.f);
        }
        if (wave > 0 && slots > (float)S.attn_slots) ends = INFINITY;
        if constexpr (!Prices::OWN) {
            __syncthreads();
            if (lane == 0) { L.wave_f[wave] = ends; L.wave_i[0][wave] = longest; }
            __syncthreads();
            float best_ends = L.wave_f[0];
#pragma unroll
            for (int w = 1; w < kCaTries; ++w)
                if (L.wave_f[w] < best_ends) { best = w; best_ends = L.wave_f[w]; }
            longest_piece = L.wave_i[0][best];
        } else {                                         // a candidate to a lane: no cut if that is best, of other equals the shorter pieces
            if (lane == 0) { L.try_f[wave] = ends; L.try_i[0][wave] = longest; L.try_i[1][wave] = longest_narrow; }
            __syncthreads();
            const int w = min(lane, kCaTries - 1);
            const float mine = L.try_f[w];
            const int mine_longest = L.try_i[0][w], mine_narrow = L.try_i[1][w];
            const uint32_t bests = (uint32_t)__builtin_amdgcn_ballot_w64(mine == -wave_max_f(-mine)) & ((1u << kCaTries) - 1);
            best = (bests & 1) ? 0 : 31 - __builtin_clz(bests);
            longest_piece = __builtin_amdgcn_readlane(mine_longest, best);
            longest_narrow = __builtin_amdgcn_readlane(mine_narrow, best);
        }
    } else {
        longest_narrow = most;
    }
    const int limit = limit_of(best), narrow_limit = narrow_limit_of(best);
    if (tid == 0) { L.first[0] = L.slot[0] = 0; L.limit = limit; L.narrow_limit = narrow_limit; L.narrow = 0; }
    auto class_of = [](bool narrow, int most_of, int len) {      // (OWN: half of the classes for each kind)
        return (narrow ? 0 : kCaClasses / 2) + max(0, min(kCaClasses / 2 - 1, (int)((float)(kCaClasses / 2 * (most_of - len)) / (float)max(most_of, 1))));
    };
    if constexpr (Prices::OWN) {
        // Up to 64 sequences: what follows, by one wavefront in registers, a sequence to a lane (2 to 3 us of a call that has ranks).
        if (io.n_seqs <= 64) {
            if (wave == 0) {
                const bool there = lane < io.n_seqs;
                const int n = there ? L.n[lane] : 0, tiles = there ? tiles_of(L.kv[lane], n) : 0;
                const bool narrow = n * grp <= kCaNarrowRows;
                const int parts = max(1, div_up(tiles, narrow ? narrow_limit : limit)), k = S.nkv * blocks_of(n, grp) * parts;
                int rank = lane, wide = 0;
                if (wave_sum_i(k) > grid && io.n_seqs > 1) {
                    const int cls = class_of(narrow, narrow ? longest_narrow : longest_piece, div_up(tiles, parts));
                    const uint64_t in_front = (1ull << lane) - 1;
                    int above = 0;
#pragma unroll
                    for (int j = 0; j < kCaClasses; ++j) {
                        const uint64_t of_it = __builtin_amdgcn_ballot_w64(there && cls == j);
                        if (cls == j) rank = above + __builtin_popcountll(of_it & in_front);
                        above += __builtin_popcountll(of_it);
                        if (j >= kCaClasses / 2) wide += __builtin_popcountll(of_it);
                    }
                }
                if (there) {
                    L.split[lane] = parts;
                    L.order[rank] = (uint16_t)lane;
                }
                in_order();
                const int b = there ? (int)L.order[lane] : lane, pieces = __shfl(k, b, 64), cut = __shfl(parts, b, 64) > 1 ? pieces : 0;
                const int upto = wave_scan_i(pieces), slots_upto = wave_scan_i(cut);
                if (there) { L.first[lane + 1] = upto; L.slot[lane + 1] = slots_upto; }
                if (wide > 0 && lane == io.n_seqs - wide) L.narrow = upto - pieces;
            }
            __syncthreads();
            return __builtin_amdgcn_readfirstlane(L.first[io.n_seqs]);
        }
    }
    auto count = [&](auto as_they_come) {                // the prefix sums; the number of pieces
        int done = 0, done_slots = 0;
        for (int i0 = 0; i0 < io.n_seqs; i0 += kCaThreads) {
            const int i = i0 + tid;
            int k = 0, sl = 0;
            __syncthreads();
            if (i < io.n_seqs) {
                int b = i, parts;
                if (as_they_come) {
                    parts = max(1, div_up(tiles_of(L.kv[i], L.n[i]), Prices::OWN && L.n[i] * grp <= kCaNarrowRows ? narrow_limit : limit));
                    L.order[i] = (uint16_t)i;
                    L.split[i] = parts;
                } else {
                    b = L.order[i];
                    parts = L.split[b];
                }
                k = S.nkv * blocks_of(L.n[b], grp) * parts;      // all together at most 2^20 tokens * 1024 heads / 256 rows + 2^20, and attn_slots
                sl = parts > 1 ? k : 0;
            }
            int sum = wave_scan_i(k), sum_sl = wave_scan_i(sl);
            if (lane == 63) { L.wave_i[0][wave] = sum; L.wave_i[1][wave] = sum_sl; }
            __syncthreads();
            for (int w = 0; w < wave; ++w) { sum += L.wave_i[0][w]; sum_sl += L.wave_i[1][w]; }
            if (i < io.n_seqs) { L.first[i + 1] = done + sum; L.slot[i + 1] = done_slots + sum_sl; }
            for (int w = 0; w < kCaWaves; ++w) { done += L.wave_i[0][w]; done_slots += L.wave_i[1][w]; }
        }
        return done;
    };
    int n_pieces = count(std::true_type());
    if (n_pieces > grid && io.n_seqs > 1) {
        // Ranks: classes by length in sevenths of the longest piece, within a class as they come.  Two classes' counts to a word.
        int before[2][kCaClasses / 2], total[kCaClasses / 2] = {}, cls[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int b = c * kCaThreads + tid, rows = b < io.n_seqs ? L.n[b] * grp : 0;
            const int len = rows > 0 ? div_up(tiles_of(L.kv[b], L.n[b]), L.split[b]) : 0;
            if constexpr (Prices::OWN) {
                cls[c] = class_of(rows <= kCaNarrowRows, rows > kCaNarrowRows ? longest_piece : longest_narrow, len);
            } else {
                cls[c] = rows > kCaNarrowRows ? kCaClasses - 1 : min(kCaClasses - 2, (int)((float)((kCaClasses - 1) * (longest_piece - len)) / (float)longest_piece));
            }
            if (c * kCaThreads >= io.n_seqs) break;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kCaClasses / 2; ++j) {
                const int mine = b < io.n_seqs && cls[c] >> 1 == j ? 1 << (cls[c] & 1) * 16 : 0;
                before[c][j] = wave_scan_i(mine);
                if (lane == 63) L.wave_i[j][wave] = before[c][j];
                before[c][j] += total[j] - mine;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kCaClasses / 2; ++j)
                for (int w = 0; w < kCaWaves; ++w) {
                    if (w < wave) before[c][j] += L.wave_i[j][w];
                    total[j] += L.wave_i[j][w];
                }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int b = c * kCaThreads + tid;
            if (b >= io.n_seqs) break;
            int rank = 0;
#pragma unroll
            for (int j = 0; j < kCaClasses; ++j) {
                const int shift = (j & 1) * 16;
                if (j < cls[c]) rank += (total[j >> 1] >> shift) & 0xFFFF;
                else if (j == cls[c]) rank += (before[c][j >> 1] >> shift) & 0xFFFF;
            }
            L.order[rank] = (uint16_t)b;
        }
        n_pieces = count(std::false_type());
        __syncthreads();
        int wide = total[kCaClasses / 2 - 1] >> 16;      // sequences
        if constexpr (Prices::OWN) {
            wide = 0;
#pragma unroll
            for (int j = kCaClasses / 4; j < kCaClasses / 2; ++j) wide += (total[j] >> 16) + (total[j] & 0xFFFF);
        }
        if (tid == 0) L.narrow = L.first[io.n_seqs - wide];
    }
    __syncthreads();
    return n_pieces;
}

// Partial results of a slot, wavefront by wavefront: [16-byte piece of a lane][lane] of the output, then m and l of 32 rows.
template <int D> constexpr int kCaPartO = D / 32 * 4 * 64 * 4;      // floats of a wavefront
template <int D> constexpr int kCaSlot = kCaWaves * (kCaPartO<D> + 64);

// ---- the products --------------------------------------------------------------------------------------------------------
// Rows of K and V in LDS, D elements without gaps; their 16-byte pieces change places with the row (exclusive or), so that the
// lanes of an access meet different banks (64 of 4 bytes): 16 rows of one piece of K, 4 rows of 4 pieces of V.  Rows of 64
// elements are half as wide as the banks: there two neighbouring rows share their places.
template <int D> __device__ __forceinline__ int k_swap(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D> __device__ __forceinline__ int v_swap(int row) { return D == 128 ? (row & 3) * 4 : (row & 2) * 2; }

template <int D>
struct Fragments {                          // LDS byte addresses of this lane's pieces in a tile that starts at 0
    uint32_t k[D / 16], v[D / 32];
    __device__ __forceinline__ Fragments(int lane)
    {
        const int half = lane >> 5, col = lane & 31, vrow = 4 * half + ((lane & 15) >> 2), piece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) k[ks] = col * D * 2 + ((ks * 2 + half) ^ k_swap<D>(col)) * 16;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) v[dt] = vrow * D * 2 + ((dt * 4 + piece) ^ v_swap<D>(vrow)) * 16 + (lane & 1) * 8;
    }
    // V^T fragment of 32 elements (tile dt) x 16 keys (step ks), the keys in the order the scores have them: rows 4 half + 0 .. 3
    // and 8 + 4 half + 0 .. 3 of the step.
    __device__ __forceinline__ u32x4 v_frag(uint32_t base, int ks, int dt) const
    {
        ETC_AS_LDS char *at = reinterpret_cast<ETC_AS_LDS char *>(v[dt] + base) + ks * 16 * D * 2;
        const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ETC_AS_LDS s16x4 *>(at)));
        const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ETC_AS_LDS s16x4 *>(at + 8 * D * 2)));
        return u32x4{a.x, a.y, b.x, b.y};
    }
};

// Softmax of a tile's scores and O^T += V^T . P^T.  l is this lane's sum, over half of the keys.
// MASKED: keys behind `limit` do not count; their rows of V hold numbers (odd_values has seen to that).
// The second product takes bf16.  Blocks of many rows (KT 2) round probabilities to it: half a unit of each, 2^-8 of the sum of p |v| at
// most and, where that sum is much larger than the result, more than the result's own rounding; l sums what was rounded, so that equal
// values come out as they are.  A second part there is exact to 2^-15 and costs 38 % (4001 tokens behind 30000 keys 3849 -> 5304 us).
// Blocks of few rows (KT 1), which wait for memory, take both parts, for up to 1 % (64 single tokens over 2000 to 4000 keys 145.7 -> 146.5
// us, 16 sequences of 5 tokens 52.1 -> 52.4, three short ones 9.7 -> 10.1).  The upper part there is below the probability, so that the
// rest is positive too: an infinity of V times either part has one sign (with probabilities above 2^-103; the rest of smaller ones can
// be less than a bf16 holds).
template <int D, int KT, bool MASKED>
__device__ __forceinline__ void attend(f32x16 (&s)[KT], f32x16 (&o)[D / 32], float &m, float &l, const Fragments<D> &F, uint32_t base,
                                       int half, float scale, int k0, int limit)
{
    constexpr int DT = D / 32;
    constexpr bool SPLIT = KT == 1;
    if constexpr (MASKED) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (k0 + kt * 32 + 8 * (i >> 2) + 4 * half + (i & 3) > limit) s[kt][i] = -INFINITY;
    }
    // V's fragments a step ahead of their products: the first ones while the maximum is found
    u32x4 w[2][DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) w[0][dt] = F.v_frag(base, 0, dt);
    float mt = s[0][0];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mt = fmaxf(mt, s[kt][i]);
    mt = partner_max(mt) * scale;
    // The reference follows the maximum only when that has grown by 2^8 (rows of a wavefront together): until then
    // probabilities up to 2^8 lose nothing, and the running output need not be multiplied.  A row's first reference multiplies nothing:
    // the output is 0 until then but for infinities of this very tile (odd_values), which a factor of 0 would make NaN.
    if (__builtin_amdgcn_ballot_w64(mt > m + 8.f) != 0) {
        const float nm = fmaxf(m, mt), sc = MASKED && m == kCaNoReference ? 1.f : exp2_fast(m - nm);
        m = nm;
        l *= sc;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= sc;
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int step = kt * 2 + h;
            u32x4 p, rest;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = exp2_fast(__builtin_fmaf(s[kt][8 * h + 2 * i], scale, -m)), b = exp2_fast(__builtin_fmaf(s[kt][8 * h + 2 * i + 1], scale, -m));
                if constexpr (SPLIT) {
                    const uint32_t ah = __builtin_elementwise_sub_sat(__float_as_uint(a), 1u), bh = __builtin_elementwise_sub_sat(__float_as_uint(b), 1u);
                    p[i] = __builtin_amdgcn_perm(bh, ah, 0x07060302u);
                    rest[i] = to_bf16x2(a - __uint_as_float(ah & 0xFFFF0000u), b - __uint_as_float(bh & 0xFFFF0000u));
                    l += a + b;
                } else {
                    const uint32_t both = to_bf16x2(a, b);
                    p[i] = both;
                    l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(s16x2, both), __builtin_bit_cast(s16x2, 0x3F803F80u), l, false);
                }
            }
            if (step + 1 < 2 * KT) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) w[(step + 1) & 1][dt] = F.v_frag(base, step + 1, dt);
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w[step & 1][dt]), __builtin_bit_cast(bf16x8, p), o[dt], 0, 0, 0);
            if constexpr (SPLIT) {                           // behind all of the first parts': none waits for the one in front of it
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w[step & 1][dt]), __builtin_bit_cast(bf16x8, rest), o[dt], 0, 0, 0);
            }
        }
}

// Values of V that are no numbers, in a tile that some rows see a part of: the probability 0 of what a row does not see would make a
// NaN of them.  They are counted by kind, in a product over the keys each row sees (+inf as 1, -inf as 2^8, NaN as 2^16, at most 64 of
// each: exact), which goes to the output as infinities and NaN; the tile then holds zeros in their place.  `mine` are the pieces of the tile this
// thread looks after, at the LDS addresses at[]; the wavefront's rows see the KEYS keys from k0 on, at `base`.  For the whole workgroup.
template <int D, int KEYS, int N>
__device__ __forceinline__ void odd_values(const u32x4 (&mine)[N], const uint32_t (&at)[N], f32x16 (&o)[D / 32], const Fragments<D> &F, uint32_t base, int half, int k0, int limit, bool live)
{
#pragma unroll
    for (int u = 0; u < N; ++u) {
        u32x4 kind;
#pragma unroll
        for (int i = 0; i < 4; ++i) kind[i] = odd_kind(mine[u][i] & 0xFFFFu) | odd_kind(mine[u][i] >> 16) << 16;
        *reinterpret_cast<ETC_AS_LDS u32x4 *>(at[u]) = kind;
    }
    __syncthreads();
    if (live) {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) {
            f32x16 n{};
#pragma unroll 1
            for (int ks = 0; ks < KEYS / 16; ++ks) {
                const u32x4 w = F.v_frag(base, ks, dt);
                u32x4 seen;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = k0 + ks * 16 + 4 * half + (i >> 1) * 8 + (i & 1) * 2;
                    seen[i] = (key <= limit ? 0x3F80u : 0u) | (key + 1 <= limit ? 0x3F800000u : 0u);
                }
                n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, seen), n, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t c = (uint32_t)n[i];
                if (c & 0xFFu) o[dt][i] += INFINITY;
                if (c & 0xFF00u) o[dt][i] -= INFINITY;
                if (c >> 16) o[dt][i] = __uint_as_float(0x7FC00000u);
                __builtin_amdgcn_sched_barrier(0);           // one after the other: the conditions of all at once fill 600 scalar registers, and
            }                                                // the lanes of eleven vector registers of the whole kernel with them (10 % of a long prompt)
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < N; ++u) {
        u32x4 w = mine[u];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] &= ((w[i] & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((w[i] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
        *reinterpret_cast<ETC_AS_LDS u32x4 *>(at[u]) = w;
    }
    __syncthreads();
}

__device__ __forceinline__ bool any_odd(u32x4 v)          // an exponent of all ones among 8 values
{
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= (v[i] & 0x7F80u) == 0x7F80u || (v[i] & 0x7F800000u) == 0x7F800000u;
    return odd;
}

// Rows go from memory to LDS without a stop in registers: 64 lanes, 16 bytes each, to 1 KB of LDS from `to` on (the same for the
// whole wavefront).  The compiler would have every LDS read wait for all such loads in flight; here their order is the
// program's own: arrived(n) waits until at most n of this wavefront's are on their way, a barrier then covers everyone's.
// The place goes by m0, which an asm statement cannot name among what it overwrites (it is reserved): it is put back.
#define ETC_FETCH_1K(address, ...)                                                                                                     \
    do {                                                                                                                               \
        int m0_;                                                                                                                       \
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 " address "\n\ts_mov_b32 m0, %0"        \
                     : "=&s"(m0_) : "s"(__builtin_amdgcn_readfirstlane(to)), __VA_ARGS__ : "memory");                                  \
    } while (0)
template <bool ONCE> __device__ __forceinline__ void fetch_1k(const char *from, uint32_t to)
{
    if (ONCE) ETC_FETCH_1K("%2, off nt", "v"(from));
    else ETC_FETCH_1K("%2, off", "v"(from));
}
template <bool ONCE> __device__ __forceinline__ void fetch_1k(const char *base, uint32_t lane_off, uint32_t to)      // base the same for the wavefront
{
    if (ONCE) ETC_FETCH_1K("%2, %3 nt", "v"(lane_off), "s"(base));
    else ETC_FETCH_1K("%2, %3", "v"(lane_off), "s"(base));
}
#undef ETC_FETCH_1K
// 64 lanes, a byte each, to 64 words of LDS from `to` on.
__device__ __forceinline__ void fetch_bytes(const uint8_t *from, uint32_t to)
{
    int m0_;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ubyte %2, off\n\ts_mov_b32 m0, %0" : "=&s"(m0_) : "s"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "memory");
}
template <int N> __device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0)" : : "i"(N) : "memory"); }

constexpr int kCaIds = 1024;                // page ids in LDS, a window of them at a time

struct Piece {
    int b, kvh, part, parts;                // part `part` of an item that has `parts` of them
    int slot0;                              // slot of part 0 (part j: j * nkv behind it)
    int tile0, tile1;                       // of the piece: [tile0, tile1)
    int n_keys;                             // that the last row of the block sees
    int grp, rows, r0;                      // query heads per KV head; rows of (sequence, KV head); first one of the block
    Seq seq;
};

template <class Prices>
__device__ __forceinline__ Piece piece_of(const ServingDev &S, const etc_serving_attention_io &io, ETC_AS_LDS const CaLds &L, int p)
{
    const int i = __builtin_amdgcn_readfirstlane(last_not_above(L.first, io.n_seqs, p)), local = p - __builtin_amdgcn_readfirstlane(L.first[i]);
    Piece P;
    P.b = __builtin_amdgcn_readfirstlane((int)L.order[i]);
    P.seq = wave_uniform(Seq{L.q0[P.b], L.n[P.b], L.kv[P.b]});
    const int split = __builtin_amdgcn_readfirstlane(L.split[P.b]);
    P.kvh = local % S.nkv;
    P.part = local / S.nkv % split;
    P.slot0 = __builtin_amdgcn_readfirstlane(L.slot[i]) + local - P.part * S.nkv;
    P.grp = S.nq / S.nkv;
    P.rows = P.seq.n * P.grp;
    P.r0 = (blocks_of(P.seq.n, P.grp) - 1 - local / S.nkv / split) * kCaRows;      // long blocks first
    P.n_keys = P.seq.kv + min(P.r0 + kCaRows - 1, P.rows - 1) / P.grp + 1;
    const int tiles = (P.n_keys - 1) / kCaKeys + 1;
    P.parts = div_up(tiles, __builtin_amdgcn_readfirstlane(Prices::OWN && P.rows <= kCaNarrowRows ? L.narrow_limit : L.limit));      // of a block shorter than its sequence's last one maybe fewer than `split`
    const int each = tiles / P.parts, more = tiles - each * P.parts;      // the first `more` have one more
    P.tile0 = P.part * each + min(P.part, more);
    P.tile1 = P.part < P.parts ? P.tile0 + each + (P.part < more) : P.tile0;
    return P;
}

// The ids of a piece's pages for the keys [key, ., .): a window, valid in front of key `end`.  Between barriers.
template <int N = kCaIds>
struct PageWindow {
    const int32_t *table;
    int first, end;                         // first page; first key that is not covered
    template <int OP> __device__ __forceinline__ void load(const ServingDev &S, const etc_serving_attention_io &io, ETC_AS_LDS int (&ids)[N], int b, int key, int key_end, int tid)
    {
        asm volatile("" : "+v"(tid));                    // addresses of this load: none of them waits in registers for the next window
        first = key >> S.page_shift;
        const int last = (key_end - 1) >> S.page_shift, n = min(last - first + 1, N);
        end = last - first < N ? key_end : (int)(((int64_t)(first + N)) << S.page_shift);
        for (int i = tid; i < n; i += kCaThreads) {
            int id = gld_i32(table + first + i);
            if ((uint32_t)id >= (uint64_t)io.n_pages) {
                refuse(S.error, SRV_BAD_PAGE, OP, b, id);
                id = 0;
            }
            ids[i] = id;
        }
    }
};

// Piece cc (of D / 8) of a lane's row: elements 8 cc + 4 half + 0 .. 3 of row r of the sequence and KV head.
template <int D>
__device__ __forceinline__ void put_out(const ServingDev &S, const etc_serving_attention_io &io, const Piece &P, int r, int cc, int half, f32x4 v)
{
    if (r >= P.rows) return;
    const int t = r / P.grp;
    uint16_t *op = (uint16_t *)io.out + ((int64_t)(P.seq.q0 + t) * S.nq + P.kvh * P.grp + (r - t * P.grp)) * D + cc * 8 + half * 4;
    *as_global(reinterpret_cast<u32x2 *>(op)) = u32x2{to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3])};
}

// Where the 32 rows rw of a part leave their partial result (device scope: the reader may be on another die).
template <int D>
__device__ __forceinline__ float *partial(const ServingDev &S, int slot, int rw)
{
    return S.attn_part + (size_t)slot * kCaSlot<D> + (size_t)rw * (kCaPartO<D> + 64);
}

// Running join of partial results (reference, sum, 4 elements of the output).
struct Join {
    float m = kCaNoReference, l = 0.f;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void add(float mj, float lj, f32x4 oj)
    {
        const float nm = fmaxf(m, mj), a = exp2_fast(m - nm), b = exp2_fast(mj - nm);
        m = nm;
        l = l * a + lj * b;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = o[i] * a + oj[i] * b;
    }
    __device__ __forceinline__ f32x4 result() const
    {
        const float inv = 1.0f / l;
        return f32x4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    }
};

// Behind a part's partial result: who arrives last at the item joins its parts, in the order of the keys.  AT_ONCE: pieces of a row that a wavefront
// asks for at once, of four parts, where an item has many rows (one piece of four parts, 4 KB, waits for memory most of the time).
template <int D, int AT_ONCE = 1>
__device__ __forceinline__ void join_parts(const ServingDev &S, const etc_serving_attention_io &io, ETC_AS_LDS CaLds &L, const Piece &P, int tid, int wave, int lane)
{
    const int half = lane >> 5, col = lane & 31;
    wg_release();
    if (tid == 0) {
        int32_t *ctr = S.attn_arrive + P.slot0;
        const int last = __hip_atomic_fetch_add(as_global(ctr), 1, __ATOMIC_RELAXED, ETC_SCOPE) + 1 == P.parts;
        if (last) st_i32(ctr, 0);
        L.last = last;
    }
    __syncthreads();
    if (!L.last) return;
    const int live = min(kCaWaves, div_up(P.rows - P.r0, 32));
    auto some = [&](auto pieces, int cc) {               // `pieces` pieces of 32 rows from piece cc on
        constexpr int N = decltype(pieces)::value;
        const int rw = cc / (D / 8), pc = cc % (D / 8);
        Join J[N];
        for (int j0 = 0; j0 < P.parts; j0 += 4) {
            f32x4 ov[4][N];
            uint64_t ml[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float *src = partial<D>(S, P.slot0 + min(j0 + u, P.parts - 1) * S.nkv, rw);
#pragma unroll
                for (int i = 0; i < N; ++i) ov[u][i] = __builtin_bit_cast(f32x4, buf_ld_16B(buf_of(src), (uint32_t)(((pc + i) * 64 + lane) * 16), 0));
                ml[u] = ld_u64(src + kCaPartO<D> + col * 2);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j0 + u < P.parts) {
#pragma unroll
                    for (int i = 0; i < N; ++i) J[i].add(__uint_as_float((uint32_t)ml[u]), __uint_as_float((uint32_t)(ml[u] >> 32)), ov[u][i]);
                }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) put_out<D>(S, io, P, P.r0 + rw * 32 + col, pc + i, half, J[i].result());
    };
    if (AT_ONCE > 1 && live > 2) {
        for (int cc = wave * AT_ONCE; cc < live * (D / 8); cc += kCaWaves * AT_ONCE) some(std::integral_constant<int, AT_ONCE>(), cc);
    } else {
        for (int cc = wave; cc < live * (D / 8); cc += kCaWaves) some(std::integral_constant<int, 1>(), cc);      // a wavefront per (32 rows, piece of them)
    }
}

// The pieces of a workgroup, one after the other.  In groups of kXcds, so that piece p stays with die p % kXcds: narrow pieces' groups
// spread evenly among the others', and in every other round of the launch the workgroups' groups in reverse.
template <class Prices = CutPrices, class F>
__device__ __forceinline__ void for_pieces(const ServingDev &S, const etc_serving_attention_io &io, ETC_AS_LDS CaLds &L, int n_pieces, F f)
{
    const int grid = (int)gridDim.x;
    const int narrow = __builtin_amdgcn_readfirstlane(L.narrow);
    const int gn = div_up(narrow, kXcds), groups = gn + div_up(n_pieces - narrow, kXcds);
    const int w = (int)blockIdx.x, all = grid & ~(kXcds - 1), back = w < all ? all - kXcds - (w & ~(kXcds - 1)) + (w & (kXcds - 1)) : w;
    for (int round = 0; round * grid < groups * kXcds; ++round) {
        int p = round * grid + ((round & 1) ? back : w), end = n_pieces;
        if (narrow > 0 && narrow < n_pieces) {
            const int g = p / kXcds, g0 = (int)((int64_t)g * gn / groups);
            const bool of_narrow = (int64_t)(g + 1) * gn / groups > g0;
            p = (of_narrow ? g0 * kXcds : narrow + (g - g0) * kXcds) + p % kXcds;
            if (of_narrow) end = narrow;
        }
        if (p >= end) continue;
        const Piece P = piece_of<Prices>(S, io, L, p);
        if (P.tile0 < P.tile1) f(P);
        __syncthreads();
    }
}

// Workgroups of a launch: one per compute unit (its registers fill one); fewer where the call cannot have as many pieces.
inline unsigned attention_grid(const ServingDev &S, const etc_serving_attention_io &io)
{
    const int64_t items = ((int64_t)io.n_tokens * (S.nq / S.nkv) / kCaRows + (io.n_seqs < io.n_tokens ? io.n_seqs : io.n_tokens)) * S.nkv;
    int64_t keys = (int64_t)io.table_cols << S.page_shift;
    if (keys > S.max_kv_len) keys = S.max_kv_len;
    const int64_t pieces = items * ((keys - 1) / (kCaKeys * kCaMinTiles) + 1);
    return (unsigned)(pieces < S.n_cus ? pieces : S.n_cus);
}

}  // namespace etc
