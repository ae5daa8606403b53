// Attention of a chunk of new tokens over the paged cache (include/etc.h, etc_serving_attention).
//
// A row of the problem is a (new token, query head) pair; the rows of one sequence and KV head, token-major, are cut into
// blocks of 32 per wavefront.  Everything runs transposed, S^T = K . Q^T and O^T = V^T . P^T on 32 x 32 x 16 matrix
// instructions: a lane then holds one row's scores (half of the keys, its partner lane + 32 the other half), so that softmax
// statistics are sums inside the lane and one exchange with the partner, and a lane's probabilities are, as they are, the
// right operand of the second product: its 16 keys are merely taken in the order the first product left them, by reading V's
// rows in that order.
#ifndef ETC_GENERIC_ONLY
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
    int limit;                              // tiles of a piece
    int narrow;                             // pieces of narrow sequences, which are in front (0: in any order)
    int odd, last;
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

// Fills L and returns the number of pieces.
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
            if (blockIdx.x == 0) refuse(S.error, SRV_BAD_LENGTH, SRV_ATTENTION, b, kv);
            n = 0;
        }
        L.q0[b] = q0;
        L.n[b] = n;
        L.kv[b] = kv;
        tokens += n;
        most = max(most, tiles_of(kv, n));
        if (n > 0) work += (float)S.nkv * blocks_of(n, grp) * 0.5f * (float)(tiles_of(kv, n) + tiles_of(kv, min(n, kCaRows / grp)));
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
        if (blockIdx.x == 0 && tid == 0) refuse(S.error, SRV_BAD_LENGTH, SRV_ATTENTION, io.n_seqs, tokens);
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
        const float f = w == 1 ? 4.f : w == 2 ? 3.f : w == 3 ? 2.f : w == 4 ? 1.5f : w == 5 ? 1.25f : w == 6 ? 1.1f : 1.f;
        return w == 0 ? 1 << 30 : max(kCaMinTiles, (int)fminf(ceilf(share * f), 1e9f));
    };
    int best = 0, longest_piece = most;
    if (most > kCaWholeTiles) {
        float pieces = 0.f, slots = 0.f;
        int longest = 0, parts = 1;
        bool whole = false;
        const int per = limit_of(wave);
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
        float ends = fmaxf((float)longest + 1.f, ceilf(pieces / (float)grid) * ((work + pieces) / fmaxf(pieces, 1.f))) + 0.5f * (float)parts + (__any(whole) ? 9.f : 0.f);
        if (wave > 0 && slots > (float)S.attn_slots) ends = INFINITY;
        __syncthreads();
        if (lane == 0) { L.wave_f[wave] = ends; L.wave_i[0][wave] = longest; }
        __syncthreads();
        float best_ends = L.wave_f[0];
#pragma unroll
        for (int w = 1; w < kCaTries; ++w)
            if (L.wave_f[w] < best_ends) { best = w; best_ends = L.wave_f[w]; }
        longest_piece = L.wave_i[0][best];
    }
    const int limit = limit_of(best);
    if (tid == 0) { L.first[0] = L.slot[0] = 0; L.limit = limit; L.narrow = 0; }
    auto count = [&](auto as_they_come) {                // the prefix sums; the number of pieces
        int done = 0, done_slots = 0;
        for (int i0 = 0; i0 < io.n_seqs; i0 += kCaThreads) {
            const int i = i0 + tid;
            int k = 0, sl = 0;
            __syncthreads();
            if (i < io.n_seqs) {
                int b = i, parts;
                if (as_they_come) {
                    parts = max(1, div_up(tiles_of(L.kv[i], L.n[i]), limit));
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
            cls[c] = rows > kCaNarrowRows ? kCaClasses - 1 : min(kCaClasses - 2, (int)((float)((kCaClasses - 1) * (longest_piece - len)) / (float)longest_piece));
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
        if (tid == 0) L.narrow = L.first[io.n_seqs - (total[kCaClasses / 2 - 1] >> 16)];
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

// S^T = K . Q^T over 32 KT keys: register i of tile kt is key 32 kt + 8 (i / 4) + 4 half + i % 4, the lane's row.
template <int D, int KT>
__device__ __forceinline__ void scores(f32x16 (&s)[KT], const Fragments<D> &F, uint32_t base, const bf16x8 (&qf)[D / 16])
{
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) s[kt] = f32x16{};
    bf16x8 a[2][KT];                                     // K's fragments a step ahead of their products
    auto k_frag = [&](int ks, int kt) {
        return *reinterpret_cast<ETC_AS_LDS const bf16x8 *>(reinterpret_cast<ETC_AS_LDS const char *>(F.k[ks] + base) + kt * 32 * D * 2);
    };
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) a[0][kt] = k_frag(0, kt);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        if (ks + 1 < D / 16) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) a[(ks + 1) & 1][kt] = k_frag(ks + 1, kt);
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[ks & 1][kt], qf[ks], s[kt], 0, 0, 0);
        // In this order: with all 256 registers taken the compiler reads one of two tiles' fragments behind the other's product (3 to 5 % of
        // a long prompt).
        if (KT > 1) __builtin_amdgcn_sched_barrier(0);
    }
}

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
template <int N> __device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0)" : : "i"(N) : "memory"); }

// LDS of a piece: rows of K and V, and the ids of its pages, a window of them at a time.
constexpr int kCaIds = 1024;
template <int D>
struct Tiles {
    uint16_t rows[512 * D];                 // 128 KB for heads of 128
    int ids[kCaIds];
};

struct Piece {
    int b, kvh, part, parts;                // part `part` of an item that has `parts` of them
    int slot0;                              // slot of part 0 (part j: j * nkv behind it)
    int tile0, tile1;                       // of the piece: [tile0, tile1)
    int n_keys;                             // that the last row of the block sees
    int grp, rows, r0;                      // query heads per KV head; rows of (sequence, KV head); first one of the block
    Seq seq;
};

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
    P.parts = div_up(tiles, __builtin_amdgcn_readfirstlane(L.limit));      // of a block shorter than its sequence's last one maybe fewer than `split`
    const int each = tiles / P.parts, more = tiles - each * P.parts;      // the first `more` have one more
    P.tile0 = P.part * each + min(P.part, more);
    P.tile1 = P.part < P.parts ? P.tile0 + each + (P.part < more) : P.tile0;
    return P;
}

// The ids of a piece's pages for the keys [key, ., .): a window, valid in front of key `end`.  Between barriers.
template <int D>
struct PageWindow {
    const int32_t *table;
    int first, end;                         // first page; first key that is not covered
    __device__ __forceinline__ void load(const ServingDev &S, const etc_serving_attention_io &io, ETC_AS_LDS Tiles<D> &B, int b, int key, int key_end, int tid)
    {
        asm volatile("" : "+v"(tid));                    // addresses of this load: none of them waits in registers for the next window
        first = key >> S.page_shift;
        const int last = (key_end - 1) >> S.page_shift, n = min(last - first + 1, kCaIds);
        end = last - first < kCaIds ? key_end : (int)(((int64_t)(first + kCaIds)) << S.page_shift);
        for (int i = tid; i < n; i += kCaThreads) {
            int id = gld_i32(table + first + i);
            if ((uint32_t)id >= (uint64_t)io.n_pages) {
                refuse(S.error, SRV_BAD_PAGE, SRV_ATTENTION, b, id);
                id = 0;
            }
            B.ids[i] = id;
        }
    }
};

// Fetches rows of the cache, KEYS of K and of V at a time, the first key a multiple of 64: load u of a wavefront brings RPL rows of
// each.  A lane's place in LDS is given, so it is the piece of memory that belongs there which it chooses.  Rows behind the last key
// are that key's again (their scores are masked).
// Where the rows of a load lie in one page (pages of RPL tokens and more) its address is a scalar and a constant of the lane: no vector
// instruction at all.  (With addresses per lane, and their page ids read from LDS on the spot, the fetches cost the long prompt 16 %.)
// ONCE, for the blocks of few rows: most rows are read by one workgroup of the launch, and by the next call only behind all other layers'
// caches, so they leave no copy in the caches on their way.  In us, with ONCE and without, caches turned over between calls / calls back to
// back: 64 single tokens over 2000 to 4000 keys 152 226 / 146 159, 16 sequences of 5 tokens 57 92 / 52 47, a mixed step 85 103 / 76 66, 16 single
// tokens over 500 to 1000 keys 26 34 / 22 22, one over 30000 45 69 / 41 39: it loses only where a call finds in the memory-side cache (256 MB) what
// the call before it read, as a model of one layer would.  Sequences that share pages read rows more than once: 64 tokens with all of 4000
// keys in common 117 113 / 101 99, with a quarter in common 144 196 / 134 138.
template <int D, int KEYS, bool ONCE>
struct Fetch {
    static constexpr int CH = D / 8, RPL = 64 / CH, LOADS = KEYS / RPL / kCaWaves;
    const etc_serving_attention_io &io;
    ETC_AS_LDS const Tiles<D> &B;
    int psh, pmask, wave, lrow, c, last_key;
    uint32_t row_bytes, head_off;
    uint32_t k_off[LOADS], v_off[LOADS];    // of the lane, from the page's row of the load's 64 keys on
    int id[LOADS];                          // page ids of the next fetch, asked for ahead of it
    __device__ __forceinline__ Fetch(const ServingDev &S, const etc_serving_attention_io &io_, ETC_AS_LDS const Tiles<D> &B_, int kvh, int last, int wave_, int lane)
        : io(io_), B(B_), psh(S.page_shift), pmask((1 << S.page_shift) - 1), wave(wave_), lrow(lane / CH), c(lane % CH), last_key(last),
          row_bytes((uint32_t)(S.nkv * D * 2)), head_off((uint32_t)(kvh * D * 2))
    {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int r = row_of(u) + lrow;
            const uint32_t in_page = (uint32_t)((r & 63) & pmask) * row_bytes + head_off;
            k_off[u] = in_page + (uint32_t)((c ^ k_swap<D>(r)) * 16);
            v_off[u] = in_page + (uint32_t)((c ^ v_swap<D>(r)) * 16);
        }
    }
    __device__ __forceinline__ int row_of(int u) const { return (wave * LOADS + u) * RPL; }
    __device__ __forceinline__ bool whole(int key0) const { return pmask + 1 >= RPL && key0 + KEYS - 1 <= last_key; }
    __device__ __forceinline__ void ask(int key0, int first_page)      // (nothing where each lane looks up its own)
    {
        if (!whole(key0)) return;
#pragma unroll
        for (int u = 0; u < LOADS; ++u) id[u] = B.ids[((key0 + row_of(u)) >> psh) - first_page];
    }
    __device__ __forceinline__ void fetch(int key0, int first_page, uint32_t kb, uint32_t vb)
    {
        const uint64_t page_bytes = (uint64_t)row_bytes << psh;
        if (whole(key0)) {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const int r = row_of(u);
                const uint64_t off = (uint32_t)__builtin_amdgcn_readfirstlane(id[u]) * page_bytes + (uint64_t)(uint32_t)((key0 + (r & ~63)) & pmask) * row_bytes;
                fetch_1k<ONCE>((const char *)io.k_pages + off, k_off[u], kb + r * D * 2);
                fetch_1k<ONCE>((const char *)io.v_pages + off, v_off[u], vb + r * D * 2);
            }
        } else {
#pragma unroll 1
            for (int u = 0; u < LOADS; ++u) {
                const int r = row_of(u), key = min(key0 + r + lrow, last_key);
                const uint64_t off = (uint32_t)B.ids[(key >> psh) - first_page] * page_bytes + (uint64_t)((uint32_t)(key & pmask)) * row_bytes + head_off;
                fetch_1k<ONCE>((const char *)io.k_pages + (off + (uint32_t)((c ^ k_swap<D>(r + lrow)) * 16)), kb + r * D * 2);
                fetch_1k<ONCE>((const char *)io.v_pages + (off + (uint32_t)((c ^ v_swap<D>(r + lrow)) * 16)), vb + r * D * 2);
            }
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

// Behind a part's partial result: who arrives last at the item joins its parts, in the order of the keys.
template <int D>
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
    for (int cc = wave; cc < live * (D / 8); cc += kCaWaves) {      // a wavefront per (32 rows, piece of them)
        const int rw = cc / (D / 8), pc = cc % (D / 8);
        Join J;
        for (int j0 = 0; j0 < P.parts; j0 += 4) {
            f32x4 ov[4];
            uint64_t ml[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float *src = partial<D>(S, P.slot0 + min(j0 + u, P.parts - 1) * S.nkv, rw);
                ov[u] = __builtin_bit_cast(f32x4, buf_ld_16B(buf_of(src), (uint32_t)((pc * 64 + lane) * 16), 0));
                ml[u] = ld_u64(src + kCaPartO<D> + col * 2);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (j0 + u < P.parts) J.add(__uint_as_float((uint32_t)ml[u]), __uint_as_float((uint32_t)(ml[u] >> 32)), ov[u]);
        }
        put_out<D>(S, io, P, P.r0 + rw * 32 + col, pc, half, J.result());
    }
}

// A block of more than 64 rows: 32 of them to a wavefront, all wavefronts over the same tiles of 64 keys, in ring slot t % 3: while
// tile t is being read, t + 1 has arrived or is about to, and the rows of t + 2 are on their way.
// Measured: 4001 tokens behind 30000 keys, 64 heads of 128 on 8 (4.2 TFLOP): 3.8 to 3.9 ms, 1.08 to 1.10 PFLOP/s, nine tenths of the rate of a large
// library product on this chip; matrix units busy 48 % of the cycles, no bank conflicts, memory idle (1 GB).  The bound is reading K and
// V from LDS, 32 KB by each of 8 wavefronts, 2048 of a tile's 4000 cycles, with the softmax of the same wavefronts in between; to delay
// half of the wavefronts, to give them priorities, or to share tiles between early and late rows changed nothing.
constexpr int kCaSlots = 3;

template <int D>
__device__ __forceinline__ void wide_piece(const ServingDev &S, const etc_serving_attention_io &io, ETC_AS_LDS CaLds &L, ETC_AS_LDS Tiles<D> &B, const Piece &P)
{
    constexpr int KS = D / 16, DT = D / 32;              // steps of the first product, tiles of the output
    constexpr int RPL = 512 / D, LOADS = kCaKeys / RPL / kCaWaves;      // rows of a load; loads of K (and of V) a wavefront has in a tile
    constexpr uint32_t BUF = kCaKeys * D * 2;            // bytes of a tile
    static_assert(2 * kCaSlots * kCaKeys <= 512, "LDS");
    int tid = (int)threadIdx.x;
    asm volatile("" : "+v"(tid));                        // of this piece: what is computed from it does not stay in registers across pieces
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int tile0 = P.tile0, n_tiles = P.tile1, key_end = min(n_tiles * kCaKeys, P.n_keys);
    PageWindow<D> W{io.block_table + (int64_t)P.b * io.table_stride, 0, 0};
    W.load(S, io, B, P.b, tile0 * kCaKeys, key_end, tid);

    // this lane's row: query fragments (right operand: 8 consecutive elements of step ks at ks * 16 + half * 8)
    const int row = P.r0 + wave * 32 + col, rr = min(row, P.rows - 1), t = rr / P.grp, head = P.kvh * P.grp + (rr - t * P.grp);
    const uint16_t *qp = (const uint16_t *)io.q + ((int64_t)(P.seq.q0 + t) * S.nq + head) * D + half * 8;
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, gld_16B(qp + ks * 16));
    const int limit = P.seq.kv + t;                      // last key this row sees
    const int first_masked = (P.seq.kv + P.r0 / P.grp + 1) / kCaKeys;      // tiles in front of it are seen whole by all rows of the block
    const int wave_last = P.seq.kv + min((P.r0 + wave * 32 + 31) / P.grp, P.seq.n - 1);
    const bool wave_live = P.r0 + wave * 32 < P.rows;
    const uint32_t k_base = (uint32_t)(uintptr_t)&B.rows[0], v_base = k_base + kCaSlots * BUF;
    Fetch<D, kCaKeys, false> G(S, io, B, P.kvh, P.n_keys - 1, wave, lane);

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x16{};
    float m = kCaNoReference, l = 0.f;                   // reference of the row's exponentials; sum over this lane's keys
    const float scale = 1.44269504088896f / sqrtf((float)D);      // scores and reference count in powers of two
    const Fragments<D> F(lane);
    f32x16 s[2];

    if (tid == 0) L.odd = -1;
    drain_vmem();                                        // nothing but tiles on their way from here on
    __syncthreads();
    uint32_t at = 0;                                     // ring slot of the tile at hand
    auto covered = [&](int tile) { return min((tile + 1) * kCaKeys, key_end) <= W.end; };
    auto after = [](uint32_t a) { return a == (kCaSlots - 1) * BUF ? 0u : a + BUF; };
    G.ask(tile0 * kCaKeys, W.first);
    G.fetch(tile0 * kCaKeys, W.first, k_base, v_base);
    if (tile0 + 1 < n_tiles && covered(tile0 + 1)) {
        G.ask((tile0 + 1) * kCaKeys, W.first);
        G.fetch((tile0 + 1) * kCaKeys, W.first, k_base + BUF, v_base + BUF);
        arrived<2 * LOADS>();
    } else {
        arrived<0>();
    }
    if (tile0 + 2 < n_tiles && covered(tile0 + 2)) G.ask((tile0 + 2) * kCaKeys, W.first);
    __syncthreads();
    // In front of a tile's work: the rows of the tile two behind it go on their way.  Behind it: the next tile's have arrived, for all.
    auto ahead = [&](int tile) {
        if (tile + 2 < n_tiles) {
            if (!covered(tile + 2)) {                    // its page ids are not here: a new window, with all loads at rest
                __syncthreads();
                W.load(S, io, B, P.b, (tile + 2) * kCaKeys, key_end, tid);
                drain_vmem();
                __syncthreads();
                G.ask((tile + 2) * kCaKeys, W.first);
            }
            const uint32_t to = after(after(at));
            G.fetch((tile + 2) * kCaKeys, W.first, k_base + to, v_base + to);
            if (tile + 3 < n_tiles && covered(tile + 3)) G.ask((tile + 3) * kCaKeys, W.first);
        }
    };
    auto next = [&](int tile) {
        if (tile + 2 < n_tiles) arrived<2 * LOADS>(); else arrived<0>();
        __syncthreads();
        at = after(at);
    };
    int tile = tile0;
    const int n_seen = min(first_masked, n_tiles);
    for (; tile < n_seen; ++tile) {
        if (wave_live) scores<D, 2>(s, F, k_base + at, qf);
        ahead(tile);                                     // while the products run: in front of them all wavefronts' fetches queue up (1 %)
        if (wave_live) attend<D, 2, false>(s, o, m, l, F, v_base + at, half, scale, 0, 0);
        next(tile);
    }
    for (; tile < n_tiles; ++tile) {
        ahead(tile);
        u32x4 mine[LOADS];
        uint32_t mine_at[LOADS];
        bool odd = false;                                // values that are no numbers, in any row of the tile
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            mine_at[u] = v_base + at + (wave * LOADS + u) * RPL * D * 2 + lane * 16;
            mine[u] = *reinterpret_cast<ETC_AS_LDS const u32x4 *>(mine_at[u]);
            odd |= any_odd(mine[u]);
        }
        if (odd) L.odd = tile;
        __syncthreads();
        const bool live = wave_live && tile * kCaKeys <= wave_last;
        if (__builtin_expect(L.odd == tile, 0)) odd_values<D, kCaKeys, LOADS>(mine, mine_at, o, F, v_base + at, half, tile * kCaKeys, limit, live);
        if (live) {
            scores<D, 2>(s, F, k_base + at, qf);
            attend<D, 2, true>(s, o, m, l, F, v_base + at, half, scale, tile * kCaKeys, limit);
        }
        next(tile);
    }
    l = partner_sum(l);
    if (P.parts == 1) {
        if (!wave_live) return;
        const float inv = 1.0f / l;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                put_out<D>(S, io, P, row, dt * 4 + q, half, f32x4{o[dt][4 * q] * inv, o[dt][4 * q + 1] * inv, o[dt][4 * q + 2] * inv, o[dt][4 * q + 3] * inv});
        return;
    }
    if (wave_live) {
        const __amdgpu_buffer_rsrc_t d_b = buf_of(partial<D>(S, P.slot0 + P.part * S.nkv, wave));
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                buf_st_16B(d_b, (uint32_t)(((dt * 4 + q) * 64 + lane) * 16),
                           __builtin_bit_cast(u32x4, f32x4{o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]}));
        if (half == 0) buf_st_8B(d_b, (uint32_t)(kCaPartO<D> * 4 + col * 8), u32x2{__float_as_uint(m), __float_as_uint(l)});
    }
    join_parts<D>(S, io, L, P, tid, wave, lane);
}

// A block of at most 64 rows is bound by the rows of the cache: all wavefronts work on the same keys' arrival, four to 128 keys (32 each)
// for the first 32 rows and four for the rest, and the keys' results are joined in LDS.  Two buffers of 128 keys: one on its
// way, or both, at any time.  Measured: 16 sequences of 5 tokens behind 2000 to 4100 keys, 32 heads of 128 on 8 (197 MB): 52 us, 3.8 TB/s, of
// which about 8 us are there for three short sequences too (launch, cut, page ids, rows and code that no cache holds yet, one after the
// other); 64 single tokens behind 2000 to 4000 keys (786 MB) 146 us, 5.4 TB/s, behind 16000 to 32000 (6.28 GB) 1040 us, 6.0 TB/s.
template <int D>
__device__ __forceinline__ void narrow_piece(const ServingDev &S, const etc_serving_attention_io &io, ETC_AS_LDS CaLds &L, ETC_AS_LDS Tiles<D> &B, const Piece &P)
{
    constexpr int KS = D / 16, DT = D / 32, KEYS = kCaNarrowKeys;
    constexpr int RPL = 512 / D, LOADS = KEYS / RPL / kCaWaves;
    constexpr uint32_t BUF = KEYS * D * 2;               // bytes of a step's K, and of its V behind that
    static_assert(4 * KEYS <= 512, "LDS");
    int tid = (int)threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int rw = wave >> 2, kg = wave & 3;             // rows 32 rw + 0 .. 31, keys 32 kg + 0 .. 31 of a step
    const int key0 = P.tile0 * kCaKeys, key_end = min(P.tile1 * kCaKeys, P.n_keys), n_steps = div_up(key_end - key0, KEYS);
    PageWindow<D> W{io.block_table + (int64_t)P.b * io.table_stride, 0, 0};
    W.load(S, io, B, P.b, key0, key_end, tid);

    const int row = rw * 32 + col, rr = min(row, P.rows - 1), t = rr / P.grp, head = P.kvh * P.grp + (rr - t * P.grp);
    const uint16_t *qp = (const uint16_t *)io.q + ((int64_t)(P.seq.q0 + t) * S.nq + head) * D + half * 8;
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, gld_16B(qp + ks * 16));
    const int limit = min(P.seq.kv + t, key_end - 1);    // last key this row sees in this piece
    const int all_see = min(P.seq.kv + 1, key_end);      // keys in front of it are seen by all rows
    const bool live = rw * 32 < P.rows;
    const uint32_t base = (uint32_t)(uintptr_t)&B.rows[0];
    Fetch<D, KEYS, true> G(S, io, B, P.kvh, key_end - 1, wave, lane);
    auto fetch = [&](int step) {
        const uint32_t to = base + (step & 1) * 2 * BUF;
        G.fetch(key0 + step * KEYS, W.first, to, to + BUF);
    };
    auto ask = [&](int step) { G.ask(key0 + step * KEYS, W.first); };
    auto covered = [&](int step) { return min(key0 + (step + 1) * KEYS, key_end) <= W.end; };

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x16{};
    float m = kCaNoReference, l = 0.f;
    const float scale = 1.44269504088896f / sqrtf((float)D);
    const Fragments<D> F(lane);
    f32x16 s[1];
    if (tid == 0) L.odd = -1;
    drain_vmem();                                        // nothing but rows on their way from here on
    __syncthreads();
    ask(0);
    fetch(0);
    if (n_steps > 1 && covered(1)) { ask(1); fetch(1); arrived<2 * LOADS>(); }
    else arrived<0>();
    if (n_steps > 2 && covered(2)) ask(2);
    __syncthreads();
    for (int step = 0; step < n_steps; ++step) {
        const int k0 = key0 + step * KEYS;
        const uint32_t kb = base + (step & 1) * 2 * BUF, kw = kb + kg * 32 * D * 2, vw = kw + BUF;
        const bool mine_live = live && k0 + kg * 32 < key_end;
        if (k0 + KEYS <= all_see) {
            if (mine_live) {
                scores<D, 1>(s, F, kw, qf);
                attend<D, 1, false>(s, o, m, l, F, vw, half, scale, 0, 0);
            }
        } else {
            u32x4 mine[LOADS];
            uint32_t at[LOADS];
            bool odd = false;
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                at[u] = kb + BUF + (wave * LOADS + u) * RPL * D * 2 + lane * 16;
                mine[u] = *reinterpret_cast<ETC_AS_LDS const u32x4 *>(at[u]);
                odd |= any_odd(mine[u]);
            }
            if (odd) L.odd = step;
            __syncthreads();
            if (__builtin_expect(L.odd == step, 0)) odd_values<D, 32, LOADS>(mine, at, o, F, vw, half, k0 + kg * 32, limit, mine_live);
            if (mine_live) {
                scores<D, 1>(s, F, kw, qf);
                attend<D, 1, true>(s, o, m, l, F, vw, half, scale, k0 + kg * 32, limit);
            }
        }
        __syncthreads();                                 // the buffer is free
        if (step + 2 < n_steps) {
            if (!covered(step + 2)) {                    // a new window of page ids, with all loads at rest
                arrived<0>();
                __syncthreads();
                W.load(S, io, B, P.b, k0 + 2 * KEYS, key_end, tid);
                drain_vmem();
                __syncthreads();
                ask(step + 2);
            }
            fetch(step + 2);
            if (step + 3 < n_steps && covered(step + 3)) ask(step + 3);
            arrived<2 * LOADS>();
        } else {
            arrived<0>();
        }
        __syncthreads();                                 // the next step's rows are here, for all
    }

    // ---- the four wavefronts of a row, in the order of the keys: output pieces of a lane as in a partial result, then m and l
    l = partner_sum(l);
    const uint32_t mine_at = base + wave * (kCaPartO<D> * 4), ml_at = (uint32_t)(uintptr_t)&B.ids[0];
    static_assert(kCaWaves * kCaPartO<D> * 4 <= 512 * D * 2, "LDS");
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<ETC_AS_LDS f32x4 *>(mine_at + ((dt * 4 + q) * 64 + lane) * 16) = f32x4{o[dt][4 * q], o[dt][4 * q + 1], o[dt][4 * q + 2], o[dt][4 * q + 3]};
    if (half == 0) *reinterpret_cast<ETC_AS_LDS f32x2_t *>(ml_at + (wave * 32 + col) * 8) = f32x2_t{m, l};
    __syncthreads();
    for (int cc = wave; cc < div_up(P.rows, 32) * (D / 8); cc += kCaWaves) {
        const int jr = cc / (D / 8), pc = cc % (D / 8);
        Join J;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x2_t ml = *reinterpret_cast<ETC_AS_LDS const f32x2_t *>(ml_at + ((jr * 4 + g) * 32 + col) * 8);
            J.add(ml[0], ml[1], *reinterpret_cast<ETC_AS_LDS const f32x4 *>(base + (jr * 4 + g) * (kCaPartO<D> * 4) + (pc * 64 + lane) * 16));
        }
        if (P.parts == 1) {
            put_out<D>(S, io, P, jr * 32 + col, pc, half, J.result());
        } else {
            const __amdgpu_buffer_rsrc_t d_b = buf_of(partial<D>(S, P.slot0 + P.part * S.nkv, jr));
            buf_st_16B(d_b, (uint32_t)((pc * 64 + lane) * 16), __builtin_bit_cast(u32x4, J.o));
            if (pc == 0 && half == 0) buf_st_8B(d_b, (uint32_t)(kCaPartO<D> * 4 + col * 8), u32x2{__float_as_uint(J.m), __float_as_uint(J.l)});
        }
    }
    if (P.parts > 1) join_parts<D>(S, io, L, P, tid, wave, lane);
}

template <int D>
__global__ __launch_bounds__(kCaThreads) void chunk_attention_kernel(ServingDev S, etc_serving_attention_io io)
{
    __shared__ CaLds s_cut;
    __shared__ __attribute__((aligned(16))) Tiles<D> s_tiles;
    ETC_AS_LDS CaLds &L = *as_lds(&s_cut);
    ETC_AS_LDS Tiles<D> &B = *as_lds(&s_tiles);
    const int n_pieces = cut(S, io, L), grid = (int)gridDim.x;
    if (n_pieces == 0) return;
    const int narrow = __builtin_amdgcn_readfirstlane(L.narrow);
    // In groups of kXcds, so that piece p stays with die p % kXcds: narrow pieces' groups spread evenly among the others', and in every
    // other round of the launch the workgroups' groups in reverse.
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
        const Piece P = piece_of(S, io, L, p);
        if (P.tile0 < P.tile1) {
            if (P.rows <= kCaNarrowRows) narrow_piece<D>(S, io, L, B, P);
            else wide_piece<D>(S, io, L, B, P);
        }
        __syncthreads();
    }
}

int64_t attention_slot_bytes(int head_dim) { return 4ll * (head_dim == 128 ? kCaSlot<128> : kCaSlot<64>); }

hipError_t launch_serving_attention(const ServingDev &S, const etc_serving_attention_io &io, hipStream_t s)
{
    // One workgroup per compute unit (its registers fill one); fewer where the call cannot have as many pieces.
    const int64_t items = ((int64_t)io.n_tokens * (S.nq / S.nkv) / kCaRows + (io.n_seqs < io.n_tokens ? io.n_seqs : io.n_tokens)) * S.nkv;
    int64_t keys = (int64_t)io.table_cols << S.page_shift;
    if (keys > S.max_kv_len) keys = S.max_kv_len;
    const int64_t pieces = items * ((keys - 1) / (kCaKeys * kCaMinTiles) + 1);
    const dim3 grid((unsigned)(pieces < S.n_cus ? pieces : S.n_cus)), block(kCaThreads);
    if (S.d == 128) hipLaunchKernelGGL((chunk_attention_kernel<128>), grid, block, 0, s, S, io);
    else hipLaunchKernelGGL((chunk_attention_kernel<64>), grid, block, 0, s, S, io);
    return hipGetLastError();
}

}  // namespace etc
#endif  // ETC_GENERIC_ONLY
