// Attention of a chunk of new tokens over a paged cache of 8 bits (include/etc.h, etc_serving_attention_codes).
//
// Rows, blocks, pieces and softmax are those of the attention over bf16 (chunk_attn.hip).  The first product takes the codes as they
// are: K's rows with the scale of their page, and q in two codes of 4 bits, q = hi + lo, each with a scale of its row, by two 32 x 32 x
// 64 instructions with scales, which take as long as the bf16 ones and read half as much.  The second product is that of bf16: V's codes
// are converted, with their page's scale, on their way to LDS.
#ifndef ETC_GENERIC_ONLY
#include "chunk_attn_rt.hip.h"
#include "codes_rt.hip.h"

namespace etc {

typedef __attribute__((ext_vector_type(8))) int i32x8;

typedef __attribute__((ext_vector_type(2))) int i32x2;

constexpr int kCa8Keys = 32;                // of a wavefront's step in a narrow piece

__device__ __forceinline__ void read_from_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }      // what was asked for is in registers

__device__ __forceinline__ i32x8 join_codes(u32x4 a, u32x4 b)
{
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// A row of q, this lane's half of it: elements half * D / 2 + 0 .. D / 2 - 1.  A scale takes the row's largest element to 224 .. 448: hi has
// 4 bits of each element, lo, of scale 2^-4, 4 more of them, down to 2^-13 of a code's unit.  Infinities and NaN are NaN.
template <int D>
struct QCodes {
    i32x8 hi[D / 64], lo[D / 64];
    int hi_scale, lo_scale;
    struct Asked { u32x4 w[D / 16]; };
    static __device__ __forceinline__ Asked ask(const uint16_t *row, int half)
    {
        Asked a;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) a.w[i] = gld_16B(row + half * (D / 2) + i * 8);
        return a;
    }
    __device__ __forceinline__ void set(const Asked &a)
    {
        const u32x4 (&w)[D / 16] = a.w;
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) most = fmaxf(most, fmaxf(fabsf(finite_or_nan(bf16_lo(w[i][j]))), fabsf(finite_or_nan(bf16_hi(w[i][j])))));
        }
        hi_scale = scale_byte(partner_max(most), 20);
        lo_scale = hi_scale - 4;
        const float inv = one_over_scale(hi_scale);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float a = finite_or_nan(bf16_lo(w[i][2 * j])) * inv, b = finite_or_nan(bf16_hi(w[i][2 * j])) * inv;
                const float c = finite_or_nan(bf16_lo(w[i][2 * j + 1])) * inv, d = finite_or_nan(bf16_hi(w[i][2 * j + 1])) * inv;
                const uint32_t h = to_f8x4(a, b, c, d);
                const f32x4 back = from_f8x4(h);
                hi[i / 4][(i & 3) * 2 + j] = (int)h;
                lo[i / 4][(i & 3) * 2 + j] = (int)to_f8x4((a - back[0]) * 16.f, (b - back[1]) * 16.f, (c - back[2]) * 16.f, (d - back[3]) * 16.f);
            }
    }
};

// S^T = K . Q^T over 32 keys: the lane's part of a key's row, as of q's, and the byte of the key's scale.
template <int D>
__device__ __forceinline__ f32x16 scores_of(const u32x4 (&k)[D / 32], int k_scale, const QCodes<D> &Q)
{
    f32x16 s{};
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
        const i32x8 a = join_codes(k[2 * j], k[2 * j + 1]);
        s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, Q.hi[j], s, 0, 0, 0, k_scale, 0, Q.hi_scale);
        s = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, Q.lo[j], s, 0, 0, 0, k_scale, 0, Q.lo_scale);
    }
    return s;
}

// Prices of a cut, in tiles of a whole block (1.55 us): 64 keys of a block of few rows are 16 KB, which a workgroup reads in less than half of that
// time; a tile of a launch's longest piece; what a piece costs besides its tiles, and where its keys are cut; what a call's last join takes; and what
// is left of a launch that takes its pieces one after the other when the first workgroup finds none, by the average piece.  Fitted to the times of all
// candidates in 34 calls (1 to 200 sequences, chunks of 1 to 4096, caches to 30000): what it chooses is 2 % behind the fastest in the mean,
// 15 % at worst (a prompt of 2000, 66 us without a cut, 57 with 1.5 shares).
// Items of up to WHOLE tiles are not cut, nor is a cut estimated; whole and as the estimate has it, in us, calls back to back:
//   tiles of the longest                          7           8          10          12          14          16
//   3 single tokens, 4 heads of 64 on 2       10.4  11.8  10.3  11.9  10.8  12.3  11.4  12.3  11.6  12.8  12.5  12.2
//   1 single token, 64 heads of 128 on 8      14.4  15.6  14.6  15.6  15.0  16.1  16.0  16.1  16.4  16.8  17.4  16.1
//   300 tokens, 32 heads of 128 on 8          24.9  26.1  26.4  28.3  29.5  34.1  32.5  29.7  35.7  35.0  38.6  31.1
struct CodesPrices {
    static constexpr bool OWN = true;
    static constexpr int WHOLE = 10;
    static __device__ __forceinline__ float factor(int w) { return w == 1 ? 4.f : w == 2 ? 2.f : w == 3 ? 1.5f : w == 4 ? 1.25f : w == 5 ? 1.1f : w == 6 ? 1.f : 0.85f; }
    static __device__ __forceinline__ float tile(bool narrow) { return narrow ? 0.44f : 1.f; }
    static __device__ __forceinline__ float alone(bool narrow) { return narrow ? 0.39f : 1.07f; }
    static __device__ __forceinline__ float piece(bool narrow) { return narrow ? 4.f : 7.6f; }
    static __device__ __forceinline__ float part(bool narrow) { return narrow ? 1.5f : 1.f; }
    static __device__ __forceinline__ float join(bool narrow, int parts) { return narrow ? 0.4f + 0.36f * (float)parts : 1.9f + 0.83f * (float)parts; }
    static __device__ __forceinline__ float left(float average) { return 0.47f * average; }
};

struct Pool8 { const uint8_t *k, *v, *k_scale, *v_scale; };

constexpr int kCa8Ids = 256;                // page ids in LDS, with their scales, a window of them at a time
constexpr int kCa8WideIds = 1024;           // of a whole block
constexpr int kCa8Tiles = 3;                // of a whole block, in LDS
template <int D>
struct Tiles8 {
    uint16_t rows[512 * D];                 // 128 KB for heads of 128
    int ids[kCa8Ids];
    int k_byte[kCa8Ids], v_byte[kCa8Ids];   // narrow pieces: scales of the pages
    float v_scale[kCaWaves][kCa8Keys];      // of a wavefront's keys
    int k_scale[kCa8Tiles][kCaKeys];        // wide pieces: of a tile's keys
};

// Where the rows of a (sequence, KV head) lie: offset of a key's row in the pools, and of its scale.
struct Rows8 {
    int psh, pmask, nkv, kvh;
    uint32_t row_bytes, head_off;
    __device__ __forceinline__ Rows8(const ServingDev &S, int kvh_, int D) : psh(S.page_shift), pmask((1 << S.page_shift) - 1), nkv(S.nkv), kvh(kvh_), row_bytes((uint32_t)(S.nkv * D)), head_off((uint32_t)(kvh_ * D)) {}
    template <int N> __device__ __forceinline__ int page(ETC_AS_LDS const int (&ids)[N], int key, int first) const { return ids[(key >> psh) - first]; }
    __device__ __forceinline__ uint64_t at(int id, int key) const { return ((uint64_t)(uint32_t)id * row_bytes << psh) + (uint32_t)(key & pmask) * (uint64_t)row_bytes + head_off; }
    __device__ __forceinline__ uint64_t scale_at(int id) const { return (uint64_t)(uint32_t)id * (uint32_t)nkv + (uint32_t)kvh; }
};

// ---- a block of more than 64 rows ------------------------------------------------------------------------------------------
// 32 rows to a wavefront, all wavefronts over the same tiles of 64 keys, in three buffers of LDS: while tile t is being read, t + 1 comes to LDS
// from registers, 16 bytes of K and of V to a thread, and t + 2 is on its way there.
// Bound by the matrix units and the power they take: 4001 tokens behind 30000 keys, 64 heads of 128 on 8 (4.2 TFLOP), take 3.46 to 3.72 ms on
// different machines, 1.13 to 1.21 PFLOP/s where a large bf16 product of a library reaches 1.29; the units are busy for half of the cycles.  Tried and slower there: K's fragments
// all asked for in front of their products (1 %), exponentials placed between the products by hand (5 %), the next tile to LDS in front of the
// products (6 %), a higher wave priority for either half of a tile (1 to 3 %).
template <int D>
__device__ __forceinline__ void wide_piece_codes(const ServingDev &S, const etc_serving_attention_io &io, const Pool8 &pool, ETC_AS_LDS CaLds &L, ETC_AS_LDS Tiles8<D> &B, const Piece &P)
{
    constexpr int DT = D / 32, PPR = D / 16;             // tiles of the output; pieces (of 16 codes) of a row
    constexpr uint32_t KBUF = kCaKeys * D, VBUF = kCaKeys * D * 2;
    static_assert(kCa8Tiles * (KBUF + VBUF) + kCa8WideIds * 4 <= 512 * D * 2, "LDS");
    static_assert(kCa8WideIds >= 2 * kCaKeys, "a window holds two tiles, whatever the pages");
    int tid = (int)threadIdx.x;
    asm volatile("" : "+v"(tid));                        // of this piece: what is computed from it does not stay in registers across pieces
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int tile0 = P.tile0, n_tiles = P.tile1, key_end = min(n_tiles * kCaKeys, P.n_keys);
    const int row = P.r0 + wave * 32 + col, rr = min(row, P.rows - 1), t = rr / P.grp, head = P.kvh * P.grp + (rr - t * P.grp);
    typename QCodes<D>::Asked q = QCodes<D>::ask((const uint16_t *)io.q + ((int64_t)(P.seq.q0 + t) * S.nq + head) * D, half);      // with the page ids
    typedef int Ids[kCa8WideIds];
    ETC_AS_LDS Ids &ids = *reinterpret_cast<ETC_AS_LDS Ids *>(&B.rows[kCa8Tiles * (KBUF + VBUF) / 2]);      // behind the tiles
    PageWindow<kCa8WideIds> W{io.block_table + (int64_t)P.b * io.table_stride, 0, 0};
    W.load<SRV_ATTENTION_CODES>(S, io, ids, P.b, tile0 * kCaKeys, key_end, tid);
    const int limit = P.seq.kv + t;                      // last key this row sees
    const int first_masked = (P.seq.kv + P.r0 / P.grp + 1) / kCaKeys;      // tiles in front of it are seen whole by all rows of the block
    const int wave_last = P.seq.kv + min((P.r0 + wave * 32 + 31) / P.grp, P.seq.n - 1);
    const bool wave_live = P.r0 + wave * 32 < P.rows;
    const uint32_t k_base = (uint32_t)(uintptr_t)&B.rows[0], v_base = k_base + kCa8Tiles * KBUF;

    // what this thread brings: row lr of a tile, codes 16 lp .. 16 lp + 15
    const Rows8 R(S, P.kvh, D);
    const int lr = tid / PPR, lp = tid % PPR;
    const bool brings = lr < kCaKeys;
    u32x4 k_in, v_in;
    uint32_t ks_in = 0, vs_in = 0;
    auto load = [&](int tile) {
        if (!brings) return;
        const int key = min(tile * kCaKeys + lr, P.n_keys - 1), id = R.page(ids, key, W.first);
        const uint64_t at = R.at(id, key) + lp * 16;
        k_in = gld_16B(pool.k + at);
        v_in = gld_16B(pool.v + at);
        ks_in = *as_global(pool.k_scale + R.scale_at(id));
        vs_in = *as_global(pool.v_scale + R.scale_at(id));
    };
    auto k_swap8 = [](int r) { return D == 128 ? (r >> 1) & 7 : (r >> 2) & 3; };
    auto put = [&](uint32_t buf) {
        if (!brings) return;
        *reinterpret_cast<ETC_AS_LDS u32x4 *>(k_base + buf * KBUF + lr * D + (lp ^ k_swap8(lr)) * 16) = k_in;
        if (lp == 0) B.k_scale[buf][lr] = (int)ks_in;
        const uint32_t to = v_base + buf * VBUF + lr * D * 2;
        const float f = scale_of(vs_in);
        *reinterpret_cast<ETC_AS_LDS u32x4 *>(to + ((2 * lp) ^ v_swap<D>(lr)) * 16) = codes_to_bf16x8(v_in[0], v_in[1], f);
        *reinterpret_cast<ETC_AS_LDS u32x4 *>(to + ((2 * lp + 1) ^ v_swap<D>(lr)) * 16) = codes_to_bf16x8(v_in[2], v_in[3], f);
    };

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x16{};
    float m = kCaNoReference, l = 0.f;                   // reference of the row's exponentials; sum over this lane's keys
    const float scale = 1.44269504088896f / sqrtf((float)D);      // scores and reference count in powers of two
    const Fragments<D> F(lane);
    uint32_t k_at[D / 32];                               // of this lane's pieces of K's rows
#pragma unroll
    for (int i = 0; i < D / 32; ++i) k_at[i] = k_base + col * D + ((half * (D / 32) + i) ^ k_swap8(col)) * 16;
    f32x16 s[2];
    QCodes<D> Q;
    auto scores = [&](uint32_t buf) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            u32x4 k[D / 32];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) k[i] = *reinterpret_cast<ETC_AS_LDS const u32x4 *>(k_at[i] + buf * KBUF + kt * 32 * D);
            s[kt] = scores_of<D>(k, B.k_scale[buf][kt * 32 + col], Q);
        }
    };
    auto next = [](uint32_t buf) { return buf + 1 == kCa8Tiles ? 0 : buf + 1; };
    auto ahead = [&](int tile, uint32_t buf) {           // the next tile to its buffer, the one behind it on its way
        if (tile + 1 < n_tiles) put(next(buf));
        if (tile + 2 < n_tiles) load(tile + 2);
    };
    int whole_tiles = 0;                                 // tiles whose pages, and those of the two behind them, are in LDS
    auto opened = [&] { whole_tiles = W.end < key_end ? W.end / kCaKeys - 2 : n_tiles; };
    auto window = [&](int tile) {                        // by all threads, none of them ahead
        __syncthreads();
        W.load<SRV_ATTENTION_CODES>(S, io, ids, P.b, (tile + 2) * kCaKeys, key_end, tid);
        __syncthreads();
        opened();
    };

    if (tid == 0) L.odd = -1;
    __syncthreads();
    load(tile0);
    Q.set(q);                                            // while the first rows are on their way
    put(0);
    if (tile0 + 1 < n_tiles) load(tile0 + 1);
    opened();
    __syncthreads();
    int tile = tile0;
    uint32_t buf = 0;
    const int n_seen = min(first_masked, n_tiles);
    // Tiles that all rows see whole.  A SIMD has a wavefront of the upper and one of the lower half of the rows: the lower ones are half a tile late, so
    // that one's products keep the matrix units busy while the other computes exponentials (7 % fewer cycles; 3 % of the time of 4001 tokens behind
    // 30000 keys, where power binds, 6 % of 1500 behind 4000, 32 heads of 128 on 4).
    const bool late = wave >= kCaWaves / 2;
    while (tile < n_seen) {
        const int stop = min(n_seen, whole_tiles);
        if (tile >= stop) {
            window(tile);
            continue;
        }
        if (late) __syncthreads();
        for (; tile < stop; ++tile, buf = next(buf)) {
            if (wave_live) scores(buf);
            ahead(tile, buf);
            __syncthreads();
            if (wave_live) attend<D, 2, false>(s, o, m, l, F, v_base + buf * VBUF, half, scale, 0, 0);
            __syncthreads();
        }
        if (!late) __syncthreads();
    }
    for (; tile < n_tiles; ++tile, buf = next(buf)) {
        if (tile >= whole_tiles) window(tile);
        const uint32_t v_tile = v_base + buf * VBUF;
        constexpr int N = D / 64;
        u32x4 mine[N];
        uint32_t mine_at[N];
        bool odd = false;                                // values that are no numbers, in any row of the tile
#pragma unroll
        for (int u = 0; u < N; ++u) {
            mine_at[u] = v_tile + (u * kCaThreads + tid) * 16;
            mine[u] = *reinterpret_cast<ETC_AS_LDS const u32x4 *>(mine_at[u]);
            odd |= any_odd(mine[u]);
        }
        if (odd) L.odd = tile;
        __syncthreads();
        const bool live = wave_live && tile * kCaKeys <= wave_last;
        if (__builtin_expect(L.odd == tile, 0)) odd_values<D, kCaKeys, N>(mine, mine_at, o, F, v_tile, half, tile * kCaKeys, limit, live);
        if (live) scores(buf);
        ahead(tile, buf);
        if (live) attend<D, 2, true>(s, o, m, l, F, v_tile, half, scale, tile * kCaKeys, limit);
        __syncthreads();
    }
    l = partner_sum(l);
    if (P.parts == 1) {
        if (!wave_live) return;
        // By way of LDS, where everyone is done with the tiles: a lane has 4 elements of a row next to its partner's 4, and writes 8 of one.
        const float inv = 1.0f / l;
        const uint32_t rows_at = (uint32_t)(uintptr_t)&B.rows[0] + wave * 32 * D * 2;
        auto piece_at = [&](int r, int piece) { return rows_at + r * D * 2 + (piece ^ (r & (D / 8 - 1))) * 16; };
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<ETC_AS_LDS u32x2 *>(piece_at(col, dt * 4 + q) + half * 8) =
                    u32x2{to_bf16x2(o[dt][4 * q] * inv, o[dt][4 * q + 1] * inv), to_bf16x2(o[dt][4 * q + 2] * inv, o[dt][4 * q + 3] * inv)};
        in_order();
        constexpr int AT_ONCE = 64 / (D / 8);            // rows
#pragma unroll
        for (int i = 0; i < 32 / AT_ONCE; ++i) {
            const int lr = i * AT_ONCE + lane / (D / 8), piece = lane % (D / 8), r = P.r0 + wave * 32 + lr, rt = r / P.grp;
            const u32x4 w = *reinterpret_cast<ETC_AS_LDS const u32x4 *>(piece_at(lr, piece));
            if (r < P.rows)
                *as_global(reinterpret_cast<u32x4 *>((uint16_t *)io.out + ((int64_t)(P.seq.q0 + rt) * S.nq + P.kvh * P.grp + (r - rt * P.grp)) * D + piece * 8)) = w;
        }
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
    join_parts<D, 4>(S, io, L, P, tid, wave, lane);
}

// ---- a block of at most 64 rows --------------------------------------------------------------------------------------------
// Bound by the rows of the cache.  Every wavefront goes through keys of its own, 32 at a time, every eighth such step, without a barrier: codes go to
// its own part of LDS, two steps of them on their way or at hand, and from there to registers as they are, K's as rows, V's transposed, so that a
// step's place is free for the one behind the next while it is worked on.  64 tokens over 4081 to 7935 keys, 32 heads of 128 on 8 (778 MB), take 160 to
// 163 us, 4.8 TB/s; without any arithmetic 148: a head's row is 128 bytes in every 1024.  Rows pass the caches by (non-temporal loads): 164 us, 175
// without, and 94 against 101 for half as many keys.  With K straight to registers and V through them to LDS, as bf16, it took 544.
// V's codes become bf16 without their scales, which the probabilities take (keys of one instruction may lie in several pages).
// The wavefronts' results are joined in LDS.

// NaN codes of V, among keys that some rows do not see: 1 in a byte of each; 0 in their place; as bf16, 1 where there is one.
__device__ __forceinline__ uint32_t nan_mask(uint32_t w) { return (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7; }
__device__ __forceinline__ uint32_t without_nan(uint32_t w) { return w & ~(nan_mask(w) * 0xFFu); }
__device__ __forceinline__ u32x4 nan_counts(u32x2 w)
{
    auto pair = [](uint32_t m, int at) { return ((m >> at & 1u) | (m >> (at + 8) & 1u) << 16) * 0x3F80u; };
    const uint32_t m = nan_mask(w[0]), n = nan_mask(w[1]);
    return u32x4{pair(m, 0), pair(m, 16), pair(n, 0), pair(n, 16)};
}

// A wavefront's steps on their way to LDS: 32 rows of K, behind them 32 of V, D bytes each; a row's 16-byte pieces change places with the row
// so that 16 rows of a piece lie in different banks.
template <int D>
struct Ring8 {
    static constexpr int PPR = D / 16, RPL = 64 / PPR, LOADS = kCa8Keys / RPL;      // pieces of a row, rows of a load, loads of K (and of V)
    static constexpr uint32_t HALF = kCa8Keys * D, STEP = 2 * HALF;
    static __device__ __forceinline__ int swap(int row) { return D == 128 ? (row >> 1) & 7 : (row >> 2) & 3; }
    const Pool8 &pool;
    ETC_AS_LDS const int (&ids)[kCa8Ids];
    const Rows8 &R;
    uint32_t base;                          // of the wavefront's part of LDS
    int lane, key0, last_key;
    uint32_t off[2];                        // of the lane, from the page's row of a load's first key on: loads with an even number, and odd ones
    __device__ __forceinline__ Ring8(const Pool8 &pool_, ETC_AS_LDS const int (&ids_)[kCa8Ids], const Rows8 &R_, uint32_t base_, int lane_, int key0_, int last)
        : pool(pool_), ids(ids_), R(R_), base(base_), lane(lane_), key0(key0_), last_key(last)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) off[u] = (lane / PPR) * R.row_bytes + R.head_off + ((lane % PPR) ^ swap(u * RPL + lane / PPR)) * 16;
    }
    template <bool K, bool V> __device__ __forceinline__ void fetch(int step, int buf, int first_page)
    {
        const int k0 = key0 + step * kCa8Keys;
        const uint32_t to = base + buf * STEP;
        if (R.pmask + 1 >= RPL && k0 + kCa8Keys - 1 <= last_key) {      // a load's rows lie in one page: scalar addresses
            int id[LOADS];
#pragma unroll
            for (int u = 0; u < LOADS; ++u) id[u] = R.page(ids, k0 + u * RPL, first_page);
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const uint64_t at = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(id[u]) * R.row_bytes << R.psh) + (uint64_t)((uint32_t)((k0 + u * RPL) & R.pmask) * (uint64_t)R.row_bytes);
                if (K) fetch_1k<true>((const char *)pool.k + at, off[u & 1], to + u * 1024);
                if (V) fetch_1k<true>((const char *)pool.v + at, off[u & 1], to + HALF + u * 1024);
            }
        } else {
#pragma unroll 1
            for (int u = 0; u < LOADS; ++u) {
                const int r = u * RPL + lane / PPR, key = min(k0 + r, last_key);
                const uint64_t at = R.at(R.page(ids, key, first_page), key) + ((lane % PPR) ^ swap(r)) * 16;
                if (K) fetch_1k<true>((const char *)pool.k + at, to + u * 1024);
                if (V) fetch_1k<true>((const char *)pool.v + at, to + HALF + u * 1024);
            }
        }
    }
};

// Softmax of a step's scores and O^T += V^T . P^T, as attend() of few rows: both parts of a probability.  v: V's codes, [16 keys][32 elements], a
// lane's 8 keys of an element in the order the scores have them; by: the scales of the lane's 16 keys.
template <int D, bool MASKED>
__device__ __forceinline__ void attend_codes(f32x16 &s, f32x16 (&o)[D / 32], float &m, float &l, const u32x2 (&v)[2][D / 32], const f32x4 (&by)[4], int half, float scale, int k0, int limit)
{
    constexpr int DT = D / 32;
    if constexpr (MASKED) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (k0 + 8 * (i >> 2) + 4 * half + (i & 3) > limit) s[i] = -INFINITY;
    }
    float mt = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mt = fmaxf(mt, s[i]);
    mt = partner_max(mt) * scale;
    if (__builtin_amdgcn_ballot_w64(mt > m + 8.f) != 0) {
        const float nm = fmaxf(m, mt), sc = MASKED && m == kCaNoReference ? 1.f : exp2_fast(m - nm);      // (NaN that are in o already stay)
        m = nm;
        l *= sc;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= sc;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        u32x4 p, rest;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = exp2_fast(__builtin_fmaf(s[8 * h + 2 * i], scale, -m)), b = exp2_fast(__builtin_fmaf(s[8 * h + 2 * i + 1], scale, -m));
            l += a + b;
            a *= by[2 * h + (i >> 1)][(i & 1) * 2];
            b *= by[2 * h + (i >> 1)][(i & 1) * 2 + 1];
            const uint32_t ah = __float_as_uint(a), bh = __float_as_uint(b);      // the upper part below the probability; codes hold no infinities, so 0 may be one
            p[i] = __builtin_amdgcn_perm(bh, ah, 0x07060302u);
            rest[i] = to_bf16x2(a - __uint_as_float(ah & 0xFFFF0000u), b - __uint_as_float(bh & 0xFFFF0000u));
        }
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const bf16x8 w = __builtin_bit_cast(bf16x8, codes_to_bf16x8(v[h][dt][0], v[h][dt][1], 1.f));
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, __builtin_bit_cast(bf16x8, p), o[dt], 0, 0, 0);
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, __builtin_bit_cast(bf16x8, rest), o[dt], 0, 0, 0);
        }
    }
}

// SHARED: 33 to 64 rows.  Two wavefronts, of 32 rows each, go through the same keys; one fetches K, the other V, in a ring of four steps, and a barrier
// in front of each step says that it is there for both (and that the one in front of it has been read).  64 sequences of 8 tokens over 8000 keys,
// 64 heads of 128 on 8: 216 to 227 us; with a ring to each wavefront, and every key fetched twice, 311.
template <int D, bool SHARED>
__device__ __forceinline__ void narrow_piece_codes(const ServingDev &S, const etc_serving_attention_io &io, const Pool8 &pool, ETC_AS_LDS CaLds &L, ETC_AS_LDS Tiles8<D> &B, const Piece &P)
{
    constexpr int DT = D / 32;
    typedef Ring8<D> Ring;
    constexpr int GROUPS = SHARED ? kCaWaves / 2 : kCaWaves, STEPS = 2 * kCaWaves / GROUPS;      // wavefronts to 32 rows; steps of a ring
    static_assert(GROUPS * STEPS * Ring::STEP <= 512 * D * 2, "LDS");
    int tid = (int)threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, half = lane >> 5, col = lane & 31;
    const int rw = wave / GROUPS, kg = wave % GROUPS;
    const int key0 = P.tile0 * kCaKeys, key_end = min(P.tile1 * kCaKeys, P.n_keys), n_steps = div_up(key_end - key0, kCa8Keys);
    const int row = rw * 32 + col, rr = min(row, P.rows - 1), t = rr / P.grp, head = P.kvh * P.grp + (rr - t * P.grp);
    typename QCodes<D>::Asked q = QCodes<D>::ask((const uint16_t *)io.q + ((int64_t)(P.seq.q0 + t) * S.nq + head) * D, half);      // with the page ids
    PageWindow<kCa8Ids> W{io.block_table + (int64_t)P.b * io.table_stride, 0, 0};
    W.load<SRV_ATTENTION_CODES>(S, io, B.ids, P.b, key0, key_end, tid);
    QCodes<D> Q;
    const int limit = min(P.seq.kv + t, key_end - 1);    // last key this row sees in this piece
    const int all_see = min(P.seq.kv + 1, key_end);      // keys in front of it are seen by all rows
    const uint32_t base = (uint32_t)(uintptr_t)&B.rows[0], mine = base + kg * STEPS * Ring::STEP;

    const Rows8 R(S, P.kvh, D);
    Ring G(pool, B.ids, R, mine, lane, key0, key_end - 1);
    uint32_t k_at[DT], v_at[DT];                         // LDS addresses of this lane's pieces of a step that starts at 0
    const int v_row = 4 * half + ((lane & 7) >> 1) + (lane & 8), v_piece = (lane >> 4) & 1;      // 8 rows to 16 lanes, 8 codes each: rows 4 half .. and 8 + 4 half ..
#pragma unroll
    for (int i = 0; i < DT; ++i) {
        k_at[i] = mine + col * D + ((half * DT + i) ^ Ring::swap(col)) * 16;
        v_at[i] = mine + Ring::HALF + v_row * D + ((i * 2 + v_piece) ^ Ring::swap(v_row)) * 16 + (lane & 1) * 8;
    }
    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x16{};
    float m = kCaNoReference, l = 0.f;
    const float scale = 1.44269504088896f / sqrtf((float)D);
    auto v_codes = [&](int buf, int h, int i) {
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<ETC_AS_LDS i32x2 *>(v_at[i] + buf * Ring::STEP + h * 16 * D)));
    };
    // NaN codes of V in a step that some rows see a part of: the probability 0 of what a row does not see would make a NaN of them.  Counted by a
    // product over the keys a row sees, which goes to the output; the second product has zeros in their place.
    auto count_nans = [&](int k0, int buf) {
        uint32_t nan = 0;
#pragma unroll
        for (int u = 0; u < Ring::LOADS; ++u) {
            const u32x4 w = *reinterpret_cast<ETC_AS_LDS const u32x4 *>(mine + buf * Ring::STEP + Ring::HALF + (u * 64 + lane) * 16);
            nan |= nan_mask(w[0]) | nan_mask(w[1]) | nan_mask(w[2]) | nan_mask(w[3]);
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(nan != 0) == 0, 1)) return;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            f32x16 n{};
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                u32x4 seen;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = k0 + h * 16 + 4 * half + (j >> 1) * 8 + (j & 1) * 2;
                    seen[j] = (key <= limit ? 0x3F80u : 0u) | (key + 1 <= limit ? 0x3F800000u : 0u);
                }
                n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, nan_counts(v_codes(buf, h, i))), __builtin_bit_cast(bf16x8, seen), n, 0, 0, 0);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                if (n[j] > 0.f) o[i][j] = __uint_as_float(0x7FC00000u);
                __builtin_amdgcn_sched_barrier(0);       // one condition at a time: all at once fill the scalar registers
            }
        }
    };
    auto fetch = [&](int step, int buf) {
        if (!SHARED) G.template fetch<true, true>(step, buf, W.first);
        else if (rw == 0) G.template fetch<true, false>(step, buf, W.first);
        else G.template fetch<false, true>(step, buf, W.first);
    };
    // A step that is there; `ahead` sends one more on its way once its place is free.
    auto work = [&](auto with_mask, int step, int buf, auto ahead) {
        constexpr bool MASKED = decltype(with_mask)::value;
        const int k0 = key0 + step * kCa8Keys;
        if constexpr (MASKED) count_nans(k0, buf);
        u32x4 k[DT];
        u32x2 v[2][DT];
#pragma unroll
        for (int i = 0; i < DT; ++i) k[i] = *reinterpret_cast<ETC_AS_LDS const u32x4 *>(k_at[i] + buf * Ring::STEP);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < DT; ++i)
                v[h][i] = v_codes(buf, h, i);
        const int page = (min(k0 + col, key_end - 1) >> R.psh) - W.first, k_scale = B.k_byte[page];
        if (half == 0) B.v_scale[wave][col] = scale_of(B.v_byte[page]);      // (each wavefront for itself)
        in_order();
        f32x4 by[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) by[j] = *reinterpret_cast<ETC_AS_LDS const f32x4 *>(&B.v_scale[wave][8 * j + 4 * half]);
        read_from_lds();                                 // the step's place is free
        ahead();
        if constexpr (MASKED) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < DT; ++i) v[h][i] = u32x2{without_nan(v[h][i][0]), without_nan(v[h][i][1])};
        }
        f32x16 s = scores_of<D>(k, k_scale, Q);
        attend_codes<D, MASKED>(s, o, m, l, v, by, half, scale, k0, limit);
    };
    constexpr int FIRST = SHARED ? STEPS - 1 : STEPS, FIRST_LOADS = FIRST * (SHARED ? 1 : 2) * Ring::LOADS;      // steps that are sent on their way at once
    int begin = 0, end = 0, step = 0;                    // a window of page ids: its steps; this wavefront's next one
    auto open = [&] {
        end = W.end < key_end ? (W.end - key0) / kCa8Keys : n_steps;
        step = begin + kg;
        if (wave < kCa8Ids / 64) {                       // the pages' scales, a page to a lane (behind the last one that one's again)
            const uint64_t at = R.scale_at(B.ids[min(wave * 64 + lane, ((min(W.end, key_end) - 1) >> R.psh) - W.first)]);
            fetch_bytes(pool.k_scale + at, (uint32_t)(uintptr_t)&B.k_byte[wave * 64]);
            fetch_bytes(pool.v_scale + at, (uint32_t)(uintptr_t)&B.v_byte[wave * 64]);
        }
#pragma unroll
        for (int a = 0; a < FIRST; ++a)
            if (step + a * GROUPS < end) fetch(step + a * GROUPS, a);
    };
    drain_vmem();                                        // nothing but rows (and scales) on their way from here on
    __syncthreads();
    open();
    Q.set(q);
    for (;;) {
        if (step + (FIRST - 1) * GROUPS < end) arrived<FIRST_LOADS>(); else arrived<0>();      // the scales, in front of the rows
        __syncthreads();
        const int seen = min(end, (all_see - key0) / kCa8Keys);      // steps that all rows see whole
        int buf = 0;
        if constexpr (!SHARED) {
            auto next = [&](auto with_mask) {
                if (step + GROUPS < end) arrived<2 * Ring::LOADS>(); else arrived<0>();
                work(with_mask, step, buf, [&] { if (step + STEPS * GROUPS < end) fetch(step + STEPS * GROUPS, buf); });
                step += GROUPS;
                buf ^= 1;
            };
            while (step < seen) next(std::false_type());
            while (step < end) next(std::true_type());
        } else {
            int first = begin;                           // of a round of steps, for all wavefronts alike
            auto next = [&](auto with_mask) {
                if (step + 2 * GROUPS < end) arrived<2 * Ring::LOADS>();
                else if (step + GROUPS < end) arrived<Ring::LOADS>();
                else arrived<0>();
                __syncthreads();
                if (step + (STEPS - 1) * GROUPS < end) fetch(step + (STEPS - 1) * GROUPS, (buf + STEPS - 1) % STEPS);
                if (step < end) work(with_mask, step, buf, [] {});
                first += GROUPS;
                step += GROUPS;
                buf = (buf + 1) % STEPS;
            };
            while (first + GROUPS <= seen) next(std::false_type());
            while (first < end) next(std::true_type());
        }
        begin = end;
        if (begin >= n_steps) break;
        __syncthreads();
        W.load<SRV_ATTENTION_CODES>(S, io, B.ids, P.b, key0 + begin * kCa8Keys, key_end, tid);
        drain_vmem();
        __syncthreads();
        open();
    }

    // ---- the wavefronts of a row, in the order of their steps: output pieces of a lane as in a partial result, then m and l
    l = partner_sum(l);
    const uint32_t mine_at = base + wave * (kCaPartO<D> * 4), ml_at = (uint32_t)(uintptr_t)&B.ids[0];      // (and the scales behind them)
    static_assert(kCaWaves * kCaPartO<D> * 4 <= 512 * D * 2 && kCaWaves * 32 * 8 <= 2 * kCa8Ids * 4, "LDS");
    __syncthreads();                                     // everyone's rows have been read, and the page ids
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
        for (int g = 0; g < GROUPS; ++g) {
            const f32x2_t ml = *reinterpret_cast<ETC_AS_LDS const f32x2_t *>(ml_at + ((jr * GROUPS + g) * 32 + col) * 8);
            J.add(ml[0], ml[1], *reinterpret_cast<ETC_AS_LDS const f32x4 *>(base + (jr * GROUPS + g) * (kCaPartO<D> * 4) + (pc * 64 + lane) * 16));
        }
        if (P.parts == 1) {
            put_out<D>(S, io, P, jr * 32 + col, pc, half, J.result());
        } else {                                         // (whole, also of few rows: their 64 bytes of each KB were slower to write)
            const __amdgpu_buffer_rsrc_t d_b = buf_of(partial<D>(S, P.slot0 + P.part * S.nkv, jr));
            buf_st_16B(d_b, (uint32_t)((pc * 64 + lane) * 16), __builtin_bit_cast(u32x4, J.o));
            if (pc == 0 && half == 0) buf_st_8B(d_b, (uint32_t)(kCaPartO<D> * 4 + col * 8), u32x2{__float_as_uint(J.m), __float_as_uint(J.l)});
        }
    }
    if (P.parts > 1) join_parts<D, 4>(S, io, L, P, tid, wave, lane);
}

// The pieces of a workgroup, one after the other, in groups of kXcds so that piece p stays with die p % kXcds: whole blocks' first, which take up to
// 45 us, then narrow ones (2 to 30).  A workgroup's first piece is its own; of the others each takes the die's next one when it has none.  Dealt out in
// advance, narrow pieces among the others, 32 mixed sequences (57 us) took 8 % longer and 40 of heads of 4 to 1 (150 us) 68 %; taken in turn in
// that order 5 % and 10 %.
template <class F>
__device__ __forceinline__ void take_pieces(const ServingDev &S, const etc_serving_attention_io &io, ETC_AS_LDS CaLds &L, ETC_AS_LDS int *next, int n_pieces, F f)
{
    const int grid = (int)gridDim.x, dies = min(grid, kXcds), w = (int)blockIdx.x, die = w % dies;
    const int narrow = __builtin_amdgcn_readfirstlane(L.narrow);
    const int gn = div_up(narrow, kXcds), groups = gn + div_up(n_pieces - narrow, kXcds), all = groups * kXcds;
    const bool asks = all > grid && threadIdx.x == 0;
    for (int k = w / dies; k * dies + die < all;) {
        int p = k * dies + die, end = n_pieces;
        if (narrow > 0 && narrow < n_pieces) {
            const int wide = (groups - gn) * kXcds;      // places
            if (p < wide) {
                p += narrow;
            } else {
                p -= wide;
                end = narrow;
            }
        }
        if (p < end) {
            const Piece P = piece_of<CodesPrices>(S, io, L, p);
            if (P.tile0 < P.tile1) f(P);
        }
        if (all <= grid) return;
        if (asks) {
            const int n = __hip_atomic_fetch_add(as_global(S.taken + die * kTakenApart), 1, __ATOMIC_RELAXED, ETC_SCOPE);
            if (n == div_up(all - die, dies) - 1) st_i32(S.taken + die * kTakenApart, 0);      // the last: every piece of the die asks once
            *next = div_up(grid - die, dies) + n;
        }
        __syncthreads();
        k = __builtin_amdgcn_readfirstlane(*next);
        __syncthreads();
    }
}

template <int D>
__global__ __launch_bounds__(kCaThreads) void chunk_attention_codes_kernel(ServingDev S, etc_serving_attention_codes_io io8)
{
    __shared__ CaLds s_cut;
    __shared__ int s_next;
    __shared__ __attribute__((aligned(16))) Tiles8<D> s_tiles;
    ETC_AS_LDS CaLds &L = *as_lds(&s_cut);
    ETC_AS_LDS Tiles8<D> &B = *as_lds(&s_tiles);
    const etc_serving_attention_io &io = io8.attention;
    const Pool8 pool{(const uint8_t *)io.k_pages, (const uint8_t *)io.v_pages, (const uint8_t *)io8.k_scale, (const uint8_t *)io8.v_scale};
    const int n_pieces = cut<SRV_ATTENTION_CODES, CodesPrices>(S, io, L);
    if (n_pieces == 0) return;
    take_pieces(S, io, L, as_lds(&s_next), n_pieces, [&](const Piece &P) {
        if (P.rows <= 32) narrow_piece_codes<D, false>(S, io, pool, L, B, P);
        else if (P.rows <= kCaNarrowRows) narrow_piece_codes<D, true>(S, io, pool, L, B, P);
        else wide_piece_codes<D>(S, io, pool, L, B, P);
    });
}

hipError_t launch_serving_attention_codes(const ServingDev &S, const etc_serving_attention_codes_io &io, hipStream_t s)
{
    const dim3 grid(attention_grid(S, io.attention)), block(kCaThreads);
    if (S.d == 128) hipLaunchKernelGGL((chunk_attention_codes_kernel<128>), grid, block, 0, s, S, io);
    else hipLaunchKernelGGL((chunk_attention_codes_kernel<64>), grid, block, 0, s, S, io);
    return hipGetLastError();
}

}  // namespace etc
#endif  // ETC_GENERIC_ONLY
