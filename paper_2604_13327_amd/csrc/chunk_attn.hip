// Attention of a chunk of new tokens over the paged cache (include/etc.h, etc_serving_attention).
//
// A row of the problem is a (new token, query head) pair; the rows of one sequence and KV head, token-major, are cut into
// blocks of 32 per wavefront.  Everything runs transposed, S^T = K . Q^T and O^T = V^T . P^T on 32 x 32 x 16 matrix
// instructions: a lane then holds one row's scores (half of the keys, its partner lane + 32 the other half), so that softmax
// statistics are sums inside the lane and one exchange with the partner, and a lane's probabilities are, as they are, the
// right operand of the second product: its 16 keys are merely taken in the order the first product left them, by reading V's
// rows in that order.
#ifndef ETC_GENERIC_ONLY
#include "chunk_attn_rt.hip.h"

namespace etc {

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

// LDS of a piece: rows of K and V, and the ids of its pages, a window of them at a time.
template <int D>
struct Tiles {
    uint16_t rows[512 * D];                 // 128 KB for heads of 128
    int ids[kCaIds];
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
    PageWindow<> W{io.block_table + (int64_t)P.b * io.table_stride, 0, 0};
    W.load<SRV_ATTENTION>(S, io, B.ids, P.b, tile0 * kCaKeys, key_end, tid);

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
                W.load<SRV_ATTENTION>(S, io, B.ids, P.b, (tile + 2) * kCaKeys, key_end, tid);
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
    PageWindow<> W{io.block_table + (int64_t)P.b * io.table_stride, 0, 0};
    W.load<SRV_ATTENTION>(S, io, B.ids, P.b, key0, key_end, tid);

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
                W.load<SRV_ATTENTION>(S, io, B.ids, P.b, k0 + 2 * KEYS, key_end, tid);
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
    const int n_pieces = cut<SRV_ATTENTION>(S, io, L);
    if (n_pieces == 0) return;
    for_pieces(S, io, L, n_pieces, [&](const Piece &P) {
        if (P.rows <= kCaNarrowRows) narrow_piece<D>(S, io, L, B, P);
        else wide_piece<D>(S, io, L, B, P);
    });
}

int64_t attention_slot_bytes(int head_dim) { return 4ll * (head_dim == 128 ? kCaSlot<128> : kCaSlot<64>); }

hipError_t launch_serving_attention(const ServingDev &S, const etc_serving_attention_io &io, hipStream_t s)
{
    const dim3 grid(attention_grid(S, io)), block(kCaThreads);
    if (S.d == 128) hipLaunchKernelGGL((chunk_attention_kernel<128>), grid, block, 0, s, S, io);
    else hipLaunchKernelGGL((chunk_attention_kernel<64>), grid, block, 0, s, S, io);
    return hipGetLastError();
}

}  // namespace etc
#endif  // ETC_GENERIC_ONLY
