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
constexpr int kCaRows = 32 * kCaWaves;      // rows of a block
constexpr int kCaKeys = 64;                 // keys of a tile

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

// Which sequence and block of rows a workgroup has.
struct Item { int b, block, row0, n_new, kv; };      // row0: first row of q; n_new == 0: nothing

// Blocks of all sequences back to back; lengths out of range leave their sequence out.
__device__ Item find_item(const ServingDev &S, const etc_serving_attention_io &io, int want, int *s_sum)
{
    __shared__ Item s_item;
    __shared__ int s_wave[kCaWaves];
    const int tid = (int)threadIdx.x, grp = S.nq / S.nkv;
    if (tid == 0) s_item = Item{0, 0, 0, 0, 0};
    int done = 0;
    for (int b0 = 0; b0 < io.n_seqs; b0 += kCaThreads) {
        const int b = b0 + tid;
        int q0 = 0, n = 0, kv = 0, blocks = 0;
        if (b < io.n_seqs) {
            q0 = gld_i32(io.q_indptr + b);
            const int q1 = gld_i32(io.q_indptr + b + 1);
            kv = gld_i32(io.kv_len + b);
            n = q1 - q0;
            const bool ok = q0 >= 0 && q1 >= q0 && q1 <= io.n_tokens && kv >= 0 && kv <= S.max_kv_len && n <= S.max_kv_len - kv &&
                            (int)(((unsigned)(kv + n) + (1u << S.page_shift) - 1) >> S.page_shift) <= io.table_cols;
            if (!ok) {
                if (blockIdx.x == 0 && blockIdx.y == 0) refuse(S.error, SRV_BAD_LENGTH, SRV_ATTENTION, b, kv);
                n = 0;
            }
            blocks = (n * grp + kCaRows - 1) / kCaRows;      // n * grp <= 2^26
        }
        int sum = wave_scan_i(blocks);
        if (lane_id() == 63) s_wave[wave_id()] = sum;
        __syncthreads();
        for (int w = 0; w < wave_id(); ++w) sum += s_wave[w];
        if (want >= done + sum - blocks && want < done + sum) s_item = Item{b, want - (done + sum - blocks), q0, n, kv};
        for (int w = 0; w < kCaWaves; ++w) done += s_wave[w];
        __syncthreads();
    }
    return lds_get_uniform(&s_item);
}

template <int D>
__global__ __launch_bounds__(kCaThreads) void chunk_attention_kernel(ServingDev S, etc_serving_attention_io io)
{
    constexpr int CH = D / 8;                            // 16-byte pieces of a row
    constexpr int KS = D / 16, DT = D / 32;              // steps of the first product, tiles of the output
    constexpr int RPT = kCaKeys * CH / kCaThreads;       // pieces of K (and of V) a thread stages
    constexpr int RSTEP = kCaThreads / CH;               // rows between them
    __shared__ __attribute__((aligned(16))) uint16_t s_k[2][kCaKeys * D], s_v[2][kCaKeys * D];
    __shared__ int s_odd[2];
    const int tid = (int)threadIdx.x, wave = wave_id(), lane = lane_id(), half = lane >> 5, col = lane & 31;
    const Item it = find_item(S, io, (int)blockIdx.x, nullptr);
    if (it.n_new == 0) return;
    const int kvh = (int)blockIdx.y, grp = S.nq / S.nkv, psh = S.page_shift, pmask = (1 << psh) - 1;
    const int rows = it.n_new * grp, r0 = it.block * kCaRows;

    // this lane's row: query fragments (right operand: 8 consecutive elements of step ks at ks * 16 + half * 8)
    const int row = r0 + wave * 32 + col, rr = min(row, rows - 1), t = rr / grp, head = kvh * grp + (rr - t * grp);
    const uint16_t *qp = (const uint16_t *)io.q + ((int64_t)(it.row0 + t) * S.nq + head) * D + half * 8;
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, gld_16B(qp + ks * 16));
    const int limit = it.kv + t;                         // last key this row sees
    const int t_last = min(r0 + kCaRows - 1, rows - 1) / grp, n_keys = it.kv + t_last + 1;      // keys of the block
    const int first_masked = (it.kv + r0 / grp + 1) / kCaKeys;      // tiles in front of it are seen whole by all rows of the block
    const int wave_last = it.kv + min((r0 + wave * 32 + 31) / grp, it.n_new - 1);
    const bool wave_live = r0 + wave * 32 < rows;
    const int n_tiles = (n_keys + kCaKeys - 1) / kCaKeys;

    // staging: thread has piece c of rows key0 + RSTEP * u of a tile
    const int c = tid % CH, key0 = tid / CH;
    const int32_t *table = io.block_table + (int64_t)it.b * io.table_stride;
    int ids[RPT];
    u32x4 kr[RPT], vr[RPT];
    auto load_ids = [&](int tile) {
#pragma unroll
        for (int u = 0; u < RPT; ++u) ids[u] = gld_i32(table + (min(tile * kCaKeys + key0 + RSTEP * u, n_keys - 1) >> psh));
    };
    auto load_rows = [&](int tile) {
#pragma unroll
        for (int u = 0; u < RPT; ++u) {
            const int key = min(tile * kCaKeys + key0 + RSTEP * u, n_keys - 1);
            int id = ids[u];
            if ((uint32_t)id >= (uint64_t)io.n_pages) {
                refuse(S.error, SRV_BAD_PAGE, SRV_ATTENTION, it.b, id);
                id = 0;
            }
            const int64_t off = (((int64_t)id << psh) + (key & pmask)) * (S.nkv * D) + kvh * D + c * 8;
            kr[u] = gld_16B((const uint16_t *)io.k_pages + off);
            vr[u] = gld_16B((const uint16_t *)io.v_pages + off);
        }
    };
    // LDS rows: the 16-byte pieces of a row change places with the row (exclusive or), so that lanes reading one piece of
    // neighbouring rows meet different banks: K by the row's low 3 bits (8 lanes an access), V by pairs of pieces (4 rows an access).
    auto store_rows = [&](int tile, int buf) {
        bool odd = false;
#pragma unroll
        for (int u = 0; u < RPT; ++u) {
            const int key = key0 + RSTEP * u;
            if ((tile + 1) * kCaKeys > n_keys && tile * kCaKeys + key >= n_keys)      // behind the last key: zero, whatever the pool holds
                kr[u] = vr[u] = u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4 *>(&s_k[buf][key * D + ((c ^ (key & 7)) * 8)]) = kr[u];
            *reinterpret_cast<u32x4 *>(&s_v[buf][key * D + ((c ^ ((key & 3) * 2)) * 8)]) = vr[u];
            if (tile >= first_masked) {
#pragma unroll
                for (int i = 0; i < 4; ++i) odd |= (vr[u][i] & 0x7F80u) == 0x7F80u || (vr[u][i] & 0x7F800000u) == 0x7F800000u;
            }
        }
        if (odd) s_odd[buf] = 1;                         // stays: the tiles behind it are masked too
    };

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x16{};
    float m = -3e38f, l = 0.f;                           // reference of the row's exponentials; sum over this lane's keys
    const float scale = 1.44269504088896f / sqrtf((float)D);      // scores and reference count in powers of two

    // Fragments in LDS.  The exchange of pieces touches the low 3 bits of a piece's number, so that every fragment lies at a constant
    // distance from one of a few addresses: K of step ks at k_at[ks % 4] (and 8 pieces behind for ks >= 4), V of tile dt at v_at[dt % 2].
    constexpr int ROW = D * 2, BUF = kCaKeys * ROW;      // bytes
    uint32_t k_at[4], v_at[2];
    {
        const uint32_t kb = (uint32_t)(uintptr_t)as_lds(&s_k[0][0]), vb = (uint32_t)(uintptr_t)as_lds(&s_v[0][0]);
#pragma unroll
        for (int i = 0; i < 4; ++i) k_at[i] = kb + col * ROW + (((i * 2 + half) ^ (col & 7)) * 16);
        const int vrow = 4 * half + ((lane & 15) >> 2), piece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
#pragma unroll
        for (int i = 0; i < 2; ++i) v_at[i] = vb + vrow * ROW + (((i * 4 + piece) ^ ((vrow & 3) * 2)) * 16) + (lane & 1) * 8;
    }
    auto k_frag = [&](int buf, int ks, int kt) {
        return *reinterpret_cast<ETC_AS_LDS const bf16x8 *>(k_at[ks & 3] + buf * BUF + kt * 32 * ROW + (ks >> 2) * 128);
    };
    // V^T fragment of 32 elements (tile dt) x 16 keys (step ks), the keys in the order the scores have them: rows 4 half + 0 .. 3
    // and 8 + 4 half + 0 .. 3 of the step.
    auto v_frag = [&](int buf, int ks, int dt) {
        const uint32_t at = v_at[dt & 1] + buf * BUF + ks * 16 * ROW + (dt >> 1) * 128;
        const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ETC_AS_LDS s16x4 *>(at)));
        const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ETC_AS_LDS s16x4 *>(at + 8 * ROW)));
        return u32x4{a.x, a.y, b.x, b.y};
    };
    // One tile.  MASKED: some row of the block does not see all of it.
    auto step = [&](auto masked_c, int tile) {
        constexpr bool MASKED = decltype(masked_c)::value;
        const int buf = tile & 1, k0 = tile * kCaKeys;
        // ---- scores: S^T[key][row], key = 32 kt + 8 (i / 4) + 4 half + i % 4 of register i
        f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(buf, ks, kt), qf[ks], s[kt], 0, 0, 0);
        if constexpr (MASKED) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (k0 + kt * 32 + 8 * (i >> 2) + 4 * half + (i & 3) > limit) s[kt][i] = -INFINITY;
        }
        float mt = s[0][0];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) mt = fmaxf(mt, s[kt][i]);
        mt = partner_max(mt) * scale;
        // The reference follows the maximum only when that has grown by 2^8 (rows of a wavefront together): until then
        // probabilities up to 2^8 lose nothing, and the running output need not be multiplied.
        if (__builtin_amdgcn_ballot_w64(mt > m + 8.f) != 0) {
            const float nm = fmaxf(m, mt), sc = exp2_fast(m - nm);
            m = nm;
            l *= sc;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] *= sc;
        }
        bool odd = false;
        if constexpr (MASKED) {
            // Keys some rows do not see: their probability 0 would make a NaN of an infinite or NaN value.  A tile that holds
            // such values (exponent all ones) has them taken out of the product, and counted by kind in a second one over the
            // keys each row sees: +inf as 1, -inf as 2^8, NaN as 2^16 (at most 64 of each: exact).
            odd = s_odd[buf] != 0;
            if (odd) {
                auto count = [&](int dt) {
                    f32x16 n{};
#pragma unroll 1
                    for (int ks = 0; ks < 4; ++ks) {
                        const u32x4 w = v_frag(buf, ks, dt);
                        u32x4 kind, seen;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = k0 + ks * 16 + 4 * half + (i >> 1) * 8 + (i & 1) * 2;
                            seen[i] = (key <= limit ? 0x3F80u : 0u) | (key + 1 <= limit ? 0x3F800000u : 0u);
                            kind[i] = odd_kind(w[i] & 0xFFFFu) | odd_kind(w[i] >> 16) << 16;
                        }
                        n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kind), __builtin_bit_cast(bf16x8, seen), n, 0, 0, 0);
                    }
                    return n;
                };
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const f32x16 n = count(dt);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t c = (uint32_t)n[i];
                        if (c & 0xFFu) o[dt][i] += INFINITY;
                        if (c & 0xFF00u) o[dt][i] -= INFINITY;
                        if (c >> 16) o[dt][i] = __uint_as_float(0x7FC00000u);
                    }
                }
            }
        }
        // ---- probabilities of 32 keys, then O^T += V^T . P^T over them
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            uint32_t p[8];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float a = exp2_fast(__builtin_fmaf(s[kt][i], scale, -m)), b = exp2_fast(__builtin_fmaf(s[kt][i + 1], scale, -m));
                p[i >> 1] = to_bf16x2(a, b);             // half a unit of bf16 of a probability: below the rounding of the output
                l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(s16x2, p[i >> 1]), __builtin_bit_cast(s16x2, 0x3F803F80u), l, false);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{p[4 * h], p[4 * h + 1], p[4 * h + 2], p[4 * h + 3]});
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    u32x4 w = v_frag(buf, kt * 2 + h, dt);
                    if constexpr (MASKED) {
                        if (odd) {
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                w[i] &= ((w[i] & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((w[i] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
                        }
                    }
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), pb, o[dt], 0, 0, 0);
                }
            }
        }
    };

    if (tid < 2) s_odd[tid] = 0;
    load_ids(0);
    load_rows(0);
    load_ids(1 < n_tiles ? 1 : 0);
    __syncthreads();
    store_rows(0, 0);
    if (n_tiles > 1) { load_rows(1); load_ids(2 < n_tiles ? 2 : 0); }
    __syncthreads();
    auto next = [&](int tile) {                          // the tile behind `tile` into the other buffer, the one behind that on its way
        if (tile + 1 < n_tiles) {
            store_rows(tile + 1, (tile & 1) ^ 1);
            if (tile + 2 < n_tiles) {
                load_rows(tile + 2);
                load_ids(tile + 3 < n_tiles ? tile + 3 : 0);
            }
        }
        __syncthreads();
    };
    int tile = 0;
    for (; tile < min(first_masked, n_tiles); ++tile) {
        if (wave_live) step(std::false_type(), tile);
        next(tile);
    }
    for (; tile < n_tiles; ++tile) {
        if (wave_live && tile * kCaKeys <= wave_last) step(std::true_type(), tile);
        next(tile);
    }
    if (row >= rows) return;
    const float inv = 1.0f / partner_sum(l);
    uint16_t *op = (uint16_t *)io.out + ((int64_t)(it.row0 + t) * S.nq + head) * D + half * 4;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *as_global(reinterpret_cast<u32x2 *>(op + dt * 32 + q * 8)) =
                u32x2{to_bf16x2(o[dt][4 * q] * inv, o[dt][4 * q + 1] * inv), to_bf16x2(o[dt][4 * q + 2] * inv, o[dt][4 * q + 3] * inv)};
}

hipError_t launch_serving_attention(const ServingDev &S, const etc_serving_attention_io &io, hipStream_t s)
{
    const int grp = S.nq / S.nkv;
    const int64_t blocks = (int64_t)io.n_tokens * grp / kCaRows + (io.n_seqs < io.n_tokens ? io.n_seqs : io.n_tokens);
    const dim3 grid((unsigned)blocks, (unsigned)S.nkv), block(kCaThreads);
    if (S.d == 128) hipLaunchKernelGGL((chunk_attention_kernel<128>), grid, block, 0, s, S, io);
    else hipLaunchKernelGGL((chunk_attention_kernel<64>), grid, block, 0, s, S, io);
    return hipGetLastError();
}

}  // namespace etc
#endif  // ETC_GENERIC_ONLY
