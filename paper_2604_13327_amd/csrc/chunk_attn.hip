// Attention of a chunk of new tokens over the paged cache (include/etc.h, etc_serving_attention).
//
// A row of the problem is a (new token, query head) pair; the rows of one sequence and KV head, token-major, are cut into
// blocks of 32 per wavefront.  Everything runs transposed, S^T = K . Q^T and O^T = V^T . P^T on 32 x 32 x 16 matrix
// instructions: a lane then holds one row's scores (half of the keys, its partner lane + 32 the other half), so that softmax
// statistics are sums inside the lane and one exchange with the partner, and a lane's probabilities are, as they are, the
// right operand of the second product: its 16 keys are merely taken in the order the first product left them, by reading V's
// rows in that order.
#ifndef ETC_GENERIC_ONLY
#include "serving_rt.hip.h"

namespace etc {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;

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
    const int t_first = (r0 + wave * 32) / grp;          // of this wavefront: all its rows see the keys up to kv + t_first
    const int wave_full = it.kv + min(t_first, it.n_new - 1), wave_last = it.kv + min((r0 + wave * 32 + 31) / grp, it.n_new - 1);
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
#pragma unroll
        for (int u = 0; u < RPT; ++u) {
            const int key = key0 + RSTEP * u;
            const bool in = tile * kCaKeys + key < n_keys;      // rows behind the last key count nothing: zero, whatever the pool holds
            *reinterpret_cast<u32x4 *>(&s_k[buf][key * D + ((c ^ (key & 7)) * 8)]) = in ? kr[u] : u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4 *>(&s_v[buf][key * D + ((c ^ ((key & 3) * 2)) * 8)]) = in ? vr[u] : u32x4{0, 0, 0, 0};
        }
    };

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x16{};
    float m = -INFINITY, l = 0.f;                        // reference of the row's exponentials; sum over this lane's keys
    const float scale = 1.44269504088896f / sqrtf((float)D);

    load_ids(0);
    load_rows(0);
    load_ids(1 < n_tiles ? 1 : 0);
    store_rows(0, 0);
    if (n_tiles > 1) { load_rows(1); load_ids(2 < n_tiles ? 2 : 0); }
    __syncthreads();
    for (int tile = 0; tile < n_tiles; ++tile) {
        const int buf = tile & 1, k0 = tile * kCaKeys;
        if (wave_live && k0 <= wave_last) {
            // ---- scores: S^T[key][row], key = 32 kt + 8 (i / 4) + 4 half + i % 4 of register i
            f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    const int key = kt * 32 + col;
                    const bf16x8 a = *reinterpret_cast<const bf16x8 *>(&s_k[buf][key * D + (((ks * 2 + half) ^ (key & 7)) * 8)]);
                    s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[ks], s[kt], 0, 0, 0);
                }
            const bool masked = k0 + kCaKeys - 1 > wave_full;      // some row of the wavefront does not see all of the tile
            float mt = -INFINITY;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x = s[kt][i] * scale;
                    if (masked) x = k0 + kt * 32 + 8 * (i >> 2) + 4 * half + (i & 3) <= limit ? x : -INFINITY;
                    s[kt][i] = x;
                    mt = fmaxf(mt, x);
                }
            mt = partner_max(mt);
            const float nm = fmaxf(m, mt), ref = fmaxf(nm, -1e30f);      // all scores -inf so far: exp2(-inf - ref) = 0, no NaN
            const float sc = exp2_fast(m - ref);
            m = nm;
            float sum = 0.f;
            uint32_t p[2][8];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float a = exp2_fast(s[kt][i] - ref), b = exp2_fast(s[kt][i + 1] - ref);
                    sum += a + b;
                    p[kt][i >> 1] = to_bf16x2(a, b);     // half a unit of bf16 of a probability: below the rounding of the output
                }
            l = l * sc + sum;
            if (__builtin_amdgcn_ballot_w64(sc != 1.0f) != 0) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] *= sc;
            }
            // ---- O^T += V^T . P^T: 16 keys a step, in the order the scores have them: rows 4 half + 0 .. 3 and 8 + 4 half + 0 .. 3
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const uint32_t *pp = &p[ks >> 1][(ks & 1) * 4];
                const bf16x8 pb = __builtin_bit_cast(bf16x8, u32x4{pp[0], pp[1], pp[2], pp[3]});
                const int vrow = ks * 16 + 4 * half + ((lane & 15) >> 2), sw = (vrow & 3) * 2;      // also of row + 8
                bf16x8 vf[DT];
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const int piece = dt * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
                    ETC_AS_LDS uint16_t *at = as_lds(&s_v[buf][vrow * D + ((piece ^ sw) * 8) + (lane & 1) * 4]);
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ETC_AS_LDS s16x4 *>(at));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<ETC_AS_LDS s16x4 *>(at + 8 * D));
                    const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
                    vf[dt] = __builtin_bit_cast(bf16x8, u32x4{a.x, a.y, b.x, b.y});
                }
                if (masked) {
                    // Keys some rows of the wavefront do not see: their probability 0 would make a NaN of an infinite or NaN
                    // value.  Such values (exponent all ones) are taken out of the product and counted by kind in a second
                    // one over the keys each row sees: +inf as 1, -inf as 2^8, NaN as 2^16 (at most 64 of each: exact).
                    uint32_t odd = 0;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        const u32x4 w = __builtin_bit_cast(u32x4, vf[dt]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) odd |= ((w[i] & 0x7F80u) == 0x7F80u) | ((w[i] & 0x7F800000u) == 0x7F800000u);
                    }
                    if (__builtin_amdgcn_ballot_w64(odd != 0) != 0) {
                        uint32_t seen[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int kk = k0 + ks * 16 + 4 * half + (i >> 1) * 8 + (i & 1) * 2;
                            seen[i] = (kk <= limit ? 0x3F80u : 0u) | (kk + 1 <= limit ? 0x3F800000u : 0u);
                        }
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            u32x4 w = __builtin_bit_cast(u32x4, vf[dt]), kind;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint32_t out = 0, keep = 0;
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const uint32_t e = (w[i] >> (16 * h)) & 0xFFFFu;
                                    const uint32_t code = (e & 0x7FFFu) > 0x7F80u ? 0x4780u : e == 0x7F80u ? 0x3F80u : e == 0xFF80u ? 0x4380u : 0u;
                                    out |= code << (16 * h);
                                    keep |= (code ? 0u : e) << (16 * h);
                                }
                                kind[i] = out;
                                w[i] = keep;
                            }
                            vf[dt] = __builtin_bit_cast(bf16x8, w);
                            const f32x16 n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kind),
                                __builtin_bit_cast(bf16x8, u32x4{seen[0], seen[1], seen[2], seen[3]}), f32x16{}, 0, 0, 0);
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const uint32_t cnt = (uint32_t)n[i];
                                if (cnt & 0xFFu) o[dt][i] += INFINITY;
                                if (cnt & 0xFF00u) o[dt][i] -= INFINITY;
                                if (cnt >> 16) o[dt][i] = __uint_as_float(0x7FC00000u);
                            }
                        }
                    }
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt], pb, o[dt], 0, 0, 0);
            }
        }
        if (tile + 1 < n_tiles) {
            store_rows(tile + 1, buf ^ 1);
            if (tile + 2 < n_tiles) {
                load_rows(tile + 2);
                load_ids(tile + 3 < n_tiles ? tile + 3 : 0);
            }
        }
        __syncthreads();
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
