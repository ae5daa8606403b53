// Per-head norms, RoPE and append of a chunk of new tokens to a paged cache of 8 bits (include/etc.h, etc_serving_append_codes).
//
// A page's tokens of one KV head share a scale, so their rows in the call, a run, are one wavefront's: it holds 16 elements of a row in
// a lane, D / 16 neighbouring lanes to a row (8 of the first half and the 8 they are rotated with), 16 rows at once, finds the largest of all
// by lane moves, and writes codes; longer runs are gone through twice.  Queries have no scale: they are rows as in serving_append_kernel, in workgroups of their own behind the others.
#ifndef ETC_GENERIC_ONLY
#include "codes_rt.hip.h"

namespace etc {

constexpr int kAp8Threads = 256, kAp8Waves = kAp8Threads / 64;
constexpr int kAp8Rows = 16;                // of the angles in LDS, and of a run in registers
constexpr int kAp8LowByte = 127 - 40;       // of a scale
constexpr int kAp8HighByte = 127 + 120;     // of 2^128 / 448

template <int D>
struct Angles { float c[kAp8Rows][D / 2], s[kAp8Rows][D / 2]; };

// Sine and cosine of the rows r0 .. r0 + n - 1.  The angle in fp64, reduced to half a turn: positions run into the millions.
template <int D>
__device__ __forceinline__ void fill_angles(ETC_AS_LDS Angles<D> &A, const ServingDev &S, const int32_t *positions, int r0, int n)
{
    for (int i = (int)threadIdx.x; i < n * (D / 2); i += kAp8Threads) {
        const int t = i / (D / 2), e = i - t * (D / 2);
        const double turns = (double)gld_i32(positions + r0 + t) * *as_global(S.inv_freq + e) * 0.15915494309189535;
        float sn, cs;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
        A.c[t][e] = cs;
        A.s[t][e] = sn;
    }
}

// The 8 + 8 elements of a lane.
template <int D, bool F32>
__device__ __forceinline__ void load_head(float (&a)[8], float (&b)[8], const void *src, int64_t at)
{
    if (F32) {
        const float *p = (const float *)src + at;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4 x = __builtin_bit_cast(f32x4, gld_16B(p + 4 * i)), y = __builtin_bit_cast(f32x4, gld_16B(p + D / 2 + 4 * i));
#pragma unroll
            for (int j = 0; j < 4; ++j) { a[4 * i + j] = x[j]; b[4 * i + j] = y[j]; }
        }
    } else {
        const uint16_t *p = (const uint16_t *)src + at;
        const u32x4 x = gld_16B(p), y = gld_16B(p + D / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) { a[2 * i] = bf16_lo(x[i]); a[2 * i + 1] = bf16_hi(x[i]); b[2 * i] = bf16_lo(y[i]); b[2 * i + 1] = bf16_hi(y[i]); }
    }
}

template <int D>
__device__ __forceinline__ void norm_head(float (&a)[8], float (&b)[8], const void *gain, int c, float eps)
{
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += a[i] * a[i] + b[i] * b[i];
    const float rn = 1.0f / sqrtf(head_sum<D>(ss) / (float)D + eps);
    const uint16_t *g = (const uint16_t *)gain + c;
    const u32x4 ga = gld_16B(g), gb = gld_16B(g + D / 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[2 * i] *= rn * bf16_lo(ga[i]); a[2 * i + 1] *= rn * bf16_hi(ga[i]);
        b[2 * i] *= rn * bf16_lo(gb[i]); b[2 * i + 1] *= rn * bf16_hi(gb[i]);
    }
}

template <int D>
__device__ __forceinline__ void rotate_head(float (&a)[8], float (&b)[8], ETC_AS_LDS const Angles<D> &A, int t, int c)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float cs = A.c[t][c + i], sn = A.s[t][c + i], x = a[i], y = b[i];
        a[i] = x * cs - y * sn;
        b[i] = x * sn + y * cs;
    }
}

// Blocks [0, kv_groups * kv_wgs): runs that begin in rows [g * rows_per_wg, ..), heads 4 h .. of K or V.  Blocks behind: queries.
template <int D, bool F32>
__global__ __launch_bounds__(kAp8Threads) void serving_append_codes_kernel(ServingDev S, etc_serving_append_codes_io io8, int rows_per_wg, int kv_groups, int kv_wgs, int q_tokens)
{
    constexpr int LPH = D / 16, RPI = 64 / LPH, ITERS = kAp8Rows / RPI;     // lanes to a row, rows at once, times
    __shared__ Angles<D> s_angles;
    ETC_AS_LDS Angles<D> &A = *as_lds(&s_angles);
    const etc_serving_append_io &io = io8.append;
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
    const int psh = S.page_shift, pmask = (1 << psh) - 1, n_slots = (int)(io.n_pages << psh), c = (lane % LPH) * 8;

    if ((int)blockIdx.x >= kv_groups * kv_wgs) {         // queries
        const int t0 = ((int)blockIdx.x - kv_groups * kv_wgs) * q_tokens, nt = min(q_tokens, io.n_tokens - t0);
        fill_angles<D>(A, S, io.positions, t0, nt);
        __syncthreads();
        for (int r = tid / LPH; r < nt * S.nq; r += kAp8Threads / LPH) {
            const int t = r / S.nq, h = r - t * S.nq, row = t0 + t;
            const int slot = gld_i32(io.slots + row);
            if (slot < 0 || slot >= n_slots) continue;   // the same for all lanes of a head
            float a[8], b[8];
            load_head<D, F32>(a, b, io.q, (int64_t)row * io.q_stride + h * D + c);
            if (S.qk_norm) norm_head<D>(a, b, io.gq, c, S.eps);
            rotate_head<D>(a, b, A, t, c);
            uint16_t *dst = (uint16_t *)io.q_out + ((int64_t)row * S.nq + h) * D + c;
            u32x4 x, y;
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = to_bf16x2(a[2 * i], a[2 * i + 1]); y[i] = to_bf16x2(b[2 * i], b[2 * i + 1]); }
            *as_global(reinterpret_cast<u32x4 *>(dst)) = x;
            *as_global(reinterpret_cast<u32x4 *>(dst + D / 2)) = y;
        }
        return;
    }

    const int part = (int)blockIdx.x % kv_wgs, group = (int)blockIdx.x / kv_wgs, head_groups = kv_wgs / 2;
    const bool is_v = part >= head_groups;
    const int h = (is_v ? part - head_groups : part) * kAp8Waves + wave;
    const bool mine = h < S.nkv;
    const void *src = is_v ? io.v : io.k;
    const int64_t stride = is_v ? io.v_stride : io.k_stride;
    uint8_t *codes = (uint8_t *)(is_v ? io.v_pages : io.k_pages), *scales = (uint8_t *)(is_v ? io8.v_scale : io8.k_scale);
    const int row0 = group * rows_per_wg, row1 = min(row0 + rows_per_wg, io.n_tokens);
    // Rows with no slot of the pool are left out, wherever they stand.  The first row of 64, from `row` on in steps of `by`, that is not; -1: none.
    auto live_from = [&](int row, int by) {
        for (; row >= 0 && row < io.n_tokens; row += 64 * by) {
            const int i = row + lane * by;
            const uint64_t live = __builtin_amdgcn_ballot_w64(i >= 0 && i < io.n_tokens && (uint32_t)gld_i32(io.slots + min(max(i, 0), io.n_tokens - 1)) < (uint32_t)n_slots);
            if (live != 0) return row + (int)__builtin_ctzll(live) * by;
        }
        return -1;
    };
    auto slot_at = [&](int row) { return __builtin_amdgcn_readfirstlane(gld_i32(io.slots + row)); };
    for (int r = row0; r < row1; ++r) {                  // (everything up to the head's part is the same for the workgroup)
        const int slot = slot_at(r), off = slot & pmask;
        if (slot < 0) continue;
        if (slot >= n_slots) {
            if (part == 0 && tid == 0) refuse(S.error, SRV_BAD_SLOT, SRV_APPEND_CODES, r, slot);
            continue;
        }
        if (off != 0 && r > 0) {
            const int before = live_from(r - 1, -1);
            if (before >= 0 && slot_at(before) == slot - 1) continue;      // of an earlier row's run
        }
        const int64_t page = slot >> psh;
        float a[ITERS][8], b[ITERS][8];
        // Rows row .. of the run, nr of them, up to kAp8Rows (those behind are the last one again): the values that are to be stored, in a and b.
        auto values = [&](int row, int nr) {
            if (!is_v) {
                __syncthreads();                         // who reads the angles of the rows before
                fill_angles<D>(A, S, io.positions, row, nr);
            }
            if (mine) {
#pragma unroll
                for (int u = 0; u < ITERS; ++u)
                    load_head<D, F32>(a[u], b[u], src, (int64_t)(row + min(u * RPI + lane / LPH, nr - 1)) * stride + h * D + c);
            }
            if (!is_v) __syncthreads();
            if (!mine) return;
#pragma unroll
            for (int u = 0; u < ITERS; ++u) {
                if (!is_v) {
                    if (S.qk_norm) norm_head<D>(a[u], b[u], io.gk, c, S.eps);
                    rotate_head<D>(a[u], b[u], A, min(u * RPI + lane / LPH, nr - 1), c);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) { a[u][i] = finite_or_nan(a[u][i]); b[u][i] = finite_or_nan(b[u][i]); }
            }
        };
        // The run, up to kAp8Rows rows without one left out between them at a time: f(first row, its slot, rows).  Returns how often.
        auto for_run = [&](auto f) {
            int row = r, at = slot, times = 0;
            for (;;) {
                const bool goes_on = lane < kAp8Rows && (at & pmask) + lane <= pmask && row + lane < io.n_tokens && gld_i32(io.slots + min(row + lane, io.n_tokens - 1)) == at + lane;
                const int nr = (int)__builtin_ctzll(~__builtin_amdgcn_ballot_w64(goes_on));      // at least 1
                f(row, at, nr);
                ++times;
                at += nr;
                if ((at & pmask) == 0 || row + nr >= io.n_tokens) return times;
                row = live_from(row + nr, 1);
                if (row < 0 || slot_at(row) != at) return times;
            }
        };
        float most = 0.f;
        const int times = for_run([&](int row, int, int nr) {
            values(row, nr);
            if (!mine) return;
#pragma unroll
            for (int u = 0; u < ITERS; ++u)
#pragma unroll
                for (int i = 0; i < 8; ++i) most = fmaxf(most, fmaxf(fabsf(a[u][i]), fabsf(b[u][i])));
        });
        int byte = scale_byte(wave_max_f(most), kAp8LowByte);
        if (mine) {
            uint8_t *const scale = scales + page * S.nkv + h;
            if (off > 0) {
                const int before = __builtin_amdgcn_readfirstlane((int)*as_global(scale));
                if (byte > before) {                     // the tokens in front, in the new scale
                    const float f = __uint_as_float((uint32_t)max(127 + before - byte, 0) << 23);
                    for (int64_t i = lane; i < (int64_t)off * (D / 8); i += 64) {
                        uint8_t *const at = codes + ((page << psh) + i / (D / 8)) * S.nkv * D + h * D + i % (D / 8) * 8;
                        u32x2 w = *as_global(reinterpret_cast<u32x2 *>(at));
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const f32x4 x = from_f8x4(w[j]);
                            w[j] = to_f8x4(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
                        }
                        *as_global(reinterpret_cast<u32x2 *>(at)) = w;
                    }
                } else {
                    byte = min(before, kAp8HighByte);
                }
            }
            if (lane == 0) *as_global(scale) = (uint8_t)byte;
        }
        const float inv = one_over_scale(byte);
        auto store = [&](int, int at, int nr) {
            if (!mine) return;
#pragma unroll
            for (int u = 0; u < ITERS; ++u) {
                const int i = u * RPI + lane / LPH;
                if (i >= nr) continue;
                uint8_t *const dst = codes + ((int64_t)at + i) * S.nkv * D + h * D + c;
                const float *x = a[u], *y = b[u];
                *as_global(reinterpret_cast<u32x2 *>(dst)) = u32x2{to_f8x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), to_f8x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv)};
                *as_global(reinterpret_cast<u32x2 *>(dst + D / 2)) = u32x2{to_f8x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), to_f8x4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
            }
        };
        if (times == 1) for_run(store);                  // the values are there still
        else for_run([&](int row, int at, int nr) { values(row, nr); store(row, at, nr); });
    }
}

hipError_t launch_serving_append_codes(const ServingDev &S, const etc_serving_append_codes_io &io, hipStream_t s)
{
    const int n = io.append.n_tokens;
    int rows = 1;                                        // that a workgroup looks for runs in
    while (rows < kAp8Rows && rows * S.n_cus < n) rows *= 2;
    int q_tokens = kAp8Threads / (S.nq * (S.d / 16));
    if (q_tokens < 1) q_tokens = 1;
    if (q_tokens > kAp8Rows) q_tokens = kAp8Rows;
    const int kv_groups = (n + rows - 1) / rows, kv_wgs = 2 * ((S.nkv + kAp8Waves - 1) / kAp8Waves);
    const dim3 grid((unsigned)kv_groups * kv_wgs + (unsigned)((n + q_tokens - 1) / q_tokens)), block(kAp8Threads);
    const bool f32 = io.append.dtype == ETC_FP32;
    if (S.d == 128) {
        if (f32) hipLaunchKernelGGL((serving_append_codes_kernel<128, true>), grid, block, 0, s, S, io, rows, kv_groups, kv_wgs, q_tokens);
        else hipLaunchKernelGGL((serving_append_codes_kernel<128, false>), grid, block, 0, s, S, io, rows, kv_groups, kv_wgs, q_tokens);
    } else {
        if (f32) hipLaunchKernelGGL((serving_append_codes_kernel<64, true>), grid, block, 0, s, S, io, rows, kv_groups, kv_wgs, q_tokens);
        else hipLaunchKernelGGL((serving_append_codes_kernel<64, false>), grid, block, 0, s, S, io, rows, kv_groups, kv_wgs, q_tokens);
    }
    return hipGetLastError();
}

}  // namespace etc
#endif  // ETC_GENERIC_ONLY
