// Per-head norms, RoPE and append of a chunk of new tokens to a paged cache of 8 bits (include/etc.h, etc_serving_append_codes).
//
// A page's tokens of one KV head share a scale, so their rows in the call, a run, are one wavefront's: it holds 16 elements of a row in
// a lane, D / 16 neighbouring lanes to a row (8 of the first half and the 8 they are rotated with), 16 rows at once, finds the largest of all
// by lane moves, and writes codes; longer runs are gone through twice.  Pages of more than 32 tokens are a workgroup's.  Queries have no scale: they are rows as in serving_append_kernel, in workgroups of
// their own behind the others (in front of them, and of the runs' chains of loads, 66 us instead of 60 for the 7328 rows below).
// Bound by memory: 7328 rows in bf16 of 64 + 2 * 8 heads of 128 take 60 us, 4.8 TB/s of the 285 MB that they read and write, a large copy's rate; 1000
// rows of 32 + 2 * 8 heads 11 us (22.5 MB: 4.6), and three tokens 4.3: there a chain of slots, rows, angles and a largest value.
#ifndef ETC_GENERIC_ONLY
#include <type_traits>

#include "codes_rt.hip.h"

namespace etc {

constexpr int kAp8Threads = 256, kAp8Waves = kAp8Threads / 64;
constexpr int kAp8Rows = 16;                // of the angles in LDS, and of a run in registers
constexpr int kAp8Heads = 2;                // queries of a lane at once
constexpr int kAp8LowByte = 127 - 40;       // of a scale
constexpr int kAp8HighByte = 127 + 120;     // of 2^128 / 448
constexpr int kAp8GridX = 1 << 23;          // workgroups in a row of the grid: a dimension takes less than 2^32 threads (2^20 rows of 128 KV heads ask for more)

template <int D, int ROWS>
struct Angles { float c[ROWS][D / 2], s[ROWS][D / 2]; };

// Sine and cosine of n rows (at most ROWS), whose positions are position(row); a thread has one frequency.  The angle in fp64, reduced to half
// a turn, since positions run into the millions, and rounded to fp32 there: 2^-25 of half a turn at most, about what a rotation's
// products and sum are rounded by.
template <int D, int ROWS, class Position>
__device__ __forceinline__ void fill_angles(ETC_AS_LDS Angles<D, ROWS> &A, double freq, int n, Position position)
{
    constexpr int AT_ONCE = kAp8Threads / (D / 2), TIMES = ROWS / AT_ONCE;
    const int t0 = (int)threadIdx.x / (D / 2), e = (int)threadIdx.x % (D / 2);
    int p[TIMES];
#pragma unroll
    for (int k = 0; k < TIMES; ++k) p[k] = position(min(t0 + k * AT_ONCE, n - 1));
#pragma unroll
    for (int k = 0; k < TIMES; ++k) {
        const int t = t0 + k * AT_ONCE;
        if (t >= n) break;
        const double turns = (double)p[k] * freq * 0.15915494309189535;
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

template <int D, int ROWS>
__device__ __forceinline__ void rotate_head(float (&a)[8], float (&b)[8], ETC_AS_LDS const Angles<D, ROWS> &A, int t, int c)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float cs = A.c[t][c + i], sn = A.s[t][c + i], x = a[i], y = b[i];
        a[i] = x * cs - y * sn;
        b[i] = x * sn + y * cs;
    }
}

// Workgroups [0, kv_blocks): runs that begin in rows [g * rows_per_wg, ..), of K or V, and SHARED: a head, whose runs the wavefronts share, 16 rows of
// 64 each; else heads 4 h .., one to a wavefront.  Those behind: queries.
// SHARED is for pages of more than 32 tokens: 8192 rows of a prompt, 32 + 2 * 8 heads of 128, not shared and shared, in us, by the page's tokens:
// 16 34 and -, 32 55 and 69, 64 89 and 59, 128 162 and 85, 256 163 and 93, 1024 604 and 230 (and of smaller pages 4 45 and -, 1 107 and -).
template <int D, bool F32, bool SHARED>
__global__ __launch_bounds__(kAp8Threads) void serving_append_codes_kernel(ServingDev S, etc_serving_append_codes_io io8, int rows_per_wg, int kv_wgs, int kv_blocks, int q_tokens)
{
    constexpr int LPH = D / 16, RPI = 64 / LPH, ITERS = kAp8Rows / RPI;     // lanes to a row, rows at once, times
    constexpr int RPP = kAp8Threads / LPH;               // heads of a workgroup at once
    constexpr int ROWS = SHARED ? kAp8Waves * kAp8Rows : kAp8Rows;          // of a run at once
    __shared__ Angles<D, ROWS> s_angles;
    __shared__ float s_most[kAp8Waves];
    ETC_AS_LDS Angles<D, ROWS> &A = *as_lds(&s_angles);
    const etc_serving_append_io &io = io8.append;
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
    const int psh = S.page_shift, pmask = (1 << psh) - 1, n_slots = (int)(io.n_pages << psh), c = (lane % LPH) * 8;
    const int wg = (int)(blockIdx.y * gridDim.x + blockIdx.x);

    if (wg >= kv_blocks) {                               // queries
        const int t0 = (wg - kv_blocks) * q_tokens, nt = min(q_tokens, io.n_tokens - t0);
        if (nt <= 0) return;                             // the rest of the grid's last row
        const double freq = *as_global(S.inv_freq + tid % (D / 2));
        bool there = false;
        for (int r0 = tid / LPH; r0 < (nt * S.nq + RPP - 1) / RPP * RPP; r0 += RPP * kAp8Heads) {
            float a[kAp8Heads][8], b[kAp8Heads][8];      // asked for in front of the angles
            int slot[kAp8Heads];
#pragma unroll
            for (int u = 0; u < kAp8Heads; ++u) {
                const int r = min(r0 + u * RPP, nt * S.nq - 1), t = r / S.nq, h = r - t * S.nq;
                slot[u] = r0 + u * RPP < nt * S.nq ? gld_i32(io.slots + t0 + t) : -1;
                load_head<D, F32>(a[u], b[u], io.q, (int64_t)(t0 + t) * io.q_stride + h * D + c);
            }
            if (!there) {
                fill_angles(A, freq, nt, [&](int t) { return gld_i32(io.positions + t0 + t); });
                __syncthreads();
                there = true;
            }
#pragma unroll
            for (int u = 0; u < kAp8Heads; ++u) {
                if (slot[u] < 0 || slot[u] >= n_slots) continue;      // the same for all lanes of a head
                const int r = r0 + u * RPP, t = r / S.nq, h = r - t * S.nq;
                if (S.qk_norm) norm_head<D>(a[u], b[u], io.gq, c, S.eps);
                rotate_head(a[u], b[u], A, t, c);
                uint16_t *dst = (uint16_t *)io.q_out + ((int64_t)(t0 + t) * S.nq + h) * D + c;
                u32x4 x, y;
#pragma unroll
                for (int i = 0; i < 4; ++i) { x[i] = to_bf16x2(a[u][2 * i], a[u][2 * i + 1]); y[i] = to_bf16x2(b[u][2 * i], b[u][2 * i + 1]); }
                *as_global(reinterpret_cast<u32x4 *>(dst)) = x;
                *as_global(reinterpret_cast<u32x4 *>(dst + D / 2)) = y;
            }
        }
        return;
    }

    const int part = wg % kv_wgs, group = wg / kv_wgs, head_groups = kv_wgs / 2;
    const bool is_v = part >= head_groups;
    const int first = is_v ? part - head_groups : part, h = SHARED ? first : first * kAp8Waves + wave;
    const int u0 = SHARED ? wave * kAp8Rows : 0;         // this wavefront's part of ROWS
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
    // The slots of the rows, of 32 in front of them and of those behind, a row to a lane: mostly that tells all.  (Everything up to the
    // head's part is the same for the workgroup.)
    const int w0 = row0 - 32, at_lane = w0 + lane;
    const int slots = at_lane >= 0 && at_lane < io.n_tokens ? gld_i32(io.slots + min(max(at_lane, 0), io.n_tokens - 1)) : -1;
    const bool asked = lane >= 32 && at_lane < row1, live = (uint32_t)slots < (uint32_t)n_slots;
    if (asked && slots >= n_slots && part == 0 && wave == 0) refuse(S.error, SRV_BAD_SLOT, SRV_APPEND_CODES, at_lane, slots);
    const uint64_t lives = __builtin_amdgcn_ballot_w64(live), in_front = lives & ((1ull << lane) - 1);
    const int before_me = __shfl(slots, in_front != 0 ? 63 - __builtin_clzll(in_front) : 0, 64);
    const bool goes_on = (slots & pmask) != 0 && in_front != 0 && before_me == slots - 1;      // an earlier row's run
    uint64_t begins = __builtin_amdgcn_ballot_w64(asked && live && !goes_on);
    if (begins == 0) return;                             // (most workgroups of a prompt: in front of loads that all of them would ask for at once)
    double freq = 0.0;
    int positions = 0;
    if (!is_v) {
        freq = *as_global(S.inv_freq + tid % (D / 2));
        positions = gld_i32(io.positions + min(max(at_lane, 0), io.n_tokens - 1));
    }
    for (; begins != 0; begins &= begins - 1) {
        const int j = __builtin_ctzll(begins), r = w0 + j, slot = __builtin_amdgcn_readlane(slots, j), off = slot & pmask;
        if (off != 0 && (lives & ((1ull << j) - 1)) == 0 && w0 > 0) {
            const int before = live_from(w0 - 1, -1);
            if (before >= 0 && slot_at(before) == slot - 1) continue;
        }
        // its rows, as far as they stand side by side within the lanes; whole: those are all, and no more than ROWS
        const int n = __builtin_ctzll(~(__builtin_amdgcn_ballot_w64(lane >= j && slots == slot + (lane - j) && off + (lane - j) <= pmask) >> j));
        const uint64_t behind = j + n < 64 ? lives >> (j + n) << (j + n) : 0;
        const bool whole = n <= ROWS && (off + n > pmask || (behind != 0 ? __builtin_amdgcn_readlane(slots, __builtin_ctzll(behind)) != slot + n : w0 + 64 >= io.n_tokens));
        const int64_t page = slot >> psh;
        uint8_t *const scale = scales + page * S.nkv + h;
        int before = 0;                                  // the page's scale; asked for behind the rows, so that those do not wait for it
        float a[ITERS][8], b[ITERS][8];
        // Rows row .. of the run, nr of them, up to ROWS (those behind are the last one again): the values that are to be stored, in a and b.
        auto values = [&](int row, int nr) {
            if (mine) {
#pragma unroll
                for (int u = 0; u < ITERS; ++u)
                    load_head<D, F32>(a[u], b[u], src, (int64_t)(row + min(u0 + u * RPI + lane / LPH, nr - 1)) * stride + h * D + c);
                if (row == r) before = (int)*as_global(scale);
            }
            if (!is_v) {
                __syncthreads();                         // who reads the angles of the rows before
                fill_angles(A, freq, nr, [&](int t) { return whole ? __shfl(positions, j + t, 64) : gld_i32(io.positions + row + t); });
                __syncthreads();
            }
            if (!mine) return;
#pragma unroll
            for (int u = 0; u < ITERS; ++u) {
                if (!is_v) {
                    if (S.qk_norm) norm_head<D>(a[u], b[u], io.gk, c, S.eps);
                    rotate_head(a[u], b[u], A, min(u0 + u * RPI + lane / LPH, nr - 1), c);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) { a[u][i] = finite_or_nan(a[u][i]); b[u][i] = finite_or_nan(b[u][i]); }
            }
        };
        float most = 0.f, inv = 0.f;
        bool once = true;                                // the run's values are in a and b
        // Up to ROWS rows of the run without one left out between them at a time, for the largest value, then to be stored.
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            for (int row = r, at = slot;;) {
                int nr = n;
                if (!whole) {
                    const bool on = lane < ROWS && (at & pmask) + lane <= pmask && row + lane < io.n_tokens && gld_i32(io.slots + min(row + lane, io.n_tokens - 1)) == at + lane;
                    const uint64_t off_it = ~__builtin_amdgcn_ballot_w64(on);
                    nr = off_it != 0 ? (int)__builtin_ctzll(off_it) : 64;      // at least 1
                }
                if (pass == 0 || !once) values(row, nr);
                if (mine && pass == 0) {
#pragma unroll
                    for (int u = 0; u < ITERS; ++u)
#pragma unroll
                        for (int i = 0; i < 8; ++i) most = fmaxf(most, fmaxf(fabsf(a[u][i]), fabsf(b[u][i])));
                } else if (mine) {
#pragma unroll
                    for (int u = 0; u < ITERS; ++u) {
                        const int i = u0 + u * RPI + lane / LPH;
                        if (i >= nr) continue;
                        uint8_t *const dst = codes + ((int64_t)at + i) * S.nkv * D + h * D + c;
                        const float *x = a[u], *y = b[u];
                        *as_global(reinterpret_cast<u32x2 *>(dst)) = u32x2{to_f8x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), to_f8x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv)};
                        *as_global(reinterpret_cast<u32x2 *>(dst + D / 2)) = u32x2{to_f8x4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv), to_f8x4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv)};
                    }
                }
                at += nr;
                if (whole || (at & pmask) == 0 || row + nr >= io.n_tokens) break;
                row = live_from(row + nr, 1);
                if (row < 0 || slot_at(row) != at) break;
                once = false;
            }
            if (pass != 0 || !mine) continue;
            most = wave_max_f(most);
            if constexpr (SHARED) {
                if (lane == 0) s_most[wave] = most;
                asm volatile("" ::"v"(before));          // it is here: another wavefront writes the page's scale behind the barrier
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kAp8Waves; ++w) most = fmaxf(most, s_most[w]);
                __syncthreads();
            }
            int byte = scale_byte(most, kAp8LowByte);
            if (off > 0 && byte > before) {              // the tokens in front, in the new scale
                const float f = __uint_as_float((uint32_t)max(127 + before - byte, 0) << 23);
                const int64_t pieces = (int64_t)off * (D / 8);
                auto piece = [&](int64_t i) { return reinterpret_cast<u32x2 *>(codes + ((page << psh) + i / (D / 8)) * S.nkv * D + h * D + i % (D / 8) * 8); };
                constexpr int N = SHARED ? kAp8Threads : 64;
                for (int64_t i0 = SHARED ? tid : lane; i0 < pieces; i0 += 4 * N) {
                    u32x2 w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] = *as_global(piece(i0 + k * N < pieces ? i0 + k * N : i0));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const f32x4 x = from_f8x4(w[k][0]), y = from_f8x4(w[k][1]);
                        w[k] = u32x2{to_f8x4(x[0] * f, x[1] * f, x[2] * f, x[3] * f), to_f8x4(y[0] * f, y[1] * f, y[2] * f, y[3] * f)};
                        if (i0 + k * N < pieces) *as_global(piece(i0 + k * N)) = w[k];
                    }
                }
            } else if (off > 0) {
                byte = min(before, kAp8HighByte);
            }
            if (SHARED ? tid == 0 : lane == 0) *as_global(scale) = (uint8_t)byte;
            inv = one_over_scale(byte);
        }
    }
}

hipError_t launch_serving_append_codes(const ServingDev &S, const etc_serving_append_codes_io &io, hipStream_t s)
{
    const int n = io.append.n_tokens;
    int rows = 1;                                        // that a workgroup looks for runs in
    while (rows < kAp8Rows && rows * S.n_cus < n) rows *= 2;
    int q_tokens = kAp8Heads * kAp8Threads / (S.nq * (S.d / 16));
    if (q_tokens < 1) q_tokens = 1;
    if (q_tokens > kAp8Rows) q_tokens = kAp8Rows;
    const bool f32 = io.append.dtype == ETC_FP32, shared = (1 << S.page_shift) > 2 * kAp8Rows;
    const int kv_wgs = 2 * (shared ? S.nkv : (S.nkv + kAp8Waves - 1) / kAp8Waves), kv_blocks = (n + rows - 1) / rows * kv_wgs;
    const int wgs = kv_blocks + (n + q_tokens - 1) / q_tokens;      // at most 2^16 * 2048 + 2^20
    const dim3 grid((unsigned)(wgs < kAp8GridX ? wgs : kAp8GridX), (unsigned)((wgs + kAp8GridX - 1) / kAp8GridX)), block(kAp8Threads);
    auto launch = [&](auto d, auto is_f32, auto is_shared) {
        hipLaunchKernelGGL((serving_append_codes_kernel<decltype(d)::value, decltype(is_f32)::value, decltype(is_shared)::value>), grid, block, 0, s, S, io, rows, kv_wgs, kv_blocks, q_tokens);
    };
    auto of_type = [&](auto d, auto is_f32) { shared ? launch(d, is_f32, std::true_type()) : launch(d, is_f32, std::false_type()); };
    auto of_heads = [&](auto d) { f32 ? of_type(d, std::true_type()) : of_type(d, std::false_type()); };
    S.d == 128 ? of_heads(std::integral_constant<int, 128>()) : of_heads(std::integral_constant<int, 64>());
    return hipGetLastError();
}

}  // namespace etc
#endif  // ETC_GENERIC_ONLY
