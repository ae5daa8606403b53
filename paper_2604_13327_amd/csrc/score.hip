// Log-probabilities of given tokens, entropy and likeliest tokens of rows of logits (include/etc.h, etc_serving_score).
//
// One pass over a row.  A thread keeps a reference r, l = sum 2^y and t = sum 2^y y of its logits, y = (x - r) / ln 2; the reference follows
// the largest logit only when that has grown by kScoreLag, so that almost no sum is scaled again.  Then ln sum exp x = r + ln l, and the
// entropy is ln l - t ln 2 / l.  The likeliest tokens are found on the way, wavefront by wavefront: vectors with something above a
// threshold wait in LDS until there is one for every lane, what is above it in them goes to a list, and a full list is cut to its first n_top,
// which raises the threshold.  The first threshold is what the first maxima of n_top lanes reach.  What is found does not depend on how rows are cut.
// Few rows are cut into slices; the workgroup that arrives last at a row joins them.
// Bound by memory where rows are many: 4096 of 128256 in bf16 (1.05 GB) with 5 alternatives take 187 to 196 us, 5.5 TB/s.  301 such rows with 10 take 28
// (77 MB: 16 us at a copy's rate): two slices to a row, and behind them 8 us of lists, join and ranks that no load covers; without alternatives 21.
// 16 rows in fp32 with 20 take 9.8 to 10.2, one row of 1024 with 5 7.0, of which a launch is 2.  With lists that take elements one by one, and are
// cut by ranks, 131 us for those 16 rows, 59 for the 301.
#ifndef ETC_GENERIC_ONLY
#include <type_traits>

#include "serving_rt.hip.h"

namespace etc {

constexpr int kScoreWaves = 4, kScoreThreads = kScoreWaves * 64;
constexpr int kScoreLoads = 4;              // of 16 bytes, of a thread, at once
constexpr int kScoreList = 128;             // entries of a wavefront: kScoreTop and one from every lane
constexpr int kScoreSlices = 32;            // of a row, at most
constexpr int kIdBits = 20;
static_assert(kServingMaxVocab <= 1 << kIdBits, "ids");
constexpr float kScoreLag = 6.f;            // weights up to e^6 lose nothing
// References from 2^30 on (of either sign): neighbours of theirs differ by 64 at least, so that only the logits equal to the largest have weight, and
// are counted.  In front of that a multiple by 1 / ln 2 is rounded by 64 at most, as far as exponents go.
constexpr float kScoreHuge = 0x1p30f;
constexpr float kLog2E = 1.44269504088896f;
constexpr double kPerLog2E = 1.0 / (double)kLog2E;      // of that very number: what it is off by scales all logits, not their differences
constexpr int kScoreMinSlice = 4096;        // tokens (one row of 32000 in bf16: 8.8 us, 8.8 with 2048, 9.3 with 8192, 9.8 with 16384)
static_assert(kScoreTop <= 64 && kScoreList >= kScoreTop + 64, "lists");

// An entry of a list: larger for the larger logit (not -0), then for the lower id; never 0.
__device__ __forceinline__ uint32_t score_key(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float score_logit(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ __forceinline__ uint64_t score_entry(float x, int id) { return (uint64_t)score_key(x + 0.f) << 32 | (uint32_t)~id; }

// A logit that is below all that a threshold lets pass, and not below others.
__device__ __forceinline__ float below(uint64_t threshold)
{
    uint32_t k = (uint32_t)(threshold >> 32);
    if (k <= 0x007FFFFFu) return -INFINITY;
    k -= k == 0x80000000u ? 2 : 1;                       // of 0: not -0
    return score_logit(k);
}

__device__ __forceinline__ uint32_t wave_max_u(uint32_t v)
{
    auto with = [&](int w) { v = max(v, (uint32_t)w); };
    with(dpp_i32<0xB1>((int)v));
    with(dpp_i32<0x4E>((int)v));
    with(dpp_i32<0x141>((int)v));
    with(dpp_i32<0x140>((int)v));
    auto row = [&](int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); };
    return max(max(row(0), row(16)), max(row(32), row(48)));
}

// A number that the `top` largest of a wavefront's entries, N to a lane, reach, and no more than 64 do (0 where there are no more): bit by
// bit, by counting, the logit's bits first.
template <int N>
__device__ __forceinline__ uint64_t threshold_of(const uint64_t (&x)[N], int top)
{
    auto reach = [&](auto at_least) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(at_least(x[i])));
        return n;
    };
    if (reach([](uint64_t e) { return e != 0; }) <= 64) return 0;
    uint32_t most = 0, least = 0xFFFFFFFFu;              // of the logits' bits: those that they have in common are the threshold's
#pragma unroll
    for (int i = 0; i < N; ++i) {
        most = max(most, (uint32_t)(x[i] >> 32));
        least = min(least, x[i] != 0 ? (uint32_t)(x[i] >> 32) : 0xFFFFFFFFu);
    }
    most = wave_max_u(most);
    least = ~wave_max_u(~least);
    uint32_t hi = most;
    if (most != least) {
        int b = 31 - __builtin_clz(most ^ least);
        hi = most >> b >> 1 << b << 1;
        for (; b >= 0; --b) {
            const uint32_t c = hi | 1u << b;
            const int n = reach([&](uint64_t e) { return (uint32_t)(e >> 32) >= c; });
            if (n < top) continue;
            hi = c;
            if (n <= 64) return (uint64_t)hi << 32;
        }
    }
    uint64_t t = (uint64_t)hi << 32 | 0xFFFFFFFFu << kIdBits;      // of equal logits the lower ids
    for (int b = kIdBits - 1; b >= 0; --b) {
        const uint64_t c = t | 1u << b;
        const int n = reach([&](uint64_t e) { return e >= c; });
        if (n < top) continue;
        t = c;
        if (n <= 64) break;
    }
    return t;
}
// Those that reach a threshold, in turn to put(i, entry): how many.
template <int N, class Put>
__device__ __forceinline__ int keep(const uint64_t (&x)[N], uint64_t threshold, Put put)
{
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool stays = x[i] != 0 && x[i] >= threshold;
        const uint64_t mask = __builtin_amdgcn_ballot_w64(stays);
        if (stays) put(n + __builtin_popcountll(mask & ((1ull << lane_id()) - 1)), x[i]);
        n += __builtin_popcountll(mask);
    }
    return n;
}

template <bool F32> struct Vec {
    static constexpr int E = F32 ? 4 : 8;
    static __device__ __forceinline__ float at(u32x4 w, int e) { return F32 ? __uint_as_float(w[e & 3]) : (e & 1) ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]); }
};
constexpr uint32_t kAllNan = 0xFFFFFFFFu;                    // as a fp32 or as two bf16

struct Pending { u32x4 w[kScoreList]; int id[kScoreList]; };      // vectors with something in them, and their first token

struct TopList {
    ETC_AS_LDS uint64_t *list;                           // [kScoreList] of this wavefront
    ETC_AS_LDS Pending *pending;
    int top, count, n_pending;                           // the same for the wavefront
    uint64_t threshold;                                  // entries from it on are taken
    float under;

    __device__ __forceinline__ void set(uint64_t t)
    {
        threshold = t;
        under = below(t);
    }
    __device__ __forceinline__ void cut()                // to 64 at most, the first `top` among them
    {
        const int lane = lane_id();
        in_order();
        const uint64_t x[2] = {lane < count ? list[lane] : 0, lane + 64 < count ? list[lane + 64] : 0};
        in_order();
        const uint64_t t = threshold_of<2>(x, top);
        if (t == 0) return;
        count = keep<2>(x, t, [&](int i, uint64_t e) { list[i] = e; });
        in_order();
        set(t);
    }
    // What at least `n` lanes' maxima reach.  Sixteen bits of it do.
    static __device__ __forceinline__ uint64_t reached(float most, int n)
    {
        const uint32_t key = score_key(most > -INFINITY ? most + 0.f : -INFINITY) >> 16;
        uint32_t t = 0;
        for (int b = 15; b >= 0; --b)
            if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= (t | 1u << b))) >= n) t |= 1u << b;
        return (uint64_t)t << 48;
    }
    // The vectors that wait, a vector to a lane.
    template <bool F32> __device__ __forceinline__ void settle()
    {
        in_order();
        for (int at = 0; at < n_pending; at += 64) {
            const bool mine = at + lane_id() < n_pending;
            const u32x4 w = pending->w[mine ? at + lane_id() : at];
            const int id = pending->id[mine ? at + lane_id() : at];
#pragma unroll
            for (int e = 0; e < Vec<F32>::E; ++e) {
                const float x = Vec<F32>::at(w, e);
                const uint64_t entry = score_entry(x, id + e);
                uint64_t takes = __builtin_amdgcn_ballot_w64(mine && x > under && entry >= threshold);
                if (takes == 0) continue;
                if (count + __builtin_popcountll(takes) > kScoreList) {
                    cut();
                    takes = __builtin_amdgcn_ballot_w64(mine && x > under && entry >= threshold);
                }
                if ((takes >> lane_id()) & 1) list[count + __builtin_popcountll(takes & ((1ull << lane_id()) - 1))] = entry;
                count += __builtin_popcountll(takes);
            }
        }
        n_pending = 0;
        in_order();
    }
    template <bool F32> __device__ __forceinline__ void take(u32x4 w, float most, int id)
    {
        const uint64_t takes = __builtin_amdgcn_ballot_w64(most > under);
        if (takes == 0) return;
        if ((takes >> lane_id()) & 1) {
            const int at = n_pending + __builtin_popcountll(takes & ((1ull << lane_id()) - 1));
            pending->w[at] = w;
            pending->id[at] = id;
        }
        n_pending += __builtin_popcountll(takes);
        if (n_pending >= 64) settle<F32>();
    }
};

struct Sums { float ref, l, t; };           // ref in logits; l and t count from in_log2(ref)
__device__ __forceinline__ float in_log2(float ref)          // rounded, wherever it stands: no part of a multiply-add
{
#pragma clang fp contract(off)
    return ref * kLog2E;
}
// By how many powers of two sums from `ref` are smaller when they count from `most`, as -300 .. 0.
__device__ __forceinline__ float log2_between(float ref, float most) { return fmaxf(in_log2(ref) - in_log2(most), -300.f); }

// Of a wavefront's sums one.
__device__ __forceinline__ Sums wave_total(Sums s)
{
    const float ref = wave_max_f(s.ref);
    float l = 0.f, t = 0.f;
    if (s.ref == ref) {
        l = s.l;
        t = s.t;
    } else if (fabsf(s.ref) < kScoreHuge && fabsf(ref) < kScoreHuge) {      // (others differ by more than an exponential can tell; -inf too)
        const float by = log2_between(s.ref, ref), f = __builtin_amdgcn_exp2f(by);
        l = f * s.l;
        t = f * __builtin_fmaf(s.l, by, s.t);
    }
    return Sums{ref, wave_sum(l), wave_sum(t)};
}

// What a slice leaves: its sums and its largest logit, and the entries it found, 64 (0: none).
__device__ __forceinline__ float *slice_sums(const ServingDev &S, int64_t slice) { return reinterpret_cast<float *>(S.smp_bins) + slice * 4; }
__device__ __forceinline__ uint64_t *slice_entries(const ServingDev &S, int64_t slice) { return S.smp_bins + (size_t)kScoreParts * 2 + slice * 64; }

template <bool F32>
__global__ __launch_bounds__(kScoreThreads) void serving_score_kernel(ServingDev S, etc_serving_score_io io, int slices, int per_slice)
{
    constexpr int E = Vec<F32>::E, SIZE = F32 ? 4 : 2, U = kScoreLoads, WAVES = kScoreWaves, THREADS = kScoreThreads;
    __shared__ uint64_t s_list[WAVES * kScoreList], s_found[64], s_begin[WAVES];
    __shared__ Pending s_pending[WAVES];
    __shared__ Sums s_sums[WAVES];
    __shared__ int s_count[WAVES], s_last;
    const int tid = (int)threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id());
    const int row = (int)blockIdx.x / slices, slice = (int)blockIdx.x - row * slices, top = io.n_top;
    int token = 0;
    if (io.tokens) {
        token = __builtin_amdgcn_readfirstlane(gld_i32(io.tokens + row));
        if (token < 0) return;                           // for all slices of the row
        if (token >= S.vocab) {
            if (slice == 0 && tid == 0) refuse(S.error, SRV_BAD_TOKEN, SRV_SCORE, row, token);
            return;
        }
    }
    const char *const logits = (const char *)io.logits + (int64_t)row * io.row_stride * SIZE;
    const int i0 = slice * per_slice, i1 = min(i0 + per_slice, S.vocab);
    const char *const from = logits + (int64_t)i0 * SIZE;
    const int a0 = min(i1, i0 + (int)((16 - ((uintptr_t)from & 15)) & 15) / SIZE), nv = (i1 - a0) / E, t0 = a0 + nv * E;
    const char *const body = logits + (int64_t)a0 * SIZE;

    TopList list{as_lds(s_list) + wave * kScoreList, as_lds(s_pending) + wave, top, 0, 0, 0, -INFINITY};
    Sums s{-INFINITY, 0.f, 0.f};
    float from_ref = INFINITY;                           // -in_log2(s.ref)
    float best = -INFINITY;                              // of what this lane has read
    int fed = 0;
    const bool short_row = nv < THREADS;
    auto feed = [&](const u32x4 (&w)[U], int id) {       // vector u: tokens id + u * THREADS * E ..; out of range: NaN
        float most[U], all = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            most[u] = Vec<F32>::at(w[u], 0);
#pragma unroll
            for (int e = 1; e < E; ++e) most[u] = fmaxf(most[u], Vec<F32>::at(w[u], e));
            all = fmaxf(all, most[u]);
        }
        if (__builtin_amdgcn_ballot_w64(all > s.ref + kScoreLag) != 0) {
            if (all > s.ref + kScoreLag) {
                const float by = log2_between(s.ref, all), f = __builtin_amdgcn_exp2f(by);
                s.t = f * (s.t + s.l * by);
                s.l *= f;
                s.ref = all;
                from_ref = -in_log2(all);
            }
        }
        float l = 0.f, t = 0.f;                          // sums of their own: the row's have one addition of each
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                // NaN and -inf: 0; against huge references, some -inf or inf in powers of two: a number, which is not used
                const float y = __builtin_amdgcn_fmed3f(__builtin_fmaf(Vec<F32>::at(w[u], e), kLog2E, from_ref), -160.f, 64.f), p = __builtin_amdgcn_exp2f(y);
                l += p;
                t = __builtin_fmaf(p, y, t);
            }
        s.l += l;
        s.t += t;
        if (top == 0) return;
        // The wavefronts' lanes together: `top` of them reach the least of this (of a row that has no vector for each of them: one wavefront's do).  Found
        // again behind the second, fourth, eighth .. load: 512 rows of 128256 in bf16 with 5 alternatives, 35.8 us -> 32.3.  Another wavefront's number
        // may be an older or a newer one then, which hold as well, and its lower word is always 0.
        best = fmaxf(best, all);
        if (fed != 1 && (fed & (fed - 1)) == 0) {
            const uint64_t t = TopList::reached(best, short_row ? top : (top + WAVES - 1) / WAVES);
            if (lane == 0) s_begin[wave] = t;
            if (fed == 0) __syncthreads(); else in_order();
            uint64_t least = s_begin[0];
#pragma unroll
            for (int i = 1; i < WAVES; ++i) least = short_row ? max(least, s_begin[i]) : min(least, s_begin[i]);
            if (least > list.threshold) list.set(least);
        }
        ++fed;
        if (__builtin_amdgcn_ballot_w64(all > list.under) == 0) return;
#pragma unroll
        for (int u = 0; u < U; ++u) list.take<F32>(w[u], most[u], id + u * THREADS * E);
    };
    u32x4 w[U], behind[U];
    auto load = [&](u32x4 (&to)[U], int v0) {
        if (v0 >= nv) return;                            // the same for the workgroup
#pragma unroll
        for (int u = 0; u < U; ++u) to[u] = gld_16B(body + (int64_t)min(v0 + u * THREADS + tid, nv - 1) * 16);
    };
    load(w, 0);
    for (int v0 = 0; v0 < nv; v0 += THREADS * U) {
        load(behind, v0 + THREADS * U);
        if (v0 + THREADS * U > nv) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v0 + u * THREADS + tid >= nv) w[u] = u32x4{kAllNan, kAllNan, kAllNan, kAllNan};
        }
        feed(w, a0 + (v0 + tid) * E);
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = behind[u];
    }
    if (a0 > i0 || t0 < i1) {                            // in front of what is aligned, and behind it: less than a vector each
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = u32x4{kAllNan, kAllNan, kAllNan, kAllNan};
        const int id = tid < E ? i0 + tid : t0 + tid - E;
        if (tid < E ? id < a0 : tid < 2 * E && id < i1)
            w[0][0] = F32 ? *as_global((const uint32_t *)(logits + (int64_t)id * SIZE)) : gld_u16((const uint16_t *)(logits + (int64_t)id * SIZE)) | 0xFFFF0000u;
        feed(w, id);
    }

    // ---- the workgroup's: by one wavefront
    const Sums mine = wave_total(s);
    if (top > 0) {
        list.settle<F32>();
        if (list.count > 64) list.cut();
    }
    if (lane == 0) {
        s_sums[wave] = mine;
        s_count[wave] = list.count;
    }
    __syncthreads();
    Sums T = wave_total(lane < WAVES ? s_sums[lane] : Sums{-INFINITY, 0.f, 0.f});
    if (T.ref != -INFINITY && fabsf(T.ref) >= kScoreHuge) {      // how many there are of the largest: nothing else has weight
        int n = 0;
        for (int i = i0 + tid; i < i1; i += THREADS)
            n += (F32 ? *as_global((const float *)logits + i) : bf16_bits_to_f32(gld_u16((const uint16_t *)logits + i))) == T.ref;
        n = wave_sum_i(n);
        __syncthreads();
        if (lane == 0) s_sums[wave].l = (float)n;
        __syncthreads();
        T.l = wave_sum(lane < WAVES ? s_sums[lane].l : 0.f);
        T.t = 0.f;
    }
    // The first `top` of the wavefronts' lists, and others up to 64.
    auto select = [&](auto put) {
        uint64_t x[WAVES];
#pragma unroll
        for (int i = 0; i < WAVES; ++i) x[i] = lane < s_count[i] ? s_list[i * kScoreList + lane] : 0;
        return keep<WAVES>(x, threshold_of<WAVES>(x, top), put);
    };
    if (slices > 1) {                                    // to memory; the last to arrive joins the row's
        const int64_t at = (int64_t)row * slices + slice;
        if (wave == 0) {
            float *const to = slice_sums(S, at);
            float largest = -INFINITY;
            if (top > 0) {
                uint64_t *const entries = slice_entries(S, at);
                uint32_t key = 0;
                const int n = select([&](int i, uint64_t e) { st_u64(entries + i, e); key = max(key, (uint32_t)(e >> 32)); });
                if (lane >= n) st_u64(entries + lane, 0);
                if (n > 0) largest = score_logit(wave_max_u(key));
            }
            if (lane < 4) st_f32(to + lane, lane == 0 ? T.ref : lane == 1 ? T.l : lane == 2 ? T.t : largest);
        }
        wg_release();
        if (tid == 0) {
            int32_t *const arrived = S.score_arrived + row * kScoreApart;
            s_last = __hip_atomic_fetch_add(as_global(arrived), 1, __ATOMIC_RELAXED, ETC_SCOPE) + 1 == slices;
            if (s_last) st_i32(arrived, 0);
        }
        __syncthreads();
        if (!s_last) return;
        Sums part{-INFINITY, 0.f, 0.f};
        float largest = -INFINITY;
        if (lane < slices) {
            const float *const from = slice_sums(S, (int64_t)row * slices + lane);
            part = Sums{ld_f32(from), ld_f32(from + 1), ld_f32(from + 2)};
            largest = ld_f32(from + 3);
        }
        if (top > 0) {                                   // a wavefront every fourth slice
            constexpr int N = kScoreSlices / WAVES;
            const uint64_t *const from = slice_entries(S, (int64_t)row * slices);
            uint64_t x[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int k = i * WAVES + wave;
                x[i] = k < slices ? ld_u64(from + k * 64 + lane) : 0;
            }
            uint64_t t = slices >= top ? TopList::reached(largest, top) : 0;      // `top` slices' largest do
            int n = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) n += __builtin_popcountll(__builtin_amdgcn_ballot_w64(x[i] != 0 && x[i] >= t));
            if (n > 64) t = threshold_of<N>(x, top);
            n = keep<N>(x, t, [&](int i, uint64_t e) { list.list[i] = e; });
            if (lane == 0) s_count[wave] = n;
        }
        T = wave_total(part);
        __syncthreads();
    }
    // ---- the row's outputs
    const double log_l = T.ref == -INFINITY ? 0.0 : log((double)T.l);
    auto logprob = [&](float x) {                        // of a logit; never positive, whatever l was rounded by
        if (!(x > -INFINITY) || T.ref == -INFINITY) return -INFINITY;
        if (fabsf(T.ref) >= kScoreHuge) return (float)((x == T.ref ? 0.0 : (double)x - (double)T.ref) - log_l);
        return (float)fmin((double)x - ((double)in_log2(T.ref) * kPerLog2E + log_l), 0.0);
    };
    if (wave == WAVES - 1 && lane == 0) {
        if (io.entropy_out) *as_global(io.entropy_out + row) = T.ref == -INFINITY ? 0.f : (float)fmax(log_l - (double)(T.t / T.l) * 0.6931471805599453, 0.0);
        if (io.logprob_out)
            *as_global(io.logprob_out + row) = logprob(F32 ? *as_global((const float *)logits + token) : bf16_bits_to_f32(gld_u16((const uint16_t *)logits + token)));
    }
    if (wave != 0 || top == 0) return;
    in_order();
    ETC_AS_LDS uint64_t *const found = as_lds(s_found);
    const int n = select([&](int i, uint64_t e) { found[i] = e; });
    in_order();
    const uint64_t entry = lane < n ? found[lane] : 0;
    int rank = 0;
    for (int i0 = 0; i0 < n; i0 += 8)
#pragma unroll
        for (int i = i0; i < i0 + 8; ++i) {              // (those behind the last are 0)
            const uint64_t e = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(entry >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)entry, i);
            rank += e > entry;
        }
    if (lane >= n) rank = lane;
    if (rank >= top) return;
    const int64_t at = (int64_t)row * top + rank;
    *as_global(io.top_ids + at) = lane < n ? (int)~(uint32_t)entry : -1;
    if (io.top_logprobs) *as_global(io.top_logprobs + at) = lane < n ? logprob(score_logit((uint32_t)(entry >> 32))) : -INFINITY;
}

hipError_t launch_serving_score(const ServingDev &S, const etc_serving_score_io &io, hipStream_t s)
{
    // Slices: where there is a workspace (long rows), enough for two workgroups on every compute unit: 64, 128 and 301 rows of 128256 in bf16 take 11.4, 16.8
    // and 27.7 us, with one 13.7, 18.9, 30.3, with three 12.5, 15.9, 28.4.
    int slices = 1;
    if (S.smp_bins && io.n_rows <= kScoreRows) {
        slices = (2 * S.n_cus + io.n_rows - 1) / io.n_rows;
        const int most = (S.vocab + kScoreMinSlice - 1) / kScoreMinSlice;
        if (slices > most) slices = most;
        if (slices > kScoreSlices) slices = kScoreSlices;
        if (slices > kScoreParts / io.n_rows) slices = kScoreParts / io.n_rows;
    }
    const int per_slice = ((S.vocab + slices - 1) / slices + 7) & ~7;
    slices = (S.vocab + per_slice - 1) / per_slice;
    const dim3 grid((unsigned)io.n_rows * (unsigned)slices), block(kScoreThreads);
    if (io.dtype == ETC_FP32) hipLaunchKernelGGL((serving_score_kernel<true>), grid, block, 0, s, S, io, slices, per_slice);
    else hipLaunchKernelGGL((serving_score_kernel<false>), grid, block, 0, s, S, io, slices, per_slice);
    return hipGetLastError();
}

}  // namespace etc
#endif  // ETC_GENERIC_ONLY
