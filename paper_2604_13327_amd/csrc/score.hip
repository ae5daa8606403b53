// Log-probabilities of given tokens, entropy and likeliest tokens of rows of logits (include/etc.h, etc_serving_score).
//
// One pass over a row.  A thread keeps a reference r, l = sum 2^y and t = sum 2^y y of its logits, y = (x - r) / ln 2; the reference follows
// the largest logit only when that has grown by kScoreLag, so that almost no sum is scaled again.  Then ln sum exp x = r + ln l, and the
// entropy is ln l - t ln 2 / l.  The likeliest tokens are found on the way, wavefront by wavefront: a list in LDS takes what is above a
// threshold, and is cut to its first n_top, the last of which is the new threshold, where it is full.  The first threshold is the n_top-th
// largest of the 64 lanes' first maxima.  Everything but the sums is a comparison, so nothing depends on how rows are cut.
// Few rows are cut into slices; the workgroup that arrives last at a row joins them.
#ifndef ETC_GENERIC_ONLY
#include "serving_rt.hip.h"

namespace etc {

constexpr int kScoreThreads = 256, kScoreWaves = kScoreThreads / 64;
constexpr int kScoreLoads = 4;              // of 16 bytes, of a thread, at once
constexpr int kScoreList = 128;             // entries of a wavefront: kScoreTop and one from every lane
constexpr int kScoreAll = 2048;             // entries of a row's slices together
constexpr float kScoreLag = 6.f;
constexpr float kScoreHuge = 1e38f;         // references from here on leave no room for their multiple by 1 / ln 2
constexpr float kLog2E = 1.44269504088896f;
constexpr double kPerLog2E = 1.0 / (double)kLog2E;      // of that very number: what it is off by scales all logits, not their differences
constexpr int kScoreRows = 2 * kSampleSharedRows;       // rows that are cut: each has a counter
constexpr int kScoreMinSlice = 4096;
static_assert(kScoreTop <= 64 && kScoreList >= kScoreTop + 64 && kScoreAll >= kScoreWaves * kScoreTop, "lists");

struct ScorePart { float ref, sum, moment; int count; uint64_t top[kScoreTop]; };      // of a slice; top sorted

__device__ __forceinline__ uint32_t score_key(float x)       // larger for the larger logit; x is not -0
{
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float score_logit(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

// Largest logit of a threshold's that is below all that it lets pass.
__device__ __forceinline__ float below(uint64_t threshold)
{
    uint32_t k = (uint32_t)(threshold >> 32);
    if (k <= 0x007FFFFFu) return -INFINITY;
    k -= k == 0x80000000u ? 2 : 1;                       // of 0: not -0
    return score_logit(k);
}

template <bool F32> struct Vec {
    static constexpr int E = F32 ? 4 : 8;
    static __device__ __forceinline__ float at(u32x4 w, int e) { return F32 ? __uint_as_float(w[e & 3]) : (e & 1) ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]); }
};
constexpr uint32_t kAllNan = 0xFFFFFFFFu;                    // as a fp32 or as two bf16

struct TopList {
    ETC_AS_LDS uint64_t *list;                           // [kScoreList] of this wavefront
    int top, count;                                      // the same for the wavefront
    uint64_t threshold;                                  // entries above it are taken
    float under;

    __device__ __forceinline__ void cut()                // to the first `top`, sorted
    {
        const int lane = lane_id();
        in_order();
        const uint64_t a = lane < count ? list[lane] : 0, b = lane + 64 < count ? list[lane + 64] : 0;
        int ra = 0, rb = 0;
        for (int j = 0; j < count; ++j) {
            const uint64_t e = list[j];
            ra += e > a;
            rb += e > b;
        }
        in_order();
        if (lane < count && ra < top) list[ra] = a;
        if (lane + 64 < count && rb < top) list[rb] = b;
        in_order();
        count = min(count, top);
    }
    __device__ __forceinline__ void raise()
    {
        if (count < top) return;
        const uint64_t last = list[top - 1];
        threshold = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(last >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)last);
        under = below(threshold);
    }
    // Of the first maxima, one from each lane: at least `top` logits are no smaller than the threshold's.
    __device__ __forceinline__ void begin(float most)
    {
        list[lane_id()] = (uint64_t)score_key(most > -INFINITY ? most + 0.f : -INFINITY) << 32 | (uint32_t)lane_id();
        count = 64;
        cut();
        raise();
        threshold &= 0xFFFFFFFF00000000ull;
        under = below(threshold);
        count = 0;
    }
    template <bool F32> __device__ __forceinline__ void take(u32x4 w, int id)
    {
#pragma unroll
        for (int e = 0; e < Vec<F32>::E; ++e) {
            const float x = Vec<F32>::at(w, e);
            const uint64_t entry = (uint64_t)score_key(x + 0.f) << 32 | (uint32_t)~(id + e);
            uint64_t takes = __builtin_amdgcn_ballot_w64(x > under && entry > threshold);
            if (takes == 0) continue;
            if (count + __builtin_popcountll(takes) > kScoreList) {
                cut();
                raise();
                takes = __builtin_amdgcn_ballot_w64(x > under && entry > threshold);
            }
            if ((takes >> lane_id()) & 1) list[count + __builtin_popcountll(takes & ((1ull << lane_id()) - 1))] = entry;
            in_order();
            count += __builtin_popcountll(takes);
        }
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

__device__ __forceinline__ double exp2_between(float ref, float most)      // factor of sums from ref where they are to count from most
{
    if (fabsf(most) >= kScoreHuge) return ref == most ? 1.0 : 0.0;      // numbers of this size differ by far more than exp can tell, or not at all
    return exp2((double)log2_between(ref, most));
}

// Sum, over n parts of ref, l, t, by all threads of a wavefront alike.
struct Total { float ref; double l, t; };
template <class At>
__device__ __forceinline__ Total total_of(int n, At at)
{
    Total T{-INFINITY, 0.0, 0.0};
    for (int i = 0; i < n; ++i) T.ref = fmaxf(T.ref, at(i).ref);
    if (T.ref == -INFINITY) return T;
    for (int i = 0; i < n; ++i) {
        const Sums s = at(i);
        if (s.ref == -INFINITY) continue;
        const double f = exp2_between(s.ref, T.ref);
        T.l += f * s.l;
        if (fabsf(T.ref) < kScoreHuge) T.t += f * ((double)s.t + (double)s.l * (double)log2_between(s.ref, T.ref));
    }
    return T;
}

template <bool F32>
__global__ __launch_bounds__(kScoreThreads) void serving_score_kernel(ServingDev S, etc_serving_score_io io, int slices, int per_slice)
{
    constexpr int E = Vec<F32>::E, SIZE = F32 ? 4 : 2, U = kScoreLoads;
    __shared__ uint64_t s_list[kScoreAll];
    __shared__ Sums s_sums[kScoreAll / 16];
    __shared__ int s_count[kScoreAll / 16];
    __shared__ int s_last;
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

    TopList list{as_lds(s_list) + wave * kScoreList, top, 0, 0, -INFINITY};
    Sums s{-INFINITY, 0.f, 0.f};
    float from_ref = INFINITY;                           // -in_log2(s.ref)
    bool first = true;
    auto feed = [&](const u32x4 (&w)[U], int id) {       // vector u: tokens id + u * kScoreThreads * E ..; out of range: NaN
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
                // NaN and -inf: 0; against a reference of the type's lowest values, which is -inf in powers of two: a number, of no weight in the end
                const float y = __builtin_amdgcn_fmed3f(__builtin_fmaf(Vec<F32>::at(w[u], e), kLog2E, from_ref), -160.f, 64.f), p = __builtin_amdgcn_exp2f(y);
                l += p;
                t = __builtin_fmaf(p, y, t);
            }
        s.l += l;
        s.t += t;
        if (top == 0) return;
        if (first) list.begin(all);
        first = false;
        if (__builtin_amdgcn_ballot_w64(all > list.under) == 0) return;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (__builtin_amdgcn_ballot_w64(most[u] > list.under) != 0) list.take<F32>(w[u], id + u * kScoreThreads * E);
    };
    u32x4 w[U], behind[U];
    auto load = [&](u32x4 (&to)[U], int v0) {
        if (v0 >= nv) return;                            // the same for the workgroup
#pragma unroll
        for (int u = 0; u < U; ++u) to[u] = gld_16B(body + (int64_t)min(v0 + u * kScoreThreads + tid, nv - 1) * 16);
    };
    load(w, 0);
    for (int v0 = 0; v0 < nv; v0 += kScoreThreads * U) {
        load(behind, v0 + kScoreThreads * U);
        if (v0 + kScoreThreads * U > nv) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v0 + u * kScoreThreads + tid >= nv) w[u] = u32x4{kAllNan, kAllNan, kAllNan, kAllNan};
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

    // ---- the workgroup's: sums by thread 0 .. in the order of the threads, lists by rank
    auto reduce = [&](Sums v) {                          // of a wavefront, in every lane; the order is that of the lanes' distances
        float ref = v.ref;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) ref = fmaxf(ref, __shfl_xor(ref, o, 64));
        double l = 0.0, t = 0.0;
        if (v.ref > -INFINITY) {
            const double f = exp2_between(v.ref, ref);
            l = f * v.l;
            if (fabsf(ref) < kScoreHuge) t = f * ((double)v.t + (double)v.l * (double)log2_between(v.ref, ref));
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) { l += __shfl_xor(l, o, 64); t += __shfl_xor(t, o, 64); }
        return Sums{ref, (float)l, (float)t};
    };
    const Sums mine = reduce(s);
    if (lane == 0) s_sums[wave] = mine;
    if (top > 0) list.cut();
    if (lane == 0) s_count[wave] = list.count;
    __syncthreads();
    Total T = total_of(kScoreWaves, [&](int i) { return s_sums[i]; });
    if (T.ref != -INFINITY && fabsf(T.ref) >= kScoreHuge) {      // how many there are of the largest: nothing else has weight
        int n = 0;
        for (int i = i0 + tid; i < i1; i += kScoreThreads)
            n += (F32 ? *as_global((const float *)logits + i) : bf16_bits_to_f32(gld_u16((const uint16_t *)logits + i))) == T.ref;
        n = wave_sum_i(n);
        __syncthreads();
        if (lane == 0) s_sums[wave].l = (float)n;
        __syncthreads();
        T.l = T.t = 0.0;
        for (int i = 0; i < kScoreWaves; ++i) T.l += (double)s_sums[i].l;
    }
    // entry i of n lists of up to `stride` entries each: how many are in front of it in all
    auto rank_of = [&](uint64_t entry, int lists, int stride) {
        int r = 0;
        for (int k = 0; k < lists; ++k) {
            const int n = s_count[k];
            for (int j = 0; j < n; ++j) r += s_list[k * stride + j] > entry;
        }
        return r;
    };
    int n_top = 0;
    for (int i = 0; i < kScoreWaves; ++i) n_top += s_count[i];
    n_top = min(n_top, top);
    uint64_t entry = 0;
    int rank = kScoreTop;
    if (top > 0 && lane < s_count[wave]) {
        entry = list.list[lane];
        rank = rank_of(entry, kScoreWaves, kScoreList);
    }
    auto finish = [&](const Total &T) {                  // (by one thread)
        if (io.entropy_out) *as_global(io.entropy_out + row) = T.ref == -INFINITY ? 0.f : (float)fmax(log(T.l) - T.t / T.l * 0.6931471805599453, 0.0);
    };
    auto logprob = [&](float x, const Total &T) {        // of a logit
        if (!(x > -INFINITY)) return -INFINITY;
        if (fabsf(T.ref) >= kScoreHuge) return x == T.ref ? (float)-log(T.l) : (float)((double)x - (double)T.ref);
        return (float)((double)x - ((double)in_log2(T.ref) * kPerLog2E + log(T.l)));
    };
    auto write_row = [&](const Total &T) {
        if (tid == 0) finish(T);
        if (tid == 64 && io.logprob_out) {
            const float x = F32 ? *as_global((const float *)logits + token) : bf16_bits_to_f32(gld_u16((const uint16_t *)logits + token));
            *as_global(io.logprob_out + row) = T.ref == -INFINITY ? -INFINITY : logprob(x, T);
        }
    };
    auto write_top = [&](uint64_t e, int r, const Total &T) {
        const int64_t at = (int64_t)row * top + r;
        *as_global(io.top_ids + at) = (int)~(uint32_t)e;
        if (io.top_logprobs) *as_global(io.top_logprobs + at) = logprob(score_logit((uint32_t)(e >> 32)), T);
    };
    auto write_none = [&](int have) {
        for (int r = have + tid; r < top; r += kScoreThreads) {
            *as_global(io.top_ids + (int64_t)row * top + r) = -1;
            if (io.top_logprobs) *as_global(io.top_logprobs + (int64_t)row * top + r) = -INFINITY;
        }
    };
    if (slices == 1) {
        write_row(T);
        if (rank < top) write_top(entry, rank, T);
        write_none(n_top);
        return;
    }
    // ---- a slice's: to memory; the last to arrive joins the row's
    ScorePart *const parts = reinterpret_cast<ScorePart *>(S.smp_bins) + (size_t)row * slices;
    if (tid == 0) {
        st_f32(&parts[slice].ref, T.ref);
        st_f32(&parts[slice].sum, (float)T.l);
        st_f32(&parts[slice].moment, (float)T.t);
        st_i32(&parts[slice].count, n_top);
    }
    if (rank < top) __hip_atomic_store(as_global(&parts[slice].top[rank]), entry, __ATOMIC_RELAXED, ETC_SCOPE);
    wg_release();
    if (tid == 0) {
        int32_t *const arrived = S.smp_listed + row;
        s_last = __hip_atomic_fetch_add(as_global(arrived), 1, __ATOMIC_RELAXED, ETC_SCOPE) + 1 == slices;
        if (s_last) st_i32(arrived, 0);
    }
    __syncthreads();
    if (!s_last) return;
    for (int i = tid; i < slices; i += kScoreThreads) {
        s_sums[i] = Sums{ld_f32(&parts[i].ref), ld_f32(&parts[i].sum), ld_f32(&parts[i].moment)};
        s_count[i] = ld_i32(&parts[i].count);
    }
    __syncthreads();
    for (int i = tid; i < slices * top; i += kScoreThreads)
        if (i % top < s_count[i / top]) s_list[i] = ld_u64(&parts[i / top].top[i % top]);
    __syncthreads();
    T = total_of(slices, [&](int i) { return s_sums[i]; });
    write_row(T);
    int have = 0;
    for (int i = 0; i < slices; ++i) have += s_count[i];
    for (int i = tid; i < slices * top; i += kScoreThreads) {
        if (i % top >= s_count[i / top]) continue;
        const int r = rank_of(s_list[i], slices, top);
        if (r < top) write_top(s_list[i], r, T);
    }
    write_none(min(have, top));
}

hipError_t launch_serving_score(const ServingDev &S, const etc_serving_score_io &io, hipStream_t s)
{
    // Slices: where there is a workspace (long rows), enough for two workgroups on every compute unit.
    int slices = 1;
    if (S.smp_bins && io.n_rows <= kScoreRows) {
        slices = (2 * S.n_cus + io.n_rows - 1) / io.n_rows;
        const int most = (S.vocab + kScoreMinSlice - 1) / kScoreMinSlice, entries = kScoreAll / (io.n_top > 16 ? io.n_top : 16);
        if (slices > most) slices = most;
        if (slices > entries) slices = entries;
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
