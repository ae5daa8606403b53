// Serving operators beside the decode step (include/etc.h): page tables and slot maps, norm + RoPE + KV append, sampling.
#ifndef ETC_GENERIC_ONLY
#include "serving_rt.hip.h"

namespace etc {

// ---- page tables and slot maps --------------------------------------------------------------------------------------
// Prefix sums over the sequences (new tokens, pages, fresh pages), one sequence to a thread; then every page entry and
// every token row finds its sequence by a search in LDS.  A workgroup computes all sums itself (at most 1024 sequences), so
// that one launch is enough.  Inputs that outputs may alias (lengths, free count) are written by the workgroup that is the
// last to have read them.
// Measured: 3 sequences in 3.8 us, hardly more than an empty launch; 200 with 32397 new tokens in 6.5: a chain of loads, sums, searches.
constexpr int kTabThreads = 1024;

struct TabSums { int tokens, pages, fresh; };

__device__ __forceinline__ int seq_of(const int *indptr, int n, int x)      // the last b with indptr[b] <= x
{
    int lo = 0, hi = n;                                                     // indptr[lo] <= x < indptr[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (indptr[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kTabThreads) void serving_tables_kernel(ServingDev S, etc_serving_tables_io io)
{
    __shared__ int s_tok[kServingMaxSeqs + 1], s_page[kServingMaxSeqs + 1], s_fresh[kServingMaxSeqs + 1], s_kv[kServingMaxSeqs];
    __shared__ int s_wave[3][kTabThreads / 64];
    __shared__ int s_bad, s_last;
    const int tid = (int)threadIdx.x, wave = wave_id(), n = io.n_seqs;
    const int psh = S.page_shift, pmask = (1 << psh) - 1;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    const int count = gld_i32(io.free_count);
    int kv = 0, fresh_len = 0, has = 0, need = 0;
    bool bad = false;
    if (tid < n) {
        kv = gld_i32(io.kv_len + tid);
        fresh_len = gld_i32(io.new_len + tid);
        bad = kv < 0 || fresh_len < 0 || kv > S.max_kv_len || fresh_len > S.max_kv_len - kv || fresh_len > io.n_tokens;
        if (!bad) {
            has = (int)(((unsigned)kv + pmask) >> psh);
            need = (int)(((unsigned)(kv + fresh_len) + pmask) >> psh);
            bad = need > io.table_cols;
        }
        if (bad) { s_bad = 1; kv = fresh_len = has = need = 0; }
    }
    // each sum is at most 1024 * 2^20 tokens, 1024 * min(2^30, table) pages: pages are summed with a bound
    int tok = wave_scan_i(fresh_len);
    long long pages = need;                              // 1024 sequences of 2^30 pages do not fit 32 bits
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const long long t = __shfl_up(pages, o, 64);
        if (lane_id() >= o) pages += t;
    }
    const bool wide = pages > 0x3FFFFFFll;               // 16 wavefronts of this fit 32 bits
    if (wide) { s_bad = 1; pages = 0; }
    int pg = (int)pages;
    int fr = wave_scan_i(min(need - has, 1 << 20));      // fresh pages of a call: at most one a token and they are checked below
    if (lane_id() == 63) { s_wave[0][wave] = tok; s_wave[1][wave] = pg; s_wave[2][wave] = fr; }
    __syncthreads();
    for (int w = 0; w < wave; ++w) { tok += s_wave[0][w]; pg += s_wave[1][w]; fr += s_wave[2][w]; }
    if (tid < n) { s_tok[tid + 1] = tok; s_page[tid + 1] = pg; s_fresh[tid + 1] = fr; s_kv[tid] = kv; }
    if (tid == 0) s_tok[0] = s_page[0] = s_fresh[0] = 0;
    __syncthreads();
    const int n_tok = s_tok[n], n_page = s_page[n], n_fresh = s_fresh[n];
    int status = 0;
    if (s_bad || n_tok > io.n_tokens || (io.page_indptr && n_page > io.page_ids_cap) || count < 0 || count > io.free_cap) status = -1;
    else if (n_fresh > count) status = n_fresh - count;

    const int stride = (int)(gridDim.x * kTabThreads), first = (int)blockIdx.x * kTabThreads + tid;
    auto page_id = [&](int b, int p, int has_b) {        // page p of sequence b
        return p < has_b ? gld_i32(io.block_table + (size_t)b * io.table_stride + p) : gld_i32(io.free_pages + (count - 1 - (s_fresh[b] + p - has_b)));
    };
    auto pages_held = [&](int b) { return (int)(((unsigned)s_kv[b] + pmask) >> psh); };
    if (status == 0) {
        for (int e = first; e < n_fresh; e += stride) {  // fresh pages into the table
            const int b = seq_of(s_fresh, n, e);
            *as_global(io.block_table + (size_t)b * io.table_stride + pages_held(b) + (e - s_fresh[b])) = gld_i32(io.free_pages + (count - 1 - e));
        }
        if (io.page_ids)
            for (int e = first; e < n_page; e += stride) {
                const int b = seq_of(s_page, n, e);
                *as_global(io.page_ids + e) = page_id(b, e - s_page[b], pages_held(b));
            }
    }
    for (int t = first; t < io.n_tokens; t += stride) {
        int slot = -1, pos = 0;
        if (status == 0 && t < n_tok) {
            const int b = seq_of(s_tok, n, t);
            pos = s_kv[b] + (t - s_tok[b]);
            const int id = page_id(b, pos >> psh, pages_held(b));
            if ((unsigned)id <= (unsigned)(INT32_MAX >> psh)) {
                slot = (id << psh) + (pos & pmask);
            } else {                                     // its slots do not fit: one that lies in no pool
                refuse(S.error, SRV_BAD_PAGE, SRV_TABLES, b, id);
                slot = INT32_MAX;
            }
        }
        *as_global(io.slots + t) = slot;
        *as_global(io.positions + t) = pos;
    }
    if (blockIdx.x == 0) {
        for (int b = tid; b <= n; b += kTabThreads) {
            *as_global(io.q_indptr + b) = status == 0 ? s_tok[b] : 0;
            if (io.page_indptr) *as_global(io.page_indptr + b) = status == 0 ? s_page[b] : 0;
        }
        if (tid == 0) *as_global(io.status) = status;
    }
    // Outputs that may be inputs: behind everyone's reads of those (which the sums above have consumed).
    bool last = true;
    if (gridDim.x > 1) {
        __syncthreads();
        if (tid == 0) {
            s_last = __hip_atomic_fetch_add(as_global(S.arrive), 1, __ATOMIC_RELAXED, ETC_SCOPE) + 1 == (int)gridDim.x;
            if (s_last) st_i32(S.arrive, 0);
        }
        __syncthreads();
        last = s_last;
    }
    if (last) {
        if (io.total_len && tid < n) {
            if (status == 0) *as_global(io.total_len + tid) = s_kv[tid] + (s_tok[tid + 1] - s_tok[tid]);
            else if (io.total_len != io.kv_len) *as_global(io.total_len + tid) = gld_i32(io.kv_len + tid);
        }
        if (tid == 0) *as_global(io.free_count_out) = status == 0 ? count - n_fresh : count;
    }
}

hipError_t launch_serving_tables(const ServingDev &S, const etc_serving_tables_io &io, hipStream_t s)
{
    // Rows and, where asked for, page ids: some per thread, at most one workgroup per compute unit.
    const long long entries = (long long)io.n_tokens > io.page_ids_cap ? io.n_tokens : io.page_ids_cap;
    long long wgs = (entries + kTabThreads - 1) / kTabThreads;
    if (wgs < 1) wgs = 1;
    if (wgs > S.n_cus) wgs = S.n_cus;
    hipLaunchKernelGGL(serving_tables_kernel, dim3((unsigned)wgs), dim3(kTabThreads), 0, s, S, io);
    return hipGetLastError();
}

// ---- per-head norms, RoPE and KV append ------------------------------------------------------------------------------
// One pass: a thread has 8 elements of the first half of a head and the 8 they are rotated with, so that a head of D
// elements is D / 16 neighbouring lanes (its sum of squares: 2 or 3 lane exchanges).  Bound by memory: every row is read and written once.
// A workgroup takes enough tokens to have work for all threads; their (cos, sin) tables are computed once, in LDS.
// Measured: 8192 tokens of 64 + 2 * 8 heads of 128, bf16 with norms (336 MB): 59 us, 5.7 TB/s (a large copy: 4.8); 1000 tokens of 32 + 2 * 8
// heads, fp32 (37 MB): 6.3 us, 5.9 TB/s.
constexpr int kAppThreads = 256;
constexpr int kAppMaxTokens = 16;

template <int D, bool F32>
__global__ __launch_bounds__(kAppThreads) void serving_append_kernel(ServingDev S, etc_serving_append_io io, int tokens_per_wg)
{
    constexpr int LPH = D / 16, HALF = D / 2, RPP = kAppThreads / LPH;      // lanes per head, pairs, heads per pass
    __shared__ float s_cos[kAppMaxTokens][HALF], s_sin[kAppMaxTokens][HALF];
    const int tid = (int)threadIdx.x, t0 = (int)blockIdx.x * tokens_per_wg, nt = min(tokens_per_wg, io.n_tokens - t0);
    for (int i = tid; i < nt * HALF; i += kAppThreads) {
        const int t = i / HALF, e = i - t * HALF;
        // the angle in double, reduced to half a turn: positions run into the millions
        const double turns = (double)gld_i32(io.positions + t0 + t) * *as_global(S.inv_freq + e) * 0.15915494309189535;
        const float r = (float)(turns - rint(turns)) * 6.2831853071795862f;
        s_cos[t][e] = __cosf(r);
        s_sin[t][e] = __sinf(r);
    }
    __syncthreads();
    const int c = (tid % LPH) * 8, heads = S.nq + 2 * S.nkv;
    for (int r = tid / LPH; r < nt * heads; r += RPP) {
        const int t = r / heads, h = r - t * heads, row = t0 + t;
        const int slot = gld_i32(io.slots + row);
        if (slot < 0) continue;                          // the same for all lanes of a head
        if (slot >= (int)(io.n_pages << S.page_shift)) {
            if (c == 0) refuse(S.error, SRV_BAD_SLOT, SRV_APPEND, row, slot);
            continue;
        }
        const bool is_q = h < S.nq, is_v = h >= S.nq + S.nkv;
        const int hh = is_q ? h : is_v ? h - S.nq - S.nkv : h - S.nq;
        const int64_t at = (int64_t)row * (is_q ? io.q_stride : is_v ? io.v_stride : io.k_stride) + hh * D + c;
        const void *src = is_q ? io.q : is_v ? io.v : io.k;
        float a[8], b[8];
        if (F32) {
            const float *p = (const float *)src + at;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const f32x4 x = __builtin_bit_cast(f32x4, gld_16B(p + 4 * i)), y = __builtin_bit_cast(f32x4, gld_16B(p + HALF + 4 * i));
#pragma unroll
                for (int j = 0; j < 4; ++j) { a[4 * i + j] = x[j]; b[4 * i + j] = y[j]; }
            }
        } else {
            const uint16_t *p = (const uint16_t *)src + at;
            const u32x4 x = gld_16B(p), y = gld_16B(p + HALF);
#pragma unroll
            for (int i = 0; i < 4; ++i) { a[2 * i] = bf16_lo(x[i]); a[2 * i + 1] = bf16_hi(x[i]); b[2 * i] = bf16_lo(y[i]); b[2 * i + 1] = bf16_hi(y[i]); }
        }
        if (!is_v) {
            if (S.qk_norm) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) ss += a[i] * a[i] + b[i] * b[i];
                const float rn = 1.0f / sqrtf(head_sum<D>(ss) / (float)D + S.eps);
                const uint16_t *g = (const uint16_t *)(is_q ? io.gq : io.gk) + c;
                const u32x4 ga = gld_16B(g), gb = gld_16B(g + HALF);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[2 * i] *= rn * bf16_lo(ga[i]); a[2 * i + 1] *= rn * bf16_hi(ga[i]);
                    b[2 * i] *= rn * bf16_lo(gb[i]); b[2 * i + 1] *= rn * bf16_hi(gb[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float cs = s_cos[t][c + i], sn = s_sin[t][c + i], x = a[i], y = b[i];
                a[i] = x * cs - y * sn;
                b[i] = x * sn + y * cs;
            }
        }
        uint16_t *dst = is_q ? (uint16_t *)io.q_out + ((int64_t)row * S.nq + hh) * D + c
                             : (uint16_t *)(is_v ? io.v_pages : io.k_pages) + ((int64_t)slot * S.nkv + hh) * D + c;
        u32x4 x, y;
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = to_bf16x2(a[2 * i], a[2 * i + 1]); y[i] = to_bf16x2(b[2 * i], b[2 * i + 1]); }
        *as_global(reinterpret_cast<u32x4 *>(dst)) = x;
        *as_global(reinterpret_cast<u32x4 *>(dst + HALF)) = y;
    }
}

hipError_t launch_serving_append(const ServingDev &S, const etc_serving_append_io &io, hipStream_t s)
{
    const int per_token = (S.nq + 2 * S.nkv) * (S.d / 16);
    int tokens = kAppThreads / per_token;
    if (tokens < 1) tokens = 1;
    if (tokens > kAppMaxTokens) tokens = kAppMaxTokens;
    const dim3 grid((unsigned)((io.n_tokens + tokens - 1) / tokens)), block(kAppThreads);
    const bool f32 = io.dtype == ETC_FP32;
    if (S.d == 128) {
        if (f32) hipLaunchKernelGGL((serving_append_kernel<128, true>), grid, block, 0, s, S, io, tokens);
        else hipLaunchKernelGGL((serving_append_kernel<128, false>), grid, block, 0, s, S, io, tokens);
    } else {
        if (f32) hipLaunchKernelGGL((serving_append_kernel<64, true>), grid, block, 0, s, S, io, tokens);
        else hipLaunchKernelGGL((serving_append_kernel<64, false>), grid, block, 0, s, S, io, tokens);
    }
    return hipGetLastError();
}

// ---- sampling ----------------------------------------------------------------------------------------------------------
// Everything the filters and the draw ask for is a beginning of the tokens in the order (larger logit, lower id): the first k, the
// first that weigh so much.  A row is sorted into kSmpBins bins by its logits' distance from the largest, with the tokens and the
// weight of each bin; running sums over the bins say in which bin a beginning ends.  The tokens of the few bins in question go
// to a list in LDS, where the same is done once more within a bin, and the handful left is compared one by one.
// Weights are whole numbers of 2^-35 of the largest and summed as such: sums are exact, so no result depends on an order of additions.
// Long rows: sample_scan (largest and smallest logit) and sample_bins over slices of the rows, as many as fill the chip, then
// sample_row; short ones: sample_row does it all.  Rows with more tokens in the bins in question than the list holds and rows with +inf
// take slow_row, which descends through the bits of the logits' keys instead.  The former are flat, or have many ties in the wrong
// place, or a low temperature and a top_k whose last token lies behind all that have weight, in the last bin, with most of the row.
// Measured: one row of 1024 in 14 us (a quarter of it the first pass, over code that no cache holds yet), 16 rows of 128256 without
// filters in 30 us (scan 4, bins 8, row 18), 64 in bf16 with all of them in 50 (7, 14, 30).  By slow_row 64 in bf16 with a top_k of 50 at a
// temperature of 0.1 in 327 us (38 at 1); one of 1024, whose last bin fits the list and is compared one by one, in 101 (13 at 1).
// One compute unit looks through a row of 128256 at 30 bytes a cycle, half of sample_row's time: where there are units for it, several do
// (33 and 55 us with one to a row).
constexpr int kSmpThreads = 1024;           // of sample_row
constexpr int kSliceThreads = 512;
constexpr int kSmpBins = 1024;              // a bin: 1 / 1024 of min(32 temperatures, the row's range); a weight below 2^-36 is 0
constexpr int kSmpList = kSampleList;       // tokens
constexpr int kSmpFew = 1024;               // compared one by one
constexpr int kUnitBits = 35;
constexpr uint64_t kTopWeight = 1ull << kUnitBits;
constexpr int kCountShift = 49;
constexpr int kBinTokens = (1 << 14) - 1;   // tokens whose count and weight fit the 64 bits of a bin, 15 and 49, all of them the largest's
static_assert((uint64_t)kBinTokens * kTopWeight < 1ull << kCountShift && kSmpList <= kBinTokens, "a bin");
constexpr int kSmpWgs = 256;                // workgroups over slices
constexpr int kSmpWhole = kBinTokens;       // longest row that sample_row does alone

template <bool F32>
__device__ __forceinline__ float raw_logit(const void *row, int i)
{
    return F32 ? *as_global((const float *)row + i) : bf16_bits_to_f32(gld_u16((const uint16_t *)row + i));
}
template <bool F32>
__device__ __forceinline__ float logit_at(const void *row, int i)
{
    float x = raw_logit<F32>(row, i);
    x = x != x ? -INFINITY : x;                              // NaN: banned
    return x + 0.f;                                          // -0 is +0: equal logits
}
// The tokens [i0, i1) of a row, by the workgroup, a thread's ids ascending; NaN as it stands.  16 bytes a load and U loads in flight
// (one after the other a row of 128256 took 73 us instead of 14): vectors(w, n, id) gets U vectors of which n are of this row, the
// first one's ids from `id` on, the next ones' THREADS * 16 bytes behind.  single(logit, id): in front of and behind what is aligned.
// meanwhile() runs while the first ones are on their way.
struct Nothing { __device__ __forceinline__ void operator()() const {} };
template <bool F32, int THREADS, int U, class Vectors, class Single, class Meanwhile = Nothing>
__device__ __forceinline__ void for_tokens(const void *row, int i0, int i1, Vectors vectors, Single single, Meanwhile meanwhile = Nothing())
{
    constexpr int SIZE = F32 ? 4 : 2, E = 16 / SIZE;
    const int tid = (int)threadIdx.x;
    const char *from = (const char *)row + (int64_t)i0 * SIZE;
    const int a0 = min(i1, i0 + (int)((16 - ((uintptr_t)from & 15)) & 15) / SIZE), nv = (i1 - a0) / E, t0 = a0 + nv * E;
    const char *body = (const char *)row + (int64_t)a0 * SIZE;
    u32x4 w[U], behind[U];
    auto load = [&](u32x4 (&to)[U], int v0) {
        if (v0 < nv) {
#pragma unroll
            for (int u = 0; u < U; ++u) to[u] = gld_16B(body + (int64_t)min(v0 + u * THREADS, nv - 1) * 16);
        }
    };
    load(w, tid);
    meanwhile();
    if (i0 + tid < a0) single(raw_logit<F32>(row, i0 + tid), i0 + tid);
    for (int v0 = tid; v0 < nv; v0 += THREADS * U) {
        load(behind, v0 + THREADS * U);
        vectors(w, min(U, (nv - v0 + THREADS - 1) / THREADS), a0 + v0 * E);
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = behind[u];
    }
    if (t0 + tid < i1) single(raw_logit<F32>(row, t0 + tid), t0 + tid);
}
template <bool F32> __device__ __forceinline__ float element(u32x4 w, int e)
{
    return F32 ? __uint_as_float(w[e & 3]) : (e & 1) ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]);
}

__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }
constexpr uint32_t kBannedKey = 0x007FFFFFu;                 // of -inf

// A token in the order: larger is earlier.
__device__ __forceinline__ float entry_logit(uint64_t e) { return key_logit((uint32_t)(e >> 32)); }

struct RowScale {
    float top;               // largest logit
    double inv_t;
    double per;              // 2^20 / width of the bins together
    double steps;            // 1024 log2(e) / T: a weight is 2^(-distance * steps / 1024)
};

// 2^(35 - j / 1024): a weight is one of these, times a polynomial in the rest of its exponent (below 2^-10: three terms in fp32
// leave 2^-34 of it), times a power of two.  Eleven operations in 64 bits; exp() took three times as long.
__device__ __forceinline__ void fill_powers(double *table)
{
    for (int j = (int)threadIdx.x; j < 1024; j += (int)blockDim.x) table[j] = exp2((double)kUnitBits - (double)j * 0x1p-10);
}
__device__ __forceinline__ uint64_t weight_of(const RowScale &R, const double *table, float x)      // exp((x - top) / T) in units
{
    // No branches: a thread's tokens then go through side by side.  From 37 on 0 (below half a unit), and what is no number as well: next
    // to +inf, where all finite ones are banned, and what is banned itself.
    const double t = fmin(((double)R.top - (double)x) * R.steps, 37.0 * 1024.0);
    const int n = (int)t;
    const float r = (float)(t - (double)n) * (float)(0.69314718055994531 / 1024.0);
    const float s = -r + r * r * (0.5f - r * 0.16666667f);
    const double base = table[n & 1023];
    const double w = __builtin_ldexp(__builtin_fma(base, (double)s, base), -(n >> 10));
    const uint64_t whole = (uint64_t)__double_as_longlong(w + 0x1p52) & ((1ull << 52) - 1);      // rounded
    return x == R.top ? kTopWeight : whole;                  // +inf among them
}
__device__ __forceinline__ uint32_t place_of(const RowScale &R, float x)      // bin << 10 | place within it; does not decrease with the distance from the top
{
    const double d = ((double)R.top - (double)x) * R.per;
    return d < 1048575.0 ? (uint32_t)d : 1048575u;
}

struct RowStats { float top, low; uint32_t first, live; };      // largest logit and its first token; smallest; tokens that are not banned

template <class T> __device__ __forceinline__ T wave_all_sum(T v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
template <class T> __device__ __forceinline__ T wave_all_max(T v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { const T t = __shfl_xor(v, o, 64); v = t > v ? t : v; }
    return v;
}

__device__ __forceinline__ void join(RowStats &st, const RowStats &t)
{
    if (t.top > st.top || (t.top == st.top && t.first < st.first)) { st.top = t.top; st.first = t.first; }
    st.low = fminf(st.low, t.low);
    st.live += t.live;
}
__device__ __forceinline__ RowStats wave_join(RowStats st)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1)
        join(st, RowStats{__shfl_xor(st.top, o, 64), __shfl_xor(st.low, o, 64), (uint32_t)__shfl_xor((int)st.first, o, 64), (uint32_t)__shfl_xor((int)st.live, o, 64)});
    return st;
}

// One pass over the tokens [i0, i1) of a row by the workgroup; the same in every thread.
template <bool F32, int THREADS, class Meanwhile = Nothing>
__device__ __forceinline__ RowStats row_stats(const void *row, int i0, int i1, RowStats *s_red, Meanwhile meanwhile = Nothing())
{
    RowStats st{-INFINITY, INFINITY, 0xFFFFFFFFu, 0};
    auto one = [&](float x, int i) {
        if (x > st.top) { st.top = x; st.first = (uint32_t)i; }
        const bool live = x > -INFINITY;                     // no NaN either
        st.low = live ? fminf(st.low, x) : st.low;
        st.live += live;
    };
    for_tokens<F32, THREADS, 4>(row, i0, i1, [&](const u32x4 (&w)[4], int n, int id) {
        constexpr int E = F32 ? 4 : 8;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (u >= n) break;
#pragma unroll
            for (int e = 0; e < E; ++e) one(element<F32>(w[u], e), id + u * THREADS * E + e);
        }
    }, one, meanwhile);
    st = wave_join(st);
    if (lane_id() == 0) s_red[wave_id()] = st;
    __syncthreads();
    st = s_red[0];
    for (int w = 1; w < THREADS / 64; ++w) join(st, s_red[w]);
    __syncthreads();
    return st;
}

__device__ __forceinline__ RowScale scale_of(const RowStats &st, float T)
{
    RowScale R{st.top, 1.0 / (double)T, 0.0, 1024.0 * 1.4426950408889634 / (double)T};
    const double range = fmin((double)st.top - (double)st.low, 32.0 * (double)T);
    R.per = range > 0.0 ? fmin(1048576.0 / range, 1e300) : 0.0;
    return R;
}

// A slice's bins, or a row's: weight, and tokens in the upper bits.
template <bool F32, int THREADS>
__device__ __forceinline__ void fill_bins(const void *row, int i0, int i1, const RowScale &R, const double *table, unsigned long long *bins)
{
    auto one = [&](float x, int) {
        const uint64_t own = weight_of(R, table, x) | 1ull << kCountShift;
        const uint32_t bin = place_of(R, x) >> 10;
        if (x > -INFINITY) atomicAdd(&bins[bin], (unsigned long long)own);
    };
    // word by word, in a loop: written out for all, the code does not stay in the instruction cache
    for_tokens<F32, THREADS, 2>(row, i0, i1, [&](const u32x4 (&w)[2], int n, int) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (u >= n) break;
            u32x4 v = w[u];
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
                if (F32) one(__uint_as_float(v.x), 0);
                else { one(bf16_lo(v.x), 0); one(bf16_hi(v.x), 0); }
                v = u32x4{v.y, v.z, v.w, v.x};
            }
        }
    }, one);
}

struct SampleArgs {
    ServingDev S;
    etc_serving_sample_io io;
    int slices, per_slice;   // of a row; tokens of one
    int shares;              // workgroups of sample_row to a row
};
template <bool F32> __device__ __forceinline__ const void *row_of(const SampleArgs &a, int r)
{
    return (const char *)a.io.logits + (int64_t)r * a.io.row_stride * (F32 ? 4 : 2);
}

template <bool F32>
__global__ __launch_bounds__(kSliceThreads) void sample_scan_kernel(SampleArgs a)
{
    __shared__ RowStats s_red[kSliceThreads / 64];
    const int r = (int)blockIdx.y, sl = (int)blockIdx.x, i0 = sl * a.per_slice, i1 = min(a.S.vocab, i0 + a.per_slice);
    const RowStats st = row_stats<F32, kSliceThreads>(row_of<F32>(a, r), i0, i1, s_red);
    if (threadIdx.x == 0) ((RowStats *)a.S.smp_stats)[(size_t)r * a.slices + sl] = st;
}

// The row's statistics from its slices', in every thread.
__device__ __forceinline__ RowStats join_stats(const SampleArgs &a, int r)
{
    RowStats st{-INFINITY, INFINITY, 0xFFFFFFFFu, 0};
    const RowStats *p = (const RowStats *)a.S.smp_stats + (size_t)r * a.slices;
    for (int i = lane_id(); i < a.slices; i += 64) join(st, p[i]);
    return wave_join(st);
}

template <bool F32>
__global__ __launch_bounds__(kSliceThreads) void sample_bins_kernel(SampleArgs a)
{
    __shared__ unsigned long long s_bins[kSmpBins];
    __shared__ double s_powers[1024];
    const int r = (int)blockIdx.y, sl = (int)blockIdx.x, i0 = sl * a.per_slice, i1 = min(a.S.vocab, i0 + a.per_slice);
    const float T = a.io.temperature ? *as_global(a.io.temperature + r) : 1.f;
    const RowStats st = join_stats(a, r);
    if (!(T > 0.f) || st.live == 0 || st.top == INFINITY) return;      // sample_row needs no bins
    for (int i = (int)threadIdx.x; i < kSmpBins; i += kSliceThreads) s_bins[i] = 0;
    fill_powers(s_powers);
    __syncthreads();
    fill_bins<F32, kSliceThreads>(row_of<F32>(a, r), i0, i1, scale_of(st, T), s_powers, s_bins);
    __syncthreads();
    uint64_t *bins = a.S.smp_bins + ((size_t)r * a.slices + sl) * kSmpBins;
    for (int i = (int)threadIdx.x; i < kSmpBins; i += kSliceThreads) bins[i] = s_bins[i];
}

// ---- the slow way ------------------------------------------------------------------------------------------------------
struct Prefix {              // a beginning of the order
    uint32_t key;            // of its last token
    uint32_t ties;           // how many tokens of that key belong to it
    uint32_t before;         // tokens of larger keys
    uint64_t mass;           // weight of all of it
};

// Sum over the workgroup, the same in every thread.
template <class T>
__device__ T wg_sum(T v, T *s_red)
{
    v = wave_all_sum(v);
    __syncthreads();
    if (lane_id() == 0) s_red[wave_id()] = v;
    __syncthreads();
    T t = 0;
    for (int w = 0; w < kSmpThreads / 64; ++w) t += s_red[w];
    return t;
}

constexpr int kSlowBins = 2048;
struct SlowLds {
    uint32_t count[kSlowBins];
    uint64_t mass[kSlowBins];
    uint64_t red[kSmpThreads / 64];
    uint32_t red_i[kSmpThreads / 64];
    uint32_t bin;
    uint32_t before;
    uint64_t mass_before;
    uint32_t id;
};

// The shortest beginning of the order that holds `want_count` tokens, or (want_count == 0) weighs `want_mass` at least; the row has
// it.  11 + 11 + 10 bits of the key at a time; equal keys have equal weights, so ties are settled by a division.
template <bool F32>
__device__ __forceinline__ Prefix find_prefix(SlowLds &L, const void *row, int vocab, const RowScale &R, const double *table, uint32_t want_count, uint64_t want_mass)
{
    const int tid = (int)threadIdx.x;
    uint32_t prefix = 0, before = 0;
    uint64_t mass_before = 0;
    const int bits[3] = {11, 11, 10};
    int shift = 32;
    for (int level = 0; level < 3; ++level) {
        const int high = shift;                              // bits above are fixed
        shift -= bits[level];
        const uint32_t bins = 1u << bits[level];
        for (int i = tid; i < kSlowBins; i += kSmpThreads) { L.count[i] = 0; L.mass[i] = 0; }
        __syncthreads();
        for (int i = tid; i < vocab; i += kSmpThreads) {
            const float x = logit_at<F32>(row, i);
            const uint32_t k = order_key(x);
            if (k == kBannedKey || (level > 0 && (k >> high) != (prefix >> high))) continue;
            const uint32_t b = (k >> shift) & (bins - 1);
            atomicAdd(&L.count[b], 1u);
            const uint64_t w = weight_of(R, table, x);
            if (w) atomicAdd((unsigned long long *)&L.mass[b], (unsigned long long)w);
        }
        __syncthreads();
        // two bins a thread, from the largest key down: prefix sums across the workgroup
        const int hi = kSlowBins - 1 - 2 * tid, lo = hi - 1;
        const uint32_t c0 = L.count[hi], c1 = L.count[lo];
        const uint64_t m0 = L.mass[hi], m1 = L.mass[lo];
        uint32_t c = c0 + c1;
        uint64_t m = m0 + m1;
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t tc = __shfl_up(c, o, 64);
            const uint64_t tm = __shfl_up(m, o, 64);
            if (lane_id() >= o) { c += tc; m += tm; }
        }
        if (lane_id() == 63) { L.red_i[wave_id()] = c; L.red[wave_id()] = m; }
        __syncthreads();
        for (int w = 0; w < wave_id(); ++w) { c += L.red_i[w]; m += L.red[w]; }
        const uint32_t cb = before + c - (c0 + c1);          // in front of this thread's bins
        const uint64_t mb = mass_before + m - (m0 + m1);
        auto holds = [&](uint32_t cc, uint64_t mm) { return want_count ? cc >= want_count : mm >= want_mass; };
        if (!holds(cb, mb)) {                                // one thread and one bin: the sums do not decrease
            if (holds(cb + c0, mb + m0)) { L.bin = hi; L.before = cb; L.mass_before = mb; }
            else if (holds(cb + c0 + c1, mb + m0 + m1)) { L.bin = lo; L.before = cb + c0; L.mass_before = mb + m0; }
        }
        __syncthreads();
        prefix |= L.bin << shift;
        before = L.before;
        mass_before = L.mass_before;
        __syncthreads();
    }
    Prefix p;
    p.key = prefix;
    p.before = before;
    const uint64_t w = weight_of(R, table, key_logit(prefix));
    p.ties = want_count ? want_count - before : (uint32_t)((want_mass - mass_before + w - 1) / w);
    p.mass = mass_before + p.ties * w;
    return p;
}

struct Drawn { uint32_t id, kept; float logprob; };
struct Settings { float T, top_p, min_p, u; int top_k; };

__device__ __forceinline__ uint64_t mass_wanted(float p, uint64_t mass)      // by a top_p below 1; sums are whole numbers
{
    const uint64_t want = (uint64_t)ceil(fmax((double)p, 0.0) * (double)mass);
    return want < 1 ? 1 : want > mass ? mass : want;
}
__device__ __forceinline__ uint64_t draw_wanted(float u, uint64_t mass)      // the first running sum above u * mass
{
    u = u > 0.f ? fminf(u, 1.f) : 0.f;
    const uint64_t want = (uint64_t)((double)u * (double)mass) + 1;
    return want > mass ? mass : want;
}
__device__ __forceinline__ bool above_min_p(const RowScale &R, float x, float min_p)
{
    return x == R.top || (R.top != INFINITY && exp(((double)x - (double)R.top) * R.inv_t) >= (double)min_p);
}
__device__ __forceinline__ float log_share(const RowScale &R, float x, uint64_t mass)      // from the logit, not from its weight in fixed point
{
    return (float)((x == R.top ? 0.0 : ((double)x - (double)R.top) * R.inv_t) - log((double)mass * 0x1p-35));
}

template <bool F32>
__device__ __forceinline__ Drawn slow_row(SlowLds &L, const void *row, int vocab, const RowScale &R, const double *table, uint32_t live, const Settings &q)
{
    const int tid = (int)threadIdx.x;
    uint32_t n_live = live;
    if (R.top == INFINITY) {                                 // next to +inf the finite ones are banned
        uint32_t inf = 0;
        for (int i = tid; i < vocab; i += kSmpThreads) inf += logit_at<F32>(row, i) == INFINITY;
        n_live = wg_sum<uint32_t>(inf, L.red_i);
    }
    uint32_t kept = q.top_k > 0 ? min((uint32_t)q.top_k, n_live) : n_live;
    uint64_t mass = find_prefix<F32>(L, row, vocab, R, table, kept, 0).mass;
    if (q.top_p < 1.f) {
        const Prefix p = find_prefix<F32>(L, row, vocab, R, table, 0, mass_wanted(q.top_p, mass));
        kept = p.before + p.ties;
        mass = p.mass;
    }
    if (q.min_p > 0.f) {
        uint32_t above = 0;
        uint64_t m = 0;
        for (int i = tid; i < vocab; i += kSmpThreads) {
            const float x = logit_at<F32>(row, i);
            if (x != -INFINITY && above_min_p(R, x, q.min_p)) { above++; m += weight_of(R, table, x); }
        }
        above = wg_sum<uint32_t>(above, L.red_i);
        m = wg_sum<uint64_t>(m, L.red);
        if (q.min_p > 1.f) { above = 1; m = kTopWeight; }
        if (above < kept) { kept = above; mass = m; }
    }
    const Prefix d = find_prefix<F32>(L, row, vocab, R, table, 0, draw_wanted(q.u, mass));
    // the ties-th token of the key, by id: a count in front of each thread's stretch of ids
    const int per = (vocab + kSmpThreads - 1) / kSmpThreads, i0 = min(vocab, tid * per), i1 = min(vocab, i0 + per);
    uint32_t n = 0;
    for (int i = i0; i < i1; ++i) n += order_key(logit_at<F32>(row, i)) == d.key;
    uint32_t upto = (uint32_t)wave_scan_i((int)n);
    if (lane_id() == 63) L.red_i[wave_id()] = upto;
    __syncthreads();
    for (int w = 0; w < wave_id(); ++w) upto += L.red_i[w];
    uint32_t left = d.ties - (upto - n);                     // which of this stretch's, from 1
    if (upto - n < d.ties && d.ties <= upto) {
        int i = i0;
        for (; i < i1; ++i)
            if (order_key(logit_at<F32>(row, i)) == d.key && --left == 0) break;
        L.id = (uint32_t)i;
    }
    __syncthreads();
    return Drawn{L.id, kept, log_share(R, key_logit(d.key), mass)};
}

// ---- a row -------------------------------------------------------------------------------------------------------------
struct FastLds {
    uint32_t upto[kSmpBins];                                 // tokens up to and with a bin
    uint64_t mass_upto[kSmpBins], sub[kSmpBins];             // their weight; the places within a bin
    uint32_t id[kSmpList], key[kSmpList], place[kSmpList];   // the tokens in question (and some next to them)
    uint64_t few[kSmpFew], few_mass[kSmpFew];
    uint32_t n_list, n_few, found[8];
    uint64_t red[kSmpThreads / 64];
    uint32_t red_i[kSmpThreads / 64];
    uint64_t end_mass, end_entry;
    uint32_t end_count;
};
union RowLds {
    FastLds f;
    SlowLds s;
    RowStats stats[kSmpThreads / 64];
};

template <int CTRL, int ROWS> __device__ __forceinline__ uint64_t dpp_u64(uint64_t v)
{
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, false);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t row_scan_u64(uint64_t v)      // over rows of 16 lanes
{
    v += dpp_u64<0x111, 0xF>(v);
    v += dpp_u64<0x112, 0xF>(v);
    v += dpp_u64<0x114, 0xF>(v);
    v += dpp_u64<0x118, 0xF>(v);
    return v;
}
__device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v)
{
    v = row_scan_u64(v);
    v += dpp_u64<0x142, 0xA>(v);
    v += dpp_u64<0x143, 0xC>(v);
    return v;
}
__device__ __forceinline__ uint64_t lane_u64(uint64_t v, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

// Running sums over the workgroup, of one value a thread: a wavefront's by lane moves, the 16 wavefronts' by the lanes of a row.
__device__ __forceinline__ void wg_scan(FastLds &L, uint32_t &c, uint64_t &m)
{
    static_assert(kSmpThreads / 64 == 16, "a row of lanes");
    c = (uint32_t)wave_scan_i((int)c);
    m = wave_scan_u64(m);
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id();
    __syncthreads();
    if (lane == 63) { L.red_i[wave] = c; L.red[wave] = m; }
    __syncthreads();
    const uint32_t cw = (uint32_t)wave_scan_i(lane < 16 ? (int)L.red_i[lane & 15] : 0);
    const uint64_t mw = row_scan_u64(L.red[lane & 15]);
    if (wave > 0) {
        c += (uint32_t)__builtin_amdgcn_readlane((int)cw, wave - 1);
        m += lane_u64(mw, wave - 1);
    }
}

struct End { uint32_t count; uint64_t mass, entry; bool ok; };      // of a beginning: its tokens, its weight, its last token

// The r-th token (from 1), by id, of those in the list that lie in `place`, which have one key.  Sorted by id into 1024 bins, the right
// one's counted one by one.
__device__ __forceinline__ uint64_t tied_token(FastLds &L, uint32_t place, uint32_t r, uint32_t vocab)
{
    const int tid = (int)threadIdx.x;
    const uint32_t n = L.n_list, per = (vocab + 1023) / 1024;
    L.sub[tid] = 0;
    if (tid == 0) L.n_few = 0;
    __syncthreads();
    for (uint32_t i = tid; i < n; i += kSmpThreads)
        if (L.place[i] == place) atomicAdd((unsigned long long *)&L.sub[L.id[i] / per], 1ull);
    __syncthreads();
    uint32_t c = (uint32_t)L.sub[tid];
    const uint32_t own = c;
    uint64_t none = 0;
    wg_scan(L, c, none);
    if (c - own < r && r <= c) { L.found[7] = tid; L.end_count = c - own; }
    __syncthreads();
    const uint32_t bin = L.found[7], left = r - L.end_count;      // at most `per` <= 1024 tokens
    for (uint32_t i = tid; i < n; i += kSmpThreads)
        if (L.place[i] == place && L.id[i] / per == bin) L.few[atomicAdd(&L.n_few, 1u)] = (uint64_t)L.key[i] << 32 | ~L.id[i];
    __syncthreads();
    const uint32_t few = L.n_few;
    if (tid < (int)few) {
        const uint64_t e = L.few[tid];
        uint32_t rank = 1;
        for (uint32_t j = 0; j < few; ++j) rank += L.few[j] > e;
        if (rank == left) L.end_entry = e;
    }
    __syncthreads();
    return L.end_entry;
}

// The beginning that ends in `bin` (whose tokens are in the list), holds `want_count` tokens or weighs `want_mass` at least.  Its last
// token is named for the draw only.
__device__ __forceinline__ End end_in_bin(FastLds &L, const RowScale &R, const double *table, uint32_t vocab, uint32_t bin, uint32_t want_count, uint64_t want_mass, bool draw)
{
    const int tid = (int)threadIdx.x;
    uint32_t before = bin ? L.upto[bin - 1] : 0;
    uint64_t mass_before = bin ? L.mass_upto[bin - 1] : 0;
    auto holds = [&](uint32_t c, uint64_t m) { return want_count ? c >= want_count : m >= want_mass; };
    L.sub[tid] = 0;
    if (tid == 0) { L.n_few = 0; L.found[6] = 0; }
    __syncthreads();
    const uint32_t n = L.n_list;
    for (uint32_t i = tid; i < n; i += kSmpThreads)
        if (L.place[i] >> 10 == bin)
            atomicAdd((unsigned long long *)&L.sub[L.place[i] & 1023], (unsigned long long)(weight_of(R, table, key_logit(L.key[i])) | 1ull << kCountShift));
    __syncthreads();
    const uint32_t c_own = (uint32_t)(L.sub[tid] >> kCountShift);
    const uint64_t m_own = L.sub[tid] & ((1ull << kCountShift) - 1);
    uint32_t c = c_own;
    uint64_t m = m_own;
    wg_scan(L, c, m);
    c += before;
    m += mass_before;
    if (!holds(c - c_own, m - m_own) && holds(c, m)) {
        L.found[7] = tid;
        L.end_count = c - c_own;
        L.end_mass = m - m_own;
    }
    __syncthreads();
    const uint32_t place = bin << 10 | L.found[7], few = (uint32_t)(L.sub[L.found[7]] >> kCountShift);
    before = L.end_count;
    mass_before = L.end_mass;
    for (uint32_t i = tid; i < n; i += kSmpThreads)          // the tokens of the place
        if (L.place[i] == place) {
            const uint32_t at = atomicAdd(&L.n_few, 1u);
            if (at < kSmpFew) L.few[at] = (uint64_t)L.key[i] << 32 | ~L.id[i];
        }
    __syncthreads();
    const uint64_t one = L.few[0];                           // have they one key?
    if (few <= kSmpFew) {
        if (tid < (int)few) {
            if ((uint32_t)(L.few[tid] >> 32) != (uint32_t)(one >> 32)) L.found[6] = 1;
            L.few_mass[tid] = weight_of(R, table, entry_logit(L.few[tid]));
        }
    } else {
        for (uint32_t i = tid; i < n; i += kSmpThreads)
            if (L.place[i] == place && L.key[i] != (uint32_t)(one >> 32)) L.found[6] = 1;
    }
    __syncthreads();
    if (!L.found[6] && few > 1) {                            // equal keys: equal weights
        const uint64_t w = weight_of(R, table, entry_logit(one));
        const uint32_t r = want_count ? want_count - before : (uint32_t)((want_mass - mass_before + w - 1) / w);
        const End e{before + r, mass_before + r * w, draw ? tied_token(L, place, r, vocab) : one, true};
        __syncthreads();
        return e;
    }
    if (few > kSmpFew) return End{0, 0, 0, false};
    if (tid < (int)few) {                                    // what is in front of this thread's token, and with it
        const uint64_t e = L.few[tid], own = L.few_mass[tid];
        uint32_t cc = before;
        uint64_t mm = mass_before;
        for (uint32_t j = 0; j < few; ++j)
            if (L.few[j] > e) { cc++; mm += L.few_mass[j]; }
        if (!holds(cc, mm) && holds(cc + 1, mm + own)) { L.end_count = cc + 1; L.end_mass = mm + own; L.end_entry = e; }
    }
    __syncthreads();
    const End e{L.end_count, L.end_mass, L.end_entry, true};
    __syncthreads();
    return e;
}

// The same by every wavefront for itself, where the tokens fit its lanes (entry, bin and weight `w` of the lane's): no barrier, no bins.
struct Few { uint64_t entry, w; uint32_t bin; int n; };
__device__ __forceinline__ End end_among_few(const FastLds &L, const Few &F, uint32_t bin, uint32_t want_count, uint64_t want_mass)
{
    auto holds = [&](uint32_t c, uint64_t m) { return want_count ? c >= want_count : m >= want_mass; };
    const bool in = lane_id() < F.n && F.bin == bin;
    uint32_t c = bin ? L.upto[bin - 1] : 0;
    uint64_t m = bin ? L.mass_upto[bin - 1] : 0;
    for (uint64_t left = __ballot(in); left; left &= left - 1) {
        const int j = __builtin_ctzll(left);
        const uint64_t w = lane_u64(F.w, j);
        if (lane_u64(F.entry, j) > F.entry) { c++; m += w; }
    }
    const uint64_t here = __ballot(in && !holds(c, m) && holds(c + 1, m + F.w));
    const int at = here ? __builtin_ctzll(here) : 0;        // there is one
    return End{(uint32_t)__builtin_amdgcn_readlane((int)c + 1, at), lane_u64(m + F.w, at), lane_u64(F.entry, at), true};
}

// The row by its bins.  Several workgroups (none of them waits): each does the sums for itself and looks through a share of the row, and
// who lists its tokens last goes on alone.  TOO_MANY: more tokens are in question than the list holds.
enum RowEnd { ROW_DRAWN, ROW_TOO_MANY, ROW_OF_ANOTHER };
template <bool F32, bool WHOLE>
__device__ __forceinline__ RowEnd fast_row(const SampleArgs &a, FastLds &L, const void *row, const RowScale &R, const double *table, const Settings &q, int r, Drawn *out)
{
    const int tid = (int)threadIdx.x, vocab = a.S.vocab;
    // ---- the bins, one a thread, and their running sums
    uint32_t c_own = 0;
    uint64_t m_own = 0;
    auto unpack = [&](uint64_t v) { c_own += (uint32_t)(v >> kCountShift); m_own += v & ((1ull << kCountShift) - 1); };
    if constexpr (WHOLE) {
        L.sub[tid] = 0;
        __syncthreads();
        fill_bins<F32, kSmpThreads>(row, 0, vocab, R, table, (unsigned long long *)L.sub);
        __syncthreads();
        unpack(L.sub[tid]);
    } else {
        const uint64_t *bins = a.S.smp_bins + (size_t)r * a.slices * kSmpBins + tid;
#pragma unroll 16
        for (int sl = 0; sl < a.slices; ++sl) unpack(bins[(size_t)sl * kSmpBins]);
    }
    uint32_t c = c_own;
    uint64_t m = m_own;
    if (tid < 8) L.found[tid] = 0;
    if (tid == 0) L.n_list = 0;
    wg_scan(L, c, m);
    L.upto[tid] = c;
    L.mass_upto[tid] = m;
    __syncthreads();
    const uint64_t total = L.mass_upto[kSmpBins - 1];
    const uint32_t n_live = L.upto[kSmpBins - 1];

    // ---- where the beginnings can end: the bins in question.  found: 0 top_k; 1, 2 top_p at its least and most; 3, 4 the draw's
    const bool use_k = q.top_k > 0 && (uint32_t)q.top_k < n_live, use_p = q.top_p < 1.f, use_m = q.min_p > 0.f;
    auto holds_mass = [&](uint64_t want) { return m - m_own < want && want <= m; };
    auto mass_in_front = [&](uint32_t b) { return b ? L.mass_upto[b - 1] : 0ull; };
    if (use_k && c - c_own < (uint32_t)q.top_k && (uint32_t)q.top_k <= c) L.found[0] = tid;
    __syncthreads();
    const uint32_t bin_k = L.found[0];
    uint64_t least = use_k ? mass_in_front(bin_k) : total, most = use_k ? L.mass_upto[bin_k] : total;
    if (use_p) {
        if (holds_mass(mass_wanted(q.top_p, least > 0 ? least : 1))) L.found[1] = tid;
        if (holds_mass(mass_wanted(q.top_p, most))) L.found[2] = tid;
        __syncthreads();
        least = min(least, mass_in_front(L.found[1]));
        most = min(most, L.mass_upto[L.found[2]]);
    }
    uint32_t bin_m0 = 0, bin_m1 = 0;
    if (use_m) {                                             // its border, and a bin to either side for the rounding of the logarithm
        const double at = q.min_p < 1.f ? -log((double)q.min_p) * (double)q.T * R.per * 0.0009765625 : 0.0;
        const uint32_t b = at < (double)(kSmpBins - 1) ? (uint32_t)at : kSmpBins - 1;
        bin_m0 = b ? b - 1 : 0;
        bin_m1 = min(b + 1, (uint32_t)kSmpBins - 1);
        least = min(least, mass_in_front(bin_m0));
        most = min(most, L.mass_upto[bin_m1]);
    }
    if (holds_mass(draw_wanted(q.u, least > 0 ? least : 1))) L.found[3] = tid;
    if (holds_mass(draw_wanted(q.u, most))) L.found[4] = tid;
    __syncthreads();
    const uint32_t p0 = L.found[1], p1 = L.found[2], d0 = L.found[3], d1 = L.found[4];
    // The tokens of the bins in question, by intervals of logits a hundredth of a bin wider, in fp32: their ids first, then all their
    // logits at once.  One interval from the first of the bins to the last where that holds few tokens (with filters the ends lie close
    // together: 64 rows of 128256 with all filters took 55 us so, 64 before, with what follows it and one workgroup to a row), else one for each end.
    const uint32_t b0[4] = {d0, p0, bin_k, bin_m0}, b1[4] = {d1, p1, bin_k, bin_m1};
    bool use[4] = {true, use_p, use_k, use_m};
    uint32_t first = d0, last = d1;
#pragma unroll
    for (int i = 1; i < 4; ++i)
        if (use[i]) { first = min(first, b0[i]); last = max(last, b1[i]); }
    const bool one = L.upto[last] - (first ? L.upto[first - 1] : 0) <= kSmpList / 4;
    float lo[4], hi[4];
    {
        const double wide = R.per > 0.0 ? 1024.0 / R.per : 0.0;
        const float slack = fabsf(R.top) * 0x1p-22f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t from = one ? first : b0[i], to = one ? last : b1[i];
            use[i] &= i == 0 || !one;
            hi[i] = from == 0 ? R.top : (float)((double)R.top - ((double)from - 0.01) * wide) + slack;
            lo[i] = R.per == 0.0 || to == kSmpBins - 1 ? -3.402823466e38f : (float)((double)R.top - ((double)to + 1.01) * wide) - slack;
        }
    }
    auto inside = [&](float x, int i) { return __builtin_amdgcn_fmed3f(x, lo[i], hi[i]) == x; };      // NaN: no
    const int per_share = WHOLE ? vocab : (vocab + a.shares - 1) / a.shares, i0 = WHOLE ? 0 : min(vocab, (int)blockIdx.y * per_share);
    for_tokens<F32, kSmpThreads, 4>(row, i0, min(vocab, i0 + per_share), [&](const u32x4 (&w)[4], int n, int id) {
        constexpr int E = F32 ? 4 : 8, ALL = 4 * E;
        uint32_t hits = 0;                                   // the first element's is the highest of ALL bits
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!use[i]) continue;
            uint32_t h = 0;
#pragma unroll
            for (int e = 0; e < ALL; ++e) h = h + h + (uint32_t)inside(element<F32>(w[e / E], e % E), i);
            hits |= h;
        }
        hits &= ~0u << ((4 - n) * E);
        const int mine = __builtin_popcount(hits);
        if (mine == 0) return;
        uint32_t at = atomicAdd(&L.n_list, (uint32_t)mine);
        for (; hits; hits &= hits - 1, ++at) {
            const int k = ALL - 1 - __builtin_ctz(hits);
            if (at < kSmpList) L.id[at] = (uint32_t)(id + (k / E) * kSmpThreads * E + k % E);
        }
    }, [&](float x, int id) {
        if (!(inside(x, 0) || (use[1] && inside(x, 1)) || (use[2] && inside(x, 2)) || (use[3] && inside(x, 3)))) return;
        const uint32_t at = atomicAdd(&L.n_list, 1u);
        if (at < kSmpList) L.id[at] = (uint32_t)id;
    });
    __syncthreads();
    if (!WHOLE && a.shares > 1) {
        int32_t *list = a.S.smp_list + (size_t)r * kSmpList;
        const uint32_t mine = L.n_list;
        if (tid == 0) L.end_count = (uint32_t)__hip_atomic_fetch_add(as_global(a.S.smp_listed + r), (int)mine, __ATOMIC_RELAXED, ETC_SCOPE);
        __syncthreads();
        for (uint32_t i = tid; i < min(mine, (uint32_t)kSmpList) && L.end_count + i < kSmpList; i += kSmpThreads) st_i32(list + L.end_count + i, (int)L.id[i]);
        wg_release();
        if (tid == 0) {
            const bool last = __hip_atomic_fetch_add(as_global(a.S.smp_done + r), 1, __ATOMIC_RELAXED, ETC_SCOPE) + 1 == a.shares;
            if (last) {
                L.n_list = (uint32_t)ld_i32(a.S.smp_listed + r);
                st_i32(a.S.smp_listed + r, 0);
                st_i32(a.S.smp_done + r, 0);
            }
            L.end_count = last;
        }
        __syncthreads();
        if (!L.end_count) return ROW_OF_ANOTHER;
        for (uint32_t i = tid; i < min(L.n_list, (uint32_t)kSmpList); i += kSmpThreads) L.id[i] = (uint32_t)ld_i32(list + i);
        __syncthreads();
    }
    if (L.n_list > kSmpList) return ROW_TOO_MANY;
    const bool is_few = L.n_list <= 64;
    Few F{0, 0, 0, (int)L.n_list};
    if (is_few) {
        if (lane_id() < F.n) {
            const uint32_t id = L.id[lane_id()];
            const float x = logit_at<F32>(row, (int)id);
            F.entry = (uint64_t)order_key(x) << 32 | (uint32_t)~id;
            F.w = weight_of(R, table, x);
            F.bin = place_of(R, x) >> 10;
        }
    } else {
        for (uint32_t j = tid; j < L.n_list; j += kSmpThreads) {
            const float x = logit_at<F32>(row, (int)L.id[j]);
            L.key[j] = order_key(x);
            L.place[j] = place_of(R, x);
        }
        __syncthreads();
    }

    // ---- exactly: top_k, top_p and, behind min_p, the draw; one after the other through the same code
    uint32_t kept = n_live;
    uint64_t mass = total;
#pragma unroll 1
    for (int stage = use_k ? 0 : use_p ? 1 : 2; stage < 3; stage += stage == 0 && !use_p ? 2 : 1) {
        uint64_t want = 0;
        uint32_t bin = bin_k;
        if (stage == 2 && use_m) {
            uint32_t above = 0;
            uint64_t am = 0;
            auto near = [&](uint32_t b, float x) { return b >= bin_m0 && b <= bin_m1 && above_min_p(R, x, q.min_p); };
            if (is_few) {
                if (lane_id() < F.n && near(F.bin, entry_logit(F.entry))) { above = 1; am = F.w; }
                above = (uint32_t)__popcll(__ballot(above));
                am = lane_u64(wave_scan_u64(am), 63);
            } else {
                for (uint32_t i = tid; i < L.n_list; i += kSmpThreads) {
                    const float x = key_logit(L.key[i]);
                    if (near(L.place[i] >> 10, x)) { above++; am += weight_of(R, table, x); }
                }
                above = wg_sum<uint32_t>(above, L.red_i);
                am = wg_sum<uint64_t>(am, L.red);
            }
            above += bin_m0 ? L.upto[bin_m0 - 1] : 0;
            am += mass_in_front(bin_m0);
            if (q.min_p > 1.f) { above = 1; am = kTopWeight; }
            if (above < kept) { kept = above; mass = am; }
        }
        if (stage > 0) {
            want = stage == 1 ? mass_wanted(q.top_p, mass) : draw_wanted(q.u, mass);
            __syncthreads();
            if (holds_mass(want)) L.found[5] = tid;
            __syncthreads();
            bin = L.found[5];
        }
        const uint32_t count = stage == 0 ? (uint32_t)q.top_k : 0;
        const uint32_t in_bin = L.upto[bin] - (bin ? L.upto[bin - 1] : 0);
        if (!is_few && in_bin <= 64) {
            if (tid == 0) L.n_few = 0;
            __syncthreads();
            for (uint32_t i = tid; i < L.n_list; i += kSmpThreads)
                if (L.place[i] >> 10 == bin) L.few[atomicAdd(&L.n_few, 1u)] = (uint64_t)L.key[i] << 32 | ~L.id[i];
            __syncthreads();
            F = Few{0, 0, bin, (int)in_bin};
            if (lane_id() < F.n) {
                F.entry = L.few[lane_id()];
                F.w = weight_of(R, table, entry_logit(F.entry));
            }
        }
        const End e = in_bin <= 64 ? end_among_few(L, F, bin, count, want) : end_in_bin(L, R, table, vocab, bin, count, want, stage == 2);
        if (!e.ok) return ROW_TOO_MANY;
        if (stage == 2) {
            *out = Drawn{~(uint32_t)e.entry, kept, log_share(R, entry_logit(e.entry), mass)};
        } else {
            kept = e.count;
            mass = e.mass;
        }
    }
    return ROW_DRAWN;
}

template <bool F32, bool WHOLE>
__global__ __launch_bounds__(kSmpThreads) void sample_row_kernel(SampleArgs a)
{
    __shared__ RowLds lds;
    __shared__ double table[1024];
    FastLds &L = lds.f;
    const int tid = (int)threadIdx.x, r = (int)blockIdx.x, vocab = a.S.vocab;
    const etc_serving_sample_io &io = a.io;
    const void *row = row_of<F32>(a, r);
    Settings q;
    q.T = io.temperature ? *as_global(io.temperature + r) : 1.f;
    q.top_k = io.top_k ? gld_i32(io.top_k + r) : 0;
    q.top_p = io.top_p ? *as_global(io.top_p + r) : 1.f;
    q.min_p = io.min_p ? *as_global(io.min_p + r) : 0.f;
    q.u = *as_global(io.u + r);
    const bool first = blockIdx.y == 0;                      // of the row's workgroups: for what all of them know
    auto answer = [&](int32_t token, float logprob, uint32_t kept) {
        if (tid != 0) return;
        *as_global(io.token_out + r) = token;
        if (io.logprob_out) gst_f32(io.logprob_out + r, logprob);
        if (io.kept_out) *as_global(io.kept_out + r) = (int32_t)kept;
    };
    RowStats st;
    if constexpr (WHOLE) {
        st = row_stats<F32, kSmpThreads>(row, 0, vocab, lds.stats, [&]() { fill_powers(table); });
    } else {
        fill_powers(table);                                  // (a barrier is in front of its first use)
        st = join_stats(a, r);
    }
    if (!first && (st.live == 0 || !(q.T > 0.f) || st.top == INFINITY)) return;
    if (st.live == 0) return answer(-1, -INFINITY, 0);
    if (!(q.T > 0.f)) return answer((int32_t)st.first, 0.f, 1);
    const RowScale R = scale_of(st, q.T);
    Drawn drawn;
    const RowEnd end = R.top == INFINITY ? ROW_TOO_MANY : fast_row<F32, WHOLE>(a, L, row, R, table, q, r, &drawn);
    if (end == ROW_OF_ANOTHER) return;
    if (end == ROW_TOO_MANY) {
        __syncthreads();
        drawn = slow_row<F32>(lds.s, row, vocab, R, table, st.live, q);
    }
    answer((int32_t)drawn.id, drawn.logprob, drawn.kept);
}

// Slices of a row: as many as give kSmpWgs workgroups, of 2048 tokens at least, and of kBinTokens at most.
static int slices_of(int vocab, int rows)
{
    const int most = (vocab + 2047) / 2048, least = (vocab + kBinTokens - 1) / kBinTokens;
    int s = kSmpWgs / rows;
    if (s > most) s = most;
    return s < least ? least : s;
}

// Workgroups of sample_row to a row: as many as there are compute units for (one fills one), with kBinTokens to look through at least.
static int shares_of(int vocab, int rows)
{
    const int room = kSmpWgs / rows, most = vocab / kBinTokens;
    static_assert(kSmpWgs / (kSampleSharedRows + 1) < 2, "rows that are shared have a list");
    return room < 2 || most < 2 ? 1 : room < most ? room : most;
}

template <bool F32>
static void launch_sample(const SampleArgs &a, hipStream_t s)
{
    if (a.S.vocab <= kSmpWhole) {
        hipLaunchKernelGGL((sample_row_kernel<F32, true>), dim3(a.io.n_rows), dim3(kSmpThreads), 0, s, a);
        return;
    }
    const dim3 grid((unsigned)a.slices, (unsigned)a.io.n_rows);
    hipLaunchKernelGGL((sample_scan_kernel<F32>), grid, dim3(kSliceThreads), 0, s, a);
    hipLaunchKernelGGL((sample_bins_kernel<F32>), grid, dim3(kSliceThreads), 0, s, a);
    hipLaunchKernelGGL((sample_row_kernel<F32, false>), dim3((unsigned)a.io.n_rows, (unsigned)a.shares), dim3(kSmpThreads), 0, s, a);
}

hipError_t launch_serving_sample(const ServingDev &S, const etc_serving_sample_io &io, hipStream_t s)
{
    SampleArgs a{S, io, slices_of(S.vocab, io.n_rows), 0, shares_of(S.vocab, io.n_rows)};
    a.per_slice = (S.vocab + a.slices - 1) / a.slices;
    if (io.dtype == ETC_FP32) launch_sample<true>(a, s); else launch_sample<false>(a, s);
    return hipGetLastError();
}

// Workspace of a handle: slices of a launch, all rows together (the bins' part holds the slices of the scores too).
static_assert((int64_t)kSmpWgs * kSmpBins * 8 >= (int64_t)kScoreParts * (16 + 8 * kScoreTop), "scores");
int64_t sample_slices(int vocab, int max_rows)
{
    if (vocab <= kSmpWhole) return 0;
    const int64_t least = (int64_t)max_rows * ((vocab + kBinTokens - 1) / kBinTokens);
    return least > kSmpWgs ? least : kSmpWgs;
}
int64_t sample_stat_bytes() { return (int64_t)sizeof(RowStats); }
int64_t sample_bins_bytes() { return kSmpBins * 8; }

}  // namespace etc
#endif  // ETC_GENERIC_ONLY
