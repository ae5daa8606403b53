// Serving operators beside the decode step (include/etc.h): page tables and slot maps, norm + RoPE + KV append, sampling.
#ifndef ETC_GENERIC_ONLY
#include "serving_rt.hip.h"

namespace etc {

// ---- page tables and slot maps --------------------------------------------------------------------------------------
// Prefix sums over the sequences (new tokens, pages, fresh pages), one sequence to a thread; then every page entry and
// every token row finds its sequence by a search in LDS.  A workgroup computes all sums itself (at most 1024 sequences), so
// that one launch is enough.  Inputs that outputs may alias (lengths, free count) are written by the workgroup that is the
// last to have read them.
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
            slot = (page_id(b, pos >> psh, pages_held(b)) << psh) + (pos & pmask);
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
constexpr int kAppThreads = 256;
constexpr int kAppMaxTokens = 16;

template <int D>
__device__ __forceinline__ float head_sum(float v)          // over D / 16 lanes
{
    v += dpp_f32<0xB1>(v);
    v += dpp_f32<0x4E>(v);
    if (D == 128) v += dpp_f32<0x141>(v);
    return v;
}

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
// Everything the filters and the draw ask for is a beginning of the tokens in the order (larger logit, lower id), named by
// the key of its last logit and how many of that key's tokens belong to it.  It is found by descending through the 32 bits
// of the (order-preserving) key, 11 + 11 + 10 of them at a time, over counts or over sums of weights.  Weights are computed in
// double and summed as 64-bit integers: sums are exact, so no result depends on an order of additions, and equal keys have
// equal weights, so ties are settled by a division.  One workgroup per row.
constexpr int kSmpThreads = 1024;
constexpr int kSmpBins = 2048;

template <bool F32>
__device__ __forceinline__ float logit_at(const void *row, int i)
{
    float x = F32 ? *as_global((const float *)row + i) : bf16_bits_to_f32(gld_u16((const uint16_t *)row + i));
    x = x != x ? -INFINITY : x;                              // NaN: banned
    return x + 0.f;                                          // -0 is +0: equal logits
}
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }
constexpr uint32_t kBannedKey = 0x007FFFFFu;                 // of -inf

struct RowScale { float top; double inv_t; };
__device__ __forceinline__ uint64_t weight_of(const RowScale &R, float x)      // exp((x - top) / T), unit 2^-43
{
    if (x == R.top) return 1ull << 43;
    if (R.top == INFINITY) return 0;
    const double w = exp(((double)x - (double)R.top) * R.inv_t);
    return (uint64_t)rint(w * 8796093022208.0);
}

struct Prefix {              // a beginning of the order
    uint32_t key;            // of its last token
    uint32_t ties;           // how many tokens of that key belong to it
    uint32_t before;         // tokens of larger keys
    uint64_t mass;           // weight of all of it
    uint64_t mass_before;    // weight of the tokens of larger keys
};

// Sum over the workgroup, the same in every thread.
template <class T>
__device__ T wg_sum(T v, T *s_red)
{
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if (lane_id() == 0) s_red[wave_id()] = v;
    __syncthreads();
    T t = 0;
    for (int w = 0; w < kSmpThreads / 64; ++w) t += s_red[w];
    return t;
}

struct SampleLds {
    uint32_t count[kSmpBins];
    uint64_t mass[kSmpBins];
    uint64_t red[kSmpThreads / 64];
    uint32_t red_i[kSmpThreads / 64];
    uint32_t bin;
    uint32_t before;
    uint64_t mass_before;
};

// The shortest beginning of the order that holds `want_count` tokens, or (want_count == 0) weighs `want_mass` at least; the row has it.
template <bool F32>
__device__ Prefix find_prefix(SampleLds &L, const void *row, int vocab, const RowScale &R, uint32_t want_count, uint64_t want_mass)
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
        for (int i = tid; i < kSmpBins; i += kSmpThreads) { L.count[i] = 0; L.mass[i] = 0; }
        __syncthreads();
        for (int i = tid; i < vocab; i += kSmpThreads) {
            const float x = logit_at<F32>(row, i);
            const uint32_t k = order_key(x);
            if (k == kBannedKey || (level > 0 && (k >> high) != (prefix >> high))) continue;
            const uint32_t b = (k >> shift) & (bins - 1);
            atomicAdd(&L.count[b], 1u);
            const uint64_t w = weight_of(R, x);
            if (w) atomicAdd((unsigned long long *)&L.mass[b], (unsigned long long)w);
        }
        __syncthreads();
        // two bins a thread, from the largest key down: prefix sums across the workgroup
        const int hi = kSmpBins - 1 - 2 * tid, lo = hi - 1;
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
        // exclusive sums in front of this thread's bins
        uint32_t cb = before + c - (c0 + c1);
        uint64_t mb = mass_before + m - (m0 + m1);
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
    p.mass_before = mass_before;
    const uint64_t w = weight_of(R, key_logit(prefix));
    p.ties = want_count ? want_count - before : (uint32_t)((want_mass - mass_before + w - 1) / w);
    p.mass = mass_before + p.ties * w;
    return p;
}

template <bool F32>
__global__ __launch_bounds__(kSmpThreads) void serving_sample_kernel(ServingDev S, etc_serving_sample_io io)
{
    __shared__ SampleLds L;
    __shared__ uint32_t s_id;
    const int tid = (int)threadIdx.x, r = (int)blockIdx.x, vocab = S.vocab;
    const void *row = (const char *)io.logits + (int64_t)r * io.row_stride * (F32 ? 4 : 2);
    const float T = io.temperature ? *as_global(io.temperature + r) : 1.f;
    const int top_k = io.top_k ? gld_i32(io.top_k + r) : 0;
    const float top_p = io.top_p ? *as_global(io.top_p + r) : 1.f, min_p = io.min_p ? *as_global(io.min_p + r) : 0.f;

    // the largest logit, and the tokens that are not banned
    uint32_t best = 0, live = 0;
    for (int i = tid; i < vocab; i += kSmpThreads) {
        const uint32_t k = order_key(logit_at<F32>(row, i));
        best = max(best, k);
        live += k != kBannedKey;
    }
    for (int o = 32; o > 0; o >>= 1) best = max(best, (uint32_t)__shfl_xor((int)best, o, 64));
    if (lane_id() == 0) L.red_i[wave_id()] = best;
    __syncthreads();
    for (int w = 0; w < kSmpThreads / 64; ++w) best = max(best, L.red_i[w]);
    live = wg_sum<uint32_t>(live, L.red_i);
    RowScale R{key_logit(best), 0.0};
    if (live == 0) {
        if (tid == 0) {
            *as_global(io.token_out + r) = -1;
            if (io.logprob_out) gst_f32(io.logprob_out + r, -INFINITY);
            if (io.kept_out) *as_global(io.kept_out + r) = 0;
        }
        return;
    }
    Prefix drawn{best, 1, 0, 1, 0};
    uint32_t kept = 1;
    float logprob = 0.f;
    if (T > 0.f) {
        R.inv_t = 1.0 / (double)T;
        uint32_t n_live = live;
        if (R.top == INFINITY) {                             // next to +inf the finite ones are banned
            uint32_t inf = 0;
            for (int i = tid; i < vocab; i += kSmpThreads) inf += logit_at<F32>(row, i) == INFINITY;
            n_live = wg_sum<uint32_t>(inf, L.red_i);
        }
        kept = top_k > 0 ? min((uint32_t)top_k, n_live) : n_live;
        uint64_t mass;
        if (kept < live) {
            mass = find_prefix<F32>(L, row, vocab, R, kept, 0).mass;
        } else {
            uint64_t m = 0;
            for (int i = tid; i < vocab; i += kSmpThreads) {
                const float x = logit_at<F32>(row, i);
                if (x != -INFINITY) m += weight_of(R, x);
            }
            mass = wg_sum<uint64_t>(m, L.red);
        }
        if (top_p < 1.f) {
            const double target = fmax((double)top_p, 0.0) * (double)mass;
            uint64_t want = (uint64_t)ceil(target);          // the sums are whole numbers
            want = want < 1 ? 1 : want > mass ? mass : want;
            const Prefix p = find_prefix<F32>(L, row, vocab, R, 0, want);
            kept = p.before + p.ties;
            mass = p.mass;
        }
        if (min_p > 0.f) {
            uint32_t above = 0;
            uint64_t m = 0;
            for (int i = tid; i < vocab; i += kSmpThreads) {
                const float x = logit_at<F32>(row, i);
                if (x == -INFINITY) continue;
                if (x == R.top || exp(((double)x - (double)R.top) * R.inv_t) >= (double)min_p) { above++; m += weight_of(R, x); }
            }
            above = wg_sum<uint32_t>(above, L.red_i);
            m = wg_sum<uint64_t>(m, L.red);
            if (min_p > 1.f) { above = 1; m = 1ull << 43; }
            if (above < kept) { kept = above; mass = m; }
        }
        float u = *as_global(io.u + r);
        u = u > 0.f ? fminf(u, 1.f) : 0.f;
        uint64_t want = (uint64_t)((double)u * (double)mass) + 1;      // first running sum above u * mass
        want = want > mass ? mass : want;
        drawn = find_prefix<F32>(L, row, vocab, R, 0, want);
        const float x = key_logit(drawn.key);                // from the logit, not from its weight in fixed point
        logprob = (float)((x == R.top ? 0.0 : ((double)x - (double)R.top) * R.inv_t) - log((double)mass * 0x1p-43));
    }
    // the ties-th token of the key, by id: a count in front of each thread's stretch of ids
    __syncthreads();
    const int per = (vocab + kSmpThreads - 1) / kSmpThreads, i0 = min(vocab, tid * per), i1 = min(vocab, i0 + per);
    uint32_t n = 0;
    for (int i = i0; i < i1; ++i) n += order_key(logit_at<F32>(row, i)) == drawn.key;
    uint32_t upto = (uint32_t)wave_scan_i((int)n);
    if (lane_id() == 63) L.red_i[wave_id()] = upto;
    __syncthreads();
    for (int w = 0; w < wave_id(); ++w) upto += L.red_i[w];
    uint32_t left = drawn.ties - (upto - n);                 // which of this stretch's, from 1
    if (upto - n < drawn.ties && drawn.ties <= upto) {
        int i = i0;
        for (; i < i1; ++i)
            if (order_key(logit_at<F32>(row, i)) == drawn.key && --left == 0) break;
        s_id = (uint32_t)i;
    }
    __syncthreads();
    if (tid == 0) {
        *as_global(io.token_out + r) = (int32_t)s_id;
        if (io.logprob_out) gst_f32(io.logprob_out + r, logprob);
        if (io.kept_out) *as_global(io.kept_out + r) = (int32_t)kept;
    }
}

hipError_t launch_serving_sample(const ServingDev &S, const etc_serving_sample_io &io, hipStream_t s)
{
    if (io.dtype == ETC_FP32) hipLaunchKernelGGL((serving_sample_kernel<true>), dim3(io.n_rows), dim3(kSmpThreads), 0, s, S, io);
    else hipLaunchKernelGGL((serving_sample_kernel<false>), dim3(io.n_rows), dim3(kSmpThreads), 0, s, S, io);
    return hipGetLastError();
}

}  // namespace etc
#endif  // ETC_GENERIC_ONLY
