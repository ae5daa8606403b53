// C ABI of the serving operators (include/etc.h, etc_serving_*): argument checks, the handle and its workspace.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>
#include <vector>

#include "serving_handle.h"

using namespace etc;

#ifdef ETC_GENERIC_ONLY      // a library generated for one graph has no kernels of these; no handle is ever made there
namespace etc {
int64_t attention_slot_bytes(int) { return 0; }
int64_t sample_slices(int, int) { return 0; }
int64_t sample_stat_bytes() { return 0; }
int64_t sample_bins_bytes() { return 0; }
hipError_t launch_serving_tables(const ServingDev &, const etc_serving_tables_io &, hipStream_t) { return hipErrorInvalidDeviceFunction; }
hipError_t launch_serving_append(const ServingDev &, const etc_serving_append_io &, hipStream_t) { return hipErrorInvalidDeviceFunction; }
hipError_t launch_serving_attention(const ServingDev &, const etc_serving_attention_io &, hipStream_t) { return hipErrorInvalidDeviceFunction; }
hipError_t launch_serving_sample(const ServingDev &, const etc_serving_sample_io &, hipStream_t) { return hipErrorInvalidDeviceFunction; }
}  // namespace etc
#endif

namespace {

template <class T>
hipError_t owned_alloc(etc_serving *s, T **p, size_t n, bool zero = true)
{
    hipError_t e = hipMalloc((void **)p, n * sizeof(T));
    if (e != hipSuccess) return e;
    s->owned[s->n_owned++] = *p;
    return zero ? hipMemset(*p, 0, n * sizeof(T)) : hipSuccess;
}

}  // namespace

extern "C" {

const char *etc_serving_last_error(const etc_serving *s) { return s ? s->err : t_create_error; }

void etc_serving_destroy(etc_serving *s)
{
    if (!s) return;
    int dev = -1;
    const bool other = hipGetDevice(&dev) == hipSuccess && dev != s->device;
    if (other) (void)hipSetDevice(s->device);
    (void)hipDeviceSynchronize();
    for (int i = 0; i < s->n_owned; ++i) (void)hipFree(s->owned[i]);
    if (s->h_error) (void)hipHostFree(s->h_error);
    if (other) (void)hipSetDevice(dev);
    delete s;
}

etc_status etc_serving_create(const etc_model_desc *m, const etc_serving_limits *l, etc_serving **out)
{
    if (!m || !l || !out) return fail(nullptr, ETC_EINVAL, "NULL argument");
    *out = nullptr;
#ifdef ETC_GENERIC_ONLY
    return fail(nullptr, ETC_ESTATE, "a library generated for one graph has no serving operators");
#else
    if (m->n_q_heads < 1 || m->n_kv_heads < 1 || m->n_q_heads % m->n_kv_heads || m->n_q_heads / m->n_kv_heads > 64 || m->n_q_heads > 1024)
        return fail(nullptr, ETC_EINVAL, "n_q_heads (<= 1024) must be 1 to 64 times n_kv_heads");
    if (m->head_dim != 64 && m->head_dim != 128) return fail(nullptr, ETC_EINVAL, "head_dim must be 64 or 128");
    if (m->page_size < 1 || (m->page_size & (m->page_size - 1))) return fail(nullptr, ETC_EINVAL, "page_size must be a power of two");
    if (!(m->rms_eps >= 0.f) || !(m->rope_theta > 0.f)) return fail(nullptr, ETC_EINVAL, "rms_eps must not be negative, rope_theta positive");
    if (m->vocab < 0 || m->vocab > kServingMaxVocab) return fail(nullptr, ETC_EINVAL, "vocab must be in 0..2^20");
    if (l->max_seqs < 1 || l->max_seqs > kServingMaxSeqs) return fail(nullptr, ETC_EINVAL, "max_seqs must be in 1..1024");
    if (l->max_tokens < 1 || l->max_tokens > kServingMaxTokens) return fail(nullptr, ETC_EINVAL, "max_tokens must be in 1..2^20");
    if (l->max_kv_len < 1 || l->max_kv_len > kServingMaxKv) return fail(nullptr, ETC_EINVAL, "max_kv_len must be in 1..2^30");
    etc_serving *s = new (std::nothrow) etc_serving();
    if (!s) return fail(nullptr, ETC_ENOMEM, "out of host memory");
    s->model = *m;
    s->limits = *l;
    auto set_up = [&]() -> etc_status {
        ServingDev &D = s->dev;
        SRV_TRY(s, hipGetDevice(&s->device));
        SRV_TRY(s, hipDeviceGetAttribute(&D.n_cus, hipDeviceAttributeMultiprocessorCount, s->device));
        D.nq = m->n_q_heads; D.nkv = m->n_kv_heads; D.d = m->head_dim; D.qk_norm = m->qk_norm ? 1 : 0; D.vocab = m->vocab;
        D.eps = m->rms_eps; D.max_kv_len = l->max_kv_len;
        while ((1 << D.page_shift) < m->page_size) ++D.page_shift;
        SRV_TRY(s, hipHostMalloc((void **)&s->h_error, 4 * sizeof(int32_t), hipHostMallocMapped));
        memset(s->h_error, 0, 4 * sizeof(int32_t));
        SRV_TRY(s, hipHostGetDevicePointer((void **)&D.error, s->h_error, 0));
        SRV_TRY(s, owned_alloc(s, &D.arrive, (size_t)kTakenApart + 8 * kTakenApart));
        D.taken = D.arrive + kTakenApart;
        D.attn_slots = attention_slots(m->n_q_heads, m->n_kv_heads, *l);
        if (D.attn_slots > 0) {
            SRV_TRY(s, owned_alloc(s, &D.attn_arrive, (size_t)D.attn_slots));
            SRV_TRY(s, owned_alloc(s, (char **)&D.attn_part, (size_t)D.attn_slots * attention_slot_bytes(m->head_dim), false));
        }
        if (m->vocab > 0) {
            const size_t n = (size_t)sample_slices(m->vocab, l->max_seqs);
            if (n > 0) {
                SRV_TRY(s, owned_alloc(s, (char **)&D.smp_stats, n * (size_t)sample_stat_bytes(), false));
                SRV_TRY(s, owned_alloc(s, (char **)&D.smp_bins, n * (size_t)sample_bins_bytes(), false));
                SRV_TRY(s, owned_alloc(s, &D.smp_listed, (size_t)kSampleSharedRows * (2 + kSampleList) + (size_t)kScoreRows * kScoreApart));
                D.smp_done = D.smp_listed + kSampleSharedRows;
                D.smp_list = D.smp_done + kSampleSharedRows;
                D.score_arrived = D.smp_list + (size_t)kSampleSharedRows * kSampleList;
            }
        }
        double inv[64], *d_inv = nullptr;
        for (int i = 0; i < m->head_dim / 2; ++i) inv[i] = pow((double)m->rope_theta, -2.0 * i / m->head_dim);
        SRV_TRY(s, owned_alloc(s, &d_inv, m->head_dim / 2));
        SRV_TRY(s, hipMemcpy(d_inv, inv, sizeof(double) * (m->head_dim / 2), hipMemcpyHostToDevice));
        D.inv_freq = d_inv;
        return ETC_OK;
    };
    const etc_status st = set_up();
    if (st != ETC_OK) {
        snprintf(t_create_error, sizeof(t_create_error), "%s", s->err);
        etc_serving_destroy(s);
        return st;
    }
    *out = s;
    return ETC_OK;
#endif
}

etc_status etc_serving_read_error(etc_serving *s, int32_t word[4])
{
    if (!s || !word) return fail(s, ETC_EINVAL, "NULL argument");
    int dev = -1;
    SRV_TRY(s, hipGetDevice(&dev));
    if (dev != s->device) SRV_TRY(s, hipSetDevice(s->device));      // whose launches the word is about
    const hipError_t synchronized = hipDeviceSynchronize();
    if (dev != s->device) SRV_TRY(s, hipSetDevice(dev));
    SRV_TRY(s, synchronized);
    return report_refusals(s, word);
}

etc_status etc_serving_tables(etc_serving *s, const etc_serving_tables_io *io, void *hip_stream)
{
    etc_status st = enter(s, io);
    if (st != ETC_OK) return st;
    if (io->n_seqs < 1 || io->n_seqs > s->limits.max_seqs) return fail(s, ETC_EINVAL, "n_seqs out of range 1..max_seqs");
    if (io->n_tokens < 0 || io->n_tokens > s->limits.max_tokens) return fail(s, ETC_EINVAL, "n_tokens out of range 0..max_tokens");
    if (!io->kv_len || !io->new_len || !io->free_count || !io->free_count_out || !io->q_indptr || !io->status ||
        (io->n_tokens > 0 && (!io->slots || !io->positions)))
        return fail(s, ETC_EINVAL, "an array is NULL");
    if (const char *e = check_table(io->block_table, io->table_stride, io->table_cols)) return fail(s, ETC_EINVAL, e);
    if (io->free_cap < 0 || (io->free_cap > 0 && !io->free_pages)) return fail(s, ETC_EINVAL, "free_pages is NULL or its size negative");
    if (io->page_ids_cap < 0 || (io->page_ids && !io->page_indptr) || (!io->page_ids && io->page_ids_cap > 0))
        return fail(s, ETC_EINVAL, "page_indptr and page_ids go together");
    const void *ints[] = {io->kv_len, io->new_len, io->free_pages, io->free_count, io->free_count_out, io->q_indptr, io->slots,
                          io->positions, io->total_len, io->page_indptr, io->page_ids, io->status};
    for (const void *p : ints)
        if (off4(p)) return fail(s, ETC_EINVAL, "an array is not aligned");
    SRV_TRY(s, launch_serving_tables(s->dev, *io, (hipStream_t)hip_stream));
    return ETC_OK;
}

etc_status etc_serving_append(etc_serving *s, const etc_serving_append_io *io, void *hip_stream)
{
    etc_status st = enter(s, io);
    if (st != ETC_OK) return st;
    if (const char *e = check_append(s, io)) return fail(s, ETC_EINVAL, e);
    if (io->n_tokens == 0) return ETC_OK;
    SRV_TRY(s, launch_serving_append(s->dev, *io, (hipStream_t)hip_stream));
    return ETC_OK;
}

etc_status etc_serving_attention(etc_serving *s, const etc_serving_attention_io *io, void *hip_stream)
{
    etc_status st = enter(s, io);
    if (st != ETC_OK) return st;
    if (const char *e = check_attention(s, io)) return fail(s, ETC_EINVAL, e);
    if (io->n_tokens == 0) return ETC_OK;
    SRV_TRY(s, launch_serving_attention(s->dev, *io, (hipStream_t)hip_stream));
    return ETC_OK;
}

etc_status etc_serving_sample(etc_serving *s, const etc_serving_sample_io *io, void *hip_stream)
{
    etc_status st = enter(s, io);
    if (st != ETC_OK) return st;
    if (s->model.vocab < 1) return fail(s, ETC_ESTATE, "the model has no vocabulary");
    if (io->n_rows < 1 || io->n_rows > s->limits.max_seqs) return fail(s, ETC_EINVAL, "n_rows out of range 1..max_seqs");
    if (io->dtype != ETC_BF16 && io->dtype != ETC_FP32) return fail(s, ETC_EINVAL, "dtype must be ETC_BF16 or ETC_FP32");
    if (!io->logits || ((uintptr_t)io->logits & (io->dtype == ETC_FP32 ? 3 : 1))) return fail(s, ETC_EINVAL, "logits missing or not aligned");
    if (io->row_stride < s->model.vocab || io->row_stride > ((int64_t)1 << 32)) return fail(s, ETC_EINVAL, "row_stride must be vocab at least");
    if (!io->u || !io->token_out) return fail(s, ETC_EINVAL, "u or token_out is NULL");
    const void *words[] = {io->u, io->temperature, io->top_k, io->top_p, io->min_p, io->token_out, io->logprob_out, io->kept_out};
    for (const void *p : words)
        if (off4(p)) return fail(s, ETC_EINVAL, "an array is not aligned");
    SRV_TRY(s, launch_serving_sample(s->dev, *io, (hipStream_t)hip_stream));
    return ETC_OK;
}

}  // extern "C"
