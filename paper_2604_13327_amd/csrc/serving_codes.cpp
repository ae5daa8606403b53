// C ABI of the operators over a cache of 8 bits and of the scores (include/etc.h): argument checks.
#include "serving_handle.h"

using namespace etc;

#ifdef ETC_GENERIC_ONLY      // a library generated for one graph has no kernels of these; no handle is ever made there
namespace etc {
hipError_t launch_serving_append_codes(const ServingDev &, const etc_serving_append_codes_io &, hipStream_t) { return hipErrorInvalidDeviceFunction; }
hipError_t launch_serving_attention_codes(const ServingDev &, const etc_serving_attention_codes_io &, hipStream_t) { return hipErrorInvalidDeviceFunction; }
hipError_t launch_serving_score(const ServingDev &, const etc_serving_score_io &, hipStream_t) { return hipErrorInvalidDeviceFunction; }
}  // namespace etc
#endif

extern "C" {

etc_status etc_serving_append_codes(etc_serving *s, const etc_serving_append_codes_io *io, void *hip_stream)
{
    etc_status st = enter(s, io);
    if (st != ETC_OK) return st;
    if (const char *e = check_append(s, &io->append)) return fail(s, ETC_EINVAL, e);
    if (io->append.n_tokens == 0) return ETC_OK;
    if (!io->k_scale || !io->v_scale) return fail(s, ETC_EINVAL, "k_scale or v_scale is NULL");
    SRV_TRY(s, launch_serving_append_codes(s->dev, *io, (hipStream_t)hip_stream));
    return ETC_OK;
}

etc_status etc_serving_attention_codes(etc_serving *s, const etc_serving_attention_codes_io *io, void *hip_stream)
{
    etc_status st = enter(s, io);
    if (st != ETC_OK) return st;
    if (const char *e = check_attention(s, &io->attention)) return fail(s, ETC_EINVAL, e);
    if (io->attention.n_tokens == 0) return ETC_OK;
    if (!io->k_scale || !io->v_scale) return fail(s, ETC_EINVAL, "k_scale or v_scale is NULL");
    SRV_TRY(s, launch_serving_attention_codes(s->dev, *io, (hipStream_t)hip_stream));
    return ETC_OK;
}

etc_status etc_serving_score(etc_serving *s, const etc_serving_score_io *io, void *hip_stream)
{
    etc_status st = enter(s, io);
    if (st != ETC_OK) return st;
    if (s->model.vocab < 1) return fail(s, ETC_ESTATE, "the model has no vocabulary");
    if (io->n_rows < 0 || io->n_rows > s->limits.max_tokens) return fail(s, ETC_EINVAL, "n_rows out of range 0..max_tokens");
    if (io->dtype != ETC_BF16 && io->dtype != ETC_FP32) return fail(s, ETC_EINVAL, "dtype must be ETC_BF16 or ETC_FP32");
    if (io->n_top < 0 || io->n_top > kScoreTop) return fail(s, ETC_EINVAL, "n_top must be in 0..64");
    if (io->n_rows == 0) return ETC_OK;
    if (!io->logits || ((uintptr_t)io->logits & (io->dtype == ETC_FP32 ? 3 : 1))) return fail(s, ETC_EINVAL, "logits missing or not aligned");
    if (io->row_stride < s->model.vocab || io->row_stride > ((int64_t)1 << 32)) return fail(s, ETC_EINVAL, "row_stride must be vocab at least");
    if ((io->tokens == nullptr) != (io->logprob_out == nullptr)) return fail(s, ETC_EINVAL, "tokens and logprob_out go together");
    if ((io->n_top > 0) != (io->top_ids != nullptr) || (io->top_logprobs && !io->top_ids)) return fail(s, ETC_EINVAL, "n_top and top_ids go together, top_logprobs with them");
    if (!io->logprob_out && !io->entropy_out && !io->top_ids) return fail(s, ETC_EINVAL, "nothing is asked for");
    const void *words[] = {io->tokens, io->logprob_out, io->entropy_out, io->top_ids, io->top_logprobs};
    for (const void *p : words)
        if (off4(p)) return fail(s, ETC_EINVAL, "an array is not aligned");
    SRV_TRY(s, launch_serving_score(s->dev, *io, (hipStream_t)hip_stream));
    return ETC_OK;
}

}  // extern "C"
