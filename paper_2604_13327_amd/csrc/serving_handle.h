// The handle of the serving operators, and what their entry points share: errors and argument checks.
#pragma once
#include <stdio.h>

#include "serving.h"

struct etc_serving {
    etc_model_desc model{};
    etc_serving_limits limits{};
    int device = 0;
    etc::ServingDev dev{};
    void *owned[8] = {nullptr};                                 // device memory
    int n_owned = 0;
    int32_t *h_error = nullptr;                                 // pinned: a kernel's first refusal
    char err[256] = "";
};

namespace etc {

inline thread_local char t_create_error[256] = "";      // plain characters: setting an error never throws

inline etc_status fail(etc_serving *s, etc_status st, const char *msg)
{
    snprintf(s ? s->err : t_create_error, sizeof(t_create_error), "%s", msg);
    return st;
}

#define SRV_TRY(s, expr)                                                                                          \
    do {                                                                                                          \
        hipError_t e_ = (expr);                                                                                   \
        if (e_ != hipSuccess) {                                                                                   \
            char buf_[256];                                                                                       \
            snprintf(buf_, sizeof(buf_), "%s: %s", #expr, hipGetErrorString(e_));                                 \
            return fail(s, e_ == hipErrorOutOfMemory ? ETC_ENOMEM : ETC_EDEVICE, buf_);                           \
        }                                                                                                         \
    } while (0)

// What finished launches refused: reported once, then cleared.
inline etc_status report_refusals(etc_serving *s, int32_t word[4])
{
    volatile int32_t *w = s->h_error;
    for (int i = 0; i < 4; ++i) word[i] = w[i];
    if (word[0] == 0) return ETC_OK;
    for (int i = 0; i < 4; ++i) w[i] = 0;
    static const char *const ops[] = {"?", "tables", "append", "attention", "sample", "append_codes", "attention_codes", "score"};
    static const char *const what[] = {"?", "a slot outside the pool", "a length out of range", "a page id outside the pool", "a token outside the vocabulary"};
    char buf[200];
    snprintf(buf, sizeof(buf), "an earlier launch refused %s (etc_serving_%s, index %d, value %d)", what[word[0] >= 1 && word[0] <= 4 ? word[0] : 0],
             ops[word[1] >= 1 && word[1] <= 7 ? word[1] : 0], word[2], word[3]);
    return fail(s, ETC_ETIMEOUT, buf);
}

// Every call: a handle, its device current, and nothing refused by an earlier launch.
inline etc_status enter(etc_serving *s, const void *io)
{
    if (!s || !io) return fail(s, ETC_EINVAL, "NULL argument");
    int dev = -1;
    SRV_TRY(s, hipGetDevice(&dev));
    if (dev != s->device) return fail(s, ETC_EINVAL, "the current device is not the one the handle was created on");
    int32_t w[4];
    return report_refusals(s, w);
}

inline bool off16(const void *p) { return ((uintptr_t)p & 15) != 0; }
inline bool off4(const void *p) { return ((uintptr_t)p & 3) != 0; }

inline const char *check_pool(const etc_serving *s, const void *k, const void *v, int64_t n_pages)
{
    if (!k || !v || off16(k) || off16(v)) return "the pools must be given, 16-byte aligned";
    if (n_pages < 1 || n_pages > INT32_MAX / s->model.page_size) return "n_pages must be positive, n_pages * page_size below 2^31";
    return nullptr;
}

inline const char *check_table(const int32_t *table, int64_t stride, int32_t cols)
{
    if (!table || off4(table)) return "block_table is NULL or not aligned";
    if (cols < 1 || stride < cols) return "table_cols must be positive, table_stride at least table_cols";
    return nullptr;
}

// The arguments that operators over pools of either type have in common; NULL, or what is wrong.
inline const char *check_append(const etc_serving *s, const etc_serving_append_io *io)
{
    if (io->n_tokens < 0 || io->n_tokens > s->limits.max_tokens) return "n_tokens out of range 0..max_tokens";
    if (io->n_tokens == 0) return nullptr;
    if (io->dtype != ETC_BF16 && io->dtype != ETC_FP32) return "dtype must be ETC_BF16 or ETC_FP32";
    const int size = io->dtype == ETC_FP32 ? 4 : 2;
    const int64_t qw = (int64_t)s->model.n_q_heads * s->model.head_dim, kw = (int64_t)s->model.n_kv_heads * s->model.head_dim;
    const void *rows[] = {io->q, io->k, io->v, io->q_out};
    for (const void *p : rows)
        if (!p || off16(p)) return "q, k, v, q_out must be given, 16-byte aligned";
    const int64_t strides[] = {io->q_stride, io->k_stride, io->v_stride};
    for (int i = 0; i < 3; ++i)
        if (strides[i] < (i ? kw : qw) || strides[i] * size % 16 || strides[i] > ((int64_t)1 << 32))
            return "a row stride is smaller than its row, or no multiple of 16 bytes";
    if (io->q_out == io->q && (io->dtype != ETC_BF16 || io->q_stride != qw)) return "q_out may be q for bf16 rows without gaps only";
    if (!io->positions || !io->slots || off4(io->positions) || off4(io->slots)) return "positions or slots missing or not aligned";
    if (s->model.qk_norm ? (!io->gq || !io->gk || off16(io->gq) || off16(io->gk)) : (io->gq || io->gk))
        return "gq and gk, 16-byte aligned, belong to models with per-head norms, and only to those";
    if (const char *e = check_pool(s, io->k_pages, io->v_pages, io->n_pages)) return e;
    return nullptr;
}

inline const char *check_attention(const etc_serving *s, const etc_serving_attention_io *io)
{
    if (io->n_seqs < 1 || io->n_seqs > s->limits.max_seqs) return "n_seqs out of range 1..max_seqs";
    if (io->n_tokens < 0 || io->n_tokens > s->limits.max_tokens) return "n_tokens out of range 0..max_tokens";
    if (io->n_tokens == 0) return nullptr;
    if (!io->q || !io->out || off16(io->q) || off16(io->out) || io->q == io->out) return "q and out must be given, 16-byte aligned, and differ";
    if (!io->q_indptr || !io->kv_len || off4(io->q_indptr) || off4(io->kv_len)) return "q_indptr or kv_len missing or not aligned";
    if (const char *e = check_table(io->block_table, io->table_stride, io->table_cols)) return e;
    if (const char *e = check_pool(s, io->k_pages, io->v_pages, io->n_pages)) return e;
    return nullptr;
}

}  // namespace etc
