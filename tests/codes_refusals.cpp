// What the entry points of the cache of codes and of the scores refuse, on the CPU: the library's argument checks over a runtime of stubs
// that counts launches.  A refused call launches nothing and leaves a text; a good one launches once.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "serving.cpp"
#include "serving_codes.cpp"

static int g_launches = 0, g_device = 0;
extern "C" {
hipError_t hipGetDevice(int *d) { *d = g_device; return hipSuccess; }
hipError_t hipSetDevice(int d) { g_device = d; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n) { *p = malloc(n < 64 ? 64 : n); return hipSuccess; }
hipError_t hipFree(void *p) { free(p); return hipSuccess; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { *p = malloc(n); return hipSuccess; }
hipError_t hipHostFree(void *p) { free(p); return hipSuccess; }
hipError_t hipHostGetDevicePointer(void **d, void *h, unsigned) { *d = h; return hipSuccess; }
hipError_t hipMemset(void *p, int v, size_t n) { if (n < (1u << 20)) memset(p, v, n); return hipSuccess; }
hipError_t hipMemcpy(void *d, const void *s, size_t n, hipMemcpyKind) { memcpy(d, s, n); return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "stub"; }
}
namespace etc {
int64_t attention_slot_bytes(int) { return 64; }
int64_t sample_slices(int, int) { return 4; }
int64_t sample_stat_bytes() { return 16; }
int64_t sample_bins_bytes() { return 64; }
hipError_t launch_serving_tables(const ServingDev &, const etc_serving_tables_io &, hipStream_t) { return hipSuccess; }
hipError_t launch_serving_append(const ServingDev &, const etc_serving_append_io &, hipStream_t) { return hipSuccess; }
hipError_t launch_serving_attention(const ServingDev &, const etc_serving_attention_io &, hipStream_t) { return hipSuccess; }
hipError_t launch_serving_sample(const ServingDev &, const etc_serving_sample_io &, hipStream_t) { return hipSuccess; }
hipError_t launch_serving_append_codes(const ServingDev &, const etc_serving_append_codes_io &, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_serving_attention_codes(const ServingDev &, const etc_serving_attention_codes_io &, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_serving_score(const ServingDev &, const etc_serving_score_io &, hipStream_t) { ++g_launches; return hipSuccess; }
}  // namespace etc

#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)
// `change` applied to a good call is refused; the good call itself is taken.
#define REFUSED(call, io_t, good, change)                                                           \
    do {                                                                                            \
        io_t x = good;                                                                              \
        change;                                                                                     \
        const int before = g_launches;                                                              \
        CHECK(call(s, &x, nullptr) == ETC_EINVAL && g_launches == before && etc_serving_last_error(s)[0]); \
        CHECK(call(s, &good, nullptr) == ETC_OK && g_launches == before + 1);                       \
    } while (0)
// ... and one that has nothing to do is taken without a launch.
#define NOTHING(call, io_t, good, change)                                                           \
    do {                                                                                            \
        io_t x = good;                                                                              \
        change;                                                                                     \
        const int before = g_launches;                                                              \
        CHECK(call(s, &x, nullptr) == ETC_OK && g_launches == before);                              \
    } while (0)

int main()
{
    etc_model_desc m{};
    m.n_q_heads = 8; m.n_kv_heads = 2; m.head_dim = 128; m.page_size = 16; m.rms_eps = 1e-5f; m.rope_theta = 1e4f; m.vocab = 1000;
    const etc_serving_limits l{4, 100, 500};
    etc_serving *s = nullptr;
    CHECK(etc_serving_create(&m, &l, &s) == ETC_OK && s);
    alignas(16) static char mem[4096];
    int32_t *i32 = (int32_t *)mem;
    float *f32 = (float *)mem;

    etc_serving_append_codes_io a{};
    a.append.n_tokens = 100; a.append.dtype = ETC_BF16; a.append.q = a.append.k = a.append.v = mem; a.append.q_stride = 1024;
    a.append.k_stride = a.append.v_stride = 256; a.append.positions = a.append.slots = i32; a.append.q_out = mem + 16;
    a.append.k_pages = a.append.v_pages = mem; a.append.n_pages = 10; a.k_scale = a.v_scale = mem + 1;
#define A(change) REFUSED(etc_serving_append_codes, etc_serving_append_codes_io, a, change)
    A(x.append.n_tokens = -1); A(x.append.n_tokens = 101); A(x.append.dtype = 2); A(x.append.q = nullptr); A(x.append.k = mem + 2); A(x.append.v = nullptr);
    A(x.append.q_out = nullptr); A(x.append.q_stride = 1023); A(x.append.k_stride = 248); A(x.append.v_stride = 1ll << 40); A(x.append.positions = nullptr);
    A(x.append.slots = (int32_t *)(mem + 2)); A(x.append.gq = mem); A(x.append.k_pages = nullptr); A(x.append.v_pages = mem + 4); A(x.append.n_pages = 0);
    A(x.append.n_pages = 1ll << 27); A(x.k_scale = nullptr); A(x.v_scale = nullptr);
    NOTHING(etc_serving_append_codes, etc_serving_append_codes_io, a, x.append.n_tokens = 0);

    etc_serving_attention_codes_io n{};
    n.attention.n_seqs = 4; n.attention.n_tokens = 100; n.attention.q = mem; n.attention.out = mem + 16;
    n.attention.q_indptr = n.attention.kv_len = n.attention.block_table = i32; n.attention.table_stride = n.attention.table_cols = 8;
    n.attention.k_pages = n.attention.v_pages = mem; n.attention.n_pages = 10; n.k_scale = n.v_scale = mem + 3;
#define N(change) REFUSED(etc_serving_attention_codes, etc_serving_attention_codes_io, n, change)
    N(x.attention.n_seqs = 0); N(x.attention.n_seqs = 5); N(x.attention.n_tokens = 101); N(x.attention.n_tokens = -1); N(x.attention.q = nullptr);
    N(x.attention.out = (void *)x.attention.q); N(x.attention.q = mem + 4); N(x.attention.q_indptr = nullptr); N(x.attention.kv_len = nullptr);
    N(x.attention.block_table = nullptr); N(x.attention.table_cols = 9); N(x.attention.k_pages = nullptr); N(x.attention.v_pages = mem + 8);
    N(x.attention.n_pages = -1); N(x.k_scale = nullptr); N(x.v_scale = nullptr);
    NOTHING(etc_serving_attention_codes, etc_serving_attention_codes_io, n, x.attention.n_tokens = 0);

    etc_serving_score_io p{};
    p.n_rows = 100; p.dtype = ETC_FP32; p.logits = mem; p.row_stride = 1000; p.tokens = i32; p.logprob_out = f32; p.entropy_out = f32; p.n_top = 64;
    p.top_ids = i32; p.top_logprobs = f32;
#define P(change) REFUSED(etc_serving_score, etc_serving_score_io, p, change)
    P(x.n_rows = -1); P(x.n_rows = 101); P(x.dtype = -1); P(x.logits = nullptr); P(x.logits = mem + 2); P((x.logits = mem + 1, x.dtype = ETC_BF16));
    P(x.row_stride = 999); P(x.row_stride = 1ll << 33); P(x.tokens = nullptr); P(x.logprob_out = nullptr); P(x.n_top = 65); P(x.n_top = -1); P(x.n_top = 0);
    P(x.top_ids = nullptr); P((x.top_ids = nullptr, x.n_top = 0)); P(x.entropy_out = (float *)(mem + 2)); P(x.top_logprobs = (float *)(mem + 1));
    P((x.tokens = nullptr, x.logprob_out = nullptr, x.entropy_out = nullptr, x.n_top = 0, x.top_ids = nullptr, x.top_logprobs = nullptr));
    NOTHING(etc_serving_score, etc_serving_score_io, p, x.n_rows = 0);
    {
        etc_serving_score_io x = p;
        const int before = g_launches;
        x.tokens = nullptr; x.logprob_out = nullptr; x.top_logprobs = nullptr;
        CHECK(etc_serving_score(s, &x, nullptr) == ETC_OK && g_launches == before + 1);
    }

    // NULL, another device, earlier refusals on the device
    CHECK(etc_serving_append_codes(nullptr, &a, nullptr) == ETC_EINVAL && etc_serving_score(s, nullptr, nullptr) == ETC_EINVAL);
    CHECK(etc_serving_last_error(nullptr)[0]);
    const int before = g_launches;
    g_device = 1;
    CHECK(etc_serving_attention_codes(s, &n, nullptr) == ETC_EINVAL && etc_serving_append_codes(s, &a, nullptr) == ETC_EINVAL && g_launches == before);
    g_device = 0;
    s->h_error[0] = SRV_BAD_TOKEN; s->h_error[1] = SRV_SCORE; s->h_error[2] = 3; s->h_error[3] = 77777;
    CHECK(etc_serving_append_codes(s, &a, nullptr) == ETC_ETIMEOUT && g_launches == before);
    CHECK(strstr(etc_serving_last_error(s), "token") && strstr(etc_serving_last_error(s), "77777") && strstr(etc_serving_last_error(s), "etc_serving_score"));
    s->h_error[0] = SRV_BAD_SLOT; s->h_error[1] = SRV_APPEND_CODES;
    int32_t w[4];
    CHECK(etc_serving_read_error(s, w) == ETC_ETIMEOUT && strstr(etc_serving_last_error(s), "etc_serving_append_codes"));
    CHECK(etc_serving_append_codes(s, &a, nullptr) == ETC_OK && g_launches == before + 1);
    etc_serving_destroy(s);
    m.vocab = 0;
    CHECK(etc_serving_create(&m, &l, &s) == ETC_OK);
    CHECK(etc_serving_score(s, &p, nullptr) == ETC_ESTATE);
    etc_serving_destroy(s);
    puts("ok");
    return 0;
}
