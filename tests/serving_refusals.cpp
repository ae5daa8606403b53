// What the serving entry points refuse, on the CPU: the library's argument checks (serving.cpp) over a runtime of stubs that
// counts launches.  A refused call launches nothing and leaves a text; a good one launches once.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "serving.cpp"

static int g_launches = 0, g_device = 0, g_fail_malloc = -1, g_allocs = 0;
extern "C" {
hipError_t hipGetDevice(int *d) { *d = g_device; return hipSuccess; }
hipError_t hipSetDevice(int d) { g_device = d; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n)
{
    if (g_fail_malloc-- == 0) return hipErrorOutOfMemory;
    *p = malloc(n < 64 ? 64 : n);
    ++g_allocs;
    return hipSuccess;
}
hipError_t hipFree(void *p) { free(p); --g_allocs; return hipSuccess; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { *p = malloc(n); ++g_allocs; return hipSuccess; }
hipError_t hipHostFree(void *p) { free(p); --g_allocs; return hipSuccess; }
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
hipError_t launch_serving_tables(const ServingDev &, const etc_serving_tables_io &, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_serving_append(const ServingDev &, const etc_serving_append_io &, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_serving_attention(const ServingDev &, const etc_serving_attention_io &, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_serving_sample(const ServingDev &, const etc_serving_sample_io &, hipStream_t) { ++g_launches; return hipSuccess; }
}  // namespace etc

#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)
// `change` applied to a good call is refused; the good call itself is taken.
#define REFUSED(call, io_t, good, status, change)                                                   \
    do {                                                                                            \
        io_t x = good;                                                                              \
        change;                                                                                     \
        const int before = g_launches;                                                              \
        CHECK(call(s, &x, nullptr) == status && g_launches == before && etc_serving_last_error(s)[0]); \
        CHECK(call(s, &good, nullptr) == ETC_OK && g_launches == before + 1);                       \
    } while (0)

int main()
{
    etc_model_desc m{};
    m.n_q_heads = 8; m.n_kv_heads = 2; m.head_dim = 128; m.page_size = 16; m.rms_eps = 1e-5f; m.rope_theta = 1e4f; m.vocab = 1000;
    const etc_serving_limits l{4, 100, 500};
    etc_serving *s = nullptr;
    {   // descriptors
        auto bad = [&](auto change) {
            etc_model_desc mm = m;
            etc_serving_limits ll = l;
            change(mm, ll);
            etc_serving *none = (etc_serving *)8;
            return etc_serving_create(&mm, &ll, &none) == ETC_EINVAL && none == nullptr && etc_serving_last_error(nullptr)[0];
        };
        typedef etc_model_desc &M;
        typedef etc_serving_limits &L;
        CHECK(bad([](M a, L) { a.head_dim = 96; }));
        CHECK(bad([](M a, L) { a.n_q_heads = 7; }));
        CHECK(bad([](M a, L) { a.n_kv_heads = 0; }));
        CHECK(bad([](M a, L) { a.n_q_heads = 130; a.n_kv_heads = 2; }));
        CHECK(bad([](M a, L) { a.page_size = 24; }));
        CHECK(bad([](M a, L) { a.page_size = 0; }));
        CHECK(bad([](M a, L) { a.rope_theta = 0.f; }));
        CHECK(bad([](M a, L) { a.rms_eps = -1.f; }));
        CHECK(bad([](M a, L) { a.vocab = (1 << 20) + 1; }));
        CHECK(bad([](M a, L) { a.vocab = -1; }));
        CHECK(bad([](M, L b) { b.max_seqs = 0; }));
        CHECK(bad([](M, L b) { b.max_seqs = 1025; }));
        CHECK(bad([](M, L b) { b.max_tokens = 0; }));
        CHECK(bad([](M, L b) { b.max_tokens = (1 << 20) + 1; }));
        CHECK(bad([](M, L b) { b.max_kv_len = 0; }));
        CHECK(etc_serving_create(nullptr, &l, &s) == ETC_EINVAL && etc_serving_create(&m, nullptr, &s) == ETC_EINVAL);
        CHECK(etc_serving_create(&m, &l, nullptr) == ETC_EINVAL);
        for (int k = 0; k < 7; ++k) {                     // no memory: everything is given back
            g_fail_malloc = k;
            CHECK(etc_serving_create(&m, &l, &s) == ETC_ENOMEM && s == nullptr && g_allocs == 0 && etc_serving_last_error(nullptr)[0]);
            g_fail_malloc = -1;
        }
    }
    CHECK(etc_serving_create(&m, &l, &s) == ETC_OK && s);
    alignas(16) static char mem[4096];
    int32_t *i32 = (int32_t *)mem;

    etc_serving_tables_io t{};
    t.n_seqs = 4; t.n_tokens = 100; t.kv_len = t.new_len = i32; t.block_table = i32; t.table_stride = 8; t.table_cols = 8; t.free_pages = i32;
    t.free_cap = 3; t.free_count = i32; t.free_count_out = i32; t.q_indptr = t.slots = t.positions = t.status = i32;
#define T(change) REFUSED(etc_serving_tables, etc_serving_tables_io, t, ETC_EINVAL, change)
    T(x.n_seqs = 0); T(x.n_seqs = 5); T(x.n_tokens = -1); T(x.n_tokens = 101); T(x.kv_len = nullptr); T(x.new_len = nullptr);
    T(x.block_table = nullptr); T(x.table_cols = 0); T(x.table_stride = 7); T(x.free_cap = -1); T(x.free_pages = nullptr);
    T(x.free_count = nullptr); T(x.free_count_out = nullptr); T(x.q_indptr = nullptr); T(x.slots = nullptr); T(x.positions = nullptr);
    T(x.status = nullptr); T(x.page_ids = i32); T((x.page_indptr = i32, x.page_ids_cap = 2)); T((x.page_indptr = x.page_ids = i32, x.page_ids_cap = -2));
    T(x.kv_len = (int32_t *)(mem + 2)); T(x.total_len = (int32_t *)(mem + 1));

    etc_serving_append_io a{};
    a.n_tokens = 100; a.dtype = ETC_BF16; a.q = a.k = a.v = mem; a.q_stride = 1024; a.k_stride = a.v_stride = 256; a.positions = a.slots = i32;
    a.q_out = mem + 16; a.k_pages = a.v_pages = mem; a.n_pages = 10;
#define A(change) REFUSED(etc_serving_append, etc_serving_append_io, a, ETC_EINVAL, change)
    A(x.n_tokens = -1); A(x.n_tokens = 101); A(x.dtype = 2); A(x.q = nullptr); A(x.k = nullptr); A(x.v = nullptr); A(x.q_out = nullptr);
    A(x.q = mem + 8); A(x.v = mem + 2); A(x.q_stride = 1023); A(x.q_stride = 1028); A(x.k_stride = 248); A(x.v_stride = 1ll << 40);
    A((x.q_out = (void *)x.q, x.q_stride = 1032)); A((x.q_out = (void *)x.q, x.dtype = ETC_FP32)); A(x.positions = nullptr); A(x.slots = nullptr);
    A(x.gq = mem); A(x.gk = mem); A(x.k_pages = nullptr); A(x.v_pages = mem + 4); A(x.n_pages = 0); A(x.n_pages = 1ll << 27);
    {
        etc_serving_append_io x = a;
        const int before = g_launches;
        x.q_out = (void *)x.q;
        CHECK(etc_serving_append(s, &x, nullptr) == ETC_OK && g_launches == before + 1);      // in place
        x.n_tokens = 0;
        CHECK(etc_serving_append(s, &x, nullptr) == ETC_OK && g_launches == before + 1);      // nothing to do
    }

    etc_serving_attention_io n{};
    n.n_seqs = 4; n.n_tokens = 100; n.q = mem; n.out = mem + 16; n.q_indptr = n.kv_len = n.block_table = i32; n.table_stride = n.table_cols = 8;
    n.k_pages = n.v_pages = mem; n.n_pages = 10;
#define N(change) REFUSED(etc_serving_attention, etc_serving_attention_io, n, ETC_EINVAL, change)
    N(x.n_seqs = 0); N(x.n_seqs = 5); N(x.n_tokens = 101); N(x.n_tokens = -1); N(x.q = nullptr); N(x.out = nullptr); N(x.out = (void *)x.q);
    N(x.q = mem + 4); N(x.q_indptr = nullptr); N(x.kv_len = nullptr); N(x.block_table = nullptr); N(x.table_cols = 9); N(x.table_cols = -1);
    N(x.k_pages = nullptr); N(x.v_pages = mem + 8); N(x.n_pages = -1); N(x.n_pages = 1ll << 28);

    etc_serving_sample_io p{};
    p.n_rows = 4; p.dtype = ETC_FP32; p.logits = mem; p.row_stride = 1000; p.u = (float *)mem; p.token_out = i32;
#define P(change) REFUSED(etc_serving_sample, etc_serving_sample_io, p, ETC_EINVAL, change)
    P(x.n_rows = 0); P(x.n_rows = 5); P(x.dtype = -1); P(x.logits = nullptr); P(x.logits = mem + 2); P((x.logits = mem + 1, x.dtype = ETC_BF16));
    P(x.row_stride = 999); P(x.row_stride = 1ll << 33); P(x.u = nullptr); P(x.token_out = nullptr); P(x.top_p = (float *)(mem + 2));

    // NULL, another device, an earlier refusal on the device
    CHECK(etc_serving_tables(nullptr, &t, nullptr) == ETC_EINVAL && etc_serving_sample(s, nullptr, nullptr) == ETC_EINVAL);
    int before = g_launches;
    g_device = 1;
    CHECK(etc_serving_attention(s, &n, nullptr) == ETC_EINVAL && g_launches == before);
    g_device = 0;
    s->h_error[0] = SRV_BAD_PAGE; s->h_error[1] = SRV_ATTENTION; s->h_error[2] = 3; s->h_error[3] = 77;
    CHECK(etc_serving_append(s, &a, nullptr) == ETC_ETIMEOUT && g_launches == before);
    CHECK(strstr(etc_serving_last_error(s), "page id") && strstr(etc_serving_last_error(s), "77"));
    CHECK(etc_serving_append(s, &a, nullptr) == ETC_OK && g_launches == before + 1);
    int32_t w[4];
    CHECK(etc_serving_read_error(s, w) == ETC_OK && w[0] == 0 && etc_serving_read_error(s, nullptr) == ETC_EINVAL);
    g_device = 1;                                         // destroyed from another device: that one stays current
    etc_serving_destroy(s);
    CHECK(g_device == 1 && g_allocs == 0);
    g_device = 0;
    etc_serving_destroy(nullptr);
    m.vocab = 0;
    CHECK(etc_serving_create(&m, &l, &s) == ETC_OK);
    CHECK(etc_serving_sample(s, &p, nullptr) == ETC_ESTATE);
    etc_serving_destroy(s);
    CHECK(g_allocs == 0);
    puts("ok");
    return 0;
}
