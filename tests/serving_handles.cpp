// Handles of the serving operators over a runtime of stubs, on the CPU: which device is waited for, what a handle allocates.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "serving.cpp"

static int g_device = 0, g_synced = -1;
static size_t g_bytes = 0;
extern "C" {
hipError_t hipGetDevice(int *d) { *d = g_device; return hipSuccess; }
hipError_t hipSetDevice(int d) { g_device = d; return hipSuccess; }
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipDeviceSynchronize() { g_synced = g_device; return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n) { g_bytes += n; *p = calloc(1, 64); return n > 0 ? hipSuccess : hipErrorInvalidValue; }
hipError_t hipFree(void *p) { free(p); return hipSuccess; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { *p = malloc(n); return hipSuccess; }
hipError_t hipHostFree(void *p) { free(p); return hipSuccess; }
hipError_t hipHostGetDevicePointer(void **d, void *h, unsigned) { *d = h; return hipSuccess; }
hipError_t hipMemset(void *, int, size_t) { return hipSuccess; }
hipError_t hipMemcpy(void *, const void *, size_t, hipMemcpyKind) { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "stub"; }
}
namespace etc {
int64_t attention_slot_bytes(int d) { return d * 1040; }
int64_t sample_slices(int, int) { return 4; }
int64_t sample_stat_bytes() { return 16; }
int64_t sample_bins_bytes() { return 8192; }
hipError_t launch_serving_tables(const ServingDev &, const etc_serving_tables_io &, hipStream_t) { return hipSuccess; }
hipError_t launch_serving_append(const ServingDev &, const etc_serving_append_io &, hipStream_t) { return hipSuccess; }
hipError_t launch_serving_attention(const ServingDev &, const etc_serving_attention_io &, hipStream_t) { return hipSuccess; }
hipError_t launch_serving_sample(const ServingDev &, const etc_serving_sample_io &, hipStream_t) { return hipSuccess; }
}  // namespace etc

#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); return 1; } } while (0)

static etc_model_desc model()
{
    etc_model_desc m{};
    m.n_q_heads = 64; m.n_kv_heads = 8; m.head_dim = 128; m.page_size = 16; m.rms_eps = 1e-5f; m.rope_theta = 1e4f; m.vocab = 100000;
    return m;
}

// The word is that of the handle's launches, so it is its device that is waited for, whatever device is current.
static int read_error_waits_for_the_handles_device()
{
    const etc_model_desc m = model();
    const etc_serving_limits l{4, 100, 500};
    etc_serving *s = nullptr;
    g_device = 2;
    CHECK(etc_serving_create(&m, &l, &s) == ETC_OK);
    for (int current : {2, 0, 5}) {
        int32_t w[4];
        g_device = current;
        g_synced = -1;
        CHECK(etc_serving_read_error(s, w) == ETC_OK && g_synced == 2 && g_device == current);
        s->h_error[0] = SRV_BAD_SLOT; s->h_error[1] = SRV_APPEND; s->h_error[2] = 4; s->h_error[3] = 9;
        CHECK(etc_serving_read_error(s, w) == ETC_ETIMEOUT && w[0] == SRV_BAD_SLOT && w[3] == 9 && g_device == current);
    }
    etc_serving_destroy(s);
    g_device = 0;
    return 0;
}

// Partial results of cut keys: a handle's limits say how many can ever be needed, none where the longest sequence is too short to be cut.
static int memory_follows_the_limits()
{
    etc_model_desc m = model();
    auto bytes = [&](int seqs, int tokens, int kv) -> size_t {
        const etc_serving_limits l{seqs, tokens, kv};
        etc_serving *s = nullptr;
        g_bytes = 0;
        if (etc_serving_create(&m, &l, &s) != ETC_OK) return (size_t)-1;
        const size_t n = g_bytes;
        etc_serving_destroy(s);
        return n;
    };
    const size_t slot = (size_t)etc::attention_slot_bytes(128), all = 1024 * slot;
    m.vocab = 0;
    CHECK(bytes(64, 64, 1) < 16384);                      // a handle that only samples, or appends
    CHECK(bytes(64, 64, 6 * 64) < 16384);                 // 6 tiles are never cut
    CHECK(bytes(1, 1, 7 * 64) >= 8 * 4 * slot && bytes(1, 1, 7 * 64) < 8 * 4 * slot + 16384);      // 8 heads, 4 parts of 2 tiles at most
    CHECK(bytes(1, 8, 1000) < 8 * 9 * slot);
    CHECK(bytes(64, 4096, 1 << 20) >= all && bytes(64, 4096, 1 << 20) < all + 16384);
    CHECK(bytes(1024, 1 << 20, 1 << 30) >= all && bytes(1024, 1 << 20, 1 << 30) < all + 16384);
    CHECK(bytes(1, 1, 1 << 30) >= all);
    return 0;
}

int main(int argc, char **argv)
{
    const char *which = argc > 1 ? argv[1] : "";
    if (!strcmp(which, "read_error")) return read_error_waits_for_the_handles_device();
    if (!strcmp(which, "memory")) return memory_follows_the_limits();
    printf("which?\n");
    return 2;
}
