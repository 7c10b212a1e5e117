// Driver of the host-layer tests of the eviction calls (built and run by tests/test_host_evict.py): tetri_evict_host.cpp with
// tetri_host.cpp, linked with a HIP runtime and kernel launchers that only write down what they are asked for.  Refusals launch
// nothing; what is launched has a workspace that holds it.  argv[1] names the check.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <string>

#include "tetri_internal.h"

#define CHECK(cond)                                                                       \
    do {                                                                                  \
        if (!(cond)) {                                                                    \
            std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #cond); \
            std::exit(1);                                                                 \
        }                                                                                 \
    } while (0)

namespace {

int g_device = 0, g_launches = 0;
hipError_t g_launch_result = hipSuccess;
DecodeParams g_decode;
AddWeightsParams g_add;
WeighParams g_weigh;
SelectParams g_select;
CompactParams g_compact;
int g_row_bytes = 0;
bool g_added = false;

}  // namespace

extern "C" {
hipError_t hipGetDeviceCount(int *n) { *n = 2; return hipSuccess; }
hipError_t hipGetDevice(int *d) { *d = g_device; return hipSuccess; }
hipError_t hipGetDeviceProperties(hipDeviceProp_t *p, int)
{
    std::memset(p, 0, sizeof *p);
    p->multiProcessorCount = 256;
    return hipSuccess;
}
const char *hipGetErrorString(hipError_t) { return "stub"; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipMalloc(void **p, size_t n) { *p = std::aligned_alloc(256, (n + 255) / 256 * 256); return hipSuccess; }
hipError_t hipFree(void *p) { std::free(p); return hipSuccess; }
hipError_t hipMemset(void *p, int v, size_t n) { std::memset(p, v, n); return hipSuccess; }
hipError_t hipMemcpy(void *d, const void *s, size_t n, hipMemcpyKind) { std::memcpy(d, s, n); return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamQuery(hipStream_t) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) { *e = nullptr; return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventQuery(hipEvent_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipPointerGetAttributes(hipPointerAttribute_t *, const void *) { return hipErrorInvalidValue; }
}

hipError_t tetri_launch_attn(const tetri_ctx *, const AttnParams &, int, bool, hipStream_t) { return hipSuccess; }
hipError_t tetri_launch_short(int, bool, const ShortParams &, int, hipStream_t) { return hipSuccess; }
hipError_t tetri_launch_decode(const tetri_ctx *, const DecodeParams &p, hipStream_t)
{
    ++g_launches;
    g_decode = p;
    return g_launch_result;
}
hipError_t tetri_decode_static_memory(DecodeStatic *) { return hipSuccess; }
hipError_t tetri_launch_kv_transfer(const tetri_ctx *, const TransferParams &, int32_t, int32_t, bool, hipStream_t) { return hipSuccess; }
hipError_t tetri_launch_kv_export_fp8(const tetri_ctx *, const TransferParams &, int32_t, hipStream_t) { return hipSuccess; }
hipError_t tetri_launch_append(const tetri_ctx *, const AppendParams &, int32_t, hipStream_t) { return hipSuccess; }
hipError_t tetri_launch_upload(const int32_t *, int32_t *, int64_t, hipStream_t, hipEvent_t) { return hipSuccess; }
hipError_t tetri_launch_upload_inline(const int32_t *, int32_t *, int64_t, hipStream_t) { return hipSuccess; }
hipError_t tetri_launch_add_weights(const AddWeightsParams &p, int32_t, hipStream_t)
{
    ++g_launches;
    g_added = true;
    g_add = p;
    return g_launch_result;
}
hipError_t tetri_launch_weigh(int, bool, const WeighParams &p, int, hipStream_t)
{
    ++g_launches;
    g_weigh = p;
    return g_launch_result;
}
hipError_t tetri_launch_select(const SelectParams &p, hipStream_t)
{
    ++g_launches;
    g_select = p;
    return g_launch_result;
}
hipError_t tetri_launch_compact(int row_bytes, const CompactParams &p, hipStream_t)
{
    ++g_launches;
    g_row_bytes = row_bytes;
    g_compact = p;
    return g_launch_result;
}

namespace {

alignas(16) char g_any[256];                  // stands for every device array: nothing is read
char *const g_off = g_any + 8;                // ... one that is not aligned

tetri_ctx *handle(int hq = 8, int hkv = 2, int d = 128, int chunk = 256, int max_blocks = 256)
{
    const tetri_config c = {hq, hkv, d, 16, chunk, 1024, max_blocks, 8, TETRI_BF16};
    tetri_ctx *h = nullptr;
    CHECK(tetri_create(&c, &h) == TETRI_OK);
    return h;
}

// The arguments of a call, for a test to spoil one of them.
struct Args {
    void *q = g_any, *k = g_any, *v = g_any, *pages = g_any, *out = g_any, *work = g_any;
    float *weights = reinterpret_cast<float *>(g_any);
    int32_t *bt = reinterpret_cast<int32_t *>(g_any), *cu = bt, *ctx = bt, *slots = bt, *lens = bt + 4;
    int32_t n = 4, max_ctx = 100, last = 32, append = 1, fp8 = 0, keep = 64, recent = 8;
    float scale = 0.1f, k_scale = 1.f, v_scale = 1.f;
    int64_t bytes = INT64_MAX;
};
typedef std::function<tetri_status(tetri_ctx *, const Args &)> Call;
const Call decode = [](tetri_ctx *h, const Args &a) {
    return tetri_decode_attn_weights(h, a.q, a.k, a.v, a.pages, a.weights, a.bt, a.ctx, a.n, a.max_ctx, a.scale, a.append, a.fp8, a.k_scale, a.v_scale, a.work,
                                     a.bytes, a.out, nullptr);
};
const Call weigh = [](tetri_ctx *h, const Args &a) {
    return tetri_chunk_prefill_weights(h, a.q, a.k, a.pages, a.weights, a.bt, a.cu, a.ctx, a.n, a.max_ctx, a.last, a.scale, a.fp8, a.k_scale, a.work, a.bytes, nullptr);
};
const Call choose = [](tetri_ctx *h, const Args &a) {
    return tetri_kv_select(h, a.weights, a.bt, a.ctx, a.n, a.max_ctx, a.keep, a.recent, a.slots, a.lens, nullptr);
};
const Call compact = [](tetri_ctx *h, const Args &a) {
    return tetri_kv_compact(h, a.slots, a.bt, a.ctx, a.n, a.keep, a.recent, a.pages, a.weights, a.fp8, nullptr);
};

void refused(const Call &call, std::function<void(Args &)> spoil, const char *word, tetri_status status = TETRI_ERR_INVALID_ARG, int max_blocks = 256)
{
    tetri_ctx *h = handle(8, 2, 128, 256, max_blocks);
    Args a;
    a.max_ctx = std::min(a.max_ctx, max_blocks * 16 - 1);
    g_launches = 0;
    CHECK(call(h, a) == TETRI_OK && g_launches > 0);
    g_launches = 0;
    spoil(a);
    const tetri_status st = call(h, a);
    if (st != status || !std::strstr(tetri_last_error(h), word)) {
        std::fprintf(stderr, "status %d, \"%s\": expected %d and \"%s\"\n", st, tetri_last_error(h), status, word);
        std::exit(1);
    }
    CHECK(g_launches == 0);
    CHECK(call(nullptr, a) == TETRI_ERR_INVALID_ARG && g_launches == 0);
    tetri_destroy(h);
}

#define SPOIL(what) [](Args &a) { a.what; }

void refusals()
{
    for (const Call &c : {decode, weigh, choose, compact}) {
        refused(c, SPOIL(weights = nullptr), "kv_weights is null");
        refused(c, SPOIL(weights = reinterpret_cast<float *>(g_off)), "kv_weights is not 16-byte aligned");
        refused(c, SPOIL(bt = nullptr), "metadata");
        refused(c, SPOIL(ctx = nullptr), "metadata");
        refused(c, SPOIL(n = 0), "num_");
        refused(c, SPOIL(n = -1), "num_");
        refused(c, SPOIL(n = INT_MAX), "num_");
        refused(c, [](Args &) { g_device = 1; }, "current device is 1");
        g_device = 0;
    }
    for (const Call &c : {decode, weigh, choose}) {
        refused(c, SPOIL(max_ctx = -1), "max_ctx_len");
        refused(c, SPOIL(max_ctx = 256 * 16 + 1), "max_ctx_len");
        refused(c, SPOIL(max_ctx = INT_MAX), "max_ctx_len");
    }
    refused(decode, SPOIL(max_ctx = 256 * 16), "max_ctx_len");             // (no slot for the new token)
    for (const Call &c : {decode, weigh}) {
        refused(c, SPOIL(q = nullptr), "q is null");
        refused(c, SPOIL(k = g_off), "k_new is not");
        refused(c, SPOIL(scale = NAN), "scale");
        refused(c, SPOIL(scale = INFINITY), "scale");
        refused(c, SPOIL(work = nullptr), "workspace");
        refused(c, SPOIL(work = g_off), "workspace");
        refused(c, SPOIL(bytes = 0), "workspace of 0 bytes");
        refused(c, [](Args &a) { a.fp8 = 1; a.k_scale = 0.f; }, "scale");
        refused(c, [](Args &a) { a.fp8 = 1; a.k_scale = NAN; }, "scale");
    }
    for (const Call &c : {decode, weigh, compact}) {
        refused(c, SPOIL(pages = nullptr), "kv_pages is null");
        refused(c, SPOIL(pages = g_off), "kv_pages is not");
        refused(c, SPOIL(fp8 = 2), "fp8");
    }
    refused(decode, SPOIL(append = 2), "append");
    refused(decode, SPOIL(v = nullptr), "v_new is null");
    refused(decode, SPOIL(out = g_off), "out is not");
    refused(decode, [](Args &a) { a.fp8 = 1; a.v_scale = -1.f; }, "scale");
    refused(weigh, SPOIL(cu = nullptr), "metadata");
    refused(weigh, SPOIL(n = 9), "num_segs");                              // (the handle's bound)
    refused(weigh, SPOIL(last = 0), "last_rows");
    refused(weigh, SPOIL(last = -3), "last_rows");
    for (const Call &c : {choose, compact}) {
        refused(c, SPOIL(slots = nullptr), "slots is null");
        refused(c, SPOIL(slots = reinterpret_cast<int32_t *>(g_off)), "slots is not");
        refused(c, SPOIL(keep = 0), "keep");
        refused(c, SPOIL(keep = 256 * 16 + 1), "keep");
        refused(c, SPOIL(recent = -1), "recent");
        refused(c, SPOIL(recent = 65), "recent");
    }
    refused(choose, SPOIL(lens = nullptr), "metadata");
    refused(choose, SPOIL(lens = a.ctx), "new_lens is ctx_lens");
    refused(choose, SPOIL(max_ctx = 524289), "at most 524288", TETRI_ERR_UNSUPPORTED, 1 << 20);
    tetri_ctx *wide = handle(66, 2);                                       // 33 query heads to a kv head
    CHECK(decode(wide, Args()) == TETRI_ERR_UNSUPPORTED);
    tetri_destroy(wide);
    // a launch that the runtime refuses
    tetri_ctx *h = handle();
    g_launch_result = hipErrorInvalidValue;
    for (const Call &c : {decode, weigh, choose, compact}) CHECK(c(h, Args()) == TETRI_ERR_HIP && std::strstr(tetri_last_error(h), "launch failed"));
    g_launch_result = hipSuccess;
    tetri_destroy(h);
}

// A workspace of exactly the bytes that are asked for is enough, one byte less is refused, and all that a launch is given lies in it.
void workspaces()
{
    for (int hq : {2, 8, 40})
        for (int chunk : {1, 64, 512, 4096})
            for (int max_ctx : {0, 1, 31, 32, 33, 4000, 65000})
                for (int n : {1, 3, 8}) {
                    tetri_ctx *h = handle(hq, 2, 128, std::max(chunk, 8), 4096);
                    Args a;
                    a.n = n; a.max_ctx = max_ctx;
                    char *const base = static_cast<char *>(a.work);        // (addresses only: nothing is read)
                    a.bytes = tetri_decode_attn_weights_workspace(h, n, max_ctx);
                    CHECK(a.bytes > 0 && decode(h, a) == TETRI_OK);
                    const int64_t heads = (int64_t)n * hq, stride = g_decode.score_stride;
                    CHECK(stride % 32 == 0 && stride > max_ctx && stride <= max_ctx + 32);
                    CHECK((char *)g_decode.scores == base && (char *)(g_decode.scores + heads * stride) <= (char *)g_decode.new_scores);
                    CHECK((char *)(g_decode.new_scores + heads) <= (char *)g_decode.lse && (char *)(g_decode.lse + heads) <= base + a.bytes);
                    --a.bytes;
                    CHECK(decode(h, a) == TETRI_ERR_INVALID_ARG);
                    for (int last : {1, 32, 5000}) {
                        a.last = last;
                        a.bytes = tetri_chunk_prefill_weights_workspace(h, n, max_ctx, last);
                        CHECK(a.bytes > 0 && weigh(h, a) == TETRI_OK);
                        const int64_t rows = (int64_t)std::max(chunk, 8) * hq;
                        CHECK(g_weigh.parts >= 1 && g_weigh.parts <= kWeighParts && g_weigh.last <= std::max(chunk, 8));
                        if (g_weigh.parts > 1) CHECK((char *)g_weigh.stats == base && (char *)(g_weigh.stats + rows * g_weigh.parts) <= (char *)g_weigh.lse);
                        CHECK((char *)g_weigh.lse >= base && (char *)(g_weigh.lse + rows) <= base + a.bytes);
                        --a.bytes;
                        CHECK(weigh(h, a) == TETRI_ERR_INVALID_ARG);
                    }
                    CHECK(tetri_decode_attn_weights_workspace(h, 0, max_ctx) == TETRI_ERR_INVALID_ARG);
                    CHECK(tetri_chunk_prefill_weights_workspace(h, n, -1, 1) == TETRI_ERR_INVALID_ARG);
                    tetri_destroy(h);
                }
    CHECK(tetri_decode_attn_weights_workspace(nullptr, 1, 1) == TETRI_ERR_INVALID_ARG);
    CHECK(tetri_chunk_prefill_weights_workspace(nullptr, 1, 1, 1) == TETRI_ERR_INVALID_ARG);
}

// What the launches are told: the factor on scores is never 0, a pool of codes has its own, and a decode's weights are added once.
void arguments()
{
    tetri_ctx *h = handle();
    for (float scale : {0.f, -0.f, 1e-40f, -0.25f, 3.f}) {
        Args a;
        a.scale = scale;
        a.fp8 = 1; a.k_scale = 0.5f;
        CHECK(weigh(h, a) == TETRI_OK);
        CHECK(g_weigh.c != 0.f && g_weigh.c_codes != 0.f && std::signbit(g_weigh.c) == std::signbit(scale) && std::signbit(g_weigh.c_codes) == std::signbit(scale));
        if (std::fabs(scale) > 0.1f) CHECK(g_weigh.c_codes == 0.5f * g_weigh.c);
    }
    for (int n : {1, 64})
        for (int max_ctx : {10, 2000, 4000}) {
            Args a;
            a.n = n; a.max_ctx = max_ctx;
            g_added = false;
            CHECK(decode(h, a) == TETRI_OK && g_decode.weights == 1);
            CHECK(g_added == (g_decode.weights_w == nullptr));             // by the launch itself or by another one
            CHECK(g_decode.weights_w == nullptr || g_decode.weights_w == a.weights);
            a.fp8 = 1;
            g_added = false;
            CHECK(decode(h, a) == TETRI_OK && (!g_added || g_add.new_scores != nullptr));
            CHECK(tetri_decode_attn(h, a.q, a.k, a.v, a.pages, a.bt, a.ctx, n, max_ctx, 0.1f, a.out, nullptr) == TETRI_OK && g_decode.weights == 0);
        }
    for (int d : {64, 128})
        for (int fp8 : {0, 1}) {
            tetri_ctx *g = handle(4, 2, d);
            Args a;
            a.fp8 = fp8;
            CHECK(compact(g, a) == TETRI_OK && g_row_bytes == d * (fp8 ? 1 : 2));
            tetri_destroy(g);
        }
    tetri_destroy(h);
}

// The kernels that shapes of tests/test_gpu_evict_instances.py go to on 256 compute units (those tests are there to run these kernels).
void instances()
{
    struct { int hq, hkv, chunk, segs, max_ctx, last, row_waves, parts, wide; } const weighs[] = {
        {32, 8, 512, 1, 16384, 32, 2, 64, 1},
        {32, 8, 512, 7, 3000, 1000, 2, 3, 0},
        {192, 48, 256, 1, 600, 1000, 4, 2, 0},
        {48, 48, 1000, 1, 33, 1000, 4, 2, 0},
        {96, 24, 480, 3, 700, 1000, 4, 2, 0},
        {192, 48, 480, 3, 1700, 1000, 4, 1, 1},
        {192, 48, 300, 1, 1500, 130, 4, 3, 0},
        {96, 24, 203, 3, 1200, 1000, 2, 2, 0},
        {144, 48, 145, 2, 2600, 1000, 2, 2, 1},
        {48, 48, 16, 1, 2600, 1000, 1, 10, 1},
    };
    for (const auto &x : weighs)
        for (int d : {64, 128})
            for (int fp8 : {0, 1}) {
                tetri_ctx *h = handle(x.hq, x.hkv, d, x.chunk, 2048);
                Args a;
                a.n = x.segs; a.max_ctx = x.max_ctx; a.last = x.last; a.fp8 = fp8;
                CHECK(weigh(h, a) == TETRI_OK);
                CHECK(g_weigh.row_waves == x.row_waves && g_weigh.parts == x.parts && g_weigh.wide_keys == x.wide);
                tetri_destroy(h);
            }
    // decode: ranges, parts, and by default; the weights by the launch itself and by one behind it
    struct { int n, max_ctx; const char *option; int value, added; } const decodes[] = {
        {5, 2100, nullptr, 0, 1}, {5, 2100, "decode_ranges", 7, 1}, {5, 2100, "decode_parts", 3, 1}, {3, 2100, nullptr, 0, 1},
        {1, 1000, nullptr, 0, 0}, {6, 260, nullptr, 0, 0}, {3, 260, nullptr, 0, 0},
    };
    for (const auto &x : decodes)
        for (int fp8 : {0, 1}) {
            tetri_ctx *h = handle();
            if (x.option) CHECK(tetri_set_option(h, x.option, x.value) == TETRI_OK);
            Args a;
            a.n = x.n; a.max_ctx = x.max_ctx; a.fp8 = fp8;
            g_added = false;
            CHECK(decode(h, a) == TETRI_OK && g_added == (x.added != 0));
            if (x.option && !std::strcmp(x.option, "decode_ranges")) CHECK(g_decode.parts == 0 && g_decode.ranges == x.value);
            if (x.option && !std::strcmp(x.option, "decode_parts")) CHECK(g_decode.parts == x.value);
            if (x.added) CHECK((g_add.new_scores != nullptr) == (fp8 != 0));
            tetri_destroy(h);
        }
}

}  // namespace

int main(int argc, char **argv)
{
    const std::string name = argc > 1 ? argv[1] : "";
    if (name == "refusals") refusals();
    else if (name == "workspaces") workspaces();
    else if (name == "arguments") arguments();
    else if (name == "instances") instances();
    else return 2;
    std::printf("%s: ok\n", name.c_str());
    return 0;
}
