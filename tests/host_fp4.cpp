// Driver of the host-layer tests of the calls over 4-bit codes and of the norm and rotation (built and run by tests/test_host_fp4.py): tetri_fp4_host.cpp and
// tetri_rope_host.cpp with tetri_host.cpp, linked with a HIP runtime and kernel launchers that only write down what they are asked for.  argv[1] names
// the check.
#include <hip/hip_runtime.h>

#include <climits>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <string>
#include <vector>

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
bool g_busy = false;
hipError_t g_result = hipSuccess;
std::string g_kernel;
DecodeParams g_decode;
AttnParams g_attn;
PrefillFp4Params g_small;
TransferParams g_transfer;
RopeParams g_rope;
int g_tiles = 0;
struct Counters {
    const int32_t *use, *clear;
    int32_t n;
};
std::vector<Counters> g_counters;

hipError_t launched(const char *kernel)
{
    ++g_launches;
    g_kernel = kernel;
    return g_result;
}

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
hipError_t hipStreamQuery(hipStream_t) { return g_busy ? hipErrorNotReady : hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) { *e = nullptr; return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventQuery(hipEvent_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t) { return hipSuccess; }
hipError_t hipPointerGetAttributes(hipPointerAttribute_t *, const void *) { return hipErrorInvalidValue; }
}

hipError_t tetri_launch_attn(const tetri_ctx *, const AttnParams &, int, bool, hipStream_t) { return launched("16-bit"); }
hipError_t tetri_launch_short(int, bool, const ShortParams &, int, hipStream_t) { return launched("16-bit"); }
hipError_t tetri_launch_decode(const tetri_ctx *, const DecodeParams &p, hipStream_t)
{
    if (p.n_counters) g_counters.push_back({p.counters, p.counters_next, p.n_counters});
    return launched("16-bit");
}
hipError_t tetri_decode_static_memory(DecodeStatic *) { return hipSuccess; }
hipError_t tetri_launch_kv_transfer(const tetri_ctx *, const TransferParams &, int32_t, int32_t, bool, hipStream_t) { return launched("16-bit"); }
hipError_t tetri_launch_kv_export_fp8(const tetri_ctx *, const TransferParams &, int32_t, hipStream_t) { return launched("16-bit"); }
hipError_t tetri_launch_append(const tetri_ctx *, const AppendParams &, int32_t, hipStream_t) { return launched("16-bit"); }
hipError_t tetri_launch_upload(const int32_t *, int32_t *, int64_t, hipStream_t, hipEvent_t) { return hipSuccess; }
hipError_t tetri_launch_upload_inline(const int32_t *, int32_t *, int64_t, hipStream_t) { return hipSuccess; }
hipError_t tetri_launch_kv_export_fp4(const tetri_ctx *, const TransferParams &p, int32_t tiles, hipStream_t)
{
    g_transfer = p;
    g_tiles = tiles;
    return launched("export");
}
hipError_t tetri_launch_kv_import_fp4(const tetri_ctx *, const TransferParams &p, int32_t tiles, hipStream_t)
{
    g_transfer = p;
    g_tiles = tiles;
    return launched("import");
}
hipError_t tetri_launch_decode_fp4(const tetri_ctx *, const DecodeParams &p, hipStream_t)
{
    g_decode = p;
    if (p.n_counters) g_counters.push_back({p.counters, p.counters_next, p.n_counters});
    return launched(p.parts == 0 ? "ranges" : "parts");
}
hipError_t tetri_launch_attn_fp4(const tetri_ctx *, const AttnParams &p, int key_parts, hipStream_t)
{
    CHECK(p.plan == nullptr && (key_parts == 1 || key_parts == 2));
    g_attn = p;
    if (p.stream_wgs > 0 || p.helpers > 0) g_counters.push_back({p.counters, p.counters_next, p.n_counters});
    return launched(p.stream_wgs > 0 ? "stream" : (p.helpers > 0 ? "tails" : "tiles"));
}
hipError_t tetri_launch_prefill_fp4(int, const PrefillFp4Params &p, hipStream_t)
{
    g_small = p;
    g_counters.push_back({p.counters, p.counters_next, p.n_counters});
    return launched("small");
}
hipError_t tetri_launch_rope(int, const RopeParams &p, hipStream_t)
{
    g_rope = p;
    return launched("rope");
}

namespace {

alignas(16) char g_any[256];                  // stands for every device array: nothing is read
char *const g_off = g_any + 8;                // ... one that is not aligned

tetri_ctx *handle(int hq = 8, int hkv = 2, int d = 128, int chunk = 256, int max_blocks = 256, int segs = 8)
{
    const tetri_config c = {hq, hkv, d, 16, chunk, 1024, max_blocks, segs, TETRI_BF16};
    tetri_ctx *h = nullptr;
    CHECK(tetri_create(&c, &h) == TETRI_OK);
    return h;
}

// The arguments of the calls, for a test to spoil one of them.
struct Args {
    void *q = g_any, *k = g_any, *v = g_any, *pages = g_any, *rows = g_any, *out = g_any, *k_out = g_any + 128, *buf = g_any, *qw = g_any, *kw = g_any;
    int32_t *bt = reinterpret_cast<int32_t *>(g_any), *cu = bt, *ctx = bt, *pos = nullptr, *first = nullptr;
    int32_t n = 4, max_ctx = 100, append = 1, num_rows = 10;
    int64_t total = 50, q_stride = 8 * 128, k_stride = 2 * 128;
    float scale = 0.1f, eps = 1e-6f;
    bool no_rope = false;
    tetri_rope rope = {};
    Args()
    {
        rope.num_pairs = 64;
        rope.num_axes = 1;
        for (float &f : rope.freq) f = 0.5f;
    }
};
tetri_status decode(tetri_ctx *h, const Args &a)
{
    return tetri_decode_attn_fp4(h, a.q, a.k, a.v, a.pages, a.bt, a.ctx, a.n, a.max_ctx, a.scale, a.append, a.out, nullptr);
}
tetri_status prefill(tetri_ctx *h, const Args &a, hipStream_t s = nullptr)
{
    return tetri_chunk_prefill_attn_fp4(h, a.q, a.k, a.v, a.pages, a.bt, a.cu, a.ctx, a.n, a.scale, a.append, a.out, s);
}
tetri_status export_codes(tetri_ctx *h, const Args &a) { return tetri_kv_export_fp4(h, a.rows, a.bt, a.cu, a.first, a.n, a.total, a.buf, nullptr); }
tetri_status import_codes(tetri_ctx *h, const Args &a) { return tetri_kv_import_fp4(h, a.buf, a.bt, a.cu, a.first, a.n, a.total, a.pages, nullptr); }
tetri_status rope(tetri_ctx *h, const Args &a)
{
    return tetri_qk_norm_rope(h, a.q, a.q_stride, a.k, a.k_stride, a.qw, a.kw, a.eps, a.no_rope ? nullptr : &a.rope, a.pos, a.cu, a.ctx, a.n, a.num_rows, a.out, a.k_out, nullptr);
}

typedef tetri_status (*Call)(tetri_ctx *, const Args &);
typedef std::function<void(Args &)> Spoil;

void refusals()
{
    tetri_ctx *h = handle();
    auto prefill0 = [](tetri_ctx *x, const Args &a) { return prefill(x, a); };
    Args in_place;                            // the outputs' rows follow each other, the inputs' do not
    in_place.out = in_place.q;
    const struct { Call call; std::vector<Spoil> spoils; } all[] = {
        {decode, {[](Args &a) { a.q = nullptr; }, [](Args &a) { a.k = g_off; }, [](Args &a) { a.v = nullptr; }, [](Args &a) { a.pages = g_off; }, [](Args &a) { a.bt = nullptr; },
                  [](Args &a) { a.ctx = nullptr; }, [](Args &a) { a.n = 0; }, [](Args &a) { a.n = -1; }, [](Args &a) { a.max_ctx = -1; }, [](Args &a) { a.max_ctx = 256 * 16; },
                  [](Args &a) { a.scale = NAN; }, [](Args &a) { a.scale = INFINITY; }, [](Args &a) { a.append = 2; }, [](Args &a) { a.append = -1; }, [](Args &a) { a.out = g_off; }}},
        {prefill0, {[](Args &a) { a.q = nullptr; }, [](Args &a) { a.k = g_off; }, [](Args &a) { a.v = nullptr; }, [](Args &a) { a.pages = nullptr; }, [](Args &a) { a.bt = nullptr; },
                    [](Args &a) { a.cu = nullptr; }, [](Args &a) { a.ctx = nullptr; }, [](Args &a) { a.n = 0; }, [](Args &a) { a.n = 9; }, [](Args &a) { a.scale = -INFINITY; },
                    [](Args &a) { a.append = 3; }, [](Args &a) { a.out = nullptr; }}},
        {export_codes, {[](Args &a) { a.rows = nullptr; }, [](Args &a) { a.rows = g_off; }, [](Args &a) { a.bt = nullptr; }, [](Args &a) { a.cu = nullptr; }, [](Args &a) { a.n = 0; },
                        [](Args &a) { a.n = INT_MAX; }, [](Args &a) { a.total = -1; }, [](Args &a) { a.total = 4 * 256 * 16 + 1; }, [](Args &a) { a.buf = nullptr; },
                        [](Args &a) { a.buf = g_off; }}},
        {import_codes, {[](Args &a) { a.pages = nullptr; }, [](Args &a) { a.pages = g_off; }, [](Args &a) { a.bt = nullptr; }, [](Args &a) { a.cu = nullptr; }, [](Args &a) { a.n = -4; },
                        [](Args &a) { a.total = -1; }, [](Args &a) { a.buf = nullptr; }, [](Args &a) { a.buf = g_off; }}},
        {rope, {[](Args &a) { a.q = nullptr; }, [](Args &a) { a.k = g_off; }, [](Args &a) { a.out = nullptr; }, [](Args &a) { a.k_out = g_off; }, [](Args &a) { a.qw = g_off; },
                [](Args &a) { a.kw = g_off; }, [](Args &a) { a.q_stride = 8 * 128 - 8; }, [](Args &a) { a.q_stride = 8 * 128 + 4; }, [](Args &a) { a.k_stride = 0; },
                [](Args &a) { a.k_stride = -256; }, [](Args &a) { a.q_stride = INT64_MAX / 8 * 8; }, [](Args &a) { a.eps = -1e-6f; }, [](Args &a) { a.eps = NAN; }, [](Args &a) { a.no_rope = true; },
                [](Args &a) { a.rope.num_pairs = 0; }, [](Args &a) { a.rope.num_pairs = 12; }, [](Args &a) { a.rope.num_pairs = 72; }, [](Args &a) { a.rope.num_axes = 0; },
                [](Args &a) { a.rope.num_axes = 9; }, [](Args &a) { a.rope.adjacent = 2; }, [](Args &a) { a.rope.freq[63] = INFINITY; }, [](Args &a) { a.rope.axis[3] = 1; },
                [](Args &a) { a.pos = a.bt; }, [](Args &a) { a.cu = nullptr; }, [](Args &a) { a.ctx = nullptr; }, [](Args &a) { a.cu = a.ctx = nullptr; }, [](Args &a) { a.n = 0; },
                [](Args &a) { a.n = 9; }, [](Args &a) { a.num_rows = 0; }, [](Args &a) { a.num_rows = -5; }, [](Args &a) { a.out = a.q; a.q_stride = 8 * 128 + 8; },
                [](Args &a) { a.k_out = a.k; a.k_stride = 2 * 128 + 8; }}},
    };
    for (const auto &x : all) {
        const Args good;
        g_launches = 0;
        CHECK(x.call(h, good) == TETRI_OK && g_launches == 1);
        g_launches = 0;
        CHECK(x.call(nullptr, good) == TETRI_ERR_INVALID_ARG);
        for (size_t i = 0; i < x.spoils.size(); ++i) {
            Args a;
            x.spoils[i](a);
            if (x.call(h, a) != TETRI_ERR_INVALID_ARG) {
                std::fprintf(stderr, "call %d, spoilt argument %d is taken\n", (int)(&x - all), (int)i);
                std::exit(1);
            }
        }
        g_device = 1;
        CHECK(x.call(h, good) == TETRI_ERR_INVALID_ARG);
        g_device = 0;
        CHECK(g_launches == 0);
        g_result = hipErrorOutOfMemory;
        CHECK(x.call(h, good) == TETRI_ERR_HIP);
        g_result = hipSuccess;
    }
    // nothing to move: nothing is launched, buffers may be null
    Args none;
    none.total = 0;
    none.buf = nullptr;
    g_launches = 0;
    CHECK(export_codes(h, none) == TETRI_OK && import_codes(h, none) == TETRI_OK && g_launches == 0);
    // a frequency and an axis behind the pairs that turn do not matter
    Args few;
    few.rope.num_pairs = 16;
    few.rope.freq[16] = NAN;
    few.rope.axis[20] = 7;
    CHECK(rope(h, few) == TETRI_OK && g_rope.freq[16] == 0.f && g_rope.axis[20] == 0);
    // a launch that uses the shared scratch memory while another stream's is pending
    Args a;
    tetri_set_option(h, "attn_variant", 3);
    CHECK(prefill(h, a, reinterpret_cast<hipStream_t>(64)) == TETRI_OK && g_kernel == "small");
    g_busy = true;
    CHECK(prefill(h, a, reinterpret_cast<hipStream_t>(128)) == TETRI_ERR_INVALID_ARG);
    CHECK(prefill(h, a, reinterpret_cast<hipStream_t>(64)) == TETRI_OK);
    g_busy = false;
    CHECK(prefill(h, a, reinterpret_cast<hipStream_t>(128)) == TETRI_OK);
    tetri_destroy(h);
}

// What launches are given fits the handle's memory, and their numbers the types that the kernels count in.
void memory()
{
    const int heads[][3] = {{40, 40, 128}, {32, 8, 128}, {8, 2, 128}, {32, 1, 128}, {6, 2, 64}, {3, 1, 64}, {1, 1, 128}, {128, 128, 128}, {128, 128, 64}, {255, 255, 64}, {64, 2, 64}};
    for (const auto &x : heads) {
        const int hq = x[0], hkv = x[1], d = x[2], g = hq / hkv;
        for (int chunk : {1, 33, 512, 8192}) {
            for (int segs : {1, 20, 64, 500}) {
                if (segs > chunk) continue;
                for (int blocks : {4, 600, 100000}) {
                    tetri_ctx *h = handle(hq, hkv, d, chunk, blocks, segs);
                    const int64_t bytes = 2 * (int64_t)h->scratch_units * h->unit_bytes;
                    for (int variant : {0, 1, 2, 3}) {
                        tetri_set_option(h, "attn_variant", variant);
                        Args a;
                        a.n = segs;
                        CHECK(prefill(h, a) == TETRI_OK);
                        if (g_kernel == "small") {
                            const PrefillFp4Params &p = g_small;
                            CHECK(p.ranges >= 1 && (int64_t)2 * p.ranges * hkv * kPrefillFp4Cols * (d + 2) * 4 <= bytes && (int64_t)p.ranges * hkv <= p.n_counters);
                            const int64_t tiles = ((int64_t)chunk * g + kPrefillFp4Cols - 1) / kPrefillFp4Cols + segs;
                            CHECK(tiles * (blocks / 2 + (chunk + 31) / 32 + 4) <= INT_MAX);
                            CHECK(p.append_blocks >= 1 && p.counters && p.counters_next && p.counters != p.counters_next);
                        } else {
                            const AttnParams &p = g_attn;
                            if (p.stream_wgs > 0) {
                                CHECK((int64_t)p.groups * p.stream_wgs * 8 <= 2 * (int64_t)h->scratch_units && segs <= 64 && p.stream_wgs <= 255);
                                CHECK((int64_t)p.groups * p.tiles * 4 <= p.n_counters);
                            }
                            if (p.helpers > 0) CHECK((int64_t)p.groups * p.tiles * 4 <= std::min<int64_t>(p.n_counters, h->scratch_units));
                            CHECK(p.append_blocks >= 1 && p.append_blocks <= std::max(chunk, 64));
                        }
                    }
                    tetri_destroy(h);
                }
            }
        }
        for (int blocks : {4, 600, 100000, 1000000}) {
            tetri_ctx *h = handle(hq, hkv, d, 256, blocks);
            const int64_t bytes = 2 * (int64_t)h->scratch_units * h->unit_bytes, part = (int64_t)4 * (g * d + (2 * g + 3) / 4 * 4);
            for (int n : {1, 2, 48, 64, 200, 1024, 1025, 5000})
                for (int ctx : {0, 1, 300, 5000, 100000, 16 * blocks - 1})
                    for (int way = 0; way < 6; ++way) {
                        if (ctx > 16 * blocks - 1) continue;
                        tetri_set_option(h, "decode_parts", way == 1 ? 1 : (way == 2 ? 1000 : 0));
                        tetri_set_option(h, "decode_ranges", way == 3 ? 2 : (way == 4 ? 300 : (way == 5 ? 100000 : 0)));
                        Args a;
                        a.n = n;
                        a.max_ctx = ctx;
                        if (decode(h, a) != TETRI_OK) { CHECK((int64_t)n * hkv * hkv > 0x7fffffff || (int64_t)n * hkv * 1024 > 0x7fffffff); continue; }
                        const DecodeParams &p = g_decode;
                        if (p.parts == 0) {
                            CHECK(p.ranges > 1 && n <= kDecodeLookup && (int64_t)n * (blocks / 2 + 9) <= INT_MAX);
                            CHECK(2 * (int64_t)p.ranges * hkv * part <= bytes && (int64_t)p.ranges * hkv <= p.n_counters);
                        } else if (p.parts > 1) {
                            CHECK((int64_t)n * hkv * p.parts * part <= bytes && (int64_t)n * hkv <= p.n_counters);
                        }
                        CHECK((p.parts == 1) == (p.n_counters == 0));
                    }
            tetri_destroy(h);
        }
    }
}

// Whatever a launch leaves in its counters is zeroed before they are used again, in any order of the launches of a handle.
void counters()
{
    tetri_ctx *h = handle(8, 2, 128);
    Args a;
    a.max_ctx = 3000;
    for (const char *seq : {"dddddddddd", "ssssssssss", "tttttttttt", "dstdstssddttdsxtxsxdxxst"}) {
        g_counters.clear();
        for (const char *c = seq; *c; ++c) {
            tetri_set_option(h, "decode_parts", 5);
            tetri_set_option(h, "attn_variant", *c == 's' ? 3 : 0);
            if (*c == 'd') CHECK(decode(h, a) == TETRI_OK);
            else if (*c == 'x') CHECK(tetri_decode_attn(h, a.q, a.k, a.v, a.pages, a.bt, a.ctx, a.n, a.max_ctx, a.scale, a.out, nullptr) == TETRI_OK);
            else CHECK(prefill(h, a) == TETRI_OK && g_kernel == (*c == 's' ? "small" : "stream"));
        }
        const size_t n = g_counters.size();
        CHECK(n == std::strlen(seq));
        for (size_t i = 0; i < n; ++i) {
            const Counters &x = g_counters[i];
            CHECK(x.n > 0 && x.clear != nullptr && x.clear != x.use);
            if (i > 0) CHECK(x.clear != g_counters[i - 1].use && x.use != g_counters[i - 1].use && x.use != g_counters[i - 1].clear);
            for (size_t j = i + 1; j < n; ++j)
                if (g_counters[j].use == x.use) {
                    bool cleared = false;
                    for (size_t k = i + 1; k < j; ++k) cleared = cleared || (g_counters[k].clear == x.use && g_counters[k].n == x.n);
                    CHECK(cleared);
                    break;
                }
        }
    }
    tetri_destroy(h);
}

// argv: heads, kv heads, head_dim, chunk, segments (prefill) or requests, longest context (decode): the kernel
void kernels(int argc, char **argv)
{
    int x[7] = {0};
    for (int i = 2; i < argc && i < 9; ++i) x[i - 2] = std::atoi(argv[i]);
    Args a;
    if (argc == 7) {
        tetri_ctx *h = handle(x[0], x[1], x[2], x[3], 1024, std::max(x[4], 1));
        a.n = x[4];
        CHECK(prefill(h, a) == TETRI_OK);
        tetri_destroy(h);
        std::printf("%s\n", g_kernel.c_str());
    } else {
        tetri_ctx *h = handle(x[0], x[1], x[2], 64, 1024);
        a.n = x[3];
        a.max_ctx = x[4];
        CHECK(decode(h, a) == TETRI_OK);
        tetri_destroy(h);
        std::printf("%d parts %d ranges\n", g_decode.parts, g_decode.parts == 0 ? g_decode.ranges : 0);
    }
}

}  // namespace

int main(int argc, char **argv)
{
    const std::string check = argc > 1 ? argv[1] : "";
    if (check == "refusals") refusals();
    else if (check == "memory") memory();
    else if (check == "counters") counters();
    else if (check == "kernels") { kernels(argc, argv); return 0; }
    else return 2;
    std::printf("%s: ok\n", check.c_str());
    return 0;
}
