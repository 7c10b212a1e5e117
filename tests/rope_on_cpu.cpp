// The kernel of tetri_rope.hip on the CPU (built and run by tests/test_host_rope_kernel.py): every array ends where memory ends that can be
// touched, so that a read or a write behind it ends the program.
#include <hip/hip_runtime.h>
#include <sys/mman.h>
#include <ucontext.h>
#include <unistd.h>

#include <csignal>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "tetri_rope.hip"

Index3 blockIdx, threadIdx;
RopeParams g_params;

namespace {

constexpr int kStack = 256 << 10;
ucontext_t g_main, g_lane[64];
bool g_ended[64];
uint64_t g_slot[64];
int g_now = 0;
void (*g_kernel)(RopeParams);
std::vector<char> g_stacks(64 * kStack);
char g_doing[200];

void lane_main()
{
    g_kernel(g_params);
    g_ended[g_now] = true;
    swapcontext(&g_lane[g_now], &g_main);
}

void on_fault(int)
{
    const char *what = "an access outside the arrays: ";
    (void)!write(2, what, std::strlen(what));
    (void)!write(2, g_doing, std::strlen(g_doing));
    _exit(1);
}

// n bytes that end at a page that cannot be touched.
template <class T> T *at_the_end(size_t n)
{
    const size_t page = 4096, bytes = n * sizeof(T), room = (bytes + page - 1) / page * page;
    char *p = static_cast<char *>(mmap(nullptr, room + page, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
    if (p == MAP_FAILED || mprotect(p + room, page, PROT_NONE) != 0) std::abort();
    return reinterpret_cast<T *>(p + room - bytes);      // (kept to the end of the program)
}

float number(uint16_t bits) { return __builtin_bit_cast(float, (uint32_t)bits << 16); }

}  // namespace

AllLanes meet(uint64_t mine)
{
    const int lane = g_now;
    g_slot[lane] = mine;
    swapcontext(&g_lane[lane], &g_main);
    AllLanes all;
    std::memcpy(all.of, g_slot, sizeof g_slot);
    swapcontext(&g_lane[lane], &g_main);
    return all;
}

void launch_on_cpu(void (*kernel)(RopeParams), dim3 grid, dim3 block, const RopeParams &p)
{
    g_params = p;
    g_kernel = kernel;
    for (unsigned b = 0; b < grid.x; ++b)
        for (unsigned w = 0; w < block.x / 64; ++w) {
            for (int i = 0; i < 64; ++i) {
                g_ended[i] = false;
                getcontext(&g_lane[i]);
                g_lane[i].uc_stack.ss_sp = g_stacks.data() + i * kStack;
                g_lane[i].uc_stack.ss_size = kStack;
                g_lane[i].uc_link = nullptr;
                makecontext(&g_lane[i], lane_main, 0);
            }
            for (bool any = true; any;) {
                any = false;
                for (int i = 0; i < 64; ++i) {
                    if (g_ended[i]) continue;
                    any = true;
                    g_now = i;
                    blockIdx.x = b;
                    threadIdx.x = w * 64 + i;
                    swapcontext(&g_main, &g_lane[i]);
                }
            }
        }
}

extern "C" hipError_t hipGetLastError() { return hipSuccess; }

// argv: heads, kv heads, head_dim, rows of the call, segments (0: given positions), rows of a segment, wavefronts of a row at most, pairs, adjacent
int main(int argc, char **argv)
{
    if (argc != 10) return 2;
    int x[10];
    for (int i = 1; i < 10; ++i) x[i] = std::atoi(argv[i]);
    const int hq = x[1], hkv = x[2], d = x[3], rows = x[4], segs = x[5], each = x[6];
    std::signal(SIGSEGV, on_fault);
    std::signal(SIGBUS, on_fault);
    for (int i = 1, at = 0; i < 10; ++i) at += std::snprintf(g_doing + at, sizeof g_doing - at, "%s ", argv[i]);
    const int real = segs ? segs * each : rows;

    const int64_t row_elements = (hq + 2 * hkv) * d;     // q and k out of one projection's rows
    uint16_t *in = at_the_end<uint16_t>(real > 0 ? real * row_elements - hkv * d : 0);       // (up to the end of the last real row's k)
    std::srand(3);
    auto any = [] { return (uint16_t)((std::rand() % 0x300 + 0x3d00) | (std::rand() & 1) << 15); };      // up to about 8
    for (int64_t i = 0; i < (real > 0 ? real * row_elements - hkv * d : 0); ++i) in[i] = any();
    uint16_t *w = at_the_end<uint16_t>(d), *q_out = at_the_end<uint16_t>((int64_t)real * hq * d), *k_out = at_the_end<uint16_t>((int64_t)real * hkv * d);
    for (int i = 0; i < d; ++i) w[i] = any();
    int32_t *cu = at_the_end<int32_t>(segs + 1), *ctx = at_the_end<int32_t>(segs), *pos = at_the_end<int32_t>(rows);
    for (int s = 0; s <= segs; ++s) cu[s] = s * each;
    for (int s = 0; s < segs; ++s) ctx[s] = 7 * s + 1;
    for (int r = 0; r < rows; ++r) pos[r] = 3 * r + 2;

    RopeParams p = {};
    p.q = in; p.k = in + hq * d;
    p.q_stride = p.k_stride = row_elements;
    p.q_weight = w; p.k_weight = nullptr;
    p.q_out = q_out; p.k_out = k_out;
    p.pos = segs ? nullptr : pos;
    p.cu = segs ? cu : nullptr; p.ctx = segs ? ctx : nullptr;
    p.eps = 1e-6f;
    p.S = segs; p.rows = rows; p.Hq = hq; p.Hkv = hkv;
    p.pairs = x[8]; p.adjacent = x[9];
    for (int i = 0; i < p.pairs; ++i) p.freq[i] = 1.0f / (1 + i);
    const int insts = (hq + hkv + 512 / d - 1) / (512 / d), want = std::min(insts, x[7]);
    p.per_split = (insts + want - 1) / want;
    p.splits = (insts + p.per_split - 1) / p.per_split;
    p.splits_magic = p.splits <= 1 ? 0u : (uint32_t)((0x100000000ull + p.splits - 1) / p.splits);
    for (int past = 0; past < 2; ++past) {
        std::memset(q_out, 0, (size_t)real * hq * d * 2);
        std::memset(k_out, 0, (size_t)real * hkv * d * 2);
        p.past_caches = past;
        if (tetri_launch_rope(d, p, nullptr) != hipSuccess) return 3;
        for (int r = 0; r < real; ++r)
            for (int h = 0; h < hq + hkv; ++h) {
                const uint16_t *src = in + r * row_elements + h * d, *got = h < hq ? q_out + ((int64_t)r * hq + h) * d : k_out + ((int64_t)r * hkv + h - hq) * d;
                double y[128], sum = 0;
                for (int i = 0; i < d; ++i) sum += (double)number(src[i]) * number(src[i]);
                for (int i = 0; i < d; ++i) y[i] = h < hq ? number(src[i]) * number(w[i]) / std::sqrt(sum / d + 1e-6) : number(src[i]);
                const double at = segs ? ctx[r / each] + r % each : pos[r];
                for (int i = 0; i < p.pairs; ++i) {
                    double &a = y[p.adjacent ? 2 * i : i], &b = y[p.adjacent ? 2 * i + 1 : i + p.pairs];
                    const double t = at * p.freq[i], c = std::cos(t), s = std::sin(t), na = a * c - b * s, nb = b * c + a * s;
                    a = na;
                    b = nb;
                }
                // one rounding to bf16, and 32-bit sums of numbers of at most 8 * 8 * 8
                for (int i = 0; i < d; ++i)
                    if (!(std::fabs(number(got[i]) - y[i]) <= std::fabs(y[i]) / 256 + 512.0 / (1 << 18))) {
                        std::fprintf(stderr, "row %d head %d element %d: %g, not %g\n", r, h, i, number(got[i]), y[i]);
                        return 4;
                    }
            }
    }
    std::printf("ok\n");
    return 0;
}
