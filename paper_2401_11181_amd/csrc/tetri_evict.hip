// Eviction from the paged cache for gfx950: which slots of a request a kv head keeps, and the moves that bring them to the front of
// the cache.  A request with L cached tokens and n = min(L, keep) to be kept gives up e = L - n of them.  The last r = min(recent, n)
// slots always stay; of the slots in front of them, [0, L - r), the n - r with the largest weight do, the lowest slot first among
// equals.  Then
//   * a kept slot below n - r stays where it is;
//   * the k-th slot below n - r that is not kept (a hole) takes the k-th kept slot of [n - r, L - r): there are as many of each;
//   * slot n - r + i takes slot L - r + i: the newest tokens close up, in their order.
// So the last slots are the newest tokens again, which is all that the next eviction needs to know, and of the others, for whose order attention
// does not care, as few move as can.  (The newest all do, by e slots, however few are given up.)
#include "attn_common.h"

namespace {

using namespace tetri_dev;

constexpr int kDigits = 2048, kCandidates = 1024, kCompared = 128;

// Value of another lane (0 where there is none, or in rows that `rows` leaves out), without a trip through LDS.
template <int CTRL, int ROWS = 15> __device__ __forceinline__ int dpp(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 15, false); }

// Sum over this lane and those in front of it.
__device__ __forceinline__ int wave_scan(int x)
{
    x += dpp<0x111>(x);                                  // one, two, four and eight lanes up inside a row of 16
    x += dpp<0x112>(x);
    x += dpp<0x114>(x);
    x += dpp<0x118>(x);
    x += dpp<0x142, 10>(x);                              // the last lane of the row before to rows 1 and 3
    x += dpp<0x143, 12>(x);                              // lane 31 to rows 2 and 3
    return x;
}
// All bits of the eight lanes of a group.
__device__ __forceinline__ uint32_t or_eight(uint32_t x)
{
    x |= (uint32_t)dpp<0xB1>((int)x);                    // neighbours, pairs, then the two halves (all lanes of a half hold the same by now)
    x |= (uint32_t)dpp<0x4E>((int)x);
    return x | (uint32_t)dpp<0x141>((int)x);
}

// Sum over the threads in front of this one; `total`: of all.
template <int THREADS> __device__ __forceinline__ int block_scan(int x, int *wave_sums, int &total)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int incl = wave_scan(x);
    __syncthreads();                                     // (everybody is done with an earlier scan's sums)
    if (lane == 63) wave_sums[wave] = incl;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
        if (i < wave) before += wave_sums[i];
        total += wave_sums[i];
    }
    return before + incl - x;
}

// A weight as an integer in the same order: NaN below all others with -infinity, -0 as 0.
__device__ __forceinline__ uint32_t ordered(float w)
{
    if (w != w) w = -INFINITY;
    const uint32_t b = __builtin_bit_cast(uint32_t, w + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A histogram's additions.  Additions to one word of LDS come one after the other: so there are COPIES of every digit's count, next to each other,
// for a quarter of the lanes each where there are four; and weights of 0, of which there may be many, are counted by each lane for itself.
// (32768 weights, 16 wavefronts: 20000 cycles with one copy.)
constexpr uint32_t kZero = 0x80000000u;                  // ordered(0)
template <int COPIES> __device__ __forceinline__ void count_digit(uint32_t *hist, uint32_t u, int shift, uint32_t digits, bool in, int &zeros)
{
    if (in && u == kZero) ++zeros;
    if (in && u != kZero) atomicAdd(&hist[((u >> shift) & digits) * COPIES + threadIdx.x % COPIES], 1u);
}
template <int COPIES> __device__ __forceinline__ void count_zeros(uint32_t *hist, int shift, uint32_t digits, int zeros)
{
    if (zeros != 0) atomicAdd(&hist[((kZero >> shift) & digits) * COPIES + threadIdx.x % COPIES], (uint32_t)zeros);
}
template <int THREADS, int COPIES> __device__ __forceinline__ void clear_digits(uint32_t *hist)
{
    for (int i = threadIdx.x; i < kDigits * COPIES / 4; i += THREADS) reinterpret_cast<uint4 *>(hist)[i] = make_uint4(0u, 0u, 0u, 0u);
}
// Where the want-th largest is, from the largest digit down: its digit, how many are wanted of that digit, and how many there are.
template <int THREADS, int COPIES> __device__ __forceinline__ void find_digit(const uint32_t *hist, int want, int *wave_sums, int (&found)[3])
{
    constexpr int MINE = kDigits / THREADS;
    const int top = kDigits - 1 - MINE * threadIdx.x;    // this thread's digits: top, top - 1, ...
    int n[MINE], sum = 0, total;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        if constexpr (COPIES == 4) {
            const uint4 x = *reinterpret_cast<const uint4 *>(hist + 4 * (top - i));
            n[i] = (int)(x.x + x.y + x.z + x.w);
        } else {
            n[i] = (int)hist[top - i];
        }
        sum += n[i];
    }
    int before = block_scan<THREADS>(sum, wave_sums, total);
    if (before < want && before + sum >= want) {
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            if (before < want && before + n[i] >= want) {
                found[0] = top - i;
                found[1] = want - before;
                found[2] = n[i];
            }
            before += n[i];
        }
    }
    __syncthreads();
}

// Choice among up to THREADS * 4 * QUADS slots, by a workgroup per (request, kv head), which reads every weight once, into registers.
// The smallest kept weight is found by its first 11 bits (a histogram in LDS), then, among those that share them, by the next 11 and 10 bits;
// as soon as they are few they are put in a list, and when they are a handful they are compared with each other.  Then every slot's bit is known: kept or not.  Counts
// of bits in front of each word give every slot its rank, by which holes and the slots that fill them find each other in a list.
// What bounds it: the chain of steps, about 3 us of it three trips to memory, where there are few workgroups; among 32768 slots (17 us) 40 % of it are
// the additions to the first histogram.  (Counting only weights between two bounds that every fourth weight gives took longer, 18.4 us: it is the
// instructions that cost, however few lanes take part, and there is another pass.)
template <int THREADS, int QUADS>
__global__ __launch_bounds__(THREADS) void select_kernel(const int32_t *ctx, const int32_t *bt, const float *weights, int max_blocks, int Hkv, int max_ctx, int keep,
                                                         int recent, int32_t *slots, int32_t *new_lens)
{
    constexpr int MOST = THREADS * 4 * QUADS, WORDS = MOST / 32;
    constexpr int COPIES = THREADS > 256 ? 4 : 1;
    static_assert(WORDS <= THREADS && MOST <= 65536, "a word to a thread, slots in 16 bits");
    __shared__ __attribute__((aligned(16))) uint32_t hist[kDigits * COPIES];
    __shared__ uint32_t kept[WORDS], front[WORDS];       // front: equals, then kept slots in front of the word
    __shared__ __attribute__((aligned(16))) uint32_t candidate[kCandidates + 4];
    __shared__ uint16_t mover[MOST / 2];                 // (there are as many holes among `heavy` slots: at most half of all)
    __shared__ int wave_sums[THREADS / 64], found[3], candidates;
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.x / Hkv, kh = blockIdx.x - b * Hkv;
    const int L = min(min(max(ctx[b], 0), max_blocks * kPage), max_ctx);
    const int n = min(L, keep), r = min(recent, n), heavy = n - r, old = L - r;
    int32_t *to = slots + ((size_t)b * Hkv + kh) * keep;
    if (kh == 0 && tid == 0) new_lens[b] = n;
    if (L <= keep || heavy == 0) {
        for (int i = tid; i < keep; i += THREADS) to[i] = i < n ? i + (L - n) : -1;
        return;
    }
    const int32_t *row = bt + (size_t)b * max_blocks;
    uint32_t u[QUADS][4];                                // 0: no old slot
    {
        int page[QUADS];
#pragma unroll
        for (int q = 0; q < QUADS; ++q) page[q] = row[min(4 * (q * THREADS + tid), old - 1) / kPage];
#pragma unroll
        for (int q = 0; q < QUADS; ++q) {
            const int j = min(4 * (q * THREADS + tid), (old - 1) & ~3);
            const f32x4 w = *reinterpret_cast<__attribute__((address_space(1))) const f32x4 *>((uintptr_t)(weights + ((size_t)page[q] * Hkv + kh) * kPage + j % kPage));
#pragma unroll
            for (int i = 0; i < 4; ++i) u[q][i] = 4 * (q * THREADS + tid) + i < old ? ordered(w[i]) : 0u;
        }
    }
    uint32_t least = 0;                                  // the smallest kept weight, and how many of the equal ones are kept, of how many
    int want = heavy, equal = 0;
    bool listed = false;
    int known = 0;                                       // bits of `least`, from the top; the others are 0
    // (one loop; as three passes laid out one after the other 64 requests of up to 2048 tokens, 40 heads, took 15.2 us instead of 14.5)
    while (true) {
        const int shift = max(0, 21 - known);
        const uint32_t digits = (1u << (32 - known - shift)) - 1u;
        // those that agree with the digits so far lie this close above `least` (a slot that does not count, 0, lies far off)
        const uint32_t span = known == 0 ? 0xffffffffu : 1u << (32 - known);
        clear_digits<THREADS, COPIES>(hist);
        if (tid == 0) candidates = 0;
        __syncthreads();
        int zeros = 0;
        if (listed) {
            for (int k = tid; k < equal; k += THREADS) {
                const uint32_t c = candidate[k];
                count_digit<COPIES>(hist, c, shift, digits, c - least < span, zeros);
            }
        } else {
#pragma unroll
            for (int q = 0; q < QUADS; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) count_digit<COPIES>(hist, u[q][i], shift, digits, u[q][i] != 0 && u[q][i] - least < span, zeros);
        }
        count_zeros<COPIES>(hist, shift, digits, zeros);
        __syncthreads();
        const int in_list = equal;
        find_digit<THREADS, COPIES>(hist, want, wave_sums, found);
        least |= (uint32_t)found[0] << shift;
        want = found[1];
        equal = found[2];
        known = 32 - shift;
        if (want == equal || known == 32) break;         // (all that share the digits so far are kept)
        const uint32_t close = 1u << shift;
        if (!listed && equal <= kCandidates) {
            int mine = 0;
#pragma unroll
            for (int q = 0; q < QUADS; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) mine += u[q][i] - least < close;
            const int incl = wave_scan(mine);
            int at = 0;
            if (lane == 63) at = atomicAdd(&candidates, incl);
            at = __builtin_amdgcn_readlane(at, 63) + incl - mine;
#pragma unroll
            for (int q = 0; q < QUADS; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (u[q][i] - least < close) candidate[at++] = u[q][i];
        } else if (listed) {                             // (once more, only those that are left)
            uint32_t c[kCandidates / THREADS];
#pragma unroll
            for (int i = 0; i < kCandidates / THREADS; ++i) c[i] = i * THREADS + tid < in_list ? candidate[i * THREADS + tid] : 0u;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kCandidates / THREADS; ++i)
                if (c[i] - least < close) candidate[atomicAdd(&candidates, 1)] = c[i];
        }
        listed = listed || equal <= kCandidates;
        if (equal <= kCompared) {
            if (tid < 4) candidate[equal + tid] = 0;     // (no candidate is 0)
            __syncthreads();
            if (tid < equal) {
                const uint32_t c = candidate[tid];
                int above = 0, same = 0;
                for (int i = 0; i < equal; i += 4) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(candidate + i);
                    above += (x.x > c) + (x.y > c) + (x.z > c) + (x.w > c);
                    same += (x.x == c) + (x.y == c) + (x.z == c) + (x.w == c);
                }
                if (above < want && above + same >= want) {      // (so do all that are equal to it, with the same to say)
                    found[0] = (int)c;
                    found[1] = want - above;
                    found[2] = same;
                }
            }
            __syncthreads();
            least = (uint32_t)found[0];
            want = found[1];
            equal = found[2];
            break;
        }
        __syncthreads();                                 // (found has been read, the list is whole)
    }
    const bool all_equals = want == equal;
    // a bit for every old slot: kept, or equal to the smallest kept weight.  (Where all that share its first digits are kept, the others of its
    // bits are 0.)
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
        uint32_t more = 0, same = 0;
        if (all_equals) {
#pragma unroll
            for (int i = 0; i < 4; ++i) more |= (uint32_t)(u[q][i] >= least) << i;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                more |= (uint32_t)(u[q][i] > least) << i;
                same |= (uint32_t)(u[q][i] == least) << i;
            }
            same = or_eight(same << 4 * (tid & 7));
        }
        more = or_eight(more << 4 * (tid & 7));
        if ((tid & 7) == 0) {
            kept[(q * THREADS + tid) / 8] = more;
            front[(q * THREADS + tid) / 8] = same;
        }
    }
    __syncthreads();
    uint32_t mine = tid < WORDS ? kept[tid] : 0u;
    int total;
    if (!all_equals) {                                   // the first `want` of the equals
        uint32_t same = tid < WORDS ? front[tid] : 0u;
        for (int at = block_scan<THREADS>(__popc(same), wave_sums, total); same != 0 && at < want; same &= same - 1, ++at) mine |= same & -same;
        if (tid < WORDS) kept[tid] = mine;
    }
    const int before = block_scan<THREADS>(__popc(mine), wave_sums, total);
    if (tid < WORDS) front[tid] = before;
    __syncthreads();
    auto kept_before = [&](int j) -> int {               // (j < MOST)
        return front[j / 32] + __popc(kept[j / 32] & ((1u << (j % 32)) - 1u));
    };
    const int stay = kept_before(heavy);                 // (heavy < old)
    if (tid < WORDS) {                                   // the kept slots from `heavy` on, in order
        int at = before;
        uint32_t x = mine;
        if (32 * tid < heavy) {
            const uint32_t low = heavy - 32 * tid >= 32 ? ~0u : (1u << (heavy - 32 * tid)) - 1u;
            at += __popc(x & low);
            x &= ~low;
        }
        for (; x != 0; x &= x - 1, ++at) mover[at - stay] = (uint16_t)(32 * tid + __builtin_ctz(x));
    }
    __syncthreads();
    for (int i = tid; i < keep; i += THREADS) {
        int src = i < n ? i + (L - n) : -1;
        if (i < heavy) src = kept[i / 32] >> (i % 32) & 1 ? i : (int)mover[i - kept_before(i)];
        to[i] = src;
    }
}

// The same among any number of slots: the weights are read again for every digit.
constexpr int kSelectThreads = 1024;

__global__ __launch_bounds__(kSelectThreads) void select_many_kernel(SelectParams p)
{
    extern __shared__ uint32_t smem[];
    __shared__ int wave_sums[kSelectThreads / 64];
    __shared__ int found[3];
    const int words = (p.max_ctx + 31) / 32;
    uint32_t *hist = smem, *kept = hist + kDigits, *other = kept + words;    // other: equals, later counts
    const int tid = threadIdx.x, b = blockIdx.x / p.Hkv, kh = blockIdx.x - b * p.Hkv;
    const int L = min(min(max(p.ctx[b], 0), p.max_blocks * kPage), p.max_ctx);
    const int n = min(L, p.keep), r = min(p.recent, n), heavy = n - r, old = L - r;
    int32_t *to = p.slots + ((size_t)b * p.Hkv + kh) * p.keep;
    if (kh == 0 && tid == 0) p.new_lens[b] = n;
    if (L <= p.keep || heavy == 0) {
        for (int i = tid; i < p.keep; i += kSelectThreads) to[i] = i < n ? i + (L - n) : -1;
        return;
    }
    const int32_t *row = p.bt + (size_t)b * p.max_blocks;
    auto load4 = [&](int j) -> f32x4 {
        const size_t at = ((size_t)row[j / kPage] * p.Hkv + kh) * kPage + j % kPage;
        return *reinterpret_cast<__attribute__((address_space(1))) const f32x4 *>((uintptr_t)(p.weights + at));
    };
    uint32_t prefix = 0;
    int want = heavy;                                    // so many of those that agree with the prefix
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, above = pass == 1 ? 21 : 10;
        const uint32_t mask = pass == 2 ? 1023 : 2047;
        for (int i = tid; i < kDigits; i += kSelectThreads) hist[i] = 0;
        __syncthreads();
        int zeros = 0;
        for (int j = 4 * tid; j < old; j += 4 * kSelectThreads) {
            const f32x4 w = load4(j);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t u = ordered(w[i]);
                count_digit<1>(hist, u, shift, mask, j + i < old && (pass == 0 || ((u ^ prefix) >> above) == 0), zeros);
            }
        }
        count_zeros<1>(hist, shift, mask, zeros);
        __syncthreads();
        find_digit<kSelectThreads, 1>(hist, want, wave_sums, found);
        prefix |= (uint32_t)found[0] << shift;
        want = found[1];
    }
    const bool all_equals = want == found[2];            // of the weights equal to the smallest kept one, `want` are kept
    // a bit for every old slot: kept, or equal to the smallest kept weight
    for (int base = 0; base < words * 32; base += 4 * kSelectThreads) {
        const int j = base + 4 * tid;
        uint32_t more = 0, equal = 0;
        if (j < old) {
            const f32x4 w = load4(j);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t u = ordered(w[i]);
                if (j + i < old) {
                    more |= (uint32_t)(u > prefix || (all_equals && u == prefix)) << i;
                    equal |= (uint32_t)(u == prefix) << i;
                }
            }
        }
        more = or_eight(more << 4 * (tid & 7));
        equal = or_eight(equal << 4 * (tid & 7));
        if ((tid & 7) == 0 && j < words * 32) {
            kept[j / 32] = more;
            other[j / 32] = equal;
        }
    }
    __syncthreads();
    const int each = (words + kSelectThreads - 1) / kSelectThreads, w0 = min(words, tid * each), w1 = min(words, w0 + each);
    int total;
    if (!all_equals) {
        // the first `want` of the equals
        int mine = 0;
        for (int w = w0; w < w1; ++w) mine += __popc(other[w]);
        int at = block_scan<kSelectThreads>(mine, wave_sums, total);
        for (int w = w0; w < w1; ++w)
            for (uint32_t x = other[w]; x != 0 && at < want; x &= x - 1, ++at) kept[w] |= x & -x;
    }
    int mine = 0;
    for (int w = w0; w < w1; ++w) mine += __popc(kept[w]);
    int at = block_scan<kSelectThreads>(mine, wave_sums, total);
    for (int w = w0; w < w1; ++w) {
        other[w] = at;                                   // kept slots in front of the word
        at += __popc(kept[w]);
    }
    __syncthreads();
    auto kept_before = [&](int j) -> int {               // (j < words * 32)
        return other[j / 32] + __popc(kept[j / 32] & ((1u << (j % 32)) - 1u));
    };
    const int stay = heavy < words * 32 ? kept_before(heavy) : total;
    for (int i = tid; i < p.keep; i += kSelectThreads) {
        int src = i < n ? i + (L - n) : -1;
        if (i < heavy) {
            src = i;
            if (!(kept[i / 32] >> (i % 32) & 1)) {
                const int k = stay + i - kept_before(i);             // its token is kept slot number k
                int lo = 0, hi = words - 1;                          // the last word with at most k in front of it
                while (lo < hi) {
                    const int mid = (lo + hi + 1) / 2;
                    if ((int)other[mid] <= k) lo = mid;
                    else hi = mid - 1;
                }
                uint32_t x = kept[lo];
                for (int skip = k - (int)other[lo]; skip > 0; --skip) x &= x - 1;
                src = lo * 32 + __builtin_ctz(x | 0x80000000u);
            }
        }
        to[i] = src;
    }
}

// The moves in place.  A token's row of K and of V goes 16 bytes to a lane.  Two kinds:
//   * to the holes from behind the new end (slots n and up): no other move writes what it reads or reads what it writes, so
//     all of them may run at once.  A workgroup has 256 slots of one kv head: it looks up the pages of those that get another
//     token, a lane each, and moves just these, as many rows of both K and V at a time as keep the memory busy;
//   * those that have to do with the last r slots [n - r, n): what a hole takes from there, and the newest tokens that come there.  Slot n - r + i
//     may be read by two moves (by a hole's, and where e < r by that of slot n - r + i - e) before it is written.  One
//     workgroup for K and one for V goes over these slots in order: it reads a stretch of slots for the holes and the tokens that come into the
//     stretch, waits until all its reads have returned, and writes.  What it reads later lies behind what it has written.
// Neighbouring workgroups have different kv heads of the same slots: what is under way at a time lies in few pages.
constexpr int kCompactThreads = 256, kBack = 1024;

template <int RB>      // bytes of a row
__global__ __launch_bounds__(kCompactThreads) void compact_kernel(const int32_t *ctx, const int32_t *bt, const int32_t *slots, int max_blocks, int Hkv, int keep,
                                                                  int recent, int tiles, char *pages, float *weights)
{
    constexpr int LPR = RB / 16, STEP = kCompactThreads / LPR, ROWS = 4, STRETCH = ROWS * STEP;
    __shared__ int32_t hole[kBack];
    __shared__ int32_t moves[kCompactThreads][3];        // pages from and to, slots in them
    __shared__ int32_t wave_moves[kCompactThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lane_row = tid / LPR, chunk = tid % LPR;
    const int rest = blockIdx.x / Hkv, kh = blockIdx.x - rest * Hkv, b = rest / (tiles + 2), tile = rest - b * (tiles + 2) - 2;
    const int32_t *map = slots + ((size_t)b * Hkv + kh) * keep, *row = bt + (size_t)b * max_blocks;
    // how far the newest tokens come is the map's to say, not the length's: of a request longer than the max_ctx_len it was made under, the
    // tokens behind that are given up too
    const int newest = tile < 0 ? map[keep - 1] : 0;
    const int L = min(max(ctx[b], 0), max_blocks * kPage), n = keep, r = recent, heavy = n - r;
    if (L <= n) return;
    auto data = [&](int page, int slot, int kv) -> char * {
        return pages + ((((size_t)page * 2 + kv) * Hkv + kh) * kPage + slot) * RB + chunk * 16;
    };
    auto ld = [&](int page, int slot, int kv) -> u32x4 { return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(data(page, slot, kv))); };
    auto st = [&](int page, int slot, int kv, u32x4 v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(data(page, slot, kv))); };
    auto weight = [&](int page, int slot) -> float & { return weights[((size_t)page * Hkv + kh) * kPage + slot]; };
    if (tile >= 0) {
        const int to = tile * kCompactThreads + tid;
        const int from = to < heavy ? map[to] : -1;
        const bool move = from >= n && from < L;
        const unsigned long long moved = __ballot(move);
        if (lane == 0) wave_moves[wave] = __popcll(moved);
        int pf = 0, pt = 0;
        float w = 0.f;
        if (move) {
            pf = row[from / kPage];
            pt = row[to / kPage];
            w = weight(pf, from % kPage);
        }
        __syncthreads();
        int at = __popcll(moved & ((1ull << lane) - 1)), count = 0;
#pragma unroll
        for (int i = 0; i < kCompactThreads / 64; ++i) {
            if (i < wave) at += wave_moves[i];
            count += wave_moves[i];
        }
        if (move) {
            moves[at][0] = pf;
            moves[at][1] = pt;
            moves[at][2] = from % kPage | to % kPage << 16;
            weight(pt, to % kPage) = w;
        }
        __syncthreads();
        for (int m0 = 0; m0 < count; m0 += STRETCH) {
            u32x4 v[ROWS][2];
            int page_to[ROWS], slot_to[ROWS];
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const int m = m0 + i * STEP + lane_row;
                slot_to[i] = -1;
                if (m < count) {
                    const int page = moves[m][0], s = moves[m][2];
                    page_to[i] = moves[m][1];
                    slot_to[i] = s >> 16;
                    v[i][0] = ld(page, s & 0xffff, 0);
                    v[i][1] = ld(page, s & 0xffff, 1);
                }
            }
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
                if (slot_to[i] >= 0) {
                    st(page_to[i], slot_to[i], 0, v[i][0]);
                    st(page_to[i], slot_to[i], 1, v[i][1]);
                }
        }
        return;
    }
    if (newest < n || newest >= L) return;               // (the map moves nothing: no more than `keep` were chosen from)
    const int kv = tile + 2, e = newest - (n - 1);
    const bool weighs = kv == 0 && chunk == 0;           // these lanes move the weights as well
    for (int base = 0; base < r; base += kBack) {
        const int many = min(r - base, kBack);
        __syncthreads();
        for (int i = tid; i < many; i += kCompactThreads) hole[i] = -1;
        __syncthreads();
        for (int i0 = tid; i0 < heavy; i0 += 16 * kCompactThreads) {
            int at[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) at[k] = map[min(i0 + k * kCompactThreads, heavy - 1)];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int i = i0 + k * kCompactThreads, x = at[k] - heavy - base;
                if (i < heavy && x >= 0 && x < many) hole[x] = i;
            }
        }
        __syncthreads();
        for (int t0 = 0; t0 < many; t0 += STRETCH) {
            u32x4 old[ROWS], now[ROWS];
            float w_old[ROWS], w_now[ROWS];
            int to[ROWS], at[ROWS], page[ROWS], page_to[ROWS];
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const int x = t0 + i * STEP + lane_row;
                at[i] = x < many ? heavy + base + x : -1;
                to[i] = x < many ? hole[x] : -1;
                if (at[i] >= 0) {
                    page[i] = row[at[i] / kPage];
                    page_to[i] = row[max(to[i], 0) / kPage];
                    const int page_now = row[(at[i] + e) / kPage];
                    if (to[i] >= 0) {
                        old[i] = ld(page[i], at[i] % kPage, kv);
                        if (weighs) w_old[i] = weight(page[i], at[i] % kPage);
                    }
                    now[i] = ld(page_now, (at[i] + e) % kPage, kv);
                    if (weighs) w_now[i] = weight(page_now, (at[i] + e) % kPage);
                }
            }
            wait_vm<0>();
            __syncthreads();
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                if (to[i] >= 0) {
                    st(page_to[i], to[i] % kPage, kv, old[i]);
                    if (weighs) weight(page_to[i], to[i] % kPage) = w_old[i];
                }
                if (at[i] >= 0) {
                    st(page[i], at[i] % kPage, kv, now[i]);
                    if (weighs) weight(page[i], at[i] % kPage) = w_now[i];
                }
            }
        }
    }
}

}  // namespace

static size_t select_lds(int32_t max_ctx) { return ((size_t)kDigits + 2 * ((size_t)(max_ctx + 31) / 32)) * sizeof(uint32_t); }

hipError_t tetri_launch_select(const SelectParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)(p.B * p.Hkv));
    if (p.max_ctx <= 32768) {
        // as many threads as give each 8 to 32 weights: 64 requests of up to 2048 tokens, 40 heads, 2560 workgroups of 256 threads
        const auto launch = [&](auto kernel, int threads) {
            hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, p.ctx, p.bt, p.weights, p.max_blocks, p.Hkv, p.max_ctx, p.keep, p.recent, p.slots, p.new_lens);
        };
        if (p.max_ctx <= 2048) launch(select_kernel<256, 2>, 256);
        else if (p.max_ctx <= 8192) launch(select_kernel<512, 4>, 512);
        else if (p.max_ctx <= 16384) launch(select_kernel<1024, 4>, 1024);
        else launch(select_kernel<1024, 8>, 1024);
        return hipGetLastError();
    }
    const size_t lds = select_lds(p.max_ctx);
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(select_many_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(select_many_kernel, grid, dim3(kSelectThreads), lds, stream, p);
    return hipGetLastError();
}

template <int RB> static hipError_t launch_compact(const CompactParams &p, hipStream_t stream)
{
    const int tiles = (p.keep - p.recent + kCompactThreads - 1) / kCompactThreads;
    const int64_t wgs = (int64_t)p.B * p.Hkv * (tiles + 2);
    if (wgs > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL((compact_kernel<RB>), dim3((unsigned)wgs), dim3(kCompactThreads), 0, stream, p.ctx, p.bt, p.slots, p.max_blocks, p.Hkv, p.keep, p.recent, tiles,
                       p.pages, p.weights);
    return hipGetLastError();
}

hipError_t tetri_launch_compact(int row_bytes, const CompactParams &p, hipStream_t stream)
{
    if (row_bytes == 256) return launch_compact<256>(p, stream);
    if (row_bytes == 128) return launch_compact<128>(p, stream);
    if (row_bytes == 64) return launch_compact<64>(p, stream);
    return hipErrorInvalidValue;
}
