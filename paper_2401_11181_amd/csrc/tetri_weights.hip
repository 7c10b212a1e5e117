// Accumulated attention weight of cached tokens for gfx950: what decode iterations and the rows of a prefill chunk give to the
// keys, kept beside the paged pool as one float per (page, kv head, slot).  The weight of key j under a query row is
//     p_j = exp2(t_j - lse),   t_j = scale * log2(e) * q . K_j,   lse = log2 sum_i exp2(t_i)
// and a slot gets the sum over the rows that see it and over the query heads that share its kv head.  It is the column sum of a
// softmax, so no weight is known before the last key of its row has been seen: everything here is in two passes.  Scores,
// exponentials and sums are fp32; nothing is rounded to fewer bits.
#include <algorithm>
#include <type_traits>

#include "attn_common.h"

namespace {

using namespace tetri_dev;

typedef __attribute__((address_space(1))) const f32x4 global_f32x4;
typedef __attribute__((address_space(1))) f32x4 global_f32x4_w;
typedef __attribute__((address_space(1))) float global_f32_w;

// ---------------------------------------------------------------- decode
// The decode kernel has written every score t and every (request, query head)'s lse; a lane turns four neighbouring keys' scores
// into weights, over the g heads of a kv head.
constexpr int kAddKeys = 1024;      // keys of a workgroup

__global__ __launch_bounds__(256) void add_weights_kernel(AddWeightsParams p)
{
    const int kh = blockIdx.y;
    for (int b = blockIdx.z; b < p.B; b += gridDim.z) {
        const int L = max(p.ctx[b], 0);                  // (a length below 0 is 0, as for the attention and the cache)
        if (L > p.max_ctx) continue;                     // (longer than the caller said)
        const int j = blockIdx.x * kAddKeys + threadIdx.x * 4;
        const size_t head = (size_t)b * p.Hq + (size_t)kh * p.g;
        if (j < L) {
            float *w = p.weights + ((size_t)p.bt[(size_t)b * p.max_blocks + j / kPage] * p.Hkv + kh) * kPage + j % kPage;
            f32x4 x = *reinterpret_cast<global_f32x4 *>((uintptr_t)w);
            const float *row = p.scores + head * p.score_stride + j;
            f32x4 given = {0.f, 0.f, 0.f, 0.f};          // (summed by itself: added to x, which may be large, head by head it could vanish)
            for (int h = 0; h < p.g; ++h, row += p.score_stride) {
                const f32x4 t = *reinterpret_cast<global_f32x4 *>((uintptr_t)row);
                const float lse = p.lse[head + h];
#pragma unroll
                for (int i = 0; i < 4; ++i) given[i] += j + i < L ? __builtin_amdgcn_exp2f(t[i] - lse) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] += given[i];
            if (j + 4 <= L) {
                *reinterpret_cast<global_f32x4_w *>((uintptr_t)w) = x;
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (j + i < L) *reinterpret_cast<global_f32_w *>((uintptr_t)(w + i)) = x[i];
            }
        }
        // the new token's slot holds nothing yet
        if (p.append && blockIdx.x == 0 && threadIdx.x == 0 && L < p.max_blocks * kPage) {
            float x = 0.f;
            for (int h = 0; h < p.g; ++h) {
                const float t = p.new_scores ? p.new_scores[head + h] : p.scores[(head + h) * p.score_stride + L];
                x += __builtin_amdgcn_exp2f(t - p.lse[head + h]);
            }
            p.weights[((size_t)p.bt[(size_t)b * p.max_blocks + L / kPage] * p.Hkv + kh) * kPage + L % kPage] = x;
        }
    }
}

// ---------------------------------------------------------------- prefill
// A segment's last rows, as seen by one kv head: row r of `rows` is token t0 + r / g, query head kh * g + r % g.
struct Segment {
    int s, first, n, L;       // segment, its first chunk row, its rows, cached tokens
    int t0, rows;             // first token looked at, query rows
    int local;                // tile inside the segment
};

// What finds a workgroup's segment: leading arguments of the kernels, in registers when a wavefront starts (the structure behind them is a
// memory read away).
struct Lookup {
    const int32_t *cu, *ctx;
    int S, C, max_tokens, max_ctx, last, g;
};

// Finds tile `tile` when the tiles of all segments are numbered segment after segment; `count` gives a segment's.  False past the last.
template <class F>
__device__ __forceinline__ bool find_segment(const Lookup &p, int tile, int lane, F count, Segment &x)
{
    int base = 0;
    for (int s0 = 0; s0 < p.S; s0 += 64) {
        const int s = s0 + lane, m = min(p.S - s0, 64);
        int first = 0, n = 0, L = 0, tiles = 0;
        if (lane < m) {
            first = min(max(p.cu[s], 0), p.C);
            n = min(max(p.cu[s + 1], first), p.C) - first;
            L = p.ctx[s];
            // (a segment that is longer than the caller said, or than the block table can describe, is left out)
            if (n > 0 && L >= 0 && L <= p.max_ctx && L <= p.max_tokens - n) tiles = count(n, L);
        }
        int incl = tiles;
#pragma unroll 1
        for (int d = 1; d < m; d <<= 1) {
            const int up = __shfl_up(incl, d);
            if (lane >= d) incl += up;
        }
        incl += base;
        const unsigned long long hit = __ballot(tile < incl && tile >= incl - tiles);
        if (hit) {
            const int src = __builtin_ctzll(hit);
            x.s = s0 + src;
            x.first = __builtin_amdgcn_readlane(first, src);
            x.n = __builtin_amdgcn_readlane(n, src);
            x.L = __builtin_amdgcn_readlane(L, src);
            x.local = tile - __builtin_amdgcn_readlane(incl - tiles, src);
            x.t0 = max(0, x.n - p.last);
            x.rows = (x.n - x.t0) * p.g;
            return true;
        }
        base = __builtin_amdgcn_readlane(incl, 63);
    }
    return false;
}

// Both passes are the same product with the parts changed: a wavefront keeps the fragments of 64 rows of one operand in registers (first
// pass: query rows, second: keys) and goes over tiles of 32 rows of the other, which come through rings in LDS; a lane has two
// columns of the result, and whatever is summed it sums by itself.  The matrix pipe needs 512 cycles for a step's 64 x 32 x 128
// products, the vector pipe as many for its 2048 exponentials (8 cycles per 64 of them) with an addition and a multiplication-addition
// each.  So that both are at work, the products of one block of 32 x 32 scores stand between the exponentials of the block before, a matrix
// instruction to two elements.  (2048 rows behind 14336 tokens, 32/8 heads, where the card's power is what bounds it: 535 us, 470 if all
// values are the same; one after the other 579; 528 to 606 on different cards.  Two products of that size by the library's rate for large
// matrices: 432.)
constexpr int kSub = 2;                  // blocks of 32 rows that a wavefront keeps
constexpr int kStreamBytes = 8192;       // a tile of 32 rows of 128 16-bit values

// next = a b; meanwhile element(v) for v = 0 .. 15 gives the exponents of the weights of the block before, whose sum is added to `sum`.
template <int KSTEPS, class F>
__device__ __forceinline__ void products_and_weights(const bf16x8 (&a)[KSTEPS], const bf16x8 (&b)[KSTEPS], f32x16 &next, float &sum, F element)
{
    constexpr int EACH = 16 / KSTEPS;
    float t[EACH], w[EACH];
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.f;
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[s], b[s], acc, 0, 0, 0);
        if (s == 0) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) t[i] = element(i);
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i) sum += w[i];
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) w[i] = __builtin_amdgcn_exp2f(t[i]);
        if (s + 1 < KSTEPS) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) t[i] = element((s + 1) * EACH + i);
        }
        asm volatile("" : "+v"(sum));                    // (a sum whose use is far away would be taken there)
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) sum += w[i];
    next = acc;
}

// Rows of 16-bit values (or codes) as they lie in a tile in LDS: 16-byte chunks XOR-ed by the row (see attn_common.h).
template <int D, bool CODES> struct StreamTile {
    static constexpr int RB = CODES ? D : 2 * D, CH = RB / 16, RPI = 1024 / RB, NI = 32 / RPI;     // a load instruction moves RPI rows
    static __device__ __forceinline__ constexpr int swizzle(int row) { return CODES ? (D == 128 ? row & 7 : (row >> 2) & 3) : k_swizzle<D>(row); }
};

// Fragments of 32 rows of a tile in LDS: 8 values of d per lane and step.
template <int D, bool CODES> __device__ __forceinline__ void read_tile(const char *tile, uint32_t base, bf16x8 (&f)[D / 16])
{
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        if constexpr (CODES) {
            const uint2 x = *reinterpret_cast<const uint2 *>(tile + (base ^ (s << 4)));
            f[s] = codes_to_bf16(x.x, x.y);
        } else {
            f[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4 *>(tile + (base ^ (s << 5))));
        }
    }
}
template <int D, bool CODES> __device__ __forceinline__ uint32_t tile_base(int lane)
{
    const int row = lane & 31, half = lane >> 5, swz = StreamTile<D, CODES>::swizzle(row);
    return row * StreamTile<D, CODES>::RB + (CODES ? (swz << 4) + 8 * half : (half ^ swz) << 4);
}

// Bit v: element v of a block of scores, row 8 * (v / 4) + v % 4 (and 4 * half, which the caller takes off), lies in front of row `end`.
// (As bits, for comparisons of which one follows from another become a chain of selections.)
__device__ __forceinline__ uint32_t rows_below(int end)
{
    const int e = min(max(end, 0), 32);
    uint32_t bits = (1u << (e / 8 * 4 + min(e % 8, 4))) - 1u;
    asm volatile("" : "+v"(bits));
    return bits;
}

// 16 bytes per lane from base + off to LDS (see dma16; base is wave-uniform).
__device__ __forceinline__ void dma16_at(const void *base, uint32_t off, uint32_t lds)
{
    dma16(reinterpret_cast<const char *>(uniform_ptr(base)) + off, lds);
}

// Fragments are in their registers from here on.  (Without this the compiler waits for them where they are used, in the loop, and there for every
// load to LDS that is in flight with them.)
template <int KSTEPS> __device__ __forceinline__ void loaded(bf16x8 (&f)[KSTEPS])
{
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) asm volatile("" : "+v"(f[s]));
}

// Fragments of 32 rows straight from memory, a row to a lane.
template <int D> __device__ __forceinline__ void load_rows(const char *row, int half, bf16x8 (&f)[D / 16])
{
    const global_u32x4 *at = reinterpret_cast<const global_u32x4 *>((uintptr_t)row) + half;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) f[s] = __builtin_bit_cast(bf16x8, u32x4(at[2 * s]));
}
template <int D> __device__ __forceinline__ void load_codes(const char *row, int half, bf16x8 (&f)[D / 16])
{
    const __attribute__((address_space(1))) u32x2 *at = reinterpret_cast<const __attribute__((address_space(1))) u32x2 *>((uintptr_t)row) + half;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        const u32x2 x = at[2 * s];
        f[s] = codes_to_bf16(x[0], x[1]);
    }
}
// Key `key` of a segment (cached: in page `page`; otherwise the chunk's own row) for kv head kh.
template <int D, bool FP8>
__device__ __forceinline__ void load_key(const WeighParams &p, const Segment &x, int kh, bool cached, int page, int key, int half, bf16x8 (&f)[D / 16])
{
    if (cached) {
        constexpr int RB = FP8 ? D : 2 * D;
        const char *row = reinterpret_cast<const char *>(p.pages) + (((size_t)page * 2 * p.Hkv + kh) * kPage + key % kPage) * RB;
        if constexpr (FP8) load_codes<D>(row, half, f);
        else load_rows<D>(row, half, f);
    } else {
        load_rows<D>(reinterpret_cast<const char *>(p.k_new + ((size_t)(x.first + key) * p.Hkv + kh) * D), half, f);
    }
}
// Query row r of a segment, as (chunk row, head).
__device__ __forceinline__ size_t query_row(const WeighParams &p, const Segment &x, int kh, int r)
{
    const int t = magic_div(r, p.g_magic);
    return (size_t)(x.first + x.t0 + t) * p.Hq + (size_t)kh * p.g + (r - t * p.g);
}

// First pass: reference exponent and sum of the softmax of every row over a part of its keys.  RW wavefronts share a stream of key tiles,
// each with 64 rows of its own; the 4 / RW streams of a workgroup take the tiles of the part in turn.  S^T = K Q^T: a lane has a
// row.  The reference is the largest score of the row's first tile and stays so as long as the sum is below 2^100: in fp32 a large
// sum is as exact as a small one.
template <int D, bool FP8, int RW>
__global__ __launch_bounds__(256, 2) void weigh_rows_kernel(const int32_t *cu, const int32_t *ctx, int S, int C, int max_tokens, int max_ctx, int last, int g,
                                                            int Hkv, int parts, WeighParams p)
{
    constexpr int KSTEPS = D / 16, KW = 4 / RW, DEPTH = KW == 4 ? 2 : 4;
    __shared__ __attribute__((aligned(1024))) char smem[KW * DEPTH * kStreamBytes];
    __shared__ float2 met[4][32 * kSub];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int rw = wave % RW, kw = wave / RW;            // which rows, which stream
    const int kh = blockIdx.x % Hkv, rest = blockIdx.x / Hkv, part = rest % parts;
    Segment x;
    if (!find_segment(Lookup{cu, ctx, S, C, max_tokens, max_ctx, last, g}, rest / parts, lane,
                      [&](int n, int) { return (min(n, last) * g + 32 * kSub * RW - 1) / (32 * kSub * RW); }, x)) return;
    const int row0 = (x.local * RW + rw) * 32 * kSub;    // the wavefront's first row
    // the wavefront's rows come through its part of the ring
    bf16x8 qf[kSub][KSTEPS];
    int t[kSub];                                         // the lane's rows see new keys 0..t
#pragma unroll
    for (int i = 0; i < kSub; ++i) t[i] = x.t0 + magic_div(min(row0 + 32 * i + l32, x.rows - 1), p.g_magic);
    {
        typedef StreamTile<D, false> T;
        constexpr int AT_ONCE = KW == 1 ? 1 : kSub;      // blocks of 32 rows
        char *mine = smem + wave * (AT_ONCE * kStreamBytes);
#pragma unroll
        for (int b0 = 0; b0 < kSub; b0 += AT_ONCE) {
#pragma unroll
            for (int b = 0; b < AT_ONCE; ++b)
#pragma unroll
                for (int i = 0; i < T::NI; ++i) {
                    const int r = T::RPI * i + lane / T::CH;
                    const size_t row = query_row(p, x, kh, min(row0 + 32 * (b0 + b) + r, x.rows - 1));
                    dma16(reinterpret_cast<const char *>(p.q + row * D) + (((lane % T::CH) ^ T::swizzle(r)) << 4), lds_address(mine) + b * kStreamBytes + i * 1024);
                }
            wait_vm<0>();
#pragma unroll
            for (int b = 0; b < AT_ONCE; ++b) {
                read_tile<D, false>(mine + b * kStreamBytes, tile_base<D, false>(lane), qf[b0 + b]);
                loaded(qf[b0 + b]);
            }
        }
    }
    const int t_first = __builtin_amdgcn_readfirstlane(x.t0 + magic_div(min(row0, x.rows - 1), p.g_magic));
    const int t_last = __builtin_amdgcn_readfirstlane(x.t0 + magic_div(min((x.local + 1) * RW * 32 * kSub, x.rows) - 1, p.g_magic));    // of the workgroup
    const int old_tiles = (x.L + 31) / 32, tiles = old_tiles + t_last / 32 + 1;
    const int each = (tiles + p.parts - 1) / p.parts, begin = min(tiles, part * each), end = min(tiles, begin + each);
    float m[kSub], l[kSub];
    const const_i32 *table = (const const_i32 *)(uintptr_t)(p.bt + (size_t)x.s * p.max_blocks);
    char *ring = smem + kw * (DEPTH * kStreamBytes);
    const uint32_t ring_lds = lds_address(ring);

    f32x16 sc[kSub];                                     // block 1's weights are taken one step late
    auto rescue = [&](int b, float c, float before) {
        // a row's first tile, or one far above its reference: another one
        if (__builtin_amdgcn_ballot_w64(!(l[b] <= 0x1p64f))) {
            float mx = sc[b][0] * c;
#pragma unroll
            for (int v = 1; v < 16; ++v) mx = fmaxf(mx, sc[b][v] * c);
            const float m_new = fmaxf(m[b], half_swap_max(mx));      // (the other half-wave has other keys of the same row)
            float sum = before * __builtin_amdgcn_exp2f(m[b] - m_new);
            m[b] = m_new;
#pragma unroll
            for (int v = 0; v < 16; ++v) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][v], c, -m_new));
            l[b] = sum;
        }
    };
    // tiles [from, to) of all of them
    auto stream = [&](auto codes_, bool careful, int from, int to) {
        constexpr bool CODES = decltype(codes_)::value;
        typedef StreamTile<D, CODES> T;
        constexpr int MY = (T::NI + RW - 1) / RW;        // load instructions of a wavefront
        int ln = lane;
        asm volatile("" : "+v"(ln));                     // (what follows from it is worked out here, not kept from one stream to the next)
        static_assert(MY <= 2 || MY == 4 || MY == 8, "they move a whole number of pages, or a part of one");
        const uint32_t base = tile_base<D, CODES>(ln);
        const int i0 = MY * rw % T::NI;                  // the first of them; its lane's row and chunk
        const int r0 = T::RPI * i0 + ln / T::CH;
        uint32_t page_off[MY];                           // where in its page a row's 16 bytes are, less the instruction's own 1 KB
#pragma unroll
        for (int j = 0; j < MY; ++j) {
            const int r = r0 + T::RPI * j;
            page_off[j] = (uint32_t)((r % kPage) * T::RB + (((ln % T::CH) ^ T::swizzle(r)) << 4));
        }
        const char *pool = reinterpret_cast<const char *>(p.pages) + (size_t)kh * (kPage * T::RB);
        const char *rows = reinterpret_cast<const char *>(p.k_new + ((size_t)x.first * p.Hkv + kh) * D);
        const size_t page_bytes = (size_t)2 * p.Hkv * (kPage * T::RB);
        const uint32_t row_bytes = (uint32_t)p.Hkv * 2 * D;
        constexpr int PAGES = (MY * T::RPI + kPage - 1) / kPage, PER = MY / PAGES;   // pages that they read from, and how many read from one
        int page[PAGES];                                 // of the tile that is issued next
        // (rows of the last tile past the end: what the last page holds; tiles of new keys have no pages)
        auto find_pages = [&](int it) {
#pragma unroll
            for (int j = 0; j < PAGES; ++j) page[j] = table[(uint32_t)max(min(32 * it + T::RPI * i0 + kPage * j, x.L - 1), 0) / kPage];
        };
        auto issue = [&](int it, int slot) {
            it = min(it, to - 1);                        // (past the end: the last tile once more, so that the waits below count the same)
            const uint32_t lds = ring_lds + slot * kStreamBytes + i0 * 1024;
            if (it < old_tiles) {
#pragma unroll
                for (int j = 0; j < MY; ++j) dma16_at(pool + page[j / PER] * page_bytes, page_off[j], lds + j * 1024);
            } else {
                const int key0 = 32 * (it - old_tiles);
#pragma unroll
                for (int j = 0; j < MY; ++j) {
                    const int r = r0 + T::RPI * j;
                    dma16_at(rows, (uint32_t)min(key0 + r, x.n - 1) * row_bytes + (((ln % T::CH) ^ T::swizzle(r)) << 4), lds + j * 1024);
                }
            }
            find_pages(min(it + KW, to - 1));
        };
        const int steps = (to - from + KW - 1) / KW;     // of every stream of the workgroup
        if (steps <= 0) return;
        const float c = CODES ? p.c_codes : p.c, none = c < 0.f ? INFINITY : -INFINITY;
        const char *at = ring;
        // scores that a row does not see are infinite, so that their weight is 0 under any reference: those of the last cached tile, of the
        // tiles from that of the wavefront's first row on, and of those past the end that even out the streams
        const int partial = x.L % 32 != 0 ? old_tiles - 1 : -1, mask_from = min(old_tiles + (t_first + 1) / 32, to);
        auto mask = [&](int it, int b) {
            if (it == partial || it >= mask_from) {
                const int most = it >= to ? -1 : it < old_tiles ? x.L - 1 - 32 * it - 4 * half : t[b] - 32 * (it - old_tiles) - 4 * half;
                const uint32_t seen = rows_below(most + 1);
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (!(seen & 1u << v)) sc[b][v] = none;
            }
        };
        lds_barrier();                                   // (the ring's last tiles have been read)
        find_pages(min(from + kw, to - 1));
#pragma unroll
        for (int i = 0; i < DEPTH - 1; ++i) issue(from + kw + KW * i, i);
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[1][v] = none;
        bf16x8 kf[2][KSTEPS];
        auto arrive = [&](int i, bf16x8 (&f)[KSTEPS]) {  // step i's tile
            wait_vm<MY *(DEPTH - 2)>();
            lds_barrier();                               // it is there, and everybody has read the one before
            issue(from + kw + KW * (i + DEPTH - 1), (i + DEPTH - 1) % DEPTH);
            read_tile<D, CODES>(at + (i % DEPTH) * kStreamBytes, base, f);
        };
        auto step = [&](int i, bf16x8 (&f)[KSTEPS], bf16x8 (&f_next)[KSTEPS]) {
            const int it = from + kw + KW * i;
            float before = l[1];
            products_and_weights<KSTEPS>(f, qf[0], sc[0], l[1], [&](int v) { return __builtin_fmaf(sc[1][v], c, -m[1]); });
            if (careful || i == 1) rescue(1, c, before);
            mask(it, 0);
            if (i + 1 < steps) arrive(i + 1, f_next);
            before = l[0];
            products_and_weights<KSTEPS>(f, qf[1], sc[1], l[0], [&](int v) { return __builtin_fmaf(sc[0][v], c, -m[0]); });
            if (careful || i == 0) rescue(0, c, before);
            mask(it, 1);
        };
        arrive(0, kf[0]);
        for (int i = 0; i < steps; i += 2) {
            step(i, kf[0], kf[1]);
            if (i + 1 < steps) step(i + 1, kf[1], kf[0]);
        }
        const float before = l[1];
#pragma unroll
        for (int v = 0; v < 16; ++v) l[1] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[1][v], c, -m[1]));
        rescue(1, c, before);
        wait_vm<0>();
    };
    // The reference is looked at in a row's first tile and then only if the sum has got too large: once more with a look at every tile.  (All
    // wavefronts of the workgroup go along, for the barriers.)
    __shared__ int overflow;
    if (tid == 0) overflow = 0;
    for (int careful = 0; careful < 2; ++careful) {
#pragma unroll
        for (int i = 0; i < kSub; ++i) m[i] = -1e30f, l[i] = 0.f;
        if constexpr (FP8) {
            const int cut = min(max(old_tiles, begin), end);
            stream(std::true_type(), careful, begin, cut);
            stream(std::false_type(), careful, cut, end);
        } else {
            stream(std::false_type(), careful, begin, end);
        }
        if (careful) break;
        if (__builtin_amdgcn_ballot_w64(!(l[0] <= 0x1p100f) || !(l[1] <= 0x1p100f))) overflow = 1;     // (sums of these do not overflow either)
        __syncthreads();
        if (!overflow) break;
    }
    // the halves of a wavefront, then the streams
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
        const float both = half_swap_sum(l[i]);
        if (half == 0) met[wave][32 * i + l32] = make_float2(m[i], both);
    }
    __syncthreads();
    const int r = x.local * RW * 32 * kSub + tid;
    if (tid < RW * 32 * kSub && r < x.rows) {
        const int w = tid / (32 * kSub), col = tid % (32 * kSub);
        float ms = met[w][col].x, sum = 0.f;
#pragma unroll
        for (int i = 1; i < KW; ++i) ms = fmaxf(ms, met[w + i * RW][col].x);
#pragma unroll
        for (int i = 0; i < KW; ++i) sum = __builtin_fmaf(met[w + i * RW][col].y, __builtin_amdgcn_exp2f(met[w + i * RW][col].x - ms), sum);
        const size_t row = query_row(p, x, kh, r);
        if (parts == 1) p.lse[row] = ms + __builtin_amdgcn_logf(sum);
        else p.stats[row * parts + part] = make_float2(ms, sum);
    }
}

// Between the passes, where the keys were cut: a row's parts put together, 16 lanes to a row.  (By every workgroup of the second pass for the rows
// it needs, this took as long as a launch: each of them waits for it, and it takes their registers.)
__global__ __launch_bounds__(256) void join_parts_kernel(const float2 *stats, float *lse, int parts, uint32_t rows)
{
    const uint32_t row = blockIdx.x * 16 + threadIdx.x / 16;
    if (row >= rows) return;
    const float2 *z = stats + (size_t)row * parts;
    float m = -1e30f, l = 0.f;
    for (int k = threadIdx.x % 16; k < parts; k += 16) {
        const float2 y = z[k];
        const float m_new = fmaxf(m, y.x);
        l = __builtin_fmaf(y.y, __builtin_amdgcn_exp2f(y.x - m_new), l * __builtin_amdgcn_exp2f(m - m_new));
        m = m_new;
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
        const float m2 = __shfl_xor(m, d), l2 = __shfl_xor(l, d), m_new = fmaxf(m, m2);
        l = __builtin_fmaf(l2, __builtin_amdgcn_exp2f(m2 - m_new), l * __builtin_amdgcn_exp2f(m - m_new));
        m = m_new;
    }
    if (threadIdx.x % 16 == 0) lse[row] = m + __builtin_amdgcn_logf(l);
}

// Second pass: the weights.  (The keys' fragments come straight from memory, beside the first tiles of rows: by way of LDS, in full cache lines, they
// were a trip of their own, and 16896 keys of 8 kv heads took 26 us instead of 18.)  A wavefront keeps 32 * SUB keys of one kv head and the workgroup goes over the query rows that see any of its
// 128 * SUB; S = Q K^T: a lane has a key.  64 keys to a wavefront halve what is read from LDS; 32 where that leaves compute units without
// work.
template <int D, bool FP8, int SUB>
__global__ __launch_bounds__(256, SUB == 2 ? 2 : 3) void weigh_keys_kernel(const int32_t *cu, const int32_t *ctx, int S, int C, int max_tokens, int max_ctx, int last,
                                                                          int g, int Hkv, WeighParams p)
{
    constexpr int KSTEPS = D / 16, DEPTH = 4, KEYS = 4 * 32 * SUB, BATCH = 256;
    typedef StreamTile<D, false> T;
    constexpr int MY = T::NI / 4;
    __shared__ __attribute__((aligned(1024))) char ring[DEPTH * kStreamBytes];
    __shared__ __attribute__((aligned(16))) float minus_lse[2 * BATCH];   // of this batch of rows and the one before
    __shared__ int no_sum[2];                            // last row that has no finite sum (-1: none), of this item and the one before
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int kh = blockIdx.x % Hkv;
    const uint32_t base = tile_base<D, false>(lane), ring_lds = lds_address(ring);
    if (tid < 2) no_sum[tid] = -1;
    for (int item = blockIdx.x / Hkv, turn = 0;; item += gridDim.x / Hkv, turn ^= 1) {
        Segment x;
        if (!find_segment(Lookup{cu, ctx, S, C, max_tokens, max_ctx, last, g}, item, lane,
                          [&](int n, int L) { return (L + KEYS - 1) / KEYS + (n + KEYS - 1) / KEYS; }, x)) return;
        const int old_tiles = (x.L + KEYS - 1) / KEYS;
        const bool cached = x.local < old_tiles;
        const int tile0 = KEYS * (cached ? x.local : x.local - old_tiles), keys = cached ? x.L : x.n;
        const int key0 = tile0 + 32 * SUB * wave;        // the wavefront's first
        const float c = FP8 && cached ? p.c_codes : p.c;
        float sum[2] = {0.f, 0.f};
        // (the rows in front of the first that sees a key of the tile are left out)
        const int from = cached ? 0 : max(0, tile0 - x.t0) * g / 32, to = (x.rows + 31) / 32, steps = to - from;
        // where the lane's query rows of the next tile are, from the segment's first on: they go up by 32 rows, that is by 32 / g tokens and
        // 32 % g heads; rows past the end are the last one
        uint32_t off[MY], head[MY];
        const uint32_t token_bytes = (uint32_t)p.Hq * 2 * D, per_tile = 32u / (uint32_t)p.g * token_bytes + 32u % (uint32_t)p.g * 2 * D;
        const uint32_t last_off = (uint32_t)(x.n - 1 - x.t0) * token_bytes + (uint32_t)(p.g - 1) * 2 * D;
        const char *queries = reinterpret_cast<const char *>(p.q + query_row(p, x, kh, 0) * D);
#pragma unroll
        for (int j = 0; j < MY; ++j) {
            const int r = from * 32 + T::RPI * (MY * wave + j) + lane / T::CH, token = magic_div(r, p.g_magic);
            head[j] = r - token * p.g;
            off[j] = token * token_bytes + head[j] * 2 * D;
        }
        auto issue = [&](int slot) {
#pragma unroll
            for (int j = 0; j < MY; ++j) {
                const int i = MY * wave + j, r = T::RPI * i + lane / T::CH;
                dma16_at(queries, min(off[j], last_off) + (((lane % T::CH) ^ T::swizzle(r)) << 4), ring_lds + slot * kStreamBytes + i * 1024);
                head[j] += 32u % (uint32_t)p.g;
                off[j] += per_tile;
                if (head[j] >= (uint32_t)p.g) {
                    head[j] -= p.g;
                    off[j] += token_bytes - (uint32_t)p.g * 2 * D;
                }
            }
        };
        f32x16 sc[2];
        const float none = c < 0.f ? INFINITY : -INFINITY;
        // a key of the chunk is seen by row first_row[b] and those behind it
        int first_row[SUB];
#pragma unroll
        for (int b = 0; b < SUB; ++b) first_row[b] = cached ? 0 : (key0 + 32 * b + l32 - x.t0) * g;
        const int all_see = cached ? 0 : (key0 + 32 * SUB - 1 - x.t0) * g;
        auto mask = [&](int rt, int b, f32x16 &s) {
            if (rt * 32 < all_see) {
                const uint32_t blind = rows_below(first_row[b] - rt * 32 - 4 * half);
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (blind & 1u << v) s[v] = none;
            }
        };
        lds_barrier();                                   // (everybody is done with the item before)
        if (tid == 0) no_sum[turn ^ 1] = -1;             // (of the item before, for the next one)
#pragma unroll
        for (int i = 0; i < DEPTH - 1; ++i) issue(i);
        bf16x8 kf[SUB][KSTEPS];
        float *weight[SUB];                              // of the lane's keys, and what they have already
        float sum_before[SUB];
#pragma unroll
        for (int b = 0; b < SUB; ++b) {
            const int key = min(key0 + 32 * b + l32, keys - 1), slot = cached ? key : x.L + key;
            const int page = p.bt[(size_t)x.s * p.max_blocks + slot / kPage];
            weight[b] = p.weights + ((size_t)page * Hkv + kh) * kPage + slot % kPage;
            load_key<D, FP8>(p, x, kh, cached, page, key, half, kf[b]);
            sum_before[b] = cached ? *weight[b] : 0.f;
        }
        // minus the logarithms of 256 rows' sums, from row r0 on; rows past the end: -infinity, that is weight 0.  So are rows whose sum is NaN or
        // infinite, for what such a row gives is NaN, also to keys that it does not see; those that see the last of these get NaN at the end.
        auto sums = [&](int r0, float *to_lds) {
            const int r = r0 + tid;
            float minus = -INFINITY;
            if (r < x.rows) {
                const float lse = p.lse[query_row(p, x, kh, r)];
                if (fabsf(lse) < INFINITY) minus = -lse;
                else atomicMax(&no_sum[turn], r);
            }
            to_lds[tid] = minus;
        };
        if (steps > 0) sums(from * 32, minus_lse);
#pragma unroll
        for (int b = 0; b < SUB; ++b) {
            loaded(kf[b]);
            asm volatile("" : "+v"(sum_before[b]));
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[1][v] = none;
        bf16x8 qf[SUB][KSTEPS];
        auto arrive = [&](int i, bf16x8 (&f)[KSTEPS]) {
            if (i > 0 && i % (BATCH / 32) == 0) sums((from + i) * 32, minus_lse + (i & (BATCH / 32)) * 32);
            wait_vm<MY *(DEPTH - 2)>();
            lds_barrier();
            issue((i + DEPTH - 1) % DEPTH);
            read_tile<D, false>(ring + (i % DEPTH) * kStreamBytes, base, f);
        };
        f32x4 neg[4];
        auto read_neg = [&](int i) {                     // of tile i
#pragma unroll
            for (int v = 0; v < 4; ++v) neg[v] = *reinterpret_cast<const f32x4 *>(minus_lse + (i & (2 * BATCH / 32 - 1)) * 32 + 8 * v + 4 * half);
        };
        if constexpr (SUB == 2) {
            // block 1's weights are taken one step late
            auto step = [&](int i, bf16x8 (&f)[KSTEPS], bf16x8 (&f_next)[KSTEPS]) {
                read_neg(i > 0 ? i - 1 : 0);
                products_and_weights<KSTEPS>(f, kf[0], sc[0], sum[1], [&](int v) { return __builtin_fmaf(sc[1][v], c, neg[v / 4][v % 4]); });
                read_neg(i);
                mask(from + i, 0, sc[0]);
                if (i + 1 < steps) arrive(i + 1, f_next);
                products_and_weights<KSTEPS>(f, kf[1], sc[1], sum[0], [&](int v) { return __builtin_fmaf(sc[0][v], c, neg[v / 4][v % 4]); });
                mask(from + i, 1, sc[1]);
            };
            if (steps > 0) arrive(0, qf[0]);
            for (int i = 0; i < steps; i += 2) {
                step(i, qf[0], qf[1]);
                if (i + 1 < steps) step(i + 1, qf[1], qf[0]);
            }
        } else {
            // a tile's weights are taken one step late
            auto step = [&](int i, f32x16 &s, const f32x16 &before) {
                arrive(i, qf[0]);
                read_neg(i > 0 ? i - 1 : 0);
                products_and_weights<KSTEPS>(qf[0], kf[0], s, sum[0], [&](int v) { return __builtin_fmaf(before[v], c, neg[v / 4][v % 4]); });
                mask(from + i, 0, s);
            };
            for (int i = 0; i < steps; i += 2) {
                step(i, sc[0], sc[1]);
                if (i + 1 < steps) step(i + 1, sc[1], sc[0]);
                else sc[1] = sc[0];
            }
        }
        // the last block
        if (steps > 0) {
            read_neg(steps - 1);
#pragma unroll
            for (int v = 0; v < 16; ++v) sum[SUB - 1] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[1][v], c, neg[v / 4][v % 4]));
        }
        wait_vm<0>();
#pragma unroll
        for (int b = 0; b < SUB; ++b) {
            float total = half_swap_sum(sum[b]);
            if (max(first_row[b], 0) <= no_sum[turn]) total = NAN;
            if (half == 0 && key0 + 32 * b + l32 < keys) *weight[b] = sum_before[b] + total;
        }
    }
}

}  // namespace

hipError_t tetri_launch_add_weights(const AddWeightsParams &p, int32_t max_ctx_len, hipStream_t stream)
{
    const dim3 grid((unsigned)(std::max(max_ctx_len, 1) + kAddKeys - 1) / kAddKeys, (unsigned)p.Hkv, (unsigned)std::min(p.B, 32768));
    hipLaunchKernelGGL(add_weights_kernel, grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

template <int D, bool FP8> static hipError_t launch_weigh(const WeighParams &p, int num_cus, hipStream_t stream)
{
    // upper bounds of the tiles: every segment may end in a partial one
    const int64_t rows = (int64_t)std::min<int64_t>(p.C, (int64_t)p.S * p.last) * p.g;
    const int64_t row_tiles = rows / (32 * kSub * p.row_waves) + p.S;
    const int max_tokens = p.max_blocks * kPage;
    const auto rows_kernel = p.row_waves == 4 ? weigh_rows_kernel<D, FP8, 4> : p.row_waves == 2 ? weigh_rows_kernel<D, FP8, 2> : weigh_rows_kernel<D, FP8, 1>;
    hipLaunchKernelGGL(rows_kernel, dim3((unsigned)(row_tiles * p.parts * p.Hkv)), dim3(256), 0, stream, p.cu, p.ctx, p.S, p.C, max_tokens, p.max_ctx, p.last, p.g,
                       p.Hkv, p.parts, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.parts > 1) {
        // (rows of the chunk that no segment's last rows are have no parts: what comes of them is not read)
        hipLaunchKernelGGL(join_parts_kernel, dim3((unsigned)(((int64_t)p.C * p.Hq + 15) / 16)), dim3(256), 0, stream, p.stats, p.lse, p.parts, (uint32_t)(p.C * p.Hq));
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    auto key_tiles = [&](int64_t keys) { return (int64_t)p.S * ((p.max_ctx + keys - 1) / keys) + p.C / keys + p.S; };
    const bool wide = p.wide_keys;
    // no more workgroups than are resident at a time: those beyond them would start when the first have ended
    const int64_t abreast = std::max<int64_t>(1, (wide ? 2 : 3) * (int64_t)num_cus / p.Hkv);
    const auto keys_kernel = wide ? weigh_keys_kernel<D, FP8, 2> : weigh_keys_kernel<D, FP8, 1>;
    hipLaunchKernelGGL(keys_kernel, dim3((unsigned)(std::min(key_tiles(wide ? 256 : 128), abreast) * p.Hkv)), dim3(256), 0, stream, p.cu, p.ctx, p.S, p.C, max_tokens,
                       p.max_ctx, p.last, p.g, p.Hkv, p);
    return hipGetLastError();
}

hipError_t tetri_launch_weigh(int head_dim, bool fp8_pool, const WeighParams &p, int num_cus, hipStream_t stream)
{
    if (head_dim == 128) return fp8_pool ? launch_weigh<128, true>(p, num_cus, stream) : launch_weigh<128, false>(p, num_cus, stream);
    if (head_dim == 64) return fp8_pool ? launch_weigh<64, true>(p, num_cus, stream) : launch_weigh<64, false>(p, num_cus, stream);
    return hipErrorInvalidValue;
}
