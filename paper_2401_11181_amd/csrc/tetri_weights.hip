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
        const int L = p.ctx[b];
        if (L < 0 || L > p.max_blocks * kPage || L >= p.score_stride) continue;      // (longer than the caller said)
        const int j = blockIdx.x * kAddKeys + threadIdx.x * 4;
        const size_t head = (size_t)b * p.Hq + (size_t)kh * p.g;
        if (j < L) {
            float *w = p.weights + ((size_t)p.bt[(size_t)b * p.max_blocks + j / kPage] * p.Hkv + kh) * kPage + j % kPage;
            f32x4 x = *reinterpret_cast<global_f32x4 *>((uintptr_t)w);
            const float *row = p.scores + head * p.score_stride + j;
            for (int h = 0; h < p.g; ++h, row += p.score_stride) {
                const f32x4 t = *reinterpret_cast<global_f32x4 *>((uintptr_t)row);
                const float lse = p.lse[head + h];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] += j + i < L ? __builtin_amdgcn_exp2f(t[i] - lse) : 0.f;
            }
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

// Finds tile `tile` when the tiles of all segments are numbered segment after segment; `count` gives a segment's.  False past the last.
template <class F>
__device__ inline bool find_segment(const WeighParams &p, int tile, int lane, F count, Segment &x)
{
    int base = 0;
    for (int s0 = 0; s0 < p.S; s0 += 64) {
        const int s = s0 + lane;
        int first = 0, n = 0, L = 0, tiles = 0;
        if (s < p.S) {
            first = min(max(p.cu[s], 0), p.C);
            n = min(max(p.cu[s + 1], first), p.C) - first;
            L = p.ctx[s];
            // (a segment that is longer than the caller said, or than the block table can describe, is left out)
            if (n > 0 && L >= 0 && L <= p.max_ctx && L <= p.max_blocks * kPage - n) tiles = count(n, L);
        }
        int incl = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
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
// products, the vector pipe 768 for its 2048 exponentials (16 cycles per 64 of them) with an addition and a multiplication-addition
// each: that is the bound where there are many rows.
constexpr int kSub = 2;                  // blocks of 32 rows that a wavefront keeps
constexpr int kStreamBytes = 8192;       // a tile of 32 rows of 128 16-bit values

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
// Key `key` of a segment (cached: through the block table; otherwise the chunk's own row) for kv head kh.
template <int D, bool FP8>
__device__ __forceinline__ void load_key(const WeighParams &p, const Segment &x, int kh, bool cached, int key, int half, bf16x8 (&f)[D / 16])
{
    if (cached) {
        constexpr int RB = FP8 ? D : 2 * D;
        const int page = p.bt[(size_t)x.s * p.max_blocks + key / kPage];
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
// row.  The reference is the largest score of the row's first tile and stays so while the sum stays below 2^64: in fp32 a large
// sum is as exact as a small one.
template <int D, bool FP8, int RW>
__global__ __launch_bounds__(256, 2) void weigh_rows_kernel(WeighParams p)
{
    constexpr int KSTEPS = D / 16, KW = 4 / RW, DEPTH = KW == 4 ? 2 : 4;
    __shared__ __attribute__((aligned(1024))) char smem[KW * DEPTH * kStreamBytes];
    __shared__ float2 met[4][32 * kSub];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int rw = wave % RW, kw = wave / RW;            // which rows, which stream
    const int kh = blockIdx.x % p.Hkv, rest = blockIdx.x / p.Hkv, part = rest % p.parts;
    Segment x;
    if (!find_segment(p, rest / p.parts, lane, [&](int n, int) { return (min(n, p.last) * p.g + 32 * kSub * RW - 1) / (32 * kSub * RW); }, x)) return;
    const int row0 = (x.local * RW + rw) * 32 * kSub;    // the wavefront's first row
    bf16x8 qf[kSub][KSTEPS];
    int t[kSub];                                         // the lane's rows see new keys 0..t
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
        const int r = min(row0 + 32 * i + l32, x.rows - 1);
        t[i] = x.t0 + magic_div(r, p.g_magic);
        load_rows<D>(reinterpret_cast<const char *>(p.q + query_row(p, x, kh, r) * D), half, qf[i]);
    }
    const int t_first = __builtin_amdgcn_readfirstlane(x.t0 + magic_div(min(row0, x.rows - 1), p.g_magic));
    const int t_last = __builtin_amdgcn_readfirstlane(x.t0 + magic_div(min((x.local + 1) * RW * 32 * kSub, x.rows) - 1, p.g_magic));    // of the workgroup
    const int old_tiles = (x.L + 31) / 32, tiles = old_tiles + t_last / 32 + 1;
    const int each = (tiles + p.parts - 1) / p.parts, begin = min(tiles, part * each), end = min(tiles, begin + each);
    float m[kSub], l[kSub];
#pragma unroll
    for (int i = 0; i < kSub; ++i) m[i] = -1e30f, l[i] = 0.f;
    const const_i32 *table = (const const_i32 *)(uintptr_t)(p.bt + (size_t)x.s * p.max_blocks);
    char *ring = smem + kw * (DEPTH * kStreamBytes);
    const uint32_t ring_lds = lds_address(ring);

    // tiles [from, to) of all of them
    auto stream = [&](auto codes_, int from, int to) {
        constexpr bool CODES = decltype(codes_)::value;
        typedef StreamTile<D, CODES> T;
        constexpr int MY = (T::NI + RW - 1) / RW;        // load instructions of a wavefront
        const uint32_t base = tile_base<D, CODES>(lane);
        auto issue = [&](int it, int slot) {
            it = min(it, to - 1);                        // (past the end: the last tile once more, so that the waits below count the same)
            const uint32_t lds = ring_lds + slot * kStreamBytes;
            const bool cached = it < old_tiles;
            const int key0 = 32 * (cached ? it : it - old_tiles);
#pragma unroll
            for (int j = 0; j < MY; ++j) {
                const int i = (MY * rw + j) % T::NI;
                const int r = T::RPI * i + lane / T::CH, chunk = (lane % T::CH) ^ T::swizzle(r);
                const char *src;
                if (cached) {
                    // (the last tile's rows past the end: what the last page holds)
                    const int page = table[min(key0 + T::RPI * i, x.L - 1) / kPage];
                    src = reinterpret_cast<const char *>(p.pages) + ((size_t)page * 2 * p.Hkv + kh) * (kPage * T::RB) + (r % kPage) * T::RB;
                } else {
                    src = reinterpret_cast<const char *>(p.k_new) + ((size_t)(x.first + min(key0 + r, x.n - 1)) * p.Hkv + kh) * (2 * D);
                }
                dma16(src + chunk * 16, lds + i * 1024);
            }
        };
        const int steps = (to - from + KW - 1) / KW;     // of every stream of the workgroup
        if (steps <= 0) return;
        lds_barrier();                                   // (the ring's last tiles have been read)
#pragma unroll
        for (int i = 0; i < DEPTH - 1; ++i) issue(from + kw + KW * i, i);
        for (int i = 0; i < steps; ++i) {
            const int it = from + kw + KW * i;
            wait_vm<MY *(DEPTH - 2)>();
            lds_barrier();                               // the tile is there, and everybody is done with the one before
            issue(it + KW * (DEPTH - 1), (i + DEPTH - 1) % DEPTH);
            const bool cached = it < old_tiles;
            const int key0 = 32 * (cached ? it : it - old_tiles);
            if (it >= to) continue;
            bf16x8 kf[KSTEPS];
            read_tile<D, CODES>(ring + (i % DEPTH) * kStreamBytes, base, kf);
            const float c = CODES ? p.c_codes : p.c;
            const bool masked = cached ? key0 + 32 > x.L : key0 + 31 > t_first;
            f32x16 sc[kSub];
#pragma unroll
            for (int b = 0; b < kSub; ++b) {
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[b][v] = 0.f;
#pragma unroll
                for (int s = 0; s < KSTEPS; ++s) sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[b][s], sc[b], 0, 0, 0);
            }
            if (masked) {                                // (as scores, so that their weight is 0 under any reference)
                const float none = c < 0.f ? INFINITY : -INFINITY;
#pragma unroll
                for (int b = 0; b < kSub; ++b) {
                    const int most = cached ? x.L - 1 : t[b];
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (key0 + 8 * (v / 4) + 4 * half + v % 4 > most) sc[b][v] = none;
                }
            }
#pragma unroll
            for (int b = 0; b < kSub; ++b) {
                float sum = l[b];
#pragma unroll
                for (int v = 0; v < 16; ++v) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][v], c, -m[b]));
                if (__builtin_amdgcn_ballot_w64(!(sum <= 0x1p64f))) {
                    // a row's first tile, or one far above it: another reference
                    float mx = sc[b][0] * c;
#pragma unroll
                    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, sc[b][v] * c);
                    const float m_new = fmaxf(m[b], mx);
                    sum = l[b] * __builtin_amdgcn_exp2f(m[b] - m_new);
                    m[b] = m_new;
#pragma unroll
                    for (int v = 0; v < 16; ++v) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][v], c, -m_new));
                }
                l[b] = sum;
            }
        }
        wait_vm<0>();
    };
    if constexpr (FP8) {
        const int cut = min(max(old_tiles, begin), end);
        stream(std::true_type(), begin, cut);
        stream(std::false_type(), cut, end);
    } else {
        stream(std::false_type(), begin, end);
    }
    // the halves of a wavefront (their references differ), then the streams
#pragma unroll
    for (int i = 0; i < kSub; ++i) {
        const float m2 = half_swap_max(m[i]), l2 = half_swap_sum(l[i] * __builtin_amdgcn_exp2f(m[i] - m2));
        if (half == 0) met[wave][32 * i + l32] = make_float2(m2, l2);
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
        p.stats[query_row(p, x, kh, r) * p.parts + part] = make_float2(ms, sum);
    }
}

// Second pass: the weights.  A wavefront keeps 64 keys of one kv head and the workgroup goes over the query rows that see any of its 256; S = Q K^T:
// a lane has a key.  The logarithms of the rows' sums are put together from the parts for 256 rows at a time.
template <int D, bool FP8>
__global__ __launch_bounds__(256, 2) void weigh_keys_kernel(WeighParams p)
{
    constexpr int KSTEPS = D / 16, DEPTH = 4, KEYS = 4 * 32 * kSub, BATCH = 256;
    typedef StreamTile<D, false> T;
    constexpr int MY = T::NI / 4;
    __shared__ __attribute__((aligned(1024))) char ring[DEPTH * kStreamBytes];
    __shared__ __attribute__((aligned(16))) float minus_lse[BATCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int kh = blockIdx.x % p.Hkv;
    const uint32_t base = tile_base<D, false>(lane), ring_lds = lds_address(ring);
    for (int item = blockIdx.x / p.Hkv;; item += gridDim.x / p.Hkv) {
        Segment x;
        if (!find_segment(p, item, lane, [&](int n, int L) { return (L + KEYS - 1) / KEYS + (n + KEYS - 1) / KEYS; }, x)) return;
        const int old_tiles = (x.L + KEYS - 1) / KEYS;
        const bool cached = x.local < old_tiles;
        const int tile0 = KEYS * (cached ? x.local : x.local - old_tiles), keys = cached ? x.L : x.n;
        const int key0 = tile0 + 32 * kSub * wave;       // the wavefront's first
        bf16x8 kf[kSub][KSTEPS];
#pragma unroll
        for (int b = 0; b < kSub; ++b) load_key<D, FP8>(p, x, kh, cached, min(key0 + 32 * b + l32, keys - 1), half, kf[b]);
        const float c = FP8 && cached ? p.c_codes : p.c;
        float sum[kSub];
#pragma unroll
        for (int b = 0; b < kSub; ++b) sum[b] = 0.f;
        // (the rows in front of the first that sees a key of the tile are left out)
        const int from = cached ? 0 : max(0, tile0 - x.t0) * p.g / 32, to = (x.rows + 31) / 32;
        auto issue = [&](int rt, int slot) {
            rt = min(rt, to - 1);
#pragma unroll
            for (int j = 0; j < MY; ++j) {
                const int i = MY * wave + j, r = T::RPI * i + lane / T::CH;
                const size_t row = query_row(p, x, kh, min(rt * 32 + r, x.rows - 1));
                dma16(reinterpret_cast<const char *>(p.q + row * D) + ((lane % T::CH) ^ T::swizzle(r)) * 16, ring_lds + slot * kStreamBytes + i * 1024);
            }
        };
        lds_barrier();                                   // (everybody is done with the item before)
#pragma unroll
        for (int i = 0; i < DEPTH - 1; ++i) issue(from + i, i);
        for (int rt = from; rt < to; ++rt) {
            const int i = rt - from;
            if (i % (BATCH / 32) == 0) {
                lds_barrier();
                const int r = rt * 32 + tid;
                float neg = -INFINITY;                   // rows past the end: weight 0
                if (r < x.rows) {
                    const float2 *z = p.stats + query_row(p, x, kh, r) * p.parts;
                    float ms = z[0].x, l = z[0].y;
                    for (int k = 1; k < p.parts; ++k) {
                        const float m_new = fmaxf(ms, z[k].x);
                        l = __builtin_fmaf(z[k].y, __builtin_amdgcn_exp2f(z[k].x - m_new), l * __builtin_amdgcn_exp2f(ms - m_new));
                        ms = m_new;
                    }
                    neg = -(ms + __builtin_amdgcn_logf(l));
                }
                minus_lse[tid] = neg;
                wait_vm<0>();                            // (the loads above have been waited for out of turn)
            } else {
                wait_vm<MY *(DEPTH - 2)>();
            }
            lds_barrier();
            issue(rt + DEPTH - 1, (i + DEPTH - 1) % DEPTH);
            bf16x8 qf[KSTEPS];
            read_tile<D, false>(ring + (i % DEPTH) * kStreamBytes, base, qf);
            f32x4 neg[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) neg[v] = *reinterpret_cast<const f32x4 *>(minus_lse + (i % (BATCH / 32)) * 32 + 8 * v + 4 * half);
            const bool masked = !cached && key0 + 32 * kSub - 1 > x.t0 + magic_div(rt * 32, p.g_magic);
            f32x16 sc[kSub];
#pragma unroll
            for (int b = 0; b < kSub; ++b) {
#pragma unroll
                for (int v = 0; v < 16; ++v) sc[b][v] = 0.f;
#pragma unroll
                for (int s = 0; s < KSTEPS; ++s) sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[s], kf[b][s], sc[b], 0, 0, 0);
            }
#pragma unroll
            for (int b = 0; b < kSub; ++b) {
                if (masked) {
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int row = x.t0 + magic_div(rt * 32 + 8 * (v / 4) + 4 * half + v % 4, p.g_magic);
                        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][v], c, neg[v / 4][v % 4]));
                        sum[b] += key0 + 32 * b + l32 <= row ? w : 0.f;
                    }
                } else {
#pragma unroll
                    for (int v = 0; v < 16; ++v) sum[b] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][v], c, neg[v / 4][v % 4]));
                }
            }
        }
        wait_vm<0>();
#pragma unroll
        for (int b = 0; b < kSub; ++b) {
            const float total = half_swap_sum(sum[b]);
            const int key = key0 + 32 * b + l32;
            if (half == 0 && key < keys) {
                const int slot = cached ? key : x.L + key;
                float *w = p.weights + ((size_t)p.bt[(size_t)x.s * p.max_blocks + slot / kPage] * p.Hkv + kh) * kPage + slot % kPage;
                *w = cached ? *w + total : total;
            }
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
    const auto rows_kernel = p.row_waves == 4 ? weigh_rows_kernel<D, FP8, 4> : p.row_waves == 2 ? weigh_rows_kernel<D, FP8, 2> : weigh_rows_kernel<D, FP8, 1>;
    hipLaunchKernelGGL(rows_kernel, dim3((unsigned)(row_tiles * p.parts * p.Hkv)), dim3(256), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t key_tiles = (int64_t)p.S * ((p.max_ctx + 255) / 256) + p.C / 256 + p.S;
    const int64_t abreast = std::max<int64_t>(1, (8 * (int64_t)num_cus + p.Hkv - 1) / p.Hkv);
    hipLaunchKernelGGL((weigh_keys_kernel<D, FP8>), dim3((unsigned)(std::min(key_tiles, abreast) * p.Hkv)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

hipError_t tetri_launch_weigh(int head_dim, bool fp8_pool, const WeighParams &p, int num_cus, hipStream_t stream)
{
    if (head_dim == 128) return fp8_pool ? launch_weigh<128, true>(p, num_cus, stream) : launch_weigh<128, false>(p, num_cus, stream);
    if (head_dim == 64) return fp8_pool ? launch_weigh<64, true>(p, num_cus, stream) : launch_weigh<64, false>(p, num_cus, stream);
    return hipErrorInvalidValue;
}
