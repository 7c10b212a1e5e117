// Accumulated attention weight of cached tokens for gfx950: what decode iterations and the rows of a prefill chunk give to the
// keys, kept beside the paged pool as one float per (page, kv head, slot).  The weight of key j under a query row is
//     p_j = exp2(t_j - lse),   t_j = scale * log2(e) * q . K_j,   lse = log2 sum_i exp2(t_i)
// and a slot gets the sum over the rows that see it and over the query heads that share its kv head.  It is the column sum of a
// softmax, so no weight is known before the last key of its row has been seen: everything here is in two passes.  Scores,
// exponentials and sums are fp32; nothing is rounded to fewer bits.
#include <algorithm>

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

// Fragment of 32 rows of a matrix product's operand: 8 values of d per lane and step, from a row of 16-bit values or of codes.
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
// Query row r of a segment.
template <int D>
__device__ __forceinline__ size_t query_row(const WeighParams &p, const Segment &x, int kh, int r)
{
    return (size_t)(x.first + x.t0 + r / p.g) * p.Hq + (size_t)kh * p.g + r % p.g;
}

// First pass: reference exponent and sum of the softmax of every row over a part of its keys.  A workgroup has 32 rows of one kv head
// and a part of the keys in tiles of 32, its wavefronts take the tiles in turn; S^T = K Q^T, so that a lane has one row.
template <int D, bool FP8>
__global__ __launch_bounds__(256) void weigh_rows_kernel(WeighParams p)
{
    constexpr int KSTEPS = D / 16;
    __shared__ float2 met[4][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, l32 = lane & 31;
    const int kh = blockIdx.x % p.Hkv, rest = blockIdx.x / p.Hkv, part = rest % p.parts;
    Segment x;
    if (!find_segment(p, rest / p.parts, lane, [&](int n, int) { return (min(n, p.last) * p.g + 31) / 32; }, x)) return;
    const int r = min(x.local * 32 + l32, x.rows - 1);
    const size_t row = query_row<D>(p, x, kh, r);
    bf16x8 qf[KSTEPS], kf[KSTEPS];
    load_rows<D>(reinterpret_cast<const char *>(p.q + row * D), half, qf);
    const int t = x.t0 + r / p.g;                        // this lane's row sees new keys 0..t
    const int t_last = x.t0 + min(x.local * 32 + 31, x.rows - 1) / p.g;
    const int old_tiles = (x.L + 31) / 32, tiles = old_tiles + t_last / 32 + 1;
    const int each = (tiles + p.parts - 1) / p.parts, begin = part * each, end = min(tiles, begin + each);
    float m = -INFINITY, l = 0.f;
    for (int it = begin + wave; it < end; it += 4) {
        const bool cached = it < old_tiles;
        const int key0 = 32 * (cached ? it : it - old_tiles);
        load_key<D, FP8>(p, x, kh, cached, min(key0 + l32, (cached ? x.L : x.n) - 1), half, kf);
        f32x16 sc;
#pragma unroll
        for (int v = 0; v < 16; ++v) sc[v] = 0.f;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[s], sc, 0, 0, 0);
        const float c = FP8 && cached ? p.c * p.k_scale : p.c;
        const int most = cached ? x.L - 1 : t;           // last key that this lane's row sees
        float mx = -INFINITY;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int key = key0 + 8 * (v / 4) + 4 * half + v % 4;
            sc[v] = key <= most ? sc[v] * c : -INFINITY;
            mx = fmaxf(mx, sc[v]);
        }
        const float m_new = fmaxf(m, mx);
        if (m_new > -INFINITY) {
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < 16; ++v) sum += __builtin_amdgcn_exp2f(sc[v] - m_new);
            l = __builtin_fmaf(l, __builtin_amdgcn_exp2f(m - m_new), sum);
            m = m_new;
        }
    }
    // the halves of a wavefront, then the wavefronts
    const float m2 = half_swap_max(m);
    const float l2 = half_swap_sum(m2 > -INFINITY ? l * __builtin_amdgcn_exp2f(m - m2) : 0.f);
    if (half == 0) met[wave][l32] = make_float2(m2, l2);
    __syncthreads();
    if (tid < 32 && x.local * 32 + tid < x.rows) {
        float ms = met[0][tid].x, sum = 0.f;
#pragma unroll
        for (int i = 1; i < 4; ++i) ms = fmaxf(ms, met[i][tid].x);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (met[i][tid].x > -INFINITY) sum = __builtin_fmaf(met[i][tid].y, __builtin_amdgcn_exp2f(met[i][tid].x - ms), sum);
        p.stats[row * p.parts + part] = make_float2(ms, sum);
    }
}

// Second pass: the weights.  A workgroup has 128 keys of one kv head, a wavefront 32 of them, whose fragments stay in registers while it goes
// over the rows that see them; S = Q K^T, so that a lane has one key and adds over the rows by itself.
template <int D, bool FP8>
__global__ __launch_bounds__(256) void weigh_keys_kernel(WeighParams p)
{
    constexpr int KSTEPS = D / 16;
    __shared__ __attribute__((aligned(16))) float lse[32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, l32 = lane & 31;
    const int kh = blockIdx.x % p.Hkv;
    for (int item = blockIdx.x / p.Hkv;; item += gridDim.x / p.Hkv) {
        Segment x;
        if (!find_segment(p, item, lane, [&](int n, int L) { return (L + 127) / 128 + (n + 127) / 128; }, x)) return;
        const int old_tiles = (x.L + 127) / 128;
        const bool cached = x.local < old_tiles;
        const int tile0 = 128 * (cached ? x.local : x.local - old_tiles), keys = cached ? x.L : x.n;
        const int key = tile0 + 32 * wave + l32;
        bf16x8 kf[KSTEPS], qf[KSTEPS];
        load_key<D, FP8>(p, x, kh, cached, min(key, keys - 1), half, kf);
        const float c = FP8 && cached ? p.c * p.k_scale : p.c;
        float sum = 0.f;
        // (the rows in front of the first that sees a key of the tile are left out)
        const int from = cached ? 0 : max(0, tile0 - x.t0) * p.g / 32;
        for (int rt = from; rt * 32 < x.rows; ++rt) {
            const size_t row = query_row<D>(p, x, kh, min(rt * 32 + l32, x.rows - 1));
            load_rows<D>(reinterpret_cast<const char *>(p.q + row * D), half, qf);
            __syncthreads();                             // everybody is done with the rows before
            if (tid < 32) {
                float ms = -INFINITY, l = 0.f;
                for (int i = 0; i < p.parts; ++i) {
                    const float2 z = p.stats[row * p.parts + i];
                    if (z.x > -INFINITY) {
                        const float m_new = fmaxf(ms, z.x);
                        l = __builtin_fmaf(z.y, __builtin_amdgcn_exp2f(z.x - m_new), l * __builtin_amdgcn_exp2f(ms - m_new));
                        ms = m_new;
                    }
                }
                lse[tid] = rt * 32 + tid < x.rows ? ms + __builtin_amdgcn_logf(l) : INFINITY;
            }
            __syncthreads();
            f32x16 sc;
#pragma unroll
            for (int v = 0; v < 16; ++v) sc[v] = 0.f;
#pragma unroll
            for (int s = 0; s < KSTEPS; ++s) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf[s], kf[s], sc, 0, 0, 0);
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int i = 8 * (v / 4) + 4 * half + v % 4;
                const bool sees = cached || key <= x.t0 + (rt * 32 + i) / p.g;
                sum += sees ? __builtin_amdgcn_exp2f(__builtin_fmaf(sc[v], c, -lse[i])) : 0.f;
            }
        }
        const float total = half_swap_sum(sum);
        if (half == 0 && key < keys) {
            const int slot = cached ? key : x.L + key;
            float *w = p.weights + ((size_t)p.bt[(size_t)x.s * p.max_blocks + slot / kPage] * p.Hkv + kh) * kPage + slot % kPage;
            *w = cached ? *w + total : total;
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
    const int64_t row_tiles = rows / 32 + p.S;
    hipLaunchKernelGGL((weigh_rows_kernel<D, FP8>), dim3((unsigned)(row_tiles * p.parts * p.Hkv)), dim3(256), 0, stream, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t key_tiles = (int64_t)p.S * ((p.max_ctx + 127) / 128) + p.C / 128 + p.S;
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
