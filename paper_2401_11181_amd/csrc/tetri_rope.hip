// Queries and keys made ready for attention (gfx950): RMS norm of every head and rotation by position, out of the rows of a projection into
// the rows that the attention calls take, in one pass.
//
//   y = x * rsqrt(mean(x^2) + eps) * w          (left out where there is no w)
//   a', b' = a cos t - b sin t, b cos t + a sin t      for the pairs (a, b) of y, t = position * frequency of the pair
//
// Bound by memory: 4 bytes per element.  A wavefront takes a row, or some of its heads where rows are few: lane l works out pair l's cosine and sine once;
// then 16 or 8 lanes take a head each time, every lane always the same elements of it, so that its cosines, sines and weights stay in registers.  A
// lane's 8 elements are two pieces of 4 that are each other's pairs (where pairs are neighbours, or elements do not turn, the pieces are): no lane needs
// another one's elements.  (With 8 neighbouring elements a lane, the other halves by way of ds_bpermute: 8192 rows of 32/8 heads, 168 MB,
// 48.7 us, now 32.7: 5.1 TB/s.  Two instructions in flight leave room for eight wavefronts to a SIMD, so that those rows are one round: four 42.6.)
// The angle is taken in 64 bits, in turns, of which whole ones are dropped: with 32 bits of a position of 10^6 times a frequency of 1 an angle
// would be off by 0.06.  Everything behind that is 32-bit, rounded once.
#include <type_traits>

#include "attn_common.h"

namespace {

using namespace tetri_dev;

constexpr int kRowWaves = 4;

typedef __attribute__((address_space(1))) const u32x2 global_u32x2;

// The sum of x over the D / 8 lanes of a head, in every one of them.
template <int D> __device__ __forceinline__ float head_sum(float x)
{
    auto add = [&](auto ctrl) { x += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true)); };
    add(std::integral_constant<int, 0xb1>());            // lane ^ 1, lane ^ 2, then 4 lanes' sums from the other half of 8 and of 16 lanes
    add(std::integral_constant<int, 0x4e>());
    add(std::integral_constant<int, 0x141>());
    if constexpr (D == 128) add(std::integral_constant<int, 0x140>());
    return x;
}

// PAST: the rows are read past the caches, for calls whose rows do not stay there anyway (see the host).
template <int D, bool PAST>
__global__ __launch_bounds__(kRowWaves * 64, 8) void qk_norm_rope_kernel(RopeParams)
{
    typedef __attribute__((address_space(4))) const RopeParams const_params;
    const const_params *p = (const const_params *)__builtin_amdgcn_kernarg_segment_ptr();
    constexpr int LPH = D / 8, HPI = 64 / LPH, U = 2;    // lanes of a head, heads of an instruction, instructions in flight
    const int lane = threadIdx.x & 63;
    const int unit = blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = magic_div(unit, p->splits_magic), split = unit - row * p->splits;
    if (row >= p->rows) return;
    // A padding row is neither read nor written.  (One word more in front of a row's loads, which are then on their way while the segment is looked up: 512 rows of 40 heads 7.2 us, 7.1 without.)
    if (p->cu != nullptr && row >= ((const const_i32 *)(uintptr_t)p->cu)[p->S]) return;
    const int heads = p->Hq + p->Hkv, Hq = p->Hq, c = lane % LPH, pairs = p->pairs, adjacent = p->adjacent;

    // ---- a lane's pieces of a head: elements at .. at + 3 and other .. other + 3
    const bool turning = 8 * c < 2 * pairs;
    const int at = adjacent || !turning ? 8 * c : 4 * c, other = adjacent || !turning ? at + 4 : at + pairs;
    const uint16_t *q_row = p->q + (size_t)row * p->q_stride, *k_row = p->k + (size_t)row * p->k_stride;
    const int first = split * p->per_split * HPI, end = min(heads, first + p->per_split * HPI);
    if (first >= end) return;
    auto load = [](const uint16_t *from) -> u32x2 {
        global_u32x2 *g = reinterpret_cast<global_u32x2 *>((uintptr_t)from);
        if constexpr (PAST) return __builtin_nontemporal_load(g);
        else return *g;
    };
    u32x2 x[U][2];
    auto fetch = [&](int h0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = min(h0 + u * HPI + lane / LPH, end - 1);
            const uint16_t *src = h < Hq ? q_row + (size_t)h * D : k_row + (size_t)(h - Hq) * D;
            x[u][0] = load(src + at);
            x[u][1] = load(src + other);
        }
    };
    fetch(first);
    const uint16_t *q_weight = p->q_weight, *k_weight = p->k_weight;
    u32x2 wq[2] = {}, wk[2] = {};
    if (q_weight) {
        wq[0] = *reinterpret_cast<global_u32x2 *>((uintptr_t)(q_weight + at));
        wq[1] = *reinterpret_cast<global_u32x2 *>((uintptr_t)(q_weight + other));
    }
    if (k_weight) {
        wk[0] = *reinterpret_cast<global_u32x2 *>((uintptr_t)(k_weight + at));
        wk[1] = *reinterpret_cast<global_u32x2 *>((uintptr_t)(k_weight + other));
    }

    // ---- the row's position, by its segment or as given (for every axis)
    double position;
    const int pair = min(lane, pairs - 1);
    if (p->cu != nullptr) {
        int seg = 0;                                     // segments that end in front of the row or at it
        for (int s0 = 0; s0 < p->S; s0 += 64) {
            const bool before = s0 + lane < p->S && p->cu[min(s0 + lane, p->S - 1) + 1] <= row;
            seg += __builtin_popcountll(__builtin_amdgcn_ballot_w64(before));
        }
        if (seg >= p->S) return;                         // (cu written to while the launch runs: no address is formed from it)
        position = (double)((int64_t)p->ctx[seg] + row - p->cu[seg]);
    } else {
        position = (double)p->pos[(size_t)p->axis[pair] * p->rows + row];
    }
    // ---- pair `lane`'s cosine and sine, then those of this lane's four pairs
    constexpr double kTurn = 0.15915494309189533576888;  // 1 / (2 pi)
    const double turns = position * (double)p->freq[pair] * kTurn;
    const float part = (float)(turns - rint(turns));
    float mys, myc;
    sincospif(2.0f * part, &mys, &myc);
    float cs[4], sn[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        cs[j] = __shfl(myc, (4 * c + j) & 63, 64);
        sn[j] = __shfl(mys, (4 * c + j) & 63, 64);
    }

    auto value = [](const u32x2 &w, int j) -> float { return __builtin_bit_cast(float, (j & 1) ? w[j / 2] & 0xffff0000u : w[j / 2] << 16); };
    const bool any_norm = q_weight != nullptr || k_weight != nullptr, both = q_weight != nullptr && k_weight != nullptr;
    for (int h0 = first; h0 < end; h0 += U * HPI) {
        u32x2 y[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) { y[u][0] = x[u][0]; y[u][1] = x[u][1]; }
        if (h0 + U * HPI < end) fetch(h0 + U * HPI);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (h0 + u * HPI >= end) break;
            const int h = h0 + u * HPI + lane / LPH;
            const bool is_q = h < Hq;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = value(y[u][j / 4], j % 4);
            if (any_norm) {
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(v[j], v[j], sum);
                const float r = __builtin_amdgcn_rsqf(head_sum<D>(sum) * (1.0f / D) + p->eps);
                if (both || (is_q ? q_weight != nullptr : k_weight != nullptr)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] *= r * value(is_q ? wq[j / 4] : wk[j / 4], j % 4);
                }
            }
            if (turning) {                               // (not by way of a product with 0, which an infinity of the head's would make NaN)
                if (adjacent) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float a = v[2 * j], b = v[2 * j + 1];
                        v[2 * j] = a * cs[j] - b * sn[j];
                        v[2 * j + 1] = b * cs[j] + a * sn[j];
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float a = v[j], b = v[4 + j];
                        v[j] = a * cs[j] - b * sn[j];
                        v[4 + j] = b * cs[j] + a * sn[j];
                    }
                }
            }
            if (h < end) {
                uint16_t *to = is_q ? p->q_out + ((size_t)row * Hq + h) * D : p->k_out + ((size_t)row * p->Hkv + (h - Hq)) * D;
                bf16x4 r[2];
#pragma unroll
                for (int j = 0; j < 8; ++j) r[j / 4][j % 4] = (__bf16)v[j];
                *reinterpret_cast<global_u32x2_w *>((uintptr_t)(to + at)) = __builtin_bit_cast(u32x2, r[0]);
                *reinterpret_cast<global_u32x2_w *>((uintptr_t)(to + other)) = __builtin_bit_cast(u32x2, r[1]);
            }
        }
    }
}

}  // namespace

hipError_t tetri_launch_rope(int head_dim, const RopeParams &p, hipStream_t stream)
{
    const int64_t units = (int64_t)p.rows * p.splits;
    auto kernel = head_dim == 128 ? (p.past_caches ? qk_norm_rope_kernel<128, true> : qk_norm_rope_kernel<128, false>)
                                  : (p.past_caches ? qk_norm_rope_kernel<64, true> : qk_norm_rope_kernel<64, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)((units + kRowWaves - 1) / kRowWaves)), dim3(kRowWaves * 64), 0, stream, p);
    return hipGetLastError();
}
