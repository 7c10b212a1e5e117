// Queries and keys made ready for attention (gfx950): RMS norm of every head and rotation by position, out of the rows of a projection into
// the rows that the attention calls take, in one pass.
//
//   y = x * rsqrt(mean(x^2) + eps) * w          (left out where there is no w)
//   a', b' = a cos t - b sin t, b cos t + a sin t      for the pairs (a, b) of y, t = position * frequency of the pair
//
// Bound by memory: 4 bytes per element.  A wavefront takes a row, or some of its heads where rows are few: lane l works out pair l's cosine and sine once,
// lanes of 16 bytes then take whole heads (16 or 8 lanes each), every lane always the same elements of a head, so that its 8 cosines and sines
// and its weights stay in registers.  A pair's other half comes from the lane that has it.
// The angle is taken in 64 bits, in turns, of which whole ones are dropped: with 32 bits of a position of 10^6 times a frequency of 1 an angle
// would be off by 0.06.  Everything behind that is 32-bit, rounded once.
#include "cache_fp4.h"

namespace {

using namespace tetri_dev;

constexpr int kRowWaves = 4;

template <int D>
__global__ __launch_bounds__(kRowWaves * 64) void qk_norm_rope_kernel(RopeParams)
{
    typedef __attribute__((address_space(4))) const RopeParams const_params;
    const const_params *p = (const const_params *)__builtin_amdgcn_kernarg_segment_ptr();
    constexpr int LPH = D / 8, HPI = 64 / LPH, U = 4;    // lanes of a head, heads of an instruction, instructions in flight
    const int lane = threadIdx.x & 63;
    const int unit = blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = magic_div(unit, p->splits_magic), split = unit - row * p->splits;
    if (row >= p->rows) return;
    const int heads = p->Hq + p->Hkv, c = lane % LPH;

    // ---- a lane's part of a head, of q or of k
    auto source = [&](int h) -> const global_u32x4 * {
        const uint16_t *x = h < p->Hq ? p->q + (size_t)row * p->q_stride + (size_t)h * D : p->k + (size_t)row * p->k_stride + (size_t)(h - p->Hq) * D;
        return reinterpret_cast<const global_u32x4 *>((uintptr_t)(x + c * 8));
    };
    const int first = split * p->per_split * HPI, end = min(heads, first + p->per_split * HPI);
    if (first >= end) return;
    u32x4 x[U];
    auto fetch = [&](int h0) {
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = *source(min(h0 + u * HPI + lane / LPH, end - 1));
    };
    fetch(first);

    // ---- the row's position, by its segment or as given (for every axis)
    double position;
    const int pairs = p->pairs, pair = min(lane, pairs - 1);
    if (p->cu != nullptr) {
        int seg = 0;                                     // segments that end in front of the row or at it
        for (int s0 = 0; s0 < p->S; s0 += 64) {
            const bool before = s0 + lane < p->S && p->cu[min(s0 + lane, p->S - 1) + 1] <= row;
            seg += __builtin_popcountll(__builtin_amdgcn_ballot_w64(before));
        }
        if (seg >= p->S) return;                         // a padding row: left as it is
        position = (double)((int64_t)p->ctx[seg] + row - p->cu[seg]);
    } else {
        position = (double)p->pos[(size_t)p->axis[pair] * p->rows + row];
    }
    // ---- pair `lane`'s cosine and sine, then those of this lane's 8 elements.  (Element j of the part that turns belongs to pair j / 2 where
    // pairs are neighbours, otherwise to pair j or j - pairs.)
    constexpr double kTurn = 0.15915494309189533576888;  // 1 / (2 pi)
    const double turns = position * (double)p->freq[pair] * kTurn;
    const float part = (float)(turns - rint(turns));
    float mys, myc;
    sincospif(2.0f * part, &mys, &myc);
    const int adjacent = p->adjacent, e0 = c * 8;
    const bool turning = e0 < 2 * pairs, upper = !adjacent && e0 >= pairs;
    float cs[8], sn[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int from = adjacent ? (e0 + j) / 2 : (upper ? e0 + j - pairs : e0 + j);
        cs[j] = __shfl(myc, from & 63, 64);
        sn[j] = __shfl(mys, from & 63, 64);
        if (!turning) { cs[j] = 1.f; sn[j] = 0.f; }
    }
    // (the lane with the other half of this lane's pairs)
    const int partner = adjacent || !turning ? lane : lane + (upper ? -pairs / 8 : pairs / 8);

    auto value = [](const u32x4 &w, int j) -> float { return __builtin_bit_cast(float, (j & 1) ? w[j / 2] & 0xffff0000u : w[j / 2] << 16); };
    u32x4 wq = {0u, 0u, 0u, 0u}, wk = wq;
    if (p->q_weight) wq = *reinterpret_cast<global_u32x4 *>((uintptr_t)(p->q_weight + c * 8));
    if (p->k_weight) wk = *reinterpret_cast<global_u32x4 *>((uintptr_t)(p->k_weight + c * 8));

    for (int h0 = first; h0 < end; h0 += U * HPI) {
        u32x4 y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) y[u] = x[u];
        if (h0 + U * HPI < end) fetch(h0 + U * HPI);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * HPI + lane / LPH;
            if (h0 + u * HPI >= end) break;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = value(y[u], j);
            const bool is_q = h < p->Hq;
            if (p->q_weight || p->k_weight) {
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(v[j], v[j], sum);
#pragma unroll
                for (int d = 1; d < LPH; d <<= 1) sum += __shfl_xor(sum, d, 64);
                const float r = 1.0f / sqrtf(sum * (1.0f / D) + p->eps);
                if (is_q ? p->q_weight != nullptr : p->k_weight != nullptr) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = v[j] * r * value(is_q ? wq : wk, j);
                }
            }
            float z[8];
            if (adjacent) {
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    z[j] = v[j] * cs[j] - v[j + 1] * sn[j];
                    z[j + 1] = v[j + 1] * cs[j] + v[j] * sn[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float other = __shfl(v[j], partner, 64);
                    z[j] = upper ? v[j] * cs[j] + other * sn[j] : v[j] * cs[j] - other * sn[j];
                }
            }
            if (!turning) {                              // (not by way of a product with 0, which an infinity of the head's would make NaN)
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = v[j];
            }
            bf16x8 r;
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = (__bf16)z[j];
            if (h < end) {
                uint16_t *to = is_q ? p->q_out + ((size_t)row * p->Hq + h) * D : p->k_out + ((size_t)row * p->Hkv + (h - p->Hq)) * D;
                *reinterpret_cast<global_u32x4_w *>((uintptr_t)(to + c * 8)) = __builtin_bit_cast(u32x4, r);
            }
        }
    }
}

}  // namespace

hipError_t tetri_launch_rope(int head_dim, const RopeParams &p, hipStream_t stream)
{
    const int64_t units = (int64_t)p.rows * p.splits;
    auto kernel = head_dim == 128 ? qk_norm_rope_kernel<128> : qk_norm_rope_kernel<64>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((units + kRowWaves - 1) / kRowWaves)), dim3(kRowWaves * 64), 0, stream, p);
    return hipGetLastError();
}
