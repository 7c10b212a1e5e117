// What tetri_rope.hip takes from the device's headers, for a build of it on the CPU (see rope_on_cpu.cpp): 64 lanes run in lockstep, each on a
// stack of its own, and meet in the operations between lanes.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "tetri_internal.h"

using std::min;

struct Index3 {
    unsigned x;
};
extern Index3 blockIdx, threadIdx;
extern RopeParams g_params;

// Every lane hands in a value and gets all of them.
struct AllLanes {
    uint64_t of[64];
};
AllLanes meet(uint64_t mine);

#define __launch_bounds__(...)
#define __forceinline__ inline
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, params) launch_on_cpu(kernel, grid, block, params)
void launch_on_cpu(void (*kernel)(RopeParams), dim3 grid, dim3 block, const RopeParams &p);

struct Bf16 {
    uint16_t bits;
    Bf16() = default;
    explicit Bf16(float x)                               // (to the nearest, ties to even)
    {
        const uint32_t w = __builtin_bit_cast(uint32_t, x);
        bits = (uint16_t)(x != x ? w >> 16 | 64 : (w + 0x7fff + (w >> 16 & 1)) >> 16);
    }
};
#define __bf16 Bf16

inline int lane_of_dpp(int lane, int ctrl)
{
    switch (ctrl) {
    case 0xb1: return lane ^ 1;
    case 0x4e: return lane ^ 2;
    case 0x141: return lane ^ 7;                         // (half a row, mirrored)
    case 0x140: return lane ^ 15;
    }
    __builtin_trap();
}
inline int my_lane() { return threadIdx.x & 63; }
inline uint64_t ballot(bool x)
{
    const AllLanes all = meet(x);
    uint64_t r = 0;
    for (int i = 0; i < 64; ++i) r |= all.of[i] << i;
    return r;
}
inline float __shfl(float x, int lane, int) { return __builtin_bit_cast(float, (uint32_t)meet(__builtin_bit_cast(uint32_t, x)).of[lane]); }
inline void sincospif(float x, float *s, float *c)
{
    *s = (float)std::sin(M_PI * x);
    *c = (float)std::cos(M_PI * x);
}
#define __builtin_amdgcn_readfirstlane(x) ((int)(uint32_t)meet((uint32_t)(x)).of[0])
#define __builtin_amdgcn_ballot_w64(x) ballot(x)
#define __builtin_amdgcn_mov_dpp(x, ctrl, rows, banks, zero) ((int)(uint32_t)meet((uint32_t)(x)).of[lane_of_dpp(my_lane(), ctrl)])
#define __builtin_amdgcn_rsqf(x) (1.0f / std::sqrt(x))
#define __builtin_amdgcn_kernarg_segment_ptr() ((uintptr_t)&g_params)

namespace tetri_dev {
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef u32x2 global_u32x2_w;
typedef const int32_t const_i32;
struct bf16x4 {
    Bf16 of[4];
    Bf16 &operator[](int i) { return of[i]; }
};
inline int magic_div(int n, uint32_t magic) { return magic != 0 ? (int)((uint64_t)(uint32_t)n * magic >> 32) : n; }
}  // namespace tetri_dev
