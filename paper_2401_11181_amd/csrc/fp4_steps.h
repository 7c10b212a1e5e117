// Steps of 32 cached keys over 4-bit codes: how they come into LDS and what the matrix cores make of them, for the kernels in which a wavefront
// takes whole steps by itself (tetri_decode_fp4.hip, tetri_prefill_fp4.hip).
//
//   * A step is two pages of one (request, kv head).  A slab comes straight into LDS: a page's codes by one instruction (D = 128), the exponents of
//     all four slabs of the step by one more.
//   * Codes become bf16 in registers, with their power of two (v_cvt_scalef32_pk_bf16_fp4, exact), and the products are 16x16x32 bf16 ones: sums are
//     32-bit numbers.  (The products that take such codes and their exponents as they are, v_mfma_scale_f32_16x16x128_f8f6f4, need Q in 8-bit
//     pieces, and they sum with fewer bits: of N(0, 1) scores of 128 products they lost 4e-6 of the root mean square, with one channel 50 times as large 3e-5 and
//     up to 0.03 of a single score; this way 1e-8.)
//   * S^T = K Q^T: the fragment of a lane is 8 neighbouring elements of a row, in any order over the lanes as long as Q's is the same: a lane takes
//     D / 4 neighbouring codes of one key, which share an exponent.
//   * O^T += V^T P^T needs several keys of one d in a lane, and codes of neighbouring d share a byte.  A lane reads D / 16 neighbouring codes of each of 8
//     keys, converts pairs of them and puts the halves of two keys together (v_perm_b32): no transposition through LDS.  Row m of the
//     product is then d = D / 16 * m + j, j its number.
//   * Which key is which row of a page's product is free too: row 4a + b is key 4b + a, so that the rows which a V instruction reads are neighbours.
//     Lane (grp, l16) then holds, of column l16, the scores of keys 16 * page + 4i + grp in element i.
#pragma once
#include "cache_fp4.h"

namespace tetri_dev {

__device__ __forceinline__ float load_coherent(const float *p)
{
    return __hip_atomic_load(reinterpret_cast<const __attribute__((address_space(1))) float *>((uintptr_t)p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 load_coherent2(const float *p)
{
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const __attribute__((address_space(1))) uint64_t *>((uintptr_t)p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__builtin_bit_cast(float, (uint32_t)v), __builtin_bit_cast(float, (uint32_t)(v >> 32)));
}
__device__ __forceinline__ void store_coherent2(float *p, float x, float y)
{
    const uint64_t v = (uint64_t)__builtin_bit_cast(uint32_t, x) | (uint64_t)__builtin_bit_cast(uint32_t, y) << 32;
    __hip_atomic_store(reinterpret_cast<__attribute__((address_space(1))) uint64_t *>((uintptr_t)p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A step in LDS: codes of K of both pages, of V of both, then the exponents of K and V of page 0 and K and V of page 1 (behind each other,
// kScaleBytes of each; D = 128: row 4a + b of a slab's at place 4b + a).
template <int D> struct Step {
    static constexpr int ROW = D / 2, PAGE_BYTES = kPage * ROW, SCALE_BYTES = kPage * D / 32;
    static constexpr int V = 2 * PAGE_BYTES, SCALES = 4 * PAGE_BYTES;
    static constexpr int BYTES = SCALES + 256;                           // (an instruction of 64 lanes of 4 bytes)
    static constexpr int LOADS = D == 128 ? 5 : 3;                       // instructions
};

// The sum of x over the lanes up to this one.
__device__ __forceinline__ int prefix_sum(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);       // (from 1, 2, 4 and 8 lanes to the left in a row of 16)
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);      // (a row's last lane to the next row, for rows 1 and 3)
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);      // (lane 31 to rows 2 and 3)
    return x;
}

// 64 lanes of 4 bytes, lane l's from p to LDS byte lds + 4 * l, and of 16 bytes; ONCE: read once, past the caches as dma16_stream's.
template <bool ONCE> __device__ __forceinline__ void dma4_lanes(const void *p, uint32_t lds)
{
    lds = __builtin_amdgcn_readfirstlane(lds);
    if constexpr (ONCE) asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dword %0, off nt" ::"v"(p), "s"(lds) : "memory", "m0");
    else asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dword %0, off" ::"v"(p), "s"(lds) : "memory", "m0");
}
template <bool ONCE> __device__ __forceinline__ void dma16_lanes(const void *p, uint32_t lds)
{
    lds = __builtin_amdgcn_readfirstlane(lds);
    if constexpr (ONCE) asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, off nt" ::"v"(p), "s"(lds) : "memory", "m0");
    else asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(lds) : "memory", "m0");
}
// 64 lanes of 16 bytes from base + off.
template <bool ONCE> __device__ __forceinline__ void dma16_base(const void *base, uint32_t off, uint32_t lds)
{
    if constexpr (ONCE) {
        const uint32_t v[1] = {off};
        dma16_stream<1>(base, v, lds);
    } else {
        base = uniform_ptr(base);
        lds = __builtin_amdgcn_readfirstlane(lds);
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
    }
}

// Where a lane's part of a step comes from.
template <int D> struct StepSource {
    uint32_t k_off, v_off, s_off;        // bytes from the slab of K (V: of V; s_off: of K, the exponents of K or V)
    bool s_second;                       // the exponents are those of the second page
    __device__ __forceinline__ StepSource(int lane, uint32_t v_delta)
    {
        const int grp = lane >> 4, l16 = lane & 15;
        if constexpr (D == 128) {
            // K: place (row, c) of LDS has chunk c ^ row / 4 of the row (16 bytes), so that the 16 lanes that read the same chunk of all rows meet no
            // bank twice
            k_off = (lane >> 2) * 64 + (((lane & 3) ^ (lane >> 4)) << 4);
            v_off = lane * 16;
            s_off = kFp4Codes<D> + (4 * (l16 & 3) + (l16 >> 2)) * 4 + ((grp & 1) ? v_delta : 0);
            s_second = grp >= 2;
        } else {                         // (lanes past 32 read exponents once more)
            k_off = v_off = (lane & 31) * 16;
            s_off = kFp4Codes<D> + (lane & 7) * 4 + ((lane & 8) ? v_delta : 0);
            s_second = (lane & 16) != 0;
        }
    }
};
// The loads of a step; a, b: the slabs of K of its pages (the same kv head), lds: its place.  ONCE: nobody else reads them.
template <int D, bool ONCE>
__device__ __forceinline__ void issue_step(const StepSource<D> &x, const char *a, const char *b, uint32_t v_delta, int lane, uint32_t lds)
{
    typedef Step<D> T;
    if constexpr (D == 128) {
        dma16_base<ONCE>(a, x.k_off, lds);
        dma16_base<ONCE>(b, x.k_off, lds + T::PAGE_BYTES);
        dma4_lanes<ONCE>((x.s_second ? b : a) + x.s_off, lds + T::SCALES);
        dma16_base<ONCE>(a + v_delta, x.v_off, lds + T::V);
        dma16_base<ONCE>(b + v_delta, x.v_off, lds + T::V + T::PAGE_BYTES);
    } else {
        const char *mine = lane < 32 ? a : b;
        dma16_lanes<ONCE>(mine + x.k_off, lds);
        dma4_lanes<ONCE>((x.s_second ? b : a) + x.s_off, lds + T::SCALES);
        dma16_lanes<ONCE>(mine + v_delta + x.v_off, lds + T::V);
    }
}

// A step's codes and exponents of a lane: K's rows, of V key 4i + grp of both pages.
template <int D> struct StepCodes {
    uint32_t kw[2][D / 32], ke[2], vw[8];
    u32x4 ve[2];                         // D = 128: exponents of all groups, a word for each key
    float vs[8];
    // reads them; they have arrived when LDS reads have been waited for
    __device__ __forceinline__ void read_k(const char *tile, int grp, int l16)
    {
        typedef Step<D> T;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
            const int row = 4 * (l16 & 3) + (l16 >> 2);
            const char *k = tile + pg * T::PAGE_BYTES, *es = tile + T::SCALES + pg * (2 * T::SCALE_BYTES);
            if constexpr (D == 128) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(k + row * 64 + ((grp ^ (row >> 2)) << 4));
#pragma unroll
                for (int s = 0; s < D / 32; ++s) kw[pg][s] = x[s];
                ke[pg] = *reinterpret_cast<const uint8_t *>(es + 4 * l16 + grp);
            } else {
                const u32x2 x = *reinterpret_cast<const u32x2 *>(k + row * 32 + grp * 8);
#pragma unroll
                for (int s = 0; s < D / 32; ++s) kw[pg][s] = x[s];
                ke[pg] = *reinterpret_cast<const uint8_t *>(es + 2 * row + (grp >> 1));
            }
        }
    }
    __device__ __forceinline__ void read_v(const char *tile, int grp, int l16)
    {
        typedef Step<D> T;
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
            const char *v = tile + T::V + pg * T::PAGE_BYTES, *es = tile + T::SCALES + (2 * pg + 1) * T::SCALE_BYTES;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (D == 128) vw[4 * pg + i] = *reinterpret_cast<const uint32_t *>(v + (4 * i + grp) * 64 + l16 * 4);
                else vw[4 * pg + i] = *reinterpret_cast<const uint16_t *>(v + (4 * i + grp) * 32 + l16 * 2);
            }
            if constexpr (D == 128) {
                ve[pg] = *reinterpret_cast<const u32x4 *>(es + 16 * grp);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) vs[4 * pg + i] = fp4_scale(*reinterpret_cast<const uint8_t *>(es + 2 * (4 * i + grp) + (l16 >> 3)));
            }
        }
    }
    // V's powers.  (The byte of the lane's group turned to where a float has its exponent; what else is in the word the conversions do not look at.)
    __device__ __forceinline__ void powers(int l16)
    {
        if constexpr (D == 128) {
#pragma unroll
            for (int x = 0; x < 8; ++x) vs[x] = __builtin_bit_cast(float, __builtin_amdgcn_alignbit(ve[x / 4][x % 4], ve[x / 4][x % 4], 9 + 8 * (l16 >> 2)));
        }
    }
    __device__ __forceinline__ void negate_k()
    {
#pragma unroll
        for (int pg = 0; pg < 2; ++pg)
#pragma unroll
            for (int s = 0; s < D / 32; ++s) kw[pg][s] ^= 0x88888888u;
    }
    __device__ __forceinline__ bf16x8 k(int pg, int s) const { return __builtin_bit_cast(bf16x8, fp4_to_bf16(kw[pg][s], fp4_scale(ke[pg]))); }
    // elements 2t and 2t + 1 of V of key x
    template <int TT> __device__ __forceinline__ uint32_t v(int x) const
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vw[x], vs[x], TT));
    }
};

// NB blocks of 16 columns (queries) and what attention over some keys has made of them.
template <int D, int NB> struct Columns {
    static constexpr int KS = D / 32, DJ = D / 16;
    f32x4 o[NB][DJ];                     // element i: row 4 * grp + i of product j
    f32x4 lsum[NB];                      // the row sum, in every element: a product of ones and the weights as rounded
    float m[NB];                         // a reference exponent, not the exact maximum

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            m[nb] = -1e30f;
            lsum[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < DJ; ++j) o[nb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // scores of a step's keys; K: something with k(page, s); q(nb, s): B operand, elements 8 s .. of a lane's D / 4 of column block nb
    template <class K, class Q> static __device__ __forceinline__ void scores(const K &codes, const Q &q, f32x4 (&sc)[NB][2])
    {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) sc[nb][0] = sc[nb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const bf16x8 k0 = codes.k(0, s), k1 = codes.k(1, s);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const bf16x8 qf = q(nb, s);
                sc[nb][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf, sc[nb][0], 0, 0, 0);
                sc[nb][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf, sc[nb][1], 0, 0, 0);
            }
        }
    }
    // their weights: rounded to bf16 for the PV product, the row sum is of the rounded ones.  c > 0
    __device__ __forceinline__ void weigh(const f32x4 (&sc)[NB][2], float c, bf16x8 (&pf)[NB])
    {
        bf16x8 ones;
#pragma unroll
        for (int i = 0; i < 8; ++i) ones[i] = (__bf16)1.0f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            // m stays as it is unless a score exceeds it by 8 (weights are floating-point numbers: no precision is lost below)
            float top = sc[nb][0][0];
#pragma unroll
            for (int x = 1; x < 8; ++x) top = fmaxf(top, sc[nb][x / 4][x % 4]);
            if (__builtin_amdgcn_ballot_w64(top * c > m[nb] + 8.f) != 0) {
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float m_new = fmaxf(m[nb], top * c), alpha = __builtin_amdgcn_exp2f(m[nb] - m_new);
                m[nb] = m_new;
                lsum[nb] *= alpha;
#pragma unroll
                for (int j = 0; j < DJ; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[nb][j][i] *= alpha;
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) pf[nb][x] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(sc[nb][x / 4][x % 4], c, -m[nb]));
            lsum[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[nb], lsum[nb], 0, 0, 0);
        }
    }
    // O^T += V^T P^T; V: something with v<t>(key)
    template <class V, int T = 0> __device__ __forceinline__ void add(const V &codes, const bf16x8 (&pf)[NB])
    {
        if constexpr (T < DJ / 2) {
            uint32_t x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = codes.template v<T>(k);
            u32x4 even, odd;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                even[k] = __builtin_amdgcn_perm(x[2 * k + 1], x[2 * k], 0x05040100u);
                odd[k] = __builtin_amdgcn_perm(x[2 * k + 1], x[2 * k], 0x07060302u);
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                o[nb][2 * T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, even), pf[nb], o[nb][2 * T], 0, 0, 0);
                o[nb][2 * T + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, odd), pf[nb], o[nb][2 * T + 1], 0, 0, 0);
            }
            add<V, T + 1>(codes, pf);
        }
    }
    // O of the lane's column of block nb to D floats
    __device__ __forceinline__ void put(int nb, float *to, int grp) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < DJ; j += 4)
                *reinterpret_cast<f32x4 *>(to + DJ * (4 * grp + i) + j) = f32x4{o[nb][j][i], o[nb][j + 1][i], o[nb][j + 2][i], o[nb][j + 3][i]};
    }
};

}  // namespace tetri_dev
