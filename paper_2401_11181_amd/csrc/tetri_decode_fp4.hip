// One decode iteration over a paged cache of 4-bit codes (cache_fp4.h) for gfx950: tetri_decode.hip's counterpart.  The batch is cut the same
// ways (a workgroup per (request, kv head), equal parts of each, or equal ranges of the whole batch's steps), partial results meet the
// same way; what a wavefront does with its steps is another thing, because codes are a quarter of the bytes: reading them is
// 4.25 * D / 8 bytes per cached token and kv head, and at that rate the work per byte counts.
//
// A step is 32 keys (fp4_steps.h).  A wavefront has a ring of steps of its own in LDS; no barrier stands between steps.
//
//   * Slots past the end of a request's cache may hold anything: their scores are masked, their exponents replaced (a code is
//     finite, an exponent may stand for NaN).  Pages past the end are not looked up.
//   * The new token is not quantised: its score is summed in 32 bits by the wavefront that has the request's last step.
#include "fp4_steps.h"

namespace {

using namespace tetri_dev;

constexpr int kMergeCols = 4;     // query heads whose partial O the merge area in LDS holds at a time
constexpr int kWaves = 4;         // wavefronts of a workgroup
constexpr int kDepth = 2;         // steps a wavefront's ring holds: three workgroups fit a compute unit (with four steps, two: 64 requests of 2048 tokens 124.6 us, 119.6)
// What a request costs a range of steps beside its steps, in steps: another page table, another Q, a merge.  A division that did not count it gave some ranges
// five short requests and let all others wait for them (48 requests of 16 to 8192 tokens, 32 heads over 8: 33.0 us, with it 20.3).
constexpr int kRequestSteps = kFp4RequestSteps;

// A workgroup's partial result: g rows of D floats (unnormalised O), then g of m and g of the row sum.
template <int D> __device__ __forceinline__ int part_floats(int g) { return g * D + ((2 * g + 3) & ~3); }

// A stretch of steps of one request; wave-uniform.  A request without a cached token has one step, without keys.
struct Job {
    int b;                      // request
    int begin, end;             // steps [begin, end)
    int L;                      // cached tokens of the request
    __device__ __forceinline__ int steps() const { return max((L + 31) >> 5, 1); }
};

constexpr int kDecodeLead = 56;   // bytes of the kernel's arguments in front of its structure (see tetri_decode.hip)

// NB: blocks of 16 query heads.  RANGES and the grid as decode_attn_kernel.
template <int D, int NB, bool RANGES>
__global__ __launch_bounds__(kWaves * 64, NB == 1 ? 3 : 2) void decode_fp4_kernel(const int32_t *ctx_lens, const int32_t *bt, const uint16_t *pages, int max_blocks, int Hkv,
                                                                    uint32_t hkv_magic, int parts, const uint16_t *q, int B, DecodeArgs)
{
    typedef __attribute__((address_space(4))) const DecodeArgs const_decode_args;
    typedef Step<D> T;
    constexpr int NW = kWaves, NT = NW * 64, KS = D / 32, DJ = D / 16, DEPTH = kDepth;
    __shared__ __attribute__((aligned(1024))) char smem[NW * DEPTH * T::BYTES];
    __shared__ __attribute__((aligned(16))) float area[NW][kMergeCols][D];
    __shared__ float stat[NW][2][32];
    __shared__ int arrived[2];
    const const_decode_args *p = (const const_decode_args *)((__attribute__((address_space(4))) const char *)__builtin_amdgcn_kernarg_segment_ptr() + kDecodeLead);

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = lane >> 4, l16 = lane & 15;
    // a context length outside what the block table can describe is clamped: whatever the device arrays hold, no address is formed
    // from a block-table index out of range
    auto ctx_of = [&](int b) -> int { return min(max(((const const_i32 *)(uintptr_t)ctx_lens)[b], 0), max_blocks * kPage); };

    // Two slabs are 17 cache lines, the one in the middle is both's: workgroups of neighbouring kv heads go to the same XCD (every 8th one),
    // whose L2 then reads it once.
    int item = blockIdx.x;
    if ((item | 15) < (int)gridDim.x) item = (item & ~15) + 2 * (item & 7) + ((item >> 3) & 1);
    const int wg = magic_div(item, hkv_magic), kh = item - wg * Hkv;
    auto clear_next = [&]() {
        const int n = p->n_counters;
        for (int i = blockIdx.x * NT + tid; i < n; i += gridDim.x * NT) store_global(p->counters_next + i, 0);
    };
    // ---- the workgroup's first job; `left` steps of its range behind it
    Job job;
    int left = 0, div_q, div_r = 0, pos;
    if constexpr (!RANGES) {
        job.b = parts == 1 ? wg : wg / parts;
        pos = wg - job.b * parts;
        job.L = ctx_of(job.b);
        div_q = parts == 1 ? job.steps() : (job.steps() + parts - 1) / parts;
        job.begin = pos * div_q;
        job.end = min(job.steps(), job.begin + div_q);
        if (job.begin >= job.end) {                      // fewer steps than parts: nobody waits for this one
            clear_next();
            return;
        }
    } else {
        // lane l looks at requests l * R .. l * R + R - 1
        const int R = (B + 63) >> 6;
        const int32_t *ctx = ctx_lens;
        auto length_of = [&](int b) -> int { return min(max(ctx[min(b, B - 1)], 0), max_blocks * kPage); };
        auto steps_of = [&](int L) -> int { return max((L + 31) >> 5, 1) + kRequestSteps; };
        const int own = length_of(lane * R);             // (all there is to look at while there are no more than 64 requests)
        int mine = lane * R < B ? steps_of(own) : 0;
        for (int i = 1; i < R; ++i)
            if (lane * R + i < B) mine += steps_of(length_of(lane * R + i));
        const int incl = prefix_sum(mine);
        const int total = __builtin_amdgcn_readlane(incl, 63);
        const int ranges = min(p->ranges, (int)((uint32_t)(total + p->min_steps - 1) / (uint32_t)p->min_steps));
        if (wg >= ranges) {
            clear_next();
            return;
        }
        div_q = __builtin_amdgcn_readfirstlane((int)((uint32_t)total / (uint32_t)ranges));
        div_r = total - div_q * ranges;
        pos = wg * div_q + min(wg, div_r);
        left = div_q + (int)(wg < div_r);
        // the request of step `pos`: its lane, then inside the lane's block
        int base = incl - mine, found = -1, fl = 0, fbase = 0;
        if (pos >= base && pos < incl) {
            if (R == 1) {
                found = lane; fl = own; fbase = base;
            } else {
                for (int i = 0; i < R; ++i) {
                    const int L = length_of(lane * R + i), n = steps_of(L);
                    if (found < 0 && pos < base + n) { found = min(lane * R + i, B - 1); fl = L; fbase = base; }
                    base += n;
                }
            }
        }
        const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(found >= 0) | (1ull << 63));
        job.b = __builtin_amdgcn_readlane(found, src);
        if (job.b < 0) return;                           // (ctx_lens written to while the launch runs: no address is formed from it)
        job.L = __builtin_amdgcn_readlane(fl, src);
        job.begin = pos - __builtin_amdgcn_readlane(fbase, src);
        job.end = min(job.steps(), job.begin + left);
        left -= min(job.steps() + kRequestSteps - job.begin, left);
    }
    // the job after `j`, with `rest` steps of the range behind j: rest goes down by the new job's steps
    auto next_job = [&](Job &j, int &rest) {
        j.b = min(j.b + 1, B - 1);                       // (there is one, unless ctx_lens is written to while the launch runs)
        j.L = ctx_of(j.b);
        j.begin = 0;
        j.end = min(j.steps(), rest);
        rest -= min(j.steps() + kRequestSteps, rest);
    };
    if constexpr (RANGES) {
        if (job.begin >= job.end) {                      // (the range begins behind a request's steps)
            if (left == 0) {
                clear_next();
                return;
            }
            pos += job.steps() + kRequestSteps - job.begin;
            next_job(job, left);
        }
    }

    const uint32_t page_bytes = 2 * Hkv * kFp4Slab<D>, v_delta = Hkv * kFp4Slab<D>;
    const char *pool = reinterpret_cast<const char *>(pages) + (size_t)kh * kFp4Slab<D>;
    char *my = smem + wave * (DEPTH * T::BYTES);
    const uint32_t my_lds = lds_address(my);

    const StepSource<D> source(lane, v_delta);

    // ---- the wavefront's cursor: the step whose loads are issued next (step fs of job fj, frest steps of the range behind that job; fs < 0: there
    // is none).  The page ids of its next 32 steps are in the lanes of `ids`, the two of step id_first + NW * i in lanes 2i and 2i + 1: read by one
    // vector load.  (Read step by step through the scalar cache they share a counter with LDS, and every wait for codes waited for them too.)
    Job fj = job;
    int fs = job.begin + wave, frest = left, id_at = 64;
    int ids = 0;
    auto settle = [&]() {
        while (fs >= fj.end) {
            if (!RANGES || frest == 0) { fs = -1; return; }
            next_job(fj, frest);
            fs = wave;
            id_at = 64;
        }
        if (id_at == 64) {
            const int n = (fj.L + kPage - 1) / kPage;    // pages of the request; of what is not one, page 0 of the pool is read and does not count
            const int e = 2 * (fs + NW * (lane >> 1)) + (lane & 1);
            ids = 0;
            if (e < n) ids = reinterpret_cast<__attribute__((address_space(1))) const int32_t *>((uintptr_t)(bt + (size_t)fj.b * max_blocks))[e];
            wait_vm<0>();                                // (here, once in 32 steps: the compiler's own wait stands at every step, where it drains the loads in flight)
            id_at = 0;
        }
    };
    auto issue = [&](int place) {
        const int pg0 = __builtin_amdgcn_readlane(ids, id_at), pg1 = __builtin_amdgcn_readlane(ids, id_at + 1);
        id_at += 2;
        issue_step<D, true>(source, pool + (size_t)pg0 * page_bytes, pool + (size_t)pg1 * page_bytes, v_delta, lane, my_lds + place * T::BYTES);
    };
    // Q fragments (B operand of S^T): column l16 is query head kh * g + l16 of the block, zero past g; element 8 s .. of a lane's D / 4 ones
    bf16x8 qf[NB][KS];
    Columns<D, NB> x;
    auto load_q = [&](int b) {
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const int g = p->g;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int col = 16 * nb + (ln & 15);
            const global_u32x4 *qp = reinterpret_cast<const global_u32x4 *>((uintptr_t)(q + ((size_t)b * p->Hq + (size_t)kh * g + min(col, g - 1)) * D + (ln >> 4) * (D / 4)));
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                u32x4 v = u32x4(qp[s]);
                if (p->neg) v ^= 0x80008000u;            // (a negative scale is Q's sign)
                if (col >= g) v = u32x4{0u, 0u, 0u, 0u};
                qf[nb][s] = __builtin_bit_cast(bf16x8, v);
            }
        }
    };

    // ---- the first loads.  The steps in flight are remembered in order: c* the current one, then what follows it
    int ahead = 0;                                       // steps in flight, the current one included
    int rb[DEPTH], rs[DEPTH], rL[DEPTH];                 // (a shift register: request, step and length of each)
    int place_in = 0, place_out = 0;
    settle();
#pragma unroll
    for (int i = 0; i < DEPTH; ++i) {
        rb[i] = 0; rs[i] = -1; rL[i] = 0;
        if (fs >= 0) {
            issue(place_in);
            if (++place_in == DEPTH) place_in = 0;
            rb[i] = fj.b; rs[i] = fs; rL[i] = fj.L;
            ++ahead;
            if (i == 0) load_q(fj.b);
            fs += NW;
            settle();
        }
    }

    const float c = p->c;
    auto write_pair = [&](uint16_t *to, float x, float y, float l) {
        const float inv = 1.0f / l;
        bf16x2 r;
        r[0] = (__bf16)(x * inv);
        r[1] = (__bf16)(y * inv);
        *reinterpret_cast<__attribute__((address_space(1))) uint32_t *>((uintptr_t)to) = __builtin_bit_cast(uint32_t, r);
    };
    // What this workgroup has left of requests cut between workgroups, two at most (of its first job and of its last one): the request, its arrival
    // counter, how many parts it has and where they are.  Settled when all jobs are done: a wait for the partial results' stores and the
    // counter's answer are two trips to memory, and the loads of the jobs behind are in flight.
    int cut_b[2], cut_counter[2], cut_pieces[2], cut_w0[2], cuts = 0;
    auto place_of = [&](float *partial, int pfl, int w0, int i) -> float * {
        return partial + ((size_t)(RANGES ? 2 * (w0 + i) + (int)(i == 0) : w0 + i) * Hkv + kh) * pfl;
    };
    for (;;) {                                           // the jobs of the range
    x.clear();
    while (rs[0] >= 0 && (!RANGES || rb[0] == job.b)) {
        const int cb = rb[0], cs = rs[0], cL = rL[0];
        const bool last = cs + 1 == max((cL + 31) >> 5, 1);          // the request's last step
        // the step has landed when only what was issued after it is outstanding
        switch (ahead) {
        case 1: wait_vm<0>(); break;
        case 2: wait_vm<T::LOADS>(); break;
        case 3: wait_vm<2 * T::LOADS>(); break;
        default: wait_vm<3 * T::LOADS>(); break;
        }
        static_assert(DEPTH <= 4, "waits for up to three steps behind the current one");
        const char *tile = my + place_out * T::BYTES;
        StepCodes<D> codes;
        codes.read_k(tile, grp, l16);
        codes.read_v(tile, grp, l16);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // everything is in registers: the place may be overwritten
        const bool far = fs >= 0;
        if (far) issue(place_in);
        if (++place_out == DEPTH) place_out = 0;
        codes.powers(l16);
        f32x4 sc[NB][2];
        x.scores(codes, [&](int nb, int s) { return qf[nb][s]; }, sc);
        // ---- slots past the end are masked
        if (last) {
            const int n = cL - 32 * cs;                              // keys of the step
#pragma unroll
            for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (16 * pg + 4 * i + grp >= n) {
                        codes.vs[4 * pg + i] = 0.f;
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb) sc[nb][pg][i] = -INFINITY;
                    }
        }
        bf16x8 pf[NB];
        x.weigh(sc, c, pf);
        x.add(codes, pf);
        if (last) {
            // the new token: a lane has D / 4 products of its score, and the rows of O that it holds
            const size_t at = ((size_t)cb * Hkv + kh) * D;
            const global_u32x4 *kp = reinterpret_cast<const global_u32x4 *>((uintptr_t)(p->k_new + at + grp * (D / 4)));
            u32x4 kn[KS], vn[4];
#pragma unroll
            for (int s = 0; s < KS; ++s) kn[s] = u32x4(kp[s]);
            // row 4 * grp + i of the products is d = DJ * (4 * grp + i) ..: DJ bf16 of v_new
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint16_t *src = p->v_new + at + DJ * (4 * grp + i);
                if constexpr (DJ == 8) {
                    vn[i] = *reinterpret_cast<global_u32x4 *>((uintptr_t)src);
                } else {
                    const u32x2 y = *reinterpret_cast<__attribute__((address_space(1))) const u32x2 *>((uintptr_t)src);
                    vn[i] = u32x4{y[0], y[1], 0u, 0u};
                }
            }
            auto value = [](const u32x4 &w, int j) -> float { return __builtin_bit_cast(float, (j & 1) ? w[j / 2] & 0xffff0000u : w[j / 2] << 16); };
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) s = __builtin_fmaf(value(kn[k], j), value(__builtin_bit_cast(u32x4, qf[nb][k]), j), s);
                s += __shfl_xor(s, 16, 64);
                s += __shfl_xor(s, 32, 64);
                s *= c;
                const float m_new = fmaxf(x.m[nb], s), alpha = __builtin_amdgcn_exp2f(x.m[nb] - m_new), w = __builtin_amdgcn_exp2f(s - m_new);
                x.m[nb] = m_new;
                x.lsum[nb] = x.lsum[nb] * alpha + w;
#pragma unroll
                for (int j = 0; j < DJ; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x.o[nb][j][i] = __builtin_fmaf(w, value(vn[i], j), x.o[nb][j][i] * alpha);
            }
        }
        // on to the next step (its Q rows, if it is another request's, are requested here)
#pragma unroll
        for (int i = 0; i + 1 < DEPTH; ++i) { rb[i] = rb[i + 1]; rs[i] = rs[i + 1]; rL[i] = rL[i + 1]; }
        rs[DEPTH - 1] = -1;
        --ahead;
        if (far) {
            rb[DEPTH - 1] = fj.b; rs[DEPTH - 1] = fs; rL[DEPTH - 1] = fj.L;
            ++ahead;
            if (++place_in == DEPTH) place_in = 0;
            fs += NW;
            settle();
        }
        if (RANGES && rs[0] >= 0 && rb[0] != cb) load_q(rb[0]);
    }

    // ---- the job is done: the wavefronts merge.  (The tiles may be receiving the next job's first steps: the merge has an area of its own in
    // LDS, for kMergeCols query heads at a time.)
    const const_decode_args *e = p;
    int te = tid;
    asm volatile("" : "+v"(te), "+s"(e));                // (values worked out and read here, not kept across the loop)
    const int grp_e = (te >> 4) & 3, l16_e = te & 15, g = e->g;
    const bool ends = job.end == job.steps(), whole = ends && job.begin == 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        if (grp_e == 0) { stat[wave][0][16 * nb + l16_e] = x.m[nb]; stat[wave][1][16 * nb + l16_e] = x.lsum[nb][0]; }
    }
    if (ends && e->pages_w != nullptr && job.L < max_blocks * kPage && wave == NW - 1 && (te & 63) < D / 4) {
        // fused append: the codes of the new token's K and V row of this kv head go to slot L % 16 of page block_table[b][L / 16], 8
        // values a lane (nothing that counts in this launch reads that slot: key L comes from k_new / v_new everywhere)
        constexpr int LR = D / 8;                            // lanes of a row
        const int which = (te & 63) / LR, chunk = te % LR;
        const int page = ((const const_i32 *)(uintptr_t)(bt + (size_t)job.b * max_blocks))[job.L / kPage];
        const uint16_t *src = (which ? e->v_new : e->k_new) + ((size_t)job.b * Hkv + kh) * D + chunk * 8;
        uint32_t exponent;
        const uint32_t codes = bf16_to_fp4(u32x4(*reinterpret_cast<global_u32x4 *>((uintptr_t)src)), exponent);
        char *slab = reinterpret_cast<char *>(e->pages_w) + (size_t)page * page_bytes + (which ? v_delta : 0) + (size_t)kh * kFp4Slab<D>;
        store_fp4<D>(slab, job.L % kPage, chunk, codes, exponent);
    }
    // a request cut between workgroups: which part of how many this is, and where the parts are (a workgroup keeps the first part of a
    // request in its second place, any other part in its first one: it has at most one of each)
    int piece = 0, pieces = 1, w0 = 0, counter = 0;
    if (!whole) {
        if constexpr (!RANGES) {
            piece = pos;
            pieces = (job.steps() + div_q - 1) / div_q;
            w0 = wg - piece;
            counter = job.b;
        } else {
            auto owner = [&](int x) -> int {             // the range that has step x of the sequence
                const int cut = div_r * (div_q + 1);
                return __builtin_amdgcn_readfirstlane(x < cut ? (int)((uint32_t)x / (uint32_t)(div_q + 1)) : div_r + (int)((uint32_t)(x - cut) / (uint32_t)div_q));
            };
            w0 = owner(pos - job.begin);                 // pos: the sequence position of the job's first step
            pieces = owner(pos - job.begin + job.steps() - 1) - w0 + 1;
            piece = wg - w0;
            counter = w0;
        }
        counter = counter * Hkv + kh;
    }
    const int pfl = part_floats<D>(g);
    float *left_part = place_of(e->partial, pfl, w0, piece);
    if (!whole) {
        const bool second = cuts != 0;
        if (!second) { cut_b[0] = job.b; cut_counter[0] = counter; cut_pieces[0] = pieces; cut_w0[0] = w0; }
        else { cut_b[1] = job.b; cut_counter[1] = counter; cut_pieces[1] = pieces; cut_w0[1] = w0; }
        ++cuts;
    }
    const size_t head = (size_t)job.b * e->Hq + (size_t)kh * g;
    uint16_t *out = e->out + head * D;
    for (int c0 = 0; c0 < g; c0 += kMergeCols) {
        if (c0 != 0) lds_barrier();                      // everybody is done with the columns before
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int col = 16 * nb + l16_e;
            if (col >= c0 && col < min(g, c0 + kMergeCols)) x.put(nb, area[wave][col - c0], grp_e);
        }
        lds_barrier();
        // two neighbouring values of one head per thread
        for (int v = te; v < min(g - c0, kMergeCols) * (D / 2); v += NT) {
            const int cc = v / (D / 2), col = c0 + cc, d = 2 * (v - cc * (D / 2));
            float ms = stat[0][0][col];
#pragma unroll
            for (int i = 1; i < NW; ++i) ms = fmaxf(ms, stat[i][0][col]);
            float v0 = 0.f, v1 = 0.f, l = 0.f;
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const float wgt = __builtin_amdgcn_exp2f(stat[i][0][col] - ms);
                const float2 z = *reinterpret_cast<const float2 *>(&area[i][cc][d]);
                v0 = __builtin_fmaf(z.x, wgt, v0);
                v1 = __builtin_fmaf(z.y, wgt, v1);
                l = __builtin_fmaf(stat[i][1][col], wgt, l);
            }
            if (whole) {
                write_pair(out + col * D + d, v0, v1, l);
            } else {
                float *mine = left_part;
                store_coherent2(mine + col * D + d, v0, v1);
                if (d == 0) {
                    store_coherent(mine + g * D + col, ms);
                    store_coherent(mine + g * D + g + col, l);
                }
            }
        }
    }
    if (!RANGES || left == 0) break;
    pos += job.steps() + kRequestSteps - job.begin;
    next_job(job, left);
    lds_barrier();                                       // everybody is done with stat and area
    }

    if (cuts != 0) {
        const const_decode_args *e = p;
        int te = tid;
        asm volatile("" : "+v"(te), "+s"(e));
        const int g = e->g, pfl = part_floats<D>(g);
        float *partial = e->partial;
        coherent_stores_done();
        lds_barrier();
        if (te < cuts) arrived[te] = atomic_add_global(e->counters + (te == 0 ? cut_counter[0] : cut_counter[1]), 1);
        lds_barrier();
        for (int k = 0; k < cuts; ++k) {
            const int pieces = k == 0 ? cut_pieces[0] : cut_pieces[1], w0 = k == 0 ? cut_w0[0] : cut_w0[1];
            if (__builtin_amdgcn_readfirstlane(arrived[k]) != pieces - 1) continue;
            // all the others have been here: the counter goes back to zero, the parts are merged in their order.  With few columns the
            // threads form groups that take every groups-th part, and the groups meet in LDS.
            if (te == 0) store_global(e->counters + (k == 0 ? cut_counter[0] : cut_counter[1]), 0);
            uint16_t *rows = e->out + ((size_t)(k == 0 ? cut_b[0] : cut_b[1]) * e->Hq + (size_t)kh * g) * D;
            const int pairs = g * (D / 2), groups = max(1, NT / pairs);
            for (int v0 = 0; v0 < pairs; v0 += NT) {
                const int grp_m = groups > 1 ? te / pairs : 0, v = groups > 1 ? te - grp_m * pairs : v0 + te;
                const bool on = grp_m < groups && v < pairs;
                const int col = v / (D / 2);
                float mm = -INFINITY, l = 0.f, x = 0.f, y = 0.f;
                if (on)
                    for (int i0 = grp_m; i0 < pieces; i0 += 8 * groups) {
                        float mi[8], li[8];
                        float2 xi[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float *src = place_of(partial, pfl, w0, min(i0 + i * groups, pieces - 1));
                            mi[i] = load_coherent(src + g * D + col);
                            li[i] = load_coherent(src + g * D + g + col);
                            xi[i] = load_coherent2(src + 2 * v);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (i0 + i * groups < pieces) {
                                const float m_new = fmaxf(mm, mi[i]);
                                const float w_old = __builtin_amdgcn_exp2f(mm - m_new), w_new = __builtin_amdgcn_exp2f(mi[i] - m_new);
                                mm = m_new;
                                l = __builtin_fmaf(li[i], w_new, l * w_old);
                                x = __builtin_fmaf(xi[i].x, w_new, x * w_old);
                                y = __builtin_fmaf(xi[i].y, w_new, y * w_old);
                            }
                    }
                if (groups > 1) {
                    // (a group without a part has m = -inf and weighs nothing; group 0 always has one)
                    float *meet = &area[0][0][0];
                    static_assert(NW * kMergeCols * D >= 4 * NT, "four floats per thread");
                    lds_barrier();                       // everybody is done with what was merged before
                    if (on) *reinterpret_cast<f32x4 *>(meet + 4 * te) = f32x4{mm, l, x, y};
                    lds_barrier();
                    if (on && grp_m == 0)
                        for (int i = 1; i < groups; ++i) {
                            const f32x4 z = *reinterpret_cast<const f32x4 *>(meet + 4 * (i * pairs + v));
                            const float m_new = fmaxf(mm, z[0]);
                            const float w_old = __builtin_amdgcn_exp2f(mm - m_new), w_new = __builtin_amdgcn_exp2f(z[0] - m_new);
                            mm = m_new;
                            l = __builtin_fmaf(z[1], w_new, l * w_old);
                            x = __builtin_fmaf(z[2], w_new, x * w_old);
                            y = __builtin_fmaf(z[3], w_new, y * w_old);
                        }
                }
                if (on && grp_m == 0) write_pair(rows + 2 * v, x, y, l);
            }
        }
    }
    clear_next();
}

template <int D, int NB> hipError_t launch(const DecodeParams &p, hipStream_t stream)
{
    const dim3 grid((p.parts > 0 ? p.B * p.parts : p.ranges) * p.Hkv);
    auto kernel = p.parts > 0 ? decode_fp4_kernel<D, NB, false> : decode_fp4_kernel<D, NB, true>;
    static_assert(KernelArgs<decltype(kernel)>::last_offset() == kDecodeLead, "where the kernel reads its structure");
    hipLaunchKernelGGL(kernel, grid, dim3(kWaves * 64), 0, stream, p.ctx, p.bt, p.pages, p.max_blocks, p.Hkv, p.hkv_magic, p.parts, p.q, p.B,
                       static_cast<const DecodeArgs &>(p));
    return hipGetLastError();
}

}  // namespace

hipError_t tetri_launch_decode_fp4(const tetri_ctx *h, const DecodeParams &p, hipStream_t stream)
{
    if (p.g > 32) return hipErrorInvalidValue;
    if (h->cfg.head_dim == 128) return p.g > 16 ? launch<128, 2>(p, stream) : launch<128, 1>(p, stream);
    return p.g > 16 ? launch<64, 2>(p, stream) : launch<64, 1>(p, stream);
}
