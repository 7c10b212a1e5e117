// Chunked-prefill attention over a paged cache of 4-bit codes for gfx950 where segments are short, or heads 64 wide: tetri_attn.hip's kernel has tiles of 128
// columns, whose keys a few workgroups walk 64 or 128 at a time, behind barriers; here a tile is a quarter as large and any number of workgroups share its keys.
//
//   * A tile is 32 columns of one kv head: neighbouring (row, query head of the kv head) pairs of a segment, rows first, so that codes become bf16
//     once for all heads that share them.  A wavefront takes whole steps of 32 keys by itself (fp4_steps.h), from a ring in LDS, for all of the
//     tile's columns; no barrier stands between steps, and a step's codes are on their way from LDS while the one before it is made.  The
//     chunk's own rows are steps as well, of bf16 rows that go straight into registers.
//   * The steps of all tiles of a kv head, tile after tile, are cut into equal ranges, a workgroup each, worked out on the device from the
//     segments' lengths, the same for every kv head.  A tile counts with all new rows of its segment, whatever its rows see of them, and with
//     kTileSteps more.  The wavefronts of a workgroup take a tile's steps in turn; when it is done every one of them gets a quarter of the others'
//     accumulators, as they lie in registers, through LDS.
//   * Tiles cut between workgroups meet through arrival counters in the same launch, as in tetri_decode.hip: the workgroup that arrives last merges the
//     parts in their order.  Nobody waits.
//   * Workgroups of a kv head run on one XCD (or two, four, eight where there are few kv heads): tiles of a segment read the same keys through its L2.
//   * The chunk's rows are cached in codes by a few workgroups in front of the others; padding rows of the output are zeroed by all.
#include <type_traits>

#include "fp4_steps.h"

namespace {

using namespace tetri_dev;

constexpr int kWaves = 4;         // wavefronts of a workgroup
constexpr int kDepth = 2;         // steps a wavefront's ring holds
constexpr int kNB = 2, kCols = 16 * kNB;        // columns of a tile
constexpr int kTileSteps = kPrefillFp4TileSteps;      // what a tile costs a range beside its steps, in steps

// A workgroup's partial result: its accumulators as they lie in registers (a vector of 4 per product and lane), then m and the row sum of the columns.
template <int D> constexpr int kPartFloats = kCols * (D + 2);

// A stretch of steps of one tile; wave-uniform.
struct Job {
    int s, t;                     // segment, tile in it
    int row0, n, L;               // the segment's first chunk row, rows, cached tokens
    int cached, steps;            // steps of cached keys, all steps
    int begin, end;               // steps [begin, end)
    int seq;                      // number of the job in its range
};

// K and V of 32 of the chunk's own rows, as a step's operands.
template <int D> struct NewRows {
    static constexpr int KS = D / 32, DJ = D / 16;
    u32x4 kw[2][KS];
    uint32_t vw[8][DJ / 2];
    __device__ __forceinline__ void load(const uint16_t *k_new, const uint16_t *v_new, size_t row_elements, int first, int most, int grp, int l16)
    {
#pragma unroll
        for (int pg = 0; pg < 2; ++pg) {
            const int key = min(first + 16 * pg + 4 * (l16 & 3) + (l16 >> 2), most);
            const global_u32x4 *src = reinterpret_cast<const global_u32x4 *>((uintptr_t)(k_new + (size_t)key * row_elements + grp * (D / 4)));
#pragma unroll
            for (int s = 0; s < KS; ++s) kw[pg][s] = u32x4(src[s]);
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int key = min(first + 16 * (x / 4) + 4 * (x % 4) + grp, most);
            const uint16_t *src = v_new + (size_t)key * row_elements + DJ * l16;
            if constexpr (DJ == 8) {
                const u32x4 y = *reinterpret_cast<global_u32x4 *>((uintptr_t)src);
#pragma unroll
                for (int t = 0; t < 4; ++t) vw[x][t] = y[t];
            } else {
                const u32x2 y = *reinterpret_cast<__attribute__((address_space(1))) const u32x2 *>((uintptr_t)src);
                vw[x][0] = y[0];
                vw[x][1] = y[1];
            }
        }
    }
    __device__ __forceinline__ void negate_k()
    {
#pragma unroll
        for (int pg = 0; pg < 2; ++pg)
#pragma unroll
            for (int s = 0; s < KS; ++s) kw[pg][s] ^= 0x80008000u;
    }
    __device__ __forceinline__ bf16x8 k(int pg, int s) const { return __builtin_bit_cast(bf16x8, kw[pg][s]); }
    template <int T> __device__ __forceinline__ uint32_t v(int x) const { return vw[x][T]; }
};

// The chunk's rows go to their slots in codes: workgroup blk of nblk, rows blk * kWaves + wavefront, ...
template <int D> __device__ __forceinline__ void append_rows(const PrefillFp4Params &p, int blk, int nblk, int wave, int lane)
{
    const int n_real = min(p.cu[p.S], p.C), chunks = p.Hkv * (D / 8);
    for (int row = blk * kWaves + wave; row < n_real; row += nblk * kWaves) {
        int lo = 0, hi = p.S - 1;                        // largest s with cu[s] <= row
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.cu[mid] <= row) lo = mid; else hi = mid - 1;
        }
        const int pos = p.ctx[lo] + (row - p.cu[lo]);
        if (pos < 0 || pos >= p.max_blocks * kPage) continue;        // (no such slot: malformed metadata)
        const int page = p.bt[(size_t)lo * p.max_blocks + pos / kPage];
        // (groups of four lanes, which settle an exponent between them, are whole: a row has a multiple of 8 chunks)
        for (int x = lane; x < 2 * chunks; x += 64) {
            const int which = x >= chunks, y = x - which * chunks, head = y / (D / 8), c = y % (D / 8);
            const u32x4 v = *reinterpret_cast<global_u32x4 *>((uintptr_t)((which ? p.v_new : p.k_new) + (size_t)row * p.Hkv * D + (size_t)y * 8));
            uint32_t exponent;
            const uint32_t codes = bf16_to_fp4(v, exponent);
            store_fp4<D>(reinterpret_cast<char *>(p.pages_w) + (((size_t)page * 2 + which) * p.Hkv + head) * kFp4Slab<D>, pos % kPage, c, codes, exponent);
        }
    }
}

// Three workgroups to a compute unit.  A step of 32 keys and 32 columns is 32 matrix instructions (about 16 clocks each) beside some 160 others: inside the loop the vector
// unit is what bounds it.  A launch is as much what stands around the loops: 256 rows of 32 heads over 8 in 32 segments behind 0 to 4000 tokens, 46.7 us, about 10 steps to a
// wavefront, have the vector unit busy for 32 % of the time and the matrix cores for 13, and write 59 MB (scratch memory, parts) where rows and codes are 2.4.  At heads of 128 the registers of a third of a SIMD do not hold everything: Q is read from LDS at every step, and 110 registers (416 bytes a lane) are
// kept in scratch memory.  Steps of cached keys use none of it; a step of the chunk's own rows, whose K and V are held together, loads 13 words and stores
// 4, and a tile puts some 64 away and fetches them around its steps.  (Heads of 64: no scratch memory.)  (With two workgroups, Q in registers and three steps in a ring, nothing in scratch: 512 rows of 32 heads over 8 in 7 segments behind 0 to 3000 tokens
// 65.9 us, 61.8 so; 256 of 8 over 2 behind 8000 43.0 and 40.1; 128 of 40 behind 0 to 4000 38.2 and 31.0.  Tiles of 64 columns: 65.0, 74.6 and 36.  Loads two
// steps ahead: 63.1, 40.8 and 31.0, they are there in time so.)
template <int D>
__global__ __launch_bounds__(kWaves * 64, 3) void prefill_fp4_kernel(PrefillFp4Params p)
{
    typedef Step<D> T;
    constexpr int NW = kWaves, NT = NW * 64, KS = D / 32, DJ = D / 16, NB = kNB;
    constexpr int UNITS = NB * DJ / NW;                  // accumulators of a wavefront's quarter: products j0 .. of block nb
    static_assert(DJ % UNITS == 0, "of one block");
    __shared__ __attribute__((aligned(1024))) char smem[NW * kDepth * T::BYTES];
    // Q's fragments, [block][s][lane] of 16 bytes, while a tile's steps are made; then what the wavefronts hand each other, [wavefront][unit][lane]
    __shared__ __attribute__((aligned(1024))) char area[NW * UNITS * 1024];
    static_assert(NB * KS * 1024 <= (int)sizeof(area), "Q's fragments");
    __shared__ float stat[NW][2][kCols];
    __shared__ int arrived[2];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = lane >> 4, l16 = lane & 15;
    int item = blockIdx.x;
    if (item < p.append_blocks) {
        append_rows<D>(p, item, p.append_blocks, wave, lane);
        return;
    }
    item -= p.append_blocks;
    const int W = p.ranges, n_items = W * p.Hkv;
    for (int i = item * NT + tid; i < p.n_counters; i += n_items * NT) store_global(p.counters_next + i, 0);
    const int wg = magic_div(item, p.hkv_magic), kh = item - wg * p.Hkv, g = p.g;
    const const_i32 *cu = (const const_i32 *)(uintptr_t)p.cu, *ctx = (const const_i32 *)(uintptr_t)p.ctx;
    {
        // padding rows of this kv head's query heads
        const int n_real = cu[p.S], per_row = g * (D / 8);
        if (n_real < p.C) {
            const int first = max(n_real, 0), many = (p.C - first) * per_row;
            for (int i = wg * NT + tid; i < many; i += W * NT) {
                const int r = i / per_row;
                reinterpret_cast<global_u32x4_w *>((uintptr_t)(p.out + ((size_t)(first + r) * p.Hq + (size_t)kh * g) * D))[i - r * per_row] = u32x4{0u, 0u, 0u, 0u};
            }
        }
    }

    // ---- the division.  A segment with n rows behind L tokens: tiles of it, and what each counts
    auto tiles_of = [&](int n) -> int { return (n * g + kCols - 1) / kCols; };
    auto counts = [&](int n, int L) -> int { return ((L + 31) >> 5) + ((n + 31) >> 5) + kTileSteps; };
    auto clamp_n = [&](int a, int b) -> int { return max(min(b, p.C) - max(a, 0), 0); };
    auto clamp_L = [&](int L) -> int { return min(max(L, 0), p.max_blocks * kPage); };
    Job job;
    int left, div_q, div_r, pos;
    auto enter = [&](Job &j, int s, int t) {             // tile t of segment s, whole
        j.s = s;
        j.t = t;
        j.row0 = max(cu[s], 0);
        j.n = clamp_n(cu[s], cu[s + 1]);
        j.L = clamp_L(ctx[s]);
    };
    auto shape = [&](Job &j) {                           // ... its steps: those of the rows that its last column sees
        const int last_row = magic_div(min(kCols * (j.t + 1), j.n * g) - 1, p.g_magic);
        j.cached = (j.L + 31) >> 5;
        j.steps = j.cached + (last_row >> 5) + 1;
    };
    {
        const int R = (p.S + 63) >> 6;                   // lane l looks at segments l * R ..
        int mine = 0;
        for (int i = 0; i < R; ++i) {
            const int s = lane * R + i;
            if (s < p.S) {
                const int n = clamp_n(p.cu[s], p.cu[s + 1]);
                mine += tiles_of(n) * counts(n, clamp_L(p.ctx[s]));
            }
        }
        const int incl = prefix_sum(mine);
        const int total = __builtin_amdgcn_readlane(incl, 63);
        const int ranges = min(W, (int)((uint32_t)(total + p.min_steps - 1) / (uint32_t)p.min_steps));
        if (wg >= ranges) return;
        div_q = __builtin_amdgcn_readfirstlane((int)((uint32_t)total / (uint32_t)ranges));
        div_r = total - div_q * ranges;
        pos = wg * div_q + min(wg, div_r);
        left = div_q + (int)(wg < div_r);
        int base = incl - mine, found = -1, fbase = 0, fn = 0, fL = 0;
        if (pos >= base && pos < incl)
            for (int i = 0; i < R; ++i) {
                const int s = min(lane * R + i, p.S - 1), n = clamp_n(p.cu[s], p.cu[s + 1]), L = clamp_L(p.ctx[s]), all = tiles_of(n) * counts(n, L);
                if (found < 0 && pos < base + all) { found = s; fbase = base; fn = n; fL = L; }
                base += all;
            }
        const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(found >= 0) | (1ull << 63));
        const int s = __builtin_amdgcn_readlane(found, src);
        if (s < 0) return;                               // (metadata written to while the launch runs: no address is formed from it)
        const int count = counts(__builtin_amdgcn_readlane(fn, src), __builtin_amdgcn_readlane(fL, src)), off = pos - __builtin_amdgcn_readlane(fbase, src);
        const int t = __builtin_amdgcn_readfirstlane((int)((uint32_t)off / (uint32_t)count));
        enter(job, s, t);
        if (t >= tiles_of(job.n)) return;                // (likewise)
        shape(job);
        job.seq = 0;
        job.begin = off - t * count;
        job.end = min(job.steps, job.begin + left);
        left -= min(count - job.begin, left);
        pos -= job.begin;                                // where the job's tile begins
    }
    // the tile behind j's, with `rest` of the range behind that
    auto next_job = [&](Job &j, int &rest, int &at) {
        at += counts(j.n, j.L);
        if (++j.t >= tiles_of(j.n)) {
            int s = j.s + 1;
            while (s < p.S && cu[s + 1] <= cu[s]) ++s;
            if (s >= p.S) { rest = 0; j.begin = j.end = j.cached = 0; ++j.seq; return; }
            enter(j, s, 0);
            if (j.n == 0) { rest = 0; j.begin = j.end = j.cached = 0; ++j.seq; return; }
        }
        shape(j);
        ++j.seq;
        j.begin = 0;
        j.end = min(j.steps, rest);
        rest -= min(counts(j.n, j.L), rest);
    };
    if (job.begin >= job.end) {                          // (the range begins behind a tile's steps)
        if (left == 0) return;
        next_job(job, left, pos);
        if (job.end == 0) return;
    }

    const uint32_t page_bytes = 2 * p.Hkv * kFp4Slab<D>, v_delta = p.Hkv * kFp4Slab<D>;
    const char *pool = reinterpret_cast<const char *>(p.pages) + (size_t)kh * kFp4Slab<D>;
    char *my = smem + wave * (kDepth * T::BYTES);
    const uint32_t my_lds = lds_address(my);
    const StepSource<D> source(lane, v_delta);

    // ---- Q's fragments: columns past the tile's end repeat the last one, their results are not stored
    const uint32_t area_lds = lds_address(area);
    auto load_q = [&](const Job &j) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int col = min(kCols * j.t + 16 * nb + l16, j.n * g - 1), r = magic_div(col, p.g_magic);
            const uint16_t *src = p.q + ((size_t)(j.row0 + r) * p.Hq + (size_t)kh * g + (col - r * g)) * D + grp * (D / 4);
#pragma unroll
            for (int s = 0; s < KS; ++s)
                if ((nb * KS + s) % NW == wave) dma16(src + 8 * s, area_lds + (nb * KS + s) * 1024);
        }
    };
    load_q(job);

    // ---- the wavefront's cursor over steps of cached keys: step fs of job fj goes next (fs < 0: there is none), the page ids of it and the 31 behind it
    // are in the lanes of `ids`
    Job fj = job;
    int fs = job.begin + wave, frest = left, fpos = 0, id_at = 64, ids = 0;
    auto settle = [&]() {
        while (fs >= min(fj.end, fj.cached)) {
            if (frest == 0) { fs = -1; return; }
            next_job(fj, frest, fpos);
            fs = wave;
            id_at = 64;
        }
        if (id_at == 64) {
            const int n = (fj.L + kPage - 1) / kPage, e = 2 * (fs + NW * (lane >> 1)) + (lane & 1);
            ids = 0;
            if (e < n) ids = reinterpret_cast<__attribute__((address_space(1))) const int32_t *>((uintptr_t)(p.bt + (size_t)fj.s * p.max_blocks))[e];
            wait_vm<0>();                                // (here, once in 32 steps: the compiler's own wait stands at every step, where it drains the loads in flight)
            id_at = 0;
        }
    };
    // steps in flight; the first one's K is on its way into registers
    int many = 0;
    uint32_t place_in = 0, place_out = 0;                // bytes
    auto turn = [](uint32_t &place) { place = place == (kDepth - 1) * T::BYTES ? 0 : place + T::BYTES; };
    auto issue = [&]() {
        const int pg0 = __builtin_amdgcn_readlane(ids, id_at), pg1 = __builtin_amdgcn_readlane(ids, id_at + 1);
        id_at += 2;
        issue_step<D, false>(source, pool + (size_t)pg0 * page_bytes, pool + (size_t)pg1 * page_bytes, v_delta, lane, my_lds + place_in);
        turn(place_in);
        ++many;
        fs += NW;
        settle();
    };
    auto lds_reads_done = [&]() {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(15 | 3 << 14 | 7 << 4);           // (vector memory is not waited for)
        asm volatile("" ::: "memory");
    };
    StepCodes<D> codes;
    settle();
    if (fs >= 0) issue();
    const bool any = many != 0;
    if (fs >= 0) issue();
    static_assert(kDepth == 2, "the first loads, and waits for what is in flight");
    if (many == 2) wait_vm<T::LOADS>();
    else wait_vm<0>();
    if (any) codes.read_k(my, grp, l16);

    // What this workgroup has left of tiles cut between workgroups, two at most: where their rows are, arrival counter, parts and where they are.
    int cut_row0[2], cut_n[2], cut_t[2], cut_counter[2], cut_pieces[2], cut_w0[2], cuts = 0;
    auto place_of = [&](int w0, int i) -> float * { return p.scratch + ((size_t)(2 * (w0 + i) + (int)(i == 0)) * p.Hkv + kh) * kPartFloats<D>; };
    const int my_nb = wave * UNITS / DJ, my_j = wave * UNITS % DJ;       // the wavefront's quarter
    // the wavefront's quarter of a finished tile: row 4 * grp + i of product j is d = DJ * (4 * grp + i) + j
    auto write_quarter = [&](int row0, int t, int cols, const f32x4 (&o)[UNITS], float inv) {
        const int col = 16 * my_nb + l16;
        if (col >= cols) return;
        const int all = kCols * t + col, r = magic_div(all, p.g_magic);
        uint16_t *to = p.out + ((size_t)(row0 + r) * p.Hq + (size_t)kh * g + (all - r * g)) * D + my_j;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w[UNITS / 2];
#pragma unroll
            for (int u = 0; u < UNITS; u += 2) {
                bf16x2 y;
                y[0] = (__bf16)(o[u][i] * inv);
                y[1] = (__bf16)(o[u + 1][i] * inv);
                w[u / 2] = __builtin_bit_cast(uint32_t, y);
            }
            uint16_t *at = to + DJ * (4 * grp + i);
            if constexpr (UNITS == 8) *reinterpret_cast<global_u32x4_w *>((uintptr_t)at) = u32x4{w[0], w[1], w[2], w[3]};
            else if constexpr (UNITS == 4) *reinterpret_cast<global_u32x2_w *>((uintptr_t)at) = u32x2{w[0], w[1]};
            else *reinterpret_cast<__attribute__((address_space(1))) uint32_t *>((uintptr_t)at) = w[0];
        }
    };
    const float c = p.c;
    const bool neg = p.neg != 0;
    Columns<D, NB> x;
    auto q_of = [&](int nb, int s) -> bf16x8 { return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(area + (nb * KS + s) * 1024 + lane * 16)); };

    lds_barrier();                                       // (everybody's part of Q is older than a wavefront's first step)
    for (;;) {                                           // the jobs of the range
        x.clear();
        int row_of[NB];                                  // the row of the lane's column
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) row_of[nb] = magic_div(min(kCols * job.t + 16 * nb + l16, job.n * g - 1), p.g_magic);
        // ---- cached keys.  A step: K's codes have arrived, V's are asked for; behind the scores the next step's K; behind the weights the place is free
        // for the loads of the last step behind it
        for (int cs = job.begin + wave; cs < min(job.end, job.cached); cs += NW) {
            lds_reads_done();
            if (neg) codes.negate_k();
            f32x4 sc[NB][2];
            x.scores(codes, q_of, sc);
            __builtin_amdgcn_sched_barrier(0);
            codes.read_v(my + place_out, grp, l16);
            --many;
            turn(place_out);
            if (many > 0) {
                wait_vm<0>();
                codes.read_k(my + place_out, grp, l16);
            }
            const int n = job.L - 32 * cs;               // slots past the end are masked
            if (n < 32) {
#pragma unroll
                for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (16 * pg + 4 * i + grp >= n) {
#pragma unroll
                            for (int nb = 0; nb < NB; ++nb) sc[nb][pg][i] = -INFINITY;
                        }
            }
            bf16x8 pf[NB];
            x.weigh(sc, c, pf);
            lds_reads_done();
            if (fs >= 0) issue();
            codes.powers(l16);
            if (n < 32) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (16 * (i / 4) + 4 * (i % 4) + grp >= n) codes.vs[i] = 0.f;
            }
            x.add(codes, pf);
        }
        // ---- the chunk's own rows
        {
            const size_t at = ((size_t)job.row0 * p.Hkv + kh) * D, row_elements = (size_t)p.Hkv * D;
            const int seen = magic_div(min(kCols * (job.t + 1), job.n * g) - 1, p.g_magic);          // the last row that a column sees
            int s = job.begin + wave;
            if (s < job.cached) s += (job.cached - s + NW - 1) / NW * NW;
            for (; s < job.end; s += NW) {
                const int first = 32 * (s - job.cached);
                NewRows<D> rows;
                rows.load(p.k_new + at, p.v_new + at, row_elements, first, seen, grp, l16);
                if (neg) rows.negate_k();
                f32x4 sc[NB][2];
                x.scores(rows, q_of, sc);
#pragma unroll
                for (int pg = 0; pg < 2; ++pg)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int nb = 0; nb < NB; ++nb)
                            if (first + 16 * pg + 4 * i + grp > row_of[nb]) sc[nb][pg][i] = -INFINITY;
                bf16x8 pf[NB];
                x.weigh(sc, c, pf);
                x.add(rows, pf);
            }
        }
        // ---- the job is done: the wavefronts merge
        Job after = job;
        int after_pos = pos;
        const bool more = left != 0 && (next_job(after, left, after_pos), after.end != 0);
        const bool whole = job.begin == 0 && job.end == job.steps;
        const int cols = min(kCols, job.n * g - kCols * job.t);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            if (grp == 0) { stat[wave][0][16 * nb + l16] = x.m[nb]; stat[wave][1][16 * nb + l16] = x.lsum[nb][0]; }
        lds_barrier();                                   // (also: everybody is done with Q)
        const int my_col = 16 * my_nb + l16;
        float top = stat[0][0][my_col], sum = 0.f;
#pragma unroll
        for (int i = 1; i < NW; ++i) top = fmaxf(top, stat[i][0][my_col]);
#pragma unroll
        for (int i = 0; i < NW; ++i) sum = __builtin_fmaf(stat[i][1][my_col], __builtin_amdgcn_exp2f(stat[i][0][my_col] - top), sum);
        f32x4 mine[UNITS];
        auto each_quarter = [&](int which, auto &&f) {   // f with the accumulators of quarter `which` (registers have no computed index)
            auto of = [&](auto w) {
                constexpr int U = decltype(w)::value * UNITS;
#pragma unroll
                for (int u = 0; u < UNITS; ++u) f(u, x.o[U / DJ][U % DJ + u]);
            };
            switch (which) {
            case 0: of(std::integral_constant<int, 0>()); break;
            case 1: of(std::integral_constant<int, 1>()); break;
            case 2: of(std::integral_constant<int, 2>()); break;
            default: of(std::integral_constant<int, 3>()); break;
            }
        };
        {
            const float w = __builtin_amdgcn_exp2f(stat[wave][0][my_col] - top);
            each_quarter(wave, [&](int u, const f32x4 &o) { mine[u] = o * w; });
        }
#pragma unroll 1
        for (int r = 1; r < NW; ++r) {
            if (r != 1) lds_barrier();                   // everybody has read the round before
            each_quarter(wave ^ r, [&](int u, const f32x4 &o) { *reinterpret_cast<f32x4 *>(area + (wave * UNITS + u) * 1024 + lane * 16) = o; });
            lds_barrier();
            const float w = __builtin_amdgcn_exp2f(stat[wave ^ r][0][my_col] - top);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const f32x4 z = *reinterpret_cast<const f32x4 *>(area + ((wave ^ r) * UNITS + u) * 1024 + lane * 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) mine[u][i] = __builtin_fmaf(z[i], w, mine[u][i]);
            }
        }
        if (whole) {
            write_quarter(job.row0, job.t, cols, mine, 1.0f / sum);
        } else {
            auto owner = [&](int y) -> int {             // the range that has position y of the sequence
                const int cut = div_r * (div_q + 1);
                return __builtin_amdgcn_readfirstlane(y < cut ? (int)((uint32_t)y / (uint32_t)(div_q + 1)) : div_r + (int)((uint32_t)(y - cut) / (uint32_t)div_q));
            };
            const int w0 = owner(pos), pieces = owner(pos + job.steps - 1) - w0 + 1;
            if (cuts == 0) { cut_row0[0] = job.row0; cut_n[0] = job.n; cut_t[0] = job.t; cut_counter[0] = w0 * p.Hkv + kh; cut_pieces[0] = pieces; cut_w0[0] = w0; }
            else { cut_row0[1] = job.row0; cut_n[1] = job.n; cut_t[1] = job.t; cut_counter[1] = w0 * p.Hkv + kh; cut_pieces[1] = pieces; cut_w0[1] = w0; }
            ++cuts;
            float *part = place_of(w0, wg - w0);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) store_coherent(reinterpret_cast<f32x4 *>(part) + (wave * UNITS + u) * 64 + lane, mine[u]);
            if (grp == 0 && my_j == 0) {
                store_coherent(part + kCols * D + my_col, top);
                store_coherent(part + kCols * D + kCols + my_col, sum);
            }
        }
        if (!more) break;
        job = after;
        pos = after_pos;
        lds_barrier();                                   // everybody is done with stat and area
        load_q(job);
        wait_vm<0>();
        lds_barrier();
    }
    if (cuts == 0) return;
    coherent_stores_done();
    lds_barrier();
    if (tid < cuts) arrived[tid] = atomic_add_global(p.counters + (tid == 0 ? cut_counter[0] : cut_counter[1]), 1);
    lds_barrier();
    for (int k = 0; k < cuts; ++k) {
        const int pieces = k == 0 ? cut_pieces[0] : cut_pieces[1], first = k == 0 ? cut_w0[0] : cut_w0[1];
        if (__builtin_amdgcn_readfirstlane(arrived[k]) != pieces - 1) continue;
        // all the others have been here: the counter goes back to zero, every wavefront merges its quarter of the parts, in their order, two at a time
        if (tid == 0) store_global(p.counters + (k == 0 ? cut_counter[0] : cut_counter[1]), 0);
        const int row0 = k == 0 ? cut_row0[0] : cut_row0[1], t = k == 0 ? cut_t[0] : cut_t[1], cols = min(kCols, (k == 0 ? cut_n[0] : cut_n[1]) * g - kCols * t);
        float top = -INFINITY, sum = 0.f;
        f32x4 o[UNITS];
#pragma unroll
        for (int u = 0; u < UNITS; ++u) o[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        constexpr int AT_ONCE = 4;
        for (int i0 = 0; i0 < pieces; i0 += AT_ONCE) {
            float mi[AT_ONCE], li[AT_ONCE];
            float2 z[AT_ONCE][UNITS][2];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const float *part = place_of(first, min(i0 + i, pieces - 1));
                mi[i] = load_coherent(part + kCols * D + 16 * my_nb + l16);
                li[i] = load_coherent(part + kCols * D + kCols + 16 * my_nb + l16);
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    z[i][u][0] = load_coherent2(part + ((wave * UNITS + u) * 64 + lane) * 4);
                    z[i][u][1] = load_coherent2(part + ((wave * UNITS + u) * 64 + lane) * 4 + 2);
                }
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i)
                if (i0 + i < pieces) {
                    const float m_new = fmaxf(top, mi[i]), w_old = __builtin_amdgcn_exp2f(top - m_new), w = __builtin_amdgcn_exp2f(mi[i] - m_new);
                    top = m_new;
                    sum = __builtin_fmaf(li[i], w, sum * w_old);
#pragma unroll
                    for (int u = 0; u < UNITS; ++u) {
                        o[u][0] = __builtin_fmaf(z[i][u][0].x, w, o[u][0] * w_old);
                        o[u][1] = __builtin_fmaf(z[i][u][0].y, w, o[u][1] * w_old);
                        o[u][2] = __builtin_fmaf(z[i][u][1].x, w, o[u][2] * w_old);
                        o[u][3] = __builtin_fmaf(z[i][u][1].y, w, o[u][3] * w_old);
                    }
                }
        }
        write_quarter(row0, t, cols, o, 1.0f / sum);
    }
}

}  // namespace

hipError_t tetri_launch_prefill_fp4(int head_dim, const PrefillFp4Params &p, hipStream_t stream)
{
    auto kernel = head_dim == 128 ? prefill_fp4_kernel<128> : prefill_fp4_kernel<64>;
    hipLaunchKernelGGL(kernel, dim3(p.append_blocks + p.ranges * p.Hkv), dim3(kWaves * 64), 0, stream, p);
    return hipGetLastError();
}
