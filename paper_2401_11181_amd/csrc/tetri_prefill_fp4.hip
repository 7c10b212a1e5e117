// Chunked-prefill attention over a paged cache of 4-bit codes for gfx950 where chunks give little work: tetri_attn.hip's kernel gives a row tile to a
// workgroup, which then walks all keys, 128 at a time, behind barriers; here a tile is a quarter as large and any number of workgroups share its keys.
//
//   * A tile is 32 columns of one kv head: neighbouring (row, query head of the kv head) pairs of a segment, rows first, so that codes become bf16
//     once for all heads that share them.  A wavefront takes whole steps of 32 keys by itself (fp4_steps.h), from a ring in LDS; no barrier
//     stands between steps.  The chunk's own rows are steps as well, of bf16 rows that go straight into registers.
//   * The steps of all tiles of a kv head, tile after tile, are cut into equal ranges, a workgroup each, worked out on the device from the
//     segments' lengths, the same for every kv head.  A tile counts with all new rows of its segment, whatever its rows see of them, and with
//     kTileSteps more.  The wavefronts of a workgroup take a tile's steps in turn and merge in LDS when it is done.
//   * Tiles cut between workgroups meet through arrival counters in the same launch, as in tetri_decode.hip: the workgroup that arrives last merges the
//     parts in their order.  Nobody waits.
//   * Workgroups of a kv head run on one XCD (or two, four, eight where there are few kv heads): tiles of a segment read the same keys through its L2.
//   * The chunk's rows are cached in codes by a few workgroups in front of the others; padding rows of the output are zeroed by all.
#include "fp4_steps.h"

namespace {

using namespace tetri_dev;

constexpr int kWaves = 4;         // wavefronts of a workgroup
constexpr int kDepth = 2;         // steps a wavefront's ring holds
constexpr int kNB = 2;            // blocks of 16 columns
constexpr int kCols = 16 * kNB;
constexpr int kMergeCols = 8;     // columns whose partial O the merge area in LDS holds at a time
constexpr int kTileSteps = 4;     // what a tile costs a range beside its steps, in steps
constexpr int kBatch = 64;        // parts whose weights the merge of a cut tile holds at a time

// A workgroup's partial result: O of the columns (unnormalised), their m, their row sums.
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

template <int D>
__global__ __launch_bounds__(kWaves * 64, 2) void prefill_fp4_kernel(PrefillFp4Params p)
{
    typedef Step<D> T;
    constexpr int NW = kWaves, NT = NW * 64, NB = kNB;
    __shared__ __attribute__((aligned(1024))) char smem[NW * kDepth * T::BYTES];
    __shared__ __attribute__((aligned(16))) float area[NW][kMergeCols][D];
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
            id_at = 0;
        }
    };
    auto issue = [&](int place) {
        const int pg0 = __builtin_amdgcn_readlane(ids, id_at), pg1 = __builtin_amdgcn_readlane(ids, id_at + 1);
        id_at += 2;
        issue_step<D>(source, pool + (size_t)pg0 * page_bytes, pool + (size_t)pg1 * page_bytes, v_delta, lane, my_lds + place * T::BYTES);
    };
    int ahead = 0, rj[kDepth], rs[kDepth], place_in = 0, place_out = 0;
    settle();
#pragma unroll
    for (int i = 0; i < kDepth; ++i) {
        rj[i] = 0; rs[i] = -1;
        if (fs >= 0) {
            issue(place_in);
            if (++place_in == kDepth) place_in = 0;
            rj[i] = fj.seq; rs[i] = fs;
            ++ahead;
            fs += NW;
            settle();
        }
    }

    // What this workgroup has left of tiles cut between workgroups, two at most: where their rows are, arrival counter, parts and where they are.
    int cut_row0[2], cut_n[2], cut_t[2], cut_counter[2], cut_pieces[2], cut_w0[2], cuts = 0;
    auto place_of = [&](int w0, int i) -> float * { return p.scratch + ((size_t)(2 * (w0 + i) + (int)(i == 0)) * p.Hkv + kh) * kPartFloats<D>; };
    auto out_of = [&](int row0, int col) -> uint16_t * {
        const int r = magic_div(col, p.g_magic);
        return p.out + ((size_t)(row0 + r) * p.Hq + (size_t)kh * g + (col - r * g)) * D;
    };
    auto write_pair = [&](uint16_t *to, float a, float b, float inv) {
        bf16x2 r;
        r[0] = (__bf16)(a * inv);
        r[1] = (__bf16)(b * inv);
        *reinterpret_cast<__attribute__((address_space(1))) uint32_t *>((uintptr_t)to) = __builtin_bit_cast(uint32_t, r);
    };
    const float c = p.c;
    Columns<D, NB> x;

    for (;;) {                                           // the jobs of the range
        x.clear();
        int row_of[NB];                                  // the row of the lane's column
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int col = min(kCols * job.t + 16 * nb + l16, job.n * g - 1);       // (columns past the end repeat the last one: their results are not stored)
            row_of[nb] = magic_div(col, p.g_magic);
            const global_u32x4 *qp = reinterpret_cast<const global_u32x4 *>((uintptr_t)(p.q + ((size_t)(job.row0 + row_of[nb]) * p.Hq + (size_t)kh * g + (col - row_of[nb] * g)) * D
                                                                                        + grp * (D / 4)));
#pragma unroll
            for (int s = 0; s < D / 32; ++s) {
                u32x4 v = u32x4(qp[s]);
                if (p.neg) v ^= 0x80008000u;             // (a negative scale is Q's sign)
                x.qf[nb][s] = __builtin_bit_cast(bf16x8, v);
            }
        }
        // ---- cached keys
        while (rs[0] >= 0 && rj[0] == job.seq) {
            const int cs = rs[0];
            if (ahead == 1) wait_vm<0>();
            else wait_vm<T::LOADS>();
            static_assert(kDepth == 2, "a wait for one step behind the current one");
            StepCodes<D> codes;
            codes.read(my + place_out * T::BYTES, grp, l16);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // everything is in registers: the place may be overwritten
            const bool far = fs >= 0;
            if (far) issue(place_in);
            if (++place_out == kDepth) place_out = 0;
            codes.powers(l16);
            f32x4 sc[NB][2];
            x.scores(codes, sc);
            if (32 * cs + 32 > job.L) {                  // slots past the end are masked
                const int n = job.L - 32 * cs;
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
            rj[0] = rj[1]; rs[0] = rs[1];
            rs[1] = -1;
            --ahead;
            if (far) {
                rj[1] = fj.seq; rs[1] = fs;
                ++ahead;
                if (++place_in == kDepth) place_in = 0;
                fs += NW;
                settle();
            }
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
                f32x4 sc[NB][2];
                x.scores(rows, sc);
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
        const bool whole = job.begin == 0 && job.end == job.steps;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            if (grp == 0) { stat[wave][0][16 * nb + l16] = x.m[nb]; stat[wave][1][16 * nb + l16] = x.lsum[nb][0]; }
        int piece = 0, w0 = 0;
        if (!whole) {
            auto owner = [&](int y) -> int {             // the range that has position y of the sequence
                const int cut = div_r * (div_q + 1);
                return __builtin_amdgcn_readfirstlane(y < cut ? (int)((uint32_t)y / (uint32_t)(div_q + 1)) : div_r + (int)((uint32_t)(y - cut) / (uint32_t)div_q));
            };
            w0 = owner(pos);
            piece = wg - w0;
            const int pieces = owner(pos + job.steps - 1) - w0 + 1;
            if (cuts == 0) { cut_row0[0] = job.row0; cut_n[0] = job.n; cut_t[0] = job.t; cut_counter[0] = w0 * p.Hkv + kh; cut_pieces[0] = pieces; cut_w0[0] = w0; }
            else { cut_row0[1] = job.row0; cut_n[1] = job.n; cut_t[1] = job.t; cut_counter[1] = w0 * p.Hkv + kh; cut_pieces[1] = pieces; cut_w0[1] = w0; }
            ++cuts;
        }
        float *part = place_of(w0, piece);
        const int cols = min(kCols, job.n * g - kCols * job.t);
        for (int c0 = 0; c0 < cols; c0 += kMergeCols) {
            if (c0 != 0) lds_barrier();                  // everybody is done with the columns before
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int col = 16 * nb + l16;
                if (col >= c0 && col < c0 + kMergeCols) x.put(nb, area[wave][col - c0], grp);
            }
            lds_barrier();
            for (int v = tid; v < min(cols - c0, kMergeCols) * (D / 2); v += NT) {
                const int cc = v / (D / 2), col = c0 + cc, d = 2 * (v - cc * (D / 2));
                float ms = stat[0][0][col];
#pragma unroll
                for (int i = 1; i < NW; ++i) ms = fmaxf(ms, stat[i][0][col]);
                float a = 0.f, b = 0.f, l = 0.f;
#pragma unroll
                for (int i = 0; i < NW; ++i) {
                    const float w = __builtin_amdgcn_exp2f(stat[i][0][col] - ms);
                    const float2 z = *reinterpret_cast<const float2 *>(&area[i][cc][d]);
                    a = __builtin_fmaf(z.x, w, a);
                    b = __builtin_fmaf(z.y, w, b);
                    l = __builtin_fmaf(stat[i][1][col], w, l);
                }
                if (whole) {
                    write_pair(out_of(job.row0, kCols * job.t + col) + d, a, b, 1.0f / l);
                } else {
                    store_coherent2(part + col * D + d, a, b);
                    if (d == 0) {
                        store_coherent(part + kCols * D + col, ms);
                        store_coherent(part + kCols * D + kCols + col, l);
                    }
                }
            }
        }
        if (left == 0) break;
        next_job(job, left, pos);
        if (job.end == 0) break;
        lds_barrier();                                   // everybody is done with stat and area
    }
    if (cuts == 0) return;
    coherent_stores_done();
    lds_barrier();
    if (tid < cuts) arrived[tid] = atomic_add_global(p.counters + (tid == 0 ? cut_counter[0] : cut_counter[1]), 1);
    lds_barrier();
    for (int k = 0; k < cuts; ++k) {
        const int pieces = k == 0 ? cut_pieces[0] : cut_pieces[1], first = k == 0 ? cut_w0[0] : cut_w0[1];
        if (__builtin_amdgcn_readfirstlane(arrived[k]) != pieces - 1) continue;
        // all the others have been here: the counter goes back to zero, the parts are merged in their order
        if (tid == 0) store_global(p.counters + (k == 0 ? cut_counter[0] : cut_counter[1]), 0);
        const int row0 = k == 0 ? cut_row0[0] : cut_row0[1], t = k == 0 ? cut_t[0] : cut_t[1], cols = min(kCols, (k == 0 ? cut_n[0] : cut_n[1]) * g - kCols * t);
        float (*wts)[kCols] = reinterpret_cast<float (*)[kCols]>(smem);              // (the ring is empty)
        float *met = &area[0][0][0];                                                 // [8][kCols] of m, [8][kCols] of the row sum
        static_assert(kBatch * kCols * 4 <= (int)sizeof(smem) && NT == 8 * kCols, "eight threads to a column");
        // the largest exponent and the sum under it: of every eighth part first
        const int col = tid % kCols, sub = tid / kCols;
        float mm = -INFINITY, l = 0.f;
        for (int i0 = sub; i0 < pieces; i0 += 8 * 4) {
            float mi[4], li[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float *src = place_of(first, min(i0 + 8 * i, pieces - 1)) + kCols * D + col;
                mi[i] = load_coherent(src);
                li[i] = load_coherent(src + kCols);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i0 + 8 * i < pieces) {
                    const float m_new = fmaxf(mm, mi[i]);
                    l = __builtin_fmaf(li[i], __builtin_amdgcn_exp2f(mi[i] - m_new), l * __builtin_amdgcn_exp2f(mm - m_new));
                    mm = m_new;
                }
        }
        lds_barrier();                                   // everybody is done with area and the ring
        met[sub * kCols + col] = mm;
        met[(8 + sub) * kCols + col] = l;
        lds_barrier();
        float top = met[col], sum = 0.f;
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, met[i * kCols + col]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(met[(8 + i) * kCols + col], __builtin_amdgcn_exp2f(met[i * kCols + col] - top), sum);
        if (sub == 0) stat[0][0][col] = 1.0f / sum;
        // ... then O, two neighbouring values of a column per thread and pass
        constexpr int PASSES = kCols * (D / 2) / NT;
        float a[PASSES], b[PASSES];
#pragma unroll
        for (int u = 0; u < PASSES; ++u) a[u] = b[u] = 0.f;
        for (int b0 = 0; b0 < pieces; b0 += kBatch) {
            const int n = min(kBatch, pieces - b0);
            if (b0 != 0) lds_barrier();                  // everybody is done with the weights before
            for (int i = sub; i < n; i += 8) wts[i][col] = __builtin_amdgcn_exp2f(load_coherent(place_of(first, b0 + i) + kCols * D + col) - top);
            lds_barrier();
            for (int i0 = 0; i0 < n; i0 += 4) {
                float2 z[4][PASSES];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int u = 0; u < PASSES; ++u) z[i][u] = load_coherent2(place_of(first, b0 + min(i0 + i, n - 1)) + 2 * (tid + u * NT));
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i0 + i < n) {
#pragma unroll
                        for (int u = 0; u < PASSES; ++u) {
                            const float w = wts[i0 + i][(tid + u * NT) / (D / 2)];
                            a[u] = __builtin_fmaf(z[i][u].x, w, a[u]);
                            b[u] = __builtin_fmaf(z[i][u].y, w, b[u]);
                        }
                    }
            }
        }
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
            const int v = tid + u * NT, cc = v / (D / 2), d = 2 * (v - cc * (D / 2));
            if (cc < cols) write_pair(out_of(row0, kCols * t + cc) + d, a[u], b[u], stat[0][0][cc]);
        }
        lds_barrier();
    }
}

}  // namespace

hipError_t tetri_launch_prefill_fp4(int head_dim, const PrefillFp4Params &p, hipStream_t stream)
{
    auto kernel = head_dim == 128 ? prefill_fp4_kernel<128> : prefill_fp4_kernel<64>;
    hipLaunchKernelGGL(kernel, dim3(p.append_blocks + p.ranges * p.Hkv), dim3(kWaves * 64), 0, stream, p);
    return hipGetLastError();
}
