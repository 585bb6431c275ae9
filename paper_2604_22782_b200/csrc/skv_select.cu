// Selection of pages by a cheap score (skv_select_pages).  For a run of rows (a decode step's row, or up to 128 / G of a chunk) and
// a kv head:  the queries in whole steps of a 127th of their largest element, c;  of every full page p before the run's last pages
//     dot(p) = max over rows and query heads of  sum_d  max(c_d, 0) highest_d(p) + min(c_d, 0) lowest_d(p),
// the largest that a key inside the page's bounds could give;  score(p) = dot(p) x the page's step;  and the `top` pages of the
// highest score, of two equal ones the lower.  dot is a sum of whole numbers below 2^24, exact in any order, so the selection does
// not depend on how the work is cut.
//
// The sum over [max(c, 0) | min(c, 0)] and [highest | lowest] is one product of length 2 D on the tensor cores in 8 bits, of
// pages against columns (rows x query heads).  Up to 16 columns: select_few_kernel, mma.sync, 16 pages against 8 columns an instruction.
// A warp loads 16 entries straight into the fragments: the order of the contracted dims is free as long as both sides agree, so a
// lane's 16 consecutive bytes serve two instructions.  Where there are few segments -- (run, kv head) -- a cluster of CTAs shares one
// and writes its scores, as whole numbers that order as they do, into the first CTA's shared memory.  More columns:
// select_many_kernel, tcgen05 (kind i8), tiles of 128 pages against all columns, whose scores a thread per page reduces.
// The CTA then finds the top-th largest score by counting into 2048 bins between lowest and highest; what lies in the bin where it is
// goes by direct comparison, or where that is more than a warp holds, through bins again.
// The scores' room in shared memory is that of the page table's width, not of the sequences: select_many_kernel's two CTAs fit an SM up to 3968 entries
// at 128 columns of 128 dims, and one where a table is wider.
// Bound by HBM with many segments of few columns (2 D + 4 bytes a page and head), by the tensor cores and their operands with many
// columns, by latency with few segments.
// Measured, 8 heads of 128, 32 query heads: one sequence of 32767 tokens 7.0 us (scores 4.7, choosing 2.3), 64 of 8192 to 32767 36.5 us (4.7 TB/s),
// two chunks of 1024 rows behind 30000 tokens, 32 to a list, 44.5 us (1.4 POP/s, 43 % of twice the bf16 rate: an item's beginning -- the
// queries' codes -- and its end -- choosing -- leave the tensor cores to the other CTA of the SM).
#include "skv_page_index.cuh"
#include "skv_prefill_parts.cuh"
#include "skv_segment.cuh"
#include "skv_tcgen05.cuh"

namespace skv {

namespace {

using chunk::mbar_arrive;
using chunk::swizzled_desc;

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int WARPS = 8, THREADS = WARPS * 32;
constexpr int BINS = 2048;
constexpr int FEW = 16;                // columns up to which mma.sync does
constexpr int MAX_PAGES = 45056, MAX_PAGES_MANY = 28672;      // of a sequence: the scores of a segment are in one CTA's shared memory
constexpr int WORDS = 96;              // of shared memory, for choose() and what comes before it

// D(16x8, s32) += A(16x32, s8, row) * B(32x8, s8, col)
__device__ __forceinline__ void mma_s8_16832(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// a page's score as a whole number that orders as the value does; -0 as +0
__device__ __forceinline__ uint32_t key_of(int dot, float scale)
{
    const float inf = __uint_as_float(0x7F800000u), x = scale == inf ? inf : (float)dot * scale + 0.f;
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// What a list is made of: pages [0, first), those chosen of [first, first + scored), pages [last, end).
struct Run {
    int b, row, rows;       // sequence; its first row of Q, rows (0: an empty list)
    int first, scored, last, end;
};

__device__ __forceinline__ Run run_of(const SelectParams &p, int list, bool report)
{
    Run r = {};
    r.b = list / p.per_seq;
    const int i = list - r.b * p.per_seq;
    int n = __ldg(p.seq_lens + r.b), pos = n - 1;
    if (p.cu_q) {
        const int first = __ldg(p.cu_q + r.b), len = __ldg(p.cu_q + r.b + 1) - first;
        if (first < 0 || len < 0 || len > n || len > p.max_q_len || (int64_t)n > (int64_t)p.pt_stride * PAGE) {
            if (report && i == 0) atomicOr(p.status, STATUS_BOUNDS);
            return r;
        }
        const int at = i * p.run;              // (below max_q_len, since i < per_seq)
        if (at >= len) return r;
        r.row = first + at;
        r.rows = rows_of_run(len - at, p.run);
        pos = n - len + at;
    } else {
        if (n <= 0) return r;
        if ((int64_t)n > (int64_t)p.pt_stride * PAGE) {
            n = p.pt_stride * PAGE;
            pos = n - 1;
            if (report) atomicOr(p.status, STATUS_BOUNDS);
        }
        r.row = r.b;
        r.rows = 1;
    }
    const int own = pos / PAGE;
    r.end = (pos + r.rows - 1) / PAGE + 1;
    r.first = p.first < r.end ? p.first : r.end;
    r.last = own >= p.last ? own - p.last + 1 : 0;
    if (r.last < r.first) r.last = r.first;
    r.scored = r.last - r.first;
    return r;
}

// every page of the sequence, where there is nothing to choose: by THREADS threads
__device__ __forceinline__ void list_all(const SelectParams &p, int seg, const Run &run, int tid)
{
    int32_t *out = p.lists + (int64_t)seg * p.stride;
    for (int i = tid; i < p.stride; i += THREADS) out[i] = i < run.end ? i : -1;
    if (tid == 0) p.counts[seg] = run.end;
}

__device__ __forceinline__ void sync_threads() { asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory"); }

// (What runs once in a CTA is kept small below, loops rolled: straight code that is new to the SM comes in at some 10 cycles an
// instruction, and made the queries' codes take 10000 cycles, choose() 8000.)

// the largest of a piece of 8 dims; an element that is not finite counts as 0
__device__ __forceinline__ uint32_t magnitude(uint32_t bits) { return bits >= 0x7F80u ? 0u : bits; }
__device__ __forceinline__ uint32_t largest(const uint4 &w)
{
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = max(top, max(magnitude(x[k] & 0x7FFFu), magnitude(x[k] >> 16 & 0x7FFFu)));
    return top;
}
// two dims in steps, in the low bytes: x * inv is 127 and a rounding at most, or x was not finite
__device__ __forceinline__ uint32_t step_of(float x, float inv)
{
    const float y = __fmul_rn(x, inv);
    return __float_as_uint(__fadd_rn(fabsf(y) < 128.f ? y : 0.f, 12582912.f));      // 1.5 * 2^23: the nearest whole number is in the low bits
}
// 8 dims of a row in steps: [max(c, 0)] and [min(c, 0)], a byte each
__device__ __forceinline__ void steps_of(const uint4 &w, float inv, uint2 &up, uint2 &down)
{
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    uint32_t c[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t lo = __byte_perm(step_of(bf16_lo(x[2 * k]), inv), step_of(bf16_hi(x[2 * k]), inv), 0x0040);
        const uint32_t hi = __byte_perm(step_of(bf16_lo(x[2 * k + 1]), inv), step_of(bf16_hi(x[2 * k + 1]), inv), 0x0040);
        c[k] = __byte_perm(lo, hi, 0x5410);
    }
    uint32_t sign0, sign1;                     // every byte's sign, all over it
    asm("prmt.b32 %0, %1, 0, 0xba98;" : "=r"(sign0) : "r"(c[0]));
    asm("prmt.b32 %0, %1, 0, 0xba98;" : "=r"(sign1) : "r"(c[1]));
    up = make_uint2(c[0] & ~sign0, c[1] & ~sign1);
    down = make_uint2(c[0] & sign0, c[1] & sign1);
}
// 127 / a for the largest element's bits in words[0 .. WARPS) (one of each warp's threads), which all THREADS have written
__device__ __forceinline__ float steps_per_unit(const uint32_t *words, int lane)
{
    const float amax = __uint_as_float(__reduce_max_sync(FULL, words[lane & (WARPS - 1)]) << 16);
    return amax < INDEX_TINY ? 0.f : __fdiv_rn(127.f, amax);
}

// The least and the largest of a segment's numbers, as they are written: one for each of lo_hi[0], lo_hi[1] of the first CTA
__device__ __forceinline__ void note_range(uint32_t lo_hi, uint32_t lo, uint32_t hi, int lane)
{
    lo = __reduce_min_sync(FULL, lo);
    hi = __reduce_max_sync(FULL, hi);
    if (lane == 0) {
        asm volatile("red.relaxed.cluster.shared::cluster.min.u32 [%0], %1;" ::"r"(lo_hi), "r"(lo) : "memory");
        asm volatile("red.relaxed.cluster.shared::cluster.max.u32 [%0], %1;" ::"r"(lo_hi + 4), "r"(hi) : "memory");
    }
}

// By THREADS threads: the list of a run whose scores' numbers are keys[0 .. run.scored), more than p.top of them, the least and the largest
// in words[0] and words[1].  keys and bins [BINS] are aligned to 16 bytes (keys may be read up to 7 past the end); bins and
// words [2 .. WORDS) are its own.  A thread has 8 pages in a row, a round of the threads 2048; where there is one round they stay in registers.
__device__ __forceinline__ void choose(const SelectParams &p, int seg, const Run &run, const uint32_t *keys, uint32_t *bins, uint32_t *words, int tid)
{
    constexpr int MINE = 8, ROUND = THREADS * MINE;
    const int lane = tid & 31, warp = tid >> 5, n = p.top > 0 ? run.scored : 0;
    int32_t *out = p.lists + (int64_t)seg * p.stride;
    uint32_t k[MINE];
    auto load = [&](int r0) {                  // (0 where there is none, which is below every score's number)
        const int i = r0 + tid * MINE;
        uint4 u = make_uint4(0, 0, 0, 0), v = u;
        if (i < n) {
            u = *reinterpret_cast<const uint4 *>(keys + i);
            v = *reinterpret_cast<const uint4 *>(keys + i + 4);
        }
        const uint32_t x[MINE] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
        for (int m = 0; m < MINE; ++m) k[m] = i + m < n ? x[m] : 0u;
    };
    uint32_t lo = words[0], hi = words[1];
    // everything above `limit` is taken, and the first `ties` that equal it
    uint32_t limit = 0xFFFFFFFFu;              // (no score's number: that of NaN)
    int need = p.top, ties = 0;
    int shift = 32 - __clz((int)(hi - lo));    // 2^shift > hi - lo
    shift = shift > 11 ? shift - 11 : 0;
    load(0);
    while (need > 0) {
#pragma unroll 1
        for (int i = tid; i < BINS / 4; i += THREADS) reinterpret_cast<uint4 *>(bins)[i] = make_uint4(0, 0, 0, 0);
        if (tid == 0) words[2] = 0;
        sync_threads();
#pragma unroll 1
        for (int r0 = 0; r0 < n; r0 += ROUND) {
            if (n > ROUND) load(r0);
#pragma unroll
            for (int m = 0; m < MINE; ++m)
                if (k[m] >= lo && k[m] <= hi) atomicAdd(&bins[(k[m] - lo) >> shift], 1u);
        }
        sync_threads();
        // bins from the top: the one where the count passes `need`
        const int from = BINS - (tid + 1) * (BINS / THREADS);          // thread 0 has the highest bins
        static_assert(BINS / THREADS == 8, "two loads a thread");
        const uint4 u = *reinterpret_cast<const uint4 *>(bins + from), v = *reinterpret_cast<const uint4 *>(bins + from + 4);
        const uint32_t sum = u.x + u.y + u.z + u.w + v.x + v.y + v.z + v.w;
        uint32_t above = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(FULL, above, d);
            if (lane >= d) above += o;
        }
        if (lane == 31) words[16 + warp] = above;
        sync_threads();
        uint32_t others = lane < warp ? words[16 + lane] : 0u;
        others = __reduce_add_sync(FULL, others);
        above += others - sum;                 // in the bins above this thread's
        if (above < (uint32_t)need && (uint32_t)need <= above + sum) {
            const uint32_t mine[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
            bool found = false;
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                if (!found && (uint32_t)need <= above + mine[i]) {
                    found = true;
                    words[24] = (uint32_t)(from + i);
                    words[25] = above;
                    words[26] = mine[i];
                }
                above += mine[i];
            }
        }
        sync_threads();
        const uint32_t bin = words[24], higher = words[25], in_bin = words[26];
        lo += bin << shift;
        need -= (int)higher;
        if ((uint32_t)need == in_bin) {        // the bin as a whole
            limit = lo - 1;                    // (a score's number is 0x007FFFFF at least)
            break;
        }
        if (shift == 0) {                      // scores that are equal
            limit = lo;
            ties = need;
            break;
        }
        hi = lo + ((1u << shift) - 1);
        if (in_bin <= 32) {
            // a warp's worth: its need-th largest by comparison.  (Which of equal ones is whose does not matter here: limit and ties do.)
#pragma unroll 1
            for (int r0 = 0; r0 < n; r0 += ROUND) {
                if (n > ROUND) load(r0);
#pragma unroll
                for (int m = 0; m < MINE; ++m)
                    if (k[m] >= lo && k[m] <= hi) words[32 + atomicAdd(&words[2], 1u)] = k[m];
            }
            sync_threads();
            const uint32_t c = lane < (int)in_bin ? words[32 + lane] : 0u;
            int higher_ones = 0, equal_before = 0;
#pragma unroll 1
            for (int i = 0; i < (int)in_bin; ++i) {
                const uint32_t o = __shfl_sync(FULL, c, i);
                higher_ones += o > c;
                equal_before += o == c && i < lane;
            }
            const int who = __ffs(__ballot_sync(FULL, c != 0u && higher_ones + equal_before == need - 1)) - 1;
            limit = __shfl_sync(FULL, c, who);
            ties = need - __shfl_sync(FULL, higher_ones, who);
            break;
        }
        shift = shift > 11 ? shift - 11 : 0;
    }
    // ---- the list, ascending ----
    int taken = 0, same = 0;                   // of the rounds before; those that equal the limit
#pragma unroll 1
    for (int r0 = 0; r0 < n; r0 += ROUND) {
        if (n > ROUND) load(r0);
        uint32_t mine = 0;                     // above the limit | << 16 equal to it (at most 2048 of each in a round)
#pragma unroll
        for (int m = 0; m < MINE; ++m) mine += (k[m] > limit ? 1u : 0u) + (k[m] == limit ? 0x10000u : 0u);
        uint32_t before = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t o = __shfl_up_sync(FULL, before, d);
            if (lane >= d) before += o;
        }
        if (lane == 31) words[64 + warp] = before;
        sync_threads();
        const uint32_t w = lane < WARPS ? words[64 + lane] : 0u;
        const uint32_t all = __reduce_add_sync(FULL, w), others = __reduce_add_sync(FULL, lane < warp ? w : 0u);
        before += others - mine;
        int place = taken + (int)(before & 0xFFFFu), equal = same + (int)(before >> 16);
        if (mine)
#pragma unroll
            for (int m = 0; m < MINE; ++m) {
                if (k[m] > limit || (k[m] == limit && equal < ties)) out[run.first + place + (equal < ties ? equal : ties)] = run.first + r0 + tid * MINE + m;
                place += k[m] > limit;
                equal += k[m] == limit;
            }
        taken += (int)(all & 0xFFFFu);
        same += (int)(all >> 16);
        if (r0 + ROUND < n) sync_threads();
    }
    const int tail = run.first + p.top, total = tail + run.end - run.last;
#pragma unroll 1
    for (int i = tid; i < run.first; i += THREADS) out[i] = i;
#pragma unroll 1
    for (int i = tail + tid; i < p.stride; i += THREADS) out[i] = i < total ? run.last + i - tail : -1;
    if (tid == 0) p.counts[seg] = total;
}

// ---- few columns -----------------------------------------------------------------------------------------------------
// Dynamic shared memory: scores [most] | bins [BINS] | query codes [NT * 8][2 D + 64 B] | words [WORDS]
template <int D>
__host__ __device__ constexpr int code_row() { return 2 * D + 64; }        // (two rows that a load touches at once are not in the same banks)
template <int D>
size_t few_smem_bytes(int most, int nt) { return (size_t)((most + 7) & ~7) * 4 + BINS * 4 + (size_t)nt * 8 * code_row<D>() + WORDS * 4; }

template <int D, int NT>
__global__ void __launch_bounds__(THREADS, 3) select_few_kernel(const __grid_constant__ SelectParams p, int G, bool by_length)
{
    extern __shared__ __align__(16) uint8_t smem_raw[];
    constexpr int J = 2 * D / 64;              // pieces of 64 bytes of an entry
    constexpr int ROW = code_row<D>();
    constexpr int PIECES = NT * 8 * (D / 8), MINE = (PIECES + THREADS - 1) / THREADS;      // of 8 dims of a column; of a thread
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, tig = lane & 3;
    uint32_t rank, ranks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    uint32_t *keys = reinterpret_cast<uint32_t *>(smem_raw), *bins = keys + ((p.most + 7) & ~7);
    uint8_t *q_codes = reinterpret_cast<uint8_t *>(bins + BINS);
    uint32_t *words = reinterpret_cast<uint32_t *>(q_codes + NT * 8 * ROW);
    if (tid == 0) {
        words[0] = 0xFFFFFFFFu;
        words[1] = 0;
    }
    pdl_wait();
    pdl_trigger();
    if (ranks > 1) cluster_arrive();           // (the first CTA has to be there before anyone writes to it)
    const int place = (int)(blockIdx.x / ranks) / p.Hkv, h = (int)(blockIdx.x / ranks) - place * p.Hkv;
    int list = place;
    if (by_length) {                           // the place-th longest of all sequences
        int *lens = reinterpret_cast<int *>(bins);
        const int n = tid < p.B ? __ldg(p.seq_lens + tid) : -0x7FFFFFFF - 1;
        lens[tid] = n;
        __syncthreads();
        int before = 0;
#pragma unroll 4
        for (int i = 0; i < p.B; i += 4) {
            const int4 o = *reinterpret_cast<const int4 *>(lens + i);
            before += (o.x > n || (o.x == n && i < tid)) + (o.y > n || (o.y == n && i + 1 < tid)) + (o.z > n || (o.z == n && i + 2 < tid)) +
                      (o.w > n || (o.w == n && i + 3 < tid));
        }
        if (tid < p.B && before == place) words[12] = (uint32_t)tid;
        __syncthreads();
        list = (int)words[12];
    }
    const int seg = list * p.Hkv + h;
    const Run run = run_of(p, list, h == 0 && rank == 0 && tid == 0);
    if (run.scored <= p.top) {                 // (the same for the whole cluster)
        if (rank == 0) list_all(p, seg, run, tid);
        if (ranks > 1) cluster_wait();
        return;
    }
    if (p.top > 0) {
        // ---- this warp's first entries are asked for before the queries ----
        const int tiles = (run.scored + 15) / 16;
        const int t_from = (int)((int64_t)tiles * rank / ranks), t_to = (int)((int64_t)tiles * (rank + 1) / ranks);
        const int32_t *table = p.page_table + (int64_t)run.b * p.pt_stride + run.first;
        auto id_of = [&](int i) {              // physical page of scored page i; past the end: the last one's
            const int id = __ldg(table + (i < run.scored ? i : run.scored - 1));
            if (id >= 0 && (int64_t)id < p.max_pages) return id;
            atomicOr(p.status, STATUS_BOUNDS);
            return 0;
        };
        uint4 a0[J], a1[J];
        float scale = 0.f;
        int id0 = 0, id1 = 0;
        auto fetch = [&]() {
            const int64_t e0 = (int64_t)id0 * p.Hkv + h, e1 = (int64_t)id1 * p.Hkv + h;
            const uint4 *s0 = reinterpret_cast<const uint4 *>(p.codes + e0 * 2 * D) + tig, *s1 = reinterpret_cast<const uint4 *>(p.codes + e1 * 2 * D) + tig;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                a0[j] = __ldg(s0 + 4 * j);
                a1[j] = __ldg(s1 + 4 * j);
            }
            scale = __ldg(p.scales + (tig & 1 ? e1 : e0));
        };
        auto ids_of = [&](int t) {
            if (t >= t_to) return;
            id0 = id_of(t * 16 + g);
            id1 = id_of(t * 16 + g + 8);
        };
        int t = t_from + warp;
        ids_of(t);
        // ---- the queries' codes, [max(c, 0) | min(c, 0)] of every row and head; columns that are left over repeat the first ----
        const int cols = run.rows * G;
        const uint16_t *q = p.Q + ((int64_t)run.row * p.Hq + (int64_t)h * G) * D;
        uint4 w[MINE];
        uint32_t top = 0;
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
            const int i = tid + m * THREADS, col = i / (D / 8) < cols ? i / (D / 8) : 0, row = col / G;
            w[m] = make_uint4(0, 0, 0, 0);
            if (i < PIECES) w[m] = __ldg(reinterpret_cast<const uint4 *>(q + ((int64_t)row * p.Hq + (col - row * G)) * D + i % (D / 8) * 8));
        }
        if (t < t_to) fetch();
        ids_of(t + WARPS);
#pragma unroll
        for (int m = 0; m < MINE; ++m) top = max(top, largest(w[m]));
        top = __reduce_max_sync(FULL, top);
        if (lane == 0) words[4 + warp] = top;
        __syncthreads();
        const float inv = steps_per_unit(words + 4, lane);
#pragma unroll
        for (int m = 0; m < MINE; ++m) {
            const int i = tid + m * THREADS, col = i / (D / 8), piece = i % (D / 8);
            uint2 up, down;
            steps_of(w[m], inv, up, down);
            if (i < PIECES) {
                *reinterpret_cast<uint2 *>(q_codes + col * ROW + piece * 8) = up;
                *reinterpret_cast<uint2 *>(q_codes + col * ROW + D + piece * 8) = down;
            }
        }
        __syncthreads();
        if (ranks > 1) cluster_wait();
        // ---- scores ----
        uint32_t to;                           // the first CTA's scores
        asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"(smem_u32(keys)));
        const uint8_t *mine = q_codes + g * ROW + tig * 16;
        uint32_t least = 0xFFFFFFFFu, most = 0;
        for (; t < t_to; t += WARPS) {
            int best0 = -0x7FFFFFFF, best1 = -0x7FFFFFFF;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                int d[4] = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const uint4 b = *reinterpret_cast<const uint4 *>(mine + nt * 8 * ROW + j * 64);
                    mma_s8_16832(d, a0[j].x, a1[j].x, a0[j].y, a1[j].y, b.x, b.y);
                    mma_s8_16832(d, a0[j].z, a1[j].z, a0[j].w, a1[j].w, b.z, b.w);
                }
                best0 = max(best0, max(d[0], d[1]));
                best1 = max(best1, max(d[2], d[3]));
            }
            const float my_scale = scale;
            if (t + WARPS < t_to) {            // the next entries, as soon as the registers are free
                fetch();
                ids_of(t + 2 * WARPS);
            }
#pragma unroll
            for (int x = 1; x < 4; x <<= 1) {
                best0 = max(best0, __shfl_xor_sync(FULL, best0, x));
                best1 = max(best1, __shfl_xor_sync(FULL, best1, x));
            }
            const int i = t * 16 + g + 8 * tig;
            if (tig < 2 && i < run.scored) {
                const uint32_t key = key_of(tig ? best1 : best0, my_scale);
                least = min(least, key);
                most = max(most, key);
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + 4u * (uint32_t)i), "r"(key) : "memory");
            }
        }
        uint32_t range;
        asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(range) : "r"(smem_u32(words)));
        note_range(range, least, most, lane);
    } else if (ranks > 1) {
        cluster_wait();
    }
    if (ranks > 1) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (rank != 0) return;
    } else {
        __syncthreads();
    }
    choose(p, seg, run, keys, bins, words, tid);
}

// ---- many columns ----------------------------------------------------------------------------------------------------
constexpr int TILE = 128;              // pages of a tile
constexpr int MANY_THREADS = THREADS + 32;
constexpr int A_STAGES = 4;            // of the ring of pages' codes; a stage is 128 bytes of each page of a tile

__device__ __forceinline__ void umma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Shared memory from a 1024-byte boundary on: pages' codes [A_STAGES][128 pages][128 B] in the 128-byte swizzle (the bins, once all scores
// are there) | columns' codes [2 D / 128][N][128 B], the same | scores [most] | words [WORDS] | barriers
constexpr int STAGE = TILE * 128;
template <int D>
size_t many_smem_bytes(int most, int N) { return 1024 + A_STAGES * (size_t)STAGE + (size_t)N * 2 * D + (size_t)((most + 7) & ~7) * 4 + WORDS * 4 + 128; }

// Nine warps.  0-3: thread = page of a tile (TMEM lane), the largest of its columns;  4-7: fetch the pages' codes;  8: issues.
template <int D>
__global__ void __launch_bounds__(MANY_THREADS, 2) select_many_kernel(const __grid_constant__ SelectParams p, int G, int N, int tmem_cols)
{
    extern __shared__ __align__(1024) uint8_t smem_many[];
    constexpr int ROW = 2 * D, ATOMS = ROW / 128;
    constexpr int PIECES = D / 8;              // of 8 dims, of a column
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);
    const uint32_t base = smem_u32(smem_many);
    const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
    const uint32_t a_smem = base + pad, b_smem = a_smem + A_STAGES * STAGE;
    uint8_t *behind = smem_many + pad + A_STAGES * STAGE + (size_t)N * ROW;
    uint32_t *bins = reinterpret_cast<uint32_t *>(smem_many + pad), *keys = reinterpret_cast<uint32_t *>(behind), *words = keys + ((p.most + 7) & ~7);
    const uint32_t bars = smem_u32(words + WORDS), full = bars, empty = full + 8 * A_STAGES, sums = empty + 8 * A_STAGES, taken = sums + 16;
    static_assert(BINS * 4 <= A_STAGES * STAGE, "the bins fit");
    volatile uint32_t *gave_up = words + 80, *tmem_slot = words + 81;
    volatile int *shared = reinterpret_cast<volatile int *>(words + 82);
    if (tid == 0) {
        for (int i = 0; i < A_STAGES; ++i) {
            mbar_init(full + 8 * i, 128);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(sums + 8 * i, 1);
            mbar_init(taken + 8 * i, 4);
        }
        *gave_up = 0;
        words[0] = 0xFFFFFFFFu;
        words[1] = 0;
        words[9] = words[10] = words[11] = 0;
        fence_barrier_init();
    }
    pdl_wait();
    // (runs of a sequence and head are neighbours in the grid: they read the same entries)
    const int pair = (int)blockIdx.x / p.per_seq, list = pair / p.Hkv * p.per_seq + (int)blockIdx.x - pair * p.per_seq, h = pair % p.Hkv, seg = list * p.Hkv + h;
    if (warp == 8) {                           // (one warp works the run out, as in skv_prefill_pages.cu)
        const Run r = run_of(p, list, h == 0 && lane == 0);
        if (lane == 0) {
            shared[0] = r.b;
            shared[1] = r.row;
            shared[2] = r.rows;
            shared[3] = r.first;
            shared[4] = r.scored;
            shared[5] = r.last;
            shared[6] = r.end;
        }
        if (r.scored > p.top && p.top > 0) {
            tc5::tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), (uint32_t)tmem_cols);
            tc5::tmem_relinquish();
        }
    }
    tc5::tc_fence_before();
    __syncthreads();
    tc5::tc_fence_after();
    Run run;
    auto get = [&](int i) { return __shfl_sync(FULL, shared[i], 0); };
    run.b = get(0);
    run.row = get(1);
    run.rows = get(2);
    run.first = get(3);
    run.scored = get(4);
    run.last = get(5);
    run.end = get(6);
    if (run.scored <= p.top) {
        if (tid < THREADS) list_all(p, seg, run, tid);
        return;
    }
    if (p.top > 0) {
        const uint32_t tmem = __shfl_sync(FULL, *tmem_slot, 0);
        const int tiles = (run.scored + TILE - 1) / TILE;
        const int32_t *table = p.page_table + (int64_t)run.b * p.pt_stride + run.first;
        auto id_of = [&](int i) {              // physical page of scored page i; past the end: the last one's
            const int id = __ldg(table + (i < run.scored ? i : run.scored - 1));
            if (id >= 0 && (int64_t)id < p.max_pages) return id;
            atomicOr(p.status, STATUS_BOUNDS);
            return 0;
        };
        if (warp >= 4 && warp < 8) {
            // ---- pages' codes: 8 lanes a row of 128 bytes; a thread has rows  t / 8 + 16 i  of every tile, their ids a tile ahead ----
            const int t = tid - 128, c = t & 7, r0 = t >> 3;
            int ids[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) ids[i] = id_of(r0 + 16 * i);
            const int8_t *codes = p.codes + (int64_t)h * ROW + c * 16;
            const int64_t page_bytes = (int64_t)p.Hkv * ROW;
            const uint32_t to = a_smem + (uint32_t)(r0 * 128 + ((c ^ (r0 & 7)) * 16));       // (rows 16 apart have the same place in the swizzle)
            int use = 0;                       // stages filled so far
            for (int tile = 0; tile < tiles; ++tile) {
                const int8_t *src[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) src[i] = codes + ids[i] * page_bytes;
                if (tile + 1 < tiles)
#pragma unroll
                    for (int i = 0; i < 8; ++i) ids[i] = id_of((tile + 1) * TILE + r0 + 16 * i);
#pragma unroll
                for (int a = 0; a < ATOMS; ++a, ++use) {
                    const int st = use & (A_STAGES - 1);
                    if (use >= A_STAGES) chunk::wait(empty + 8 * st, (uint32_t)((use / A_STAGES - 1) & 1), gave_up);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + (uint32_t)(st * STAGE + i * 16 * 128)), "l"(src[i] + a * 128) : "memory");
                    // the barrier hears of it when they are there; whoever issues the products sees to the proxies
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full + 8 * st) : "memory");
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
        // ---- the queries' codes, by warps 0 to 3 and 8; columns that are left over repeat the first ----
        if (warp < 4 || warp == 8) {
            const int me = warp < 4 ? tid : 128 + lane, cols = run.rows * G;
            const uint16_t *q = p.Q + ((int64_t)run.row * p.Hq + (int64_t)h * G) * D;
            // 160 threads: a thread has the same piece of every 160 / PIECES-th column
            constexpr int STEP = 160 / PIECES, AT_ONCE = (128 + STEP - 1) / STEP <= 7 ? (128 + STEP - 1) / STEP : 7;
            const int piece = me % PIECES, c0 = me / PIECES;
            const uint32_t by_G = 65535u / (uint32_t)G + 1u;         // col / G = col by_G >> 16 for the columns there are
            auto piece_of = [&](int col) {
                const int x = col < cols ? col : 0, row = (int)((uint32_t)x * by_G >> 16);
                return __ldg(reinterpret_cast<const uint4 *>(q + ((int64_t)row * p.Hq + (x - row * G)) * D + piece * 8));
            };
            auto chunk_at = [&](int byte) { return (uint32_t)(byte / 128 * N * 128 + byte % 128 / 16 * 16); };
            const uint32_t up_at = chunk_at(piece * 8), down_at = chunk_at(D + piece * 8), half = (uint32_t)(piece & 1) * 8;
            auto up_of = [&](int col) { return b_smem + (uint32_t)(col * 128) + half + (up_at ^ (uint32_t)(col & 7) * 16); };
            auto down_of = [&](int col) { return b_smem + (uint32_t)(col * 128) + half + (down_at ^ (uint32_t)(col & 7) * 16); };
            // first as they are, in the 16 bytes that the piece's steps will have (asking for them a second time took 700 cycles each)
            uint32_t top = 0;
#pragma unroll 1
            for (int col = c0; col < N; col += AT_ONCE * STEP) {
                uint4 w[AT_ONCE];
#pragma unroll
                for (int m = 0; m < AT_ONCE; ++m) w[m] = piece_of(col + STEP * m);     // (past the last column: the first again)
#pragma unroll
                for (int m = 0; m < AT_ONCE; ++m) {
                    top = max(top, largest(w[m]));
                    if (col + STEP * m < N) {
                        asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(up_of(col + STEP * m)), "r"(w[m].x), "r"(w[m].y) : "memory");
                        asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(down_of(col + STEP * m)), "r"(w[m].z), "r"(w[m].w) : "memory");
                    }
                }
            }
            top = __reduce_max_sync(FULL, top);
            if (lane == 0) words[warp < 4 ? 4 + warp : 8] = top;
            asm volatile("bar.sync 2, 160;" ::: "memory");
            const float inv = steps_per_unit(words + 4, lane);
#pragma unroll 2
            for (int col = c0; col < N; col += STEP) {
                uint4 w;
                asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w.x), "=r"(w.y) : "r"(up_of(col)) : "memory");
                asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w.z), "=r"(w.w) : "r"(down_of(col)) : "memory");
                uint2 up, down;
                steps_of(w, inv, up, down);
                asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(up_of(col)), "r"(up.x), "r"(up.y) : "memory");
                asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(down_of(col)), "r"(down.x), "r"(down.y) : "memory");
            }
            fence_proxy_async();
            asm volatile("bar.sync 2, 160;" ::: "memory");
        }
        if (warp == 8) {
            // ---- products: one lane issues ----
            const bool leader = chunk::elect_one();
            const uint32_t idesc = (2u << 4) /* s32 */ | (1u << 7) | (1u << 10) /* s8 by s8 */ | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
            const uint64_t a_desc = swizzled_desc(a_smem), b_desc = swizzled_desc(b_smem);
            const uint64_t b_atom = (uint64_t)((N * 128) >> 4);
            int use = 0;
            for (int tile = 0; tile < tiles; ++tile) {
                const int buf = tile & 1;
                if (tile >= 2) chunk::wait(taken + 8 * buf, (uint32_t)((tile / 2 - 1) & 1), gave_up);
#pragma unroll
                for (int a = 0; a < ATOMS; ++a, ++use) {
                    const int st = use & (A_STAGES - 1);
                    chunk::wait(full + 8 * st, (uint32_t)((use / A_STAGES) & 1), gave_up);
                    fence_proxy_async();       // (the codes came through the generic proxy)
                    tc5::tc_fence_after();
                    if (leader) {
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            umma_i8(tmem + (uint32_t)(buf * N), a_desc + (uint64_t)((st * STAGE + ks * 32) >> 4), b_desc + (uint64_t)a * b_atom + (uint64_t)((ks * 32) >> 4),
                                    idesc, a > 0 || ks > 0);
                        tc5::tc_commit(empty + 8 * st);
                        if (a == ATOMS - 1) tc5::tc_commit(sums + 8 * buf);
                    }
                    __syncwarp();
                }
            }
            for (int j = use > A_STAGES ? use - A_STAGES : 0; j < use; ++j)            // the last commits arrive while the barriers are still there
                chunk::wait(empty + 8 * (j & (A_STAGES - 1)), (uint32_t)((j / A_STAGES) & 1), gave_up);
        } else if (warp < 4) {
            // ---- scores ----
            const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16);
            // (a page's scale is asked for a tile ahead, its id two)
            auto raw_id = [&](int i) { return __ldg(table + (i < run.scored ? i : run.scored - 1)); };
            auto scale_of = [&](int id) { return __ldg(p.scales + (int64_t)(id >= 0 && (int64_t)id < p.max_pages ? id : 0) * p.Hkv + h); };
            int id = raw_id(tid + TILE);
            float scale = scale_of(raw_id(tid));
            uint32_t least = 0xFFFFFFFFu, most = 0;
#pragma unroll 1
            for (int tile = 0; tile < tiles; ++tile) {
                const int buf = tile & 1, i = tile * TILE + tid;
                const float next = scale_of(id);
                id = raw_id(i + 2 * TILE);
                chunk::wait(sums + 8 * buf, (uint32_t)((tile >> 1) & 1), gave_up);
                tc5::tc_fence_after();
                int best[2] = {-0x7FFFFFFF, -0x7FFFFFFF};
                int n = 0;
#pragma unroll 1
                for (; n + 64 <= N; n += 64) {
                    uint32_t u[32], v[32];
                    tc5::tmem_ld32(mine + (uint32_t)(buf * N + n), u);
                    tc5::tmem_ld32(mine + (uint32_t)(buf * N + n + 32), v);
                    tc5::tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 32; ++x) best[x & 1] = max(best[x & 1], max((int)u[x], (int)v[x]));
                }
#pragma unroll 1
                for (; n < N; n += 16) {
                    uint32_t v[16];
                    tc5::tmem_ld16(mine + (uint32_t)(buf * N + n), v);
                    tc5::tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 16; ++x) best[x & 1] = max(best[x & 1], (int)v[x]);
                }
                tc5::tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(taken + 8 * buf);
                if (i < run.scored) {
                    const uint32_t key = key_of(max(best[0], best[1]), scale);
                    least = min(least, key);
                    most = max(most, key);
                    keys[i] = key;
                }
                scale = next;
            }
            note_range(smem_u32(words), least, most, lane);
        }
        tc5::tc_fence_before();
        __syncthreads();
        if (warp == 8) tc5::tmem_dealloc(tmem, (uint32_t)tmem_cols);
        if (tid == 0 && *gave_up) atomicOr(p.status, STATUS_TIMEOUT);
    }
    if (tid < THREADS) choose(p, seg, run, keys, bins, words, tid);
}

template <class Kernel, class... Args>
cudaError_t launch(Kernel kern, int64_t ctas, int threads, size_t smem, int ranks, bool pdl, cudaStream_t s, Args... args)
{
    if (ctas > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    const cudaError_t e = ensure_dynamic_smem(kern, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (ranks > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)ranks;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (pdl) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

template <int D>
cudaError_t launch_d(const SelectParams &p, int G, int sm_count, bool pdl, cudaStream_t s)
{
    const int cols = (p.run < p.max_q_len ? p.run : p.max_q_len) * G;
    const int64_t segments = (int64_t)p.B * p.per_seq * p.Hkv;
    if (cols <= FEW) {
        // a cluster where the segments leave SMs idle, a rank with a tile for each of its warps
        int ranks = 1;
        while (2 * ranks <= 8 && segments * 2 * ranks <= 2 * (int64_t)sm_count && p.most >= 2 * ranks * WARPS * 16) ranks *= 2;
        // Where there is more than a CTA for every SM, the longest sequences go first: the CTAs' loads differ as the lengths do, and the last
        // to begin are then the shortest.  (64 sequences of 8192 to 32768 tokens: 36.3 us, 40.6 without.)
        const bool by_length = !p.cu_q && p.B <= THREADS && ranks == 1 && segments > sm_count;
        const int nt = (cols + 7) / 8;
        return nt == 1 ? launch(select_few_kernel<D, 1>, segments * ranks, THREADS, few_smem_bytes<D>(p.most, 1), ranks, pdl, s, p, G, by_length)
                       : launch(select_few_kernel<D, 2>, segments * ranks, THREADS, few_smem_bytes<D>(p.most, 2), ranks, pdl, s, p, G, by_length);
    }
    const int N = (cols + 15) / 16 * 16;
    int tmem_cols = 32;
    while (tmem_cols < 2 * N) tmem_cols *= 2;
    return launch(select_many_kernel<D>, segments, MANY_THREADS, many_smem_bytes<D>(p.most, N), 1, pdl, s, p, G, N, tmem_cols);
}

}  // namespace

int select_max_pages(int columns) { return columns <= FEW ? MAX_PAGES : MAX_PAGES_MANY; }

cudaError_t launch_select_pages(const SelectParams &p, int D, int sm_count, bool pdl, cudaStream_t s)
{
    const int G = p.Hq / p.Hkv;
    return D == 128 ? launch_d<128>(p, G, sm_count, pdl, s) : D == 64 ? launch_d<64>(p, G, sm_count, pdl, s) : cudaErrorInvalidValue;
}

}  // namespace skv
