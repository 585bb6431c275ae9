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
// Bound by HBM with many segments of few columns (2 D + 4 bytes a page and head), by the tensor cores and their operands with many
// columns, by latency with few segments.
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
constexpr int HELD = 8;                // scores of a segment that a thread keeps in registers: THREADS * HELD pages of it
constexpr int FEW = 16;                // columns up to which mma.sync does
constexpr int MAX_PAGES = 45056, MAX_PAGES_MANY = 28672;      // of a sequence: the scores of a segment are in one CTA's shared memory
constexpr int WORDS = 256;             // of shared memory that choose() has for itself

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
        const int64_t at = (int64_t)i * p.run;
        if (at >= len) return r;
        r.row = first + (int)at;
        r.rows = len - (int)at < p.run ? len - (int)at : p.run;
        pos = n - len + (int)at;
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

// 8 dims of a row in steps: [max(c, 0)] and [min(c, 0)], a byte each; an element that is not finite counts as 0
__device__ __forceinline__ uint32_t magnitude(uint32_t bits) { return bits >= 0x7F80u ? 0u : bits; }
__device__ __forceinline__ uint32_t largest(const uint4 &w)
{
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = max(top, max(magnitude(x[k] & 0x7FFFu), magnitude(x[k] >> 16 & 0x7FFFu)));
    return top;
}
__device__ __forceinline__ void steps_of(const uint4 &w, float inv, uint2 &up, uint2 &down)
{
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
    uint32_t u[2] = {0, 0}, d[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t bits = (k & 1) ? x[k / 2] >> 16 : x[k / 2] & 0xFFFFu;
        const int c = magnitude(bits & 0x7FFFu) ? __float2int_rn(__uint_as_float(bits << 16) * inv) : 0;
        u[k / 4] |= ((uint32_t)max(c, 0) & 0xFFu) << (8 * (k & 3));
        d[k / 4] |= ((uint32_t)min(c, 0) & 0xFFu) << (8 * (k & 3));
    }
    up = make_uint2(u[0], u[1]);
    down = make_uint2(d[0], d[1]);
}
// 127 / a for the largest element's bits in words[0 .. WARPS) (one of each warp's threads), which all THREADS have written
__device__ __forceinline__ float steps_per_unit(const uint32_t *words, int lane)
{
    const float amax = __uint_as_float(__reduce_max_sync(FULL, words[lane & (WARPS - 1)]) << 16);
    return amax < INDEX_TINY ? 0.f : __fdiv_rn(127.f, amax);
}

// By THREADS threads: the list of a run whose scores' numbers are keys[0 .. run.scored), more than p.top of them.
// bins [BINS] and words [WORDS] are its own.
__device__ void choose(const SelectParams &p, int seg, const Run &run, const uint32_t *keys, uint32_t *bins, uint32_t *words, int tid)
{
    const int lane = tid & 31, warp = tid >> 5, n = p.top > 0 ? run.scored : 0;
    int32_t *out = p.lists + (int64_t)seg * p.stride;
    // (a page that is not there: 0, below every score's number, which is 0x007FFFFF at least)
    uint32_t held[HELD];
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
        held[j] = j * THREADS + tid < n ? keys[j * THREADS + tid] : 0u;
        lo = min(lo, held[j] - 1);             // (0 wraps to the top)
        hi = max(hi, held[j]);
    }
    for (int i = HELD * THREADS + tid; i < n; i += THREADS) {
        lo = min(lo, keys[i] - 1);
        hi = max(hi, keys[i]);
    }
    lo = __reduce_min_sync(FULL, lo);
    hi = __reduce_max_sync(FULL, hi);
    if (lane == 0) {
        words[warp] = lo;
        words[WARPS + warp] = hi;
    }
    for (int i = tid; i < BINS / 4; i += THREADS) reinterpret_cast<uint4 *>(bins)[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) words[48] = 0;
    sync_threads();
    lo = __reduce_min_sync(FULL, words[lane & (WARPS - 1)]) + 1;
    hi = __reduce_max_sync(FULL, words[WARPS + (lane & (WARPS - 1))]);
    // everything above `limit` is taken, and the first `ties` that equal it
    uint32_t limit = 0xFFFFFFFFu;              // (no score's number: that of NaN)
    int need = p.top, ties = 0;
    int shift = 32 - __clz((int)(hi - lo));    // 2^shift > hi - lo
    shift = shift > 11 ? shift - 11 : 0;
    while (need > 0) {
#pragma unroll
        for (int j = 0; j < HELD; ++j)
            if (held[j] >= lo && held[j] <= hi) atomicAdd(&bins[(held[j] - lo) >> shift], 1u);
        for (int i = HELD * THREADS + tid; i < n; i += THREADS) {
            const uint32_t k = keys[i];
            if (k >= lo && k <= hi) atomicAdd(&bins[(k - lo) >> shift], 1u);
        }
        sync_threads();
        // bins from the top: the one where the count passes `need`
        uint32_t mine[BINS / THREADS], sum = 0;
        const int from = BINS - (tid + 1) * (BINS / THREADS);          // thread 0 has the highest bins
#pragma unroll
        for (int i = 0; i < BINS / THREADS; i += 4) {
            const uint4 w = *reinterpret_cast<const uint4 *>(bins + from + i);
            mine[i] = w.x;
            mine[i + 1] = w.y;
            mine[i + 2] = w.z;
            mine[i + 3] = w.w;
            sum += w.x + w.y + w.z + w.w;
        }
        uint32_t above = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t u = __shfl_up_sync(FULL, above, d);
            if (lane >= d) above += u;
        }
        if (lane == 31) words[16 + warp] = above;
        sync_threads();
        for (int w = 0; w < warp; ++w) above += words[16 + w];
        above -= sum;                          // in the bins above this thread's
        if (above < (uint32_t)need && (uint32_t)need <= above + sum) {
            bool found = false;
#pragma unroll
            for (int i = BINS / THREADS - 1; i >= 0; --i) {
                if (!found && (uint32_t)need <= above + mine[i]) {
                    found = true;
                    words[24] = (uint32_t)(from + i);
                    words[25] = above;
                    words[26] = mine[i];
                }
                if (!found) above += mine[i];
            }
        }
        sync_threads();
        const uint32_t bin = words[24], higher = words[25], in_bin = words[26];
        lo += bin << shift;
        need -= (int)higher;
        if ((uint32_t)need == in_bin) {        // the bin as a whole
            limit = lo - 1;
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
            auto note = [&](uint32_t k) {
                if (k >= lo && k <= hi) words[64 + atomicAdd(&words[48], 1u)] = k;
            };
#pragma unroll
            for (int j = 0; j < HELD; ++j) note(held[j]);
            for (int i = HELD * THREADS + tid; i < n; i += THREADS) note(keys[i]);
            sync_threads();
            const uint32_t k = lane < (int)in_bin ? words[64 + lane] : 0u;
            int higher_ones = 0, equal_before = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t o = __shfl_sync(FULL, k, i);
                higher_ones += o > k;
                equal_before += o == k && i < lane;
            }
            const unsigned at = __ballot_sync(FULL, k != 0u && higher_ones + equal_before == need - 1);
            const int who = __ffs(at) - 1;
            limit = __shfl_sync(FULL, k, who);
            ties = need - __shfl_sync(FULL, higher_ones, who);
            break;
        }
        sync_threads();
        for (int i = tid; i < BINS / 4; i += THREADS) reinterpret_cast<uint4 *>(bins)[i] = make_uint4(0, 0, 0, 0);
        sync_threads();
        shift = shift > 11 ? shift - 11 : 0;
    }
    // ---- the list, ascending: 32 pages a warp at a time, their places from the counts of those before them ----
    const unsigned lower = (1u << lane) - 1;
    int taken = 0, same = 0;                   // of the pages before the round; those that equal the limit
    for (int i0 = 0; i0 < n; i0 += HELD * THREADS) {
        unsigned gt[HELD], eq[HELD];
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            if (i0 > 0) {
                const int i = i0 + j * THREADS + tid;
                held[j] = i < n ? keys[i] : 0u;
            }
            gt[j] = __ballot_sync(FULL, held[j] > limit);
            eq[j] = __ballot_sync(FULL, held[j] == limit);
            if (lane == 0) words[128 + j * WARPS + warp] = (uint32_t)(__popc(gt[j]) | __popc(eq[j]) << 16);
        }
        sync_threads();
        // two counts a lane, in order
        const uint32_t c0 = words[128 + 2 * lane], c1 = words[128 + 2 * lane + 1];
        uint32_t sum = c0 + c1;                // (both halves at once: at most 2048 in each)
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t u = __shfl_up_sync(FULL, sum, d);
            if (lane >= d) sum += u;
        }
        const uint32_t all = __shfl_sync(FULL, sum, 31), before0 = sum - c0 - c1, before1 = sum - c1;
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            const int x = j * WARPS + warp;
            const uint32_t b0 = __shfl_sync(FULL, before0, x / 2), b1 = __shfl_sync(FULL, before1, x / 2), before = x & 1 ? b1 : b0;
            const int eq_before = same + (int)(before >> 16) + __popc(eq[j] & lower);
            if (held[j] > limit || (held[j] == limit && eq_before < ties))
                out[run.first + taken + (int)(before & 0xFFFFu) + __popc(gt[j] & lower) + (eq_before < ties ? eq_before : ties)] = run.first + i0 + j * THREADS + tid;
        }
        taken += (int)(all & 0xFFFFu);
        same += (int)(all >> 16);
        if (i0 + HELD * THREADS < n) sync_threads();
    }
    const int tail = run.first + p.top, total = tail + run.end - run.last;
    for (int i = tid; i < run.first; i += THREADS) out[i] = i;
    for (int i = tail + tid; i < p.stride; i += THREADS) out[i] = i < total ? run.last + i - tail : -1;
    if (tid == 0) p.counts[seg] = total;
}

// ---- few columns -----------------------------------------------------------------------------------------------------
// Dynamic shared memory: scores [most] | bins [BINS] | query codes [NT * 8][2 D + 64 B] | words [WORDS]
template <int D>
__host__ __device__ constexpr int code_row() { return 2 * D + 64; }        // (two rows that a load touches at once are not in the same banks)
template <int D>
size_t few_smem_bytes(int most, int nt) { return (size_t)((most + 3) & ~3) * 4 + BINS * 4 + (size_t)nt * 8 * code_row<D>() + WORDS * 4; }

template <int D, int NT>
__global__ void __launch_bounds__(THREADS, 3) select_few_kernel(SelectParams p, int G)
{
    extern __shared__ __align__(16) uint8_t smem_raw[];
    constexpr int J = 2 * D / 64;              // pieces of 64 bytes of an entry
    constexpr int ROW = code_row<D>();
    constexpr int PIECES = NT * 8 * (D / 8), MINE = (PIECES + THREADS - 1) / THREADS;      // of 8 dims of a column; of a thread
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, tig = lane & 3;
    uint32_t rank, ranks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    uint32_t *keys = reinterpret_cast<uint32_t *>(smem_raw), *bins = keys + ((p.most + 3) & ~3);
    uint8_t *q_codes = reinterpret_cast<uint8_t *>(bins + BINS);
    uint32_t *words = reinterpret_cast<uint32_t *>(q_codes + NT * 8 * ROW);
    pdl_wait();
    pdl_trigger();
    if (ranks > 1) cluster_arrive();           // (the first CTA has to be there before anyone writes to it)
    const int seg = (int)(blockIdx.x / ranks), list = seg / p.Hkv, h = seg - list * p.Hkv;
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
        if (lane == 0) words[warp] = top;
        __syncthreads();
        const float inv = steps_per_unit(words, lane);
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
            if (tig < 2 && i < run.scored)
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + 4u * (uint32_t)i), "r"(key_of(tig ? best1 : best0, my_scale)) : "memory");
        }
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
constexpr int A_STAGES = 2;

__device__ __forceinline__ void umma_i8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Shared memory from a 1024-byte boundary on: pages' codes [A_STAGES][2 D / 128][128 pages][128 B] in the 128-byte swizzle (the bins, once
// all scores are there) | columns' codes [2 D / 128][N][128 B], the same | scores [most] | words [WORDS] | barriers
template <int D>
__host__ __device__ constexpr int a_stage_bytes() { return TILE * 2 * D; }
template <int D>
size_t many_smem_bytes(int most, int N) { return 1024 + A_STAGES * (size_t)a_stage_bytes<D>() + (size_t)N * 2 * D + (size_t)((most + 3) & ~3) * 4 + WORDS * 4 + 64; }

// Nine warps.  0-3: thread = page of a tile (TMEM lane), the largest of its columns;  4-7: fetch the pages' codes;  8: issues.
template <int D>
__global__ void __launch_bounds__(MANY_THREADS, 2) select_many_kernel(const __grid_constant__ SelectParams p, int G, int N, int tmem_cols)
{
    extern __shared__ __align__(1024) uint8_t smem_many[];
    constexpr int ROW = 2 * D, ATOMS = ROW / 128, STAGE = a_stage_bytes<D>();
    constexpr int PIECES = D / 8;              // of 8 dims, of a column
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);
    const uint32_t base = smem_u32(smem_many);
    const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
    const uint32_t a_smem = base + pad, b_smem = a_smem + A_STAGES * STAGE;
    uint8_t *behind = smem_many + pad + A_STAGES * STAGE + (size_t)N * ROW;
    uint32_t *bins = reinterpret_cast<uint32_t *>(smem_many + pad), *keys = reinterpret_cast<uint32_t *>(behind), *words = keys + ((p.most + 3) & ~3);
    const uint32_t bars = smem_u32(words + WORDS), full = bars, empty = full + 8 * A_STAGES, sums = empty + 8 * A_STAGES, taken = sums + 16;
    static_assert(BINS * 4 <= A_STAGES * a_stage_bytes<D>(), "the bins fit");
    volatile uint32_t *gave_up = words + 200, *tmem_slot = words + 201;
    volatile int *shared = reinterpret_cast<volatile int *>(words + 202);
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
            auto landed = [&](int tile) {      // (the tensor core reads through the async proxy)
                fence_proxy_async();
                mbar_arrive(full + 8 * (tile & (A_STAGES - 1)));
            };
            for (int tile = 0; tile < tiles; ++tile) {
                const int st = tile & (A_STAGES - 1);
                if (tile >= A_STAGES) chunk::wait(empty + 8 * st, (uint32_t)((tile / A_STAGES - 1) & 1), gave_up);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int row = r0 + 16 * i;
                    const int8_t *src = p.codes + ((int64_t)ids[i] * p.Hkv + h) * ROW + c * 16;
                    const uint32_t dst = a_smem + (uint32_t)(st * STAGE + row * 128 + ((c ^ (row & 7)) * 16));
#pragma unroll
                    for (int a = 0; a < ATOMS; ++a)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + (uint32_t)(a * TILE * 128)), "l"(src + a * 128) : "memory");
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                if (tile + 1 < tiles)
#pragma unroll
                    for (int i = 0; i < 8; ++i) ids[i] = id_of((tile + 1) * TILE + r0 + 16 * i);
                if (tile > 0) {
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    landed(tile - 1);
                }
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            landed(tiles - 1);
        }
        // ---- the queries' codes, by warps 0 to 3 and 8; columns that are left over repeat the first ----
        if (warp < 4 || warp == 8) {
            const int me = warp < 4 ? tid : 128 + lane, cols = run.rows * G;
            const uint16_t *q = p.Q + ((int64_t)run.row * p.Hq + (int64_t)h * G) * D;
            auto piece_of = [&](int i) {
                const int col = i / PIECES < cols ? i / PIECES : 0, row = col / G;
                return __ldg(reinterpret_cast<const uint4 *>(q + ((int64_t)row * p.Hq + (col - row * G)) * D + i % PIECES * 8));
            };
            uint32_t top = 0;
#pragma unroll 4
            for (int i = me; i < cols * PIECES; i += 160) top = max(top, largest(piece_of(i)));
            top = __reduce_max_sync(FULL, top);
            if (lane == 0) words[warp < 4 ? warp : 4] = top;
            if (tid < 3) words[5 + tid] = 0;
            asm volatile("bar.sync 2, 160;" ::: "memory");
            const float inv = steps_per_unit(words, lane);
#pragma unroll 4
            for (int i = me; i < N * PIECES; i += 160) {
                const int col = i / PIECES, piece = i % PIECES;
                uint2 up, down;
                steps_of(piece_of(i), inv, up, down);
                auto at = [&](int byte) { return b_smem + (uint32_t)(byte / 128 * N * 128 + col * 128 + (((byte % 128 / 16) ^ (col & 7)) * 16) + byte % 16); };
                asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at(piece * 8)), "r"(up.x), "r"(up.y) : "memory");
                asm volatile("st.shared.v2.u32 [%0], {%1,%2};" ::"r"(at(D + piece * 8)), "r"(down.x), "r"(down.y) : "memory");
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
            for (int tile = 0; tile < tiles; ++tile) {
                const int st = tile & (A_STAGES - 1), buf = tile & 1;
                chunk::wait(full + 8 * st, (uint32_t)((tile / A_STAGES) & 1), gave_up);
                if (tile >= 2) chunk::wait(taken + 8 * buf, (uint32_t)((tile / 2 - 1) & 1), gave_up);
                tc5::tc_fence_after();
                if (leader) {
#pragma unroll
                    for (int ks = 0; ks < ROW / 32; ++ks)
                        umma_i8(tmem + (uint32_t)(buf * N), a_desc + (uint64_t)((st * STAGE + (ks >> 2) * TILE * 128 + (ks & 3) * 32) >> 4),
                                b_desc + (uint64_t)(ks >> 2) * b_atom + (uint64_t)(((ks & 3) * 32) >> 4), idesc, ks > 0);
                    tc5::tc_commit(sums + 8 * buf);
                    tc5::tc_commit(empty + 8 * st);
                }
                __syncwarp();
            }
            for (int j = tiles > A_STAGES ? tiles - A_STAGES : 0; j < tiles; ++j)      // the last commits arrive while the barriers are still there
                chunk::wait(empty + 8 * (j & (A_STAGES - 1)), (uint32_t)((j / A_STAGES) & 1), gave_up);
        } else if (warp < 4) {
            // ---- scores ----
            const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16);
            float scale = __ldg(p.scales + (int64_t)id_of(tid) * p.Hkv + h);
            for (int tile = 0; tile < tiles; ++tile) {
                const int buf = tile & 1, i = tile * TILE + tid;
                const float next = tile + 1 < tiles ? __ldg(p.scales + (int64_t)id_of(i + TILE) * p.Hkv + h) : 0.f;
                chunk::wait(sums + 8 * buf, (uint32_t)((tile >> 1) & 1), gave_up);
                tc5::tc_fence_after();
                int best[4] = {-0x7FFFFFFF, -0x7FFFFFFF, -0x7FFFFFFF, -0x7FFFFFFF};
                int n = 0;
                for (; n + 32 <= N; n += 32) {
                    uint32_t v[32];
                    tc5::tmem_ld32(mine + (uint32_t)(buf * N + n), v);
                    tc5::tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 32; ++x) best[x & 3] = max(best[x & 3], (int)v[x]);
                }
                if (n < N) {
                    uint32_t v[16];
                    tc5::tmem_ld16(mine + (uint32_t)(buf * N + n), v);
                    tc5::tmem_wait_ld();
#pragma unroll
                    for (int x = 0; x < 16; ++x) best[x & 3] = max(best[x & 3], (int)v[x]);
                }
                tc5::tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(taken + 8 * buf);
                if (i < run.scored) keys[i] = key_of(max(max(best[0], best[1]), max(best[2], best[3])), scale);
                scale = next;
            }
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
        const int nt = (cols + 7) / 8;
        return nt == 1 ? launch(select_few_kernel<D, 1>, segments * ranks, THREADS, few_smem_bytes<D>(p.most, 1), ranks, pdl, s, p, G)
                       : launch(select_few_kernel<D, 2>, segments * ranks, THREADS, few_smem_bytes<D>(p.most, 2), ranks, pdl, s, p, G);
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
