// Selection of pages by a cheap score (skv_select_pages).  For a run of rows (a decode step's row, or up to 32 of a chunk) and a
// kv head:  the queries in whole steps of a 127th of their largest element, c;  of every full page p before the run's last pages
//     dot(p) = max over rows and query heads of  sum_d  max(c_d, 0) highest_d(p) + min(c_d, 0) lowest_d(p),
// the largest that a key inside the page's bounds could give;  score(p) = dot(p) x the page's step;  and the `top` pages of the
// highest score, of two equal ones the lower.  dot is a sum of whole numbers below 2^24, exact in any order, so the selection does
// not depend on how the work is cut.
//
// The sum over [max(c, 0) | min(c, 0)] and [highest | lowest] is one product of length 2 D on the tensor cores in 8 bits: 16 pages
// against 8 columns (rows x query heads) an instruction.  A warp loads 16 entries straight into the fragments: the order of the
// contracted dims is free as long as both sides agree, so a lane's 16 consecutive bytes serve two instructions.
// A CTA scores a part of a segment's pages -- (run, kv head) --, a cluster of CTAs shares a segment where there are few, and writes
// its scores, as whole numbers that order as they do, into the first CTA's shared memory.  That one then finds the
// top-th largest by counting into 2048 bins between lowest and highest, again inside the bin where it lies until that is
// resolved, and lists the chosen in ascending order.
// Bound by HBM with many segments (2 D + 4 bytes a page and head), by latency with few.
#include "skv_page_index.cuh"
#include "skv_segment.cuh"

namespace skv {

namespace {

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int WARPS = 8, THREADS = WARPS * 32;
constexpr int BINS = 2048;
constexpr int MAX_PAGES = 45056;       // of a sequence: the scores of a segment are in one CTA's shared memory

// D(16x8, s32) += A(16x32, s8, row) * B(32x8, s8, col)
__device__ __forceinline__ void mma_s8_16832(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// a whole number that orders as the value does; -0 as +0
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
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

// Dynamic shared memory: scores [most] | bins [BINS] | query codes [NT * 8][2 D + 64 B] | words [64]
template <int D>
__host__ __device__ constexpr int code_row() { return 2 * D + 64; }        // (two rows that a load touches at once are not in the same banks)

template <int D, int NT>
__global__ void __launch_bounds__(THREADS) select_pages_kernel(SelectParams p, int G)
{
    extern __shared__ __align__(16) uint8_t smem_raw[];
    constexpr int J = 2 * D / 64;              // pieces of 64 bytes of an entry
    constexpr int ROW = code_row<D>();
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
    int32_t *out = p.lists + (int64_t)seg * p.stride;
    const bool choose = run.scored > p.top;    // the same for the whole cluster
    if (!choose) {
        if (rank == 0) {
            for (int i = tid; i < p.stride; i += THREADS) out[i] = i < run.end ? i : -1;
            if (tid == 0) p.counts[seg] = run.end;
        }
        if (ranks > 1) cluster_wait();
        return;
    }
    if (p.top > 0) {
        // ---- the queries' codes, [max(c, 0) | min(c, 0)] of every row and head; columns that are left over repeat the first ----
        const int cols = run.rows * G, pieces = cols * (D / 8);
        const uint16_t *q = p.Q + ((int64_t)run.row * p.Hq + (int64_t)h * G) * D;
        auto piece_of = [&](int i) {           // 8 dims of a column
            const int col = i / (D / 8), row = col / G;
            return *reinterpret_cast<const uint4 *>(q + ((int64_t)row * p.Hq + (col - row * G)) * D + i % (D / 8) * 8);
        };
        auto magnitude = [](uint32_t bits) { return bits >= 0x7F80u ? 0u : bits; };       // an element that is not finite counts as 0
        uint32_t top = 0;
        for (int i = tid; i < pieces; i += THREADS) {
            const uint4 w = piece_of(i);
            const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) top = max(top, max(magnitude(x[k] & 0x7FFFu), magnitude(x[k] >> 16 & 0x7FFFu)));
        }
        top = __reduce_max_sync(FULL, top);
        if (lane == 0) words[warp] = top;
        __syncthreads();
        top = __reduce_max_sync(FULL, words[lane & (WARPS - 1)]);
        const float amax = __uint_as_float(top << 16), inv = amax < INDEX_TINY ? 0.f : __fdiv_rn(127.f, amax);
        for (int i = tid; i < NT * 8 * (D / 8); i += THREADS) {
            const int col = i / (D / 8), piece = i % (D / 8);
            const uint4 w = piece_of(col < cols ? i : piece);
            const uint32_t x[4] = {w.x, w.y, w.z, w.w};
            uint32_t up[2] = {0, 0}, down[2] = {0, 0};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t bits = (k & 1) ? x[k / 2] >> 16 : x[k / 2] & 0xFFFFu;
                const int c = magnitude(bits & 0x7FFFu) ? __float2int_rn(__uint_as_float(bits << 16) * inv) : 0;
                up[k / 4] |= ((uint32_t)max(c, 0) & 0xFFu) << (8 * (k & 3));
                down[k / 4] |= ((uint32_t)min(c, 0) & 0xFFu) << (8 * (k & 3));
            }
            *reinterpret_cast<uint2 *>(q_codes + col * ROW + piece * 8) = make_uint2(up[0], up[1]);
            *reinterpret_cast<uint2 *>(q_codes + col * ROW + D + piece * 8) = make_uint2(down[0], down[1]);
        }
        __syncthreads();
    }
    if (ranks > 1) cluster_wait();
    if (p.top > 0) {
        // ---- scores ----
        uint32_t to;                           // the first CTA's scores
        asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"(smem_u32(keys)));
        const int tiles = (run.scored + 15) / 16;
        const int t_from = (int)((int64_t)tiles * rank / ranks), t_to = (int)((int64_t)tiles * (rank + 1) / ranks);
        const int32_t *table = p.page_table + (int64_t)run.b * p.pt_stride + run.first;
        const uint8_t *mine = q_codes + g * ROW + tig * 16;
        uint4 b_regs[NT <= 2 ? NT * J : 1];
        if (NT <= 2)
#pragma unroll
            for (int i = 0; i < NT * J; ++i) b_regs[i] = *reinterpret_cast<const uint4 *>(mine + i / J * 8 * ROW + i % J * 64);
        auto id_of = [&](int i) {              // physical page of scored page i; past the end: the last one's
            const int id = __ldg(table + (i < run.scored ? i : run.scored - 1));
            if (id >= 0 && (int64_t)id < p.max_pages) return id;
            atomicOr(p.status, STATUS_BOUNDS);
            return 0;
        };
        int id0 = 0, id1 = 0;
        if (t_from + warp < t_to) {
            id0 = id_of((t_from + warp) * 16 + g);
            id1 = id_of((t_from + warp) * 16 + g + 8);
        }
        for (int t = t_from + warp; t < t_to; t += WARPS) {
            const int64_t e0 = (int64_t)id0 * p.Hkv + h, e1 = (int64_t)id1 * p.Hkv + h;
            const uint4 *s0 = reinterpret_cast<const uint4 *>(p.codes + e0 * 2 * D) + tig, *s1 = reinterpret_cast<const uint4 *>(p.codes + e1 * 2 * D) + tig;
            uint4 a0[J], a1[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                a0[j] = __ldg(s0 + 4 * j);
                a1[j] = __ldg(s1 + 4 * j);
            }
            const float scale = __ldg(p.scales + (tig & 1 ? e1 : e0));
            if (t + WARPS < t_to) {
                id0 = id_of((t + WARPS) * 16 + g);
                id1 = id_of((t + WARPS) * 16 + g + 8);
            }
            int best0 = -0x7FFFFFFF, best1 = -0x7FFFFFFF;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                int d[4] = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const uint4 b = NT <= 2 ? b_regs[nt * J + j] : *reinterpret_cast<const uint4 *>(mine + nt * 8 * ROW + j * 64);
                    mma_s8_16832(d, a0[j].x, a1[j].x, a0[j].y, a1[j].y, b.x, b.y);
                    mma_s8_16832(d, a0[j].z, a1[j].z, a0[j].w, a1[j].w, b.z, b.w);
                }
                best0 = max(best0, max(d[0], d[1]));
                best1 = max(best1, max(d[2], d[3]));
            }
#pragma unroll
            for (int x = 1; x < 4; x <<= 1) {
                best0 = max(best0, __shfl_xor_sync(FULL, best0, x));
                best1 = max(best1, __shfl_xor_sync(FULL, best1, x));
            }
            const int i = t * 16 + g + 8 * tig;
            if (tig < 2 && i < run.scored) {
                const float inf = __uint_as_float(0x7F800000u);
                const uint32_t key = order_of(scale == inf ? inf : (float)(tig ? best1 : best0) * scale);
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + 4u * (uint32_t)i), "r"(key) : "memory");
            }
        }
    }
    if (ranks > 1) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        if (rank != 0) return;
    } else {
        __syncthreads();
    }
    // ---- the top-th largest: everything above `limit` is taken, and the first `ties` that equal it ----
    uint32_t lo = 0xFFFFFFFFu, hi = 0;
    for (int i = tid; i < run.scored && p.top > 0; i += THREADS) {
        lo = min(lo, keys[i]);
        hi = max(hi, keys[i]);
    }
    lo = __reduce_min_sync(FULL, lo);
    hi = __reduce_max_sync(FULL, hi);
    if (lane == 0) {
        words[16 + warp] = lo;
        words[24 + warp] = hi;
    }
    __syncthreads();
    lo = __reduce_min_sync(FULL, words[16 + (lane & (WARPS - 1))]);
    hi = __reduce_max_sync(FULL, words[24 + (lane & (WARPS - 1))]);
    uint32_t limit = 0xFFFFFFFFu;              // (no score's number: that of NaN)
    int need = p.top, ties = 0;
    int shift = 32 - __clz((int)(hi - lo));    // 2^shift > hi - lo
    shift = shift > 11 ? shift - 11 : 0;
    while (need > 0) {
        for (int i = tid; i < BINS; i += THREADS) bins[i] = 0;
        __syncthreads();
        for (int i = tid; i < run.scored; i += THREADS) {
            const uint32_t k = keys[i];
            if (k >= lo && k <= hi) atomicAdd(&bins[(k - lo) >> shift], 1u);
        }
        __syncthreads();
        // bins from the top: the one where the count passes `need`
        uint32_t mine[BINS / THREADS], sum = 0;
        const int from = BINS - (tid + 1) * (BINS / THREADS);          // thread 0 has the highest bins
#pragma unroll
        for (int i = 0; i < BINS / THREADS; ++i) sum += mine[i] = bins[from + i];
        uint32_t above = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t u = __shfl_up_sync(FULL, above, d);
            if (lane >= d) above += u;
        }
        if (lane == 31) words[32 + warp] = above;
        __syncthreads();
        for (int w = 0; w < warp; ++w) above += words[32 + w];
        above -= sum;                          // in the bins above this thread's
        if (above < (uint32_t)need && (uint32_t)need <= above + sum) {
#pragma unroll
            for (int i = BINS / THREADS - 1; i >= 0; --i) {
                if (above < (uint32_t)need && (uint32_t)need <= above + mine[i]) {
                    words[40] = (uint32_t)(from + i);
                    words[41] = above;
                    words[42] = mine[i];
                    break;
                }
                above += mine[i];
            }
        }
        __syncthreads();
        const uint32_t bin = words[40], higher = words[41], in_bin = words[42];
        __syncthreads();
        lo += bin << shift;
        need -= (int)higher;
        if ((uint32_t)need == in_bin) {        // the bin as a whole
            limit = lo - 1;                    // (a score's number is at least 0x007FFFFF)
            break;
        }
        if (shift == 0) {                      // scores that are equal
            limit = lo;
            ties = need;
            break;
        }
        hi = lo + ((1u << shift) - 1);
        shift = shift > 11 ? shift - 11 : 0;
    }
    // ---- the list, ascending ----
    const int per_warp = (run.scored + THREADS - 1) / THREADS * 32;
    const int w_from = warp * per_warp < run.scored ? warp * per_warp : run.scored, w_to = w_from + per_warp < run.scored ? w_from + per_warp : run.scored;
    int more = 0, same = 0;
    for (int i0 = w_from; i0 < w_to && p.top > 0; i0 += 32) {
        const uint32_t k = i0 + lane < w_to ? keys[i0 + lane] : 0;
        more += __popc(__ballot_sync(FULL, k > limit));
        same += __popc(__ballot_sync(FULL, k == limit));
    }
    if (lane == 0) {
        words[44 + warp] = (uint32_t)more;
        words[52 + warp] = (uint32_t)same;
    }
    __syncthreads();
    int taken = 0, before = 0;                 // by the warps before this one; scores equal to the limit there
    for (int w = 0; w < warp; ++w) {
        taken += (int)words[44 + w];
        before += (int)words[52 + w];
    }
    taken += before < ties ? before : ties;
    for (int i0 = w_from; i0 < w_to && p.top > 0; i0 += 32) {
        const uint32_t k = i0 + lane < w_to ? keys[i0 + lane] : 0;
        const unsigned gt = __ballot_sync(FULL, k > limit), eq = __ballot_sync(FULL, k == limit), lower = (1u << lane) - 1;
        const int eq_before = before + __popc(eq & lower), eq_taken = eq_before < ties ? eq_before : ties;
        const bool take = k > limit || (k == limit && eq_before < ties);
        const int eq_base = before < ties ? before : ties;
        if (take) out[run.first + taken + __popc(gt & lower) + eq_taken - eq_base] = run.first + i0 + lane;
        const int eq_end = before + __popc(eq);
        taken += __popc(gt) + (eq_end < ties ? eq_end : ties) - eq_base;
        before = eq_end;
    }
    const int tail = run.first + p.top, total = tail + run.end - run.last;
    for (int i = tid; i < run.first; i += THREADS) out[i] = i;
    for (int i = tail + tid; i < p.stride; i += THREADS) out[i] = i < total ? run.last + i - tail : -1;
    if (tid == 0) p.counts[seg] = total;
}

template <int D>
size_t smem_bytes(int most, int nt) { return (size_t)((most + 3) & ~3) * 4 + BINS * 4 + (size_t)nt * 8 * code_row<D>() + 64 * 4; }

template <int D, int NT>
cudaError_t launch_t(const SelectParams &p, int G, int sm_count, bool pdl, cudaStream_t s)
{
    const int64_t segments = (int64_t)p.B * p.per_seq * p.Hkv;
    // a cluster where the segments leave SMs idle, a rank with at least four tiles for each of its warps
    int ranks = 1;
    while (2 * ranks <= 8 && segments * 2 * ranks <= 2 * (int64_t)sm_count && p.most >= 2 * ranks * WARPS * 16) ranks *= 2;
    if (segments * ranks > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    const size_t smem = smem_bytes<D>(p.most, NT);
    auto kern = select_pages_kernel<D, NT>;
    cudaError_t e = ensure_dynamic_smem(kern, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(segments * ranks));
    cfg.blockDim = dim3(THREADS);
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
    return cudaLaunchKernelEx(&cfg, kern, p, G);
}

template <int D>
cudaError_t launch_d(const SelectParams &p, int G, int sm_count, bool pdl, cudaStream_t s)
{
    const int rows = p.run < p.max_q_len ? p.run : p.max_q_len, tiles = (rows * G + 7) / 8;
    if (tiles <= 1) return launch_t<D, 1>(p, G, sm_count, pdl, s);
    if (tiles <= 2) return launch_t<D, 2>(p, G, sm_count, pdl, s);
    if (tiles <= 4) return launch_t<D, 4>(p, G, sm_count, pdl, s);
    if (tiles <= 8) return launch_t<D, 8>(p, G, sm_count, pdl, s);
    if (tiles <= 16) return launch_t<D, 16>(p, G, sm_count, pdl, s);
    return cudaErrorInvalidValue;
}

}  // namespace

int select_max_pages() { return MAX_PAGES; }

cudaError_t launch_select_pages(const SelectParams &p, int D, int sm_count, bool pdl, cudaStream_t s)
{
    const int G = p.Hq / p.Hkv;
    if (p.most > MAX_PAGES) return cudaErrorInvalidValue;
    return D == 128 ? launch_d<128>(p, G, sm_count, pdl, s) : D == 64 ? launch_d<64>(p, G, sm_count, pdl, s) : cudaErrorInvalidValue;
}

}  // namespace skv
