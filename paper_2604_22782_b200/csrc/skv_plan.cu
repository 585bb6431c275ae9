// A step's tables, made on the GPU from the requests' lengths: new pages off a stack of free ones into the page
// table, the slot and position of every new token, the row offsets and the new lengths; and the way back, pages
// from the table onto the stack.
//
// All of it follows from prefix sums over the requests (which are admitted, how many pages and tokens come before
// each), so it is a matter of latency, not of bytes: every CTA reads all requests' lengths and repeats the scans for
// itself in shared memory -- cheaper than a second launch or a trip through global memory -- and then writes its
// share of the tokens and pages, each found by a binary search in the sums.  Where an output may be the same memory
// as the input it comes from (seq_lens, n_free: a loop that keeps its state in place), the CTAs are one cluster and
// that output is written after a cluster barrier behind everybody's reads; no counter in memory, nothing to reset.
// 64 requests of a token each 3.7 us, little more than a launch; 256 requests with some thousand tokens 5.8.
#include "skv_common.cuh"

namespace skv {

namespace {

constexpr int PLAN_MAX_BATCH = 16384;
constexpr unsigned ALL = 0xFFFFFFFFu;

__device__ __forceinline__ int pages_of(int64_t tokens) { return (int)((tokens + PAGE - 1) / PAGE); }

// exclusive prefix of two sums over the threads of the CTA; tot: the CTA's sums.  part: [2][32] words of shared memory
__device__ __forceinline__ void block_scan2(int64_t &a, int64_t &b, int64_t &tot_a, int64_t &tot_b, int64_t *part)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (int)(blockDim.x >> 5);
    int64_t ia = a, ib = b;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t ua = __shfl_up_sync(ALL, ia, d), ub = __shfl_up_sync(ALL, ib, d);
        if (lane >= d) { ia += ua; ib += ub; }
    }
    __syncthreads();                               // (part may still be read from the scan before)
    if (lane == 31) { part[warp] = ia; part[32 + warp] = ib; }
    __syncthreads();
    int64_t wa = lane < warps ? part[lane] : 0, wb = lane < warps ? part[32 + lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t ua = __shfl_up_sync(ALL, wa, d), ub = __shfl_up_sync(ALL, wb, d);
        if (lane >= d) { wa += ua; wb += ub; }
    }
    tot_a = __shfl_sync(ALL, wa, 31);
    tot_b = __shfl_sync(ALL, wb, 31);
    const int64_t ba = __shfl_sync(ALL, wa, (warp + 31) & 31), bb = __shfl_sync(ALL, wb, (warp + 31) & 31);
    a = ia - a + (warp ? ba : 0);
    b = ib - b + (warp ? bb : 0);
}

// the largest i with sums[i] <= x (sums[0] = 0, non-decreasing, x < sums[n])
__device__ __forceinline__ int owner_of(const int32_t *sums, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// Dynamic shared memory: cached[B] | tokens before [B+1] | pages before [B+1]
template <bool IN_PLACE>
__global__ void __launch_bounds__(1024) plan_step_kernel(const __grid_constant__ PlanParams p)
{
    extern __shared__ int32_t tables[];
    __shared__ int64_t part[64];
    int32_t *cached = tables, *tok_before = cached + p.B, *page_before = tok_before + p.B + 1;
    const int tid = threadIdx.x, nt = blockDim.x, rank = blockIdx.x, ranks = gridDim.x;
    pdl_wait();
    pdl_trigger();
    int64_t row_tokens = (int64_t)p.pt_stride * PAGE;
    if (row_tokens > 0x7FFFFFFF) row_tokens = 0x7FFFFFFF;      // lengths and positions are 32-bit
    int n_free = __ldcg(p.n_free);                  // (may be written below: not through the read-only path)
    n_free = n_free < 0 ? 0 : n_free > p.free_capacity ? p.free_capacity : n_free;
    // ---- which requests are admitted: inclusive sums of what all requests ask for, in request order ----
    const int per = (p.B + nt - 1) / nt, b0 = tid * per < p.B ? tid * per : p.B, b1 = b0 + per < p.B ? b0 + per : p.B;
    auto asks = [&](int b, int &n, int64_t &a, int64_t &need) {
        n = cached[b];
        a = tok_before[b];                         // (as it was put there below)
        need = pages_of((int64_t)n + a) - pages_of(n);
    };
    for (int b = tid; b < p.B; b += nt) {          // whole lines, once
        const int n = __ldcg(p.seq_lens + b), a = __ldg(p.new_lens + b);
        cached[b] = n > 0 ? n : 0;
        tok_before[b] = a > 0 ? a : 0;
    }
    __syncthreads();
    if (IN_PLACE) asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");       // this CTA has read seq_lens and n_free
    int64_t sum_a = 0, sum_p = 0, tot_a, tot_p;
    for (int b = b0; b < b1; ++b) {
        int n;
        int64_t a, need;
        asks(b, n, a, need);
        sum_a += a;
        sum_p += need;
    }
    block_scan2(sum_a, sum_p, tot_a, tot_p, part);
    int64_t in_a = 0, in_p = 0;                    // admitted ones of this thread
    int flags = 0;
    for (int b = b0; b < b1; ++b) {
        int n;
        int64_t a, need;
        asks(b, n, a, need);
        sum_a += a;
        sum_p += need;
        const bool fits_row = n + a <= row_tokens, ok = (need == 0 || sum_p <= n_free) && sum_a <= p.max_tokens && fits_row;
        if (!ok && a > 0) flags |= fits_row ? STATUS_NOMEM : STATUS_BOUNDS;
        if (!ok) tok_before[b] = 0;                // (this thread's own entry)
        else { in_a += a; in_p += need; }
    }
    if (flags && rank == 0) atomicOr(p.status, flags);
    block_scan2(in_a, in_p, tot_a, tot_p, part);
    const int n_tok = (int)tot_a, n_page = (int)tot_p;       // (at most max_tokens < 2^31 and n_free)
    for (int b = b0; b < b1; ++b) {
        int n;
        int64_t a, need;
        asks(b, n, a, need);
        tok_before[b] = (int)in_a;
        page_before[b] = (int)in_p;
        in_a += a;
        in_p += need;
    }
    if (tid == 0) {
        tok_before[p.B] = n_tok;
        page_before[p.B] = n_page;
    }
    __syncthreads();
    // ---- the tokens' slots and positions; pages taken in this step are looked up on the stack, not in the table ----
    const int step = ranks * nt, first = rank * nt + tid;
    bool bad = false;
    for (int64_t i = first; i < n_tok; i += step) {
        const int b = owner_of(tok_before, p.B, (int)i), n = cached[b], pos = n + ((int)i - tok_before[b]), pg = pos >> 4, old = pages_of(n);
        const int id = pg < old ? p.page_table[(int64_t)b * p.pt_stride + pg] : __ldg(p.free_pages + (n_free - 1 - (page_before[b] + pg - old)));
        const bool good = id >= 0 && (int64_t)id < p.max_pages;
        bad |= !good;
        p.slot_map[i] = good ? (int64_t)id * PAGE + (pos & (PAGE - 1)) : -1;
        if (p.positions) p.positions[i] = pos;
    }
    if (bad) atomicOr(p.status, STATUS_BOUNDS);
    for (int64_t k = first; k < n_page; k += step) {
        const int b = owner_of(page_before, p.B, (int)k), at = pages_of(cached[b]) + ((int)k - page_before[b]);
        p.page_table[(int64_t)b * p.pt_stride + at] = __ldg(p.free_pages + (n_free - 1 - (int)k));
    }
    for (int b = first; b <= p.B; b += step) p.cu_q_lens[b] = tok_before[b];
    if (IN_PLACE) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    for (int b = first; b < p.B; b += step) p.seq_lens_out[b] = cached[b] + (tok_before[b + 1] - tok_before[b]);
    if (first == 0) *p.n_free_out = n_free - n_page;
}

// One CTA.  The rows that give pages back are listed first (usually few), then a warp per row counts the
// entries that hold a page, and after a scan of the counts writes them onto the stack in row order.
// Dynamic shared memory: listed rows [B] | their counts, then offsets [B]
__global__ void __launch_bounds__(1024) plan_release_kernel(const __grid_constant__ ReleaseParams p)
{
    extern __shared__ int32_t tables[];
    __shared__ int64_t part[64];
    int32_t *rows = tables, *count = tables + p.B;
    const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5, warps = nt >> 5;
    pdl_wait();
    pdl_trigger();
    int n_free = __ldcg(p.n_free);
    n_free = n_free < 0 ? 0 : n_free > p.free_capacity ? p.free_capacity : n_free;
    auto range = [&](int b, int &from, int &to) {
        from = __ldg(p.first_page + b);
        to = __ldg(p.end_page + b);
        from = from < 0 ? 0 : from;
        to = to > p.pt_stride ? p.pt_stride : to;
    };
    const int per = (p.B + nt - 1) / nt, b0 = tid * per < p.B ? tid * per : p.B, b1 = b0 + per < p.B ? b0 + per : p.B;
    int64_t mine = 0, none = 0, n_rows, tot;
    for (int b = b0; b < b1; ++b) {
        int from, to;
        range(b, from, to);
        mine += from < to;
    }
    block_scan2(mine, none, n_rows, tot, part);
    for (int b = b0; b < b1; ++b) {
        int from, to;
        range(b, from, to);
        if (from < to) rows[mine++] = b;
    }
    __syncthreads();
    auto holds = [&](int32_t id) { return id >= 0 && (int64_t)id < p.max_pages; };
    bool bad = false;
    for (int r = warp; r < n_rows; r += warps) {
        int from, to, n = 0;
        range(rows[r], from, to);
        const int32_t *row = p.page_table + (int64_t)rows[r] * p.pt_stride;
        for (unsigned at = from; at < (unsigned)to; at += 32) {                // (unsigned: the last step may pass 31 bits)
            const int32_t id = at + lane < (unsigned)to ? row[at + lane] : -1;
            bad |= id >= 0 && !holds(id);
            n += __popc(__ballot_sync(ALL, holds(id)));
        }
        if (lane == 0) count[r] = n;
    }
    if (bad) atomicOr(p.status, STATUS_BOUNDS);
    __syncthreads();
    const int rper = ((int)n_rows + nt - 1) / nt, r0 = tid * rper < n_rows ? tid * rper : (int)n_rows, r1 = r0 + rper < n_rows ? r0 + rper : (int)n_rows;
    int64_t sum = 0, zero = 0, total;
    for (int r = r0; r < r1; ++r) sum += count[r];
    block_scan2(sum, zero, total, tot, part);
    const uint32_t room = (uint32_t)(p.free_capacity - n_free);
    for (int r = r0; r < r1; ++r) {
        const int n = count[r];
        count[r] = (int)release_start(sum, room);
        sum += n;
    }
    __syncthreads();
    for (int r = warp; r < n_rows; r += warps) {
        int from, to;
        range(rows[r], from, to);
        uint32_t start = (uint32_t)count[r];
        int32_t *row = p.page_table + (int64_t)rows[r] * p.pt_stride;
        for (unsigned at = from; at < (unsigned)to; at += 32) {
            const int32_t id = at + lane < (unsigned)to ? row[at + lane] : -1;
            const unsigned have = __ballot_sync(ALL, holds(id));
            const uint32_t k = release_next(start, __popc(have & ((1u << lane) - 1u)), room);
            if (holds(id) && k < room) {
                p.free_pages[n_free + (int)k] = id;
                row[at + lane] = -1;
            }
            start = release_next(start, __popc(have), room);
        }
    }
    if (tid == 0) {
        *p.n_free_out = n_free + (int)(total < room ? total : room);
        if (total > room) atomicOr(p.status, STATUS_NOMEM);
    }
}

}  // namespace

int plan_max_batch() { return PLAN_MAX_BATCH; }

cudaError_t launch_plan_step(const PlanParams &p, bool in_place, int sm_count, bool pdl, cudaStream_t s)
{
    // A token per thread (the scans are repeated by each CTA), at most a CTA per SM, or one cluster of the portable
    // size where outputs may lie on inputs.
    const int most = in_place ? 8 : sm_count;
    int64_t ctas = (p.max_tokens + 1023) / 1024;
    ctas = ctas < 1 ? 1 : ctas > most ? most : ctas;
    const int threads = p.B <= 256 && p.max_tokens <= 1024 ? 256 : 1024;
    const size_t smem = (size_t)(3 * p.B + 2) * sizeof(int32_t);
    auto kern = in_place ? plan_step_kernel<true> : plan_step_kernel<false>;
    const cudaError_t e = ensure_dynamic_smem(kern, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (in_place) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)ctas;
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
    return cudaLaunchKernelEx(&cfg, kern, p);
}

cudaError_t launch_plan_release(const ReleaseParams &p, bool pdl, cudaStream_t s)
{
    const size_t smem = (size_t)2 * p.B * sizeof(int32_t);
    const cudaError_t e = ensure_dynamic_smem(plan_release_kernel, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1);
    cfg.blockDim = dim3(1024);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, plan_release_kernel, p);
}

}  // namespace skv
