// Decode attention over listed pages (skv_decode_attn_pages): Eq. (3.1) over the tokens of the pages that a list names for
// each (row, kv head), and the same for rows of a chunk, a row as a sequence that ends with its own token
// (skv_prefill_attn_pages where that is the quicker way).
//
// A segment -- a (row, kv head) with its list -- is one piece of work of a CTA's warps or, where the segments do not fill the GPU,
// of a cluster of CTAs, as over a window (skv_decode_window.cu): the warps take the listed pages in turn through
// rings of bulk copies of their own and the states are joined in shared memory.  Two loads stand between a warp and its first
// page, the list's entry and the page table's: a lane has them done for a page of its own, for 32 pages ahead.
#include "skv_decode_states.cuh"
#include "skv_page_index.cuh"
#include "skv_segment.cuh"
#include <atomic>
#include <type_traits>

namespace skv {

namespace {

// Dynamic shared memory: rings [NW][ST] blocks | states [NW] | the CTA's state | barriers [NW][ST]
template <int D, class State, int NW, bool EARLY, bool CHUNK>
__global__ void __launch_bounds__(NW * 32) decode_pages_kernel(DecodeParams p, PageLists l, int G, int ST)
{
    extern __shared__ __align__(128) uint8_t smem_raw[];
    constexpr int BLOCK = State::BLOCK;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t rank, ranks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    const uint32_t base = smem_u32(smem_raw);
    const uint32_t pad = (128u - (base & 127u)) & 127u;
    const uint32_t ring = base + pad + (uint32_t)(warp * ST * BLOCK);
    const int PF = part_floats(G, D);
    float *states = reinterpret_cast<float *>(smem_raw + pad + (size_t)NW * ST * BLOCK), *mine = states + (size_t)warp * PF;
    float *cta_state = states + (size_t)NW * PF;
    const uint32_t bars = base + pad + (uint32_t)((size_t)NW * ST * BLOCK + (size_t)(NW + 1) * PF * 4) + (uint32_t)(warp * ST * 8);
    if (lane == 0) {
        for (int s = 0; s < ST; ++s) mbar_init(bars + 8 * s, 1);
        fence_barrier_init();
    }
    __syncwarp();
    pdl_wait();
    if (EARLY) pdl_trigger();
    const int seg = (int)(blockIdx.x / ranks), slot = seg / p.Hkv, h = seg - slot * p.Hkv;
    int b = slot, row = slot, list = slot, n;  // sequence, row of Q and out, list, tokens up to the row's own
    int pages;                                 // of the sequence
    if (CHUNK) {                               // (every exit is the whole cluster's)
        b = slot / p.max_q_len;
        const int i = slot - b * p.max_q_len, first = __ldg(p.cu_q + b), q_len = __ldg(p.cu_q + b + 1) - first;
        n = __ldg(p.seq_lens + b);
        if (first < 0 || q_len < 0 || q_len > n || q_len > p.max_q_len || (int64_t)n > (int64_t)p.pt_stride * PAGE) {
            if (i == 0 && h == 0 && rank == 0 && threadIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
            return;
        }
        if (i >= q_len) return;
        pages = (n + PAGE - 1) / PAGE;
        n -= q_len - 1 - i;
        row = first + i;
        list = b * l.per_seq + i / l.run;
    } else {
        n = __ldg(p.seq_lens + b);
        n = n > 0 ? n : 0;
        if ((int64_t)n > (int64_t)p.pt_stride * PAGE) {
            n = p.pt_stride * PAGE;
            if (rank == 0 && h == 0 && threadIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
        }
        pages = (n + PAGE - 1) / PAGE;
    }
    const int64_t at = (int64_t)list * p.Hkv + h;
    int listed = n > 0 ? __ldg(l.counts + at) : 0;
    if (listed > l.stride) {
        listed = l.stride;
        if (rank == 0 && threadIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
    }
    uint32_t *rows = reinterpret_cast<uint32_t *>(p.out + ((int64_t)row * p.Hq + (int64_t)h * G) * D);     // pairs of bf16
    if (listed <= 0) {                         // (the same for the whole cluster: no barrier is left half-way)
        if (rank == 0)
            for (int i = threadIdx.x; i < G * D / 2; i += NW * 32) rows[i] = 0u;
        return;
    }
    const int from = (int)((int64_t)listed * rank / ranks), to = (int)((int64_t)listed * (rank + 1) / ranks);
    const int count = to - from > warp ? (to - from - warp + NW - 1) / NW : 0;       // this warp's entries: from + warp + i * NW
    const int32_t *entries = l.lists + at * l.stride + from + warp, *table = p.page_table + (int64_t)b * p.pt_stride;
    const uint64_t policy = p.keep_pct > 0 ? make_policy_evict_normal() : make_policy_evict_first();
    // Entry i: physical page and the tokens of it that the row sees.  Where those are none (an entry out of range is one of these) the
    // page that is copied in its place is not looked at.
    auto entry = [&](int i, int &id, uint32_t &bits) {
        id = 0;
        bits = 0;
        if (i >= count) return;
        const int page = __ldg(entries + i * NW);
        if (page < 0 || page >= pages) {
            atomicOr(p.status, STATUS_BOUNDS);
            return;
        }
        const int left = n - page * PAGE;
        bits = left >= PAGE ? 0xFFFFu : left > 0 ? (1u << left) - 1 : 0u;
        id = __ldg(table + page);
        if (id < 0 || (int64_t)id >= p.max_pages) {
            atomicOr(p.status, STATUS_BOUNDS);
            id = 0;
        }
    };
    auto send = [&](int i, int id) {           // by one lane
        const int s = i % ST;
        mbar_expect_tx(bars + 8 * s, BLOCK);
        bulk_copy_g2s_hint(ring + (uint32_t)(s * BLOCK), p.layer_base + (int64_t)id * p.page_stride + (int64_t)h * BLOCK, BLOCK, bars + 8 * s, policy);
    };
    int id, next_id = 0;                       // lane i: of entry 32 k + i, and of the 32 after those
    uint32_t bits, next_bits = 0;
    entry(lane, id, bits);
    int sent = count < ST ? count : ST, done = 0;
    if (lane < sent) send(lane, id);
    if (count > 32) entry(32 + lane, next_id, next_bits);
    State st;
    st.begin(p, row, h, G, lane);
    bool ok = true;
    for (; done < count; ++done) {
        if (done > 0 && (done & 31) == 0) {
            id = next_id;
            bits = next_bits;
            entry(done + 32 + lane, next_id, next_bits);
        }
        const int s = done % ST;
        ok = __all_sync(FULL, mbar_wait_bounded(bars + 8 * s, (uint32_t)((done / ST) & 1)));
        if (!ok) break;
        const uint32_t seen = __shfl_sync(FULL, bits, done & 31);
        if (seen) st.page_bits(ring + (uint32_t)(s * BLOCK), seen, p.scale_log2, lane);
        __syncwarp();                          // every lane is done reading this stage
        if (sent < count) {
            const int ahead = __shfl_sync(FULL, (sent & ~31) == (done & ~31) ? id : next_id, sent & 31);
            if (lane == 0) send(sent, ahead);
            ++sent;
        }
    }
    if (!ok) {
        // the copies still in flight get their (bounded) wait before the shared memory goes away
        if (lane == 0) {
            atomicOr(p.status, STATUS_TIMEOUT);
            for (int i = done + 1; i < sent; ++i) mbar_wait_bounded(bars + 8 * (i % ST), (uint32_t)((i / ST) & 1));
        }
        __syncwarp();
    }
    if (count > 0) st.finish(mine, mine + G * D, 0, G, lane);
    else if (lane < G) *reinterpret_cast<float2 *>(mine + G * D + 2 * lane) = make_float2(-INFINITY, 0.f);
    __syncthreads();
    auto write_row = [&](int e2, float L, float2 a) {
        const float inv = L == 0.f ? 0.f : 1.f / L;          // (a NaN stays one)
        rows[e2] = pack_bf16x2(a.x * inv, a.y * inv);
    };
    for (int e2 = threadIdx.x; e2 < G * D / 2; e2 += NW * 32) {
        float M, L;
        float2 a;
        join_states<NW>(NW, 2 * e2 / D, e2, [&](int c, int g) { return *reinterpret_cast<const float2 *>(states + (size_t)c * PF + G * D + 2 * g); },
                        [&](int c, int e) { return *reinterpret_cast<const float2 *>(states + (size_t)c * PF + 2 * e); }, M, L, a);
        if (ranks == 1) {
            write_row(e2, L, a);
            continue;
        }
        *reinterpret_cast<float2 *>(cta_state + 2 * e2) = a;
        if (2 * e2 % D == 0) *reinterpret_cast<float2 *>(cta_state + G * D + 2 * (2 * e2 / D)) = make_float2(M, L);
    }
    if (ranks == 1) return;
    __syncwarp();
    cluster_arrive();                          // this CTA's state is complete ...
    cluster_wait();                            // ... and so is everybody's
    const uint32_t theirs = smem_u32(cta_state);
    const int e_from = G * D / 2 * (int)rank / (int)ranks, e_to = G * D / 2 * (int)(rank + 1) / (int)ranks;
    for (int e2 = e_from + (int)threadIdx.x; e2 < e_to; e2 += NW * 32) {
        float M, L;
        float2 a;
        join_states<MAX_RANKS>((int)ranks, 2 * e2 / D, e2, [&](int c, int g) { return ld_cluster_f2(at_rank(theirs, (uint32_t)c) + (uint32_t)(G * D + 2 * g) * 4); },
                               [&](int c, int e) { return ld_cluster_f2(at_rank(theirs, (uint32_t)c) + (uint32_t)(2 * e) * 4); }, M, L, a);
        write_row(e2, L, a);
    }
    __syncwarp();
    cluster_arrive();                          // nobody leaves while its state is being read
    cluster_wait();
}

template <int D, class State, bool CHUNK>
cudaError_t launch_t(const DecodeParams &p, const PageLists &l, int G, int sm_count, bool pdl, cudaStream_t s)
{
    const int64_t segments = (int64_t)p.B * p.Hkv;
    const Shape f = shape_of(State::BLOCK, segments, l.stride < p.pt_stride ? l.stride : p.pt_stride, sm_count);
    if (segments * f.ranks > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    const size_t smem = 128 + (size_t)f.warps * f.stages * State::BLOCK + (size_t)(f.warps + 1) * part_floats(G, D) * 4 + (size_t)f.warps * f.stages * 8;
    const bool early = segments * f.ranks <= sm_count;       // (as over a window: the next launch may fill the SMs that this one leaves free)
    auto kern = CHUNK        ? (f.warps == 8 ? decode_pages_kernel<D, State, 8, false, CHUNK> : decode_pages_kernel<D, State, 4, false, CHUNK>)
                : f.warps == 8 ? (early ? decode_pages_kernel<D, State, 8, true, CHUNK> : decode_pages_kernel<D, State, 8, false, CHUNK>)
                               : (early ? decode_pages_kernel<D, State, 4, true, CHUNK> : decode_pages_kernel<D, State, 4, false, CHUNK>);
    cudaError_t e = ensure_dynamic_smem(kern, smem);
    if (e != cudaSuccess) return e;
    if (f.ranks > 8) {
        static std::atomic<uint64_t> allowed[4];           // (bit per device: asking every time costs more than the launch)
        int dev = 0;
        if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
        const uint64_t bit = 1ull << (dev & 63);
        if (dev > 63 || !(allowed[2 * (f.warps == 8) + early] & bit)) {
            e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            if (e != cudaSuccess) return e;
            allowed[2 * (f.warps == 8) + early] |= bit;
        }
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(segments * f.ranks));
    cfg.blockDim = dim3((unsigned)(f.warps * 32));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (f.ranks > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)f.ranks;
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
    return cudaLaunchKernelEx(&cfg, kern, p, l, G, f.stages);
}

}  // namespace

cudaError_t launch_decode_pages(const DecodeParams &p, const PageLists &l, int D, int G, int kernel, int sm_count, bool pdl, cudaStream_t s)
{
    auto go = [&](auto dim) {
        constexpr int N = decltype(dim)::value;
        if (kernel == 2) return p.cu_q ? launch_t<N, Fp8State<N>, true>(p, l, G, sm_count, pdl, s) : launch_t<N, Fp8State<N>, false>(p, l, G, sm_count, pdl, s);
        if (kernel == 1) return p.cu_q ? launch_t<N, TensorCoreState<N>, true>(p, l, G, sm_count, pdl, s) : launch_t<N, TensorCoreState<N>, false>(p, l, G, sm_count, pdl, s);
        return p.cu_q ? launch_t<N, CudaCoreState<N>, true>(p, l, G, sm_count, pdl, s) : launch_t<N, CudaCoreState<N>, false>(p, l, G, sm_count, pdl, s);
    };
    return D == 128 ? go(std::integral_constant<int, 128>()) : D == 64 ? go(std::integral_constant<int, 64>()) : cudaErrorInvalidValue;
}

}  // namespace skv
