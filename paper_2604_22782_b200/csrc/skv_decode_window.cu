// Decode attention over a sliding window with sinks (skv_decode_attn_window): Eq. (3.1) over the tokens
// t >= n - window  or  t < sinks  of a sequence, i.e. over the pages of window_pages() with a few tokens of them masked.
//
// A window makes the segments -- the (sequence, kv head) pairs -- short and nearly equal, so a segment is one piece
// of work: a CTA's warps take its pages in turn, each through a small ring of bulk copies of its own (a page's K and V of
// one kv head are one contiguous block), keep a running (max, sum, output), and combine in shared memory.  Where the
// segments alone do not fill the GPU, a cluster of CTAs shares a segment and combines through distributed shared
// memory: after a cluster barrier every CTA reads all CTAs' states for its share of the rows.  One launch, no partials in
// global memory, no merge kernel.
// Bound by HBM where there is work for every SM: 32 sequences of 8 kv heads, window 2048 (262 MB) 42.3 us, 6.2 TB/s; 32 kv heads,
// window 4096 (539 MB) 80 us, 6.7 TB/s, above the measured copy peak; by latency below that: one sequence, window 1024, 8 kv
// heads 5.6 us, an empty window 4.6 us.  Cutting the block list into a range per SM and merging, as the unwindowed call does,
// costs 16.8 us there and 83 us where this kernel takes 73 (128 sequences, window 1024), because the short segments are cut and
// joined again.
#include "skv_common.cuh"
#include "skv_decode_states.cuh"
#include "skv_segment.cuh"
#include "skv_walk.cuh"
#include <atomic>

namespace skv {

namespace {

// Dynamic shared memory: rings [NW][ST] blocks | states [NW] | the CTA's state | barriers [NW][ST]
template <int D, class State, int NW, bool EARLY, bool CHUNK>
__global__ void __launch_bounds__(NW * 32) decode_window_kernel(DecodeParams p, int G, int ST)
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
    int b = slot, row = slot, n;               // sequence, row of Q and out, tokens up to the row's own
    if (CHUNK) {                               // (every exit is the whole cluster's)
        b = slot / p.max_q_len;
        const int i = slot - b * p.max_q_len, first = __ldg(p.cu_q + b), q_len = __ldg(p.cu_q + b + 1) - first;
        n = __ldg(p.seq_lens + b);
        if (first < 0 || q_len < 0 || q_len > n || q_len > p.max_q_len || (int64_t)n > (int64_t)p.pt_stride * PAGE) {
            if (i == 0 && h == 0 && rank == 0 && threadIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
            return;
        }
        if (i >= q_len) return;
        n -= q_len - 1 - i;
        row = first + i;
    } else {
        n = __ldg(p.seq_lens + b);
        n = n > 0 ? n : 0;
        if ((int64_t)n > (int64_t)p.pt_stride * PAGE) {
            n = p.pt_stride * PAGE;
            if (rank == 0 && h == 0 && threadIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
        }
    }
    uint32_t *rows = reinterpret_cast<uint32_t *>(p.out + ((int64_t)row * p.Hq + (int64_t)h * G) * D);     // pairs of bf16
    if (n == 0) {                              // (the same for the whole cluster: no barrier is left half-way)
        if (rank == 0)
            for (int i = threadIdx.x; i < G * D / 2; i += NW * 32) rows[i] = 0u;
        return;
    }
    const WindowPages win = window_pages(n - 1, n, p.window, p.sinks);
    const int from = (int)((int64_t)win.count * rank / ranks), to = (int)((int64_t)win.count * (rank + 1) / ranks);
    const int count = to - from > warp ? (to - from - warp + NW - 1) / NW : 0;       // this warp's pages: from + warp + i * NW
    const int32_t *table = p.page_table + (int64_t)b * p.pt_stride;
    const uint64_t policy = p.keep_pct > 0 ? make_policy_evict_normal() : make_policy_evict_first();
    auto send = [&](int i, int id) {           // by one lane
        if (id < 0 || (int64_t)id >= p.max_pages) {
            atomicOr(p.status, STATUS_BOUNDS);
            id = 0;
        }
        const int s = i % ST;
        mbar_expect_tx(bars + 8 * s, BLOCK);
        bulk_copy_g2s_hint(ring + (uint32_t)(s * BLOCK), p.layer_base + (int64_t)id * p.page_stride + (int64_t)h * BLOCK, BLOCK, bars + 8 * s, policy);
    };
    auto id_of = [&](int i) { return i < count ? __ldg(table + win.page(from + warp + i * NW)) : 0; };
    int next_id = id_of(lane < ST ? lane : ST);                      // lanes < ST: the first pages; lane ST on: page ST's
    if (lane < ST && lane < count) send(lane, next_id);
    next_id = __shfl_sync(FULL, next_id, ST);
    State st;
    st.begin(p, row, h, G, lane);
    int sent = count < ST ? count : ST, done = 0;
    bool ok = true;
    for (; done < count; ++done) {
        const int s = done % ST;
        ok = __all_sync(FULL, mbar_wait_bounded(bars + 8 * s, (uint32_t)((done / ST) & 1)));
        if (!ok) break;
        st.page_bits(ring + (uint32_t)(s * BLOCK), window_bits(win.page(from + warp + done * NW), win.lo, n, p.sinks), p.scale_log2, lane);
        __syncwarp();                          // every lane is done reading this stage
        if (sent < count) {
            if (lane == 0) send(sent, next_id);
            ++sent;
            next_id = id_of(sent);
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
cudaError_t launch_t(const DecodeParams &p, int G, int sm_count, bool pdl, cudaStream_t s)
{
    const int64_t segments = (int64_t)p.B * p.Hkv;
    int64_t pages = ((int64_t)p.window + PAGE - 2) / PAGE + 1 + ((int64_t)p.sinks + PAGE - 1) / PAGE;      // of a segment, at most
    if (pages > p.pt_stride) pages = p.pt_stride;
    const Shape f = shape_of(State::BLOCK, segments, pages, sm_count, wide_ctas<State>());
    if (segments * f.ranks > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    const size_t smem = 128 + (size_t)f.warps * f.stages * State::BLOCK + (size_t)(f.warps + 1) * part_floats(G, D) * 4 + (size_t)f.warps * f.stages * 8;
    // The next launch may be let in at once where there is an SM for every CTA; else it would fill what this one leaves
    // free, two CTAs here and none there, and run as unevenly (64 x 129 pages: 42 us, and 51 let in at once; 1024 x 257 pages
    // 79 and 84; 8 x 65 pages 6.0 and 5.6).
    const bool early = segments * f.ranks <= sm_count;
    auto kern = CHUNK        ? (f.warps == 8 ? decode_window_kernel<D, State, 8, false, CHUNK> : decode_window_kernel<D, State, 4, false, CHUNK>)
                : f.warps == 8 ? (early ? decode_window_kernel<D, State, 8, true, CHUNK> : decode_window_kernel<D, State, 8, false, CHUNK>)
                               : (early ? decode_window_kernel<D, State, 4, true, CHUNK> : decode_window_kernel<D, State, 4, false, CHUNK>);
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
    return cudaLaunchKernelEx(&cfg, kern, p, G, f.stages);
}

}  // namespace

cudaError_t launch_decode_window(const DecodeParams &p, int D, int G, int kernel, int sm_count, bool pdl, cudaStream_t s)
{
    if (D == 128) {
        if (kernel == 2) return p.cu_q ? launch_t<128, Fp8State<128>, true>(p, G, sm_count, pdl, s) : launch_t<128, Fp8State<128>, false>(p, G, sm_count, pdl, s);
        if (kernel == 1) return p.cu_q ? launch_t<128, TensorCoreState<128>, true>(p, G, sm_count, pdl, s) : launch_t<128, TensorCoreState<128>, false>(p, G, sm_count, pdl, s);
        return p.cu_q ? launch_t<128, CudaCoreState<128>, true>(p, G, sm_count, pdl, s) : launch_t<128, CudaCoreState<128>, false>(p, G, sm_count, pdl, s);
    }
    if (D == 64) {
        if (kernel == 2) return p.cu_q ? launch_t<64, Fp8State<64>, true>(p, G, sm_count, pdl, s) : launch_t<64, Fp8State<64>, false>(p, G, sm_count, pdl, s);
        if (kernel == 1) return p.cu_q ? launch_t<64, TensorCoreState<64>, true>(p, G, sm_count, pdl, s) : launch_t<64, TensorCoreState<64>, false>(p, G, sm_count, pdl, s);
        return p.cu_q ? launch_t<64, CudaCoreState<64>, true>(p, G, sm_count, pdl, s) : launch_t<64, CudaCoreState<64>, false>(p, G, sm_count, pdl, s);
    }
    return cudaErrorInvalidValue;
}

#ifdef SKV_TEST_HOOKS
void decode_window_shape(int D, int kernel, int64_t segments, int64_t pages, int sm_count, int *out)
{
    auto ask = [&](auto state) {
        using State = typename decltype(state)::type;
        const Shape f = shape_of(State::BLOCK, segments, pages, sm_count, wide_ctas<State>());
        out[0] = f.warps;
        out[1] = f.stages;
        out[2] = f.ranks;
        out[3] = f.warps == 8 ? wide_ctas<State>() : 2;
    };
    if (D == 128) kernel == 2 ? ask(Type<Fp8State<128>>()) : kernel == 1 ? ask(Type<TensorCoreState<128>>()) : ask(Type<CudaCoreState<128>>());
    else kernel == 2 ? ask(Type<Fp8State<64>>()) : kernel == 1 ? ask(Type<TensorCoreState<64>>()) : ask(Type<CudaCoreState<64>>());
}
#endif

}  // namespace skv
