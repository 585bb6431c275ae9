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
#include "skv_walk.cuh"
#include <atomic>
#include <type_traits>

namespace skv {

namespace {

constexpr int MAX_RANKS = 16;          // CTAs that may share a segment

__host__ __device__ constexpr int part_floats(int G, int D) { return G * D + ((2 * G + 3) & ~3); }

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// shared-memory address `a` of this CTA as the CTA of the given rank has it
__device__ __forceinline__ uint32_t at_rank(uint32_t a, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
    return r;
}
__device__ __forceinline__ float2 ld_cluster_f2(uint32_t a)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
    return v;
}

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
    // sum of n_states states, weighted: the pair e2 of the segment's rows and its head's (max, sum)
    auto combine = [&](auto most, int n_states, int e2, auto ml_of, auto pair_of, float &M, float &L, float2 &a) {
        constexpr int N = decltype(most)::value;
        float2 ml[N], v[N];
#pragma unroll
        for (int c = 0; c < N; ++c) {
            ml[c] = make_float2(-INFINITY, 0.f);
            v[c] = make_float2(0.f, 0.f);
            if (c < n_states) {
                ml[c] = ml_of(c, 2 * e2 / D);
                v[c] = pair_of(c, e2);
            }
        }
        M = -INFINITY;
#pragma unroll
        for (int c = 0; c < N; ++c) M = fmaxf(M, ml[c].x);
        L = 0.f;
        a = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < N; ++c) {
            // No page there, or not there: the sum says so, which is 1 or more where there is one, or NaN.  (Not the maximum:
            // that is -inf too where every score is NaN, and the result has to be NaN then.)
            if (ml[c].y == 0.f) continue;
            const float w = fast_exp2(ml[c].x - M);
            L = fmaf(w, ml[c].y, L);
            a.x = fmaf(w, v[c].x, a.x);
            a.y = fmaf(w, v[c].y, a.y);
        }
    };
    auto write_row = [&](int e2, float L, float2 a) {
        const float inv = L == 0.f ? 0.f : 1.f / L;          // (a NaN stays one)
        rows[e2] = pack_bf16x2(a.x * inv, a.y * inv);
    };
    for (int e2 = threadIdx.x; e2 < G * D / 2; e2 += NW * 32) {
        float M, L;
        float2 a;
        combine(std::integral_constant<int, NW>(), NW, e2, [&](int c, int g) { return *reinterpret_cast<const float2 *>(states + (size_t)c * PF + G * D + 2 * g); },
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
        combine(std::integral_constant<int, MAX_RANKS>(), (int)ranks, e2, [&](int c, int g) { return ld_cluster_f2(at_rank(theirs, (uint32_t)c) + (uint32_t)(G * D + 2 * g) * 4); },
                [&](int c, int e) { return ld_cluster_f2(at_rank(theirs, (uint32_t)c) + (uint32_t)(2 * e) * 4); }, M, L, a);
        write_row(e2, L, a);
    }
    __syncwarp();
    cluster_arrive();                          // nobody leaves while its state is being read
    cluster_wait();
}

// How a call is laid out: warps per CTA, pages in flight per warp, CTAs per segment.
struct Shape { int warps, stages, ranks; };

// `block` bytes per page and kv head, `segments` of at most `pages` pages.  Measured (us; rows of the sweep: segments x
// pages at 8 KB blocks; W warps, S stages, R ranks):
//       8 x   65   W8 S1 R16  5.7   W8 S2 R8  6.0   W4 S2 R16  5.8
//       8 x  513   W8 S1 R16 11.1   W4 S2 R16 12.2
//      16 x   65   W4 S2 R16  6.3   W8 S2 R8 11.1
//      16 x  513   W4 S2 R16 14.9   W8 S2 R8 25.2
//      64 x   65   W8 S2 R2   9.7   W4 S2 R4 10.0   W8 S1 R4 10.1
//     128 x   65   W8 S2 R1  13.1   W8 S1 R2 14.1   W4 S2 R2 14.5
//     256 x  129   W4 S2 R1  37.2   W8 S1 R1 37.1   W8 S2 R1 41.5
//     320 x  257   W4 S2 R1  93.0   W4 S2 R2 100
//    1024 x   65   W4 S2 R1  72.8   W8 S1 R1 75.7   W8 S2 R1 80.5
// So: a CTA of 8 warps and two stages (one per SM) where a power of two of them per segment comes close to one for every
// SM, and 4 warps with two stages (three per SM) else, as many ranks as still leave all CTAs resident at once.  A cluster's CTAs
// share a GPC, whose SMs are not a multiple of 8: of 8 CTAs with an SM each 15 clusters run at once, and the 16th doubles the time.
// Blocks of half the size (FP8, head_dim 64) take 8 warps in the same space, and 16 ranks of them only with an SM for each
// (16 segments x 257 pages: 11.5 us, in clusters of 8 7.8).  A rank has at least four pages.
Shape shape_of(int block, int64_t segments, int64_t pages, int sm)
{
    Shape best = {block >= 8192 ? 4 : 8, 2, 1};
    auto ranks_up_to = [&](int64_t ctas, int most) {
        int r = 1;
        while (2 * r <= most && segments * 2 * r <= ctas && pages >= 4 * 2 * r) r *= 2;
        return r;
    };
    best.ranks = ranks_up_to(2 * (int64_t)sm + sm / 4, block >= 8192 || 16 * segments <= sm ? MAX_RANKS : 8);
    if (block >= 8192) {
        const int r = ranks_up_to(sm, MAX_RANKS);
        const int64_t room = r == 8 ? 3 * (int64_t)sm / 4 : r == 4 ? 7 * (int64_t)sm / 8 : sm;
        const bool fills = 4 * segments * r >= 3 * (int64_t)sm && segments * r <= room;
        if (fills) best = {8, r > 8 ? 1 : 2, r};             // (a cluster of 16 needs two CTAs to an SM: a GPC may not have 16 SMs)
    }
    const int64_t per_warp = (pages + (int64_t)best.ranks * best.warps - 1) / ((int64_t)best.ranks * best.warps);
    if (per_warp < best.stages) best.stages = 1;
    return best;
}

template <int D, class State, bool CHUNK>
cudaError_t launch_t(const DecodeParams &p, int G, int sm_count, bool pdl, cudaStream_t s)
{
    const int64_t segments = (int64_t)p.B * p.Hkv;
    int64_t pages = ((int64_t)p.window + PAGE - 2) / PAGE + 1 + ((int64_t)p.sinks + PAGE - 1) / PAGE;      // of a segment, at most
    if (pages > p.pt_stride) pages = p.pt_stride;
    const Shape f = shape_of(State::BLOCK, segments, pages, sm_count);
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

}  // namespace skv
