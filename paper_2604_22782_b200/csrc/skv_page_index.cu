// The page index (skv_index_pages): of every full page and kv head the highest and the lowest value of each dim of its 16
// keys, in steps of a 127th of the largest of them, and that step -- what skv_select_pages scores a page by.
//
// A warp takes one (page, kv head).  bf16 pages: the K half is one bulk copy; a lane then holds 8 dims (a chunk) of some of the
// tokens, in an order of the tokens that differs from lane to lane so that no two lanes of a shared-memory access are in one bank, and
// keeps highest and lowest as packed bf16.  FP8 pages: the codes times the tokens' scales in fp32, 16 dims a lane.  Bound by HBM
// in prompts (a page's K is read once, 1/16 as much is written), by the launch in a decode step, in which one
// sequence in 16 fills a page.
// Measured: 8 prompts of 4096 tokens, 8 heads of 128, 15 us (4.8 TB/s; some 4 us are the launch and the first copies), a step of 64 sequences
// 2.6 us, 23 ragged chunks on FP8 pages 12.7 us: 12000 pages and heads of 540 instructions are 6 us of issue, which a scheduler has in half of its
// busy cycles; warps wait for shared memory and its exchanges, at the barriers around the list, and the start is a launch and three dependent trips.
#include "skv_common.cuh"
#include "skv_page_index.cuh"

namespace skv {

namespace {

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int WARPS = 8;

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float min_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float min3_nan(float a, float b, float c)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// What a lane has in the end: highest and lowest of N dims in a row, from dim d on.
template <int N>
struct Ends { float hi[N], lo[N]; int d; };

// blk: [D/8 chunks of 8 dims][16 tokens][16 B].  A lane keeps a chunk over some of the tokens; lanes that have the same chunk then
// share its dims among them.
template <int D>
__device__ __forceinline__ Ends<D / 32> ends_of_bf16(uint32_t blk, int lane)
{
    constexpr int CH = D / 8, PARTS = 32 / CH, TP = PAGE / PARTS;
    const int c = lane % CH, part = lane / CH;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < TP; ++i) {
        const int t = part * TP + ((i + c) & (TP - 1));
        uint32_t x[4];
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(blk + (uint32_t)((c * PAGE + t) * 16)) : "memory");
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            hi[k] = i ? max_bf16x2(hi[k], x[k]) : x[k];
            lo[k] = i ? min_bf16x2(lo[k], x[k]) : x[k];
        }
    }
    // half of the words go to the lane with the other tokens, for half of its
    const bool upper = part & 1;
    uint32_t h[2], l[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        h[k] = max_bf16x2(upper ? hi[2 + k] : hi[k], __shfl_xor_sync(FULL, upper ? hi[k] : hi[2 + k], CH));
        l[k] = min_bf16x2(upper ? lo[2 + k] : lo[k], __shfl_xor_sync(FULL, upper ? lo[k] : lo[2 + k], CH));
    }
    Ends<D / 32> e;
    e.d = 8 * c + (upper ? 4 : 0);
    if constexpr (PARTS == 4) {
        const bool top = part & 2;
        h[0] = max_bf16x2(top ? h[1] : h[0], __shfl_xor_sync(FULL, top ? h[0] : h[1], 2 * CH));
        l[0] = min_bf16x2(top ? l[1] : l[0], __shfl_xor_sync(FULL, top ? l[0] : l[1], 2 * CH));
        e.d += top ? 2 : 0;
    }
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
        e.hi[2 * k] = bf16_lo(h[k]);
        e.hi[2 * k + 1] = bf16_hi(h[k]);
        e.lo[2 * k] = bf16_lo(l[k]);
        e.lo[2 * k + 1] = bf16_hi(l[k]);
    }
    return e;
}

// blk: K codes [2 groups of 8 tokens][D/16 chunks of 16 dims][8 tokens][16 B], then the tokens' scales
template <int D>
__device__ __forceinline__ Ends<D / 32> ends_of_fp8(uint32_t blk, int lane)
{
    constexpr int CH = D / 16, PARTS = 32 / CH, TP = PAGE / PARTS;
    const int c = lane % CH, part = lane / CH;
    float hi[16], lo[16];
    // two tokens at a time: highest and lowest then take an instruction each for both (of three inputs), the products one for a pair of dims
    static_assert(TP % 2 == 0, "a lane has an even number of tokens");
#pragma unroll
    for (int i = 0; i < TP; i += 2) {
        uint32_t x[2][4];
        float s[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int t = part * TP + i + m;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x[m][0]), "=r"(x[m][1]), "=r"(x[m][2]), "=r"(x[m][3]) : "r"(blk + (uint32_t)fp8_k_pos(D, t, 16 * c)) : "memory");
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(s[m]) : "r"(blk + (uint32_t)(PAGE * D + t * 4)) : "memory");
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float v[2][4];                             // [token][dim]
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                uint32_t w[2];
                e4m3x4_to_f16x2(x[m][k], w[0], w[1]);
#pragma unroll
                for (int q = 0; q < 2; ++q)
                    asm("{\n\t.reg .b16 u, v;\n\t.reg .f32 a, b;\n\t.reg .b64 p, t;\n\tmov.b32 {u, v}, %2;\n\tcvt.f32.f16 a, u;\n\tcvt.f32.f16 b, v;\n\t"
                        "mov.b64 p, {a, b};\n\tmov.b64 t, {%3, %3};\n\tmul.rn.f32x2 p, p, t;\n\tmov.b64 {%0, %1}, p;\n\t}"
                        : "=f"(v[m][2 * q]), "=f"(v[m][2 * q + 1]) : "r"(w[q]), "f"(s[m]));
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                hi[4 * k + d] = i ? max3_nan(hi[4 * k + d], v[0][d], v[1][d]) : max_nan(v[0][d], v[1][d]);
                lo[4 * k + d] = i ? min3_nan(lo[4 * k + d], v[0][d], v[1][d]) : min_nan(v[0][d], v[1][d]);
            }
        }
    }
    Ends<D / 32> e;
    e.d = 16 * c;
    // from exchange to exchange half as many dims
#pragma unroll
    for (int x = 1, n = 8; x < PARTS; x <<= 1, n >>= 1) {
        const bool upper = part & x;
#pragma unroll
        for (int d = 0; d < n; ++d) {
            hi[d] = max_nan(upper ? hi[n + d] : hi[d], __shfl_xor_sync(FULL, upper ? hi[d] : hi[n + d], x * CH));
            lo[d] = min_nan(upper ? lo[n + d] : lo[d], __shfl_xor_sync(FULL, upper ? lo[d] : lo[n + d], x * CH));
        }
        e.d += upper ? n : 0;
    }
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
        e.hi[d] = hi[d];
        e.lo[d] = lo[d];
    }
    return e;
}

// Codes and scale of one (page, kv head) from a warp's ends
template <int D>
__device__ __forceinline__ void write_entry(const Ends<D / 32> &e, int8_t *codes, float *scale, int lane)
{
    constexpr int N = D / 32;
    uint32_t top = 0;                                  // largest |x| as bits: they order as the values do, and those of a NaN are above all
#pragma unroll
    for (int d = 0; d < N; ++d) top = max(top, max(__float_as_uint(e.hi[d]) & 0x7FFFFFFFu, __float_as_uint(e.lo[d]) & 0x7FFFFFFFu));
    top = __reduce_max_sync(FULL, top);
    const float amax = __uint_as_float(top);
    const bool wild = top >= 0x7F800000u, none = !wild && amax < INDEX_TINY;
    const float inv = wild || none ? 0.f : __fdiv_rn(127.f, amax);
    if (lane == 0) *scale = wild ? __uint_as_float(0x7F800000u) : none ? 0.f : __fdiv_rn(amax, 127.f);
    uint32_t h = 0, l = 0;
#pragma unroll
    for (int m = 0; m < N; ++m) {                      // (at most 127: the product rounds to 127 at most)
        h |= ((uint32_t)(wild || none ? 0 : __float2int_rn(e.hi[m] * inv)) & 0xFFu) << (8 * m);
        l |= ((uint32_t)(wild || none ? 0 : __float2int_rn(e.lo[m] * inv)) & 0xFFu) << (8 * m);
    }
    if constexpr (N == 4) {
        *reinterpret_cast<uint32_t *>(codes + e.d) = h;
        *reinterpret_cast<uint32_t *>(codes + D + e.d) = l;
    } else {
        *reinterpret_cast<uint16_t *>(codes + e.d) = (uint16_t)h;
        *reinterpret_cast<uint16_t *>(codes + D + e.d) = (uint16_t)l;
    }
}

// Copies a warp has under way, and CTAs to an SM: some 200 KB of an SM's memory.  (With two copies of 2 KB a warp, a chunk's FP8 pages took 16 us.)
template <int D, bool FP8>
struct Ring {
    static constexpr int BYTES = FP8 ? PAGE * D + PAGE * 4 : half_bytes(D);
    static constexpr int STAGES = BYTES > 2200 ? 2 : 4, CTAS = 3;
    static constexpr size_t SMEM = WARPS * STAGES * ((size_t)BYTES + 8);
};

template <int D, bool FP8>
__global__ void __launch_bounds__(WARPS * 32, 3) index_pages_kernel(const __grid_constant__ IndexParams p)
{
    using R = Ring<D, FP8>;
    constexpr int BYTES = R::BYTES, ST = R::STAGES;
    extern __shared__ __align__(128) uint8_t smem_raw[];       // [WARPS][ST] blocks, then [WARPS][ST] barriers
    __shared__ int2 list[WARPS * 32];                          // page id and kv head of what there is to do
    __shared__ int counts[WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t ring = smem_u32(smem_raw) + (uint32_t)(warp * ST * BYTES), bars = smem_u32(smem_raw) + (uint32_t)(WARPS * ST * BYTES + warp * ST * 8);
    if (lane == 0) {
        for (int i = 0; i < ST; ++i) mbar_init(bars + 8 * i, 1);
        fence_barrier_init();
    }
    __syncwarp();
    pdl_wait();
    pdl_trigger();
    // Items are (sequence, page among those that its new tokens can fill, kv head); a CTA's are `gridDim.x` apart, so that every CTA has about
    // as many that are there, whatever the sequences' lengths.  A thread finds out about one; the warps take in turn what is found.
    const int64_t items = (int64_t)p.B * p.max_new_pages * p.Hkv;
    uint32_t sent = 0, done = 0;                       // this warp's copies; number n goes to stage n % ST
    for (int64_t i0 = blockIdx.x; i0 < items; i0 += (int64_t)gridDim.x * (WARPS * 32)) {
        const int64_t item = i0 + (int64_t)threadIdx.x * gridDim.x;
        int id = -1, h = 0;
        if (item < items) {
            const int64_t place = item / p.Hkv;
            h = (int)(item - place * p.Hkv);
            const int b = (int)(place / p.max_new_pages), j = (int)(place - (int64_t)b * p.max_new_pages);
            const int n = __ldg(p.seq_lens + b), first = p.cu_q ? __ldg(p.cu_q + b) : 0, a = p.cu_q ? __ldg(p.cu_q + b + 1) - first : 1;
            if (!p.cu_q && n <= 0) {
            } else if ((int64_t)n > (int64_t)p.pt_stride * PAGE || first < 0 || a < 0 || a > n || a > p.max_q_len) {
                if (h == 0 && j == 0) atomicOr(p.status, STATUS_BOUNDS);
            } else if ((n - a) / PAGE + j < n / PAGE) {
                id = __ldg(p.page_table + (int64_t)b * p.pt_stride + (n - a) / PAGE + j);
                if (id < 0 || (int64_t)id >= p.max_pages) {
                    atomicOr(p.status, STATUS_BOUNDS);
                    id = -1;
                }
            }
        }
        const unsigned there = __ballot_sync(FULL, id >= 0);
        if (lane == 0) counts[warp] = __popc(there);
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            before += w < warp ? counts[w] : 0;
            all += counts[w];
        }
        if (id >= 0) list[before + __popc(there & ((1u << lane) - 1))] = make_int2(id, h);
        __syncthreads();
        auto send = [&](int x) {                       // the list's entry x, by one lane
            if (lane == 0) {
                const int2 at = list[x];
                const uint8_t *src = p.layer_base + (int64_t)at.x * p.page_stride + (int64_t)at.y * (FP8 ? fp8_block_bytes(D) : block_bytes(D));
                const uint32_t dst = ring + (sent % ST) * BYTES, bar = bars + 8 * (sent % ST);
                mbar_expect_tx(bar, BYTES);
                if (FP8) {
                    bulk_copy_g2s(dst, src, PAGE * D, bar);
                    bulk_copy_g2s(dst + PAGE * D, src + fp8_ks_off(D), PAGE * 4, bar);
                } else {
                    bulk_copy_g2s(dst, src, BYTES, bar);
                }
            }
            ++sent;
        };
        for (int i = 0; i < ST && warp + i * WARPS < all; ++i) send(warp + i * WARPS);
        bool ok = true;
#pragma unroll 1
        for (int x = warp; x < all && ok; x += WARPS) {
            const uint32_t st = done % ST;
            ok = __all_sync(FULL, mbar_wait_bounded(bars + 8 * st, done / ST & 1u));
            if (!ok) break;
            ++done;
            const Ends<D / 32> e = FP8 ? ends_of_fp8<D>(ring + st * BYTES, lane) : ends_of_bf16<D>(ring + st * BYTES, lane);
            __syncwarp();                              // (the stage may be filled again)
            if (x + ST * WARPS < all) send(x + ST * WARPS);
            const int64_t at = (int64_t)list[x].x * p.Hkv + list[x].y;
            write_entry<D>(e, p.codes + at * 2 * D, p.scales + at, lane);
        }
        if (!__syncthreads_and(ok)) {                  // (the list is also free again)
            if (!ok && lane == 0) atomicOr(p.status, STATUS_TIMEOUT);
            // the copies under way get their time before the shared memory goes away
            for (uint32_t n = done; n != sent; ++n) mbar_wait_bounded(bars + 8 * (n % ST), n / ST & 1u);
            return;
        }
    }
}

}  // namespace

namespace {
template <int D, bool FP8>
cudaError_t launch_t(const IndexParams &p, int sm_count, bool pdl, cudaStream_t s)
{
    const size_t smem = Ring<D, FP8>::SMEM;
    const int64_t items = (int64_t)p.B * p.max_new_pages * p.Hkv, most = (int64_t)sm_count * Ring<D, FP8>::CTAS;
    const int64_t ctas = (items + WARPS - 1) / WARPS < most ? (items + WARPS - 1) / WARPS : most;
    auto kern = index_pages_kernel<D, FP8>;
    const cudaError_t e = ensure_dynamic_smem(kern, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(WARPS * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, p);
}
}  // namespace

cudaError_t launch_index_pages(const IndexParams &p, int D, bool fp8, int sm_count, bool pdl, cudaStream_t s)
{
    if (D == 128) return fp8 ? launch_t<128, true>(p, sm_count, pdl, s) : launch_t<128, false>(p, sm_count, pdl, s);
    if (D == 64) return fp8 ? launch_t<64, true>(p, sm_count, pdl, s) : launch_t<64, false>(p, sm_count, pdl, s);
    return cudaErrorInvalidValue;
}

}  // namespace skv
