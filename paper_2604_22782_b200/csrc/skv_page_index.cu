// The page index (skv_index_pages): of every full page and kv head the highest and the lowest value of each dim of its 16
// keys, in steps of a 127th of the largest of them, and that step -- what skv_select_pages scores a page by.
//
// A warp takes one (page, kv head).  bf16 pages: the K half is one bulk copy; a lane then holds 8 dims (a chunk) of some of the
// tokens, in an order of the tokens that differs from lane to lane so that no two lanes of a shared-memory access are in one bank, and
// keeps highest and lowest as packed bf16.  FP8 pages: the codes times the tokens' scales in fp32, 16 dims a lane.  Bound by HBM
// in prompts (a page's K is read once, 1/16 as much is written), by the launch in a decode step, in which one
// sequence in 16 fills a page.
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

// dims of one lane: N highest and N lowest, the same in all lanes of a group that differ only in their tokens
template <int N>
struct Ends { float hi[N], lo[N]; };

template <int D>
__device__ __forceinline__ Ends<8> ends_of_bf16(const uint8_t *blk, int lane)
{
    constexpr int CH = D / 8, PARTS = 32 / CH, TP = PAGE / PARTS;
    const int c = lane % CH, part = lane / CH;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < TP; ++i) {
        const int t = part * TP + ((i + c) & (TP - 1));
        const uint4 w = *reinterpret_cast<const uint4 *>(blk + (c * PAGE + t) * 16);
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            hi[k] = i ? max_bf16x2(hi[k], x[k]) : x[k];
            lo[k] = i ? min_bf16x2(lo[k], x[k]) : x[k];
        }
    }
#pragma unroll
    for (int d = CH; d < 32; d <<= 1)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            hi[k] = max_bf16x2(hi[k], __shfl_xor_sync(FULL, hi[k], d));
            lo[k] = min_bf16x2(lo[k], __shfl_xor_sync(FULL, lo[k], d));
        }
    Ends<8> e;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        e.hi[2 * k] = bf16_lo(hi[k]);
        e.hi[2 * k + 1] = bf16_hi(hi[k]);
        e.lo[2 * k] = bf16_lo(lo[k]);
        e.lo[2 * k + 1] = bf16_hi(lo[k]);
    }
    return e;
}

// blk: K codes [2 groups of 8 tokens][D/16 chunks][8 tokens][16 B], then the tokens' scales
template <int D>
__device__ __forceinline__ Ends<16> ends_of_fp8(const uint8_t *blk, int lane)
{
    constexpr int CH = D / 16, PARTS = 32 / CH, TP = PAGE / PARTS;
    const int c = lane % CH, part = lane / CH;
    const float *scales = reinterpret_cast<const float *>(blk + PAGE * D);
    Ends<16> e;
#pragma unroll
    for (int i = 0; i < TP; ++i) {
        const int t = part * TP + i;
        const uint4 w = *reinterpret_cast<const uint4 *>(blk + fp8_k_pos(D, t, 16 * c));
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
        const float s = scales[t];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t h[2];
            e4m3x4_to_f16x2(x[k], h[0], h[1]);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                float a, b;
                asm("{\n\t.reg .b16 u, v;\n\tmov.b32 {u, v}, %2;\n\tcvt.f32.f16 %0, u;\n\tcvt.f32.f16 %1, v;\n\t}" : "=f"(a), "=f"(b) : "r"(h[m]));
                const int d = 4 * k + 2 * m;
                a *= s;
                b *= s;
                e.hi[d] = i ? max_nan(e.hi[d], a) : a;
                e.lo[d] = i ? min_nan(e.lo[d], a) : a;
                e.hi[d + 1] = i ? max_nan(e.hi[d + 1], b) : b;
                e.lo[d + 1] = i ? min_nan(e.lo[d + 1], b) : b;
            }
        }
    }
#pragma unroll
    for (int x = CH; x < 32; x <<= 1)
#pragma unroll
        for (int d = 0; d < 16; ++d) {
            e.hi[d] = max_nan(e.hi[d], __shfl_xor_sync(FULL, e.hi[d], x));
            e.lo[d] = min_nan(e.lo[d], __shfl_xor_sync(FULL, e.lo[d], x));
        }
    return e;
}

// Codes and scale of one (page, kv head) from a warp's ends; c: which N dims the lane has, part: which of the lanes that have them
template <int D, int N>
__device__ __forceinline__ void write_entry(const Ends<N> &e, int c, int part, int8_t *codes, float *scale, int lane)
{
    uint32_t top = 0;                                  // largest |x| as bits: they order as the values do, and those of a NaN are above all
#pragma unroll
    for (int d = 0; d < N; ++d) {
        const uint32_t a = __float_as_uint(e.hi[d]) & 0x7FFFFFFFu, b = __float_as_uint(e.lo[d]) & 0x7FFFFFFFu;
        top = max(top, max(a, b));
    }
    top = __reduce_max_sync(FULL, top);
    const float amax = __uint_as_float(top);
    const bool wild = top >= 0x7F800000u, none = !wild && amax < INDEX_TINY;
    const float inv = wild || none ? 0.f : __fdiv_rn(127.f, amax);
    if (lane == 0) *scale = wild ? __uint_as_float(0x7F800000u) : none ? 0.f : __fdiv_rn(amax, 127.f);
    if (part < 2) {
        uint32_t w[N / 4];
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            w[k] = 0;
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                const float x = part ? e.lo[4 * k + m] : e.hi[4 * k + m];
                const int q = wild || none ? 0 : __float2int_rn(x * inv);      // (at most 127: the product rounds to 127 at most)
                w[k] |= ((uint32_t)q & 0xFFu) << (8 * m);
            }
        }
        int8_t *dst = codes + part * D + c * N;
        if (N == 16) *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[N / 4 - 2], w[N / 4 - 1]);
        else *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
    }
}

template <int D, bool FP8>
__global__ void __launch_bounds__(WARPS * 32) index_pages_kernel(IndexParams p)
{
    constexpr int BYTES = FP8 ? PAGE * D + PAGE * 4 : half_bytes(D);
    __shared__ __align__(128) uint8_t blocks[WARPS][BYTES];
    __shared__ __align__(8) unsigned long long bars[WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t bar = smem_u32(&bars[warp]);
    if (lane == 0) {
        mbar_init(bar, 1);
        fence_barrier_init();
    }
    __syncwarp();
    pdl_wait();
    pdl_trigger();
    // (sequence, page among those that its new tokens can fill, kv head)
    const int64_t item = (int64_t)blockIdx.x * WARPS + warp;
    const int64_t place = item / p.Hkv;
    const int h = (int)(item - place * p.Hkv), b = (int)(place / p.max_new_pages), j = (int)(place - (int64_t)b * p.max_new_pages);
    if (b >= p.B) return;
    const int n = __ldg(p.seq_lens + b), first = p.cu_q ? __ldg(p.cu_q + b) : 0, a = p.cu_q ? __ldg(p.cu_q + b + 1) - first : 1;
    if (!p.cu_q && n <= 0) return;
    if ((int64_t)n > (int64_t)p.pt_stride * PAGE || first < 0 || a < 0 || a > n || a > p.max_q_len) {
        if (h == 0 && j == 0 && lane == 0) atomicOr(p.status, STATUS_BOUNDS);
        return;
    }
    const int page = (n - a) / PAGE + j;
    if (page >= n / PAGE) return;
    const int id = __ldg(p.page_table + (int64_t)b * p.pt_stride + page);
    if (id < 0 || (int64_t)id >= p.max_pages) {
        if (lane == 0) atomicOr(p.status, STATUS_BOUNDS);
        return;
    }
    const uint8_t *src = p.layer_base + (int64_t)id * p.page_stride + (int64_t)h * (FP8 ? fp8_block_bytes(D) : block_bytes(D));
    if (lane == 0) {
        mbar_expect_tx(bar, BYTES);
        if (FP8) {
            bulk_copy_g2s(smem_u32(blocks[warp]), src, PAGE * D, bar);
            bulk_copy_g2s(smem_u32(blocks[warp]) + PAGE * D, src + fp8_ks_off(D), PAGE * 4, bar);
        } else {
            bulk_copy_g2s(smem_u32(blocks[warp]), src, BYTES, bar);
        }
    }
    __syncwarp();
    if (!__all_sync(FULL, mbar_wait_bounded(bar, 0))) {
        if (lane == 0) atomicOr(p.status, STATUS_TIMEOUT);
        mbar_wait_bounded(bar, 0);                     // (the copy gets its time before the shared memory goes away)
        return;
    }
    const int64_t entry = (int64_t)id * p.Hkv + h;
    int8_t *codes = p.codes + entry * 2 * D;
    if (FP8) {
        const Ends<16> e = ends_of_fp8<D>(blocks[warp], lane);
        write_entry<D, 16>(e, lane % (D / 16), lane / (D / 16), codes, p.scales + entry, lane);
    } else {
        const Ends<8> e = ends_of_bf16<D>(blocks[warp], lane);
        write_entry<D, 8>(e, lane % (D / 8), lane / (D / 8), codes, p.scales + entry, lane);
    }
}

}  // namespace

cudaError_t launch_index_pages(const IndexParams &p, int D, bool fp8, bool pdl, cudaStream_t s)
{
    const int64_t warps = (int64_t)p.B * p.max_new_pages * p.Hkv, ctas = (warps + WARPS - 1) / WARPS;
    if (ctas > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(WARPS * 32);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 1 : 0;
    if (D == 128) return fp8 ? cudaLaunchKernelEx(&cfg, index_pages_kernel<128, true>, p) : cudaLaunchKernelEx(&cfg, index_pages_kernel<128, false>, p);
    if (D == 64) return fp8 ? cudaLaunchKernelEx(&cfg, index_pages_kernel<64, true>, p) : cudaLaunchKernelEx(&cfg, index_pages_kernel<64, false>, p);
    return cudaErrorInvalidValue;
}

}  // namespace skv
