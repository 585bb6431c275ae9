// Pieces of the chunk attention kernels on the 5th-generation tensor cores (skv_prefill_window.cu, skv_prefill_pages.cu).
#pragma once
#include "skv_common.cuh"
#include "skv_tcgen05.cuh"

#include <cuda.h>
#include <math.h>

namespace skv {
namespace chunk {

constexpr float RESCALE_STEP = 8.f;   // the softmax's reference maximum moves when it has grown by more than 2^8

__host__ __device__ constexpr uint32_t instr_desc(int M, int N, bool b_mn_major)
{
    return (1u << 4) /* D fp32 */ | (1u << 7) /* A bf16 */ | (1u << 10) /* B bf16 */ |
           ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// By a whole warp.  Bounded, by a number of tries (some seconds).  A wait that runs out raises gave_up; everybody's waits
// then end after a few tries, and the CTA runs through to its end on whatever it finds, which stays inside its buffers.
// As small a loop as it gets and nothing to ask afterwards: with a clock read in it, and a vote and a branch on the outcome
// after it, a wait that was already over cost 340 cycles, several of them per tile and block.
__device__ __forceinline__ void wait(uint32_t bar, uint32_t parity, volatile uint32_t *gave_up)
{
#pragma unroll 1
    for (uint32_t n = 1; !mbar_try_wait(bar, parity); ++n)
        if ((n & 255u) == 0 && (n >> 24 || *gave_up)) {
            *gave_up = 1;
            break;
        }
    __syncwarp();
}

// operand rows of 128 bytes in the 128-byte swizzle, groups of 8 rows 1024 bytes apart
__device__ __forceinline__ uint64_t swizzled_desc(uint32_t saddr)
{
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// K half of page `page`, kv head `h`
__device__ __forceinline__ void tensor_copy_k(uint32_t dst, const CUtensorMap *map, int h, int page, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(0), "r"(h), "r"(page), "r"(bar)
                 : "memory");
}

// a pair of fp32 in one 64-bit register: one instruction works on both
__device__ __forceinline__ uint64_t pair_of(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void halves(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float ex2(float x)          // (fast_exp2 without its place in the order of volatile instructions)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// one lane of the warp, the same one every time
__device__ __forceinline__ bool elect_one()
{
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}

template <int REGS>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS)); }
template <int REGS>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS)); }

// K halves of an owner layer's pages as a tensor: [page][head][2 groups of 8 tokens][D/8 chunks][8 tokens x 8 dims]; a box is one
// page's half of one head.  (The encoder is the driver's; asked for through the runtime, nothing is linked.)
inline bool encode_k_map(CUtensorMap *map, const uint8_t *layer_base, int64_t page_stride, int64_t max_pages, int Hkv, int D)
{
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    if (!encode) return false;
    const cuuint64_t dims[5] = {64, (cuuint64_t)(D / 8), 2, (cuuint64_t)Hkv, (cuuint64_t)max_pages};
    const cuuint64_t strides[4] = {256, 128, (cuuint64_t)block_bytes(D), (cuuint64_t)page_stride};
    const cuuint32_t box[5] = {64, (cuuint32_t)(D / 8), 2, 1, 1}, steps[5] = {1, 1, 1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<uint8_t *>(layer_base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace chunk
}  // namespace skv
