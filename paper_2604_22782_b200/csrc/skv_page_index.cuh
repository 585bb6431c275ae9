// The page index of a cache and the lists of selected pages: parameter blocks and launchers.
//
// The index of one owner layer: codes int8 [max_pages][kv heads][highest | lowest][D], padded to 256 bytes, then scales
// fp32 [max_pages][kv heads], padded to 256 bytes.  An entry belongs to a physical page, as its keys do, so pages that sequences
// share have one entry.
#pragma once
#include "skv_common.cuh"

namespace skv {

constexpr float INDEX_TINY = 7.888609052210118e-31f;       // 2^-100: a page or query whose largest element is below counts as zero

__host__ __device__ inline int64_t index_codes_bytes(int64_t max_pages, int Hkv, int D) { return (max_pages * Hkv * 2 * D + 255) / 256 * 256; }
__host__ __device__ inline int64_t index_layer_bytes(int64_t max_pages, int Hkv, int D)
{
    return index_codes_bytes(max_pages, Hkv, D) + (max_pages * Hkv * 4 + 255) / 256 * 256;
}

// Rows of a run, of which `left` are there.  As an instruction of its own: written as a comparison, the lesser of the two came out as
// run in kernels that take it from a __grid_constant__ parameter (nvcc 12.9.86, whole kernels only, not where the value was also printed), and
// rows behind the last were read and written.  No small kernel shows it, so that its cause is not known; the tests' guard rows hold it down.
__device__ __forceinline__ int rows_of_run(int left, int run)
{
    int r;
    asm volatile("min.s32 %0, %1, %2;" : "=r"(r) : "r"(left), "r"(run));
    return r;
}

struct IndexParams {
    const uint8_t *layer_base;  // first page of the owner layer
    int64_t page_stride;
    int64_t max_pages;
    const int32_t *page_table;  // [B][pt_stride]
    const int32_t *seq_lens;    // [B] cached tokens including the new ones
    const int32_t *cu_q;        // [B+1] as in PrefillParams, or null: one new token per sequence
    int B, Hkv, pt_stride, max_q_len;
    int max_new_pages;          // pages that max_q_len new tokens fill at most
    int8_t *codes;              // the layer's part of the index
    float *scales;
    int *status;
};

struct SelectParams {
    const int8_t *codes;
    const float *scales;
    int64_t max_pages;
    const uint16_t *Q;          // rows [Hq][D] bf16 bits
    const int32_t *page_table;
    const int32_t *seq_lens;
    const int32_t *cu_q;        // null: one row per sequence
    int32_t *lists;             // [B * per_seq][Hkv][stride]
    int32_t *counts;            // [B * per_seq][Hkv]
    int B, Hq, Hkv, pt_stride, max_q_len;
    int run, per_seq;           // rows that share a list; lists of a sequence
    int top, first, last;
    int stride;
    int most;                   // pages that a list's score can be asked of, at most
    int *status;
};

// Lists that an attention call reads.
struct PageLists {
    const int32_t *lists;       // [B * per_seq][Hkv][stride]
    const int32_t *counts;      // [B * per_seq][Hkv]
    int stride;
    int run, per_seq;
};

cudaError_t launch_index_pages(const IndexParams &p, int D, bool fp8, int sm_count, bool pdl, cudaStream_t s);
int select_max_pages(int columns);      // of a sequence; columns: min(run, max_q_len) * G
cudaError_t launch_select_pages(const SelectParams &p, int D, int sm_count, bool pdl, cudaStream_t s);
// decode attention over listed pages (skv_decode_pages.cu); kernel as in launch_decode_splitk.  p.cu_q: rows of chunks, a row as a
// sequence of its own (p.B = sequences * p.max_q_len)
cudaError_t launch_decode_pages(const DecodeParams &p, const PageLists &l, int D, int G, int kernel, int sm_count, bool pdl, cudaStream_t s);
// chunk attention over listed pages on the tensor cores (skv_prefill_pages.cu): min(run, max_q_len) * G <= 128
size_t prefill_pages_smem_bytes(int D, bool fp8);
int prefill_pages_parts(int64_t lists, int pages, int sm_count);         // CTAs that share a list
cudaError_t launch_prefill_pages(const PrefillParams &p, const PageLists &l, int D, int G, int max_q_len, bool fp8, int sm_count, bool pdl, cudaStream_t s);

}  // namespace skv
