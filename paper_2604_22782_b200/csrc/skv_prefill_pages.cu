// Attention of chunks over listed pages (skv_prefill_attn_pages) on the 5th-generation tensor cores: the row at position pos
// attends the tokens t <= pos of the pages that its run's list names for the kv head.
//
// An item is a list: (sequence, run of rows, kv head), one tile of 128 query rows, row r = token r / G, head r % G.  Lists of
// neighbouring tiles differ, so tiles share no K and V read (as the windowed kernel's two do) and a CTA has one item.  Two CTAs
// share an SM, 256 or 384 threads, about 100 KB and 256 columns of tensor memory each: while one's softmax works the other's instructions
// do, and what an item's beginning and end leave idle the other CTA uses.  Keys go in blocks of 64, 4 listed pages.
// Warps 0-3 fetch the queries, then softmax: thread = row (TMEM lane).  The others, on bf16 pages:
//   warp 4     issues the scores Q K^T,  warp 5  the outputs P V
//   warp 6     copies K and V of the key blocks; the entries' page ids are had 32 at a time
//   warp 7     zeroes the V rows of tokens that no row of the item sees, whatever they hold
// On FP8 pages K's codes are the scores' operand as they are.  A query is the sum of two E4M3 numbers, times a power of two that brings a
// row's largest to [128, 256): the nearest, and the nearest to what that leaves, which hold bf16's 8 bits exactly, but for elements below
// 2^-9 of the largest, which may be off by 2^-17 of it.  V's codes are turned into f16, which holds every one of them exactly, on the way
// into the operand.  The tokens' scales are applied in fp32, K's to the scores and V's to the probabilities, which are taken relative to c,
// the power of two at or above every V scale that the row has seen, so that they fit f16 whatever the scales:
//   warps 4-7  convert V (tokens that no row sees: zero),  warp 8  scales, issues Q K^T,  9  P V,  warps 10, 11  copy K and V
// On bf16 pages probabilities are bf16, as both operands of the instruction are of V's type: 2^-8 of a weight at most, as in the other bf16 chunk
// kernels.  (A second term for the rest, as skv_decode_pages.cu has it, is not free here: half as much again for the tensor cores, and five
// instructions a pair for a softmax that waits for issue.)  Sums and references are fp32.
// Few lists leave SMs without one: then a cluster of CTAs shares a list, each has a part of its blocks, and their unnormalised outputs, with
// each row's reference and sum, are joined through shared memory, every CTA some of the dims (prefill_pages_parts has the figures).
// Operand layouts, softmax and waits are those of skv_prefill_window.cu, but for its exponentials on the FMA units: here the softmax waits for
// issue, not for the exponential's unit (every eighth pair, as there: 79.9 / 55.4 us below, none 79.3 / 54.2, every other 59.3 on FP8).  Runs of one sequence and head are neighbours in the grid:
// their lists have pages in common, which are then in L2.
// Measured, 8 kv heads of 128, 32 query heads: 2 x 1024 rows, 32 to a list of 126 pages, 79 us on bf16 pages, 0.85 PFLOP/s, in short loops (90 to 96, 0.72,
// in long ones, under the power limit); 4 chunks of 129 to 256 rows on FP8 pages 54 us.  Neither tensor cores (45 % and 31 %) nor shared memory (45 % and 62 %) are
// busy throughout: with two CTAs to an SM it is the chain copy, scores, softmax, P V, and 512 items in 296 places.
#include "skv_page_index.cuh"
#include "skv_prefill_parts.cuh"
#include "skv_segment.cuh"
#include "skv_tcgen05.cuh"

namespace skv {

namespace {

using namespace tc5;
using namespace chunk;

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int ROWS = 128;             // query rows of an item
constexpr int KB = 4;                 // pages of a key block
constexpr int KEYS = KB * PAGE;
__host__ __device__ constexpr int threads_of(bool fp8) { return fp8 ? 384 : 256; }
constexpr int COL_O = 2 * KEYS;       // scores at columns 0 and 64, output from 128 on
constexpr int TMEM_COLS = 256;
constexpr int MAX_PARTS = 8;          // CTAs that may share a list
constexpr int NO_PAGE = 0x07FFFFFF;   // no row sees a token of it

// Shared memory (from a 1024-byte boundary on).  bf16: Q [D/64][128 rows][128 B] | K ring [8 groups][D/8 chunks][8 keys][16 B] | V ring
// [4 pages][V half].  FP8: Q [128 rows][two terms][D dims], D = 128 the terms one after the other | two V tiles [4 pages][2 halves of
// 8 tokens][D dims][16 B] | K ring: codes of 4 pages [8 groups][D/16 chunks][8 keys][16 B], their K and V scales | V ring: codes | scales of
// 4 blocks: K scale x log2(e) / sqrt(d) [64] | V scale [64] | the largest V scale.  Then barriers and words.
template <int D, bool FP8>
struct Layout {
    static constexpr int STAGES = D == 128 ? 2 : 4;                  // bf16: of the K ring and of the V ring
    static constexpr int SCALE_STAGE = (2 * KEYS + 4) * 4;
    static constexpr int K_STAGES = FP8 ? 3 : STAGES, V_STAGES = FP8 ? 2 : STAGES;
    static constexpr int Q_BYTES = ROWS * D * 2, TILE = KEYS * D * 2;
    static constexpr int K_STAGE = FP8 ? KEYS * D + KB * 2 * PAGE * 4 : TILE, V_STAGE = FP8 ? KEYS * D : TILE;
    static constexpr int K_RING = Q_BYTES + (FP8 ? 2 * TILE : 0), V_RING = K_RING + K_STAGES * K_STAGE;
    static constexpr int SCALES = V_RING + V_STAGES * V_STAGE, BARS = SCALES + (FP8 ? 4 * SCALE_STAGE : 0);
    static constexpr int N_BARS = 2 * K_STAGES + 2 * V_STAGES + (FP8 ? 2 : V_STAGES) + 3 * 2 + 1;
    static constexpr int WORDS = BARS + 8 * N_BARS + (8 * N_BARS & 8);
    static constexpr int BYTES = 1024 + WORDS + 48;
};

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// 16 E4M3 codes -> two times 8 f16 (exact)
__device__ __forceinline__ void convert16(const uint4 &w, uint4 &a, uint4 &b)
{
    e4m3x4_to_f16x2(w.x, a.x, a.y);
    e4m3x4_to_f16x2(w.y, a.z, a.w);
    e4m3x4_to_f16x2(w.z, b.x, b.y);
    e4m3x4_to_f16x2(w.w, b.z, b.w);
}

__device__ __forceinline__ float2 f16x2_to_f32x2(uint32_t w)
{
    float2 f;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(w));
    return f;
}

// exponent of the power of two at or above x >= 0, at least LEAST_C: a probability of up to 2^8 over c stays far from fp32's end
constexpr int LEAST_C = -100;
__device__ __forceinline__ float ceil_log2(float x)
{
    const int e = (int)((__float_as_uint(x) + 0x007FFFFFu) >> 23) - 127;
    return (float)(e < LEAST_C ? LEAST_C : e);
}

__device__ __forceinline__ uint4 ld_shared(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void st_shared(uint32_t a, const uint4 &v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// zeros where it is not there
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t a, bool there)
{
    float4 v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.f32 %0, 0f00000000;\n\tmov.f32 %1, %0;\n\tmov.f32 %2, %0;\n\tmov.f32 %3, %0;\n\t"
                 "@p ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];\n\t}" : "=&f"(v.x), "=&f"(v.y), "=&f"(v.z), "=&f"(v.w) : "r"(a), "r"((int)there) : "memory");
    return v;
}

// Groups [first, last) of 8 dims of this thread's row from the parts of up to N CTAs, U groups at a time.  `mine`: the row's O in this CTA's shared
// memory, `sum` its reference and sum.
template <int N, int U>
__device__ __forceinline__ void join_parts(uint32_t mine, uint32_t sum, int parts, int first, int last, bool row_ok, uint16_t *dst)
{
    float w[N], top = -INFINITY, total = 0.f;
    float2 ml[N];
#pragma unroll
    for (int c = 0; c < N; ++c) ml[c] = ld_cluster_f2(at_rank(sum, (uint32_t)(c < parts ? c : 0)));
#pragma unroll
    for (int c = 0; c < N; ++c)
        if (c < parts) top = fmaxf(top, ml[c].x);
#pragma unroll
    for (int c = 0; c < N; ++c) {
        w[c] = c >= parts ? 0.f : ml[c].x == top ? 1.f : ex2(ml[c].x - top);       // (1 too where all are -inf: nothing seen, or only NaN)
        total = fmaf(w[c], c < parts ? ml[c].y : 0.f, total);
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll 1
    for (int u0 = first; u0 < last; u0 += U) {
        float4 x[U][N][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < N; ++c)
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    x[u][c][half] = ld_cluster_f4(at_rank(mine, (uint32_t)(c < parts ? c : 0)) + (uint32_t)((2 * (u0 + u) + half) * ROWS * 16), c < parts && u0 + u < last);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t y[4];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int c = 0; c < N; ++c) {
                    a.x = fmaf(w[c], x[u][c][half].x, a.x);
                    a.y = fmaf(w[c], x[u][c][half].y, a.y);
                    a.z = fmaf(w[c], x[u][c][half].z, a.z);
                    a.w = fmaf(w[c], x[u][c][half].w, a.w);
                }
                y[2 * half] = pack_bf16x2(a.x * inv, a.y * inv);
                y[2 * half + 1] = pack_bf16x2(a.z * inv, a.w * inv);
            }
            if (row_ok && u0 + u < last) *reinterpret_cast<uint4 *>(dst + 8 * (u0 + u)) = make_uint4(y[0], y[1], y[2], y[3]);
        }
    }
}

// the tokens of page `page` (NO_PAGE: none) up to position pos
__device__ __forceinline__ uint32_t bits_up_to(int pos, int page)
{
    const int left = pos + 1 - page * PAGE;
    return (1u << (left < 0 ? 0 : left < PAGE ? left : PAGE)) - 1;
}

template <int D, bool FP8>
__global__ void __launch_bounds__(threads_of(FP8), 2) prefill_pages_kernel(const __grid_constant__ PrefillParams p, const __grid_constant__ PageLists l,
                                                                      const __grid_constant__ CUtensorMap k_map, int G, int max_q_len)
{
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    using L = Layout<D, FP8>;
    constexpr int THREADS = threads_of(FP8);
    constexpr int BLOCK = FP8 ? fp8_block_bytes(D) : block_bytes(D), HALF = half_bytes(D), CH = D / 8, KS = L::K_STAGES, VS = L::V_STAGES;
    constexpr uint32_t F16 = FP8 ? (1u << 7) | (1u << 10) : 0u;              // the operands' type bits of P V: bf16, or neither
    constexpr uint32_t IDESC_QK = FP8 ? instr_desc_e4m3(ROWS, KEYS) : instr_desc(ROWS, KEYS, false), IDESC_PV = instr_desc(ROWS, D, !FP8) & ~F16;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);      // (known to be the same for the warp)
    const uint32_t base = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
    const uint32_t q_smem = base + pad, v_tiles = q_smem + L::Q_BYTES, k_ring = q_smem + L::K_RING, v_ring = q_smem + L::V_RING,
                   scale_ring = q_smem + L::SCALES;
    const uint32_t k_full = q_smem + L::BARS, k_empty = k_full + 8 * KS, v_full = k_empty + 8 * KS, v_empty = v_full + 8 * VS;
    // bf16: a V stage with tokens that nobody sees has landed; FP8: a V tile is complete
    const uint32_t v_landed = v_empty + 8 * VS, v_ready = v_landed;
    const uint32_t s_ready = v_landed + 8 * (FP8 ? 2 : VS), p_ready = s_ready + 16, pv_done = p_ready + 16, q_full = pv_done + 16;
    uint8_t *words = smem_raw + pad + L::WORDS;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(words), *gave_up = tmem_slot + 1;
    volatile int32_t *item = reinterpret_cast<volatile int32_t *>(words + 8);      // rows, first position, tokens of the sequence, first row, entries

    if (tid == 0) {
        for (int i = 0; i < KS; ++i) {
            mbar_init(k_full + 8 * i, 1);
            mbar_init(k_empty + 8 * i, 1);
        }
        for (int i = 0; i < VS; ++i) {
            mbar_init(v_full + 8 * i, 1);
            mbar_init(v_empty + 8 * i, FP8 ? 4 : 1);
            if (!FP8) mbar_init(v_landed + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            if (FP8) mbar_init(v_ready + 8 * i, 4);
            mbar_init(s_ready + 8 * i, FP8 ? 2 : 1);                         // (FP8: the block's scales are there too)
            mbar_init(p_ready + 8 * i, 4);
            mbar_init(pv_done + 8 * i, 1);
        }
        mbar_init(q_full, 4);
        *gave_up = 0;
        fence_barrier_init();
    }
    pdl_wait();
    uint32_t rank, ranks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    const int index = (int)(blockIdx.x / ranks), pair = index / l.per_seq, r = index - pair * l.per_seq, b = pair / p.Hkv, h = pair - b * p.Hkv;
    const int64_t list_no = ((int64_t)b * l.per_seq + r) * p.Hkv + h;
    // The item, worked out by one warp and handed over in shared memory.
    if (warp == 4) {
        const int q_begin = __ldg(p.cu_q + b), q_len = __ldg(p.cu_q + b + 1) - q_begin, n = __ldg(p.seq_lens + b);
        const int at = r * l.run;                                        // the run's first row (below max_q_len, since r < per_seq)
        int rows = 0, listed = 0;
        if (q_begin < 0 || q_len < 0 || q_len > n || q_len > max_q_len || (int64_t)n > (int64_t)p.pt_stride * PAGE) {
            if (r == 0 && h == 0 && lane == 0) atomicOr(p.status, STATUS_BOUNDS);
        } else if (at < q_len) {
            rows = rows_of_run(q_len - at, l.run);
            listed = __ldg(l.counts + list_no);
            if (listed > l.stride) {
                listed = l.stride;
                if (lane == 0) atomicOr(p.status, STATUS_BOUNDS);
            }
        }
        if (rows > 0 && ((int64_t)listed + KEYS / PAGE - 1) / KB > (int64_t)rank) {
            tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), TMEM_COLS);
            tmem_relinquish();
        }
        if (lane == 0) {
            item[0] = rows;
            item[1] = n - q_len + at;
            item[2] = n;
            item[3] = q_begin + at;
            item[4] = listed;
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // (by a shuffle: then they are known to be the same for the warp, and what is worked out from them stays in uniform registers, from
    // which the tensor core's instructions take their operands)
    auto shared = [&](int i) { return __shfl_sync(FULL, item[i], 0); };
    const int rows = shared(0), p0 = shared(1), p1 = p0 + rows - 1, pages = (shared(2) + PAGE - 1) / PAGE, all_listed = shared(4);
    const int64_t first_row = shared(3);
    const uint16_t *q_rows = p.Q + (first_row * p.Hq + (int64_t)h * G) * D;
    uint16_t *out_rows = p.out + (first_row * p.Hq + (int64_t)h * G) * D;
    if (rows <= 0) return;                     // (the whole cluster, here and where nothing is listed)
    if (all_listed <= 0) {
        for (int i = tid + (int)rank * THREADS; i < rows * G * (D / 4); i += THREADS * (int)ranks) {
            const int row = i / (D / 4), token = row / G;
            *reinterpret_cast<uint2 *>(out_rows + ((int64_t)token * p.Hq + row - token * G) * D + i % (D / 4) * 4) = make_uint2(0, 0);
        }
        return;
    }
    // Each of the cluster's CTAs has a part of the list's blocks; where there are fewer of these than CTAs, the last ones have none.
    const int all_blocks = (all_listed + KB - 1) / KB, parts = all_blocks < (int)ranks ? all_blocks : (int)ranks;
    if ((int)rank >= parts) {
        for (int i = 0; i < 2; ++i) {
            cluster_arrive();
            cluster_wait();
        }
        return;
    }
    const int from = (int)((int64_t)all_blocks * rank / parts), blocks = (int)((int64_t)all_blocks * (rank + 1) / parts) - from;
    const int listed = all_listed - from * KB < blocks * KB ? all_listed - from * KB : blocks * KB;
    const int32_t *entries = l.lists + list_no * l.stride + (int64_t)from * KB, *table = p.page_table + (int64_t)b * p.pt_stride;
    const uint32_t tmem = __shfl_sync(FULL, *tmem_slot, 0);
    // a listed page's number, NO_PAGE where it is none of the sequence's
    auto page_at = [&](int i) {
        const int page = i < listed ? __ldg(entries + i) : NO_PAGE;
        return page >= 0 && page < pages ? page : NO_PAGE;
    };
    // physical page of entry i; where there is none, one whose content is not looked at
    auto id_at = [&](int i) {
        if (i >= listed) return 0;
        const int page = page_at(i), id = page != NO_PAGE ? __ldg(table + page) : -1;
        if (id >= 0 && (int64_t)id < p.max_pages) return id;
        atomicOr(p.status, STATUS_BOUNDS);
        return 0;
    };

    if (warp < 4) {
        more_registers<FP8 ? 160 : 200>();
        // =================== queries ===================
        float row_scale = 0.f;                             // FP8: the power of two that was taken out of this thread's row
        {
            // 8 lanes a row of 128 bytes, a warp its 32 rows; rows that the item does not have are zero
            const int c = lane & 7;
#pragma unroll 1
            for (int i = 0; i < 8; ++i) {
                const int row = warp * 32 + i * 4 + (lane >> 3), token = row / G;
                const uint16_t *src = q_rows + ((int64_t)token * p.Hq + row - token * G) * D + c * 8;
                const uint32_t dst = q_smem + (uint32_t)(row * 128 + ((c ^ (row & 7)) * 16));
#pragma unroll
                for (int half = 0; half < D / 64; ++half) {
                    if (token < rows)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + (uint32_t)(half * ROWS * 128)), "l"(src + half * 64) : "memory");
                    else
                        st_shared(dst + (uint32_t)(half * ROWS * 128), make_uint4(0, 0, 0, 0));
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            if constexpr (FP8) {
                // a row's two terms take the place of its bf16 values
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {
                    const int row = warp * 32 + i * 4 + (lane >> 3);
                    const uint32_t at = q_smem + (uint32_t)(row * 128);
                    uint4 w[D / 64];
                    uint32_t top = 0;
#pragma unroll
                    for (int half = 0; half < D / 64; ++half) {
                        w[half] = ld_shared(at + (uint32_t)(half * ROWS * 128 + (c ^ (row & 7)) * 16));
                        const uint32_t x[4] = {w[half].x, w[half].y, w[half].z, w[half].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) top = max(top, max(x[k] & 0x7FFFu, x[k] >> 16 & 0x7FFFu));
                    }
#pragma unroll
                    for (int x = 1; x < 8; x <<= 1) top = max(top, __shfl_xor_sync(FULL, top, x));
                    __syncwarp();                          // every lane has its part of the row
                    // the row's largest comes to [128, 256); both powers are normal numbers
                    const int e = min(max((int)(top >> 7) - 127, -119), 127) - 7;
                    const float out = __int_as_float((127 - e) << 23), in = __int_as_float((127 + e) << 23);
#pragma unroll
                    for (int half = 0; half < D / 64; ++half) {
                        const uint32_t x[4] = {w[half].x, w[half].y, w[half].z, w[half].w};
                        uint32_t term[2][2];                             // 8 dims each
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float v[4] = {bf16_lo(x[2 * k]) * out, bf16_hi(x[2 * k]) * out, bf16_lo(x[2 * k + 1]) * out, bf16_hi(x[2 * k + 1]) * out};
#pragma unroll
                            for (int n = 0; n < 4; ++n) v[n] += v[n] - v[n];             // what is not finite becomes NaN
                            term[0][k] = pack_e4m3x2(v[0], v[1]) | pack_e4m3x2(v[2], v[3]) << 16;
                            uint32_t a, b;
                            e4m3x4_to_f16x2(term[0][k], a, b);
                            const float2 f = f16x2_to_f32x2(a), g = f16x2_to_f32x2(b);
                            term[1][k] = pack_e4m3x2(v[0] - f.x, v[1] - f.y) | pack_e4m3x2(v[2] - g.x, v[3] - g.y) << 16;
                        }
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            const int col = t * D + half * 64 + c * 8;   // byte of the row's two terms, in tiles of 128
                            asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(at + (uint32_t)((col >> 7) * ROWS * 128 + (((col >> 4 & 7) ^ (row & 7)) * 16) + (col & 8))),
                                         "r"(term[t][0]), "r"(term[t][1]) : "memory");
                        }
                    }
                    const float theirs = __shfl_sync(FULL, in, (lane & 3) * 8);
                    if (lane >> 2 == i) row_scale = theirs;
                }
            }
            fence_proxy_async();                           // the tensor core reads them through the async proxy
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
        }
        // =================== softmax ===================
        const uint32_t lane_base = tmem + ((uint32_t)(warp * 32) << 16), output = lane_base + COL_O;
        const int token = tid / G, g = tid - token * G;
        const bool row_ok = token < rows;
        const int pos = row_ok ? p0 + token : 0x7FFFFFF0;
        const float scale = FP8 ? row_scale : p.scale_log2;       // of what the loop below takes for scores (FP8: K's scales times the rest are in them)
        const uint64_t scale2 = pair_of(scale, scale);
        float m_used = -INFINITY, l_sum = 0.f, c_used = LEAST_C;    // c_used: log2 c
        int page32 = page_at(lane), next32 = page_at(32 + lane);       // lane: entry 8 k + lane
        for (int kb = 0; kb < blocks; ++kb) {
            if (kb > 0 && (kb & 7) == 0) {
                page32 = next32;
                next32 = page_at((kb + 8) * KB + lane);
            }
            int page[KB];
            bool clear = true;
#pragma unroll
            for (int j = 0; j < KB; ++j) {
                page[j] = __shfl_sync(FULL, page32, (kb & 7) * KB + j);
                clear = clear && page[j] * PAGE + PAGE - 1 <= p0;        // every row sees every token of it
            }
            const int buf = kb & 1, bar = 8 * buf;
            const uint32_t phase = (uint32_t)((kb >> 1) & 1), scores = lane_base + (uint32_t)(buf * KEYS);
            const uint32_t scales = scale_ring + (uint32_t)((kb & 3) * L::SCALE_STAGE);
            wait(s_ready + bar, phase, gave_up);
            tc_fence_after();
            uint32_t raw[2][32];
#pragma unroll
            for (int i = 0; i < 2; ++i) tmem_ld32(scores + 32 * i, raw[i]);
            tmem_wait_ld();
            float c_block = 0.f;
            if (FP8) {
                // before anything is hidden: a hidden token's scale may be anything
#pragma unroll
                for (int c = 0; c < KEYS; c += 4) {
                    const uint4 s = ld_shared(scales + 4 * c);
                    const uint32_t f[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int k = 0; k < 4; k += 2) {
                        uint32_t &a = raw[c / 32][c % 32 + k], &b = raw[c / 32][c % 32 + k + 1];
                        float x, y;
                        halves(mul2(pair_of(__uint_as_float(a), __uint_as_float(b)), pair_of(__uint_as_float(f[k]), __uint_as_float(f[k + 1]))), x, y);
                        a = __float_as_uint(x);
                        b = __float_as_uint(y);
                    }
                }
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(c_block) : "r"(scales + 2 * KEYS * 4));
            }
            if (!clear) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t bits = bits_up_to(pos, page[2 * i]) | bits_up_to(pos, page[2 * i + 1]) << PAGE;
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (!((bits >> c) & 1u)) raw[i][c] = 0xFF800000u;      // -inf
                }
                if (FP8) {                                 // the largest V scale of what this row sees
                    c_block = 0.f;
                    for (int c = 0; c < KEYS; ++c) {
                        float v;
                        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(scales + (uint32_t)(4 * (KEYS + c))));
                        if (bits_up_to(pos, __shfl_sync(FULL, page32, (kb & 7) * KB + c / PAGE)) >> (c % PAGE) & 1u) c_block = fmaxf(c_block, v);
                    }
                }
            }
            const float c_now = FP8 ? fmaxf(c_used, ceil_log2(c_block)) : 0.f;
            // Against the reference as it stands; again if the block's maximum turns out to have run away from it.
            for (;;) {
                const float neg_m = (m_used == -INFINITY ? 0.f : -m_used) - (FP8 ? c_used : 0.f);
                const uint64_t neg2 = pair_of(neg_m, neg_m);
                uint64_t sum2[2] = {0ull, 0ull};
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                uint32_t pk[32];
                uint4 vs = make_uint4(0, 0, 0, 0);                     // FP8: V scales of 4 tokens
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    const float s0 = __uint_as_float(raw[c >> 4][(2 * c) & 31]), s1 = __uint_as_float(raw[c >> 4][(2 * c + 1) & 31]);
                    const uint64_t x = fma2(pair_of(s0, s1), scale2, neg2);
                    float e0, e1;
                    halves(x, e0, e1);
                    e0 = ex2(e0);
                    e1 = ex2(e1);
                    mx4[c & 3] = max3(mx4[c & 3], s0, s1);
                    sum2[c & 1] = add2(sum2[c & 1], pair_of(e0, e1));
                    if (FP8) {
                        if (c % 2 == 0) vs = ld_shared(scales + (uint32_t)(4 * (KEYS + 2 * c)));
                        halves(mul2(pair_of(e0, e1), pair_of(__uint_as_float(c % 2 == 0 ? vs.x : vs.z), __uint_as_float(c % 2 == 0 ? vs.y : vs.w))), e0, e1);
                    }
                    pk[c] = FP8 ? pack_f16x2(e0, e1) : pack_bf16x2(e0, e1);
                }
                const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * scale;      // the scale is positive
                const bool higher = mx > m_used + RESCALE_STEP;    // also true for the first key that the row sees
                const bool move = higher || (FP8 && c_now > c_used);
                if (!__any_sync(FULL, move)) {
                    float s0, s1;
                    halves(add2(sum2[0], sum2[1]), s0, s1);
                    l_sum += s0 + s1;
                    tmem_st32(scores, pk);                         // P over the first half of its scores
                    break;
                }
                float alpha = higher ? ex2(m_used - mx) : 1.f;             // 0 when m_used = -inf
                if (higher) m_used = mx;
                if (FP8) {
                    alpha *= ex2(c_used - c_now);
                    c_used = c_now;
                }
                l_sum *= alpha;
                if (kb > 0) {
                    // O has to hold all blocks so far (P V two blocks back is over: these scores were issued after it)
                    wait(pv_done + 8 * (buf ^ 1), (uint32_t)(((kb - 1) >> 1) & 1), gave_up);
                    tc_fence_after();
#pragma unroll
                    for (int q = 0; q < D / 16; ++q) {
                        uint32_t ov[16];
                        tmem_ld16(output + 16 * q, ov);
                        tmem_wait_ld();
#pragma unroll
                        for (int c = 0; c < 16; ++c) ov[c] = __float_as_uint(__uint_as_float(ov[c]) * alpha);
                        tmem_st16(output + 16 * q, ov);
                    }
                }
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_ready + bar);
        }
        wait(pv_done + 8 * ((blocks - 1) & 1), (uint32_t)(((blocks - 1) >> 1) & 1), gave_up);
        tc_fence_after();
        if (ranks == 1) {
            const float inv = l_sum == 0.f ? 0.f : 1.f / l_sum;                // (a row that sees nothing)
            uint32_t packed[D / 2];
#pragma unroll
            for (int q = 0; q < D / 32; ++q) {
                uint32_t ov[32];
                tmem_ld32(output + 32 * q, ov);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 16; ++c) packed[16 * q + c] = pack_bf16x2(__uint_as_float(ov[2 * c]) * inv, __uint_as_float(ov[2 * c + 1]) * inv);
            }
            if (row_ok) {
                uint16_t *dst = out_rows + ((int64_t)token * p.Hq + g) * D;
                if ((reinterpret_cast<uintptr_t>(p.out) & 31) == 0) {          // whole sectors: half as many, and none written twice
#pragma unroll
                    for (int c = 0; c < D / 2; c += 8)
                        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + 2 * c), "r"(packed[c]), "r"(packed[c + 1]),
                                     "r"(packed[c + 2]), "r"(packed[c + 3]), "r"(packed[c + 4]), "r"(packed[c + 5]), "r"(packed[c + 6]), "r"(packed[c + 7]) : "memory");
                } else {
#pragma unroll
                    for (int c = 0; c < D / 2; c += 4)
                        *reinterpret_cast<uint4 *>(dst + 2 * c) = make_uint4(packed[c], packed[c + 1], packed[c + 2], packed[c + 3]);
                }
            }
        } else {
            // O [D/4 groups][128 rows][4], then each row's reference and sum, to where the operands were; every CTA joins some of the dims
            const uint32_t mine = q_smem + (uint32_t)(tid * 16), sums = q_smem + ROWS * D * 4;
#pragma unroll
            for (int q = 0; q < D / 32; ++q) {
                uint32_t ov[32];
                tmem_ld32(output + 32 * q, ov);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 8; ++c) st_shared(mine + (uint32_t)((8 * q + c) * ROWS * 16), make_uint4(ov[4 * c], ov[4 * c + 1], ov[4 * c + 2], ov[4 * c + 3]));
            }
            asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(sums + (uint32_t)(tid * 8)), "f"(m_used + (FP8 ? c_used : 0.f)), "f"(l_sum) : "memory");
            __syncwarp();
            cluster_arrive();                      // this part is complete ...
            cluster_wait();                        // ... and so is everybody's
            uint16_t *dst = out_rows + ((int64_t)token * p.Hq + g) * D;
            const int first = D / 8 * (int)rank / parts, last = D / 8 * ((int)rank + 1) / parts;       // groups of 8 dims
            if (parts <= 2) join_parts<2, 4>(mine, sums + (uint32_t)(tid * 8), parts, first, last, row_ok, dst);
            else if (parts <= 4) join_parts<4, 2>(mine, sums + (uint32_t)(tid * 8), parts, first, last, row_ok, dst);
            else join_parts<MAX_PARTS, 1>(mine, sums + (uint32_t)(tid * 8), parts, first, last, row_ok, dst);
            __syncwarp();
            cluster_arrive();                      // nobody leaves while its part is being read
            cluster_wait();
        }
    } else {
        if (!FP8) fewer_registers<56>();
        else fewer_registers<40>();
        const bool leader = elect_one(), values = (warp & 1) != 0;
        const uint32_t output = tmem + COL_O;
        const uint64_t q_desc = swizzled_desc(q_smem);
        // scores of block kb from the K at k_desc / output of block kb from the V at v_desc, whose pages and halves of 8 tokens are
        // `half` bytes apart and whose 8-dim groups are `group` bytes: by one lane of a warp that has waited for its operands
        auto issue_scores = [&](int kb, uint64_t k_desc) {
            const uint32_t scores = tmem + (uint32_t)((kb & 1) * KEYS);
            if constexpr (FP8) {                       // both terms of the queries on the codes as they are, 32 dims at a time
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int ks = 0; ks < D / 32; ++ks) {
                        const int col = t * D + ks * 32;
                        umma_ss_f8(scores, q_desc + (uint64_t)(((col >> 7) * ROWS * 128 + (col & 127)) >> 4), k_desc + (uint64_t)((ks * 2 * 128) >> 4), IDESC_QK,
                                   t > 0 || ks > 0);
                    }
            } else {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma_ss(scores, q_desc + (uint64_t)(((ks >> 2) * ROWS * 128 + (ks & 3) * 32) >> 4), k_desc + (uint64_t)((ks * 2 * 128) >> 4), IDESC_QK, ks > 0);
            }
            tc_commit(s_ready + 8 * (kb & 1));
        };
        auto issue_output = [&](int kb, uint64_t v_desc) {
            const uint32_t scores = tmem + (uint32_t)((kb & 1) * KEYS);
            const int np = listed - kb * KB;
#pragma unroll
            for (int j = 0; j < KB; ++j)
                if (j < np) umma_ts(output, scores + (uint32_t)(8 * j), v_desc + (uint64_t)((j * HALF) >> 4), IDESC_PV, j > 0 || kb > 0 ? 1u : 0u);
            tc_commit(pv_done + 8 * (kb & 1));
        };
        if (FP8) {
            if (warp < 8) {
                // =================== conversion of V ===================
                const int me = tid - 128;
                int page32 = page_at(lane), next32 = page_at(32 + lane);
                for (int kb = 0; kb < blocks; ++kb) {
                    if (kb > 0 && (kb & 7) == 0) {
                        page32 = next32;
                        next32 = page_at((kb + 8) * KB + lane);
                    }
                    const int st = kb % VS, np = listed - kb * KB < KB ? listed - kb * KB : KB;
                    const uint32_t from = v_ring + (uint32_t)(st * L::V_STAGE), tile = v_tiles + (uint32_t)((kb & 1) * L::TILE);
                    // tokens that some row sees, of this lane's entry of the block
                    const uint32_t seen = bits_up_to(p1, page32);
                    const bool partial = __any_sync(FULL, seen != 0xFFFFu && lane >> 2 == (kb & 7));
                    wait(v_full + 8 * st, (uint32_t)((kb / VS) & 1), gave_up);
                    if (kb >= 2) wait(pv_done + 8 * (kb & 1), (uint32_t)(((kb >> 1) - 1) & 1), gave_up);       // the tile: P V two blocks back is over
                    // unit: a dim of a page, 16 tokens (a warp's units are of one page)
#pragma unroll 1
                    for (int u0 = me; u0 < np * D; u0 += 256) {
                        uint4 w[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (u0 + 128 * i < np * D) w[i] = ld_shared(from + (uint32_t)((u0 + 128 * i) * 16));
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int u = u0 + 128 * i, j = u / D, dim = u % D;
                            if (u >= np * D) break;
                            if (partial) {
                                const uint32_t bits = __shfl_sync(FULL, seen, (kb & 7) * KB + j);
                                auto keep = [&](int k) {
                                    const uint32_t f = bits >> (4 * k) & 0xFu;
                                    return ((f & 1u) | (f & 2u) << 7 | (f & 4u) << 14 | (f & 8u) << 21) * 0xFFu;
                                };
                                w[i] = make_uint4(w[i].x & keep(0), w[i].y & keep(1), w[i].z & keep(2), w[i].w & keep(3));
                            }
                            uint4 x, y;
                            convert16(w[i], x, y);
                            st_shared(tile + (uint32_t)(j * HALF + dim * 16), x);
                            st_shared(tile + (uint32_t)(j * HALF + (D + dim) * 16), y);
                        }
                    }
                    fence_proxy_async();               // the tensor core reads the tile through the async proxy
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(v_ready + 8 * (kb & 1));
                        mbar_arrive(v_empty + 8 * st);
                    }
                }
            } else if (warp == 8) {
                // =================== scales, and scores from the codes as they are ===================
                const uint64_t ring_desc = smem_desc(k_ring, 128, 8 * D);
                int page32 = page_at(lane), next32 = page_at(32 + lane);
                wait(q_full, 0, gave_up);
                for (int kb = 0; kb < blocks; ++kb) {
                    if (kb > 0 && (kb & 7) == 0) {
                        page32 = next32;
                        next32 = page_at((kb + 8) * KB + lane);
                    }
                    const int st = kb % KS, np = listed - kb * KB < KB ? listed - kb * KB : KB;
                    const uint32_t bar = 8 * ((uint32_t)kb & 1u), seen = bits_up_to(p1, page32);
                    // (this slot's last scales were those of four blocks back, whose P V was over when the block before this was issued)
                    const uint32_t from = k_ring + (uint32_t)(st * L::K_STAGE + KEYS * D), slot = scale_ring + (uint32_t)((kb & 3) * L::SCALE_STAGE);
                    wait(k_full + 8 * st, (uint32_t)((kb / KS) & 1), gave_up);
                    uint32_t most = 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        // a token's K scale into units of log2, V scale (0 where no row sees it)
                        const int x = lane + 32 * i, j = x / PAGE, t = x % PAGE;
                        const uint32_t bits = __shfl_sync(FULL, seen, (kb & 7) * KB + j);
                        float ks = 0.f, vs = 0.f;
                        if (j < np && (bits >> t & 1u)) {
                            const uint32_t a = from + (uint32_t)((j * 2 * PAGE + t) * 4);
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ks) : "r"(a) : "memory");
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(vs) : "r"(a + PAGE * 4) : "memory");
                        }
                        most = max(most, __float_as_uint(vs));           // (0 or more; the bits of a NaN are above all)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(slot + (uint32_t)(x * 4)), "f"(ks * p.scale_log2) : "memory");
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(slot + (uint32_t)((KEYS + x) * 4)), "f"(vs) : "memory");
                    }
                    most = __reduce_max_sync(FULL, most);
                    if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(slot + (uint32_t)(2 * KEYS * 4)), "r"(most) : "memory");
                    __syncwarp();
                    if (kb >= 2) wait(pv_done + bar, (uint32_t)(((kb >> 1) - 1) & 1), gave_up);        // the buffer: P V two blocks back is over
                    tc_fence_after();
                    if (leader) {
                        mbar_arrive(s_ready + bar);
                        issue_scores(kb, ring_desc + (uint64_t)((st * L::K_STAGE) >> 4));
                        tc_commit(k_empty + 8 * st);
                    }
                    __syncwarp();
                }
                // the last commits arrive while the barriers are still there
                for (int j = blocks > KS ? blocks - KS : 0; j < blocks; ++j) wait(k_empty + 8 * (j % KS), (uint32_t)((j / KS) & 1), gave_up);
            } else if (warp == 9) {
                // =================== outputs ===================
                const uint64_t desc = smem_desc(v_tiles, D * 16, 128);
                for (int kb = 0; kb < blocks; ++kb) {
                    const uint32_t bar = 8 * ((uint32_t)kb & 1u), turn = (uint32_t)(kb >> 1);
                    wait(v_ready + bar, turn & 1u, gave_up);
                    wait(p_ready + bar, turn & 1u, gave_up);
                    tc_fence_after();
                    if (leader) issue_output(kb, desc + (uint64_t)(((kb & 1) * L::TILE) >> 4));
                    __syncwarp();
                }
            } else {
                // =================== copies: K and the scales, or V ===================
                const int stages = values ? VS : KS;
                const uint32_t ring = values ? v_ring : k_ring, stage_bytes = values ? L::V_STAGE : L::K_STAGE, full = values ? v_full : k_full,
                               empty = values ? v_empty : k_empty;
                int id = id_at(lane), next_id = id_at(32 + lane);        // lane 4 (kb % 8) + j has entry j of block kb
                for (int kb = 0; kb < blocks; ++kb) {
                    if (kb > 0 && (kb & 7) == 0) {
                        id = next_id;
                        next_id = id_at((kb + 8) * KB + lane);
                    }
                    const int st = kb % stages, np = listed - kb * KB < KB ? listed - kb * KB : KB, j = lane - (kb & 7) * KB;
                    if (kb >= stages) wait(empty + 8 * st, (uint32_t)((kb / stages - 1) & 1), gave_up);
                    if (lane == 0) mbar_expect_tx(full + 8 * st, (uint32_t)(np * (values ? PAGE * D : PAGE * D + 2 * PAGE * 4)));
                    __syncwarp();
                    if (j >= 0 && j < np) {
                        const uint8_t *src = p.layer_base + (int64_t)id * p.page_stride + (int64_t)h * BLOCK;
                        const uint32_t dst = ring + (uint32_t)st * stage_bytes;
                        bulk_copy_g2s(dst + (uint32_t)(j * PAGE * D), src + (values ? fp8_v_off(D) : 0), PAGE * D, full + 8 * st);
                        if (!values) bulk_copy_g2s(dst + (uint32_t)(KEYS * D + j * 2 * PAGE * 4), src + fp8_ks_off(D), 2 * PAGE * 4, full + 8 * st);
                    }
                    __syncwarp();
                }
                // leave only when every copy has landed (as on bf16 pages)
                for (int j = blocks > stages ? blocks - stages : 0; j < blocks; ++j) wait(full + 8 * (j % stages), (uint32_t)((j / stages) & 1), gave_up);
                if (*gave_up) {
                    const uint64_t t = global_timer_ns();
                    while (global_timer_ns() - t < 1000000ull) __nanosleep(1000);
                }
            }
        } else if (warp < 6) {
            // =================== tensor-core issue: the whole warp walks along, one lane issues ===================
            const uint64_t ring_desc = values ? smem_desc(v_ring, 128, PAGE * 16) : smem_desc(k_ring, 128, CH * 128);
            const uint32_t full = values ? v_full : k_full, empty = values ? v_empty : k_empty;
            if (!values) wait(q_full, 0, gave_up);
            for (int kb = 0; kb < blocks; ++kb) {
                const uint32_t st = (uint32_t)kb & (KS - 1), bar = 8 * ((uint32_t)kb & 1u), turn = (uint32_t)(kb >> 1);
                const uint64_t desc = ring_desc + (uint64_t)(st * (L::TILE >> 4));
                wait(full + 8 * st, (uint32_t)(kb / KS) & 1u, gave_up);
                if (!values) {
                    if (kb >= 2) wait(pv_done + bar, (turn - 1) & 1u, gave_up);        // the buffer: P V two blocks back is over
                    tc_fence_after();
                    if (leader) issue_scores(kb, desc);
                } else {
                    wait(p_ready + bar, turn & 1u, gave_up);
                    tc_fence_after();
                    if (leader) issue_output(kb, desc);
                }
                if (leader) tc_commit(empty + 8 * st);
                __syncwarp();
            }
            // the last commits arrive while the barriers are still there
            for (int j = blocks > KS ? blocks - KS : 0; j < blocks; ++j) wait(empty + 8 * (j & (KS - 1)), (uint32_t)((j / KS) & 1), gave_up);
        } else if (warp == 6) {
            // =================== copies of K and V ===================
            if (lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
            // lane: entry 8 k + lane; a page no row sees a token of is some page's copy, whose V is zeroed
            auto whole_at = [&](int i) { return i >= listed || bits_up_to(p1, page_at(i)) == 0xFFFFu; };
            int id = id_at(lane), next_id = id_at(32 + lane);
            bool whole = whole_at(lane), next_whole = whole_at(32 + lane);
            for (int kb = 0; kb < blocks; ++kb) {
                if (kb > 0 && (kb & 7) == 0) {
                    id = next_id;
                    whole = next_whole;
                    next_id = id_at((kb + 8) * KB + lane);
                    next_whole = whole_at((kb + 8) * KB + lane);
                }
                const int st = kb & (KS - 1), np = listed - kb * KB < KB ? listed - kb * KB : KB, j = lane - (kb & 7) * KB;
                const uint32_t again = (uint32_t)((kb / KS - 1) & 1);
                const bool mine = j >= 0 && j < np;
                // a block with tokens that no row sees passes through the hands of warp 7 first
                const bool partial = __any_sync(FULL, mine && !whole);
                const uint32_t v_bar = (partial ? v_landed : v_full) + 8 * st;
                if (kb >= KS) wait(k_empty + 8 * st, again, gave_up);
                if (lane == 0) mbar_expect_tx(k_full + 8 * st, (uint32_t)(np * HALF));
                __syncwarp();
                if (mine) tensor_copy_k(k_ring + (uint32_t)(st * L::TILE + j * HALF), &k_map, h, id, k_full + 8 * st);
                if (kb >= KS) wait(v_empty + 8 * st, again, gave_up);
                if (lane == 0) mbar_expect_tx(v_bar, (uint32_t)(np * HALF));
                __syncwarp();
                if (mine)
                    bulk_copy_g2s(v_ring + (uint32_t)(st * L::TILE + j * HALF), p.layer_base + (int64_t)id * p.page_stride + (int64_t)h * BLOCK + HALF, HALF, v_bar);
            }
            // leave only when every copy has landed (normally long the case; after a failure it is not known which barrier one
            // still in flight will come through, and it is given time)
            for (int j = blocks > KS ? blocks - KS : 0; j < blocks; ++j) {
                wait(k_full + 8 * (j & (KS - 1)), (uint32_t)((j / KS) & 1), gave_up);
                wait(v_full + 8 * (j & (KS - 1)), (uint32_t)((j / KS) & 1), gave_up);
            }
            if (*gave_up) {
                const uint64_t t = global_timer_ns();
                while (global_timer_ns() - t < 1000000ull) __nanosleep(1000);
            }
        } else {
            // =================== V rows that no row of the item sees ===================
            uint32_t landed = 0;                       // bit per ring stage: parity of the blocks that came through v_landed
            for (int kb0 = 0; kb0 < blocks; kb0 += 8) {
                const uint32_t bits = kb0 * KB + lane < listed ? bits_up_to(p1, page_at(kb0 * KB + lane)) : 0xFFFFu;
                unsigned todo = __ballot_sync(FULL, bits != 0xFFFFu);
                while (todo) {                         // (few have any: the last page of a list)
                    const int x = __ffs(todo) - 1, kb = kb0 + x / KB, st = kb & (KS - 1);
                    const unsigned block = todo & (((1u << KB) - 1) << (x / KB * KB));
                    wait(v_landed + 8 * st, (landed >> st) & 1u, gave_up);
                    landed ^= 1u << st;
                    for (unsigned rest = block; rest; rest &= rest - 1) {
                        const int y = __ffs(rest) - 1;
                        const uint32_t set = __shfl_sync(FULL, bits, y);
                        for (int i = lane; i < CH * PAGE; i += 32)
                            if (!((set >> (i & (PAGE - 1))) & 1u))
                                st_shared(v_ring + (uint32_t)(st * L::TILE + (y & (KB - 1)) * HALF + i * 16), make_uint4(0, 0, 0, 0));
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(v_full + 8 * st);
                    todo &= ~block;
                }
            }
        }
    }
    if (ranks > 1 && warp >= 4) {              // (the softmax warps have been there)
        __syncwarp();
        for (int i = 0; i < 2; ++i) {
            cluster_arrive();
            cluster_wait();
        }
    }
    // ---- common exit ----
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && *gave_up) atomicOr(p.status, STATUS_TIMEOUT);
    if (warp == 4) {
        __syncwarp();
        tmem_dealloc(tmem, TMEM_COLS);
    }
}

template <int D, bool FP8>
cudaError_t launch_t(const PrefillParams &p, const PageLists &l, int G, int max_q_len, int sm_count, bool pdl, cudaStream_t s)
{
    const int64_t ctas = (int64_t)p.B * l.per_seq * p.Hkv;
    const int ranks = prefill_pages_parts(ctas, l.stride < p.pt_stride ? l.stride : p.pt_stride, sm_count);
    if (ctas * ranks > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    CUtensorMap k_map = {};
    if (!FP8 && !encode_k_map(&k_map, p.layer_base, p.page_stride, p.max_pages, p.Hkv, D)) return cudaErrorNotSupported;
    auto kern = prefill_pages_kernel<D, FP8>;
    const size_t smem = Layout<D, FP8>::BYTES;
    const cudaError_t e = ensure_dynamic_smem(kern, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(ctas * ranks));
    cfg.blockDim = dim3(threads_of(FP8));
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
    return cudaLaunchKernelEx(&cfg, kern, p, l, k_map, G, max_q_len);
}

}  // namespace

// CTAs to a list.  A list is a chain of blocks, 0.6 us each on bf16 pages and 0.9 on FP8, and few lists leave SMs without one; what a part
// costs besides is its beginning and the joining, 5 us.  (us by CTAs to a list, 1 / 2 / 4 / 8, lists of 8 and of 32 blocks, bf16:
//     8 lists  10.8 10.4  9.6  9.6   25.6 17.6 13.3 11.5        64 lists  11.4 11.1 13.2 26.4   31.3 22.0 20.1 33.4
//    16        11.0 10.6  9.8 12.2   25.9 17.9 13.6 14.8       128        11.9 14.7 24.2 48.4   34.1 30.0 39.2 63.4
//    32        11.1 10.6 10.2 14.8   26.5 18.5 14.2 17.7       192        16.3 24.5 35.8 71.8   42.0 48.7 56.5 92.3
//  FP8, 32 lists 17.5 15.8 14.9 18.9, 40.5 27.5 20.7 23.2; 128 lists 18.4 21.1 33.9 62.5, 44.0 40.5 54.1 85.0.)  So: powers of two, of two
// blocks a part while there is an SM for each, of eight where two share one; 8 CTAs only with two SMs for each, as clusters share a GPC.
int prefill_pages_parts(int64_t lists, int pages, int sm_count)
{
    const int blocks = (pages + KB - 1) / KB;
    int r = 1;
    for (int next = 2; next <= MAX_PARTS; next *= 2) {
        const int64_t ctas = lists * next;
        const bool alone = ctas <= (next == 8 ? sm_count / 2 : sm_count);
        if (alone ? blocks < 2 * next : next == 8 || ctas > 2 * sm_count || blocks < 8 * next) break;
        r = next;
    }
    return r;
}

size_t prefill_pages_smem_bytes(int D, bool fp8)
{
    if (D == 128) return fp8 ? Layout<128, true>::BYTES : Layout<128, false>::BYTES;
    return D == 64 ? (fp8 ? Layout<64, true>::BYTES : Layout<64, false>::BYTES) : 0;
}

cudaError_t launch_prefill_pages(const PrefillParams &p, const PageLists &l, int D, int G, int max_q_len, bool fp8, int sm_count, bool pdl, cudaStream_t s)
{
    if (D == 128) return fp8 ? launch_t<128, true>(p, l, G, max_q_len, sm_count, pdl, s) : launch_t<128, false>(p, l, G, max_q_len, sm_count, pdl, s);
    if (D == 64) return fp8 ? launch_t<64, true>(p, l, G, max_q_len, sm_count, pdl, s) : launch_t<64, false>(p, l, G, max_q_len, sm_count, pdl, s);
    return cudaErrorInvalidValue;
}

}  // namespace skv
