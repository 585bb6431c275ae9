// Attention of prompts and chunks over a sliding window with sinks (skv_prefill_attn_window) on the 5th-generation
// tensor cores: the row at position pos attends  t <= pos  and  (t > pos - window  or  t < sinks).
//
// An item is (sequence, kv head, two neighbouring tiles of 128 query rows): row r of a tile = token r / G, head r % G.
// The tiles share every K and V read.  A persistent CTA per SM takes its share of the items, which are dealt out by their
// place in the sequence, furthest first (those have the most keys, where the window does not make all alike), back and forth
// over the CTAs: within 2 % of the mean where every CTA has some, by count (dealt in the order of the rows: 15 % over it).
// Sixteen warps:
//   warps 0-3, 4-7  softmax of tile 0 / tile 1: thread = row (TMEM lane)
//   warps 8, 9      issue the scores Q K^T of tile 0 / tile 1,  warps 10, 11 the outputs P V
//   warp 12         copies K and V of the key blocks (64 keys = 4 pages of the item's list of pages, window_pages)
//   warps 13, 14    copy the queries of the next item's tile 0 / tile 1 as soon as the last scores of this one are done
//   warp 15         zeroes the V rows of tokens that no row of the item sees, whatever they hold
// Shared memory: Q of both tiles (rows of 128 bytes in the 128-byte swizzle), K ring and V ring of four blocks each.  A page's
// K half, [chunk of 8 dims][16 tokens][16 B], is fetched by one tensor copy that puts its two groups of 8 tokens one
// behind the other, [group][chunk][8 tokens][16 B]: the groups of a block's pages then follow each other at one stride, and the
// block is one operand.  V pages are copied as they are: an MN-major operand.
// Tensor memory (512 columns): per tile two score buffers [64 each], each overwritten in place by the probabilities (bf16)
// of its block, and the outputs of tile 0 and 1.
//
// A tile's scores of block kb + 1 are issued before its softmax of block kb has finished, so the softmax warps find the next
// scores ready.  (A first form had blocks of 128 keys and one buffer per tile: each block then waited for its own chain
// softmax -> P V -> Q K^T, 6500 cycles of which the tensor core worked 2100, 306 us in all.  Blocks of 64 keys came together with
// shorter waits, tensor copies of K and uniform issue, which would have served 128 keys as well, so the 190 us of today do not
// tell the two apart; 128 keys have not been timed with the rest as it is now.  What 64 keys cost: an N = 64 instruction reads 6 KB
// of operands for 32 cycles of work, which take 48 cycles at 128 bytes a cycle.)  A warp per tile
// issues the instructions: one thread for both took 600 cycles of bookkeeping per tile and block and was slower than the tensor
// core.  The tiles need not be in step -- a block that one tile does not see is skipped by that tile alone.  A ring stage
// goes back to its copy warp when both tiles have done with it.
// Softmax as in skv_prefill_umma.cu: the reference maximum moves only when it has grown by more than 2^8, so O is rarely
// rescaled.  A row that has seen nothing yet counts from reference 0.
// Every wait is bounded; copies in flight get their wait before the end.
// Few rows behind long windows (a chunk of a prompt, a drafted run of tokens) leave most SMs idle and each item a long chain of
// blocks: there a cluster of CTAs shares an item's blocks and joins the outputs over distributed shared memory.
// Measured: 2 prompts of 4096 tokens, 32 query / 8 kv heads, head_dim 128, window 2048: 190 us, 1.09 PFLOP/s of visible pairs (0.67 of
// the measured bf16 peak) alone, 222 us (0.93 PFLOP/s) in a long loop, at the clock the power limit leaves; 8 chunks of 257 to 512 rows behind 3000 to
// 6000 tokens, window 1024: 64 to 77 us.  The tensor pipe has work in flight in 70 % of the cycles and computes in 55 %, the exponentials
// take 50 %, issue slots 48 %: what is left is operand reads (above), the chain scores -> maximum -> probabilities -> store of two tiles
// that overlap in part, and, in items of few blocks, an item's beginning (queries, first scores, a softmax taken twice), which nothing
// overlaps: the queries' one buffer comes back with the last scores of the item before.  Tried and slower:
// two threads to a row (199 us), the first maximum of an item before its exponentials (199), masks page by page (189).
#include "skv_common.cuh"
#include "skv_prefill_parts.cuh"
#include "skv_tcgen05.cuh"
#include "skv_walk.cuh"

namespace skv {

namespace {

using namespace tc5;
using namespace chunk;

constexpr int BY_FMA = 8;             // every eighth pair of exponentials is computed on the FMA units

// 2^x of a pair on the FMA units: x = n + f with n the nearest integer, a polynomial for 2^f on [-1/2, 1/2] (least largest
// relative error, by Remez exchange: 2.7e-6 in fp32, a thousandth of the rounding to bf16 that follows), times 2^n.
// x is clamped to -127, whose power of two has the bits of 0: a hidden key (x = -inf) gets exactly 0, as from ex2, and its V,
// however large, does not show.
__device__ __forceinline__ void exp2_by_fma(uint64_t x, float &lo, float &hi)
{
    const float magic = 12582912.f;                    // 1.5 * 2^23: x + magic has the nearest integer in its low bits
    float x0, x1;
    halves(x, x0, x1);
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(x0) : "f"(x0), "f"(-127.f));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(x1) : "f"(x1), "f"(-127.f));
    x = pair_of(x0, x1);
    const uint64_t r = add2(x, pair_of(magic, magic));
    const uint64_t n = add2(r, pair_of(-magic, -magic));
    const uint64_t f = fma2(n, pair_of(-1.f, -1.f), x);
    uint64_t y = pair_of(0.009570102207362652f, 0.009570102207362652f);
    y = fma2(y, f, pair_of(0.05591785907745361f, 0.05591785907745361f));
    y = fma2(y, f, pair_of(0.240247443318367f, 0.240247443318367f));
    y = fma2(y, f, pair_of(0.6931217908859253f, 0.6931217908859253f));
    y = fma2(y, f, pair_of(0.9999992847442627f, 0.9999992847442627f));
    float r0, r1;
    halves(r, r0, r1);
    const uint64_t power = pair_of(__int_as_float((__float_as_int(r0) << 23) + 0x3F800000), __int_as_float((__float_as_int(r1) << 23) + 0x3F800000));
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(y), "l"(power));       // (a NaN stays one)
    halves(y, lo, hi);
}

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int ROWS = 128;             // query rows of a tile
constexpr int KB = 4;                 // pages of a key block
constexpr int KEYS = KB * PAGE;
constexpr int THREADS = 512;
constexpr int STAGES = 4;             // key blocks of the K ring and of the V ring
constexpr int COL_O = 4 * KEYS;       // scores of tile s, buffer i at column 128 s + 64 i, its output at 256 + 128 s
constexpr int BAR_BYTES = 5 * 8 * STAGES + 3 * 32 + 3 * 16;
constexpr int MAX_RANKS = 8;          // CTAs that may share an item
constexpr int MAX_BATCH = 1024;       // sequences of a launch: their tables are in shared memory

// What an item is made of.
struct Item {
    int b, h, q_begin;      // sequence, kv head, the sequence's first query row
    int q0, q_len;          // first token of the item among the sequence's new ones; all of those
    int pos0;               // position of the sequence's first new token
    int n[2];               // tokens of the two tiles
    int rows;               // tokens of tile 0, also where none of its blocks is this CTA's
    int n_keys;             // keys below this one are visible to some row
    int kb0, blocks;        // blocks [kb0, blocks) of its list are this CTA's
    WindowPages win;
    // tokens of tile s: positions first(s) .. last(s)
    __device__ __forceinline__ int first(int s, int TQ) const { return pos0 + q0 + s * TQ; }
    __device__ __forceinline__ int last(int s, int TQ) const { return first(s, TQ) + n[s] - 1; }
};

// In shared memory.  Of the sequences, most items first: how many items (per kv head) the r-th has, and how many lie at
// places below that number in all sequences together, below[r] = r count[r] + count[r] + ... + count[B-1].
struct Tables {
    const int32_t *order, *count, *below;
    const int32_t *q_begin, *q_len, *lens;
    int rank, ranks;        // SPLIT: of this CTA in its cluster
};

// item of round `round` of this CTA; per_item: tokens of an item.  False: no more.
template <bool SPLIT>
__device__ __forceinline__ bool item_at(Item &it, const PrefillParams &p, const Tables &t, int total, int round, int TQ, int per_item)
{
    if (SPLIT && round > 0) return false;                   // (there is a cluster for every item)
    const int x = SPLIT ? (int)blockIdx.x / t.ranks : round * (int)gridDim.x + ((round & 1) ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
    if (x >= total) return false;
    const int back = total - 1 - x, y = back / p.Hkv;       // places ascending, over the sequences that have one
    it.h = back - y * p.Hkv;
    int lo = 0, hi = p.B;                                   // the smallest r with below[r] <= y  (below[0] is all, below[B] = 0)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.below[mid] <= y) hi = mid; else lo = mid;
    }
    const int d = y - t.below[hi], place = d / hi;          // the first hi sequences have an item there
    it.b = t.order[d - place * hi];
    it.q_begin = t.q_begin[it.b];
    it.q_len = t.q_len[it.b];
    it.q0 = (t.count[hi] + place) * per_item;
    it.pos0 = t.lens[it.b] - it.q_len;
    const int left = it.q_len - it.q0;
    it.n[0] = left < TQ ? left : TQ;
    const int second = (left < per_item ? left : per_item) - TQ;
    it.n[1] = second > 0 ? second : 0;
    it.n_keys = it.pos0 + it.q0 + it.n[0] + it.n[1];
    it.win = window_pages(it.pos0 + it.q0, it.n_keys, p.window, p.sinks);
    it.kb0 = 0;
    it.blocks = (it.win.count + KB - 1) / KB;
    it.rows = it.n[0];
    if (SPLIT) {
        const int all = it.blocks;
        it.kb0 = all * t.rank / t.ranks;
        it.blocks = all * (t.rank + 1) / t.ranks;
    }
    return true;
}

// The blocks that some row of tile s sees: [0, sinks) and [from, to), sinks <= from; and those of them, [clear_from, clear_to),
// of which every row of the tile sees every key.
struct Plan { int sinks, from, to, clear_from, clear_to; };

__device__ __forceinline__ Plan plan_of(const Item &it, int s, int TQ, int window, int sinks)
{
    const int first = it.first(s, TQ), last = it.last(s, TQ);
    const int lo = first >= window ? first - window + 1 : 0;                  // first key that the tile's first row sees, sinks apart
    const int lo_last = last >= window ? last - window + 1 : 0;              // ... and its last row
    const int gap = it.win.gap, sink_blocks = sinks > 0 ? (it.win.sink_pages + KB - 1) / KB : 0;
    Plan q;
    q.to = (last / PAGE - gap) / KB + 1;                                     // (the page of a row's own key is behind the gap)
    q.sinks = sink_blocks < q.to ? sink_blocks : q.to;
    const int x = lo / PAGE - gap;
    q.from = x > 0 ? x / KB : 0;
    if (q.from < q.sinks) q.from = q.sinks;
    const int c = (lo_last + PAGE - 1) / PAGE - gap, behind_gap = gap > 0 ? (it.win.sink_pages + KB - 1) / KB : 0;
    q.clear_from = c > 0 ? (c + KB - 1) / KB : 0;
    if (q.clear_from < behind_gap) q.clear_from = behind_gap;
    const int e = (first + 1) / PAGE - gap;
    q.clear_to = e > 0 ? e / KB : 0;
    // this CTA's part of them
    if (q.sinks > it.blocks) q.sinks = it.blocks;
    if (q.from < it.kb0) q.from = it.kb0;
    if (q.to > it.blocks) q.to = it.blocks;
    return q;
}

// The items of a CTA, round by round, as a warp goes through them.  Working one out takes some two thousand cycles, all of
// latency: every lane does it for a round of its own, once in 32 rounds, and the rounds then only read their lane's.
template <bool SPLIT>
struct Items {
    Item mine;
    Plan plans[2];
    bool any;

    __device__ __forceinline__ bool at(Item &it, const PrefillParams &p, const Tables &t, int total, int round, int lane, int TQ, int per_item)
    {
        if ((round & 31) == 0) {
            any = item_at<SPLIT>(mine, p, t, total, round + lane, TQ, per_item);
            if (any)
                for (int s = 0; s < 2; ++s)
                    if (mine.n[s] > 0) plans[s] = plan_of(mine, s, TQ, p.window, p.sinks);
        }
        const int from = round & 31;
        if (!__shfl_sync(FULL, (int)any, from)) return false;
        auto get = [&](int v) { return __shfl_sync(FULL, v, from); };
        it.b = get(mine.b);
        it.h = get(mine.h);
        it.q_begin = get(mine.q_begin);
        it.q_len = get(mine.q_len);
        it.q0 = get(mine.q0);
        it.pos0 = get(mine.pos0);
        it.n[0] = get(mine.n[0]);
        it.n[1] = get(mine.n[1]);
        it.n_keys = get(mine.n_keys);
        it.blocks = get(mine.blocks);
        it.kb0 = SPLIT ? get(mine.kb0) : 0;
        if (SPLIT && it.kb0 == it.blocks) it.n[0] = 0;          // nothing to do for this CTA
        it.win.lo = get(mine.win.lo);
        it.win.sink_pages = get(mine.win.sink_pages);
        it.win.gap = get(mine.win.gap);
        it.win.count = get(mine.win.count);
        return true;
    }
    // of the round that at() was asked for last
    __device__ __forceinline__ Plan plan(int s, int round) const
    {
        const Plan &q = plans[s];
        const int from = round & 31;
        return {__shfl_sync(FULL, q.sinks, from), __shfl_sync(FULL, q.from, from), __shfl_sync(FULL, q.to, from),
                __shfl_sync(FULL, q.clear_from, from), __shfl_sync(FULL, q.clear_to, from)};
    }
};

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
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t a)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}

// Dynamic shared memory: Q [2][D/64][128 rows][128 B] | K ring [4][8 groups][D/8 chunks][8 keys][16 B] | V ring [4][4 pages][V half]
//                        | barriers | tensor-memory address, gave_up, items | tables [6][B + 1]
// SPLIT: a cluster of CTAs to an item of one tile, each with its part of the key blocks, where that leaves no SM out: the outputs
// are joined over distributed shared memory.
template <int D, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1) prefill_window_kernel(const __grid_constant__ PrefillParams p, const __grid_constant__ CUtensorMap k_map,
                                                                       int G, int tiles, int max_q_len)
{
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    constexpr int BLOCK = block_bytes(D), HALF = half_bytes(D), CH = D / 8;
    constexpr int Q_BYTES = ROWS * D * 2, STAGE = KEYS * D * 2;
    constexpr uint32_t IDESC_QK = instr_desc(ROWS, KEYS, false), IDESC_PV = instr_desc(ROWS, D, true);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);      // (known to be the same for the warp)
    const int TQ = ROWS / G, per_item = TQ * tiles;

    const uint32_t base = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
    const uint32_t q_smem = base + pad, k_ring = q_smem + 2 * Q_BYTES, v_ring = k_ring + STAGES * STAGE, bars = v_ring + STAGES * STAGE;
    // a barrier per ring stage: copied, given back; per tile and score buffer: scores, probabilities, P V; per tile: the rest
    const uint32_t k_full = bars, v_full = k_full + 8 * STAGES, v_landed = v_full + 8 * STAGES, k_empty = v_landed + 8 * STAGES, v_empty = k_empty + 8 * STAGES;
    const uint32_t s_ready = v_empty + 8 * STAGES, p_ready = s_ready + 32, pv_done = p_ready + 32;
    const uint32_t q_full = pv_done + 32, q_free = q_full + 16, o_free = q_free + 16;
    uint8_t *words = smem_raw + pad + 2 * Q_BYTES + 2 * STAGES * STAGE + BAR_BYTES;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(words), *gave_up = tmem_slot + 1;
    int32_t *order = reinterpret_cast<int32_t *>(words + 16), *count = order + p.B + 1, *below = count + p.B + 1;
    int32_t *q_begin = below + p.B + 1, *q_len = q_begin + p.B + 1, *lens = q_len + p.B + 1;
    uint32_t rank = 0, ranks = 1;
    if (SPLIT) {
        asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    }
    const Tables tables = {order, count, below, q_begin, q_len, lens, (int)rank, (int)ranks};
    // SPLIT, in place of the K ring once the item is done: a row's output [128][D + 4] (four words of padding: no two lanes in one
    // bank), and its reference and sum [128]
    constexpr int STATE_ROW = D + 4;
    const uint32_t state = k_ring, state_ml = state + (uint32_t)(ROWS * STATE_ROW * 4);
    static_assert(ROWS * (STATE_ROW + 2) * 4 <= 2 * STAGES * STAGE, "the joined state fits the rings");

    if (tid == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(k_full + 8 * i, 1);
            mbar_init(v_full + 8 * i, 1);
            mbar_init(v_landed + 8 * i, 1);
            mbar_init(k_empty + 8 * i, 2);
            mbar_init(v_empty + 8 * i, 2);
            mbar_init(s_ready + 8 * i, 1);         // (two tiles x two buffers)
            mbar_init(p_ready + 8 * i, 4);
            mbar_init(pv_done + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(q_full + 8 * i, 1);
            mbar_init(q_free + 8 * i, 1);
            mbar_init(o_free + 8 * i, 4);
        }
        *gave_up = 0;
        fence_barrier_init();
    }
    if (warp == 8) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), 512);
        tmem_relinquish();
    }
    pdl_wait();
    pdl_trigger();
    // the sequences' tables
    for (int i = tid; i < p.B; i += THREADS) {
        const int qb = __ldg(p.cu_q + i), ql = __ldg(p.cu_q + i + 1) - qb, n = __ldg(p.seq_lens + i);
        const bool fits = qb >= 0 && ql >= 0 && ql <= n && ql <= max_q_len && (int64_t)n <= (int64_t)p.pt_stride * PAGE;
        if (!fits && blockIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
        q_begin[i] = qb;
        q_len[i] = ql;
        lens[i] = n;
        below[i] = fits ? (ql + per_item - 1) / per_item : 0;            // (for now: the sequence's items)
    }
    __syncthreads();
    for (int i = tid; i < p.B; i += THREADS) {                           // its place among the others, most items first
        const int mine = below[i];
        int before = 0;
        for (int j = 0; j < p.B; ++j) before += below[j] > mine || (below[j] == mine && j < i);
        order[before] = i;
        count[before] = mine;
    }
    if (tid == 0) count[p.B] = 0;
    __syncthreads();
    if (warp == 0) {                                                     // sums from the back
        int carry = 0;
        for (int i0 = 0; i0 <= p.B; i0 += 32) {
            const int r = p.B - i0 - lane;
            const int c = r >= 0 ? count[r] : 0;
            int sum = c;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int u = __shfl_up_sync(FULL, sum, d);
                if (lane >= d) sum += u;
            }
            if (r >= 0) below[r] = r * c + carry + sum;
            carry += __shfl_sync(FULL, sum, 31);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const int total = below[0] * p.Hkv;

    if (warp < 8) {
        // =================== softmax ===================
        more_registers<208>();
        const int s = warp >> 2, row = tid & (ROWS - 1);
        const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16), scores0 = lane_base + (uint32_t)(2 * s * KEYS),
                       output = lane_base + (uint32_t)(COL_O + 2 * s * KEYS);
        const int qi = row / G, g = row - qi * G;
        const uint64_t scale2 = pair_of(p.scale_log2, p.scale_log2);
        const bool wide_out = (reinterpret_cast<uintptr_t>(p.out) & 31) == 0;
        int count = 0;                             // blocks of this tile so far
        Item it;
        Items<SPLIT> items = {};
        for (int round = 0; items.at(it, p, tables, total, round, lane, TQ, per_item); ++round) {
            if (it.n[s] == 0) continue;
            const Plan plan = s == 0 ? items.plan(0, round) : items.plan(1, round);
            const bool row_ok = qi < it.n[s];
            const int pos = row_ok ? it.first(s, TQ) + qi : 0x7FFFFFFE, lo = pos >= p.window ? pos - p.window + 1 : 0;
            float m_used = -INFINITY, l_sum = 0.f;
            const int first = plan.sinks > it.kb0 ? it.kb0 : plan.from;
            for (int kb = first; kb < plan.to; kb = (kb + 1 < plan.sinks || kb + 1 >= plan.from) ? kb + 1 : plan.from) {
                const int buf = count & 1, bar = 8 * (2 * s + buf);
                const uint32_t phase = (uint32_t)((count >> 1) & 1), scores = scores0 + (uint32_t)(buf * KEYS);
                wait(s_ready + bar, phase, gave_up);
                tc_fence_after();
                uint32_t raw[2][32];
#pragma unroll
                for (int i = 0; i < 2; ++i) tmem_ld32(scores + 32 * i, raw[i]);
                tmem_wait_ld();
                if (kb < plan.clear_from || kb >= plan.clear_to) {
                    // the causal edge, the window's, a gap or an end: key by key
                    const int j0 = kb * KB;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t b0 = j0 + 2 * i < it.win.count ? window_bits(it.win.page(j0 + 2 * i), lo, pos + 1, p.sinks) : 0u;
                        const uint32_t b1 = j0 + 2 * i + 1 < it.win.count ? window_bits(it.win.page(j0 + 2 * i + 1), lo, pos + 1, p.sinks) : 0u;
                        const uint32_t bits = b0 | (b1 << 16);
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (!((bits >> c) & 1u)) raw[i][c] = 0xFF800000u;      // -inf
                    }
                }
                // The probabilities are taken against the reference as it stands while the block's maximum is being found; should that
                // turn out to have run away from it (an item's first block, rarely another), they are taken again.  The maximum first
                // and the exponentials then cost 280 cycles more a block.
                for (;;) {
                    const float neg_m = m_used == -INFINITY ? 0.f : -m_used;
                    const uint64_t neg2 = pair_of(neg_m, neg_m);
                    uint64_t sum2[2] = {0ull, 0ull};
                    float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    uint32_t pk[32];
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        const float s0 = __uint_as_float(raw[c >> 4][(2 * c) & 31]), s1 = __uint_as_float(raw[c >> 4][(2 * c + 1) & 31]);
                        const uint64_t x = fma2(pair_of(s0, s1), scale2, neg2);
                        float p0, p1;
                        if (c % BY_FMA == BY_FMA - 1) {
                            exp2_by_fma(x, p0, p1);
                        } else {
                            halves(x, p0, p1);
                            p0 = ex2(p0);
                            p1 = ex2(p1);
                        }
                        mx4[c & 3] = fmaxf(mx4[c & 3], fmaxf(s0, s1));
                        sum2[c & 1] = add2(sum2[c & 1], pair_of(p0, p1));
                        pk[c] = pack_bf16x2(p0, p1);
                    }
                    const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * p.scale_log2;      // the scale is positive
                    const bool move = mx > m_used + RESCALE_STEP;      // also true for the first key that the row sees
                    if (!__any_sync(FULL, move)) {
                        float s0, s1;
                        halves(add2(sum2[0], sum2[1]), s0, s1);
                        l_sum += s0 + s1;
                        tmem_st32(scores, pk);                         // P over the first half of its scores
                        break;
                    }
                    const float alpha = move ? ex2(m_used - mx) : 1.f;         // 0 when m_used = -inf
                    if (move) m_used = mx;
                    l_sum *= alpha;
                    if (kb != first) {
                        // O has to hold all blocks so far (P V two blocks back is over: these scores were issued after it)
                        wait(pv_done + 8 * (2 * s + (buf ^ 1)), (uint32_t)(((count - 1) >> 1) & 1), gave_up);
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
                ++count;
            }
            // the item's last P V
            wait(pv_done + 8 * (2 * s + ((count - 1) & 1)), (uint32_t)(((count - 1) >> 1) & 1), gave_up);
            tc_fence_after();
            if (SPLIT) {
#pragma unroll
                for (int q = 0; q < D / 32; ++q) {
                    uint32_t ov[32];
                    tmem_ld32(output + 32 * q, ov);
                    tmem_wait_ld();
#pragma unroll
                    for (int c = 0; c < 32; c += 4)
                        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(state + (uint32_t)((row * STATE_ROW + 32 * q + c) * 4)), "r"(ov[c]), "r"(ov[c + 1]), "r"(ov[c + 2]), "r"(ov[c + 3]) : "memory");
                }
                asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(state_ml + (uint32_t)(row * 8)), "f"(m_used), "f"(l_sum) : "memory");
                continue;
            }
            const float inv = 1.f / l_sum;
            uint16_t *dst = p.out + ((int64_t)(it.q_begin + it.q0 + s * TQ + qi) * p.Hq + (int64_t)it.h * G + g) * D;
            uint32_t packed[D / 2];
#pragma unroll
            for (int q = 0; q < D / 32; ++q) {
                uint32_t ov[32];
                tmem_ld32(output + 32 * q, ov);
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 16; ++c) packed[16 * q + c] = pack_bf16x2(__uint_as_float(ov[2 * c]) * inv, __uint_as_float(ov[2 * c + 1]) * inv);
            }
            tc_fence_before();                     // the output's columns may be used again
            __syncwarp();
            if (lane == 0) mbar_arrive(o_free + 8 * s);
            if (row_ok) {
                if (wide_out) {                    // whole sectors: half as many, and none written twice
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
        }
        if (SPLIT) {
            const bool any = item_at<SPLIT>(it, p, tables, total, 0, TQ, per_item);
            if (any && it.kb0 == it.blocks && tid < ROWS)          // no block of the item is this CTA's
                asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(state_ml + (uint32_t)(tid * 8)), "f"(-INFINITY), "f"(0.f) : "memory");
            __syncwarp();
            cluster_arrive();                      // every CTA's part is in place
            cluster_wait();
            // rows row_from .. row_to - 1 of the tile are joined by this CTA, four dims a thread at a time
            const int row_from = ROWS * (int)rank / (int)ranks, row_to = ROWS * (int)(rank + 1) / (int)ranks;
            for (int i = tid; any && i < (row_to - row_from) * (D / 4); i += 256) {
                const int r = row_from + i / (D / 4), d = i % (D / 4) * 4, token = r / G, g = r - token * G;
                if (token >= it.rows) break;       // (rows ascend)
                float2 ml[MAX_RANKS];
                float4 v[MAX_RANKS];
#pragma unroll
                for (int c = 0; c < MAX_RANKS; ++c) {
                    ml[c] = make_float2(-INFINITY, 0.f);
                    v[c] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (c < (int)ranks) {
                        ml[c] = ld_cluster_f2(at_rank(state_ml + (uint32_t)(r * 8), (uint32_t)c));
                        if (ml[c].y != 0.f) v[c] = ld_cluster_f4(at_rank(state + (uint32_t)((r * STATE_ROW + d) * 4), (uint32_t)c));
                    }
                }
                float M = -INFINITY, L = 0.f;
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int c = 0; c < MAX_RANKS; ++c) M = fmaxf(M, ml[c].x);
#pragma unroll
                for (int c = 0; c < MAX_RANKS; ++c) {
                    // The row sees nothing there: its weights, and so their sum, are exactly 0.  (Its maximum is -inf, but that is
                    // so too where all the scores are NaN; their sum is NaN, and the result has to be.)
                    if (ml[c].y == 0.f) continue;
                    const float w = ex2(ml[c].x - M);
                    L = fmaf(w, ml[c].y, L);
                    o = make_float4(fmaf(w, v[c].x, o.x), fmaf(w, v[c].y, o.y), fmaf(w, v[c].z, o.z), fmaf(w, v[c].w, o.w));
                }
                const float inv = 1.f / L;
                *reinterpret_cast<uint2 *>(p.out + ((int64_t)(it.q_begin + it.q0 + token) * p.Hq + (int64_t)it.h * G + g) * D + d) =
                    make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
            }
        }
    } else if (warp < 12) {
        // =================== tensor-core issue ===================
        // The whole warp walks along and one lane issues: descriptors and barriers are then the same for the warp as far as the
        // compiler can see, and stay in uniform registers.  (In a branch of lane 0 alone every instruction moved them there anew:
        // 60 to 100 cycles each, 2600 per tile and block.)
        fewer_registers<48>();
        const bool leader = elect_one(), values = warp >= 10;
        const int s = warp & 1;
        const uint32_t scores0 = tmem + (uint32_t)(2 * s * KEYS), output = tmem + (uint32_t)(COL_O + 2 * s * KEYS);
        // descriptors of the first instruction of each kind; the others are a constant further on in the address field
        const uint64_t q_desc = swizzled_desc(q_smem + (uint32_t)(s * Q_BYTES));
        const uint64_t ring_desc = values ? smem_desc(v_ring, 128, PAGE * 16) : smem_desc(k_ring, 128, CH * 128);
        const uint32_t full = values ? v_full : k_full, empty = values ? v_empty : k_empty;
        int g = 0, turn = 0, count = 0;            // blocks before this one; items and blocks of the tile before it
        Item it;
        Items<SPLIT> items = {};
        for (int round = 0; items.at(it, p, tables, total, round, lane, TQ, per_item); ++round) {
            const int blocks = it.blocks, pages = it.win.count;
            const bool mine = it.n[s] > 0;
            const Plan plan = s == 0 ? items.plan(0, round) : items.plan(1, round);
            const int sinks_to = mine ? plan.sinks : 0, from = mine ? plan.from : 0, to = mine ? plan.to : 0;
            const int final = from < to ? to - 1 : sinks_to - 1;
            bool begun = false;
            for (int kb = it.kb0; kb < blocks; ++kb, ++g) {
                const uint32_t st = (uint32_t)g & (STAGES - 1), parity = (uint32_t)(g / STAGES) & 1u;
                const uint32_t buf = (uint32_t)count & 1u, turn_of_buf = (uint32_t)(count >> 1), bar = 8 * (2 * s + buf), scores = scores0 + buf * KEYS;
                const uint64_t desc = ring_desc + (uint64_t)(st * (STAGE >> 4));
                if (kb >= to || (kb >= sinks_to && kb < from)) {
                    // not this tile's: once it is there (and the stage's block before it thus gone), it may go
                    wait(full + 8 * st, parity, gave_up);
                    if (leader) mbar_arrive(empty + 8 * st);
                    continue;
                }
                if (!values) {
                    if (!begun) wait(q_full + 8 * s, (uint32_t)(turn & 1), gave_up);
                    // the buffer: P V two blocks back is over
                    if (count >= 2) wait(pv_done + bar, (turn_of_buf - 1) & 1u, gave_up);
                    wait(full + 8 * st, parity, gave_up);
                    tc_fence_after();
                    if (leader) {
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)
                            umma_ss(scores, q_desc + (uint64_t)(((ks >> 2) * ROWS * 128 + (ks & 3) * 32) >> 4), desc + (uint64_t)((ks * 2 * 128) >> 4), IDESC_QK, ks > 0);
                        tc_commit(s_ready + bar);
                        tc_commit(empty + 8 * st);
                        if (kb == final) tc_commit(q_free + 8 * s);
                    }
                } else {
                    wait(full + 8 * st, parity, gave_up);
                    // an item's first block: the output of the item before has been read
                    if (!begun && turn > 0) wait(o_free + 8 * s, (uint32_t)((turn - 1) & 1), gave_up);
                    wait(p_ready + bar, turn_of_buf & 1u, gave_up);
                    tc_fence_after();
                    if (leader) {
                        const int np = pages - kb * KB;
#pragma unroll
                        for (int j = 0; j < KB; ++j)
                            if (j < np)
                                umma_ts(output, scores + (uint32_t)(8 * j), desc + (uint64_t)((j * HALF) >> 4), IDESC_PV, j > 0 || begun ? 1u : 0u);
                        tc_commit(pv_done + bar);
                        tc_commit(empty + 8 * st);
                    }
                }
                __syncwarp();
                begun = true;
                ++count;
            }
            if (mine) ++turn;
        }
        // the last commits arrive while the barriers are still there
        for (int j = g > STAGES ? g - STAGES : 0; j < g; ++j) wait(empty + 8 * (j & (STAGES - 1)), (uint32_t)((j / STAGES) & 1), gave_up);
    } else if (warp == 12) {
        // =================== copies of K and V ===================
        fewer_registers<48>();
        if (lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        int g = 0;
        Item it;
        Items<SPLIT> items = {};
        for (int round = 0; items.at(it, p, tables, total, round, lane, TQ, per_item); ++round) {
            const int32_t *row = p.page_table + (int64_t)it.b * p.pt_stride;
            auto load_id = [&](int kb) -> int {                // lane j: page j of a block
                const int j = kb * KB + lane;
                if (lane >= KB || j >= it.win.count) return 0;
                const int id = __ldg(row + it.win.page(j));
                if (id >= 0 && (int64_t)id < p.max_pages) return id;
                atomicOr(p.status, STATUS_BOUNDS);
                return 0;
            };
            int id = load_id(it.kb0), next_id = load_id(it.kb0 + 1);
            for (int kb = it.kb0; kb < it.blocks; ++kb, ++g) {
                const int st = g & (STAGES - 1), np = it.win.count - kb * KB < KB ? it.win.count - kb * KB : KB;
                const uint32_t again = (uint32_t)((g / STAGES - 1) & 1);
                // a block with tokens that no row sees passes through the hands of warp 15 first
                const bool partial = __any_sync(FULL, lane < np && window_bits(it.win.page(kb * KB + lane), it.win.lo, it.n_keys, p.sinks) != 0xFFFFu);
                const uint32_t v_bar = (partial ? v_landed : v_full) + 8 * st;
                if (g >= STAGES) wait(k_empty + 8 * st, again, gave_up);
                if (lane == 0) mbar_expect_tx(k_full + 8 * st, (uint32_t)(np * HALF));
                __syncwarp();
                if (lane < np) tensor_copy_k(k_ring + (uint32_t)(st * STAGE + lane * HALF), &k_map, it.h, id, k_full + 8 * st);
                if (g >= STAGES) wait(v_empty + 8 * st, again, gave_up);
                if (lane == 0) mbar_expect_tx(v_bar, (uint32_t)(np * HALF));
                __syncwarp();
                if (lane < np)
                    bulk_copy_g2s(v_ring + (uint32_t)(st * STAGE + lane * HALF),
                                  p.layer_base + (int64_t)id * p.page_stride + (int64_t)it.h * BLOCK + HALF, HALF, v_bar);
                id = next_id;
                next_id = load_id(kb + 2);
            }
        }
        // leave only when every copy has landed (normally long the case; after a failure it is not known which barrier one
        // still in flight will come through, and it is given time)
        for (int j = g > STAGES ? g - STAGES : 0; j < g; ++j) {
            wait(k_full + 8 * (j & (STAGES - 1)), (uint32_t)((j / STAGES) & 1), gave_up);
            wait(v_full + 8 * (j & (STAGES - 1)), (uint32_t)((j / STAGES) & 1), gave_up);
        }
        if (*gave_up) {
            const uint64_t t = global_timer_ns();
            while (global_timer_ns() - t < 1000000ull) __nanosleep(1000);
        }
    } else if (warp < 15) {
        // =================== queries ===================
        fewer_registers<48>();
        const int s = warp - 13;
        int turn = 0;                              // items of the tile before this one
        Item it;
        Items<SPLIT> items = {};
        for (int round = 0; items.at(it, p, tables, total, round, lane, TQ, per_item); ++round) {
            if (it.n[s] == 0) continue;
            if (turn > 0) wait(q_free + 8 * s, (uint32_t)((turn - 1) & 1), gave_up);
            // 8 lanes a row of 128 bytes: whole lines from memory, and no two lanes of a row's eight in one bank.  Rows r, r + 4, ...
            // of a lane: the token and head are counted along (a division per row made this the slowest part of an item).
            const int c = lane & 7, r4 = lane >> 3;
            int qi = r4 / G, g8 = r4 - qi * G;
            const int step_q = 4 / G, step_g = 4 - step_q * G;
            const uint16_t *src = p.Q + ((int64_t)(it.q_begin + it.q0 + s * TQ + qi) * p.Hq + (int64_t)it.h * G + g8) * D + c * 8;
            const int64_t step = (int64_t)(step_q * p.Hq + step_g) * D, wrap = (int64_t)(p.Hq - G) * D;
            const uint32_t dst = q_smem + (uint32_t)(s * Q_BYTES + r4 * 128);
            const uint32_t at[2] = {(uint32_t)((c ^ r4) * 16), (uint32_t)(512 + ((c ^ (r4 + 4)) * 16))};
            for (int r0 = 0; r0 < ROWS * 128; r0 += 1024) {
#pragma unroll
                for (int odd = 0; odd < 2; ++odd) {
                    if (qi < it.n[s])                      // (another row runs on whatever is there; nothing of it is stored)
#pragma unroll
                        for (int half = 0; half < D / 64; ++half)
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + at[odd] + (uint32_t)(r0 + half * ROWS * 128)), "l"(src + half * 64) : "memory");
                    qi += step_q;
                    g8 += step_g;
                    src += step;
                    if (g8 >= G) {
                        g8 -= G;
                        ++qi;
                        src += wrap;
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            fence_proxy_async();                           // the tensor core reads them through the async proxy
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full + 8 * s);
            ++turn;
        }
    } else {
        // =================== V rows that no row of the item sees ===================
        fewer_registers<48>();
        int g = 0;                                 // blocks before this one
        uint32_t landed = 0;                       // bit per ring stage: parity of the blocks that came through v_landed
        Item it;
        Items<SPLIT> items = {};
        for (int round = 0; items.at(it, p, tables, total, round, lane, TQ, per_item); ++round) {
            for (int kb = it.kb0; kb < it.blocks; ++kb, ++g) {
                const int st = g & (STAGES - 1), np = it.win.count - kb * KB < KB ? it.win.count - kb * KB : KB;
                const uint32_t bits = lane < np ? window_bits(it.win.page(kb * KB + lane), it.win.lo, it.n_keys, p.sinks) : 0xFFFFu;
                unsigned todo = __ballot_sync(FULL, bits != 0xFFFFu);
                if (!todo) continue;                           // (few have any: the first and the last of an item, and the sinks')
                wait(v_landed + 8 * st, (landed >> st) & 1u, gave_up);
                landed ^= 1u << st;
                for (; todo; todo &= todo - 1) {
                    const int j = __ffs(todo) - 1;
                    const uint32_t set = __shfl_sync(FULL, bits, j);
                    for (int i = lane; i < CH * PAGE; i += 32)
                        if (!((set >> (i & (PAGE - 1))) & 1u))
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(v_ring + (uint32_t)(st * STAGE + j * HALF + i * 16)), "r"(0u) : "memory");
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(v_full + 8 * st);
            }
        }
    }
    // ---- common exit ----
    if (SPLIT) {
        __syncwarp();
        if (warp >= 8) {                           // (the softmax warps were there before they joined the parts)
            cluster_arrive();
            cluster_wait();
        }
        cluster_arrive();                          // nobody leaves while its part is being read
        cluster_wait();
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && *gave_up) atomicOr(p.status, STATUS_TIMEOUT);
    if (warp == 8) {
        __syncwarp();
        tmem_dealloc(tmem, 512);
    }
}

}  // namespace

bool prefill_window_supported(int D, int G) { return (D == 64 || D == 128) && G >= 1 && G <= 8; }
int prefill_window_max_batch() { return MAX_BATCH; }

size_t prefill_window_smem_bytes(int D, int B)
{
    if (D != 64 && D != 128) return 0;
    return 1024 + 2 * (size_t)ROWS * D * 2 + 2 * STAGES * (size_t)KEYS * D * 2 + BAR_BYTES + 16 + 6 * (size_t)(B + 1) * sizeof(int32_t);
}

cudaError_t launch_prefill_window(const PrefillParams &p, int D, int G, int max_q_len, int sm_count, bool pdl, cudaStream_t s)
{
    if (!prefill_window_supported(D, G) || p.B > MAX_BATCH || max_q_len <= 0) return cudaErrorInvalidValue;
    // two tiles an item, or one where that leaves SMs without work
    const int64_t TQ = ROWS / G, most = (int64_t)p.B * p.Hkv;
    const int tiles = most * (((int64_t)max_q_len + 2 * TQ - 1) / (2 * TQ)) >= sm_count ? 2 : 1;
    int64_t ctas = most * (((int64_t)max_q_len + tiles * TQ - 1) / (tiles * TQ));
    if (ctas > sm_count) ctas = sm_count;
    // A cluster to an item, as large as leaves every CTA an SM and three key blocks, from 14 blocks on: joining costs some 5 us.  (A
    // cluster's SMs are of one GPC: of 8 CTAs 15 fit beside each other here, and 16 items of 66 blocks take 33 us in them, 24 in clusters of 4.)  (16 rows of one sequence, 32 / 8 heads, by blocks: 9 11.6 us, and 14.7 in a
    // cluster of two; 14 15.5, and 13.4 in one of four; 17 17.9 / 13.9; 33 30.2 / 14.6 in one of eight; 66 54 / 17.  Four
    // sequences: 14 15.9 / 16.3, 17 18.3 / 16.4, 66 55 / 25.)
    int64_t tokens = (int64_t)p.window + p.sinks + TQ, blocks;
    if (tokens > (int64_t)p.pt_stride * PAGE) tokens = (int64_t)p.pt_stride * PAGE;
    blocks = (tokens + KEYS - 1) / KEYS;
    int ranks = 1;
    while (tiles == 1 && blocks >= 14 && 2 * ranks <= MAX_RANKS && ctas * 2 * ranks <= (2 * ranks == 8 ? 6 : 7) * (int64_t)sm_count / 8 && blocks >= 3 * 2 * ranks) ranks *= 2;
    CUtensorMap k_map;
    if (!encode_k_map(&k_map, p.layer_base, p.page_stride, p.max_pages, p.Hkv, D)) return cudaErrorNotSupported;
    const size_t smem = prefill_window_smem_bytes(D, p.B);
    auto kern = ranks > 1 ? (D == 128 ? prefill_window_kernel<128, true> : prefill_window_kernel<64, true>)
                          : (D == 128 ? prefill_window_kernel<128, false> : prefill_window_kernel<64, false>);
    const cudaError_t e = ensure_dynamic_smem(kern, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(ctas * ranks));
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
    return cudaLaunchKernelEx(&cfg, kern, p, k_map, G, tiles, max_q_len);
}

}  // namespace skv
