// Attention of prompts and chunks over a sliding window with sinks (skv_prefill_attn_window) on the 5th-generation
// tensor cores: the row at position pos attends  t <= pos  and  (t > pos - window  or  t < sinks).
//
// An item is (sequence, kv head, two neighbouring tiles of 128 query rows): row r of a tile = token r / G, head r % G.
// The tiles share every K and V read.  A persistent CTA per SM takes items in turn; twelve warps:
//   warps 0-3, 4-7  softmax of tile 0 / tile 1: thread = row (TMEM lane)
//   warp 8          lane 0 issues the tensor-core instructions of both tiles
//   warp 9          copies K and V of the key blocks (128 keys = 8 pages of the item's list of pages, window_pages)
//   warp 10         copies the queries of the next item as soon as the last scores of this one are done
//   warp 11         blocks with tokens that no row of the item sees: zeroes their V rows, whatever they hold
// Shared memory: Q of both tiles, K ring and V ring of two blocks each.  K is brought in 256-byte pieces (16 keys x one
// 8-dim chunk) that interleave the pages by chunk, so that a block is ONE N = 128 operand: with N = 64 the tensor core reads
// 6 KB of operands per 32 cycles of work and waits for shared memory.  V pages are copied as they are: an MN-major operand.
// Tensor memory (512 columns): scores of tile 0 and 1 [128 each], overwritten in place by the probabilities (bf16), and
// the outputs of tile 0 and 1.
//
// While one tile's softmax runs, the tensor core works on the other's products: per tile and block  P V(kb), then
// Q K^T(kb + 1).  The tiles need not be in step -- a block that one tile does not see is skipped by that tile alone, and
// one may be an item ahead -- so the issuing thread polls: whichever instruction has its operands ready goes out.
// Blocks return to the copy warp in order, when neither tile needs them any more.
// Softmax as in skv_prefill_umma.cu: the reference maximum moves only when it has grown by more than 2^8, so O is rarely
// rescaled.  A row that has seen nothing yet counts from reference 0.
// Every wait is bounded and ends early when another warp has given up; copies in flight get their wait before the end.
#include "skv_common.cuh"
#include "skv_tcgen05.cuh"
#include "skv_walk.cuh"

#include <math.h>

namespace skv {

namespace {

using namespace tc5;

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int ROWS = 128;             // query rows of a tile
constexpr int KB = 8;                 // pages of a key block
constexpr int KEYS = KB * PAGE;
constexpr int THREADS = 384;
constexpr int COL_O = 2 * KEYS;       // scores of tile s at column 128 s, its output at 256 + 128 s
constexpr float RESCALE_STEP = 8.f;
constexpr int MAX_BATCH = 1024;       // sequences of a launch: their tables are in shared memory

__host__ __device__ constexpr uint32_t instr_desc(int M, int N, bool b_mn_major)
{
    return (1u << 4) /* D fp32 */ | (1u << 7) /* A bf16 */ | (1u << 10) /* B bf16 */ |
           ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// a look that never suspends the thread
__device__ __forceinline__ bool test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// bounded (two seconds); ends early when another warp of the CTA has given up
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile uint32_t *gave_up)
{
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return true;
        if (*gave_up || global_timer_ns() - t0 > 2000000000ull) return false;
    }
}

// What an item is made of.
struct Item {
    int b, h, q_begin;      // sequence, kv head, the sequence's first query row
    int q0, q_len;          // first token of the item among the sequence's new ones; all of those
    int pos0;               // position of the sequence's first new token
    int n[2];               // tokens of the two tiles
    int n_keys;             // keys below this one are visible to some row
    int blocks;
    WindowPages win;
    // tokens of tile s: positions first(s) .. last(s)
    __device__ __forceinline__ int first(int s, int TQ) const { return pos0 + q0 + s * TQ; }
    __device__ __forceinline__ int last(int s, int TQ) const { return first(s, TQ) + n[s] - 1; }
};

struct Tables {             // in shared memory, per sequence
    const int32_t *prefix;  // items per kv head of the sequences before
    const int32_t *q_begin, *q_len, *lens;
};

// item x of the call; per_item: tokens of an item
__device__ __forceinline__ Item item_at(const PrefillParams &p, const Tables &t, int64_t x, int TQ, int per_item)
{
    const Cursor c = locate(t.prefix, p.B, p.Hkv, x);
    Item it;
    it.b = c.b;
    it.h = c.h;
    it.q_begin = t.q_begin[c.b];
    it.q_len = t.q_len[c.b];
    it.q0 = (c.pages - 1 - c.pg) * per_item;                  // the sequence's last tokens, with the most keys, first
    it.pos0 = t.lens[c.b] - it.q_len;
    const int left = it.q_len - it.q0;
    it.n[0] = left < TQ ? left : TQ;
    const int second = (left < per_item ? left : per_item) - TQ;
    it.n[1] = second > 0 ? second : 0;
    it.n_keys = it.pos0 + it.q0 + it.n[0] + it.n[1];
    it.win = window_pages(it.pos0 + it.q0, it.n_keys, p.window, p.sinks);
    it.blocks = (it.win.count + KB - 1) / KB;
    return it;
}

// whether some row of tile s sees a key of block kb
__device__ __forceinline__ bool needs(const Item &it, int s, int kb, int TQ, int window, int sinks)
{
    if (it.n[s] == 0) return false;
    const int j0 = kb * KB, j1 = (j0 + KB < it.win.count ? j0 + KB : it.win.count) - 1;
    if (sinks > 0 && j0 < it.win.sink_pages) return true;
    const int first = it.first(s, TQ), lo = first >= window ? first - window + 1 : 0;
    return it.win.page(j1) * PAGE + PAGE > lo && it.win.page(j0) * PAGE <= it.last(s, TQ);
}

// A tile's walk over its blocks, item by item.  Every role that walks it gets the same sequence.
struct Walk {
    int64_t x;              // item
    int kb;                 // block of the item
    int g;                  // blocks of the CTA before it, of either tile
    int turn;               // items of this tile before this one
    bool first, last;       // block of this tile in the item
    bool over;
    Item it;
};

__device__ __forceinline__ void find(Walk &w, const PrefillParams &p, const Tables &t, int s, int64_t total, int TQ, int per_item, int from)
{
    // the next block >= from of the item that the tile needs, else the first one of the next item
    for (;;) {
        int kb = from;
        if (w.it.n[s] > 0)
            while (kb < w.it.blocks && !needs(w.it, s, kb, TQ, p.window, p.sinks)) ++kb;
        else
            kb = w.it.blocks;
        if (kb < w.it.blocks) {
            w.g += kb - w.kb;
            w.kb = kb;
            int after = kb + 1;
            while (after < w.it.blocks && !needs(w.it, s, after, TQ, p.window, p.sinks)) ++after;
            w.last = after >= w.it.blocks;
            return;
        }
        w.g += w.it.blocks - w.kb;
        w.kb = 0;
        if (w.it.n[s] > 0) ++w.turn;
        w.first = true;
        w.x += gridDim.x;
        if (w.x >= total) {
            w.over = true;
            return;
        }
        w.it = item_at(p, t, w.x, TQ, per_item);
        from = 0;
    }
}

__device__ __forceinline__ Walk begin_walk(const PrefillParams &p, const Tables &t, int s, int64_t total, int TQ, int per_item)
{
    Walk w;
    w.x = blockIdx.x;
    w.kb = w.g = w.turn = 0;
    w.first = true;
    w.last = false;
    w.over = w.x >= total;
    if (w.over) return w;
    w.it = item_at(p, t, w.x, TQ, per_item);
    find(w, p, t, s, total, TQ, per_item, 0);
    return w;
}

__device__ __forceinline__ void next_block(Walk &w, const PrefillParams &p, const Tables &t, int s, int64_t total, int TQ, int per_item)
{
    w.first = false;
    find(w, p, t, s, total, TQ, per_item, w.kb + 1);
}

// Dynamic shared memory: Q [2][D/8 chunks][128 rows][16 B] | K ring [2][D/8][128 keys][16 B] | V ring [2][8 pages][V half]
//                        | barriers | tensor-memory address, gave_up | tables [4][B + 1]
template <int D>
__global__ void __launch_bounds__(THREADS, 1) prefill_window_kernel(const __grid_constant__ PrefillParams p, int G, int tiles, int max_q_len)
{
    extern __shared__ __align__(128) uint8_t smem_raw[];
    constexpr int BLOCK = block_bytes(D), HALF = half_bytes(D), CH = D / 8;
    constexpr int Q_BYTES = ROWS * D * 2, STAGE = KEYS * D * 2;
    constexpr uint32_t IDESC_QK = instr_desc(ROWS, KEYS, false), IDESC_PV = instr_desc(ROWS, D, true);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int TQ = ROWS / G, per_item = TQ * tiles;

    const uint32_t base = smem_u32(smem_raw);
    const uint32_t pad = (128u - (base & 127u)) & 127u;
    const uint32_t q_smem = base + pad, k_ring = q_smem + 2 * Q_BYTES, v_ring = k_ring + 2 * STAGE, bars = v_ring + 2 * STAGE;
    // one barrier per ring stage: copied, given back; per tile: the rest
    const uint32_t k_full = bars, v_full = bars + 16, v_landed = bars + 32, k_empty = bars + 48, v_empty = bars + 64;
    const uint32_t q_full = bars + 80, q_free = bars + 96, s_ready = bars + 112, p_ready = bars + 128, o_ready = bars + 144, o_free = bars + 160;
    uint8_t *words = smem_raw + pad + 2 * Q_BYTES + 4 * STAGE + 176;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(words), *gave_up = tmem_slot + 1;
    int32_t *prefix = reinterpret_cast<int32_t *>(words + 16), *q_begin = prefix + p.B + 1, *q_len = q_begin + p.B + 1, *lens = q_len + p.B + 1;
    const Tables tables = {prefix, q_begin, q_len, lens};

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(k_full + 8 * i, 1);
            mbar_init(v_full + 8 * i, 1);
            mbar_init(v_landed + 8 * i, 1);
            mbar_init(k_empty + 8 * i, 1);
            mbar_init(v_empty + 8 * i, 1);
            mbar_init(q_full + 8 * i, 1);
            mbar_init(q_free + 8 * i, 1);
            mbar_init(s_ready + 8 * i, 1);
            mbar_init(p_ready + 8 * i, 4);
            mbar_init(o_ready + 8 * i, 1);
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
    // the sequences' tables: items per kv head of the sequences before (warp 0)
    if (warp == 0) {
        int carry = 0;
        for (int i0 = 0; i0 < p.B; i0 += 32) {
            const int i = i0 + lane;
            int items = 0;
            if (i < p.B) {
                const int qb = __ldg(p.cu_q + i), ql = __ldg(p.cu_q + i + 1) - qb, n = __ldg(p.seq_lens + i);
                const bool fits = ql >= 0 && ql <= n && ql <= max_q_len && (int64_t)n <= (int64_t)p.pt_stride * PAGE;
                if (!fits && blockIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
                items = fits ? (ql + per_item - 1) / per_item : 0;
                q_begin[i] = qb;
                q_len[i] = ql;
                lens[i] = n;
            }
            int sum = items;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int u = __shfl_up_sync(FULL, sum, d);
                if (lane >= d) sum += u;
            }
            if (i < p.B) prefix[i + 1] = carry + sum;
            carry += __shfl_sync(FULL, sum, 31);
        }
        if (lane == 0) prefix[0] = 0;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const int64_t total = (int64_t)prefix[p.B] * p.Hkv;
    auto give_up = [&]() {
        atomicOr(p.status, STATUS_TIMEOUT);
        *gave_up = 1;
    };
    int copied = 0;                                // copy warp: blocks sent

    if (warp < 8) {
        // =================== softmax ===================
        const int s = warp >> 2, row = tid & (ROWS - 1);
        const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16), scores = lane_base + (uint32_t)(s * KEYS),
                       output = lane_base + (uint32_t)(COL_O + s * KEYS);
        const int qi = row / G, g = row - qi * G;
        float m_used = -INFINITY, l_sum = 0.f;
        bool ok = true;
        int count = 0;                             // blocks of this tile so far
        for (Walk w = begin_walk(p, tables, s, total, TQ, per_item); !w.over && ok; ++count) {
            const Item &it = w.it;
            if (w.first) {
                m_used = -INFINITY;
                l_sum = 0.f;
            }
            const bool row_ok = qi < it.n[s];
            const int pos = row_ok ? it.first(s, TQ) + qi : 0x7FFFFFFF;
            ok = __all_sync(FULL, wait(s_ready + 8 * s, (uint32_t)(count & 1), gave_up));
            if (!ok) break;
            tc_fence_after();
            uint32_t raw[4][32];
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_ld32(scores + 32 * i, raw[i]);
            tmem_wait_ld();
            // most blocks are visible to every row of the tile: neither the causal edge, nor the window's, nor a gap or an end
            const int j0 = w.kb * KB, np = it.win.count - j0 < KB ? it.win.count - j0 : KB;
            const int t0 = it.win.page(j0) * PAGE, t1 = it.win.page(j0 + np - 1) * PAGE + PAGE - 1;
            const int last = it.last(s, TQ), lo_last = last >= p.window ? last - p.window + 1 : 0;
            const bool whole = np == KB && t1 - t0 == KEYS - 1 && t1 <= it.first(s, TQ) && (t0 >= lo_last || t1 < p.sinks);
            if (!whole) {
                const int lo = pos >= p.window ? pos - p.window + 1 : 0;
#pragma unroll
                for (int j = 0; j < KB; ++j) {
                    const uint32_t bits = j < np ? window_bits(it.win.page(j0 + j), lo, pos < 0x7FFFFFFF ? pos + 1 : pos, p.sinks) : 0u;
#pragma unroll
                    for (int i = 0; i < PAGE; ++i)
                        if (!((bits >> i) & 1u)) raw[j / 2][(j & 1) * PAGE + i] = 0xFF800000u;      // -inf
                }
            }
            float mx4[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                mx4[i] = __uint_as_float(raw[i][0]);
#pragma unroll
                for (int c = 1; c < 32; ++c) mx4[i] = fmaxf(mx4[i], __uint_as_float(raw[i][c]));
            }
            const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * p.scale_log2;      // the scale is positive
            float alpha = 1.f;
            const bool move = mx > m_used + RESCALE_STEP;      // also true for the first key that the row sees
            if (move) {
                alpha = fast_exp2(m_used - mx);                // 0 when m_used = -inf
                m_used = mx;
            }
            if (!w.first && __any_sync(FULL, move)) {
                // (the scores of this block were issued after P V of the one before: O holds all blocks so far)
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
            const float neg_m = m_used == -INFINITY ? 0.f : -m_used;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t pk[32];
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    const int i = 2 * half + (c >> 4), cc = (2 * c) & 31;
                    const float p0 = fast_exp2(fmaf(__uint_as_float(raw[i][cc]), p.scale_log2, neg_m));
                    const float p1 = fast_exp2(fmaf(__uint_as_float(raw[i][cc + 1]), p.scale_log2, neg_m));
                    sum[c & 3] += p0 + p1;
                    pk[c] = pack_bf16x2(p0, p1);
                }
                tmem_st32(scores + 32 * half, pk);             // P over the first half of the tile's scores
            }
            l_sum = l_sum * alpha + ((sum[0] + sum[1]) + (sum[2] + sum[3]));
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_ready + 8 * s);
            if (w.last) {
                ok = __all_sync(FULL, wait(o_ready + 8 * s, (uint32_t)(w.turn & 1), gave_up));
                if (!ok) break;
                tc_fence_after();
                const float inv = 1.f / l_sum;
                uint16_t *dst = p.out + ((int64_t)(it.q_begin + it.q0 + s * TQ + qi) * p.Hq + (int64_t)it.h * G + g) * D;
#pragma unroll
                for (int q = 0; q < D / 32; ++q) {
                    uint32_t ov[32];
                    tmem_ld32(output + 32 * q, ov);
                    tmem_wait_ld();
                    if (q == D / 32 - 1) {                     // the output's columns may be used again
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(o_free + 8 * s);
                    }
                    if (row_ok) {
#pragma unroll
                        for (int c = 0; c < 32; c += 8) {
                            uint4 v;
                            v.x = pack_bf16x2(__uint_as_float(ov[c]) * inv, __uint_as_float(ov[c + 1]) * inv);
                            v.y = pack_bf16x2(__uint_as_float(ov[c + 2]) * inv, __uint_as_float(ov[c + 3]) * inv);
                            v.z = pack_bf16x2(__uint_as_float(ov[c + 4]) * inv, __uint_as_float(ov[c + 5]) * inv);
                            v.w = pack_bf16x2(__uint_as_float(ov[c + 6]) * inv, __uint_as_float(ov[c + 7]) * inv);
                            *reinterpret_cast<uint4 *>(dst + 32 * q + c) = v;
                        }
                    }
                }
            }
            next_block(w, p, tables, s, total, TQ, per_item);
        }
        if (!ok && lane == 0) give_up();
    } else if (warp == 8) {
        // =================== tensor-core issue ===================
        if (lane == 0) {
            struct Block { int g, np, turn; bool first, last; };
            Walk w[2];
            Block cur[2];
            bool held[2] = {false, false};         // scores are out, P V of them is not
            int count[2] = {0, 0};
            int freed_k = -1, freed_v = -1;        // blocks given back
#pragma unroll
            for (int s = 0; s < 2; ++s) w[s] = begin_walk(p, tables, s, total, TQ, per_item);
            uint64_t t0 = global_timer_ns();
            bool ok = true;
            int idle = 0;
            while (ok && !(w[0].over && w[1].over && !held[0] && !held[1])) {
                bool issued = false;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (held[s]) {
                        const Block &c = cur[s];
                        const int st = c.g & 1;
                        // P of this block; V (the stage's phase before this one is over: the block before it has been given back);
                        // for an item's first block, the output of the item before has been read
                        if (test(p_ready + 8 * s, (uint32_t)(count[s] & 1)) && c.g <= freed_v + 2 &&
                            test(v_full + 8 * st, (uint32_t)((c.g >> 1) & 1)) &&
                            (!c.first || c.turn == 0 || test(o_free + 8 * s, (uint32_t)((c.turn - 1) & 1)))) {
                            tc_fence_after();
                            for (int j = 0; j < c.np; ++j)
                                umma_ts(tmem + (uint32_t)(COL_O + s * KEYS), tmem + (uint32_t)(s * KEYS + 8 * j),
                                        smem_desc(v_ring + (uint32_t)(st * STAGE + j * HALF), 128, PAGE * 16), IDESC_PV, (c.first && j == 0) ? 0u : 1u);
                            if (c.last) tc_commit(o_ready + 8 * s);
                            held[s] = false;
                            ++count[s];
                            issued = true;
                        }
                    }
                    if (!held[s] && !w[s].over) {
                        const int gk = w[s].g, st = gk & 1;
                        if (gk <= freed_k + 2 && test(k_full + 8 * st, (uint32_t)((gk >> 1) & 1)) &&
                            (!w[s].first || test(q_full + 8 * s, (uint32_t)(w[s].turn & 1)))) {
                            tc_fence_after();
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks)
                                umma_ss(tmem + (uint32_t)(s * KEYS), smem_desc(q_smem + (uint32_t)(s * Q_BYTES + ks * 2 * ROWS * 16), ROWS * 16, 128),
                                        smem_desc(k_ring + (uint32_t)(st * STAGE + ks * 2 * KEYS * 16), KEYS * 16, 128), IDESC_QK, ks > 0);
                            tc_commit(s_ready + 8 * s);
                            if (w[s].last) tc_commit(q_free + 8 * s);
                            const int np = w[s].it.win.count - w[s].kb * KB;
                            cur[s] = {gk, np < KB ? np : KB, w[s].turn, w[s].first, w[s].last};
                            held[s] = true;
                            next_block(w[s], p, tables, s, total, TQ, per_item);
                            issued = true;
                        }
                    }
                }
                if (issued) {
                    // blocks that neither tile needs any more go back, in order (a commit arrives when all work issued so far is done)
                    const int k0 = w[0].over ? 0x7FFFFFFF : w[0].g, k1 = w[1].over ? 0x7FFFFFFF : w[1].g;
                    const int v0 = held[0] ? cur[0].g : k0, v1 = held[1] ? cur[1].g : k1;
                    int to_k = (k0 < k1 ? k0 : k1) - 1, to_v = (v0 < v1 ? v0 : v1) - 1;
                    const int most_k = freed_k + 2, most_v = freed_v + 2;        // (never more than the ring holds)
                    to_k = to_k < most_k ? to_k : most_k;
                    to_v = to_v < most_v ? to_v : most_v;
                    while (freed_k < to_k) tc_commit(k_empty + 8 * (++freed_k & 1));
                    while (freed_v < to_v) tc_commit(v_empty + 8 * (++freed_v & 1));
                    idle = 0;
                } else if (++idle == 1024) {
                    idle = 0;
                    if (*gave_up) ok = false;
                    const uint64_t now = global_timer_ns();
                    if (now - t0 > 2000000000ull) ok = false;
                }
                if (issued) t0 = global_timer_ns();
            }
            // the last commits arrive while the barriers are still there
            if (ok && freed_k >= 0) ok = wait(k_empty + 8 * (freed_k & 1), (uint32_t)((freed_k >> 1) & 1), gave_up);
            if (ok && freed_v >= 0) ok = wait(v_empty + 8 * (freed_v & 1), (uint32_t)((freed_v >> 1) & 1), gave_up);
            if (!ok) give_up();
        }
        __syncwarp();
    } else if (warp == 9) {
        // =================== copies of K and V ===================
        bool ok = true;
        int g = 0;
        for (int64_t x = blockIdx.x; x < total && ok; x += gridDim.x) {
            const Item it = item_at(p, tables, x, TQ, per_item);
            const int32_t *row = p.page_table + (int64_t)it.b * p.pt_stride;
            auto load_id = [&](int kb) -> int {                // lane j: page j of a block
                const int j = kb * KB + lane;
                if (lane >= KB || j >= it.win.count) return 0;
                const int id = __ldg(row + it.win.page(j));
                if (id >= 0 && (int64_t)id < p.max_pages) return id;
                atomicOr(p.status, STATUS_BOUNDS);
                return 0;
            };
            int id = load_id(0);
            for (int kb = 0; kb < it.blocks && ok; ++kb, ++g) {
                const int st = g & 1, np = it.win.count - kb * KB < KB ? it.win.count - kb * KB : KB;
                const uint32_t again = (uint32_t)(((g >> 1) - 1) & 1);
                bool partial = false;
                if (lane < np) partial = window_bits(it.win.page(kb * KB + lane), it.win.lo, it.n_keys, p.sinks) != 0xFFFFu;
                partial = __any_sync(FULL, partial);
                if (g >= 2) ok = __all_sync(FULL, wait(k_empty + 8 * st, again, gave_up));
                if (!ok) break;
                if (lane == 0) mbar_expect_tx(k_full + 8 * st, (uint32_t)(np * HALF));
                __syncwarp();
                // a piece: 16 keys of one chunk, 256 bytes of the page; lane = (page, every 4th chunk)
                const int pj = lane & 7;
                const int page_id = __shfl_sync(FULL, id, pj);
                if (pj < np) {
                    const uint8_t *src = p.layer_base + (int64_t)page_id * p.page_stride + (int64_t)it.h * BLOCK;
                    const uint32_t dst = k_ring + (uint32_t)(st * STAGE + pj * PAGE * 16);
#pragma unroll
                    for (int c = lane >> 3; c < CH; c += 4) bulk_copy_g2s(dst + (uint32_t)(c * KEYS * 16), src + c * PAGE * 16, PAGE * 16, k_full + 8 * st);
                }
                const int next_id = load_id(kb + 1);
                if (g >= 2) ok = __all_sync(FULL, wait(v_empty + 8 * st, again, gave_up));
                const uint32_t bar = (partial ? v_landed : v_full) + 8 * st;
                if (ok) {
                    if (lane == 0) mbar_expect_tx(bar, (uint32_t)(np * HALF));
                    __syncwarp();
                    if (lane < np)
                        bulk_copy_g2s(v_ring + (uint32_t)(st * STAGE + lane * HALF),
                                      p.layer_base + (int64_t)id * p.page_stride + (int64_t)it.h * BLOCK + HALF, HALF, bar);
                }
                copied = g + 1;
                id = next_id;
            }
        }
        if (!ok && lane == 0) give_up();
        // leave only when every copy has landed (normally long the case)
        for (int j = copied > 2 ? copied - 2 : 0; j < copied; ++j) {
            mbar_wait_bounded(k_full + 8 * (j & 1), (uint32_t)((j >> 1) & 1));
            if (ok) mbar_wait_bounded(v_full + 8 * (j & 1), (uint32_t)((j >> 1) & 1));
        }
        if (!ok) {
            // (after a failure a block's V may have come through either barrier, or not have been sent for: give it time instead)
            const uint64_t t = global_timer_ns();
            while (global_timer_ns() - t < 1000000ull) __nanosleep(1000);
        }
    } else if (warp == 10) {
        // =================== queries ===================
        bool ok = true;
        int turn[2] = {0, 0};
        for (int64_t x = blockIdx.x; x < total && ok; x += gridDim.x) {
            const Item it = item_at(p, tables, x, TQ, per_item);
            for (int s = 0; s < 2 && ok; ++s) {
                if (it.n[s] == 0) continue;
                if (turn[s] > 0) ok = __all_sync(FULL, wait(q_free + 8 * s, (uint32_t)((turn[s] - 1) & 1), gave_up));
                if (!ok) break;
                for (int r0 = 0; r0 < ROWS; r0 += 32) {
                    const int r = r0 + lane, qi = r / G, g = r - qi * G;
                    if (qi >= it.n[s]) continue;               // (such a row runs on whatever is there; nothing of it is stored)
                    const uint16_t *src = p.Q + ((int64_t)(it.q_begin + it.q0 + s * TQ + qi) * p.Hq + (int64_t)it.h * G + g) * D;
                    const uint32_t dst = q_smem + (uint32_t)(s * Q_BYTES + r * 16);
#pragma unroll
                    for (int c = 0; c < CH; ++c)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + (uint32_t)(c * ROWS * 16)), "l"(src + c * 8) : "memory");
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                fence_proxy_async();                           // the tensor core reads Q through the async proxy
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full + 8 * s);
                ++turn[s];
            }
        }
        if (!ok && lane == 0) give_up();
    } else {
        // =================== V rows that no row of the item sees ===================
        bool ok = true;
        int g = 0, seen[2] = {0, 0};
        for (int64_t x = blockIdx.x; x < total && ok; x += gridDim.x) {
            const Item it = item_at(p, tables, x, TQ, per_item);
            for (int kb = 0; kb < it.blocks && ok; ++kb, ++g) {
                const int st = g & 1, np = it.win.count - kb * KB < KB ? it.win.count - kb * KB : KB;
                const uint32_t bits = lane < np ? window_bits(it.win.page(kb * KB + lane), it.win.lo, it.n_keys, p.sinks) : 0xFFFFu;
                unsigned todo = __ballot_sync(FULL, bits != 0xFFFFu);
                if (!todo) continue;
                ok = __all_sync(FULL, wait(v_landed + 8 * st, (uint32_t)(seen[st] & 1), gave_up));
                if (!ok) break;
                ++seen[st];
                for (; todo; todo &= todo - 1) {
                    const int j = __ffs(todo) - 1;
                    const uint32_t set = __shfl_sync(FULL, bits, j);
                    const uint32_t sV = v_ring + (uint32_t)(st * STAGE + j * HALF);
                    for (int i = lane; i < CH * PAGE; i += 32)
                        if (!((set >> (i & (PAGE - 1))) & 1u))
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(sV + (uint32_t)(i * 16)), "r"(0u) : "memory");
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(v_full + 8 * st);
            }
        }
        if (!ok && lane == 0) give_up();
    }
    // ---- common exit ----
    tc_fence_before();
    __syncthreads();
    if (warp == 10) asm volatile("cp.async.wait_group 0;" ::: "memory");
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
    return 128 + 2 * (size_t)ROWS * D * 2 + 4 * (size_t)KEYS * D * 2 + 176 + 16 + 4 * (size_t)(B + 1) * sizeof(int32_t);
}

cudaError_t launch_prefill_window(const PrefillParams &p, int D, int G, int max_q_len, int sm_count, bool pdl, cudaStream_t s)
{
    if (!prefill_window_supported(D, G) || p.B > MAX_BATCH || max_q_len <= 0) return cudaErrorInvalidValue;
    // two tiles an item, or one where that leaves SMs without work
    const int64_t TQ = ROWS / G, most = (int64_t)p.B * p.Hkv;
    const int tiles = most * (((int64_t)max_q_len + 2 * TQ - 1) / (2 * TQ)) >= sm_count ? 2 : 1;
    int64_t ctas = most * (((int64_t)max_q_len + tiles * TQ - 1) / (tiles * TQ));
    if (ctas > sm_count) ctas = sm_count;
    const size_t smem = prefill_window_smem_bytes(D, p.B);
    auto kern = D == 128 ? prefill_window_kernel<128> : prefill_window_kernel<64>;
    const cudaError_t e = ensure_dynamic_smem(kern, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, p, G, tiles, max_q_len);
}

}  // namespace skv
