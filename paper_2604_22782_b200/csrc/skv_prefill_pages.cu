// Attention of chunks over listed pages (skv_prefill_attn_pages) on the 5th-generation tensor cores: the row at position pos
// attends the tokens t <= pos of the pages that its run's list names for the kv head.
//
// An item is a list: (sequence, run of rows, kv head), one tile of 128 query rows, row r = token r / G, head r % G.  Lists of
// neighbouring tiles differ, so tiles share no K and V read (as the windowed kernel's two do) and a CTA has one item.  Two CTAs
// share an SM, 256 threads, 98 KB and 256 columns of tensor memory each: while one's softmax works the other's instructions do,
// and what an item's beginning and end leave idle the other CTA uses.  Eight warps:
//   warps 0-3  fetch the queries, then softmax: thread = row (TMEM lane)
//   warp 4     issues the scores Q K^T,  warp 5  the outputs P V
//   warp 6     copies K and V of the key blocks (64 keys = 4 listed pages); the entries' page ids are had 32 at a time
//   warp 7     zeroes the V rows of tokens that no row of the item sees, whatever they hold
// Operand layouts, softmax and waits are those of skv_prefill_window.cu.  Runs of one sequence and head are neighbours in the grid:
// their lists have pages in common, which are then in L2.
#include "skv_page_index.cuh"
#include "skv_prefill_parts.cuh"
#include "skv_tcgen05.cuh"

namespace skv {

namespace {

using namespace tc5;
using namespace chunk;

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int ROWS = 128;             // query rows of an item
constexpr int KB = 4;                 // pages of a key block
constexpr int KEYS = KB * PAGE;
constexpr int THREADS = 256;
constexpr int COL_O = 2 * KEYS;       // scores at columns 0 and 64, output from 128 on
constexpr int TMEM_COLS = 256;
constexpr int NO_PAGE = 0x07FFFFFF;   // no row sees a token of it

__host__ __device__ constexpr int stages_of(int D) { return D == 128 ? 2 : 4; }

// Dynamic shared memory: Q [D/64][128 rows][128 B] | K ring [8 groups][D/8 chunks][8 keys][16 B] | V ring [4 pages][V half] | barriers | words
template <int D>
constexpr size_t smem_bytes_of() { return 1024 + (size_t)ROWS * D * 2 + 2 * stages_of(D) * (size_t)KEYS * D * 2 + 5 * 8 * stages_of(D) + 3 * 16 + 8 + 32; }

template <int D>
__global__ void __launch_bounds__(THREADS, 2) prefill_pages_kernel(const __grid_constant__ PrefillParams p, const __grid_constant__ PageLists l,
                                                                      const __grid_constant__ CUtensorMap k_map, int G, int max_q_len)
{
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    constexpr int BLOCK = block_bytes(D), HALF = half_bytes(D), CH = D / 8, STAGES = stages_of(D);
    constexpr int Q_BYTES = ROWS * D * 2, STAGE = KEYS * D * 2;
    constexpr uint32_t IDESC_QK = instr_desc(ROWS, KEYS, false), IDESC_PV = instr_desc(ROWS, D, true);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(FULL, tid >> 5, 0);      // (known to be the same for the warp)
    const uint32_t base = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
    const uint32_t q_smem = base + pad, k_ring = q_smem + Q_BYTES, v_ring = k_ring + STAGES * STAGE, bars = v_ring + STAGES * STAGE;
    const uint32_t k_full = bars, v_full = k_full + 8 * STAGES, v_landed = v_full + 8 * STAGES, k_empty = v_landed + 8 * STAGES, v_empty = k_empty + 8 * STAGES;
    const uint32_t s_ready = v_empty + 8 * STAGES, p_ready = s_ready + 16, pv_done = p_ready + 16, q_full = pv_done + 16;
    uint8_t *words = smem_raw + pad + Q_BYTES + 2 * STAGES * STAGE + 5 * 8 * STAGES + 3 * 16 + 8;
    volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(words), *gave_up = tmem_slot + 1;
    volatile int32_t *item = reinterpret_cast<volatile int32_t *>(words + 8);      // rows, first position, tokens of the sequence, first row, entries

    if (tid == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(k_full + 8 * i, 1);
            mbar_init(v_full + 8 * i, 1);
            mbar_init(v_landed + 8 * i, 1);
            mbar_init(k_empty + 8 * i, 1);
            mbar_init(v_empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_ready + 8 * i, 1);
            mbar_init(p_ready + 8 * i, 4);
            mbar_init(pv_done + 8 * i, 1);
        }
        mbar_init(q_full, 4);
        *gave_up = 0;
        fence_barrier_init();
    }
    pdl_wait();
    const int pair = (int)blockIdx.x / l.per_seq, r = (int)blockIdx.x - pair * l.per_seq, b = pair / p.Hkv, h = pair - b * p.Hkv;
    const int64_t list_no = ((int64_t)b * l.per_seq + r) * p.Hkv + h;
    // The item, worked out by one warp and handed over in shared memory.  (Worked out by every thread for itself, the lesser of run and
    // the rows that are left came out as run in code compiled by nvcc 12.9.86, though not where it was also printed.)
    if (warp == 4) {
        const int q_begin = __ldg(p.cu_q + b), q_len = __ldg(p.cu_q + b + 1) - q_begin, n = __ldg(p.seq_lens + b);
        const int64_t at = (int64_t)r * l.run;                           // the run's first row
        int rows = 0, listed = 0;
        if (q_begin < 0 || q_len < 0 || q_len > n || q_len > max_q_len || (int64_t)n > (int64_t)p.pt_stride * PAGE) {
            if (r == 0 && h == 0 && lane == 0) atomicOr(p.status, STATUS_BOUNDS);
        } else if (at < q_len) {
            rows = q_len - (int)at < l.run ? q_len - (int)at : l.run;
            listed = __ldg(l.counts + list_no);
            if (listed > l.stride) {
                listed = l.stride;
                if (lane == 0) atomicOr(p.status, STATUS_BOUNDS);
            }
        }
        if (lane == 0) {
            item[0] = rows;
            item[1] = n - q_len + (int)at;
            item[2] = n;
            item[3] = q_begin + (int)at;
            item[4] = listed;
        }
        if (rows > 0 && listed > 0) {
            tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_slot)), TMEM_COLS);
            tmem_relinquish();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const int rows = item[0], p0 = item[1], p1 = p0 + rows - 1, pages = (item[2] + PAGE - 1) / PAGE, listed = item[4];
    const int64_t first_row = item[3];
    const uint16_t *q_rows = p.Q + (first_row * p.Hq + (int64_t)h * G) * D;
    uint16_t *out_rows = p.out + (first_row * p.Hq + (int64_t)h * G) * D;
    if (rows <= 0) return;
    if (listed <= 0) {
        for (int i = tid; i < rows * G * (D / 4); i += THREADS) {
            const int row = i / (D / 4), token = row / G;
            *reinterpret_cast<uint2 *>(out_rows + ((int64_t)token * p.Hq + row - token * G) * D + i % (D / 4) * 4) = make_uint2(0, 0);
        }
        return;
    }
    const int blocks = (listed + KB - 1) / KB;
    const int32_t *entries = l.lists + list_no * l.stride, *table = p.page_table + (int64_t)b * p.pt_stride;
    const uint32_t tmem = *tmem_slot;

    if (warp < 4) {
        more_registers<208>();
        // =================== queries ===================
        {
            // 8 lanes a row of 128 bytes; rows that the item does not have are zero
            const int c = lane & 7;
            for (int row = warp * 4 + (lane >> 3); row < ROWS; row += 16) {
                const int token = row / G;
                const uint16_t *src = q_rows + ((int64_t)token * p.Hq + row - token * G) * D + c * 8;
                const uint32_t dst = q_smem + (uint32_t)(row * 128 + ((c ^ (row & 7)) * 16));
#pragma unroll
                for (int half = 0; half < D / 64; ++half) {
                    if (token < rows)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + (uint32_t)(half * ROWS * 128)), "l"(src + half * 64) : "memory");
                    else
                        asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(dst + (uint32_t)(half * ROWS * 128)), "r"(0u) : "memory");
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            fence_proxy_async();                           // the tensor core reads them through the async proxy
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
        }
        // =================== softmax ===================
        const uint32_t lane_base = tmem + ((uint32_t)(warp * 32) << 16), output = lane_base + COL_O;
        const int token = tid / G, g = tid - token * G;
        const bool row_ok = token < rows;
        const int pos = row_ok ? p0 + token : 0x7FFFFFF0;
        const uint64_t scale2 = pair_of(p.scale_log2, p.scale_log2);
        float m_used = -INFINITY, l_sum = 0.f;
        auto entry = [&](int i) {                          // a listed page's number
            const int page = i < listed ? __ldg(entries + i) : NO_PAGE;
            return page >= 0 && page < pages ? page : NO_PAGE;
        };
        int page32 = entry(lane), next32 = entry(32 + lane);           // lane: entry 8 k + lane
        for (int kb = 0; kb < blocks; ++kb) {
            if (kb > 0 && (kb & 7) == 0) {
                page32 = next32;
                next32 = entry((kb + 8) * KB + lane);
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
            wait(s_ready + bar, phase, gave_up);
            tc_fence_after();
            uint32_t raw[2][32];
#pragma unroll
            for (int i = 0; i < 2; ++i) tmem_ld32(scores + 32 * i, raw[i]);
            tmem_wait_ld();
            if (!clear) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t bits = 0;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int left = pos + 1 - page[2 * i + j] * PAGE;
                        bits |= ((1u << (left < 0 ? 0 : left < PAGE ? left : PAGE)) - 1) << (PAGE * j);
                    }
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (!((bits >> c) & 1u)) raw[i][c] = 0xFF800000u;      // -inf
                }
            }
            // Against the reference as it stands; again if the block's maximum turns out to have run away from it.
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
                    float e0, e1;
                    if (c % BY_FMA == BY_FMA - 1) {
                        exp2_by_fma(x, e0, e1);
                    } else {
                        halves(x, e0, e1);
                        e0 = ex2(e0);
                        e1 = ex2(e1);
                    }
                    mx4[c & 3] = fmaxf(mx4[c & 3], fmaxf(s0, s1));
                    sum2[c & 1] = add2(sum2[c & 1], pair_of(e0, e1));
                    pk[c] = pack_bf16x2(e0, e1);
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
        fewer_registers<48>();
        if (warp < 6) {
            // =================== tensor-core issue: the whole warp walks along, one lane issues ===================
            const bool leader = elect_one(), values = warp == 5;
            const uint32_t output = tmem + COL_O;
            const uint64_t q_desc = swizzled_desc(q_smem);
            const uint64_t ring_desc = values ? smem_desc(v_ring, 128, PAGE * 16) : smem_desc(k_ring, 128, CH * 128);
            const uint32_t full = values ? v_full : k_full, empty = values ? v_empty : k_empty;
            if (!values) wait(q_full, 0, gave_up);
            for (int kb = 0; kb < blocks; ++kb) {
                const uint32_t st = (uint32_t)kb & (STAGES - 1), parity = (uint32_t)(kb / STAGES) & 1u;
                const uint32_t buf = (uint32_t)kb & 1u, turn = (uint32_t)(kb >> 1), bar = 8 * buf, scores = tmem + buf * KEYS;
                const uint64_t desc = ring_desc + (uint64_t)(st * (STAGE >> 4));
                wait(full + 8 * st, parity, gave_up);
                if (!values) {
                    if (kb >= 2) wait(pv_done + bar, (turn - 1) & 1u, gave_up);        // the buffer: P V two blocks back is over
                    tc_fence_after();
                    if (leader) {
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)
                            umma_ss(scores, q_desc + (uint64_t)(((ks >> 2) * ROWS * 128 + (ks & 3) * 32) >> 4), desc + (uint64_t)((ks * 2 * 128) >> 4), IDESC_QK, ks > 0);
                        tc_commit(s_ready + bar);
                        tc_commit(empty + 8 * st);
                    }
                } else {
                    wait(p_ready + bar, turn & 1u, gave_up);
                    tc_fence_after();
                    if (leader) {
                        const int np = listed - kb * KB;
#pragma unroll
                        for (int j = 0; j < KB; ++j)
                            if (j < np)
                                umma_ts(output, scores + (uint32_t)(8 * j), desc + (uint64_t)((j * HALF) >> 4), IDESC_PV, j > 0 || kb > 0 ? 1u : 0u);
                        tc_commit(pv_done + bar);
                        tc_commit(empty + 8 * st);
                    }
                }
                __syncwarp();
            }
            // the last commits arrive while the barriers are still there
            for (int j = blocks > STAGES ? blocks - STAGES : 0; j < blocks; ++j) wait(empty + 8 * (j & (STAGES - 1)), (uint32_t)((j / STAGES) & 1), gave_up);
        } else if (warp == 6) {
            // =================== copies of K and V ===================
            if (lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
            // lane: entry 8 k + lane; a page no row sees a token of is some page's copy, whose V is zeroed
            auto entry = [&](int i, int &id, bool &whole) {
                id = 0;
                whole = true;
                if (i >= listed) return;
                const int page = __ldg(entries + i);
                whole = page >= 0 && page < pages && page * PAGE + PAGE - 1 <= p1;
                if (page >= 0 && page < pages) id = __ldg(table + page);
                if (page < 0 || page >= pages || id < 0 || (int64_t)id >= p.max_pages) {
                    atomicOr(p.status, STATUS_BOUNDS);
                    id = 0;
                }
            };
            int id, next_id;
            bool whole, next_whole;
            entry(lane, id, whole);
            entry(32 + lane, next_id, next_whole);
            for (int kb = 0; kb < blocks; ++kb) {
                if (kb > 0 && (kb & 7) == 0) {
                    id = next_id;
                    whole = next_whole;
                    entry((kb + 8) * KB + lane, next_id, next_whole);
                }
                const int st = kb & (STAGES - 1), np = listed - kb * KB < KB ? listed - kb * KB : KB, j = lane - (kb & 7) * KB;
                const uint32_t again = (uint32_t)((kb / STAGES - 1) & 1);
                const bool mine = j >= 0 && j < np;
                // a block with tokens that no row sees passes through the hands of warp 7 first
                const bool partial = __any_sync(FULL, mine && !whole);
                const uint32_t v_bar = (partial ? v_landed : v_full) + 8 * st;
                if (kb >= STAGES) wait(k_empty + 8 * st, again, gave_up);
                if (lane == 0) mbar_expect_tx(k_full + 8 * st, (uint32_t)(np * HALF));
                __syncwarp();
                if (mine) tensor_copy_k(k_ring + (uint32_t)(st * STAGE + j * HALF), &k_map, h, id, k_full + 8 * st);
                if (kb >= STAGES) wait(v_empty + 8 * st, again, gave_up);
                if (lane == 0) mbar_expect_tx(v_bar, (uint32_t)(np * HALF));
                __syncwarp();
                if (mine)
                    bulk_copy_g2s(v_ring + (uint32_t)(st * STAGE + j * HALF), p.layer_base + (int64_t)id * p.page_stride + (int64_t)h * BLOCK + HALF, HALF, v_bar);
            }
            // leave only when every copy has landed (normally long the case; after a failure it is not known which barrier one
            // still in flight will come through, and it is given time)
            for (int j = blocks > STAGES ? blocks - STAGES : 0; j < blocks; ++j) {
                wait(k_full + 8 * (j & (STAGES - 1)), (uint32_t)((j / STAGES) & 1), gave_up);
                wait(v_full + 8 * (j & (STAGES - 1)), (uint32_t)((j / STAGES) & 1), gave_up);
            }
            if (*gave_up) {
                const uint64_t t = global_timer_ns();
                while (global_timer_ns() - t < 1000000ull) __nanosleep(1000);
            }
        } else {
            // =================== V rows that no row of the item sees ===================
            uint32_t landed = 0;                       // bit per ring stage: parity of the blocks that came through v_landed
            auto tokens = [&](int i) -> uint32_t {     // of entry i, those that some row sees
                if (i >= listed) return 0xFFFFu;
                const int page = __ldg(entries + i);
                if (page < 0 || page >= pages) return 0;
                const int left = p1 + 1 - page * PAGE;
                return (1u << (left < 0 ? 0 : left < PAGE ? left : PAGE)) - 1;
            };
            for (int kb0 = 0; kb0 < blocks; kb0 += 8) {
                const uint32_t bits = tokens(kb0 * KB + lane);
                unsigned todo = __ballot_sync(FULL, bits != 0xFFFFu);
                while (todo) {                         // (few have any: the last page of a list)
                    const int x = __ffs(todo) - 1, kb = kb0 + x / KB, st = kb & (STAGES - 1);
                    const unsigned block = todo & (((1u << KB) - 1) << (x / KB * KB));
                    wait(v_landed + 8 * st, (landed >> st) & 1u, gave_up);
                    landed ^= 1u << st;
                    for (unsigned rest = block; rest; rest &= rest - 1) {
                        const int y = __ffs(rest) - 1;
                        const uint32_t set = __shfl_sync(FULL, bits, y);
                        for (int i = lane; i < CH * PAGE; i += 32)
                            if (!((set >> (i & (PAGE - 1))) & 1u))
                                asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(v_ring + (uint32_t)(st * STAGE + (y & (KB - 1)) * HALF + i * 16)), "r"(0u) : "memory");
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(v_full + 8 * st);
                    todo &= ~block;
                }
            }
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

template <int D>
cudaError_t launch_t(const PrefillParams &p, const PageLists &l, int G, int max_q_len, bool pdl, cudaStream_t s)
{
    const int64_t ctas = (int64_t)p.B * l.per_seq * p.Hkv;
    if (ctas > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    CUtensorMap k_map;
    if (!encode_k_map(&k_map, p.layer_base, p.page_stride, p.max_pages, p.Hkv, D)) return cudaErrorNotSupported;
    auto kern = prefill_pages_kernel<D>;
    const size_t smem = smem_bytes_of<D>();
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
    return cudaLaunchKernelEx(&cfg, kern, p, l, k_map, G, max_q_len);
}

}  // namespace

size_t prefill_pages_smem_bytes(int D) { return D == 128 ? smem_bytes_of<128>() : D == 64 ? smem_bytes_of<64>() : 0; }

cudaError_t launch_prefill_pages(const PrefillParams &p, const PageLists &l, int D, int G, int max_q_len, bool pdl, cudaStream_t s)
{
    if (D == 128) return launch_t<128>(p, l, G, max_q_len, pdl, s);
    if (D == 64) return launch_t<64>(p, l, G, max_q_len, pdl, s);
    return cudaErrorInvalidValue;
}

}  // namespace skv
