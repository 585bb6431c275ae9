// Decode attention over listed pages (skv_decode_attn_pages): Eq. (3.1) over the tokens of the pages that a list names for
// each (row, kv head), and the same for rows of a chunk, a row as a sequence that ends with its own token
// (skv_prefill_attn_pages where that is the quicker way).
//
// A segment -- a (row, kv head) with its list -- is one piece of work of a CTA's warps or, where the segments do not fill the GPU,
// of a cluster of CTAs, as over a window (skv_decode_window.cu): the warps take the listed pages in turn through
// rings of bulk copies of their own and the states are joined in shared memory.  Two loads stand between a warp and its first
// page, the list's entry and the page table's: a lane has them done for a page of its own, for 32 pages ahead.
// Probabilities: fp32 on the CUDA cores; on the tensor cores, whose operands are of V's type, two bf16 terms, the second in the half of the instruction's
// rows that the heads leave empty, at 0 to 2 % of the time (one term: 2^-8 of every weight, which showed beside the result's own rounding);
// on FP8 pages f16 relative to a power of two, 2^-11 of a weight.
// Measured, 8 kv heads of 128, 32 query heads: one sequence, 128 pages 7.5 us (launch, count, entry, page id, copies, cluster exchange); 32 sequences
// 44.6 us, 6.0 TB/s; 128 sequences of 256 FP8 pages 185 us, 6.0 TB/s (198 in a long loop, at the clocks that the power limit leaves).
// Registers: of 128 dims the 8-warp form has 128 and spills some 50 to 130 bytes, FP8 pages some 40 (two and four CTAs to an SM count for more).
#include "skv_decode_states.cuh"
#include "skv_page_index.cuh"
#include "skv_segment.cuh"
#include <atomic>
#include <type_traits>

namespace skv {

namespace {

// What a warp does with what it has copied: a page at a time on bf16 pages.
template <class State>
struct ByPage : State {
    static constexpr int PAGES = 1;
    __device__ __forceinline__ void fold_unit(uint32_t blk, uint32_t seen, float scale_log2, int lane) { State::page_bits(blk, seen, scale_log2, lane); }
};

// FP8 pages, two at a time: one softmax step, one turn of the ring for both.  Arithmetic and token orders are Fp8State's -- codes to f16,
// K's scales on the scores, V's on the probabilities relative to c, the power of two at or above every V scale so far --, but the
// output is transposed, O^T += V^T P^T, with the dims as the instruction's 16 rows and the heads as its 8 columns: half as many
// instructions and registers as with the heads as half-empty rows.  A thread's probabilities, head g and tokens 4 tig .. 4 tig + 3, are
// the column operand as they are.
// What bounds it is issue: 430 instructions a page taken one by one, 314 by twos.  (The same on E4M3 operands, mma.sync's e4m3 form, is no way out: it
// is some 14 instructions of its own, 420 a page in all.)
template <int D>
struct Fp8PairState {
    static constexpr int PAGES = 2, BLOCK = fp8_block_bytes(D);
    static constexpr int KS = D / 16, DT = D / 4;       // k-steps of Q K^T; dims per thread of a quad
    static constexpr float STEP = 8.f;                  // the reference follows a maximum 2^8 above it
    uint32_t qa[KS][2];                                 // f16x2: dims DT tig + 4 ks + {0, 1} and + {2, 3} of Q / qmax, head g
    float o[D / 16][4];                                 // dims 16 i + g and 16 i + 8 + g, of heads 2 tig and 2 tig + 1 each
    float m, l, qmax, cs;                               // of head g

    __device__ __forceinline__ void begin(const DecodeParams &p, int b, int h, int G, int lane)
    {
        Fp8State<D> s;
        s.begin(p, b, h, G, lane);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qa[ks][0] = s.qa[ks][0];
            qa[ks][1] = s.qa[ks][1];
        }
        qmax = s.qmax;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
        m = -INFINITY;
        l = 0.f;
        cs = 0.f;
    }

    // blk: two pages' blocks; seen: the tokens in use of the first, and of the second << 16 (not both none)
    __device__ __forceinline__ void fold_unit(uint32_t blk, uint32_t seen, float scale_log2, int lane)
    {
        const int g = lane >> 2, tig = lane & 3, tok = 4 * (g >> 1) + (g & 1);
        const float qs = qmax * scale_log2;
        float v[8], sv[8];                              // tokens 4 tig .. 4 tig + 3 of each page: scores, V scales
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t page = blk + (uint32_t)(j * BLOCK);
            const uint32_t k0 = page + (uint32_t)((tok >> 3) * 8 * D + (DT / 16) * tig * 128 + (tok & 7) * 16), k1 = k0 + 2 * 16;
            uint32_t w0[DT / 4], w1[DT / 4];
#pragma unroll
            for (int c = 0; c < DT / 16; ++c) {
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w0[4 * c]), "=r"(w0[4 * c + 1]), "=r"(w0[4 * c + 2]), "=r"(w0[4 * c + 3]) : "r"(k0 + 128 * c));
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w1[4 * c]), "=r"(w1[4 * c + 1]), "=r"(w1[4 * c + 2]), "=r"(w1[4 * c + 3]) : "r"(k1 + 128 * c));
            }
            float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint32_t b0, b1;
                e4m3x4_to_f16x2(w0[ks], b0, b1);
                mma_f16_16816(s0, qa[ks][0], 0u, qa[ks][1], 0u, b0, b1);
                e4m3x4_to_f16x2(w1[ks], b0, b1);
                mma_f16_16816(s1, qa[ks][0], 0u, qa[ks][1], 0u, b0, b1);
            }
            float4 sk;
            asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(sk.x), "=f"(sk.y), "=f"(sk.z), "=f"(sk.w) : "r"(page + (uint32_t)(fp8_ks_off(D) + 16 * tig)));
            asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(sv[4 * j]), "=f"(sv[4 * j + 1]), "=f"(sv[4 * j + 2]), "=f"(sv[4 * j + 3])
                         : "r"(page + (uint32_t)(fp8_vs_off(D) + 16 * tig)));
            v[4 * j + 0] = s0[0] * (qs * sk.x);
            v[4 * j + 1] = s0[1] * (qs * sk.y);
            v[4 * j + 2] = s1[0] * (qs * sk.z);
            v[4 * j + 3] = s1[1] * (qs * sk.w);
        }
        uint32_t keep[2] = {0xFFFFFFFFu, 0xFFFFFFFFu};  // bytes of a V word that are in use: other slots may hold anything
        if (seen != 0xFFFFFFFFu)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t b = seen >> (16 * j + 4 * tig) & 0xFu;
                keep[j] = ((b & 1u) | (b & 2u) << 7 | (b & 4u) << 14 | (b & 8u) << 21) * 0xFFu;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(b >> i & 1u)) {
                        v[4 * j + i] = -INFINITY;
                        sv[4 * j + i] = 0.f;
                    }
            }
        float mx = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
        float top = fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])), fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
#pragma unroll
        for (int x = 1; x < 4; x <<= 1) {
            mx = fmaxf(mx, __shfl_xor_sync(FULL, mx, x));
            top = fmaxf(top, __shfl_xor_sync(FULL, top, x));
        }
        const float m_new = mx > m + STEP ? mx : m;     // (finite: some token is in use)
        float alpha = fast_exp2(m - m_new);
        const float up = __uint_as_float((__float_as_uint(top) + 0x007FFFFFu) & 0x7F800000u);
        const float cs_new = fmaxf(cs, up);
        const float inv_cs = cs_new > 0.f ? 1.f / cs_new : 0.f;          // exact: a power of two
        uint32_t pb[2][2];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = fast_exp2(v[4 * j + i] - m_new);
                sum += x[i];
                x[i] *= sv[4 * j + i] * inv_cs;
            }
            pb[j][0] = pack_f16x2(x[0], x[1]);
            pb[j][1] = pack_f16x2(x[2], x[3]);
        }
        l = l * alpha + sum;
        m = m_new;
        alpha *= cs * inv_cs;                           // 1 unless the reference grew
        cs = cs_new;
        if (__any_sync(FULL, alpha != 1.f)) {           // rare once the references have settled
            const float a0 = __shfl_sync(FULL, alpha, 8 * tig), a1 = __shfl_sync(FULL, alpha, 8 * tig + 4);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                o[i][0] *= a0;
                o[i][1] *= a1;
                o[i][2] *= a0;
                o[i][3] *= a1;
            }
        }
        const uint32_t v_lane = blk + (uint32_t)(fp8_v_off(D) + g * PAGE + 4 * tig);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t w[D / 8];                          // all loads first: the volatile loads keep their order
#pragma unroll
            for (int i = 0; i < D / 8; ++i) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[i]) : "r"(v_lane + (uint32_t)(j * BLOCK + i * 8 * PAGE)));
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                uint32_t a0, a1, a2, a3;
                e4m3x4_to_f16x2(w[2 * i] & keep[j], a0, a2);
                e4m3x4_to_f16x2(w[2 * i + 1] & keep[j], a1, a3);
                mma_f16_16816(o[i], a0, a1, a2, a3, pb[j][0], pb[j][1]);
            }
        }
    }

    __device__ __forceinline__ void finish(float *part_o, float *part_ml, int64_t slot, int G, int lane)
    {
        const int g = lane >> 2, tig = lane & 3;
        l += __shfl_xor_sync(FULL, l, 1);
        l += __shfl_xor_sync(FULL, l, 2);
        const float c0 = __shfl_sync(FULL, cs, 8 * tig), c1 = __shfl_sync(FULL, cs, 8 * tig + 4);
        float *po = part_o + (slot * G + 2 * tig) * D + g;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            if (2 * tig < G) {
                po[16 * i] = o[i][0] * c0;
                po[16 * i + 8] = o[i][2] * c0;
            }
            if (2 * tig + 1 < G) {
                po[D + 16 * i] = o[i][1] * c1;
                po[D + 16 * i + 8] = o[i][3] * c1;
            }
        }
        if (g < G && tig == 0) *reinterpret_cast<float2 *>(part_ml + (slot * G + g) * 2) = make_float2(m, l);
    }
};

// CTAs of NW warps whose registers an SM is to hold. bf16 pages: a cluster of 16 CTAs needs two of 8 warps an SM, as a
// GPC may have fewer than 16 SMs; the CUDA cores' state of 128 dimensions is too large for that, and takes no such clusters.  Of 4 warps three,
// which shape_of counts on.  (That state with two of 4 warps an SM: 16 segments of 128 pages 14.5 us, 9.0 with three; 12 of 512, which need
// no more than two, 14.1 and 15.6.)
template <class State>
constexpr int ctas_per_sm(int warps)
{
    return State::PAGES == 2 ? 16 / warps : warps == 8 ? wide_ctas<State>() : 3;
}

// Dynamic shared memory: rings [NW][ST] units of State::PAGES blocks | the CTA's state | barriers [NW][ST]
template <int D, class State, int NW, bool EARLY, bool CHUNK>
__global__ void __launch_bounds__(NW * 32, ctas_per_sm<State>(NW)) decode_pages_kernel(DecodeParams p, PageLists l, int G, int ST)
{
    extern __shared__ __align__(128) uint8_t smem_raw[];
    constexpr int BLOCK = State::BLOCK, U = State::PAGES, UNIT = U * BLOCK;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t rank, ranks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(ranks));
    const uint32_t base = smem_u32(smem_raw);
    const uint32_t pad = (128u - (base & 127u)) & 127u;
    const uint32_t ring = base + pad + (uint32_t)(warp * ST * UNIT);
    // (a warp's state goes to the beginning of its ring, once that is done with: then three CTAs of four warps fit an SM)
    const int PF = part_floats(G, D), SF = ST * UNIT / 4;
    static_assert(part_floats(8, D) * 4 <= UNIT, "a state fits");
    float *states = reinterpret_cast<float *>(smem_raw + pad), *mine = states + (size_t)warp * SF;
    float *cta_state = states + (size_t)NW * SF;
    const uint32_t bars = base + pad + (uint32_t)((size_t)NW * ST * UNIT + (size_t)PF * 4) + (uint32_t)(warp * ST * 8);
    if (lane == 0) {
        for (int s = 0; s < ST; ++s) mbar_init(bars + 8 * s, 1);
        fence_barrier_init();
    }
    __syncwarp();
    pdl_wait();
    if (EARLY) pdl_trigger();
    const int seg = (int)(blockIdx.x / ranks), slot = seg / p.Hkv, h = seg - slot * p.Hkv;
    // sequence, which of its rows, list; row of Q and out, tokens up to the row's own
    const int b = CHUNK ? slot / p.max_q_len : slot, i = CHUNK ? slot - b * p.max_q_len : 0, list = CHUNK ? b * l.per_seq + i / l.run : slot;
    int row = slot, n;
    int pages;                                 // of the sequence
    const int64_t at = (int64_t)list * p.Hkv + h;
    const int length = __ldg(l.counts + at);   // (with the lengths: one trip for both)
    if (CHUNK) {                               // (every exit is the whole cluster's)
        const int first = __ldg(p.cu_q + b), q_len = __ldg(p.cu_q + b + 1) - first;
        n = __ldg(p.seq_lens + b);
        if (first < 0 || q_len < 0 || q_len > n || q_len > p.max_q_len || (int64_t)n > (int64_t)p.pt_stride * PAGE) {
            if (i == 0 && h == 0 && rank == 0 && threadIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
            return;
        }
        if (i >= q_len) return;
        pages = (n + PAGE - 1) / PAGE;
        n -= q_len - 1 - i;
        row = first + i;
    } else {
        n = __ldg(p.seq_lens + b);
        n = n > 0 ? n : 0;
        if ((int64_t)n > (int64_t)p.pt_stride * PAGE) {
            n = p.pt_stride * PAGE;
            if (rank == 0 && h == 0 && threadIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
        }
        pages = (n + PAGE - 1) / PAGE;
    }
    int listed = n > 0 ? length : 0;
    if (listed > l.stride) {
        listed = l.stride;
        if (rank == 0 && threadIdx.x == 0) atomicOr(p.status, STATUS_BOUNDS);
    }
    uint32_t *rows = reinterpret_cast<uint32_t *>(p.out + ((int64_t)row * p.Hq + (int64_t)h * G) * D);     // pairs of bf16
    if (listed <= 0) {                         // (the same for the whole cluster: no barrier is left half-way)
        if (rank == 0)
            for (int i = threadIdx.x; i < G * D / 2; i += NW * 32) rows[i] = 0u;
        return;
    }
    // units of U entries: this warp's are  from + warp + i * NW
    const int units = (listed + U - 1) / U, from = (int)((int64_t)units * rank / ranks), to = (int)((int64_t)units * (rank + 1) / ranks);
    const int count = to - from > warp ? (to - from - warp + NW - 1) / NW : 0;
    const int32_t *entries = l.lists + at * l.stride, *table = p.page_table + (int64_t)b * p.pt_stride;
    const uint64_t policy = p.keep_pct > 0 ? make_policy_evict_normal() : make_policy_evict_first();
    // A lane has an entry of its own, of 32 that follow each other (32 / U units): physical page and the tokens of it that the row sees.  Where
    // those are none (an entry out of range is one of these) the page that is copied in its place is not looked at; id -1: no entry.
    auto entry = [&](int i, int &id, uint32_t &bits) {
        id = -1;
        bits = 0;
        const int x = (from + warp + i / U * NW) * U + i % U;
        if (i / U >= count || x >= listed) return;
        const int page = __ldg(entries + x);
        id = 0;
        if (page < 0 || page >= pages) {
            atomicOr(p.status, STATUS_BOUNDS);
            return;
        }
        const int left = n - page * PAGE;
        bits = left >= PAGE ? 0xFFFFu : left > 0 ? (1u << left) - 1 : 0u;
        id = __ldg(table + page);
        if (id < 0 || (int64_t)id >= p.max_pages) {
            atomicOr(p.status, STATUS_BOUNDS);
            id = 0;
        }
    };
    constexpr int ROUND = 32 / U;              // units that the lanes have entries of
    int id, next_id;                           // of this round and of the next
    uint32_t bits, next_bits;
    entry(lane, id, bits);
    // unit i of this round or the next; the whole warp
    auto send = [&](int i, bool next) {
        int ids[U], there = 0;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            ids[j] = __shfl_sync(FULL, next ? next_id : id, i % ROUND * U + j);
            there += ids[j] >= 0;
        }
        if (lane == 0) {
            const uint32_t to_bar = bars + 8 * (i % ST), dst = ring + (uint32_t)(i % ST * UNIT);
            mbar_expect_tx(to_bar, (uint32_t)(there * BLOCK));
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (ids[j] >= 0)
                    bulk_copy_g2s_hint(dst + (uint32_t)(j * BLOCK), p.layer_base + (int64_t)ids[j] * p.page_stride + (int64_t)h * BLOCK, BLOCK, to_bar, policy);
        }
    };
    int sent = count < ST ? count : ST, done = 0;
    for (int i = 0; i < sent; ++i) send(i, false);
    entry(32 + lane, next_id, next_bits);
    State st;
    st.begin(p, row, h, G, lane);
    bool ok = true;
    for (; done < count; ++done) {
        if (done > 0 && done % ROUND == 0) {
            id = next_id;
            bits = next_bits;
            entry((done + ROUND) * U + lane, next_id, next_bits);
        }
        const int s = done % ST;
        ok = __all_sync(FULL, mbar_wait_bounded(bars + 8 * s, (uint32_t)((done / ST) & 1)));
        if (!ok) break;
        uint32_t seen = 0;
#pragma unroll
        for (int j = 0; j < U; ++j) seen |= __shfl_sync(FULL, bits, done % ROUND * U + j) << (PAGE * j);
        if (seen) st.fold_unit(ring + (uint32_t)(s * UNIT), seen, p.scale_log2, lane);
        __syncwarp();                          // every lane is done reading this stage
        if (sent < count) {
            send(sent, sent / ROUND != done / ROUND);
            ++sent;
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
        join_states<NW>(NW, 2 * e2 / D, e2, [&](int c, int g) { return *reinterpret_cast<const float2 *>(states + (size_t)c * SF + G * D + 2 * g); },
                        [&](int c, int e) { return *reinterpret_cast<const float2 *>(states + (size_t)c * SF + 2 * e); }, M, L, a);
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

// The shape of a call of `segments`, of at most `most` listed pages each
template <int D, class State>
Shape pages_shape(int64_t segments, int64_t most, int sm_count)
{
    Shape f = shape_of(State::PAGES * State::BLOCK, segments, (most + State::PAGES - 1) / State::PAGES, sm_count, wide_ctas<State>());
    // Segments are much of a size, so with a CTA each they come in waves, of which the last may be nearly empty.  What share of the slots
    // that `ways` to cut the segments fill, in waves of 4-warp CTAs:
    auto filled = [&](int ways, int per_sm) {
        const int64_t n = segments * ways, slots = (int64_t)per_sm * sm_count;
        return (double)n / (double)((n + slots - 1) / slots * slots);
    };
    if (State::PAGES == 2) {
        // FP8 pages of 128 dims are bound by issue and by the chain of a warp's steps, so warps count for more than bytes under way: as many ranks as
        // leave all CTAs resident at once, three to an SM with two stages or, over long lists, three and a half with one (clusters of 4 and 8 share a
        // GPC: 576 CTAs in fours do not fit 592 places, 45 us for 34); and of two to a segment a CTA of 8 warps.  (us, 256 pages, shape_of / these: 48
        // segments 20.5 / 16.9, 64 22.0 / 19.4, 96 33.9 / 25.3, 128 34.2 / 30.5, 192 59.2 / 41.4, 256 60.0 / 51.1; 26 pages: 16 segments 8.3 / 7.1,
        // 48 8.6 / 7.4, 256 12.2 / 11.3, but 128 8.2 / 9.4, where shape_of has as many warps.  Of 64 dims: 32 segments 9.7 / 10.2, 256 33.6 / 35.8.)
        int r = 1;
        for (int next = 2; D == 128 && next <= 8; next *= 2) {
            const int64_t ctas = segments * next;
            if (ctas <= 3 * (int64_t)sm_count ? most < 3 * next : next == 2 ? ctas > 4 * (int64_t)sm_count || most < 16 : 2 * ctas > 7 * (int64_t)sm_count || most < 128) break;
            r = next;
        }
        if (4 * r > f.warps * f.ranks) f = segments * r <= 3 * (int64_t)sm_count ? Shape{4, 2, r} : r == 2 ? Shape{8, 1, 1} : Shape{4, 1, r};
        // And with a CTA to a segment, four to an SM with a stage less, where three would leave more empty.  (us, 256 pages, three / four: 384 segments
        // 72 / 81, 512 131 / 95, 768 142 / 168, 1024 208 / 186.)
        if (f.ranks == 1 && f.warps == 4 && filled(1, 4) > filled(1, 3)) f.stages = 1;
    } else if (f.ranks == 1 && f.warps == 4 && filled(2, 3) > 1.25 * filled(1, 3) && most >= 64) {
        // bf16 pages: a cluster of two to a segment, where that fills a quarter more.  (One / two: 512 segments, 128 pages 99.8 / 91.9, 256 pages
        // 195 / 169; 384 segments 67.4 / 68.2; 768 120 / 127; 1024 165 / 163.)
        f.ranks = 2;
    }
    return f;
}

template <int D, class State, bool CHUNK>
cudaError_t launch_t(const DecodeParams &p, const PageLists &l, int G, int sm_count, bool pdl, cudaStream_t s)
{
    const int64_t segments = (int64_t)p.B * p.Hkv;
    constexpr int UNIT = State::PAGES * State::BLOCK;
    const Shape f = pages_shape<D, State>(segments, l.stride < p.pt_stride ? l.stride : p.pt_stride, sm_count);
    if (segments * f.ranks > 0x7FFFFFFF) return cudaErrorInvalidConfiguration;
    const size_t smem = 128 + (size_t)f.warps * f.stages * UNIT + (size_t)part_floats(G, D) * 4 + (size_t)f.warps * f.stages * 8;
    const bool early = segments * f.ranks <= sm_count;       // (as over a window: the next launch may fill the SMs that this one leaves free)
    auto kern = CHUNK        ? (f.warps == 8 ? decode_pages_kernel<D, State, 8, false, CHUNK> : decode_pages_kernel<D, State, 4, false, CHUNK>)
                : f.warps == 8 ? (early ? decode_pages_kernel<D, State, 8, true, CHUNK> : decode_pages_kernel<D, State, 8, false, CHUNK>)
                               : (early ? decode_pages_kernel<D, State, 4, true, CHUNK> : decode_pages_kernel<D, State, 4, false, CHUNK>);
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
    return cudaLaunchKernelEx(&cfg, kern, p, l, G, f.stages);
}

}  // namespace

cudaError_t launch_decode_pages(const DecodeParams &p, const PageLists &l, int D, int G, int kernel, int sm_count, bool pdl, cudaStream_t s)
{
    auto go = [&](auto dim) {
        constexpr int N = decltype(dim)::value;
        if (kernel == 2) return p.cu_q ? launch_t<N, Fp8PairState<N>, true>(p, l, G, sm_count, pdl, s) : launch_t<N, Fp8PairState<N>, false>(p, l, G, sm_count, pdl, s);
        if (kernel == 1) return p.cu_q ? launch_t<N, ByPage<TensorCoreState<N, true>>, true>(p, l, G, sm_count, pdl, s) : launch_t<N, ByPage<TensorCoreState<N, true>>, false>(p, l, G, sm_count, pdl, s);
        return p.cu_q ? launch_t<N, ByPage<CudaCoreState<N>>, true>(p, l, G, sm_count, pdl, s) : launch_t<N, ByPage<CudaCoreState<N>>, false>(p, l, G, sm_count, pdl, s);
    };
    return D == 128 ? go(std::integral_constant<int, 128>()) : D == 64 ? go(std::integral_constant<int, 64>()) : cudaErrorInvalidValue;
}

#ifdef SKV_TEST_HOOKS
void decode_pages_shape(int D, int kernel, int64_t segments, int64_t pages, int sm_count, int *out)
{
    auto ask = [&](auto state, auto dim) {
        using State = typename decltype(state)::type;
        const Shape f = pages_shape<decltype(dim)::value, State>(segments, pages, sm_count);
        out[0] = f.warps;
        out[1] = f.stages;
        out[2] = f.ranks;
        out[3] = ctas_per_sm<State>(f.warps);
    };
    auto go = [&](auto dim) {
        constexpr int N = decltype(dim)::value;
        if (kernel == 2) ask(Type<Fp8PairState<N>>(), dim);
        else if (kernel == 1) ask(Type<ByPage<TensorCoreState<N, true>>>(), dim);
        else ask(Type<ByPage<CudaCoreState<N>>>(), dim);
    };
    if (D == 128) go(std::integral_constant<int, 128>());
    else go(std::integral_constant<int, 64>());
}
#endif

}  // namespace skv
