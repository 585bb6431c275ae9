// Rotary embedding of a call's queries and keys, and Algorithm 2's "Update" with the turned keys, in one pass.
//
// Frequency i of a token turns the pair (x1, x2) of a row by  angle = position * inv_freq[i]:
//     x1' = x1 cos - x2 sin,   x2' = x2 cos + x1 sin.
// The angle is kept as a fraction of a turn in 64-bit fixed point: with F = 2^64 inv_freq / 2 pi (mod 2^64, from
// the host, off by half at most) the product position * F mod 2^64 IS the angle modulo a full turn, for every 32-bit
// position, with an error of 2^-34 of a turn at most.  (A product in fp32 is off by 0.03 rad at position 10^6.)  Only then does it
// become a float, between -1 and 1 half turns (2^-26 of a turn at most), and cos / sin of it are taken with sincospi.  The rows are turned in fp32 and rounded once: to bf16, or
// on FP8 pages to the code of the row's own scale.
//
// Work split.  A lane owns a pair of 16-byte pieces of a row (a chunk of 8 elements and its partners), so a head
// is D/16 lanes and a warp holds 32 / (D/16) tokens: 4 at head_dim 128.  The lane's eight cos / sin belong to its
// token and chunk alone, so it computes them itself, once, and then runs over heads: no table, no shared memory,
// nothing is computed twice inside a warp.  Loads and stores of Q are whole 128-byte lines; a page's chunk-major
// layout takes the same lanes as 64-byte runs (4 tokens x 16 bytes), whatever the slots are.  The heads are dealt
// to `head_parts` warps per token group: for few tokens (a decode step) to have warps at all, for many so that the
// last ones to finish are short.  Only V of FP8 pages, which is dim-major there, is done by warps of its own, a page (16
// tokens) and kv head each: four lanes swap words so that each ends up with 16 tokens of four dims and stores 16 bytes
// at a time (byte by byte it took longer than all the rest).
// Bound by memory: every row is read once and written once.  32768 tokens of 32 query and 8 kv heads onto FP8 pages 120 us,
// 6.2 TB/s (0.94 of the measured copy peak); 8191 tokens with three axes 36.1 us, 5.6 TB/s (0.85);
// 64 tokens 3.6 us, a launch.
#include "skv_common.cuh"

#include <math.h>

namespace skv {

namespace {

constexpr int ROPE_THREADS = 128;

// 8 bf16 of a 16-byte piece
__device__ __forceinline__ void unpack8(const uint4 &w, float (&x)[8])
{
    x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
    x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8])
{
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// 4 x 4 bytes transposed: word i of the input holds bytes [i][0..3], word j of the output bytes [0..3][j]
__device__ __forceinline__ void transpose_bytes(const uint32_t (&a)[4], uint32_t (&o)[4])
{
    const uint32_t t0 = __byte_perm(a[0], a[1], 0x5140), t1 = __byte_perm(a[0], a[1], 0x7362);
    const uint32_t t2 = __byte_perm(a[2], a[3], 0x5140), t3 = __byte_perm(a[2], a[3], 0x7362);
    o[0] = __byte_perm(t0, t2, 0x5410);
    o[1] = __byte_perm(t0, t2, 0x7632);
    o[2] = __byte_perm(t1, t3, 0x5410);
    o[3] = __byte_perm(t1, t3, 0x7632);
}

__device__ __forceinline__ uint32_t codes4(const float *x, float inv)
{
    return pack_e4m3x2(__fmul_rn(x[0], inv), __fmul_rn(x[1], inv)) | (pack_e4m3x2(__fmul_rn(x[2], inv), __fmul_rn(x[3], inv)) << 16);
}

// V rows of tokens 16 group .. +15 and kv head kh onto FP8 pages, by one warp.
template <int D>
__device__ __forceinline__ void store_v_fp8(const RopeParams &p, int64_t group, int kh, int lane)
{
    constexpr unsigned ALL = 0xFFFFFFFFu;
    constexpr int LPR = D / 16, TOK = 32 / LPR, ROUNDS = PAGE / TOK;         // lanes of a row, tokens at once: 4 (8 at head_dim 64)
    const int64_t t0 = group * PAGE;
    const int c = lane % LPR, r = lane / LPR;                               // 16-dim piece and token of a round
    uint4 in[ROUNDS][2];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int64_t tok = t0 + k * TOK + r;
        const uint4 *src = reinterpret_cast<const uint4 *>(p.V + tok * p.v_stride + (int64_t)kh * D) + 2 * c;
        in[k][0] = in[k][1] = make_uint4(0u, 0u, 0u, 0u);
        if (tok < p.n_tokens) {
            in[k][0] = __ldg(src);
            in[k][1] = __ldg(src + 1);
        }
    }
    const int64_t mine = lane < PAGE && t0 + lane < p.n_tokens ? (int64_t)__ldg(reinterpret_cast<const long long *>(p.slot_map) + t0 + lane) : -1;
    if (mine >= p.n_slots) atomicOr(p.status, STATUS_BOUNDS);
    const int64_t first = __shfl_sync(ALL, mine, 0);
    const bool whole = __all_sync(ALL, lane >= PAGE || (first >= 0 && (first & (PAGE - 1)) == 0 && mine == first + lane && mine < p.n_slots));
    uint32_t code[ROUNDS][4];                                               // [round][quad of dims]
    float scale[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        float x[16], amax = 0.f;
        float (&lo)[8] = *reinterpret_cast<float (*)[8]>(x), (&hi)[8] = *reinterpret_cast<float (*)[8]>(x + 8);
        unpack8(in[k][0], lo);
        unpack8(in[k][1], hi);
#pragma unroll
        for (int i = 0; i < 16; ++i) amax = fmaxf(amax, fabsf(x[i]));
#pragma unroll
        for (int d = 1; d < LPR; d <<= 1) amax = fmaxf(amax, __shfl_xor_sync(ALL, amax, d));
        const float inv = amax > 0.f ? __fdiv_rn(448.f, amax) : 0.f;
        scale[k] = __fdiv_rn(amax, 448.f);
#pragma unroll
        for (int j = 0; j < 4; ++j) code[k][j] = codes4(x + 4 * j, inv);
    }
    if (whole) {
        uint8_t *blk = p.layer_base + (first >> 4) * p.page_stride + (int64_t)kh * fp8_block_bytes(D);
        // the four lanes of a piece and of four neighbouring tokens swap quads: lane r & 3 gets quad r & 3 of all four
        uint32_t word[4][ROUNDS];                                           // [dim of the quad][round]: four tokens
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) {
#pragma unroll
            for (int bit = 0; bit < 2; ++bit) {
                const bool up = (r >> bit) & 1;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!((j >> bit) & 1)) {
                        const int jh = j | (1 << bit);
                        const uint32_t got = __shfl_xor_sync(ALL, up ? code[k][j] : code[k][jh], LPR << bit);
                        if (up) code[k][j] = got;
                        else code[k][jh] = got;
                    }
            }
            uint32_t o[4];
            transpose_bytes(code[k], o);
#pragma unroll
            for (int i = 0; i < 4; ++i) word[i][k] = o[i];
            if (c == 0) *reinterpret_cast<float *>(blk + fp8_vs_off(D) + 4 * (k * TOK + r)) = scale[k];
        }
        uint8_t *dst = blk + fp8_v_off(D) + (16 * c + 4 * (r & 3)) * PAGE;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (ROUNDS == 4) *reinterpret_cast<uint4 *>(dst + i * PAGE) = make_uint4(word[i][0], word[i][1 % ROUNDS], word[i][2 % ROUNDS], word[i][3 % ROUNDS]);
            else
#pragma unroll
                for (int k = 0; k < ROUNDS; ++k) *reinterpret_cast<uint32_t *>(dst + i * PAGE + TOK * k + 4 * (r >> 2)) = word[i][k];
        }
        return;
    }
    // loose tokens, holes, the ragged end: each token's column, a byte per dim
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int64_t slot = __shfl_sync(ALL, mine, k * TOK + r);
        if (slot < 0 || slot >= p.n_slots) continue;
        const int off = (int)(slot & (PAGE - 1));
        uint8_t *blk = p.layer_base + (slot >> 4) * p.page_stride + (int64_t)kh * fp8_block_bytes(D);
        if (c == 0) *reinterpret_cast<float *>(blk + fp8_vs_off(D) + 4 * off) = scale[k];
        uint8_t *dst = blk + fp8_v_off(D) + 16 * c * PAGE + off;
#pragma unroll
        for (int i = 0; i < 16; ++i) dst[i * PAGE] = (uint8_t)(code[k][i >> 2] >> (8 * (i & 3)));
    }
}

// ADJACENT: pairs (2i, 2i+1) instead of (i, i + rotary_dim / 2)
template <int D, bool FP8, bool ADJACENT>
// (six blocks to an SM: 8191 tokens 36.1 us, five 37.6; FP8 pages want the registers)
__global__ void __launch_bounds__(ROPE_THREADS, FP8 ? 5 : 6) rope_append_kernel(const __grid_constant__ RopeParams p)
{
    constexpr int CP = D / 16;                     // lanes of a head
    constexpr int TOK = 32 / CP;                   // tokens of a warp
    constexpr int AHEAD = 4;
    constexpr unsigned ALL = 0xFFFFFFFFu;
    const int lane = threadIdx.x & 31;
    int64_t item = (int64_t)blockIdx.x * (ROPE_THREADS / 32) + (threadIdx.x >> 5);
    const int64_t n_groups = (p.n_tokens + TOK - 1) / TOK;
    pdl_wait();
    pdl_trigger();
    if (FP8 && item >= n_groups * p.head_parts) {  // V
        item -= n_groups * p.head_parts;
        if (item < (p.n_tokens + PAGE - 1) / PAGE * p.Hkv) store_v_fp8<D>(p, item / p.Hkv, (int)(item % p.Hkv), lane);
        return;
    }
    const int64_t group = item / p.head_parts;
    const int part = (int)(item - group * p.head_parts);
    if (group >= n_groups) return;
    const int cp = lane % CP;
    const int64_t tok = group * TOK + lane / CP;
    const bool there = tok < p.n_tokens;
    // this lane's two pieces of a row: c0 and its partner c1 (or, past the rotary dims, two pieces that are copied)
    const int turned = p.rotary_dim / 16;          // lanes of a head whose pieces are turned
    const bool turns = cp < turned;
    const int c0 = turns ? (ADJACENT ? 2 * cp : cp) : 2 * cp, c1 = turns && !ADJACENT ? cp + turned : c0 + 1;
    float cs[8], sn[8];
    if (turns) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int f = 8 * cp + i;              // (half: elements 8 c0 + i and 8 c1 + i; adjacent: pairs 4 c0 .. 4 c0 + 7)
            const int pos = there ? __ldg(p.positions + (int64_t)p.axis[f] * p.pos_stride + tok) : 0;
            const uint64_t phase = p.freq[f] * (uint64_t)(int64_t)pos;       // fraction of a turn, modulo one
            sincospif((float)(int64_t)phase * 1.0842021724855044e-19f, &sn[i], &cs[i]);       // 2^-63: half turns in [-1, 1)
        }
    }
    auto turn = [&](float (&a)[8], float (&b)[8]) {
        if (!turns) return;
        if (ADJACENT) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float x = a[2 * i], y = a[2 * i + 1];
                a[2 * i] = x * cs[i] - y * sn[i];
                a[2 * i + 1] = y * cs[i] + x * sn[i];
                const float u = b[2 * i], v = b[2 * i + 1];
                b[2 * i] = u * cs[i + 4] - v * sn[i + 4];
                b[2 * i + 1] = v * cs[i + 4] + u * sn[i + 4];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = a[i], y = b[i];
                a[i] = x * cs[i] - y * sn[i];
                b[i] = y * cs[i] + x * sn[i];
            }
        }
    };
    // ---- heads of this warp among [Q heads | K heads | V heads] (FP8 pages: V has warps of its own) ----
    const int heads = p.Hq + (FP8 ? 1 : 2) * p.Hkv;
    const int h_from = (int)((int64_t)heads * part / p.head_parts), h_to = (int)((int64_t)heads * (part + 1) / p.head_parts);
    {
        const int to = h_to < p.Hq ? h_to : p.Hq;
        const uint4 *src = reinterpret_cast<const uint4 *>(p.Q + tok * p.q_stride);
        uint4 *dst = reinterpret_cast<uint4 *>(p.Q_out + tok * p.qo_stride);
        // (a few heads' loads ahead of their stores: Q_out may be Q, so the compiler must keep the order it is given)
        for (int h0 = h_from; h0 < to; h0 += AHEAD) {
            uint4 wa[AHEAD], wb[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (there && h0 + i < to) {
                    wa[i] = src[(h0 + i) * (D / 8) + c0];
                    wb[i] = src[(h0 + i) * (D / 8) + c1];
                }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (there && h0 + i < to) {
                    if (turns) {
                        float a[8], b[8];
                        unpack8(wa[i], a);
                        unpack8(wb[i], b);
                        turn(a, b);
                        wa[i] = pack8(a);
                        wb[i] = pack8(b);
                    }
                    dst[(h0 + i) * (D / 8) + c0] = wa[i];
                    dst[(h0 + i) * (D / 8) + c1] = wb[i];
                }
        }
    }
    if (h_to <= p.Hq) return;
    int64_t slot = there ? __ldg(reinterpret_cast<const long long *>(p.slot_map) + tok) : -1;
    if (slot >= p.n_slots) {
        atomicOr(p.status, STATUS_BOUNDS);
        slot = -1;
    }
    const int off = (int)(slot & (PAGE - 1));
    uint8_t *page = p.layer_base + (slot >> 4) * p.page_stride;              // (not touched for slot < 0)
    for (int h0 = h_from > p.Hq ? h_from : p.Hq; h0 < h_to; h0 += AHEAD) {
        uint4 wa[AHEAD], wb[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int h = h0 + i, which = h >= p.Hq + p.Hkv, kh = h - p.Hq - (which ? p.Hkv : 0);
            wa[i] = wb[i] = make_uint4(0u, 0u, 0u, 0u);
            if (slot >= 0 && h < h_to) {
                const uint4 *src = reinterpret_cast<const uint4 *>(which ? p.V + tok * p.v_stride : p.K + tok * p.k_stride) + kh * (D / 8);
                wa[i] = __ldg(src + c0);
                wb[i] = __ldg(src + c1);
            }
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int h = h0 + i, which = h >= p.Hq + p.Hkv, kh = h - p.Hq - (which ? p.Hkv : 0);
            if (h >= h_to) break;                                            // (the same for the warp)
            float a[8], b[8];
            unpack8(wa[i], a);
            unpack8(wb[i], b);
            if (!which) turn(a, b);
            if (!FP8) {
                if (slot < 0) continue;
                uint4 *dst = reinterpret_cast<uint4 *>(page + (int64_t)kh * block_bytes(D) + (which ? half_bytes(D) : 0)) + off;
                const bool raw = which || !turns;                            // (bits as they are, NaN payloads among them)
                dst[c0 * PAGE] = raw ? wa[i] : pack8(a);
                dst[c1 * PAGE] = raw ? wb[i] : pack8(b);
            } else {
                float amax = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fmaxf(fabsf(a[j]), fabsf(b[j])));
#pragma unroll
                for (int d = 1; d < CP; d <<= 1) amax = fmaxf(amax, __shfl_xor_sync(ALL, amax, d));
                if (slot < 0) continue;                                      // (after the shuffles)
                const float inv = amax > 0.f ? __fdiv_rn(448.f, amax) : 0.f;
                uint8_t *blk = page + (int64_t)kh * fp8_block_bytes(D);
                if (cp == 0) *reinterpret_cast<float *>(blk + fp8_ks_off(D) + 4 * off) = __fdiv_rn(amax, 448.f);
                *reinterpret_cast<uint2 *>(blk + fp8_k_pos(D, off, 8 * c0)) = make_uint2(codes4(a, inv), codes4(a + 4, inv));
                *reinterpret_cast<uint2 *>(blk + fp8_k_pos(D, off, 8 * c1)) = make_uint2(codes4(b, inv), codes4(b + 4, inv));
            }
        }
    }
}

template <int D, bool FP8>
cudaError_t launch_rope(const RopeParams &p, bool adjacent, bool pdl, cudaStream_t s)
{
    const int64_t groups = (p.n_tokens + 32 / (D / 16) - 1) / (32 / (D / 16));
    const int64_t warps = groups * p.head_parts + (FP8 ? (p.n_tokens + PAGE - 1) / PAGE * p.Hkv : 0), blocks = (warps * 32 + ROPE_THREADS - 1) / ROPE_THREADS;
    if (blocks > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(ROPE_THREADS);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl ? 1 : 0;
    return adjacent ? cudaLaunchKernelEx(&cfg, rope_append_kernel<D, FP8, true>, p)
                    : cudaLaunchKernelEx(&cfg, rope_append_kernel<D, FP8, false>, p);
}

}  // namespace

cudaError_t launch_rope_append(const RopeParams &p, int D, bool fp8, bool adjacent, bool pdl, cudaStream_t s)
{
    if (p.n_tokens <= 0 || p.head_parts < 1) return cudaSuccess;
    if (D == 128) return fp8 ? launch_rope<128, true>(p, adjacent, pdl, s) : launch_rope<128, false>(p, adjacent, pdl, s);
    if (D == 64) return fp8 ? launch_rope<64, true>(p, adjacent, pdl, s) : launch_rope<64, false>(p, adjacent, pdl, s);
    return cudaErrorInvalidValue;
}

}  // namespace skv
