// A segment -- one (row, kv head) with its pages -- as one piece of work of a CTA or of a cluster of CTAs: what the decode
// kernels over a window (skv_decode_window.cu) and over listed pages (skv_decode_pages.cu) share.
#pragma once
#include "skv_common.cuh"

#include <math.h>
#include <type_traits>

namespace skv {

constexpr int MAX_RANKS = 16;          // CTAs that may share a segment

__host__ __device__ constexpr int part_floats(int G, int D) { return G * D + ((2 * G + 3) & ~3); }

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

// sum of n_states states, weighted: the pair e2 of the segment's rows and its head's (max, sum)
template <int N, class MlOf, class PairOf>
__device__ __forceinline__ void join_states(int n_states, int head, int e2, MlOf ml_of, PairOf pair_of, float &M, float &L, float2 &a)
{
    float2 ml[N], v[N];
#pragma unroll
    for (int c = 0; c < N; ++c) {
        ml[c] = make_float2(-INFINITY, 0.f);
        v[c] = make_float2(0.f, 0.f);
        if (c < n_states) {
            ml[c] = ml_of(c, head);
            v[c] = pair_of(c, e2);
        }
    }
    M = -INFINITY;
#pragma unroll
    for (int c = 0; c < N; ++c) M = fmaxf(M, ml[c].x);
    L = 0.f;
    a = make_float2(0.f, 0.f);
#pragma unroll
    for (int c = 0; c < N; ++c) {
        // No page there, or not there: the sum says so, which is 1 or more where there is one, or NaN.  (Not the maximum:
        // that is -inf too where every score is NaN, and the result has to be NaN then.)
        if (ml[c].y == 0.f) continue;
        const float w = fast_exp2(ml[c].x - M);
        L = fmaf(w, ml[c].y, L);
        a.x = fmaf(w, v[c].x, a.x);
        a.y = fmaf(w, v[c].y, a.y);
    }
}

// CTAs of 8 warps of it that an SM's registers hold: two, but one of the CUDA cores' state of 128 dims (128 floats a thread for queries
// and outputs alone).
template <class State>
constexpr int wide_ctas() { return sizeof(State) > 400 ? 1 : 2; }

// How a call is laid out: warps per CTA, pages in flight per warp, CTAs per segment.
struct Shape { int warps, stages, ranks; };

// `block` bytes per page and kv head, `segments` of at most `pages` pages; `wide`: wide_ctas of the state.  Measured (us; rows of the sweep: segments x
// pages at 8 KB blocks; W warps, S stages, R ranks):
//       8 x   65   W8 S1 R16  5.7   W8 S2 R8  6.0   W4 S2 R16  5.8
//       8 x  513   W8 S1 R16 11.1   W4 S2 R16 12.2
//      16 x   65   W4 S2 R16  6.3   W8 S2 R8 11.1
//      16 x  513   W4 S2 R16 14.9   W8 S2 R8 25.2
//      64 x   65   W8 S2 R2   9.7   W4 S2 R4 10.0   W8 S1 R4 10.1
//     128 x   65   W8 S2 R1  13.1   W8 S1 R2 14.1   W4 S2 R2 14.5
//     256 x  129   W4 S2 R1  37.2   W8 S1 R1 37.1   W8 S2 R1 41.5
//     320 x  257   W4 S2 R1  93.0   W4 S2 R2 100
//    1024 x   65   W4 S2 R1  72.8   W8 S1 R1 75.7   W8 S2 R1 80.5
// So: a CTA of 8 warps and two stages (one per SM) where a power of two of them per segment comes close to one for every
// SM, and 4 warps with two stages (three per SM) else, as many ranks as still leave all CTAs resident at once.  A cluster's CTAs
// share a GPC, whose SMs are not a multiple of 8: of 8 CTAs with an SM each 15 clusters run at once, and the 16th doubles the time.
// Blocks of half the size (FP8, head_dim 64) take 8 warps in the same space, and 16 ranks of them only with an SM for each
// (16 segments x 257 pages: 11.5 us, in clusters of 8 7.8).  A rank has at least four pages.  Of 8 warps of which an SM holds one CTA, clusters
// of 16 would need 16 free SMs of one GPC each (7 run at once here, and where no GPC has as many none): these take 4 warps (8 segments x 128
// pages 7.6 us, 12.6 to 13.2 in clusters of 16 x 8 warps).
inline Shape shape_of(int block, int64_t segments, int64_t pages, int sm, int wide)
{
    Shape best = {block >= 8192 ? 4 : 8, 2, 1};
    auto ranks_up_to = [&](int64_t ctas, int most) {
        int r = 1;
        while (2 * r <= most && segments * 2 * r <= ctas && pages >= 4 * 2 * r) r *= 2;
        return r;
    };
    best.ranks = ranks_up_to(2 * (int64_t)sm + sm / 4, block >= 8192 || 16 * segments <= sm ? MAX_RANKS : 8);
    if (block >= 8192) {
        const int r = ranks_up_to(sm, wide > 1 ? MAX_RANKS : 8);
        const int64_t room = r == 8 ? 3 * (int64_t)sm / 4 : r == 4 ? 7 * (int64_t)sm / 8 : sm;
        const bool fills = 4 * segments * r >= 3 * (int64_t)sm && segments * r <= room;
        if (fills) best = {8, r > 8 ? 1 : 2, r};             // (a cluster of 16 needs two CTAs to an SM: a GPC may not have 16 SMs)
    }
    const int64_t per_warp = (pages + (int64_t)best.ranks * best.warps - 1) / ((int64_t)best.ranks * best.warps);
    if (per_warp < best.stages) best.stages = 1;
    return best;
}

#ifdef SKV_TEST_HOOKS
template <class T>
struct Type { using type = T; };
// {warps, stages, ranks, CTAs of it that an SM's registers hold} of a call; kernel as in launch_decode_splitk
void decode_pages_shape(int D, int kernel, int64_t segments, int64_t pages, int sm_count, int *out);
void decode_window_shape(int D, int kernel, int64_t segments, int64_t pages, int sm_count, int *out);
#endif

}  // namespace skv
