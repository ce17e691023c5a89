// Eviction from a sequence cache by accumulated attention weight: of the len keys of a (sequence, key/value head) the
// kept = min(n_keep, len) stay: the last min(n_recent, kept) ones, and of the older ones those of largest weight (equal weights: the lower
// position; NaN counts as less than everything).  They keep their order.
//
//   evict_select_kernel  a cluster of 1 to 16 CTAs per (sequence, head): the weight of the last key kept is found digit by digit (radix
//                        12 + 12 + 8 bits of the weight's order-preserving integer), by a histogram of the keys that agree with the digits
//                        found so far, until all that are left in a bin stay.  Each CTA counts its share of the keys, held in its shared
//                        memory where they fit, and the cluster's counts are added over distributed shared memory.  Then every thread, which
//                        has a run of adjacent keys, counts what it keeps and writes positions and weights behind what is kept before it.
//   evict_gather_kernel  copies the kept K and V rows, all heads of a few output positions per CTA: bound by HBM (each row read and
//                        written once; 32 sequences, 1024 rows of 8 heads kept, d = 128: 268 MB in 38 us).  It writes the new lengths too: they may
//                        take the place of the old ones, which the selection of any head, whenever its CTAs get their turn, has to read.
//
// The selection is a chain of short phases, bound by their latencies (per CTA of 8192 keys some 8 us: 2.3 the weights' way here, 2 each of the two or three
// passes, 2.5 counting and writing).  us, both kernels: 32 x 8192 keys to 1024, 8 heads 53; 131001 keys to 16001, 8 heads, d = 64 31; 2176 to 2048 8.6.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "launch_rules.h"
#include "sm100_ptx.cuh"

namespace moda {

struct EvictParams {
    const __nv_bfloat16* K;       // [B][T_cap][Hk][d]
    const __nv_bfloat16* V;
    const float* mass;            // [B][Hk][T_cap]
    const int* seq_lens;          // [B], each 0 .. T, or null: T for all
    __nv_bfloat16* K_out;         // [B][T_out][Hk][d]
    __nv_bfloat16* V_out;
    float* mass_out;              // [B][Hk][T_out], may be null
    int* index;                   // [B][Hk][n_keep]
    int* lens_out;                // [B], may be null, may be seq_lens
    int B, T, T_cap, T_out, Hk, n_keep, n_recent;
};

__device__ __forceinline__ int evict_len(const EvictParams& p, int b) {
    return p.seq_lens ? min(max(p.seq_lens[b], 0), p.T) : p.T;
}

// Unsigned integers in the order of the floats: NaN first, -0 and +0 equal.
__device__ __forceinline__ uint32_t evict_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u ^ ((u & 0x80000000u) ? 0xffffffffu : 0x80000000u);
}

constexpr int kEvictBins = 4096, kEvictGroups = kEvictBins / 32, kEvictWarps = kEvictMostThreads / 32;

struct EvictShared {
    uint32_t hist[2][kEvictBins], hist3[256];     // of a pass each: nobody waits until another CTA has read the one before
    uint32_t group[3][kEvictGroups];              // sums over 32 bins
    uint32_t rank_group[kEvictMostRanks][kEvictGroups], rank_bin[kEvictMostRanks][32];   // what the cluster's CTAs have
    uint32_t warp_gt[kEvictWarps], warp_eq[kEvictWarps];
    __align__(8) uint32_t cta_gt;
    uint32_t cta_eq;
    uint32_t pad[2];                              // the keys behind start on a 16-byte boundary
};
static_assert(sizeof(EvictShared) % 16 == 0, "alignment of the keys");
inline int evict_select_smem(int run, int threads) { return int(sizeof(EvictShared)) + run * threads * 4; }

__device__ __forceinline__ uint4 ld_cluster_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint2 ld_cluster_v2(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cp_async_4(uint32_t smem_dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_dst), "l"(src) : "memory");
}

// grid (cluster, Hk, B).  RUN: most keys of a thread (evict_form); they are in shared memory and, where the registers hold them, there as integers.  0: more
// than shared memory holds, they are read again for every pass.  CTAS: that share an SM.
template <int RUN, int NT, int CTAS>
__global__ void __launch_bounds__(NT, CTAS)
evict_select_kernel(const EvictParams p) {
    constexpr bool kHeld = RUN > 0, kRegs = RUN > 0 && RUN <= (CTAS == 1 && NT == 512 ? 33 : 17);
    extern __shared__ __align__(16) uint8_t evict_smem[];
    EvictShared& s = *reinterpret_cast<EvictShared*>(evict_smem);
    float* held = reinterpret_cast<float*>(evict_smem + sizeof(EvictShared));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int ranks = gridDim.x, rank = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
    const int len = evict_len(p, b);
    const int kept = min(p.n_keep, len), recent = min(p.n_recent, kept);
    const int old = len - recent, want = kept - recent;              // `want` of the `old` first keys stay
    const float* mass = p.mass + (size_t(b) * p.Hk + hk) * p.T_cap;
    int* index = p.index + (size_t(b) * p.Hk + hk) * p.n_keep;
    float* mass_out = p.mass_out ? p.mass_out + (size_t(b) * p.Hk + hk) * p.T_out : nullptr;

    // a thread has a run of adjacent keys
    const int run = evict_run(old, ranks, NT), share = run * NT;
    const int first = min(rank * share, old), n = min(share, old - first);
    const int r0 = min(tid * run, n), mine = min(run, n - r0);
    const bool some = want > 0 && want < old;
    grid_launch_dependents();

    if (kHeld && want > 0) {
        const uint32_t dst = smem_u32(held);
        const int quads = (reinterpret_cast<uintptr_t>(mass + first) & 15u) == 0 ? n / 4 : 0;   // rows of any length and start
#pragma unroll 4
        for (int i = tid; i < quads; i += NT)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + i * 16), "l"(mass + first + i * 4) : "memory");
#pragma unroll 4
        for (int i = quads * 4 + tid; i < n; i += NT) cp_async_4(dst + i * 4, mass + first + i);
    }
#pragma unroll
    for (int i = 0; i < 2 * kEvictBins / 4; i += NT) reinterpret_cast<uint4*>(s.hist[0])[i + tid] = make_uint4(0u, 0u, 0u, 0u);
    if (tid < 64) reinterpret_cast<uint4*>(s.hist3)[tid] = make_uint4(0u, 0u, 0u, 0u);
    if (kHeld) asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    auto weight = [&](int j) -> float {                              // of key j of this thread's run
        if constexpr (kHeld) return held[r0 + j];
        else return mass[first + r0 + j];
    };
    uint32_t keys[kRegs ? RUN : 1];
    if constexpr (kRegs) {
        if (some) {
#pragma unroll
            for (int j = 0; j < RUN; ++j) keys[j] = j < mine ? evict_key(weight(j)) : 0u;
        }
    }
    // f(j, integer) for the keys of the run
    auto each = [&](auto&& f) {
        if constexpr (kRegs) {
#pragma unroll
            for (int j = 0; j < RUN; ++j)
                if (j < mine) f(j, keys[j]);
        } else {
#pragma unroll 4
            for (int j = 0; j < mine; ++j) f(j, evict_key(weight(j)));
        }
    };

    uint32_t thr = 0u, ties = uint32_t(old);                         // kept: key > thr, and the first `ties` keys equal to it
    if (some) {
        uint32_t prefix = 0, left = uint32_t(want);                  // digits found; keys still to take among those that agree
        uint32_t count = 0;
        int shift = 32;
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int bits = pass == 2 ? 8 : 12, agree = shift;
            shift -= bits;
            uint32_t* hist = pass == 2 ? s.hist3 : s.hist[pass];
            const uint32_t mask = (1u << bits) - 1u;
            if (pass == 0) each([&](int, uint32_t k) { atomicAdd(&hist[k >> 20], 1u); });
            else each([&](int, uint32_t k) { if ((k >> agree) == prefix) atomicAdd(&hist[(k >> shift) & mask], 1u); });
            __syncthreads();
            {
                uint32_t sum = 0;
                if (tid < (pass < 2 ? kEvictBins / 8 : 32)) {                          // 8 bins a thread
                    const uint4 c = *reinterpret_cast<const uint4*>(&hist[tid * 8]), e = *reinterpret_cast<const uint4*>(&hist[tid * 8 + 4]);
                    sum = ((c.x + c.y) + (c.z + c.w)) + ((e.x + e.y) + (e.z + e.w));
                }
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                if ((tid & 3) == 0 && tid < kEvictBins / 8) s.group[pass][tid >> 2] = sum;
            }
            // The bin in two steps: its group of 32, by the groups' sums, then the bin.  Every warp finds it for itself; a warp per CTA of the
            // cluster fetches that CTA's counts (128 and 32 words: all 2048 of a smaller digit from all CTAs took 3 us a pass).
            uint4 g = make_uint4(0u, 0u, 0u, 0u);                    // of the groups 4 lane .. 4 lane + 3, all CTAs
            if (ranks > 1) {
                cluster_sync_all();
                if (warp < ranks)
                    *reinterpret_cast<uint4*>(&s.rank_group[warp][4 * lane]) = ld_cluster_v4(cluster_map_shared(smem_u32(&s.group[pass][4 * lane]), uint32_t(warp)));
                __syncthreads();
#pragma unroll 8
                for (int r = 0; r < ranks; ++r) {
                    const uint4 v = *reinterpret_cast<const uint4*>(&s.rank_group[r][4 * lane]);
                    g.x += v.x; g.y += v.y; g.z += v.z; g.w += v.w;
                }
            } else {
                __syncthreads();
                g = *reinterpret_cast<const uint4*>(&s.group[pass][4 * lane]);
            }
            auto above = [&](uint32_t v) {                           // sum over the lanes above this one
                uint32_t incl = v;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const uint32_t up = __shfl_down_sync(0xffffffffu, incl, off);
                    if (lane + off < 32) incl += up;
                }
                return incl - v;
            };
            const uint32_t sum4 = (g.x + g.y) + (g.z + g.w);
            uint32_t over = above(sum4);                             // keys above this lane's groups
            int at = __ffs(__ballot_sync(0xffffffffu, over < left && over + sum4 >= left)) - 1;   // one lane
            int group = 4 * lane + 3;
            if (over + g.w < left) { over += g.w; --group;
                if (over + g.z < left) { over += g.z; --group;
                    if (over + g.y < left) { over += g.y; --group; } } }
            group = __shfl_sync(0xffffffffu, group, at);
            left -= __shfl_sync(0xffffffffu, over, at);
            uint32_t c = 0;                                          // of this lane's bin of the group, all CTAs
            if (ranks > 1) {
                if (warp < ranks) {
                    uint32_t v;
                    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_map_shared(smem_u32(&hist[group * 32 + lane]), uint32_t(warp))) : "memory");
                    s.rank_bin[warp][lane] = v;
                }
                __syncthreads();
#pragma unroll 8
                for (int r = 0; r < ranks; ++r) c += s.rank_bin[r][lane];
            } else {
                c = hist[group * 32 + lane];
            }
            over = above(c);
            at = __ffs(__ballot_sync(0xffffffffu, over < left && over + c >= left)) - 1;
            prefix = (prefix << bits) | uint32_t(group * 32 + at);
            left -= __shfl_sync(0xffffffffu, over, at);
            count = __shfl_sync(0xffffffffu, c, at);
            if (count == left) break;                                // all that agree stay (the same in every CTA)
        }
        if (shift > 0 || count == left) {
            // key >= prefix << shift; where that is 0, every key, as `thr` and `ties` have it already
            const uint32_t least = prefix << shift;
            if (least != 0u) {
                thr = least - 1u;
                ties = 0u;
            }
        } else {
            thr = prefix;
            ties = left;
        }
    }

    // ---- positions and weights of the kept keys, in order ----
    uint32_t gt = 0, eq = 0;
    if (some) {
        each([&](int, uint32_t k) {
            gt += k > thr;
            eq += k == thr;
        });
    } else if (want > 0) {
        gt = uint32_t(mine);                                         // every key
    }
    uint32_t gt_incl = gt, eq_incl = eq;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t a = __shfl_up_sync(0xffffffffu, gt_incl, off), e = __shfl_up_sync(0xffffffffu, eq_incl, off);
        if (lane >= off) { gt_incl += a; eq_incl += e; }
    }
    if (lane == 31) { s.warp_gt[warp] = gt_incl; s.warp_eq[warp] = eq_incl; }
    __syncthreads();
    const uint32_t w_gt = lane < NT / 32 ? s.warp_gt[lane] : 0u, w_eq = lane < NT / 32 ? s.warp_eq[lane] : 0u;
    uint32_t gt_before = __reduce_add_sync(0xffffffffu, lane < warp ? w_gt : 0u) + gt_incl - gt;
    uint32_t eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? w_eq : 0u) + eq_incl - eq;
    if (ranks > 1) {
        const uint32_t gt_all = __reduce_add_sync(0xffffffffu, w_gt), eq_all = __reduce_add_sync(0xffffffffu, w_eq);
        if (tid == 0) { s.cta_gt = gt_all; s.cta_eq = eq_all; }
        cluster_sync_all();
        // a lane per CTA before this one
        const uint2 v = lane < rank ? ld_cluster_v2(cluster_map_shared(smem_u32(&s.cta_gt), uint32_t(lane))) : make_uint2(0u, 0u);
        gt_before += __reduce_add_sync(0xffffffffu, v.x);
        eq_before += __reduce_add_sync(0xffffffffu, v.y);
        cluster_arrive();                                            // no CTA leaves before all have read the others' counts
    }
    uint32_t at = gt_before + min(eq_before, ties);
    auto keep = [&](int j) {
        index[at] = first + r0 + j;
        if (mass_out) mass_out[at] = weight(j);
        ++at;
    };
    if (some) {
        each([&](int j, uint32_t k) {
            const bool tie = k == thr;
            if (k > thr || (tie && eq_before < ties)) keep(j);
            eq_before += tie;
        });
    } else if (want > 0) {
        for (int j = 0; j < mine; ++j) keep(j);
    }
    // the recent keys, and -1 behind the last one kept
    for (int i = rank * NT + tid; i < p.n_keep - want; i += ranks * NT) {
        index[want + i] = i < recent ? old + i : -1;
        if (i < recent && mass_out) mass_out[want + i] = mass[old + i];
    }
    if (ranks > 1) cluster_wait();
}

constexpr int kEvictGatherThreads = 256;
constexpr int kEvictGatherPieces = 1024;          // 16-byte pieces of K (and as many of V) of a CTA: 4 a thread, all on their way at once

// grid (blocks of output positions, B): a block copies K and V of `rows` consecutive output positions, all heads.
template <int D>
__global__ void __launch_bounds__(kEvictGatherThreads)
evict_gather_kernel(const EvictParams p, int rows) {
    constexpr int CH = D / 8;                                        // 16-byte pieces of a row
    extern __shared__ int s_index[];                                 // [rows][Hk]
    const int b = blockIdx.y, n0 = int(blockIdx.x) * rows;
    const int kept = min(p.n_keep, evict_len(p, b));                 // the same of the old length and of the new one
    grid_dependency_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0 && p.lens_out) p.lens_out[b] = kept;   // every head's selection has ended
    const int here = min(rows, kept - n0);
    if (here <= 0) return;
    for (int e = threadIdx.x; e < here * p.Hk; e += kEvictGatherThreads) {
        const int hk = e / here, r = e - hk * here;
        s_index[r * p.Hk + hk] = __ldcg(p.index + (size_t(b) * p.Hk + hk) * p.n_keep + n0 + r);
    }
    __syncthreads();
    const uint4* K = reinterpret_cast<const uint4*>(p.K) + size_t(b) * p.T_cap * p.Hk * CH;
    const uint4* V = reinterpret_cast<const uint4*>(p.V) + size_t(b) * p.T_cap * p.Hk * CH;
    uint4* K_out = reinterpret_cast<uint4*>(p.K_out) + (size_t(b) * p.T_out + n0) * p.Hk * CH;
    uint4* V_out = reinterpret_cast<uint4*>(p.V_out) + (size_t(b) * p.T_out + n0) * p.Hk * CH;
    const int pieces = here * p.Hk * CH;
    constexpr int UN = 4;
    for (int e0 = threadIdx.x; e0 < pieces; e0 += UN * kEvictGatherThreads) {
        uint4 k[UN], v[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int e = e0 + u * kEvictGatherThreads;
            if (e < pieces) {
                const int row = e / CH, hk = row % p.Hk;
                const size_t src = (size_t(s_index[row]) * p.Hk + hk) * CH + e % CH;
                k[u] = __ldcs(K + src);
                v[u] = __ldcs(V + src);
            }
        }
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int e = e0 + u * kEvictGatherThreads;
            if (e < pieces) {
                K_out[e] = k[u];
                V_out[e] = v[u];
            }
        }
    }
}

}  // namespace moda
