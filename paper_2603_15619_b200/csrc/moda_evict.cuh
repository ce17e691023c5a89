// Eviction from a sequence cache by accumulated attention weight: of the len keys of a (sequence, key/value head) the
// kept = min(n_keep, len) stay: the last min(n_recent, kept) ones, and of the older ones those of largest weight (equal weights: the lower
// position; NaN counts as less than everything).  They keep their order.
//
//   evict_select_kernel  a cluster of 1 to 8 CTAs per (sequence, head): the weight of the last key kept is found digit by digit (radix
//                        11 + 11 + 10 bits of the weight's order-preserving integer), by a histogram of the keys that agree with the digits
//                        found so far; each CTA counts its share of the keys, held in its shared memory where they fit, and the
//                        cluster's counts are added over distributed shared memory.  Then every warp counts what it keeps of its share and writes
//                        positions and weights behind what is kept before it.
//   evict_gather_kernel  copies the kept K and V rows, all heads of a few output positions per CTA: bound by HBM (each row read and
//                        written once).
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

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
    int* lens_out;                // [B], may be null
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

constexpr int kEvictThreads = 512;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictBins = 2048;
constexpr int kEvictKeys = 48 * 1024;             // keys of a CTA's share that its shared memory holds

struct EvictShared {
    uint32_t hist[kEvictBins];
    uint32_t scan[kEvictWarps];
    uint32_t found_bin, found_above;
    uint32_t warp_gt[kEvictWarps], warp_eq[kEvictWarps];
    uint32_t cta_gt, cta_eq;
};
inline int evict_select_smem(int keys) { return int(sizeof(EvictShared)) + (keys < kEvictKeys ? keys : kEvictKeys) * 4; }

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

// grid (cluster, Hk, B)
__global__ void __launch_bounds__(kEvictThreads)
evict_select_kernel(const EvictParams p) {
    extern __shared__ __align__(16) uint8_t evict_smem[];
    EvictShared& s = *reinterpret_cast<EvictShared*>(evict_smem);
    uint32_t* held = reinterpret_cast<uint32_t*>(evict_smem + sizeof(EvictShared));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int ranks = gridDim.x, rank = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
    const int len = evict_len(p, b);
    const int kept = min(p.n_keep, len), recent = min(p.n_recent, kept);
    const int old = len - recent, want = kept - recent;              // `want` of the `old` first keys stay
    const float* mass = p.mass + (size_t(b) * p.Hk + hk) * p.T_cap;
    int* index = p.index + (size_t(b) * p.Hk + hk) * p.n_keep;
    float* mass_out = p.mass_out ? p.mass_out + (size_t(b) * p.Hk + hk) * p.T_out : nullptr;

    // the shares of CTAs and, within them, of warps are runs of whole 32-key steps
    const int share = ((old + ranks - 1) / ranks + 32 * kEvictWarps - 1) / (32 * kEvictWarps) * (32 * kEvictWarps);
    const int first = min(rank * share, old), n = min(share, old - first);
    const bool fits = n <= kEvictKeys;
    grid_launch_dependents();

    uint32_t above_thr = 0xffffffffu, ties = 0;                      // kept: key > above_thr, and the first `ties` keys equal to it
    if (want == old) {
        above_thr = 0u;
        ties = uint32_t(old);                                        // everything: keys above 0, and all that equal 0
    } else if (want > 0) {
        if (fits)
            for (int i = tid; i < n; i += kEvictThreads) held[i] = evict_key(mass[first + i]);
        uint32_t prefix = 0, left = uint32_t(want);                  // digits found; keys still to take among those that agree
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
            for (int i = tid; i < kEvictBins; i += kEvictThreads) s.hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < n; i += kEvictThreads) {
                const uint32_t k = fits ? held[i] : evict_key(mass[first + i]);
                const bool agrees = pass == 0 || (pass == 1 ? (k >> 21) == prefix : (k >> 10) == prefix);
                if (agrees) atomicAdd(&s.hist[(k >> shift) & uint32_t(bins - 1)], 1u);
            }
            // the cluster's counts of this thread's four bins
            uint4 c;
            if (ranks > 1) {
                cluster_sync_all();
                c = make_uint4(0u, 0u, 0u, 0u);
                const uint32_t at = smem_u32(&s.hist[tid * 4]);
#pragma unroll 4
                for (int r = 0; r < ranks; ++r) {
                    const uint4 v = ld_cluster_v4(cluster_map_shared(at, uint32_t(r)));
                    c.x += v.x; c.y += v.y; c.z += v.z; c.w += v.w;
                }
            } else {
                __syncthreads();
                c = *reinterpret_cast<const uint4*>(&s.hist[tid * 4]);
            }
            // keys in this thread's bins and those above (a scan from the top bin down)
            const uint32_t mine = c.x + c.y + c.z + c.w;
            uint32_t incl = mine;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const uint32_t v = __shfl_down_sync(0xffffffffu, incl, off);
                if (lane + off < 32) incl += v;
            }
            if (lane == 0) s.scan[warp] = incl;
            __syncthreads();
            uint32_t over = incl - mine;                             // keys above this thread's bins
#pragma unroll
            for (int w = 0; w < kEvictWarps; ++w)
                if (w > warp) over += s.scan[w];
            const uint32_t cc[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int j = 3; j >= 0; --j) {
                if (over < left && over + cc[j] >= left) { s.found_bin = uint32_t(tid * 4 + j); s.found_above = over; }
                over += cc[j];
            }
            if (ranks > 1) cluster_sync_all();                       // the counts have been read: they may be cleared
            else __syncthreads();
            prefix = (prefix << (pass == 2 ? 10 : 11)) | s.found_bin;
            left -= s.found_above;
        }
        above_thr = prefix;
        ties = left;
    }

    // ---- positions and weights of the kept keys, in order ----
    const int seg = share / kEvictWarps;                             // keys of a warp, a multiple of 32
    const int w0 = min(warp * seg, n), w1 = min(w0 + seg, n);
    auto key_of = [&](int i) { return fits && want > 0 && want < old ? held[i] : evict_key(mass[first + i]); };
    uint32_t gt = 0, eq = 0;
    if (want > 0) {
        for (int i0 = w0; i0 < w1; i0 += 32) {
            const int i = i0 + lane;
            const uint32_t k = i < w1 ? key_of(i) : 0u;
            gt += __popc(__ballot_sync(0xffffffffu, i < w1 && k > above_thr));
            eq += __popc(__ballot_sync(0xffffffffu, i < w1 && k == above_thr));
        }
    }
    if (lane == 0) { s.warp_gt[warp] = gt; s.warp_eq[warp] = eq; }
    __syncthreads();
    if (tid == 0) {
        uint32_t a = 0, e = 0;
        for (int w = 0; w < kEvictWarps; ++w) { a += s.warp_gt[w]; e += s.warp_eq[w]; }
        s.cta_gt = a;
        s.cta_eq = e;
    }
    if (ranks > 1) cluster_sync_all();
    else __syncthreads();
    uint32_t gt_before = 0, eq_before = 0;
    for (int r = 0; r < rank; ++r) {
        const uint2 v = ld_cluster_v2(cluster_map_shared(smem_u32(&s.cta_gt), uint32_t(r)));
        gt_before += v.x;
        eq_before += v.y;
    }
    for (int w = 0; w < warp; ++w) { gt_before += s.warp_gt[w]; eq_before += s.warp_eq[w]; }
    if (want > 0) {
        const uint32_t below = (1u << lane) - 1u;
        for (int i0 = w0; i0 < w1; i0 += 32) {
            const int i = i0 + lane;
            const uint32_t k = i < w1 ? key_of(i) : 0u;
            const uint32_t bg = __ballot_sync(0xffffffffu, i < w1 && k > above_thr);
            const uint32_t be = __ballot_sync(0xffffffffu, i < w1 && k == above_thr);
            const uint32_t my_eq = eq_before + __popc(be & below);   // equal keys before this one
            const bool is_gt = (bg >> lane) & 1u, is_eq = ((be >> lane) & 1u) && my_eq < ties;
            if (is_gt || is_eq) {
                const uint32_t at = gt_before + __popc(bg & below) + min(my_eq, ties);
                index[at] = first + i;
                if (mass_out) mass_out[at] = mass[first + i];
            }
            gt_before += __popc(bg);
            eq_before += __popc(be);
        }
    }
    // the recent keys, and -1 behind the last one kept
    for (int i = rank * kEvictThreads + tid; i < p.n_keep - want; i += ranks * kEvictThreads) {
        index[want + i] = i < recent ? old + i : -1;
        if (i < recent && mass_out) mass_out[want + i] = mass[old + i];
    }
    if (rank == 0 && hk == 0 && tid == 0 && p.lens_out) p.lens_out[b] = kept;
    if (ranks > 1) cluster_sync_all();                               // no CTA leaves while another reads its counts
}

constexpr int kEvictGatherThreads = 256;
constexpr int kEvictGatherRows = 32;              // (output position, head) pairs of a CTA, per 16 bytes of a row and 8 threads

// grid (blocks of output positions, B): a block copies K and V of `rows` consecutive output positions, all heads.
template <int D>
__global__ void __launch_bounds__(kEvictGatherThreads)
evict_gather_kernel(const EvictParams p, int rows) {
    constexpr int CH = D / 8;                                        // 16-byte pieces of a row
    extern __shared__ int s_index[];                                 // [rows][Hk]
    const int b = blockIdx.y, n0 = int(blockIdx.x) * rows;
    const int kept = min(p.n_keep, evict_len(p, b));
    grid_dependency_wait();
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
