// Decode step of a batch whose sequences share a prefix: every token attends, under one softmax, to the P keys of the prefix (one
// copy for the batch), to the keys of its sequence's own cache and to its l depth pairs.
//
//   shared_prefix_kernel   the prefix part, once for all sequences: the B G query rows that share a key/value head are the rows of
//                          tcgen05 tiles (128 rows = S = 128 / G sequences with the G heads of the group), so a key is read once per 256 rows
//                          instead of once per sequence, and the products run at the tensor cores' rate.
//   decode_split_tma_kernel  the sequences' own caches (moda_decode.cuh)
//   shared_merge_kernel    joins the partials of both with the depth pairs; short own caches it reads itself.
//
// shared_prefix_kernel: teams of CTAs take the same key tiles at the same time.  With one row tile, where the bytes of K and V set the pace, a
// team has adjacent kv heads, whose rows are adjacent in memory (a head alone is read in pieces of 2 d bytes: B = 37, 131072 keys,
// 8 heads, d = 64: 85 us, 58 us with teams of 8); with several it has the row tiles of a kv head, so that all but one find K and V in L2 (B = 128, 131072 keys, 32
// heads on 8, alone -> in teams: d = 128 249 -> 218 us, d = 64 228 -> 174).  The 128-key tiles of all groups of a team's size (heads, or a head's pairs of row tiles), in this
// order, are cut into equal runs, one per team; a CTA leaves a partial (m, l, o) per row for the part of each group that its run covers (a piece).  384 threads:
//
//   warps 0-3, 4-7   two streams, one thread per row: a score tile goes into registers at once, so that its columns can take the next one; maximum,
//                    exponentials and sum; P to columns of its own, in bf16 as the product with V takes it (a probability off by 2^-9 at most; the sum is that of the
//                    fp32 values; with V's and O's own bf16 the output is 0.0023 off in rel. L2, of which the rounding of O alone makes 0.0017)
//   warp 8 TMA producer (K tiles one ahead of V tiles)      warp 9 issues S = Q K^T of both streams, owns TMEM      warp 10 O += P V of both
//
// With a pair of row tiles the streams are its two tiles and both use every K, V tile.  With one row tile (few rows: bound by the bytes
// of K and V) they take the key tiles in turn and each leaves a partial of its own.
// ptxas gives the kernel 168 registers and spills 76 bytes (148 to 152 loaded), in the softmax warps around their 128 scores.
// TMEM columns: d = 128: [0,128) scores, of the streams in turn, [128,256) P, [256,512) O; d = 64: [0,256) scores, [256,384) P, [384,512) O.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda.h>
#include <cuda_runtime.h>

#include "moda_decode.cuh"
#include "moda_keymass.cuh"      // PipeWait
#include "sm100_ptx.cuh"

namespace moda {

constexpr int kSpThreads = 384;
constexpr int kSharedCtas = 148;       // most runs of a call: the workspace has room for their partials

struct SharedParams {
    int B, P, H, Hk, G;
    int S;                        // sequences of a row tile: 128 / G
    int row_tiles, pairs;         // row tiles; groups of two of them (1: one stream per key tile in turn)
    int key_tiles;                // 128-key tiles of the prefix
    int team;                     // CTAs of a team: divides Hk (one row tile) or pairs
    int total, run;               // key tiles of all groups, of a team
    int pieces;                   // partials that a row has room for
    int k_slots, v_slots;         // of shared memory, behind one or two row tiles
    float* o;                     // [pieces][B][H][d]
    float2* ml;                   // [pieces][B][H]: maximum (log2 domain), row sum
    float scale_log2;
};

// The group of a team's size that kv head `hk` and pair `pair` of row tiles belong to.
__host__ __device__ inline int shared_group(const SharedParams& p, int hk, int pair) {
    return p.row_tiles > 1 ? hk * (p.pairs / p.team) + pair / p.team : hk / p.team;
}
// Partials of a row: a piece per run that touches its group, two with one row tile (a stream each).
inline __host__ __device__ int shared_first_run(int group, int key_tiles, int run) { return int((long long)group * key_tiles / run); }

template <int D>
struct SharedSmem {
    static constexpr int kTileBytes = 128 * D * 2;
    static constexpr int kSubBytes = 128 * 128;
    static constexpr int kTiles = D == 128 ? 7 : 14;               // row tiles, K slots, V slots
    static constexpr int kMaxSlots = 6;
    static constexpr int kBars = kTiles * kTileBytes;
    static constexpr int kNumBars = 4 * kMaxSlots + 12;
    static constexpr int kMisc = kBars + kNumBars * 8;             // tmem base, abort word
    static constexpr int kTotal = kMisc + 16;
    static constexpr int kDynamic = kTotal + 1024;
    static_assert(kDynamic <= 232448, "shared memory");
};
inline void shared_slots(int d, bool paired, int& k_slots, int& v_slots) {
    k_slots = d == 64 ? 6 : paired ? 2 : 3;
    v_slots = d == 64 ? 6 : 3;
}

enum SharedBar : int {
    kSpKFull = 0,      // +slot (<= 6)
    kSpKEmpty = 6,
    kSpVFull = 12,
    kSpVEmpty = 18,
    kSpQFull = 24,
    kSpSFull = 25,     // +stream
    kSpXFree = 27,     // +stream (d = 64), one for both (d = 128): the scores are in registers
    kSpPFull = 29,     // +stream
    kSpODone = 31,     // +stream: P has been read, O holds everything up to this tile
    kSpPieceDone = 33, // O has been read
    kSpDrain = 34,     // +issuer
};

// A CTA's run, piece by piece.
struct SharedWalk {
    int group, j0, j1;            // key tiles of the piece
    int at, end;
    __device__ __forceinline__ void set(const SharedParams& p) {
        group = at / p.key_tiles;
        j0 = at - group * p.key_tiles;
        j1 = min(p.key_tiles, j0 + end - at);
    }
    __device__ __forceinline__ void next(const SharedParams& p) {
        at += j1 - j0;
        if (at < end) set(p);
    }
};

template <int D>
__global__ void __launch_bounds__(kSpThreads, 1)
shared_prefix_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
                     const __grid_constant__ CUtensorMap mapV, const SharedParams p) {
    using L = SharedSmem<D>;
    constexpr int NSUB = D / 64;
    constexpr int NX = D == 64 ? 2 : 1;                                // score buffers
    constexpr uint32_t kColP = NX * 128, kColO = kColP + 128;
    if (g_moda_status != 0) return;   // an earlier kernel gave up a wait: do not pile up more timeouts
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sbase = smem_u32(smem);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kMisc + 4);
    auto bar = [&](int i) { return sbase + L::kBars + 8u * uint32_t(i); };
    const PipeWait wait{abort_flag};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool paired = p.row_tiles > 1;
    const int rows = p.S * p.G, q_tiles = paired ? 2 : 1;
    const uint32_t sK = sbase + q_tiles * L::kTileBytes, sV = sK + p.k_slots * L::kTileBytes;

    if (tid == 0) {
        *abort_flag = 0;
        for (int s = 0; s < L::kMaxSlots; ++s) {
            mbar_init(bar(kSpKFull + s), 1);
            mbar_init(bar(kSpKEmpty + s), 1);
            mbar_init(bar(kSpVFull + s), 1);
            mbar_init(bar(kSpVEmpty + s), 1);
        }
        mbar_init(bar(kSpQFull), 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(kSpSFull + s), 1);
            mbar_init(bar(kSpXFree + s), 128);
            mbar_init(bar(kSpPFull + s), 128);
            mbar_init(bar(kSpODone + s), 1);
            mbar_init(bar(kSpDrain + s), 1);
        }
        mbar_init(bar(kSpPieceDone), 256);
        fence_mbar_init();
    }
    if (warp == 9) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    // rows of the Q tiles that no box covers stay zero
    if (rows < 128) {
        for (int e = tid; e < q_tiles * NSUB * (128 - rows) * 8; e += kSpThreads) {
            const int piece = e & 7, r = rows + (e >> 3) % (128 - rows), sub = (e >> 3) / (128 - rows);
            *reinterpret_cast<uint4*>(smem + sub * L::kSubBytes + r * 128 + piece * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async_smem();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    grid_launch_dependents();                                          // the split kernel of the sequences' own caches takes the SMs that this one leaves
    const uint32_t tmem = *tmem_slot;
    SharedWalk w;
    const int my_team = int(blockIdx.x) / p.team, member = int(blockIdx.x) % p.team;
    auto place = [&](int group) {                                      // kv head and pair of row tiles of this CTA
        if (!paired) return make_int2(group * p.team + member, 0);
        const int per_head = p.pairs / p.team, hk = group / per_head;
        return make_int2(hk, (group - hk * per_head) * p.team + member);
    };
    w.at = my_team * p.run;
    w.end = min(w.at + p.run, p.total);
    w.set(p);

    if (warp < 8) {
        // =========================== softmax of stream s: thread = row ===========================
        setmaxnreg_inc<208>();
        const int s = warp >> 2, r = tid & 127;
        const uint32_t lane_addr = uint32_t((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lane_addr + (NX == 2 ? s * 128 : 0), tP = tmem + lane_addr + kColP + s * 64, tO = tmem + lane_addr + kColO + s * D;
        const uint32_t x_free = bar(kSpXFree + (NX == 2 ? s : 0));
        int n = 0, tile0 = 0;                                          // tiles of this stream so far; key tiles of the CTA before the piece
#pragma unroll 1
        while (w.at < w.end) {
            const int2 at = place(w.group);
            const int hk = at.x, pair = at.y;
            float m_ref = -INFINITY, l_sum = 0.f;
            int in_piece = 0;
            // one row tile: the CTA's key tiles in turn, whatever piece they belong to
#pragma unroll 1
            for (int j = w.j0 + (paired ? 0 : (tile0 ^ s) & 1); j < w.j1; j += paired ? 1 : 2, ++n, ++in_piece) {
                wait(bar(kSpSFull + s), n & 1, 150);
                tc_fence_after_sync();
                uint32_t sv[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, sv[c]);
                tmem_wait_ld();
                tc_fence_before_sync();
                mbar_arrive(x_free);
                const int keys = p.P - j * 128;
                if (keys < 128) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c * 32 + i >= keys) sv[c][i] = 0xff800000u;
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        m0 = max3(m0, __uint_as_float(sv[c][i]), __uint_as_float(sv[c][i + 1]));
                        m1 = max3(m1, __uint_as_float(sv[c][i + 2]), __uint_as_float(sv[c][i + 3]));
                    }
                    mx[c] = fmaxf(m0, m1);
                }
                const float m_new = fmaxf(m_ref, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2);
                // The reference moves only when some row of the warp grew by more than 2^8 (the accesses to tensor memory are warp-wide).
                const bool move = in_piece == 0 || __any_sync(0xffffffffu, m_new - m_ref > 8.f);
                if (n > 0) wait(bar(kSpODone + s), (n - 1) & 1, 151);  // P of the tile before has been read, O is complete up to it
                if (move) {
                    if (in_piece > 0) {
                        tc_fence_after_sync();
                        const float f = fast_exp2(m_ref - m_new);
                        l_sum *= f;
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t o[16];
                            tmem_ld16(tO + c * 16, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tmem_st16(tO + c * 16, o);
                        }
                    }
                    m_ref = m_new;
                }
                const float neg_m = -m_ref;
                tc_fence_after_sync();
                float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        float a0, a1, b0, b1;
                        fma2_scale(__uint_as_float(sv[c][2 * i]), __uint_as_float(sv[c][2 * i + 1]), p.scale_log2, neg_m, a0, a1);
                        fma2_scale(__uint_as_float(sv[c][2 * i + 2]), __uint_as_float(sv[c][2 * i + 3]), p.scale_log2, neg_m, b0, b1);
                        a0 = fast_exp2(a0);
                        a1 = fast_exp2(a1);
                        b0 = fast_exp2(b0);
                        b1 = fast_exp2(b1);
                        add2_f32(a0, a1, s0, s1);
                        add2_f32(b0, b1, s2, s3);
                        pk[i] = pack_bf16x2(a0, a1);
                        pk[i + 1] = pack_bf16x2(b0, b1);
                    }
                    tmem_st16(tP + c * 16, pk);
                }
                l_sum += (s0 + s1) + (s2 + s3);
                tmem_wait_st();
                tc_fence_before_sync();
                mbar_arrive(bar(kSpPFull + s));
            }
            tile0 += w.j1 - w.j0;
            // ---- the piece's partial of this row ----
            const int cta0 = shared_first_run(w.group, p.key_tiles, p.run);
            const int index = paired ? my_team - cta0 : 2 * (my_team - cta0) + s;
            const int b = (paired ? 2 * pair + s : 0) * p.S + r / p.G;
            const bool there = r < rows && b < p.B;
            const size_t row = (size_t(index) * p.B + b) * p.H + hk * p.G + r % p.G;
            if (in_piece > 0) {
                wait(bar(kSpODone + s), (n - 1) & 1, 152);
                tc_fence_after_sync();
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tO + c * 32, o);
                    tmem_wait_ld();
                    if (there) {
                        float4* dst = reinterpret_cast<float4*>(p.o + row * D + c * 32);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            dst[i] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]), __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
                    }
                }
            }
            if (there) p.ml[row] = make_float2(m_ref, l_sum);         // -inf, 0: a stream without a key tile in the piece
            tc_fence_before_sync();
            mbar_arrive(bar(kSpPieceDone));
            w.next(p);
        }
    } else {
      setmaxnreg_dec<88>();
      if (warp == 8) {
        // =========================== TMA producer ===========================
        if (lane == 0) {
            tma_prefetch_desc(&mapQ);
            tma_prefetch_desc(&mapK);
            tma_prefetch_desc(&mapV);
            RingAt ka, va;
            auto load = [&](const CUtensorMap& map, RingAt& at, uint32_t ring, int full, int empty, int slots, int hk, int j) {
                if (at.round > 0) wait(bar(empty + at.slot), (at.round - 1) & 1, 161);
                mbar_arrive_expect_tx(bar(full + at.slot), L::kTileBytes);
#pragma unroll
                for (int s = 0; s < NSUB; ++s)
                    tma_load_4d(ring + at.slot * L::kTileBytes + s * L::kSubBytes, &map, bar(full + at.slot), s * 64, hk, j * 128, 0);
                at.next(slots);
            };
            int piece = 0;
#pragma unroll 1
            for (; w.at < w.end; ++piece) {
                const int2 at = place(w.group);
                const int hk = at.x, pair = at.y;
                load(mapK, ka, sK, kSpKFull, kSpKEmpty, p.k_slots, hk, w.j0);
                if (piece > 0) wait(bar(kSpPieceDone), (piece - 1) & 1, 160);   // every product of the piece before is complete
                mbar_arrive_expect_tx(bar(kSpQFull), uint32_t(q_tiles * rows) * D * 2);
                for (int t = 0; t < q_tiles; ++t)
#pragma unroll
                    for (int s = 0; s < NSUB; ++s)
                        tma_load_4d(sbase + t * L::kTileBytes + s * L::kSubBytes, &mapQ, bar(kSpQFull), s * 64, hk * p.G, (2 * pair + t) * p.S, 0);
#pragma unroll 1
                for (int j = w.j0; j < w.j1; ++j) {
                    if (j + 1 < w.j1) load(mapK, ka, sK, kSpKFull, kSpKEmpty, p.k_slots, hk, j + 1);
                    load(mapV, va, sV, kSpVFull, kSpVEmpty, p.v_slots, hk, j);
                }
                w.next(p);
            }
        }
      } else if (warp == 9) {
        // =========================== S = Q K^T of both streams ===========================
        constexpr uint32_t idesc = make_idesc_bf16(128, 128, false, false);
        const uint64_t dq0 = desc_kmajor_sw128(sbase, 0), dk0 = desc_kmajor_sw128(sK, 0);
        RingAt ka;
        int n = 0, piece = 0;                                          // products so far: stream n % 2
#pragma unroll 1
        for (; w.at < w.end; ++piece) {
            wait(bar(kSpQFull), piece & 1, 170);
#pragma unroll 1
            for (int j = w.j0; j < w.j1; ++j, ka.next(p.k_slots)) {
                wait(bar(kSpKFull + ka.slot), ka.round & 1, 171);
                const uint64_t dk = dk0 + uint64_t((ka.slot * L::kTileBytes) >> 4);
#pragma unroll 1
                for (int t = 0; t < q_tiles; ++t, ++n) {
                    const int s = n & 1;
                    // the buffer's last scores are in registers
                    if (NX == 1) { if (n > 0) wait(bar(kSpXFree), (n - 1) & 1, 172); }
                    else { if (n > 1) wait(bar(kSpXFree + s), ((n >> 1) - 1) & 1, 173); }
                    tc_fence_after_sync();
                    const uint64_t dq = dq0 + uint64_t((t * L::kTileBytes) >> 4);
                    const uint32_t tS = tmem + (NX == 2 ? s * 128 : 0);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint64_t o = uint64_t(((kk >> 2) * L::kSubBytes + (kk & 3) * 32) >> 4);
                        umma_ss(tS, dq + o, dk + o, idesc, kk > 0);
                    }
                    umma_commit(bar(kSpSFull + s));
                }
                umma_commit(bar(kSpKEmpty + ka.slot));
            }
            w.next(p);
        }
        if (*abort_flag != 0) {
            // A wait gave up somewhere: make sure no MMA of this warp is still in flight before TMEM is released.
            umma_commit(bar(kSpDrain));
            const uint64_t t0 = globaltimer_ns();
            while (!mbar_try_wait(bar(kSpDrain), 0) && globaltimer_ns() - t0 < 20000000ull) {}
        }
      } else if (warp == 10) {
        // =========================== O += P V of both streams ===========================
        constexpr uint32_t idesc = make_idesc_bf16(128, D, false, true);
        const uint64_t dv0 = desc_mnmajor_sw128(sV, 0, L::kSubBytes);
        RingAt va;
        int n = 0;
#pragma unroll 1
        while (w.at < w.end) {
#pragma unroll 1
            for (int j = w.j0; j < w.j1; ++j, va.next(p.v_slots)) {
                wait(bar(kSpVFull + va.slot), va.round & 1, 174);
                const uint64_t dv = dv0 + uint64_t((va.slot * L::kTileBytes) >> 4);
#pragma unroll 1
                for (int t = 0; t < q_tiles; ++t, ++n) {
                    const int s = n & 1;
                    wait(bar(kSpPFull + s), (n >> 1) & 1, 175);
                    tc_fence_after_sync();
                    const uint32_t tP = tmem + kColP + s * 64, tO = tmem + kColO + s * D;
                    const bool first = paired ? j == w.j0 : j - w.j0 < 2;     // of the stream in the piece
                    umma_ts(tO, tP, dv, idesc, !first);
#pragma unroll
                    for (int kk = 1; kk < 8; ++kk) umma_ts(tO, tP + kk * 8, dv + uint64_t(kk * 128), idesc, 1);
                    umma_commit(bar(kSpODone + s));
                }
                umma_commit(bar(kSpVEmpty + va.slot));
            }
            w.next(p);
        }
        if (*abort_flag != 0) {
            umma_commit(bar(kSpDrain + 1));
            const uint64_t t0 = globaltimer_ns();
            while (!mbar_try_wait(bar(kSpDrain + 1), 0) && globaltimer_ns() - t0 < 20000000ull) {}
        }
      }
    }

    tc_fence_before_sync();
    __syncthreads();
    abort_teardown(abort_flag, 256);
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 512);
}

// Per (b, query head): the prefix partials, the sequence's own pieces (or, of a short cache, its keys) and the token's depth pairs, by WPR
// warps.  It starts beside the kernels before it (programmatic dependent launch) and has the keys and depth pairs done when they end.
// Bound by latency and by the rows that an SM holds: few dependent loads, and few registers where there are many rows (l = 24, d = 128, one warp a row: with
// 4 loads of 16 bytes in flight 80 registers, with 2 64; 4096 rows 52.8 -> 47.1 us, 14240 rows of d = 64 35.5 -> 33.3).
constexpr int kSharedMergeThreads = 128;

struct SharedMergeParams {
    DecodeParams dec;             // own caches and depth pairs (T_kv == 0: none of the former)
    SharedParams pre;             // prefix (P == 0: none)
    int own_here;                 // the own caches are short: no split kernel has run, this one reads them
};

template <int D, int WPR>
__global__ void __launch_bounds__(kSharedMergeThreads)
shared_merge_kernel(const SharedMergeParams p) {
    constexpr int LPR = D / 8, KPL = 32 / LPR;                       // lanes of a key (16 bytes each), keys of a warp's load
    constexpr int ROWS = kSharedMergeThreads / 32 / WPR, UN = WPR > 1 ? 4 : 2;
    constexpr int kMost = 2 * (kSharedCtas + 1) + kDecodeMaxSplits;  // partials of a row: streams of the prefix, own pieces
    __shared__ float s_w[ROWS][kMost], s_red[2][ROWS][WPR];
    __shared__ __align__(16) float s_acc[ROWS][WPR][D];
    const DecodeParams& q = p.dec;
    const int warp = int(threadIdx.x >> 5) % WPR, lane = threadIdx.x & 31, tid = warp * 32 + lane;   // in the row
    const int sub = lane / LPR, col = lane % LPR * 8;                // key of a load, first of the lane's 8 elements
    const int row_in = int(threadIdx.x >> 5) / WPR;
    const int row = int(blockIdx.x) * ROWS + row_in;                 // b * H + h
    const bool there = ROWS == 1 || row < q.B * q.H;
    const int b = there ? row / q.H : 0, h = there ? row - b * q.H : 0;
    const int G = q.H / q.Hk, hk = h / G, g = h - hk * G;            // groups of at most 8 heads, as the split kernel has them
    const int Hk_real = q.Hk / q.kv_rep, hk_real = hk / q.kv_rep;
    float* w_of = s_w[row_in];
    auto sync = [] {
        if constexpr (WPR > 1) __syncthreads();
        else __syncwarp();
    };
    auto warp_max = [](float v) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
        return v;
    };
    auto warp_sum = [](float v) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
        return v;
    };
    auto unpack = [](const uint4& v, float (&x)[8]) {
        x[0] = bf16_lo_to_f32(v.x); x[1] = bf16_hi_to_f32(v.x); x[2] = bf16_lo_to_f32(v.y); x[3] = bf16_hi_to_f32(v.y);
        x[4] = bf16_lo_to_f32(v.z); x[5] = bf16_hi_to_f32(v.z); x[6] = bf16_lo_to_f32(v.w); x[7] = bf16_hi_to_f32(v.w);
    };
    // ---- a short own cache and the depth pairs, one pass: LPR lanes keep the running maximum, sum and o of every WPR KPL-th key ----
    const int own_len = q.T_kv == 0 ? 0 : q.seq_lens ? min(max(q.seq_lens[b], 0), q.T_kv) : q.T_kv;
    const int n_here = p.own_here ? own_len : 0, n_near = n_here + q.l;
    float acc[8], m_d = -INFINITY, l_d = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[c] = 0.f;
    if (n_near > 0) {
        float qv[8];
        unpack(*reinterpret_cast<const uint4*>(q.q + size_t(there ? row : 0) * D + col), qv);
#pragma unroll
        for (int c = 0; c < 8; ++c) qv[c] *= q.scale_log2;
        const size_t own0 = (size_t(b) * q.T_cap * Hk_real + hk_real) * D + col, own_stride = size_t(Hk_real) * D;
        const size_t depth0 = (size_t(b) * Hk_real + hk_real) * 2 * D + col, slot_stride = size_t(q.B) * Hk_real * 2 * D;
#pragma unroll 1
        for (int i0 = warp * KPL; i0 < n_near; i0 += WPR * KPL * UN) {
            uint4 k[UN], v[UN];
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                const int i = min(i0 + u * WPR * KPL + sub, n_near - 1);
                const bool own = i < n_here;
                const size_t at = own ? own0 + i * own_stride : depth0 + (i - n_here) * slot_stride;
                k[u] = *reinterpret_cast<const uint4*>((own ? q.K : q.depth) + at);
                v[u] = *reinterpret_cast<const uint4*>((own ? q.V : q.depth + D) + at);
            }
            float a[UN];
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                float x[8];
                unpack(k[u], x);
                a[u] = 0.f;
#pragma unroll
                for (int c = 0; c < 8; ++c) a[u] = fmaf(qv[c], x[c], a[u]);
            }
#pragma unroll
            for (int off = LPR / 2; off > 0; off >>= 1)
#pragma unroll
                for (int u = 0; u < UN; ++u) a[u] += __shfl_xor_sync(0xffffffffu, a[u], off);
            float m = m_d;
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                if (i0 + u * WPR * KPL + sub >= n_near) a[u] = -INFINITY;
                m = fmaxf(m, a[u]);
            }
            const float m_safe = m == -INFINITY ? 0.f : m, old = fast_exp2(m_d - m_safe);
            m_d = m;
            l_d *= old;
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[c] *= old;
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                const bool in = i0 + u * WPR * KPL + sub < n_near;
                const float f = fast_exp2(a[u] - m_safe);
                float x[8];
                unpack(in ? v[u] : make_uint4(0, 0, 0, 0), x);
                l_d += f;
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = fmaf(f, x[c], acc[c]);
            }
        }
    }
    int n_pre = 0;
    if (p.pre.P > 0) {
        const int group = shared_group(p.pre, h / p.pre.G, p.pre.row_tiles > 1 ? b / (2 * p.pre.S) : 0);
        const int c0 = shared_first_run(group, p.pre.key_tiles, p.pre.run);
        const int c1 = int(((long long)(group + 1) * p.pre.key_tiles - 1) / p.pre.run);
        n_pre = (c1 - c0 + 1) * (p.pre.row_tiles > 1 ? 1 : 2);
    }
    const float* group = q.part + (size_t(b) * q.Hk + hk) * kDecodeMaxSplits * G * (D + 2);
    const float* part = group + g * (D + 2);
    const size_t split_stride = size_t(G) * (D + 2);
    const size_t pre_stride = size_t(q.B) * q.H, pre_row = size_t(there ? row : 0);
    grid_dependency_wait();
    // ---- from here on: what the kernels before have written ----
    int n_own = 0;
    if (own_len > n_here)
        n_own = q.seq_lens ? min(max(__float_as_int(__ldcg(group + (kDecodeMaxSplits - 1) * split_stride)), 1), q.max_pieces)
                           : decode_pieces_equal(q.cut, b * (q.Hk / q.team) + hk / q.team, q.T_kv, q.unit_log2);
    const int n = n_pre + n_own;
    auto fetch_ml = [&](int i) {                                     // maximum, row sum of a partial
        if (i < n_pre) return __ldcg(p.pre.ml + i * pre_stride + pre_row);
        if (i < n) return __ldcg(reinterpret_cast<const float2*>(part + (i - n_pre) * split_stride));
        return make_float2(-INFINITY, 0.f);
    };
    // one partial a thread in registers, the others (very long prefixes, many runs) in shared memory
    const float2 ml = fetch_ml(tid);
    float mx = fmaxf(m_d, ml.x);
    for (int i = tid + 32 * WPR; i < n; i += 32 * WPR) mx = fmaxf(mx, fetch_ml(i).x);
    mx = warp_max(mx);
    if constexpr (WPR > 1) {
        if (lane == 0) s_red[0][row_in][warp] = mx;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WPR; ++w) mx = fmaxf(mx, s_red[0][row_in][w]);
    }
    // no key: 0; only NaN among the scores: NaN, as their sum is
    auto weight = [&](const float2& v) { return v.x == -INFINITY ? v.y : fast_exp2(v.x - mx); };
    float f = weight(ml), lt = f * ml.y;
    if (tid < n) w_of[tid] = f;
    for (int i = tid + 32 * WPR; i < n; i += 32 * WPR) {
        const float2 v = fetch_ml(i);
        w_of[i] = f = weight(v);
        lt = fmaf(f, v.y, lt);
    }
    const float f_d = weight(make_float2(m_d, l_d));
    lt = warp_sum(col == 0 ? fmaf(f_d, l_d, lt) : lt);
    if constexpr (WPR > 1) {
        if (lane == 0) s_red[1][row_in][warp] = lt;
    }
    sync();
    if constexpr (WPR > 1) {
        lt = s_red[1][row_in][0];
#pragma unroll
        for (int w = 1; w < WPR; ++w) lt += s_red[1][row_in][w];
    }
    // ---- weighted sum: LPR lanes take every WPR KPL-th partial, in pairs of columns so that a load takes whole sectors ----
    float2 o[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = make_float2(0.f, 0.f);
#pragma unroll 1
    for (int i0 = warp * KPL; i0 < n; i0 += WPR * KPL * UN) {
        float2 x[UN][4];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int i = min(i0 + u * WPR * KPL + sub, n - 1);
            const float* src = (i < n_pre ? p.pre.o + (i * pre_stride + pre_row) * D : part + (i - n_pre) * split_stride + 2) + col / 4;
#pragma unroll
            for (int c = 0; c < 4; ++c) x[u][c] = __ldcg(reinterpret_cast<const float2*>(src) + c * LPR);
        }
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int i = i0 + u * WPR * KPL + sub;
            const float wt = i < n ? w_of[i] : 0.f;
            if (wt != 0.f) {                                         // a stream without a key has written no o
#pragma unroll
                for (int c = 0; c < 4; ++c) o[c] = make_float2(fmaf(wt, x[u][c].x, o[c].x), fmaf(wt, x[u][c].y, o[c].y));
            }
        }
    }
#pragma unroll
    for (int off = LPR; off < 32; off <<= 1)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            o[c].x += __shfl_xor_sync(0xffffffffu, o[c].x, off);
            o[c].y += __shfl_xor_sync(0xffffffffu, o[c].y, off);
        }
    float* sum_of = s_acc[row_in][warp];
    if (n_near > 0) {
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[c] *= f_d;
#pragma unroll
        for (int off = LPR; off < 32; off <<= 1)
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[c] += __shfl_xor_sync(0xffffffffu, acc[c], off);
        if (sub == 0) {
#pragma unroll
            for (int c = 0; c < 8; c += 4) *reinterpret_cast<float4*>(sum_of + col + c) = make_float4(acc[c], acc[c + 1], acc[c + 2], acc[c + 3]);
        }
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float2 near = reinterpret_cast<const float2*>(sum_of + col / 4)[c * LPR];
            o[c] = make_float2(o[c].x + near.x, o[c].y + near.y);
        }
        __syncwarp();
    }
    // a row without any key: O = 0, LSE = -inf
    const float inv = lt > 0.f || lt != lt ? 1.f / lt : 0.f;
    if constexpr (WPR > 1) {
        if (sub == 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c) reinterpret_cast<float2*>(sum_of + col / 4)[c * LPR] = o[c];
        }
        __syncthreads();
        for (int c = tid; there && c < D; c += 32 * WPR) {
            float a = s_acc[row_in][0][c];
#pragma unroll
            for (int w = 1; w < WPR; ++w) a += s_acc[row_in][w][c];
            q.O[size_t(row) * D + c] = __float2bfloat16(inv == 0.f ? 0.f : a * inv);
        }
    } else if (there && sub == 0) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            reinterpret_cast<uint32_t*>(q.O + size_t(row) * D + col / 4)[c * LPR] = inv == 0.f ? 0u : pack_bf16x2(o[c].x * inv, o[c].y * inv);
    }
    if (tid == 0 && there) q.LSE[row] = (mx + log2f(lt)) * kDecodeLn2;
}

}  // namespace moda
