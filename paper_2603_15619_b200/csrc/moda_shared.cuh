// Decode step of a batch whose sequences share a prefix: every token attends, under one softmax, to the P keys of the prefix (one
// copy for the batch), to the keys of its sequence's own cache and to its l depth pairs.
//
//   shared_prefix_kernel   the prefix part, once for all sequences: the B G query rows that share a key/value head are the rows of
//                          tcgen05 tiles (128 rows = S = 128 / G sequences with the G heads of the group), so a key is read once per 256 rows
//                          instead of once per sequence, and the products run at the tensor cores' rate.
//   decode_split_tma_kernel  the sequences' own caches (moda_decode.cuh)
//   shared_merge_kernel    joins the partials of both with the depth pairs.
//
// shared_prefix_kernel: the 128-key tiles of all (kv head, pair of row tiles) groups, in this order, are cut into equal runs, one per
// CTA; a CTA leaves a partial (m, l, o) per row for the part of each group that its run covers (a piece).  384 threads:
//
//   warps 0-3, 4-7   two streams, one thread per row: maximum, exponentials and sum of a score tile; P goes back over the scores
//   warp 8 TMA producer      warps 9, 10 issue the products of streams 0, 1 (S = Q K^T, then O += P V); warp 9 owns TMEM
//
// With a pair of row tiles the streams are its two tiles and both use every K, V tile.  With one row tile (few rows: bound by the bytes
// of K and V) they take the key tiles in turn and each leaves a partial of its own.
// TMEM columns of a stream: [0,128) scores, P in the first 64 of them, [128, 128 + D) O.
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

struct SharedParams {
    int B, P, H, Hk, G;
    int S;                        // sequences of a row tile: 128 / G
    int row_tiles, pairs;         // row tiles; groups of two of them (1: one stream per key tile in turn)
    int key_tiles;                // 128-key tiles of the prefix
    int total, run;               // key tiles of all groups, of a CTA
    int pieces;                   // partials that a row has room for
    float* o;                     // [pieces][B][H][d]
    float2* ml;                   // [pieces][B][H]: maximum (log2 domain), row sum
    float scale_log2;
};

// Partials of a row: a piece per run that touches its group, two with one row tile (a stream each).
inline __host__ __device__ int shared_first_run(int group, int key_tiles, int run) { return int((long long)group * key_tiles / run); }

template <int D>
struct SharedSmem {
    static constexpr int kTileBytes = 128 * D * 2;
    static constexpr int kSubBytes = 128 * 128;
    static constexpr int kQ = 0;                                   // two row tiles
    static constexpr int kRing = 2 * kTileBytes;                   // K_0 V_0 K_1 V_1 ...
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int kBars = kRing + kStages * kTileBytes;
    static constexpr int kNumBars = 2 * kStages + 8;
    static constexpr int kMisc = kBars + kNumBars * 8;             // tmem base, abort word
    static constexpr int kTotal = kMisc + 16;
    static constexpr int kDynamic = kTotal + 1024;
    static_assert(kDynamic <= 232448, "shared memory");
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
    constexpr int NSUB = D / 64, NST = L::kStages;
    constexpr int kFull = 0, kEmpty = NST, kQFull = 2 * NST, kSFull = 2 * NST + 1, kPFull = 2 * NST + 3, kODone = 2 * NST + 5, kPieceDone = 2 * NST + 7;
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
    const int rows = p.S * p.G;

    if (tid == 0) {
        *abort_flag = 0;
        for (int s = 0; s < NST; ++s) {
            mbar_init(bar(kFull + s), 1);
            mbar_init(bar(kEmpty + s), paired ? 2 : 1);
        }
        mbar_init(bar(kQFull), 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(kSFull + s), 1);
            mbar_init(bar(kPFull + s), 128);
            mbar_init(bar(kODone + s), 1);
        }
        mbar_init(bar(kPieceDone), 256);
        fence_mbar_init();
    }
    if (warp == 9) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    // rows of the Q tiles that no box covers stay zero
    if (rows < 128) {
        for (int e = tid; e < 2 * NSUB * (128 - rows) * 8; e += kSpThreads) {
            const int piece = e & 7, r = rows + (e >> 3) % (128 - rows), sub = (e >> 3) / (128 - rows);
            *reinterpret_cast<uint4*>(smem + L::kQ + sub * L::kSubBytes + r * 128 + piece * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async_smem();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    SharedWalk w;
    w.at = int(blockIdx.x) * p.run;
    w.end = min(w.at + p.run, p.total);
    w.set(p);
    // Key tiles of a stream in a piece: all of them, or (one row tile) every second one.
    const int step = paired ? 1 : 2;

    if (warp < 8) {
        // =========================== softmax of stream s: thread = row ===========================
        const int s = warp >> 2, r = tid & 127;
        const uint32_t tS = tmem + (uint32_t((warp & 3) * 32) << 16) + s * 256, tO = tS + 128;
        int n = 0;                                                    // tiles of this stream so far
#pragma unroll 1
        while (w.at < w.end) {
            const int hk = w.group / p.pairs, pair = w.group - hk * p.pairs;
            float m_ref = -INFINITY, l_sum = 0.f;
            int in_piece = 0;
#pragma unroll 1
            for (int j = w.j0 + (paired ? 0 : s); j < w.j1; j += step, ++n, ++in_piece) {
                wait(bar(kSFull + s), n & 1, 150);
                tc_fence_after_sync();
                uint32_t sv[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, sv[c]);
                tmem_wait_ld();
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
                if (move) {
                    if (in_piece > 0) {
                        wait(bar(kODone + s), (n - 1) & 1, 151);      // O holds everything up to the tile before
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
                float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        float a0, a1, b0, b1;
                        fma2_scale(__uint_as_float(sv[c][2 * i]), __uint_as_float(sv[c][2 * i + 1]), p.scale_log2, -m_ref, a0, a1);
                        fma2_scale(__uint_as_float(sv[c][2 * i + 2]), __uint_as_float(sv[c][2 * i + 3]), p.scale_log2, -m_ref, b0, b1);
                        a0 = fast_exp2(a0);
                        a1 = fast_exp2(a1);
                        b0 = fast_exp2(b0);
                        b1 = fast_exp2(b1);
                        add2_f32(a0, a1, s0, s1);
                        add2_f32(b0, b1, s2, s3);
                        pk[i] = pack_bf16x2(a0, a1);
                        pk[i + 1] = pack_bf16x2(b0, b1);
                    }
                    tmem_st16(tS + c * 16, pk);
                }
                l_sum += (s0 + s1) + (s2 + s3);
                tmem_wait_st();
                tc_fence_before_sync();
                mbar_arrive(bar(kPFull + s));
            }
            // ---- the piece's partial of this row ----
            const int cta0 = shared_first_run(w.group, p.key_tiles, p.run);
            const int index = paired ? int(blockIdx.x) - cta0 : 2 * (int(blockIdx.x) - cta0) + s;
            const int b = (paired ? 2 * pair + s : 0) * p.S + r / p.G;
            const bool there = r < rows && b < p.B;
            const size_t row = (size_t(index) * p.B + b) * p.H + hk * p.G + r % p.G;
            if (in_piece > 0) {
                wait(bar(kODone + s), (n - 1) & 1, 152);
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
            mbar_arrive(bar(kPieceDone));
            w.next(p);
        }
    } else if (warp == 8) {
        // =========================== TMA producer ===========================
        if (lane == 0) {
            tma_prefetch_desc(&mapQ);
            tma_prefetch_desc(&mapK);
            tma_prefetch_desc(&mapV);
            int n = 0, piece = 0;
#pragma unroll 1
            for (; w.at < w.end; ++piece) {
                const int hk = w.group / p.pairs, pair = w.group - hk * p.pairs;
                if (piece > 0) wait(bar(kPieceDone), (piece - 1) & 1, 160);   // every product of the piece before is complete
                const int tiles = paired ? 2 : 1;
                mbar_arrive_expect_tx(bar(kQFull), uint32_t(tiles * rows) * D * 2);
                for (int t = 0; t < tiles; ++t)
#pragma unroll
                    for (int s = 0; s < NSUB; ++s)
                        tma_load_4d(sbase + L::kQ + t * L::kTileBytes + s * L::kSubBytes, &mapQ, bar(kQFull), s * 64, hk * p.G, (2 * pair + t) * p.S, 0);
#pragma unroll 1
                for (int j = w.j0; j < w.j1; ++j)
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv, ++n) {
                        const int st = n % NST;
                        if (n >= NST) wait(bar(kEmpty + st), (n / NST - 1) & 1, 161);
                        mbar_arrive_expect_tx(bar(kFull + st), L::kTileBytes);
#pragma unroll
                        for (int s = 0; s < NSUB; ++s)
                            tma_load_4d(sbase + L::kRing + st * L::kTileBytes + s * L::kSubBytes, kv ? &mapV : &mapK, bar(kFull + st), s * 64, hk, j * 128, 0);
                    }
                w.next(p);
            }
        }
    } else if (warp < 11) {
        // =========================== products of stream s ===========================
        const int s = warp - 9;
        constexpr uint32_t idesc_s = make_idesc_bf16(128, 128, false, false), idesc_o = make_idesc_bf16(128, D, false, true);
        const uint64_t dq0 = desc_kmajor_sw128(sbase + L::kQ + (paired ? s * L::kTileBytes : 0), 0);
        const uint64_t dk0 = desc_kmajor_sw128(sbase + L::kRing, 0), dv0 = desc_mnmajor_sw128(sbase + L::kRing, 0, L::kSubBytes);
        const uint32_t tS = tmem + s * 256, tO = tS + 128;
        int n = 0, base = 0, piece = 0;                               // tiles of this stream; ring index of the piece's first K tile
#pragma unroll 1
        for (; w.at < w.end; ++piece) {
            wait(bar(kQFull), piece & 1, 170);
            bool first = true;
#pragma unroll 1
            for (int j = w.j0; j < w.j1; ++j) {
                const int ik = base + 2 * (j - w.j0), iv = ik + 1;
                const int sk = ik % NST, sv = iv % NST;
                wait(bar(kFull + sk), (ik / NST) & 1, 171);
                if (!paired && ((j - w.j0) & 1) != s) {
                    // the other stream's tile: its barriers are waited for all the same, since a wait tells only one phase from the next
                    wait(bar(kFull + sv), (iv / NST) & 1, 175);
                    continue;
                }
                if (n > 0) wait(bar(kODone + s), (n - 1) & 1, 174);   // P, in the columns of the scores, has been read
                tc_fence_after_sync();
                const uint64_t dk = dk0 + uint64_t((sk * L::kTileBytes) >> 4);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint64_t o = uint64_t(((kk >> 2) * L::kSubBytes + (kk & 3) * 32) >> 4);
                    umma_ss(tS, dq0 + o, dk + o, idesc_s, kk > 0);
                }
                umma_commit(bar(kSFull + s));
                umma_commit(bar(kEmpty + sk));
                wait(bar(kFull + sv), (iv / NST) & 1, 172);
                wait(bar(kPFull + s), n & 1, 173);
                tc_fence_after_sync();
                const uint64_t dv = dv0 + uint64_t((sv * L::kTileBytes) >> 4);
                umma_ts(tO, tS, dv, idesc_o, !first);
#pragma unroll
                for (int kk = 1; kk < 8; ++kk) umma_ts(tO, tS + kk * 8, dv + uint64_t(kk * 128), idesc_o, 1);
                umma_commit(bar(kODone + s));
                umma_commit(bar(kEmpty + sv));
                first = false;
                ++n;
            }
            base += 2 * (w.j1 - w.j0);
            // O is read by the stream's warps before the next piece's first product writes it: they arrive on kPieceDone, which the
            // next Q tiles wait for
            w.next(p);
        }
        if (*abort_flag != 0) {
            // A wait gave up somewhere: make sure no MMA of this warp is still in flight before TMEM is released.
            umma_commit(bar(kODone + s));
            const uint64_t t0 = globaltimer_ns();
            while (globaltimer_ns() - t0 < 1000000ull) {}
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    abort_teardown(abort_flag, 256);
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 512);
}

// One CTA per (b, query head): the prefix partials, the sequence's own pieces and the token's depth pairs.
constexpr int kSharedMergeThreads = 128;

struct SharedMergeParams {
    DecodeParams dec;             // own caches and depth pairs (T_kv == 0: none of the former)
    SharedParams pre;             // prefix (P == 0: none)
};

template <int D>
__global__ void __launch_bounds__(kSharedMergeThreads)
shared_merge_kernel(const SharedMergeParams p) {
    constexpr int FPL = D / 32, NW = kSharedMergeThreads / 32;
    __shared__ float s_w[2 * 160], s_own[kDecodeMaxSplits], s_d[256], s_red[NW];
    __shared__ __align__(16) float s_acc[NW][D];
    const DecodeParams& q = p.dec;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = q.H / q.Hk, hk = h / G, g = h - hk * G;            // groups of at most 8 heads, as the split kernel has them
    const int Hk_real = q.Hk / q.kv_rep;

    auto load_row = [&](const __nv_bfloat16* row, float (&x)[FPL]) {
        if constexpr (FPL == 4) {
            const uint2 v = *reinterpret_cast<const uint2*>(row + lane * 4);
            x[0] = bf16_lo_to_f32(v.x); x[1] = bf16_hi_to_f32(v.x); x[2] = bf16_lo_to_f32(v.y); x[3] = bf16_hi_to_f32(v.y);
        } else {
            const uint32_t v = *reinterpret_cast<const uint32_t*>(row + lane * 2);
            x[0] = bf16_lo_to_f32(v); x[1] = bf16_hi_to_f32(v);
        }
    };
    // ---- depth scores ----
    float qv[FPL];
    load_row(q.q + (size_t(b) * q.H + h) * D, qv);
#pragma unroll
    for (int c = 0; c < FPL; ++c) qv[c] *= q.scale_log2;
    const size_t slot_stride = size_t(q.B) * Hk_real * 2 * D;
    const __nv_bfloat16* depth0 = q.depth + (size_t(b) * Hk_real + hk / q.kv_rep) * 2 * D;
    for (int i = warp; i < q.l; i += NW) {
        float kd[FPL], a = 0.f;
        load_row(depth0 + size_t(i) * slot_stride, kd);
#pragma unroll
        for (int c = 0; c < FPL; ++c) a = fmaf(qv[c], kd[c], a);
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) a += __shfl_xor_sync(0xffffffffu, a, off);
        if (lane == 0) s_d[i] = a;
    }
    const int own_len = q.T_kv == 0 ? 0 : q.seq_lens ? min(max(q.seq_lens[b], 0), q.T_kv) : q.T_kv;
    int n_pre = 0;
    if (p.pre.P > 0) {
        const int group = (h / p.pre.G) * p.pre.pairs + (p.pre.row_tiles > 1 ? b / (2 * p.pre.S) : 0);
        const int c0 = shared_first_run(group, p.pre.key_tiles, p.pre.run);
        const int c1 = int(((long long)(group + 1) * p.pre.key_tiles - 1) / p.pre.run);
        n_pre = (c1 - c0 + 1) * (p.pre.row_tiles > 1 ? 1 : 2);
    }
    __syncthreads();
    grid_dependency_wait();
    int n_own = 0;
    const float* group = q.part + (size_t(b) * q.Hk + hk) * kDecodeMaxSplits * G * (D + 2);
    const float* part = group + g * (D + 2);
    const size_t split_stride = size_t(G) * (D + 2);
    if (own_len > 0)
        n_own = q.seq_lens ? min(max(__float_as_int(__ldcg(group + (kDecodeMaxSplits - 1) * split_stride)), 1), q.max_pieces)
                           : decode_pieces_equal(q.cut, b * (q.Hk / q.team) + hk / q.team, q.T_kv, q.unit_log2);
    const size_t pre_stride = size_t(q.B) * q.H, pre_row = size_t(b) * q.H + h;
    // ---- maximum, weights, row sum ----
    float mx = -INFINITY;
    for (int i = tid; i < n_pre; i += kSharedMergeThreads) mx = fmaxf(mx, __ldcg(&p.pre.ml[i * pre_stride + pre_row].x));
    for (int i = tid; i < n_own; i += kSharedMergeThreads) mx = fmaxf(mx, __ldcg(part + i * split_stride));
    for (int i = tid; i < q.l; i += kSharedMergeThreads) mx = fmaxf(mx, s_d[i]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
    if (lane == 0) s_red[warp] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
    __syncthreads();
    float lt = 0.f;
    for (int i = tid; i < n_pre; i += kSharedMergeThreads) {
        const float2 v = __ldcg(&p.pre.ml[i * pre_stride + pre_row]);
        const float f = v.x == -INFINITY ? 0.f : fast_exp2(v.x - mx);
        s_w[i] = f;
        lt = fmaf(f, v.y, lt);
    }
    for (int i = tid; i < n_own; i += kSharedMergeThreads) {
        const float m = __ldcg(part + i * split_stride);
        const float f = m == -INFINITY ? 0.f : fast_exp2(m - mx);
        s_own[i] = f;
        lt = fmaf(f, __ldcg(part + i * split_stride + 1), lt);
    }
    for (int i = tid; i < q.l; i += kSharedMergeThreads) {
        const float f = fast_exp2(s_d[i] - mx);
        s_d[i] = f;
        lt += f;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) lt += __shfl_xor_sync(0xffffffffu, lt, off);
    if (lane == 0) s_red[warp] = lt;
    __syncthreads();
    lt = (s_red[0] + s_red[1]) + (s_red[2] + s_red[3]);
    // ---- weighted sums: a warp takes every fourth partial and every fourth depth value ----
    float acc[FPL];
#pragma unroll
    for (int c = 0; c < FPL; ++c) acc[c] = 0.f;
#pragma unroll 4
    for (int i = warp; i < n_pre; i += NW) {
        const float f = s_w[i];
        if (f == 0.f) continue;                                       // also a stream without keys, whose o is not written
        const float* src = p.pre.o + (i * pre_stride + pre_row) * D + lane * FPL;
#pragma unroll
        for (int c = 0; c < FPL; ++c) acc[c] = fmaf(f, __ldcg(src + c), acc[c]);
    }
#pragma unroll 4
    for (int i = warp; i < n_own; i += NW) {
        const float f = s_own[i];
        const float* src = part + i * split_stride + 2 + lane * FPL;
#pragma unroll
        for (int c = 0; c < FPL; ++c) acc[c] = fmaf(f, __ldcg(src + c), acc[c]);
    }
#pragma unroll 4
    for (int i = warp; i < q.l; i += NW) {
        const float f = s_d[i];
        float vd[FPL];
        load_row(depth0 + size_t(i) * slot_stride + D, vd);
#pragma unroll
        for (int c = 0; c < FPL; ++c) acc[c] = fmaf(f, vd[c], acc[c]);
    }
#pragma unroll
    for (int c = 0; c < FPL; ++c) s_acc[warp][lane * FPL + c] = acc[c];
    __syncthreads();
    // a row without any key: O = 0, LSE = -inf
    if (tid < D) {
        const float a = (s_acc[0][tid] + s_acc[1][tid]) + (s_acc[2][tid] + s_acc[3][tid]);
        q.O[(size_t(b) * q.H + h) * D + tid] = __float2bfloat16(lt > 0.f || lt != lt ? a / lt : 0.f);
    }
    if (tid == 0) q.LSE[size_t(b) * q.H + h] = (mx + log2f(lt)) * kDecodeLn2;
}

}  // namespace moda
