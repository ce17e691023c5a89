// Attention weight of the sequence keys: how much probability the rows of a call, and the query heads of a group, gave to each key of
// the cache (Sec. 2.2: the probabilities of the one softmax over sequence and depth keys, hence the LSE of the call that is meant).
//
//     mass[b, hk, j] = old[b, hk, j] + sum_{h in group hk} sum_{i : i + T_kv - T_q >= j} exp( scale <q_i, k_j> - LSE[b, h, i] )
//
// decode_key_mass_kernel   T_q = 1, behind the decode step's merge: the split kernel has left its scores, which are G floats a key beside
//                          the 4 d bytes of the key's K and V rows; reading K a second time would be 2 d bytes.
//
// key_mass_kernel          T_q rows: one product S^T = K Q^T per (key tile, unit), the keys as the 128 rows of the tcgen05 tile, so that
//                          a thread holds a key and the sum over the query rows stays in one register.  A unit is up to 128 query
//                          rows: P = 128 / G positions with the G heads of the group (row = position in the unit * G + head), as one TMA box
//                          of the [T][H][d] tensor leaves them.
//
//   Every CTA takes an equal run of the units of all (b, hk, key tile) in this order (within a key tile only the units that see it), so
//   all SMs end together whatever the causal triangle looks like; the part of a key tile that a run covers is a piece.  A piece that is its whole key
//   tile is stored at once; the others leave partial sums, at most two a CTA, that key_mass_join_kernel adds in order of the units
//   (no atomics: the result is reproducible bit for bit).
//
//   20 warps: 0-15 four warpgroups on the units in turn (weights of a 128 x 128 tile: thread = key), 16 TMA producer, 17 issues the
//   products and owns TMEM, 18 loads the LSE of a unit's rows.  Unit n uses stage n % 4 of the Q ring, of the LSE ring and of the four
//   score buffers in tensor memory.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda.h>
#include <cuda_runtime.h>

#include "moda_bwd.cuh"          // kLog2e
#include "sm100_ptx.cuh"

namespace moda {

// ---------------------------------------------------------------------------------------------------------- decode step
struct DecodeKeyMassParams {
    const float* scores;          // [B][Hk][kv_rep * G][stride], times log2(e)
    const float* LSE;             // [B][H]
    const float* mass_in;         // [B][Hk][T_cap], or null
    float* mass;                  // [B][Hk][T_cap]
    const int* seq_lens;          // [B] or null
    size_t stride;
    int T_kv, T_cap, H, Hk;
};

constexpr int kDecodeMassThreads = 256;

// grid (blocks of 4 x 256 keys, Hk, B)
__global__ void __launch_bounds__(kDecodeMassThreads)
decode_key_mass_kernel(const DecodeKeyMassParams p) {
    __shared__ float s_lse[32];
    const int hk = blockIdx.y, b = blockIdx.z, G = p.H / p.Hk;
    const int len = p.seq_lens ? min(max(p.seq_lens[b], 1), p.T_kv) : p.T_kv;
    const int t0 = (int(blockIdx.x) * kDecodeMassThreads + int(threadIdx.x)) * 4;
    const size_t row = (size_t(b) * p.Hk + hk) * p.T_cap;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    if (p.mass_in != nullptr) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t0 + i < len - 1) acc[i] = p.mass_in[row + t0 + i];
    }
    grid_dependency_wait();
    if (int(threadIdx.x) < G) s_lse[threadIdx.x] = __ldcg(p.LSE + size_t(b) * p.H + hk * G + threadIdx.x) * kLog2e;
    __syncthreads();
    if (t0 >= len) return;
    const float* src = p.scores + (size_t(b) * p.Hk + hk) * G * p.stride + t0;
#pragma unroll 8
    for (int g = 0; g < G; ++g) {
        const float4 s = __ldcg(reinterpret_cast<const float4*>(src + g * p.stride));
        const float lse = s_lse[g];
        acc[0] += fast_exp2(s.x - lse);
        acc[1] += fast_exp2(s.y - lse);
        acc[2] += fast_exp2(s.z - lse);
        acc[3] += fast_exp2(s.w - lse);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (t0 + i < len) p.mass[row + t0 + i] = acc[i];
}

// ------------------------------------------------------------------------------------------------------------ T_q rows
constexpr int kKmThreads = 640;
constexpr int kKmStages = 4;

struct KeyMassParams {
    const float* LSE;             // [B][H][T_q]
    const float* mass_in;         // [B][Hk][T_cap], or null
    float* mass;                  // [B][Hk][T_cap]
    float* part;                  // [CTA][2][128] partial sums, then [CTA][2] int2 {key tile of all, kPieceStart | kPieceEnd}
    int T_q, T_kv, T_cap, H, Hk, G;
    int P, n_units;               // positions of a unit; units that cover T_q
    int tiles;                    // key tiles of a (b, hk)
    long long per_head, total;    // units of a (b, hk), of all
    int run;                      // units of a CTA
    float scale_log2;
};
enum : int { kPieceStart = 1, kPieceEnd = 2, kPieceNone = 4 };

template <int D>
struct KeyMassSmem {
    static constexpr int kTileBytes = 128 * D * 2;
    static constexpr int kSubBytes = 128 * 128;
    static constexpr int kK = 0;                                   // 2 stages
    static constexpr int kQ = kK + 2 * kTileBytes;                 // kKmStages
    static constexpr int kLse = kQ + kKmStages * kTileBytes;       // [stage][128]
    static constexpr int kAcc = kLse + kKmStages * 512;            // [2][4][128]
    static constexpr int kBars = kAcc + 2 * 4 * 512;
    static constexpr int kNumBars = 24;
    static constexpr int kMisc = kBars + kNumBars * 8;             // tmem base, abort word, start of the run
    static constexpr int kTotal = kMisc + 32;
    static constexpr int kDynamic = kTotal + 1024;
    static_assert(kDynamic <= 232448, "shared memory");
};

enum KeyMassBar : int {
    kKmKFull = 0,      // +(piece & 1)
    kKmKEmpty = 2,     // +(piece & 1): every product of the piece is complete
    kKmQFull = 4,      // +stage
    kKmLFull = 8,      // +stage
    kKmSFull = 12,     // +stage: the scores are there, the Q stage is free
    kKmSEmpty = 16,    // +stage: the scores and the LSE have been read
    kKmDone = 20,      // +(piece & 1): the four warpgroups' sums of a piece are in shared memory
    kKmDrain = 22,
};

// A wait of the kernels for serving: mbar_wait, as a call that takes the CTA's abort word along.
struct PipeWait {
    volatile int* abort_flag;
    __device__ __forceinline__ void operator()(uint32_t bar, uint32_t parity, int site) const { mbar_wait(bar, parity, abort_flag, site); }
};

// First unit that sees key tile `jt`: the one of the first position i with i + off >= 128 jt.
__device__ __forceinline__ int key_mass_first_unit(int jt, int off, int P) {
    const int i = jt * 128 - off;
    return i > 0 ? i / P : 0;
}

// The units of a CTA's run, piece by piece.
struct KeyMassWalk {
    int bh, jt, u;                // of the next unit
    int left;                     // units of the run that are left
    __device__ __forceinline__ bool last_of_tile(const KeyMassParams& p) const { return u + 1 == p.n_units; }
    __device__ __forceinline__ bool last_of_piece(const KeyMassParams& p) const { return left == 1 || u + 1 == p.n_units; }
    __device__ __forceinline__ void next(const KeyMassParams& p) {
        --left;
        if (++u == p.n_units) {
            if (++jt == p.tiles) { jt = 0; ++bh; }
            u = key_mass_first_unit(jt, p.T_kv - p.T_q, p.P);
        }
    }
};

template <int D>
__global__ void __launch_bounds__(kKmThreads, 1)
key_mass_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const KeyMassParams p) {
    using L = KeyMassSmem<D>;
    constexpr int NSUB = D / 64;
    if (g_moda_status != 0) return;   // an earlier kernel gave up a wait: do not pile up more timeouts
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t sbase = smem_u32(smem);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + L::kMisc + 4);
    int* s_start = reinterpret_cast<int*>(smem + L::kMisc + 8);
    auto bar = [&](int i) { return sbase + L::kBars + 8u * uint32_t(i); };
    const PipeWait wait{abort_flag};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int off = p.T_kv - p.T_q;
    const int rows = p.P * p.G;                       // query rows of a unit, at most 128

    if (tid < 2) reinterpret_cast<int2*>(p.part + size_t(gridDim.x) * 256)[blockIdx.x * 2 + tid] = make_int2(0, kPieceNone);
    if (tid == 0) {
        *abort_flag = 0;
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(kKmKFull + s), 1);
            mbar_init(bar(kKmKEmpty + s), 1);
            mbar_init(bar(kKmDone + s), 512);
        }
        for (int s = 0; s < kKmStages; ++s) {
            mbar_init(bar(kKmQFull + s), 1);
            mbar_init(bar(kKmLFull + s), 32);
            mbar_init(bar(kKmSFull + s), 1);
            mbar_init(bar(kKmSEmpty + s), 128);
        }
        mbar_init(bar(kKmDrain), 1);
        fence_mbar_init();
    }
    if (warp == 17) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    if (warp == 16) {
        // where the run starts: (b, hk), then its key tile by the lanes' sums over equal shares of the tiles
        const long long at = (long long)blockIdx.x * p.run;
        const int bh = int(at / p.per_head);
        const int in_head = int(at - bh * p.per_head);
        const int per_lane = (p.tiles + 31) / 32;
        const int j0 = min(lane * per_lane, p.tiles), j1 = min(j0 + per_lane, p.tiles);
        int sum = 0;
        for (int j = j0; j < j1; ++j) sum += p.n_units - key_mass_first_unit(j, off, p.P);
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (in_head >= incl - sum && in_head < incl) {
            int before = incl - sum, j = j0;
            for (;; ++j) {
                const int n = p.n_units - key_mass_first_unit(j, off, p.P);
                if (in_head < before + n) break;
                before += n;
            }
            s_start[0] = bh;
            s_start[1] = j;
            s_start[2] = key_mass_first_unit(j, off, p.P) + in_head - before;
        }
    }
    // rows of the Q stages that no box covers stay zero (their LSE is +inf: weight 0)
    if (rows < 128) {
        for (int e = tid; e < kKmStages * NSUB * (128 - rows) * 8; e += kKmThreads) {
            const int piece = e & 7, r = rows + (e >> 3) % (128 - rows), sub = (e >> 3) / (128 - rows);
            *reinterpret_cast<uint4*>(smem + L::kQ + sub * L::kSubBytes + r * 128 + piece * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
        fence_proxy_async_smem();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    const long long begin = (long long)blockIdx.x * p.run;
    KeyMassWalk w;
    w.bh = s_start[0];
    w.jt = s_start[1];
    w.u = s_start[2];
    w.left = int(min((long long)p.run, p.total - begin));

    if (warp < 16) {
        // =========================== weights and their sums: thread = key ===========================
        const int wg = warp >> 2, r = tid & 127;
        const uint32_t tS = tmem + (uint32_t((warp & 3) * 32) << 16) + wg * 128;
        float* s_acc = reinterpret_cast<float*>(smem + L::kAcc);
        const float4* s_lse = reinterpret_cast<const float4*>(smem + L::kLse + wg * 512);
        float acc = 0.f;
        int n = 0, piece = 0;
        bool starts = w.u == key_mass_first_unit(w.jt, off, p.P);        // the piece starts its key tile
#pragma unroll 1
        for (; w.left > 0; ++n) {
            if ((n & 3) == wg) {
                const int par = (n >> 2) & 1;
                wait(bar(kKmLFull + wg), par, 110);
                wait(bar(kKmSFull + wg), par, 111);
                tc_fence_after_sync();
                const int key = w.jt * 128 + r, i0 = w.u * p.P;
                // row c of the unit sees this key iff c / G + i0 + off >= key
                const int hidden = i0 + off >= w.jt * 128 + 127 ? 0 : (key - off - i0) * p.G;
                float a0 = 0.f, a1 = 0.f, a2 = 0.f, a3 = 0.f;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t s[32];
                    tmem_ld32(tS + c * 32, s);
                    tmem_wait_ld();
                    if (hidden > c * 32) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c * 32 + i < hidden) s[i] = 0xff800000u;
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 nl = s_lse[c * 8 + i / 4];
                        float x0 = nl.x, x1 = nl.y, x2 = nl.z, x3 = nl.w;
                        fma2_f32(__uint_as_float(s[i]), __uint_as_float(s[i + 1]), p.scale_log2, p.scale_log2, x0, x1);
                        fma2_f32(__uint_as_float(s[i + 2]), __uint_as_float(s[i + 3]), p.scale_log2, p.scale_log2, x2, x3);
                        add2_f32(fast_exp2(x0), fast_exp2(x1), a0, a1);
                        add2_f32(fast_exp2(x2), fast_exp2(x3), a2, a3);
                    }
                }
                acc += (a0 + a1) + (a2 + a3);
                tc_fence_before_sync();
                mbar_arrive(bar(kKmSEmpty + wg));
            }
            if (w.last_of_piece(p)) {
                // the four warpgroups' sums meet in shared memory; the piece's owner adds them while the others go on.  (Behind piece - 1's
                // barrier the owner of piece - 2 has read this buffer: it arrived there after that.)
                if (piece >= 2) wait(bar(kKmDone + ((piece - 1) & 1)), ((piece - 1) >> 1) & 1, 112);
                float* buf = s_acc + (piece & 1) * 512;
                buf[wg * 128 + r] = acc;
                mbar_arrive(bar(kKmDone + (piece & 1)));
                const bool ends = w.last_of_tile(p);
                if ((piece & 3) == wg) {
                    wait(bar(kKmDone + (piece & 1)), (piece >> 1) & 1, 113);
                    const float sum = (buf[r] + buf[128 + r]) + (buf[256 + r] + buf[384 + r]);
                    const int key = w.jt * 128 + r;
                    if (starts && ends) {
                        if (key < p.T_kv) {
                            const size_t at = size_t(w.bh) * p.T_cap + key;
                            p.mass[at] = sum + (p.mass_in != nullptr && key < off ? p.mass_in[at] : 0.f);
                        }
                    } else {
                        const int slot = int(blockIdx.x) * 2 + (piece > 0);
                        p.part[size_t(slot) * 128 + r] = sum;
                        if (r == 0)
                            reinterpret_cast<int2*>(p.part + size_t(gridDim.x) * 256)[slot] =
                                make_int2(w.bh * p.tiles + w.jt, (starts ? kPieceStart : 0) | (ends ? kPieceEnd : 0));
                    }
                }
                ++piece;
                acc = 0.f;
                starts = true;
            }
            w.next(p);
        }
    } else if (warp == 16) {
        // =========================== TMA producer ===========================
        if (lane == 0) {
            tma_prefetch_desc(&mapQ);
            tma_prefetch_desc(&mapK);
            const uint32_t unit_bytes = uint32_t(rows) * D * 2;
            int n = 0, piece = 0;
            bool fresh = true;
#pragma unroll 1
            for (; w.left > 0; ++n) {
                const int b = w.bh / p.Hk, hk = w.bh - b * p.Hk;
                if (fresh) {
                    const int st = piece & 1;
                    if (piece >= 2) wait(bar(kKmKEmpty + st), ((piece - 2) >> 1) & 1, 120);
                    mbar_arrive_expect_tx(bar(kKmKFull + st), L::kTileBytes);
#pragma unroll
                    for (int s = 0; s < NSUB; ++s)
                        tma_load_4d(sbase + L::kK + st * L::kTileBytes + s * L::kSubBytes, &mapK, bar(kKmKFull + st), s * 64, hk, w.jt * 128, b);
                    ++piece;
                }
                const int st = n & 3;
                if (n >= 4) wait(bar(kKmSFull + st), ((n - 4) >> 2) & 1, 121);
                mbar_arrive_expect_tx(bar(kKmQFull + st), unit_bytes);
#pragma unroll
                for (int s = 0; s < NSUB; ++s)
                    tma_load_4d(sbase + L::kQ + st * L::kTileBytes + s * L::kSubBytes, &mapQ, bar(kKmQFull + st), s * 64, hk * p.G, w.u * p.P, b);
                fresh = w.last_of_tile(p);
                w.next(p);
            }
        }
    } else if (warp == 17) {
        // =========================== MMA issuer: S^T = K Q^T ===========================
        constexpr uint32_t idesc = make_idesc_bf16(128, 128, false, false);
        const uint64_t dk0 = desc_kmajor_sw128(sbase + L::kK, 0), dq0 = desc_kmajor_sw128(sbase + L::kQ, 0);
        int n = 0, piece = 0;
        bool fresh = true;
#pragma unroll 1
        for (; w.left > 0; ++n) {
            const int st = n & 3, kst = piece & 1;
            if (fresh) wait(bar(kKmKFull + kst), (piece >> 1) & 1, 130);
            wait(bar(kKmQFull + st), (n >> 2) & 1, 131);
            if (n >= 4) wait(bar(kKmSEmpty + st), ((n - 4) >> 2) & 1, 132);
            tc_fence_after_sync();
            const uint64_t dk = dk0 + uint64_t((kst * L::kTileBytes) >> 4), dq = dq0 + uint64_t((st * L::kTileBytes) >> 4);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint64_t o = uint64_t(((kk >> 2) * L::kSubBytes + (kk & 3) * 32) >> 4);
                umma_ss(tmem + st * 128, dk + o, dq + o, idesc, kk > 0);
            }
            umma_commit(bar(kKmSFull + st));
            fresh = w.last_of_tile(p);
            if (w.last_of_piece(p)) {
                umma_commit(bar(kKmKEmpty + kst));
                ++piece;
            }
            w.next(p);
        }
        if (*abort_flag != 0) {
            // A wait gave up somewhere: make sure no MMA of this thread is still in flight before TMEM is released.
            umma_commit(bar(kKmDrain));
            const uint64_t t0 = globaltimer_ns();
            while (!mbar_try_wait(bar(kKmDrain), 0) && globaltimer_ns() - t0 < 20000000ull) {}
        }
    } else if (warp == 18) {
        // =========================== LSE of a unit's rows: -LSE log2(e), -inf where there is no row ===========================
        float* s_lse = reinterpret_cast<float*>(smem + L::kLse);
        int pos[4];
        size_t at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = lane * 4 + i;
            pos[i] = c < rows ? c / p.G : p.T_q;                     // T_q: no position of any unit
            at[i] = size_t(c % p.G) * p.T_q + (c < rows ? c / p.G : 0);
        }
        auto fetch = [&](const KeyMassWalk& k, float (&v)[4]) {
            const int b = k.bh / p.Hk, hk = k.bh - b * p.Hk, i0 = k.u * p.P;
            const float* src = p.LSE + (size_t(b) * p.H + hk * p.G) * p.T_q + i0;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pos[i] < p.T_q - i0 ? src[at[i]] : INFINITY;
        };
        float v[4];
        fetch(w, v);
#pragma unroll 1
        for (int n = 0; w.left > 0; ++n) {
            const int st = n & 3;
            KeyMassWalk after = w;
            after.next(p);
            float ahead[4] = {0.f, 0.f, 0.f, 0.f};
            if (after.left > 0) fetch(after, ahead);
            if (n >= 4) wait(bar(kKmSEmpty + st), ((n - 4) >> 2) & 1, 140);
            // a row without keys has the LSE -inf; its weights are 0
            float4 o;
            o.x = v[0] == -INFINITY ? -INFINITY : -v[0] * kLog2e;
            o.y = v[1] == -INFINITY ? -INFINITY : -v[1] * kLog2e;
            o.z = v[2] == -INFINITY ? -INFINITY : -v[2] * kLog2e;
            o.w = v[3] == -INFINITY ? -INFINITY : -v[3] * kLog2e;
            *reinterpret_cast<float4*>(s_lse + st * 128 + lane * 4) = o;
            mbar_arrive(bar(kKmLFull + st));
            w = after;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = ahead[i];
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    abort_teardown(abort_flag, 512);
    __syncthreads();
    if (warp == 17) tmem_dealloc(tmem, 512);
}

// Adds the pieces of the key tiles that several runs share: CTA c takes the tile that starts in run c and does not end there.
__global__ void __launch_bounds__(128)
key_mass_join_kernel(const KeyMassParams p) {
    const int ctas = gridDim.x, c = blockIdx.x, r = threadIdx.x;
    const int2* dir = reinterpret_cast<const int2*>(p.part + size_t(ctas) * 256);
    grid_dependency_wait();
    // the piece at the end of run c: its second entry, or its first where the run is one piece
    int slot = 2 * c + 1;
    int2 d = dir[slot];
    if (d.y == kPieceNone) d = dir[--slot];
    if (d.y != kPieceStart) return;                   // ends in its run (or nothing is shared), or does not start in it
    float sum = p.part[size_t(slot) * 128 + r];
    for (int k = c + 1; k < ctas; ++k) {
        sum += p.part[size_t(2 * k) * 128 + r];
        if (dir[2 * k].y & kPieceEnd) break;
    }
    const int bh = d.x / p.tiles, key = (d.x - bh * p.tiles) * 128 + r;
    if (key < p.T_kv) {
        const size_t at = size_t(bh) * p.T_cap + key;
        p.mass[at] = sum + (p.mass_in != nullptr && key < p.T_kv - p.T_q ? p.mass_in[at] : 0.f);
    }
}

}  // namespace moda
