// Attention weight of the sequence keys: how much probability the rows of a call, and the query heads of a group, gave to each key of
// the cache (Sec. 2.2: the probabilities of the one softmax over sequence and depth keys, hence the LSE of the call that is meant).
//
//     mass[b, hk, j] = old[b, hk, j] + sum_{h in group hk} sum_{i : i + T_kv - T_q >= j} exp( scale <q_i, k_j> - LSE[b, h, i] )
//
// decode_key_mass_kernel   T_q = 1, behind the decode step's merge: the split kernel has left its scores, which are G floats a key beside
//                          the 4 d bytes of the key's K and V rows; reading K a second time would be 2 d bytes.
//
// key_mass_kernel          T_q rows: products S^T = K Q^T of a tile, two adjacent 128-key tiles, and a unit, up to 128 query rows.  The keys are the rows of the
//                          tcgen05 products, so that a thread holds a key and the sum over the query rows stays in a register.  A
//                          unit is P = 128 / G positions with the G heads of the group (row = position in the unit * G + head), as one TMA box of the
//                          [T][H][d] tensor leaves them.  One more step of 16 contraction elements subtracts LSE / scale (three bf16 terms a row,
//                          whose sum is the fp32 value, against ones), so the weight is exp2(scale log2(e) S) as it comes.
//
//   Every CTA takes an equal run of the units of all (b, hk, tile) in this order (within a tile only the units that see it), so all SMs end
//   together whatever the causal triangle looks like; the part of a tile that a run covers is a piece.  With few units a tile, where the
//   bytes of K set the pace, the runs are those of teams of CTAs that take adjacent heads, whose rows are adjacent in memory, at the same time.  A piece that is its whole tile
//   is stored at once; the others leave partial sums, at most two a CTA, that key_mass_join_kernel adds in order of the units (no
//   atomics: the result is reproducible bit for bit).
//
//   20 warps: 0-15 four warpgroups (even units: tiles' first and second 128 keys, odd units: likewise), 16 TMA producer, 17 and 19 issue the
//   products of the two halves (17 owns TMEM), 18 prepares the LSE terms and clears the queries of rows that saw no key (LSE -inf;
//   a test of every unit by the weights' warps instead: 67.9 -> 69.7 us in the second case below, this way 68.1).  With few units a tile the warpgroups and issuers take even and
//   odd tiles instead: their sums need not meet (64 rows over 8192 keys, B = 4, 32 heads on 8, two units: d = 128 32.7 -> 30.4 us, d = 64 29.7 -> 27.5; 300 rows over
//   6000, B = 2, 16 heads, d = 64, three: 29.6 -> 27.7).
//
//   What bounds it: the exponentials, one per visible (row, key), of which a quarter goes to the FMA pipe: 768 cycles of the SFU a 128 x 128 tile
//   against 576 of the tensor cores at d = 128, 320 at 64.  us, SFU time of its three quarters / the kernel: 64 rows over 8192 as above 11 / 31 (8.5 of it the
//   launch, its start and end); 1000 rows over 5003, B = 3, 16 heads, d = 64 38 / 68; 32768 rows and keys, 16 heads on 8, d = 128 1430 / 2140, and 1750 / 2500
//   under a lasting load, when the power limit of 1000 W holds the SMs at 1.57 GHz.  The kernels stand at 1.4 to 1.8 of that bound (the first case, with its
//   start and end, at 2.8): scores come from tensor memory 16 columns a wait, and the form for many units a tile spills 28 bytes (48 loaded).
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
constexpr int kKmTile = 256;          // keys of a tile
struct KeyMassParams {
    const float* LSE;             // [B][H][T_q]
    const float* mass_in;         // [B][Hk][T_cap], or null
    float* mass;                  // [B][Hk][T_cap]
    float* part;                  // [CTA][2][kKmTile] partial sums, then [CTA][2] int2 {tile of all, kPieceStart | kPieceEnd}
    int T_q, T_kv, T_cap, Hk, G;
    int P, n_units;               // positions of a unit; units that cover T_q
    int tiles;                    // tiles of a (b, hk)
    int team;                     // CTAs of a team (divides Hk): CTA c takes the heads c % team of the groups of `team` heads
    long long per_head, total;    // units of a (b, hk), of all groups of heads
    int run;                      // units of a team
    int k_slots, q_slots;         // of shared memory: halves of tiles, units
    int stay;                     // every tile sees every unit, and a unit comes round to its slot again with every tile: it stays there
    float scale_log2, inv_scale, least;   // least: -127 / scale_log2
};
enum : int { kPieceStart = 1, kPieceEnd = 2, kPieceNone = 4 };

// Slots of 128 rows: the ring of tile halves takes the first k_slots, the ring of units the next q_slots.
template <int D>
struct KeyMassSmem {
    static constexpr int kSlotBytes = 128 * D * 2;
    static constexpr int kSubBytes = 128 * 128;
    static constexpr int kSlots = D == 128 ? 6 : 10;
    static constexpr int kMaxUnits = 6;
    static constexpr int kTermBytes = 128 * 16;                    // 8 contraction elements of 128 rows
    static constexpr int kOnes = kSlots * kSlotBytes;              // the keys' side of the LSE step
    static constexpr int kTerms = kOnes + kTermBytes;              // [unit slot]
    static constexpr int kZero = kTerms + kMaxUnits * kTermBytes;  // the second 8 elements, of both sides
    static constexpr int kAcc = kZero + kTermBytes;                // [2][4][128]
    static constexpr int kBars = kAcc + 2 * 4 * 512;
    static constexpr int kNumBars = 48;
    static constexpr int kMisc = kBars + kNumBars * 8;             // tmem base, abort word, start of the run
    static constexpr int kTotal = kMisc + 32;
    static constexpr int kDynamic = kTotal + 1024;
    static_assert(kDynamic <= 232448, "shared memory");
};
// Few units a tile (the last rows of a prompt): they stay in their slots, and the tiles stream.  Many: two units on their way while one is used.
inline void key_mass_slots(int d, int n_units, int& k_slots, int& q_slots) {
    if (d == 64) { k_slots = 4; q_slots = 6; return; }
    k_slots = n_units <= 2 ? 4 : 3;
    q_slots = 6 - k_slots;
}

enum KeyMassBar : int {
    kKmKFull = 0,      // +slot of a tile's half (<= 4)
    kKmKEmpty = 4,     // +slot: every product with it is complete
    kKmQFull = 8,      // +slot of a unit (<= 6): its LSE terms, and rows that saw no key are zero
    kKmQEmpty = 14,    // +slot: the products of both halves with it are complete
    kKmQHere = 20,     // +slot: its rows are there
    kKmSFull = 26,     // +(n % 2) * 2 + half: the scores are there
    kKmSEmpty = 30,    // +(n % 2) * 2 + half: the scores have been read
    kKmDone = 34,      // +(piece % 2): the warpgroups' sums of a piece are in shared memory
    kKmDrain = 36,     // +half
};

// A place in a ring of `slots` slots and how often the ring has gone round.
struct RingAt {
    int slot = 0, round = 0;
    __device__ __forceinline__ void next(int slots) {
        if (++slot == slots) { slot = 0; ++round; }
    }
};

// A wait of the kernels for serving: mbar_wait, as a call that takes the CTA's abort word along.
struct PipeWait {
    volatile int* abort_flag;
    __device__ __forceinline__ void operator()(uint32_t bar, uint32_t parity, int site) const { mbar_wait(bar, parity, abort_flag, site); }
    __device__ __forceinline__ void both(uint32_t bar_a, uint32_t parity_a, uint32_t bar_b, uint32_t parity_b, int site_a, int site_b) const {
        mbar_wait2(bar_a, parity_a, bar_b, parity_b, abort_flag, site_a, site_b);
    }
};

// First unit that sees tile `jt`: the one of the first position i with i + off >= 256 jt.
__host__ __device__ __forceinline__ int key_mass_first_unit(int jt, int off, int P) {
    const int i = jt * kKmTile - off;
    return i > 0 ? i / P : 0;
}

// Columns of a unit's scores: its rows, at T_q's end fewer than of the others, in steps of 32.
__device__ __forceinline__ int key_mass_filled(const KeyMassParams& p, int u) { return (min(p.P, p.T_q - u * p.P) * p.G + 31) & ~31; }

// The pieces of a CTA's run.
struct KeyMassWalk {
    int bh, jt, u0, u1;           // (b, kv head), tile, units of the piece
    int left;                     // units of the run from u0 on
    bool starts;                  // the piece starts its tile
    __device__ __forceinline__ void begin(const KeyMassParams& p, const int* start) {
        bh = start[0] * p.team + int(blockIdx.x) % p.team;
        jt = start[1];
        u0 = start[2];
        left = int(min((long long)p.run, p.total - (long long)(int(blockIdx.x) / p.team) * p.run));
        u1 = min(p.n_units, u0 + left);
        starts = u0 == key_mass_first_unit(jt, p.T_kv - p.T_q, p.P);
    }
    __device__ __forceinline__ bool ends(const KeyMassParams& p) const { return u1 == p.n_units; }
    __device__ __forceinline__ void next(const KeyMassParams& p) {
        left -= u1 - u0;
        if (++jt == p.tiles) {
            jt = 0;
            bh += p.team;
        }
        u0 = key_mass_first_unit(jt, p.T_kv - p.T_q, p.P);
        u1 = min(p.n_units, u0 + left);
        starts = true;
    }
};

// FEW: few units a tile.  The warpgroups take tiles in turn, and of a unit only the rows that there are.
template <int D, bool FEW>
__global__ void __launch_bounds__(kKmThreads, 1)
key_mass_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const KeyMassParams p) {
    using L = KeyMassSmem<D>;
    constexpr int NSUB = D / 64;
    // first of all, whatever happens then: the join takes places in `mass` from here, and the workspace holds anything
    int2* dir = reinterpret_cast<int2*>(p.part + size_t(gridDim.x) * 2 * kKmTile) + blockIdx.x * 2;
    if (threadIdx.x < 2) dir[threadIdx.x] = make_int2(0, kPieceNone);
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

    if (tid == 0) {
        *abort_flag = 0;
        for (int s = 0; s < 4; ++s) {
            mbar_init(bar(kKmKFull + s), 1);
            mbar_init(bar(kKmKEmpty + s), 1);
            mbar_init(bar(kKmSFull + s), 1);
            mbar_init(bar(kKmSEmpty + s), 128);
        }
        for (int s = 0; s < L::kMaxUnits; ++s) {
            mbar_init(bar(kKmQFull + s), 1);
            mbar_init(bar(kKmQHere + s), 1);
            mbar_init(bar(kKmQEmpty + s), 2);
        }
        for (int s = 0; s < 2; ++s) mbar_init(bar(kKmDone + s), 512);
        for (int s = 0; s < 2; ++s) mbar_init(bar(kKmDrain + s), 1);
        fence_mbar_init();
    }
    if (warp == 17) {
        tmem_alloc(smem_u32(tmem_slot), 512);
        tmem_relinquish();
    }
    if (warp == 16) {
        // where the run starts: (b, group of heads), then its tile by the lanes' sums over equal shares of the tiles
        const long long at = (long long)(int(blockIdx.x) / p.team) * p.run;
        const int group = int(at / p.per_head);
        const int in_head = int(at - group * p.per_head);
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
            s_start[0] = group;
            s_start[1] = j;
            s_start[2] = key_mass_first_unit(j, off, p.P) + in_head - before;
        }
    }
    // rows of the unit slots that no box covers stay zero (their LSE terms make their weights 0)
    if (rows < 128) {
        for (int e = tid; e < p.q_slots * NSUB * (128 - rows) * 8; e += kKmThreads) {
            const int piece = e & 7, r = rows + (e >> 3) % (128 - rows), sub = (e >> 3) / (128 - rows);
            *reinterpret_cast<uint4*>(smem + p.k_slots * L::kSlotBytes + sub * L::kSubBytes + r * 128 + piece * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
    }
    // the keys' side of the LSE step: 1, 1, 1, 0 ...
    if (tid < 128) {
        *reinterpret_cast<uint4*>(smem + L::kOnes + tid * 16) = make_uint4(0x3f803f80u, 0x00003f80u, 0u, 0u);
        *reinterpret_cast<uint4*>(smem + L::kZero + tid * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    fence_proxy_async_smem();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    KeyMassWalk w;
    w.begin(p, s_start);

    if (warp < 16) {
        // =========================== weights and their sums: thread = key ===========================
        setmaxnreg_inc<104>();
        const int wg = warp >> 2, r = tid & 127;
        const int half = wg & 1, st = wg >> 1;                           // half of the tile; the units n % 2 == st are this warpgroup's
        const uint32_t tS = tmem + (uint32_t((warp & 3) * 32) << 16) + st * 256 + half * 128;
        float* s_acc = reinterpret_cast<float*>(smem + L::kAcc);
        const int step = FEW ? 1 : 2;
        int n0 = 0, q0 = 0;                                              // units before the piece, slot of its first one
        int cnt = 0;                                                     // units of this warpgroup so far
#pragma unroll 1
        for (int piece = 0; w.left > 0; ++piece) {
            uint64_t y0 = 0, y1 = 0;
            const int key0 = w.jt * kKmTile + half * 128;
            const bool mine = !FEW || (piece & 1) == st;
            const int skip = FEW ? 0 : (n0 ^ st) & 1;
            int q_slot = q0 + skip;
#pragma unroll 1
            for (int u = mine ? w.u0 + skip : w.u1; u < w.u1; u += step, ++cnt) {
                wait(bar(kKmSFull + wg), cnt & 1, 111);
                tc_fence_after_sync();
                if (q_slot >= p.q_slots) q_slot -= p.q_slots;
                if (r == 0) mbar_arrive(bar(kKmQEmpty + q_slot));
                q_slot += step;
                // row c of the unit sees key r iff c / G + i0 + off >= key0 + r
                const int i0 = u * p.P;
                const bool masked = i0 + off < key0 + 127;
                const int hidden = (key0 + r - off - i0) * p.G;
                if (key0 < p.T_kv) {
                    auto add_chunk = [&](uint32_t (&s)[16], int c) {
                        if (masked) {
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (c * 16 + i < hidden) s[i] = 0xff800000u;
                        }
                        add_exp2_16<2>(s, p.scale_log2, p.least, y0, y1);
                    };
                    auto read = [&]() {                                  // the scores are in registers
                        tc_fence_before_sync();
                        mbar_arrive(bar(kKmSEmpty + wg));
                    };
                    uint32_t sa[16], sb[16];
                    const int filled = FEW ? key_mass_filled(p, u) : 128;  // the columns behind have not been computed
                    tmem_ld16(tS, sa);
#pragma unroll
                    for (int c = 0; c < 8; c += 2) {
                        if (FEW && c * 16 >= filled) break;
                        tmem_wait_ld();
                        tmem_ld16(tS + c * 16 + 16, sb);
                        add_chunk(sa, c);
                        tmem_wait_ld();
                        if (c < 6 && (!FEW || (c + 2) * 16 < filled)) tmem_ld16(tS + c * 16 + 32, sa);
                        else read();
                        add_chunk(sb, c + 1);
                    }
                } else {
                    mbar_arrive(bar(kKmSEmpty + wg));
                }
            }
            n0 += w.u1 - w.u0;
            q0 = (q0 + w.u1 - w.u0) % p.q_slots;
            float sum = (__uint_as_float(uint32_t(y0)) + __uint_as_float(uint32_t(y0 >> 32))) +
                        (__uint_as_float(uint32_t(y1)) + __uint_as_float(uint32_t(y1 >> 32)));
            if (!FEW) {
                // The warpgroups' sums meet in shared memory; a pair of them adds them up while the others go on.  (Behind piece - 1's
                // barrier the pair that had piece - 2 has read this buffer: it arrived there after that.)
                if (piece >= 2) wait(bar(kKmDone + ((piece - 1) & 1)), ((piece - 1) >> 1) & 1, 112);
                float* buf = s_acc + (piece & 1) * 512;
                buf[wg * 128 + r] = sum;
                mbar_arrive(bar(kKmDone + (piece & 1)));
                if ((piece & 1) == st) {
                    wait(bar(kKmDone + (piece & 1)), (piece >> 1) & 1, 113);
                    sum = buf[half * 128 + r] + buf[(half + 2) * 128 + r];
                }
            }
            if ((piece & 1) == st) {
                const int key = key0 + r;
                if (w.starts && w.ends(p)) {
                    if (key < p.T_kv) {
                        const size_t at = size_t(w.bh) * p.T_cap + key;
                        p.mass[at] = sum + (p.mass_in != nullptr && key < off ? p.mass_in[at] : 0.f);
                    }
                } else {
                    const int slot = piece > 0;
                    p.part[size_t(blockIdx.x * 2 + slot) * kKmTile + half * 128 + r] = sum;
                    if (half == 0 && r == 0) dir[slot] = make_int2(w.bh * p.tiles + w.jt, (w.starts ? kPieceStart : 0) | (w.ends(p) ? kPieceEnd : 0));
                }
            }
            w.next(p);
        }
    } else {
      setmaxnreg_dec<64>();
      if (warp == 16) {
        // =========================== TMA producer ===========================
        if (lane == 0) {
            tma_prefetch_desc(&mapQ);
            tma_prefetch_desc(&mapK);
            const uint32_t unit_bytes = uint32_t(rows) * D * 2;
            RingAt ka, qa;
            int held = -1;                                               // (b, hk) that the slots' units are of
            int fresh = 0;                                               // slots to fill with its units (p.stay)
            int b = w.bh / p.Hk, hk = w.bh - b * p.Hk, bh = w.bh;
#pragma unroll 1
            while (w.left > 0) {
                if (bh != w.bh) {
                    bh = w.bh;
                    if ((hk += p.team) >= p.Hk) { hk -= p.Hk; ++b; }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h, ka.next(p.k_slots)) {
                    if (ka.round > 0) wait(bar(kKmKEmpty + ka.slot), (ka.round - 1) & 1, 120);
                    mbar_arrive_expect_tx(bar(kKmKFull + ka.slot), L::kSlotBytes);
#pragma unroll
                    for (int s = 0; s < NSUB; ++s)
                        tma_load_4d(sbase + ka.slot * L::kSlotBytes + s * L::kSubBytes, &mapK, bar(kKmKFull + ka.slot), s * 64, hk, w.jt * kKmTile + h * 128, b);
                }
                if (held != bh) { held = bh; fresh = p.q_slots; }
#pragma unroll 1
                for (int u = w.u0; u < w.u1; ++u, qa.next(p.q_slots)) {
                    if (qa.round > 0) wait(bar(kKmQEmpty + qa.slot), (qa.round - 1) & 1, 121);
                    if (p.stay && fresh == 0) {
                        mbar_arrive(bar(kKmQHere + qa.slot));
                        continue;
                    }
                    --fresh;
                    mbar_arrive_expect_tx(bar(kKmQHere + qa.slot), unit_bytes);
#pragma unroll
                    for (int s = 0; s < NSUB; ++s)
                        tma_load_4d(sbase + (p.k_slots + qa.slot) * L::kSlotBytes + s * L::kSubBytes, &mapQ, bar(kKmQHere + qa.slot), s * 64, hk * p.G, u * p.P, b);
                }
                w.next(p);
            }
        }
      } else if (warp != 18) {
        // =========================== MMA issuers: S^T = K Q^T - LSE / scale ===========================
        // a warp for each half of the tiles, or for every second tile: one for all needs 890 to 1000 cycles a 128 x 128 product, of which the
        // tensor cores take 576 (d = 128)
        const int id = warp == 17 ? 0 : 1;
        const uint64_t dk0 = desc_kmajor_sw128(sbase, 0), dq0 = dk0 + uint64_t((p.k_slots * L::kSlotBytes) >> 4);
        const uint64_t d_ones = make_smem_desc_noswz(sbase + L::kOnes, uint32_t(L::kZero - L::kOnes), 128u);
        int n = 0, m = 0;                                                // units so far, of this warp's pieces
        RingAt ka, qa;
#pragma unroll 1
        for (int piece = 0; w.left > 0; ++piece) {
            const bool mine = !FEW || (piece & 1) == id;
            RingAt kb = ka;
            kb.next(p.k_slots);
            if (mine) {                                                  // both halves, also the other warp's: of three slots each is now one's, now the other's,
                wait(bar(kKmKFull + ka.slot), ka.round & 1, 130);        // and a wait tells only one phase from the next
                wait(bar(kKmKFull + kb.slot), kb.round & 1, 134);
            }
#pragma unroll 1
            for (int u = w.u0; u < w.u1; ++u, ++n, qa.next(p.q_slots)) {
                wait.both(bar(kKmQFull + qa.slot), qa.round & 1, bar(kKmQHere + qa.slot), qa.round & 1, 131, 135);   // likewise of every unit
                if (!mine) continue;
                const uint64_t dq = dq0 + uint64_t((qa.slot * L::kSlotBytes) >> 4);
                const int terms = L::kTerms + qa.slot * L::kTermBytes;
                const uint64_t dt = make_smem_desc_noswz(sbase + terms, uint32_t(L::kZero - terms), 128u);
                const int before = FEW ? m : n >> 1;               // units that the score buffer has had
                const uint32_t idesc = make_idesc_bf16(128, FEW ? key_mass_filled(p, u) : 128, false, false);
#pragma unroll 1
                for (int h = FEW ? 0 : id; h < (FEW ? 2 : id + 1); ++h) {
                    const int buf = (FEW ? id : n & 1) * 2 + h;
                    if (before > 0) wait(bar(kKmSEmpty + buf), (before - 1) & 1, 132);
                    tc_fence_after_sync();
                    const uint64_t dk = dk0 + uint64_t(((h ? kb.slot : ka.slot) * L::kSlotBytes) >> 4);
                    const uint32_t t = tmem + buf * 128;
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint64_t o = uint64_t(((kk >> 2) * L::kSubBytes + (kk & 3) * 32) >> 4);
                        umma_ss(t, dk + o, dq + o, idesc, kk > 0);
                    }
                    umma_ss(t, d_ones, dt, idesc, 1);
                    umma_commit(bar(kKmSFull + buf));
                }
                ++m;
            }
            if (mine && (FEW || id == 0)) umma_commit(bar(kKmKEmpty + ka.slot));
            if (mine && (FEW || id == 1)) umma_commit(bar(kKmKEmpty + kb.slot));
            kb.next(p.k_slots);
            ka = kb;
            w.next(p);
        }
        if (*abort_flag != 0) {
            // A wait gave up somewhere: make sure no MMA of this thread is still in flight before TMEM is released.
            umma_commit(bar(kKmDrain + id));
            const uint64_t t0 = globaltimer_ns();
            while (!mbar_try_wait(bar(kKmDrain + id), 0) && globaltimer_ns() - t0 < 20000000ull) {}
        }
      } else if (warp == 18) {
        // =========================== LSE terms of a unit's rows; rows that saw no key ===========================
        int pos[4], at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = lane + i * 32;
            pos[i] = c < rows ? c / p.G : p.T_q;                         // T_q: no position of any unit
            at[i] = (c < rows ? c % p.G : 0) * p.T_q + (c < rows ? c / p.G : 0);
        }
        // The values of the next two units are on their way while one is written.
        int units = w.left, u = w.u0;
        auto fetch = [&](float (&v)[4]) {
            if (w.left <= 0) return;
            const int i0 = u * p.P;
            const float* src = p.LSE + size_t(w.bh) * p.G * p.T_q + i0;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pos[i] < p.T_q - i0 ? __ldg(src + at[i]) : INFINITY;
            if (++u == w.u1) {
                w.next(p);
                u = w.u0;
            }
        };
        float v[4], v1[4], v2[4];
        fetch(v);
        fetch(v1);
        RingAt qa;
#pragma unroll 1
        for (; units > 0; --units, qa.next(p.q_slots)) {
            fetch(v2);
            if (qa.round > 0) wait(bar(kKmQEmpty + qa.slot), (qa.round - 1) & 1, 140);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4 t = make_uint4(0x0000ff80u, 0u, 0u, 0u);           // -inf: no row, or one without keys (LSE -inf)
                if (fabsf(v[i]) != INFINITY) split3_bf16(-v[i] * p.inv_scale, t.x, t.y);
                *reinterpret_cast<uint4*>(smem + L::kTerms + qa.slot * L::kTermBytes + (lane + i * 32) * 16) = t;
            }
            if (__any_sync(0xffffffffu, v[0] == -INFINITY || v[1] == -INFINITY || v[2] == -INFINITY || v[3] == -INFINITY)) {
                // -inf takes up any number, but not NaN: the query of a row that saw no key may hold anything
                wait(bar(kKmQHere + qa.slot), qa.round & 1, 141);
#pragma unroll 1
                for (int e = 0; e < 4 * NSUB * 8; ++e) {
                    const int i = e / (NSUB * 8), r = lane + i * 32, sub = e / 8 % NSUB;
                    if ((i == 0 ? v[0] : i == 1 ? v[1] : i == 2 ? v[2] : v[3]) == -INFINITY)
                        *reinterpret_cast<uint4*>(smem + (p.k_slots + qa.slot) * L::kSlotBytes + sub * L::kSubBytes + r * 128 + (e & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = v1[i];
                v1[i] = v2[i];
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kKmQFull + qa.slot));
        }
      }
    }

    tc_fence_before_sync();
    __syncthreads();
    abort_teardown(abort_flag, 512);
    __syncthreads();
    if (warp == 17) tmem_dealloc(tmem, 512);
}

// Adds the pieces of the tiles that several runs share: CTA c takes the tile that starts in run c and does not end there.  First how many there are, 32 runs
// at a look, then the sums, 16 on their way at once and added in order (one after the other: 1409 rows, 8 heads on 1, d = 64, 25 pieces a tile: 19.4 -> 12.7 us).
__global__ void __launch_bounds__(kKmTile)
key_mass_join_kernel(const KeyMassParams p) {
    const int ctas = gridDim.x, c = blockIdx.x, r = threadIdx.x;
    const int2* dir = reinterpret_cast<const int2*>(p.part + size_t(ctas) * 2 * kKmTile);
    grid_dependency_wait();                           // launched when key_mass_kernel's last CTA has gone, which lets nothing start earlier
    if (g_moda_status != 0) return;                   // a wait was given up before or in key_mass_kernel: there are no sums
    // the piece at the end of run c: its second entry, or its first where the run is one piece
    int slot = 2 * c + 1;
    int2 d = dir[slot];
    if (d.y == kPieceNone) d = dir[--slot];
    if (d.y != kPieceStart) return;                   // ends in its run (or nothing is shared), or does not start in it
    float sum = p.part[size_t(slot) * kKmTile + r];
    int more = 0;
    for (bool found = false; !found;) {
        const int k = c + (more + (r & 31) + 1) * p.team;
        const unsigned there = __ballot_sync(0xffffffffu, k < ctas), last = __ballot_sync(0xffffffffu, k < ctas && (dir[2 * k].y & kPieceEnd));
        found = last != 0u || there != 0xffffffffu;
        more += last != 0u ? __ffs(last) : __popc(there);
    }
    constexpr int UN = 16;
    for (int i0 = 1; i0 <= more; i0 += UN) {
        float x[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) x[u] = p.part[size_t(2 * (c + min(i0 + u, more) * p.team)) * kKmTile + r];
#pragma unroll
        for (int u = 0; u < UN; ++u)
            if (i0 + u <= more) sum += x[u];
    }
    const int bh = d.x / p.tiles, key = (d.x - bh * p.tiles) * kKmTile + r;
    if (key < p.T_kv) {
        const size_t at = size_t(bh) * p.T_cap + key;
        p.mass[at] = sum + (p.mass_in != nullptr && key < p.T_kv - p.T_q ? p.mass_in[at] : 0.f);
    }
}

}  // namespace moda
