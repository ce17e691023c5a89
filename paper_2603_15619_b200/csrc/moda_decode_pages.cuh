// The decode step over the paged sequence cache in 8 bits (moda_pages.cuh): a token's query heads against all blocks of its sequence, or against those
// that an index names, and its l depth pairs, under one softmax.
//
//   pages_split_kernel    a block of a (sequence, key/value head) is a unit; the units of all, in this order, are cut into equal runs, one per warp of the
//                         device, and every warp works through its own: nothing waits for another warp.  A lane's share of a block's keys is the operand of its
//                         matrix products as it lies in memory, and so is its share of the values: nothing is turned on the way.  A warp has a ring of
//                         its own for three or four pieces (a block's keys, or its values) in shared memory, all but one on their way: 192 KiB an SM at d = 128.
//                         Other warps of the CTA take the depth pairs, a partial result like the rest.  Groups of 16 or 32 query heads are sets of 8, whose runs
//                         take the same blocks at the same time.
//   pages_merge_kernel    one or four warps per (sequence, query head) join the partial results.
//
// One block, lane = (g, t) = (lane / 4, lane % 4), products m16n8k16 of f16 with fp32 sums, eight heads as columns:
//
//   S^T = K Q^T, keys as rows.  Rows g and g + 8 of the j-th sixteen are keys a = 16 (g / 2) + g % 2 + 4 j and a + 2; the lane holds their codes 64 i + 16 t .. + 15, and a
//   product pairs the same four of them with the same four of q, so that their order in it is no matter.  It ends up with the scores of those keys for heads 2 t, 2 t + 1.
//   O^T = V^T P^T, features as rows: the lane's value codes are those of feature g (and g + 8) of keys 16 t .. 16 t + 15, whose weights for head g are what the scores'
//   lanes have, turned 8 x 8 at a time.
//
// Codes are exact in f16 and so is q once a row is scaled by a power of two, its elements above 2^-31 of the largest at least (those below by up to 2^-39 of it).  Keys'
// scales multiply scores, in fp32.
// Values' scales go into the weights: w = exp2(s + log2(scale) - m'), with a running maximum m' of its own, so that the largest weight is 2^14;
// weights are rounded to f16 for the product (2^-11; below 2^-28 of the largest by up to 2^-39 of it), the row sum and both maxima are fp32.  A row of zeros, whose scale is 1
// by the format, has weight 0 in the product and leaves m' alone: beside it, rows below 2^-28 of it would lose bits for nothing.
//
// 32 sequences to 8192, 64 heads on 8, d = 128, 24 depth pairs: 59.4 us, of which the merge is 5; the bytes take 43.6 at the copy rate.  Read in this order by these warps
// without any arithmetic they take 45 (5.97 TB/s); the rest is that SMs which share their path to L2 with more others stream up to 20 % slower (equal runs end
// after 45 to 61 us).  Runs that others take over when they are done cost more in partial results and in queries that wait behind the stream than they win (63 us
// and more).  96 sequences to 1500, 24 heads on 8, d = 64: 31 to 32 us against 13.2: a block of half the bytes has the same softmax, three heads in columns for eight.
// Products of e4m3 codes as they are (m16n8k32) are no faster, 67.0 against 66.2 us at that stage.
#pragma once

#include <cstdint>
#include <type_traits>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "moda_depth_gqa.cuh"
#include "moda_pages.cuh"
#include "sm100_ptx.cuh"

namespace moda {

struct PagesDecodeParams : PagesParams {
    // The query heads of a key/value head in kv_rep sets of at most 8; set s of head hk of sequence b is number (b Hk + hk) kv_rep + s, heads number * G ..
    const __nv_bfloat16* q;       // [B][H][d]
    const uint8_t* pages;
    const int* lens;              // [B], each 0 .. max_len
    const int* index;             // [B][Hk][n_index]: blocks, or null: all
    const __nv_bfloat16* depth;   // [l][B][Hk][2][d]
    __nv_bfloat16* O;             // [B][H][d]
    float* LSE;                   // [B][H]
    float* part;                  // [warps + sets][G][d + 2], then [sets][G][d + 2] of the depth pairs: m (log2 domain), l, o[d]
    int* before;                  // [B + 1]: blocks of the sequences before each
    int G, H, l, kv_rep, max_len, n_index, warps;
    float scale_log2;
    __device__ __forceinline__ int sets() const { return B * Hk * kv_rep; }
    __device__ __forceinline__ int len(int b) const { return min(max(lens[b], 0), max_len); }
    // Blocks of a sequence that a group takes.
    __device__ __forceinline__ int units(int b) const {
        const int n = pages_blocks(len(b));
        return index ? min(n, n_index) : n;
    }
};

constexpr int kPagesMostBatch = 2048;                                // sequences of a call: their blocks are counted in shared memory
template <int D>
struct PagesSplit {
    static constexpr int kWarps = D == 64 ? 9 : 8, kDepthWarps = D == 64 ? 3 : 4;   // of a CTA, one an SM
    static constexpr int kThreads = (kWarps + kDepthWarps) * 32;
    static constexpr int kPiece = kPageBlock * D;                    // bytes: a block's key codes, or its value codes
    static constexpr int kPieces = D == 64 ? 4 : 3;                  // that a warp has in shared memory or on the way
    static constexpr int kScaleSets = D == 64 ? 3 : 2;               // blocks whose scales it has there
    static constexpr int kWarpBytes = kPieces * kPiece + kScaleSets * 8 * kPageBlock;
    static constexpr int smem(int B) { return kWarps * kWarpBytes + (B + 1) * 4; }
    static_assert(smem(kPagesMostBatch) + 4096 <= 232448, "shared memory");
};
constexpr int kPagesMergeThreads = 128;

__device__ __forceinline__ void mma_f16_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// An 8 x 8 matrix of 16-bit numbers, two adjacent ones of a row a lane, turned.
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// Where a warp is in the order of all units.
struct PagesWalk {
    int b, r, j, n;               // sequence, group of it, unit of that group, units of a group of this sequence
    __device__ __forceinline__ void begin(const int* before, int B, int Hk, long long u) {
        int lo = 0, hi = B;                                          // before[lo] Hk <= u < before[hi] Hk
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((long long)before[mid] * Hk <= u) lo = mid; else hi = mid;
        }
        b = lo;
        n = before[b + 1] - before[b];
        const int rest = int(u - (long long)before[b] * Hk);
        r = rest / n;
        j = rest - r * n;
    }
    __device__ __forceinline__ bool next(const int* before, int Hk) {   // true: another group
        if (++j < n) return false;
        j = 0;
        if (++r == Hk) {
            r = 0;
            do { ++b; n = before[b + 1] - before[b]; } while (n == 0);   // there is another unit
        }
        return true;
    }
};

// The depth pairs of a group's token by one warp: a partial result like those of the cached keys.  Scores by m16n8k16 products of bf16 (heads as rows, slots as
// columns), weights in fp32 through shared memory, and the weighted values on the CUDA cores, each lane D / 32 features of all heads.
template <int D>
__device__ __forceinline__ void pages_depth(const PagesDecodeParams& p, int set, float (*s_w)[8], float* out, int lane) {
    constexpr int FPL = D / 32, SLOTS = 32;
    const int g = lane >> 2, t = lane & 3;
    const size_t stride = size_t(p.B) * p.Hk * 2 * D;                // elements between depth slots
    const __nv_bfloat16* depth0 = p.depth + size_t(set / p.kv_rep) * 2 * D;
    uint4 q[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        q[i] = make_uint4(0u, 0u, 0u, 0u);
        if (g < p.G) q[i] = *reinterpret_cast<const uint4*>(p.q + (size_t(set) * p.G + g) * D + 32 * i + 8 * t);
    }
    float m = -INFINITY, sum = 0.f, acc[8][FPL];
#pragma unroll
    for (int h = 0; h < 8; ++h)
#pragma unroll
        for (int c = 0; c < FPL; ++c) acc[h][c] = 0.f;
    constexpr int BATCH = 64 / FPL;                                  // value rows that are on their way together
    using Row = typename std::conditional<FPL == 4, uint2, uint32_t>::type;
#pragma unroll 1
    for (int i0 = 0; i0 < p.l; i0 += SLOTS) {
        const int n_slot = min(p.l - i0, SLOTS);
        uint4 k[4][D / 32];                                          // rows past the last slot are that one's again
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const uint4* row = reinterpret_cast<const uint4*>(depth0 + size_t(i0 + min(8 * n + g, n_slot - 1)) * stride);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) k[n][i] = row[4 * i + t];
        }
        Row v[BATCH];
        auto load_v = [&](int j0) {
#pragma unroll
            for (int j = 0; j < BATCH; ++j) v[j] = *reinterpret_cast<const Row*>(depth0 + size_t(i0 + min(j0 + j, n_slot - 1)) * stride + D + lane * FPL);
        };
        if (FPL == 2) load_v(0);                                     // (both at once are more than the registers hold at d = 128)
        float s[4][2];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                mma_bf16_16x8x16(c, q[i].x, 0u, q[i].y, 0u, k[n][i].x, k[n][i].y);
                mma_bf16_16x8x16(c, q[i].z, 0u, q[i].w, 0u, k[n][i].z, k[n][i].w);
            }
            s[n][0] = 8 * n + 2 * t < n_slot ? c[0] * p.scale_log2 : -INFINITY;
            s[n][1] = 8 * n + 2 * t + 1 < n_slot ? c[1] * p.scale_log2 : -INFINITY;
        }
        if (FPL == 4) load_v(0);
        float top = m;
#pragma unroll
        for (int n = 0; n < 4; ++n) top = fmaxf(top, fmaxf(s[n][0], s[n][1]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float base = top == -INFINITY ? 0.f : top, alpha = fast_exp2(m - base);
        m = top;
        sum *= alpha;
        __syncwarp();
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float w = fast_exp2(s[n][i] - base);
                sum += w;
                s_w[8 * n + 2 * t + i][g] = w;
            }
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 8; ++h) {
            const float f = __shfl_sync(0xffffffffu, alpha, 4 * h);
#pragma unroll
            for (int c = 0; c < FPL; ++c) acc[h][c] *= f;
        }
#pragma unroll
        for (int j0 = 0; j0 < SLOTS; j0 += BATCH) {
            if (j0 >= n_slot) break;
            if (j0 > 0) load_v(j0);
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                if (j0 + j >= n_slot) break;
                float x[FPL];
                if constexpr (FPL == 4) {
                    x[0] = bf16_lo_to_f32(v[j].x); x[1] = bf16_hi_to_f32(v[j].x); x[2] = bf16_lo_to_f32(v[j].y); x[3] = bf16_hi_to_f32(v[j].y);
                } else {
                    x[0] = bf16_lo_to_f32(v[j]); x[1] = bf16_hi_to_f32(v[j]);
                }
                const float4 w0 = *reinterpret_cast<const float4*>(&s_w[j0 + j][0]), w1 = *reinterpret_cast<const float4*>(&s_w[j0 + j][4]);
                const float w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
                for (int h = 0; h < 8; ++h)
#pragma unroll
                    for (int c = 0; c < FPL; ++c) acc[h][c] = fmaf(w[h], x[c], acc[h][c]);
            }
        }
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    if (t == 0 && g < p.G) *reinterpret_cast<float2*>(out + g * (D + 2)) = make_float2(m, sum);
#pragma unroll
    for (int h = 0; h < 8; ++h)
        if (h < p.G) {
#pragma unroll
            for (int c = 0; c < FPL; c += 2) *reinterpret_cast<float2*>(out + h * (D + 2) + 2 + lane * FPL + c) = make_float2(acc[h][c], acc[h][c + 1]);
        }
}

template <int D>
__global__ void __launch_bounds__(PagesSplit<D>::kThreads, 1)
pages_split_kernel(const PagesDecodeParams p) {
    using L = PagesSplit<D>;
    constexpr int NW = L::kWarps, NP = L::kPieces, PIECE = L::kPiece;
    constexpr int KP = D / 64, FB = D / 16, CH = D / 16;             // 64-feature parts of a key; 16-feature rows of the value product; 16-byte pieces of a key
    constexpr int AHEAD = (1 + NP) / 2;                              // units that the ring is ahead, at most
    extern __shared__ __align__(16) uint8_t split_smem[];
    int* s_before = reinterpret_cast<int*>(split_smem + NW * L::kWarpBytes);      // [B + 1]
    __shared__ int s_sum[NW];
    __shared__ __align__(16) float s_w[L::kDepthWarps][32][8];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;
    grid_dependency_wait();
    if (warp >= NW) {
        // ---- warps for the depth pairs ----
        const int sets = p.l > 0 ? p.sets() : 0;
        for (int i = (warp - NW) * gridDim.x + blockIdx.x; i < sets; i += L::kDepthWarps * gridDim.x)
            pages_depth<D>(p, i, s_w[warp - NW], p.part + (size_t(p.warps) + p.sets() + i) * p.G * (D + 2), lane);
        return;
    }
    // ---- blocks of the sequences before each ----
    {
        const int per = (p.B + NW * 32 - 1) / (NW * 32);
        const int b0 = min(tid * per, p.B), b1 = min(b0 + per, p.B);
        int sum = 0;
        for (int b = b0; b < b1; ++b) sum += p.units(b);
        int incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += up;
        }
        if (lane == 31) s_sum[warp] = incl;
        asm volatile("bar.sync 1, %0;" ::"n"(NW * 32) : "memory");
        int at = incl - sum;
        for (int w = 0; w < warp; ++w) at += s_sum[w];
        for (int b = b0; b < b1; ++b) {
            s_before[b] = at;
            at += p.units(b);
        }
        if (b0 < b1 && b1 == p.B) s_before[p.B] = at;
        asm volatile("bar.sync 1, %0;" ::"n"(NW * 32) : "memory");
        if (blockIdx.x == 0)
            for (int b = tid; b <= p.B; b += NW * 32) p.before[b] = s_before[b];
    }
    // neighbours in the order are on different SMs; the sets of a head take the same blocks at the same time, so that one of them finds them in L2
    const long long total = (long long)s_before[p.B] * p.Hk, runs = min(total, (long long)(p.warps / p.kv_rep));
    const int w = warp * gridDim.x + blockIdx.x, run = w / p.kv_rep, set = w - run * p.kv_rep;
    if (run >= runs) return;
    const int first = int(total * run / runs), n_unit = int(total * (run + 1) / runs) - first;

    // ---- the ring: pieces (a unit's keys, then its values) in order, the next ones on their way while one is worked on ----
    uint8_t* ring = split_smem + warp * L::kWarpBytes;
    const uint32_t ring_u32 = smem_u32(ring);
    float* scales = reinterpret_cast<float*>(ring + NP * PIECE);     // [kScaleSets][128], of consecutive units
    PagesWalk ahead;                                                 // the unit that is looked up next
    ahead.begin(s_before, p.B, p.Hk, first);
    int left = n_unit;                                               // units not yet looked up
    uint32_t qf[KP][8];                                              // this lane's features of head g, f16
    float q_scale[2];                                                // scale log2(e) over the power of two of heads 2 t, 2 t + 1
    auto load_q = [&](uint4 (&v)[KP][2], int group) {
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            v[i][0] = v[i][1] = make_uint4(0u, 0u, 0u, 0u);
            if (g < p.G) {
                const uint4* src = reinterpret_cast<const uint4*>(p.q + (size_t(group) * p.G + g) * D + 64 * i + 16 * t);
                v[i][0] = src[0];
                v[i][1] = src[1];
            }
        }
    };
    auto take_q = [&](const uint4 (&v)[KP][2]) {
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < KP; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t words[4] = {v[i][k].x, v[i][k].y, v[i][k].z, v[i][k].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) most = fmaxf(most, fmaxf(fabsf(bf16_lo_to_f32(words[j])), fabsf(bf16_hi_to_f32(words[j]))));
            }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int e = max(int(__float_as_uint(most) >> 23), 20) - 127;          // most < 2^(e + 1): times 2^(14 - e), below 2^15
        const float up = __uint_as_float(uint32_t(127 + 14 - e) << 23);
        const float down = p.scale_log2 * __uint_as_float(uint32_t(127 - 14 + e) << 23);
        q_scale[0] = __shfl_sync(0xffffffffu, down, 8 * t);
        q_scale[1] = __shfl_sync(0xffffffffu, down, 8 * t + 4);
#pragma unroll
        for (int i = 0; i < KP; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t words[4] = {v[i][k].x, v[i][k].y, v[i][k].z, v[i][k].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) qf[i][4 * k + j] = pack_f16x2(bf16_lo_to_f32(words[j]) * up, bf16_hi_to_f32(words[j]) * up);
            }
    };
    uint4 raw[KP][2];
    load_q(raw, (ahead.b * p.Hk + ahead.r) * p.kv_rep + set);        // ahead of the pieces, behind which it would wait
    struct Place { const uint8_t* rec; int rows, group; };           // where a unit lies (null: nowhere), its keys, its set of heads
    auto block_of = [&]() -> int {
        return p.index ? p.index[(size_t(ahead.b) * p.Hk + ahead.r) * p.n_index + ahead.j] : ahead.j;
    };
    auto look_up = [&](int blk) -> Place {
        const int len = p.len(ahead.b);
        const int tile = blk >= 0 && blk < pages_blocks(len) ? p.tile(ahead.b, blk) : -1;
        Place x;
        x.rec = tile >= 0 ? p.pages + (size_t(tile) * p.Hk + ahead.r) * page_block_bytes(D) : nullptr;
        x.rows = tile >= 0 ? min(len - blk * kPageBlock, kPageBlock) : 0;
        x.group = (ahead.b * p.Hk + ahead.r) * p.kv_rep + set;
        if (--left > 0) ahead.next(s_before, p.Hk);
        return x;
    };
    // The keys (i = 0) or the values of a unit into a slot of the ring.  16-byte piece c of key row r lies at c ^ 4 (r % 2) where a row has 8, so that two
    // adjacent rows of four lanes each are in different banks.
    auto request = [&](const uint8_t* rec, int unit, int i, int slot) {
        if (rec) {
            const uint32_t dst = ring_u32 + slot * PIECE;
            if (i == 0) {
                const int r = lane / CH, c = lane % CH;
                const uint32_t to = dst + r * D + 16 * (D == 128 ? c ^ ((r & 1) << 2) : c);
#pragma unroll
                for (int k = 0; k < PIECE / 512; ++k) cp_async_16(to + k * 512, rec + k * 512 + lane * 16);
                cp_async_16(smem_u32(scales) + unit % L::kScaleSets * 512 + lane * 16, rec + 2 * PIECE + lane * 16);
            } else {
#pragma unroll
                for (int k = 0; k < PIECE / 512; ++k) cp_async_16(dst + k * 512 + lane * 16, rec + PIECE + k * 512 + lane * 16);
            }
        }
        cp_async_commit();
    };
    Place place[AHEAD + 1];                                          // of units u .. u + AHEAD
#pragma unroll
    for (int i = 0; i <= AHEAD; ++i) place[i] = left > 0 ? look_up(block_of()) : Place{nullptr, 0, -1};
#pragma unroll
    for (int i = 0; i <= AHEAD; ++i) {
        if (2 * i < NP) request(place[i].rec, i, 0, 2 * i);
        if (2 * i + 1 < NP) request(place[i].rec, i, 1, 2 * i + 1);
    }
    take_q(raw);
    if (place[1].group != place[0].group && place[1].group >= 0) load_q(raw, place[1].group);
    int slot = 0;                                                    // of the piece in work, which the one NP behind it takes over
    auto pass_on = [&](int u, int i) {
        request(place[(i + NP) / 2].rec, u + (i + NP) / 2, (i + NP) % 2, slot);
        slot = slot + 1 == NP ? 0 : slot + 1;
    };

    // of heads 2 t, 2 t + 1: maxima of the scores and of the weights' exponents, row sums (this lane's keys)
    float m[2] = {-INFINITY, -INFINITY}, mw[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
    float o[FB][4];                                                  // features 16 f + g (c0 c1) and + 8 (c2 c3) of heads 2 t, 2 t + 1
#pragma unroll
    for (int f = 0; f < FB; ++f) { o[f][0] = 0.f; o[f][1] = 0.f; o[f][2] = 0.f; o[f][3] = 0.f; }
#pragma unroll 1
    for (int u = 0; u < n_unit; ++u) {
        const int rows = place[0].rows;
        const int blk = left > 0 ? block_of() : 0;                   // of unit u + AHEAD + 1
        float* own = scales + u % L::kScaleSets * 128;
        float c[4][4];                                               // of keys a = 16 (g / 2) + 4 j + g % 2 and a + 2: heads 2 t, 2 t + 1 of either
#pragma unroll
        for (int j = 0; j < 4; ++j) { c[j][0] = 0.f; c[j][1] = 0.f; c[j][2] = 0.f; c[j][3] = 0.f; }
        cp_async_wait<NP - 1>();
        __syncwarp();
        bool one = false;                                            // a value row of this lane's has scale 1, so that it may be one of zeros
        if (rows > 0) {
            {
                // scales in the order in which the lanes have the keys: [2 (key / 16) + key % 2][key % 16 / 2]; of the values, their logarithms
                const float2 k = *reinterpret_cast<const float2*>(own + 2 * lane), v = *reinterpret_cast<const float2*>(own + kPageBlock + 2 * lane);
                one = v.x == 1.f || v.y == 1.f;
                __syncwarp();
                float* to = own + (lane >> 3) * 16 + (lane & 7);
                to[0] = k.x;
                to[8] = k.y;
                to[kPageBlock] = __log2f(v.x);
                to[kPageBlock + 8] = __log2f(v.y);
            }
#pragma unroll
            for (int i = 0; i < KP; ++i) {
                const uint8_t* row = ring + slot * PIECE + (16 * (g >> 1) + (g & 1)) * D + 16 * (D == 128 ? (4 * i + t) ^ ((g & 1) << 2) : t);
                uint4 x[4], y[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] = *reinterpret_cast<const uint4*>(row + 4 * j * D);
                    y[j] = *reinterpret_cast<const uint4*>(row + (4 * j + 2) * D);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t a0, a1, a2, a3;
                        e4m3x4_to_f16(k == 0 ? x[j].x : k == 1 ? x[j].y : k == 2 ? x[j].z : x[j].w, a0, a2);
                        e4m3x4_to_f16(k == 0 ? y[j].x : k == 1 ? y[j].y : k == 2 ? y[j].z : y[j].w, a1, a3);
                        mma_f16_16x8x16(c[j], a0, a1, a2, a3, qf[i][2 * k], qf[i][2 * k + 1]);
                    }
            }
        }
        __syncwarp();                                                // everyone has read the keys; the scales are in order
        pass_on(u, 0);
        if (__any_sync(0xffffffffu, one)) {
            // Rows of zeros add nothing to the weighted sum, and their scale is not of their size: weight 0 there, so that the others' keep their bits (in the row sum they count).
            cp_async_wait<NP - 1>();
            __syncwarp();
            uint32_t some[4] = {0u, 0u, 0u, 0u};                     // a byte per position 16 (lane % 4) ..: not 0 where it has a code that is not
#pragma unroll 4
            for (int k = 0; k < PIECE / 512; ++k) {
                const uint4 x = *reinterpret_cast<const uint4*>(ring + slot * PIECE + k * 512 + lane * 16);
                some[0] |= x.x; some[1] |= x.y; some[2] |= x.z; some[3] |= x.w;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) some[i] |= __shfl_xor_sync(0xffffffffu, some[i], off);
                if (lane < 4) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if ((some[i] >> (8 * k) & 0x7fu) == 0u) own[kPageBlock + 16 * lane + 8 * (k & 1) + 2 * i + (k >> 1)] = -INFINITY;
                }
            }
            __syncwarp();
        }
        uint32_t pw[8];                                              // weights of keys 16 t + 4 j, + 1 (and + 2, + 3) of head g
        if (rows > 0) {
            float s[8][2], x[8];                                     // scores of this lane's keys a, a + 2, ..; log2 of the values' scales
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 a = *reinterpret_cast<const float4*>(own + 8 * g + 4 * i);
                const float4 y = *reinterpret_cast<const float4*>(own + kPageBlock + 8 * g + 4 * i);
                const float sk[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[4 * i + j][0] = c[2 * i + j / 2][2 * (j & 1)] * sk[j] * q_scale[0];
                    s[4 * i + j][1] = c[2 * i + j / 2][2 * (j & 1) + 1] * sk[j] * q_scale[1];
                }
                x[4 * i] = y.x; x[4 * i + 1] = y.y; x[4 * i + 2] = y.z; x[4 * i + 3] = y.w;
            }
            if (rows < kPageBlock) {                                 // what lies past the last key may hold anything
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (16 * (g >> 1) + (g & 1) + 2 * j >= rows) { s[j][0] = s[j][1] = -INFINITY; x[j] = 0.f; }
            }
            float f[2], base[2], base_w[2], part[2] = {0.f, 0.f};
            bool moved = false;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float mx = s[0][h], mxw = s[0][h] + x[0];
#pragma unroll
                for (int j = 1; j < 8; ++j) { mx = fmaxf(mx, s[j][h]); mxw = fmaxf(mxw, s[j][h] + x[j]); }
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) {
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
                    mxw = fmaxf(mxw, __shfl_xor_sync(0xffffffffu, mxw, off));
                }
                mx = fmaxf(m[h], mx);
                mxw = fmaxf(mw[h], mxw);
                base[h] = mx == -INFINITY ? 0.f : mx;
                base_w[h] = mxw == -INFINITY ? 0.f : mxw - 14.f;
                sum[h] *= fast_exp2(m[h] - base[h]);
                f[h] = mw[h] != mxw && mw[h] != -INFINITY ? fast_exp2(mw[h] - mxw) : 1.f;
                moved |= f[h] != 1.f;
                m[h] = mx;
                mw[h] = mxw;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                part[0] += fast_exp2(s[j][0] - base[0]);
                part[1] += fast_exp2(s[j][1] - base[1]);
                pw[j] = transpose_8x8(pack_f16x2(fast_exp2(s[j][0] + x[j] - base_w[0]), fast_exp2(s[j][1] + x[j] - base_w[1])));
            }
            sum[0] += part[0];
            sum[1] += part[1];
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int i = 0; i < FB; ++i) { o[i][0] *= f[0]; o[i][1] *= f[1]; o[i][2] *= f[0]; o[i][3] *= f[1]; }
            }
        }
        Place behind = left > 0 ? look_up(blk) : Place{nullptr, 0, -1};
        cp_async_wait<NP - 1>();
        __syncwarp();
        if (rows > 0) {
            uint8_t* sv = ring + slot * PIECE;
            if (rows < kPageBlock) {                                 // value codes past the last key: zero, their weights are 0
                for (int e = lane; e < PIECE / 16; e += 32) {
                    uint4* at16 = reinterpret_cast<uint4*>(sv) + e;
                    uint32_t word[4] = {at16->x, at16->y, at16->z, at16->w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int some = min(max(rows - 16 * (e & 3) - 4 * k, 0), 4);
                        word[k] = some == 4 ? word[k] : word[k] & ((1u << (8 * some)) - 1u);
                    }
                    *at16 = make_uint4(word[0], word[1], word[2], word[3]);
                }
                __syncwarp();
            }
#pragma unroll
            for (int f0 = 0; f0 < FB; f0 += 4) {
                uint4 x[4], y[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    x[f] = *reinterpret_cast<const uint4*>(sv + (16 * (f0 + f) + g) * kPageBlock + 16 * t);
                    y[f] = *reinterpret_cast<const uint4*>(sv + (16 * (f0 + f) + 8 + g) * kPageBlock + 16 * t);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        uint32_t a0, a1, a2, a3;
                        e4m3x4_to_f16(k == 0 ? x[f].x : k == 1 ? x[f].y : k == 2 ? x[f].z : x[f].w, a0, a2);
                        e4m3x4_to_f16(k == 0 ? y[f].x : k == 1 ? y[f].y : k == 2 ? y[f].z : y[f].w, a1, a3);
                        mma_f16_16x8x16(o[f0 + f], a0, a1, a2, a3, pw[2 * k], pw[2 * k + 1]);
                    }
            }
        }
        __syncwarp();                                                // everyone has read the values
        pass_on(u, 1);
        if (u + AHEAD + 1 >= n_unit) grid_launch_dependents();       // all loads are on their way: the merge may come up
        const int group = place[0].group;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) place[i] = place[i + 1];
        place[AHEAD] = behind;
        if (place[0].group != group) {
            // ---- the group's partial result of this warp ----
            float* out = p.part + (size_t(run) * p.kv_rep + group) * p.G * (D + 2);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], off);
                if (2 * t + h < p.G) {
                    float* to = out + (2 * t + h) * (D + 2);
                    if (g == 0) *reinterpret_cast<float2*>(to) = make_float2(m[h], sum[h]);
                    // the weighted sums are relative to 2^(mw - 14), the row sum to 2^m
                    const float f = mw[h] == -INFINITY ? 0.f : fast_exp2(mw[h] - 14.f - m[h]);
#pragma unroll
                    for (int i = 0; i < FB; ++i) {
                        to[2 + 16 * i + g] = o[i][h] * f;
                        to[2 + 16 * i + 8 + g] = o[i][2 + h] * f;
                    }
                }
                m[h] = mw[h] = -INFINITY;
                sum[h] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < FB; ++i) { o[i][0] = 0.f; o[i][1] = 0.f; o[i][2] = 0.f; o[i][3] = 0.f; }
        }
        // the queries of the next unit's group; those of the one behind it are on their way for a unit's time
        if (place[0].group != group && place[0].group >= 0) take_q(raw);
        if (place[1].group != place[0].group && place[1].group >= 0) load_q(raw, place[1].group);
    }
}

// W warps per row (sequence, query head); lanes hold D / 32 adjacent features, a warp takes every W-th partial result.  A token without any key has O = 0 and LSE = -inf.
template <int D, int W>
__global__ void __launch_bounds__(kPagesMergeThreads)
pages_merge_kernel(const PagesDecodeParams p) {
    constexpr int FPL = D / 32, NW = kPagesMergeThreads / 32, UN = 8;
    __shared__ float s_red[NW], s_sum[NW];
    __shared__ __align__(16) float s_acc[W > 1 ? NW : 1][D];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long row = (long long)blockIdx.x * (NW / W) + warp / W;
    const int part_of = warp % W;
    const bool there = row < (long long)p.B * p.H;
    const int b = there ? int(row / p.H) : 0, h = there ? int(row - (long long)b * p.H) : 0;
    const int r = h / p.G, g = h - r * p.G;
    int own = 0, before = 0, all = 0;                                // blocks of this sequence, of those before it, of all
    const bool few = p.B <= 128;
    if (few) {
        for (int i = lane; i < p.B; i += 32) {
            const int v = p.units(i);
            all += v;
            if (i < b) before += v;
        }
        all = __reduce_add_sync(0xffffffffu, all);
        before = __reduce_add_sync(0xffffffffu, before);
        own = p.units(b);
    }
    // ---- from here on: what the split kernel wrote ----
    grid_dependency_wait();
    if (!few) {
        before = __ldcg(p.before + b);
        own = __ldcg(p.before + b + 1) - before;
        all = __ldcg(p.before + p.B);
    }
    const long long total = (long long)all * p.Hk, first = (long long)before * p.Hk + (long long)(r / p.kv_rep) * own;
    // run of a unit
    const long long runs = min(total, (long long)(p.warps / p.kv_rep));
    const int w0 = own > 0 ? int(((first + 1) * runs - 1) / total) : 0, w1 = own > 0 ? int(((first + own) * runs - 1) / total) : -1;
    const int S = w1 - w0 + 1, n = S + (p.l > 0 ? 1 : 0);            // the last one is that of the depth pairs
    const size_t stride = size_t(p.kv_rep) * p.G * (D + 2), group = size_t(b) * p.Hk * p.kv_rep + r;
    const float* part = p.part + (size_t(w0) * p.kv_rep + group) * p.G * (D + 2) + g * (D + 2);
    const float* depth = p.part + (size_t(p.warps) + p.sets() + group) * p.G * (D + 2) + g * (D + 2);
    float m = -INFINITY, lt = 0.f, acc[FPL];
#pragma unroll
    for (int c = 0; c < FPL; ++c) acc[c] = 0.f;
    for (int s0 = there ? part_of : n; s0 < n; s0 += W * UN) {
        float2 ml[UN];
        float x[UN][FPL];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int s = s0 + u * W;
            ml[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int c = 0; c < FPL; ++c) x[u][c] = 0.f;
            if (s < n) {
                const float* src = s < S ? part + size_t(s) * stride : depth;
                ml[u] = __ldcg(reinterpret_cast<const float2*>(src));
#pragma unroll
                for (int c = 0; c < FPL; c += 2) {
                    const float2 v = __ldcg(reinterpret_cast<const float2*>(src + 2 + lane * FPL + c));
                    x[u][c] = v.x; x[u][c + 1] = v.y;
                }
            }
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < UN; ++u) top = fmaxf(top, ml[u].x);
        const float base = top == -INFINITY ? 0.f : top, alpha = fast_exp2(m - base);
        m = top;
        lt *= alpha;
#pragma unroll
        for (int c = 0; c < FPL; ++c) acc[c] *= alpha;
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const float f = fast_exp2(ml[u].x - base);               // 0 for a partial without keys, whose sums are 0 (or NaN: then so is the row)
            lt = fmaf(f, ml[u].y, lt);
#pragma unroll
            for (int c = 0; c < FPL; ++c) acc[c] = fmaf(f, x[u][c], acc[c]);
        }
    }
    float top = m;
    if constexpr (W > 1) {
        if (lane == 0) { s_red[warp] = m; s_sum[warp] = lt; }
#pragma unroll
        for (int c = 0; c < FPL; ++c) s_acc[warp][lane * FPL + c] = acc[c];
        __syncthreads();
        if (part_of != 0) return;
        top = s_red[warp];
#pragma unroll
        for (int i = 1; i < W; ++i) top = fmaxf(top, s_red[warp + i]);
        const float base = top == -INFINITY ? 0.f : top;
        lt = 0.f;
#pragma unroll
        for (int c = 0; c < FPL; ++c) acc[c] = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float f = fast_exp2(s_red[warp + i] - base);
            lt = fmaf(f, s_sum[warp + i], lt);
#pragma unroll
            for (int c = 0; c < FPL; ++c) acc[c] = fmaf(f, s_acc[warp + i][lane * FPL + c], acc[c]);
        }
    }
    if (!there) return;
#pragma unroll
    for (int c = 0; c < FPL; ++c) acc[c] = lt == 0.f ? 0.f : acc[c] / lt;
    __nv_bfloat16* O = p.O + size_t(row) * D + lane * FPL;
    if constexpr (FPL == 4) *reinterpret_cast<uint2*>(O) = make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
    else *reinterpret_cast<uint32_t*>(O) = pack_bf16x2(acc[0], acc[1]);
    if (lane == 0) p.LSE[row] = lt == 0.f ? -INFINITY : (top + log2f(lt)) * 0.6931471805599453f;
}

}  // namespace moda
