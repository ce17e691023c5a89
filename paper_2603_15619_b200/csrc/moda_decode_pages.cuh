// The decode step over the paged sequence cache in 8 bits (moda_pages.cuh): a token's query heads against all blocks of its sequence, or against those
// that an index names, and its l depth pairs, under one softmax.
//
//   pages_split_kernel    a block of a (sequence, key/value head) is a unit; the units of all, in this order, are cut into equal runs, one per warp of the
//                         device, and every warp works through its own: nothing waits for another warp.  A lane's share of a block's keys is the operand of its
//                         matrix products as it lies in memory, and so is its share of the values: nothing is turned on the way.  A warp has a ring of
//                         its own for three pieces (a block's keys, or its values) in shared memory, two on their way while one is worked on: 128 KiB an SM.
//   pages_merge_kernel    a CTA per (sequence, query head): the depth pairs, then the partial results of the group's warps.
//
// One block, lane = (g, t) = (lane / 4, lane % 4), products m16n8k16 of f16 with fp32 sums:
//
//   S = Q K^T, heads as rows.  Column g of the n-th eight keys is key 16 (g / 2) + 2 n + g % 2 of the block, whose codes 64 i + 16 t .. + 15 the lane holds:
//   a product pairs the same four of them with the same four of q, so that their order in it is no matter.  Thread t of a row then has the
//   scores of keys 16 t + 2 n, + 1: in all, of keys 16 t .. 16 t + 15.
//   O^T = V^T P^T, features as rows: the lane's value codes are those of feature g (and g + 8) of keys 16 t .. 16 t + 15, the keys whose weights it has.
//
// Codes are exact in f16 and so is q once a row is scaled by a power of two (below 2^-40 of its largest element it is rounded).  Keys' scales multiply scores, in fp32.
// Values' scales go into the weights: w = exp2(s + log2(scale) - m'), with a running maximum m' of its own, 2^14 below the largest f16 power;
// weights are rounded to f16 (2^-11) for the product, the row sum and both maxima are fp32.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "moda_depth_gqa.cuh"
#include "moda_pages.cuh"
#include "sm100_ptx.cuh"

namespace moda {

struct PagesDecodeParams : PagesParams {
    // Hk counts groups of at most 8 query heads; kv_rep of them read one key/value head
    const __nv_bfloat16* q;       // [B][H][d]
    const uint8_t* pages;
    const int* lens;              // [B], each 0 .. max_len
    const int* index;             // [B][Hk / kv_rep][n_index]: blocks, or null: all
    const __nv_bfloat16* depth;   // [l][B][Hk / kv_rep][2][d]
    __nv_bfloat16* O;             // [B][H][d]
    float* LSE;                   // [B][H]
    float* part;                  // [warps + B Hk][G][d + 2]: m (log2 domain), l, o[d]
    int* before;                  // [B + 1]: blocks of the sequences before each
    int G, H, l, kv_rep, max_len, n_index, warps;
    float scale_log2;
    __device__ __forceinline__ int len(int b) const { return min(max(lens[b], 0), max_len); }
    // Blocks of a sequence that a group takes.
    __device__ __forceinline__ int units(int b) const {
        const int n = pages_blocks(len(b));
        return index ? min(n, n_index) : n;
    }
};

constexpr int kPagesMostBatch = 2048;                                // sequences of a call: their blocks are counted in shared memory
constexpr int kPagesWarps = 11, kPagesDepthWarps = 1;                // of a CTA, one an SM
constexpr int kPagesSplitThreads = (kPagesWarps + kPagesDepthWarps) * 32;
constexpr int kPagesPiece = 64 * kPageBlock;                         // bytes: 64 features of a block's keys, or of its values
constexpr int kPagesPieces = 4;                                      // that a warp has in shared memory or on the way
constexpr int kPagesScaleSets = 3;                                   // blocks whose scales it has there
constexpr int kPagesWarpBytes = kPagesPieces * kPagesPiece + kPagesScaleSets * 8 * kPageBlock;
constexpr int kPagesSplitSmem(int B) { return kPagesWarps * kPagesWarpBytes + (B + 1) * 4; }
static_assert(kPagesSplitSmem(kPagesMostBatch) + 4096 <= 232448, "shared memory");
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
__device__ __forceinline__ void pages_depth(const PagesDecodeParams& p, int b, int r, float (*s_w)[8], float* out, int lane) {
    constexpr int FPL = D / 32, SLOTS = 32;
    const int g = lane >> 2, t = lane & 3;
    const int heads = p.Hk / p.kv_rep;
    const size_t stride = size_t(p.B) * heads * 2 * D;               // elements between depth slots
    const __nv_bfloat16* depth0 = p.depth + (size_t(b) * heads + r / p.kv_rep) * 2 * D;
    uint4 q[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        q[i] = make_uint4(0u, 0u, 0u, 0u);
        if (g < p.G) q[i] = *reinterpret_cast<const uint4*>(p.q + (size_t(b) * p.H + r * p.G + g) * D + 32 * i + 8 * t);
    }
    float m = -INFINITY, sum = 0.f, acc[8][FPL];
#pragma unroll
    for (int h = 0; h < 8; ++h)
#pragma unroll
        for (int c = 0; c < FPL; ++c) acc[h][c] = 0.f;
#pragma unroll 1
    for (int i0 = 0; i0 < p.l; i0 += SLOTS) {
        const int n_slot = min(p.l - i0, SLOTS);
        float s[4][2];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            float c[4] = {0.f, 0.f, 0.f, 0.f};
            if (8 * n < n_slot) {
                const uint4* row = reinterpret_cast<const uint4*>(depth0 + size_t(i0 + min(8 * n + g, n_slot - 1)) * stride);
                uint4 k[D / 32];
#pragma unroll
                for (int i = 0; i < D / 32; ++i) k[i] = row[4 * i + t];
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    mma_bf16_16x8x16(c, q[i].x, 0u, q[i].y, 0u, k[i].x, k[i].y);
                    mma_bf16_16x8x16(c, q[i].z, 0u, q[i].w, 0u, k[i].z, k[i].w);
                }
            }
            s[n][0] = 8 * n + 2 * t < n_slot ? c[0] * p.scale_log2 : -INFINITY;
            s[n][1] = 8 * n + 2 * t + 1 < n_slot ? c[1] * p.scale_log2 : -INFINITY;
        }
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
#pragma unroll 8
        for (int i = 0; i < n_slot; ++i) {
            const __nv_bfloat16* row = depth0 + size_t(i0 + i) * stride + D + lane * FPL;
            float v[FPL];
            if constexpr (FPL == 4) {
                const uint2 x = *reinterpret_cast<const uint2*>(row);
                v[0] = bf16_lo_to_f32(x.x); v[1] = bf16_hi_to_f32(x.x); v[2] = bf16_lo_to_f32(x.y); v[3] = bf16_hi_to_f32(x.y);
            } else {
                const uint32_t x = *reinterpret_cast<const uint32_t*>(row);
                v[0] = bf16_lo_to_f32(x); v[1] = bf16_hi_to_f32(x);
            }
            const float4 w0 = *reinterpret_cast<const float4*>(&s_w[i][0]), w1 = *reinterpret_cast<const float4*>(&s_w[i][4]);
            const float w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
            for (int h = 0; h < 8; ++h)
#pragma unroll
                for (int c = 0; c < FPL; ++c) acc[h][c] = fmaf(w[h], v[c], acc[h][c]);
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
__global__ void __launch_bounds__(kPagesSplitThreads, 1)
pages_split_kernel(const PagesDecodeParams p) {
    constexpr int NW = kPagesWarps;
    constexpr int KP = D / 64, FB = D / 16;                          // 64-feature parts of keys and values; 16-feature rows of the value product
    constexpr int AHEAD = kPagesPieces / (2 * KP);                   // units that the ring is ahead
    extern __shared__ __align__(16) uint8_t split_smem[];
    int* s_before = reinterpret_cast<int*>(split_smem + NW * kPagesWarpBytes);      // [B + 1]
    __shared__ int s_sum[NW];
    __shared__ __align__(16) float s_w[kPagesDepthWarps][32][8];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;
    if (p.index) grid_dependency_wait();                             // launched beside what comes before it in the stream
    if (warp >= NW) {
        // ---- two warps for the depth pairs ----
        const int groups = p.l > 0 ? p.B * p.Hk : 0;
        for (int i = (warp - NW) * gridDim.x + blockIdx.x; i < groups; i += kPagesDepthWarps * gridDim.x)
            pages_depth<D>(p, i / p.Hk, i % p.Hk, s_w[warp - NW], p.part + (size_t(p.warps) + size_t(p.B) * p.Hk + i) * p.G * (D + 2), lane);
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
    const long long total = (long long)s_before[p.B] * p.Hk, runs = min(total, (long long)p.warps);
    const int w = warp * gridDim.x + blockIdx.x;                     // neighbours in the order are on different SMs
    if (w >= runs) return;
    const int first = int(total * w / runs), n_unit = int(total * (w + 1) / runs) - first;

    // ---- the ring: pieces (64 features of a unit's keys, then of its values) in order, three on their way while one is worked on ----
    uint8_t* ring = split_smem + warp * kPagesWarpBytes;
    const uint32_t ring_u32 = smem_u32(ring);
    float* scales = reinterpret_cast<float*>(ring + kPagesPieces * kPagesPiece);    // [kPagesScaleSets][128], of consecutive units
    PagesWalk ahead;                                                 // the unit that is looked up next
    ahead.begin(s_before, p.B, p.Hk, first);
    PagesWalk at = ahead;                                            // the one in work
    int left = n_unit;                                               // units not yet looked up
    struct Place { const uint8_t* rec; int rows; };                  // where a unit lies (null: nowhere), its keys
    auto block_of = [&]() -> int {
        return p.index ? p.index[(size_t(ahead.b) * (p.Hk / p.kv_rep) + ahead.r / p.kv_rep) * p.n_index + ahead.j] : ahead.j;
    };
    auto look_up = [&](int blk) -> Place {
        const int len = p.len(ahead.b);
        const int tile = blk >= 0 && blk < pages_blocks(len) ? p.tile(ahead.b, blk) : -1;
        Place x;
        x.rec = tile >= 0 ? p.pages + (size_t(tile) * (p.Hk / p.kv_rep) + ahead.r / p.kv_rep) * page_block_bytes(D) : nullptr;
        x.rows = tile >= 0 ? min(len - blk * kPageBlock, kPageBlock) : 0;
        if (--left > 0) ahead.next(s_before, p.Hk);
        return x;
    };
    // Piece `i` of a unit (0 .. KP - 1: keys, then values) into its slot of the ring.
    auto request = [&](const uint8_t* rec, int unit, int i) {
        if (rec) {
            const uint32_t dst = ring_u32 + (unit % AHEAD * 2 * KP + i) * kPagesPiece + lane * 16;
            if (i < KP) {
                const uint8_t* src = rec + (lane >> 2) * D + 64 * i + 16 * (lane & 3);
#pragma unroll
                for (int k = 0; k < 8; ++k) cp_async_16(dst + k * 512, src + k * 8 * D);
                if (i == 0) cp_async_16(smem_u32(scales) + unit % kPagesScaleSets * 512 + lane * 16, rec + 2 * kPageBlock * D + lane * 16);
            } else {
                const uint8_t* src = rec + kPageBlock * D + (i - KP) * kPagesPiece + lane * 16;
#pragma unroll
                for (int k = 0; k < 8; ++k) cp_async_16(dst + k * 512, src + k * 512);
            }
        }
        cp_async_commit();
    };
    Place place[AHEAD + 1];                                          // of units u .. u + AHEAD
#pragma unroll
    for (int i = 0; i <= AHEAD; ++i) {
        place[i] = left > 0 ? look_up(block_of()) : Place{nullptr, 0};
        if (i < AHEAD)
#pragma unroll
            for (int k = 0; k < 2 * KP; ++k) request(place[i].rec, i, k);
    }

    uint32_t qf[KP][8];                                              // this lane's features of head g, f16
    float q_scale;                                                   // their power of two, times scale log2(e)
    auto load_q = [&]() {
        uint4 v[KP][2];
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            v[i][0] = v[i][1] = make_uint4(0u, 0u, 0u, 0u);
            if (g < p.G) {
                const uint4* src = reinterpret_cast<const uint4*>(p.q + (size_t(at.b) * p.H + at.r * p.G + g) * D + 64 * i + 16 * t);
                v[i][0] = src[0];
                v[i][1] = src[1];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t words[4] = {v[i][k].x, v[i][k].y, v[i][k].z, v[i][k].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) most = fmaxf(most, fmaxf(fabsf(bf16_lo_to_f32(words[j])), fabsf(bf16_hi_to_f32(words[j]))));
            }
        }
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int e = max(int(__float_as_uint(most) >> 23), 20) - 127;          // most < 2^(e + 1): times 2^(14 - e), below 2^15
        const float up = __uint_as_float(uint32_t(127 + 14 - e) << 23);
        q_scale = p.scale_log2 * __uint_as_float(uint32_t(127 - 14 + e) << 23);
#pragma unroll
        for (int i = 0; i < KP; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t words[4] = {v[i][k].x, v[i][k].y, v[i][k].z, v[i][k].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) qf[i][4 * k + j] = pack_f16x2(bf16_lo_to_f32(words[j]) * up, bf16_hi_to_f32(words[j]) * up);
            }
    };
    load_q();

    float m = -INFINITY, mw = -INFINITY, sum = 0.f;                  // of head g: maxima of the scores and of the weights' exponents, row sum (this lane's keys)
    float o[FB][4];                                                  // features 16 f + g (c0 c1) and + 8 (c2 c3) of heads 2 t, 2 t + 1
#pragma unroll
    for (int f = 0; f < FB; ++f) { o[f][0] = 0.f; o[f][1] = 0.f; o[f][2] = 0.f; o[f][3] = 0.f; }
#pragma unroll 1
    for (int u = 0; u < n_unit; ++u) {
        const int rows = place[0].rows;
        const uint8_t* then = place[AHEAD].rec;                      // of unit u + AHEAD
        const int blk = left > 0 ? block_of() : 0;                   // of the one behind it
        const uint8_t* mine = ring + u % AHEAD * 2 * KP * kPagesPiece;
        float* own = scales + u % kPagesScaleSets * 128;
        float c[8][4];                                               // eight products side by side: each waits for the one before it in its sum
#pragma unroll
        for (int n = 0; n < 8; ++n) { c[n][0] = 0.f; c[n][1] = 0.f; c[n][2] = 0.f; c[n][3] = 0.f; }
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            cp_async_wait<kPagesPieces - 1>();
            __syncwarp();
            if (rows > 0) {
                if (i == 0) {
                    const float2 v = *reinterpret_cast<const float2*>(own + kPageBlock + 2 * lane);
                    *reinterpret_cast<float2*>(own + kPageBlock + 2 * lane) = make_float2(__log2f(v.x), __log2f(v.y));
                }
#pragma unroll
                for (int n0 = 0; n0 < 8; n0 += 4) {
                    uint4 x[4];
#pragma unroll
                    for (int n = 0; n < 4; ++n) x[n] = *reinterpret_cast<const uint4*>(mine + i * kPagesPiece + (16 * (g >> 1) + 2 * (n0 + n) + (g & 1)) * 64 + 16 * t);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            uint32_t b0, b1;
                            e4m3x4_to_f16(k == 0 ? x[n].x : k == 1 ? x[n].y : k == 2 ? x[n].z : x[n].w, b0, b1);
                            mma_f16_16x8x16(c[n0 + n], qf[i][2 * k], 0u, qf[i][2 * k + 1], 0u, b0, b1);
                        }
                }
            }
            __syncwarp();                                            // everyone has read the piece; the logarithms are there
            request(then, u + AHEAD, i);
        }
        uint32_t pw[8];                                              // weights of keys 16 t + 2 n, + 1
        if (rows > 0) {
            float s[8][2], x[8][2];                                  // scores over q_scale; log2 of the values' scales, then the weights' exponents
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 a = *reinterpret_cast<const float4*>(own + 16 * t + 4 * i);
                const float4 y = *reinterpret_cast<const float4*>(own + kPageBlock + 16 * t + 4 * i);
                s[2 * i][0] = c[2 * i][0] * a.x; s[2 * i][1] = c[2 * i][1] * a.y;
                s[2 * i + 1][0] = c[2 * i + 1][0] * a.z; s[2 * i + 1][1] = c[2 * i + 1][1] * a.w;
                x[2 * i][0] = y.x; x[2 * i][1] = y.y; x[2 * i + 1][0] = y.z; x[2 * i + 1][1] = y.w;
            }
            if (rows < kPageBlock) {                                 // what lies past the last key may hold anything
#pragma unroll
                for (int n = 0; n < 8; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        if (16 * t + 2 * n + i >= rows) { s[n][i] = -INFINITY; x[n][i] = 0.f; }
            }
            float mx = -INFINITY, mxw = -INFINITY;
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    s[n][i] *= q_scale;
                    x[n][i] += s[n][i];
                    mx = fmaxf(mx, s[n][i]);
                    mxw = fmaxf(mxw, x[n][i]);
                }
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mxw = fmaxf(mxw, __shfl_xor_sync(0xffffffffu, mxw, 1));
            mx = fmaxf(m, fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)));
            mxw = fmaxf(mw, fmaxf(mxw, __shfl_xor_sync(0xffffffffu, mxw, 2)));
            const float base = mx == -INFINITY ? 0.f : mx, alpha = fast_exp2(m - base);
            const float base_w = mxw == -INFINITY ? 0.f : mxw - 14.f, alpha_w = fast_exp2(mw - mxw);
            float part = 0.f;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                part += fast_exp2(s[n][0] - base) + fast_exp2(s[n][1] - base);
                pw[n] = pack_f16x2(fast_exp2(x[n][0] - base_w), fast_exp2(x[n][1] - base_w));
            }
            sum = sum * alpha + part;
            const bool moved = mw != mxw && mw != -INFINITY;
            m = mx;
            mw = mxw;
            if (__any_sync(0xffffffffu, moved)) {
                const float f = moved ? alpha_w : 1.f;
                const float a0 = __shfl_sync(0xffffffffu, f, 8 * t), a1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
#pragma unroll
                for (int i = 0; i < FB; ++i) { o[i][0] *= a0; o[i][1] *= a1; o[i][2] *= a0; o[i][3] *= a1; }
            }
        }
        const bool leaves = u + 1 < n_unit && at.j + 1 == at.n;
        Place behind = left > 0 ? look_up(blk) : Place{nullptr, 0};
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            cp_async_wait<kPagesPieces - 1>();
            __syncwarp();
            uint8_t* sv = ring + (u % AHEAD * 2 * KP + KP + i) * kPagesPiece;
            if (rows > 0) {
                if (rows < kPageBlock) {                             // value codes past the last key: zero, their weights are 0
                    for (int e = lane; e < kPagesPiece / 16; e += 32) {
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
                uint4 x[4], y[4];
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    x[f] = *reinterpret_cast<const uint4*>(sv + (16 * f + g) * kPageBlock + 16 * t);
                    y[f] = *reinterpret_cast<const uint4*>(sv + (16 * f + 8 + g) * kPageBlock + 16 * t);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        uint32_t a0, a1, a2, a3;
                        e4m3x4_to_f16(k == 0 ? x[f].x : k == 1 ? x[f].y : k == 2 ? x[f].z : x[f].w, a0, a2);
                        e4m3x4_to_f16(k == 0 ? y[f].x : k == 1 ? y[f].y : k == 2 ? y[f].z : y[f].w, a1, a3);
                        mma_f16_16x8x16(o[4 * i + f], a0, a1, a2, a3, pw[2 * k], pw[2 * k + 1]);
                    }
            }
            __syncwarp();                                            // everyone has read the piece
            request(then, u + AHEAD, KP + i);
        }
        if (u + AHEAD + 1 >= n_unit) grid_launch_dependents();       // all loads are on their way: the merge may come up
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) place[i] = place[i + 1];
        place[AHEAD] = behind;
        if (leaves || u + 1 == n_unit) {
            // ---- the group's partial result of this warp ----
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            float* out = p.part + (size_t(w) + size_t(at.b) * p.Hk + at.r) * p.G * (D + 2);
            // the weighted sums are relative to 2^(mw - 14), the row sum to 2^m
            const float f = mw == -INFINITY ? 0.f : fast_exp2(mw - 14.f - m);
            const float a0 = __shfl_sync(0xffffffffu, f, 8 * t), a1 = __shfl_sync(0xffffffffu, f, 8 * t + 4);
            if (t == 0 && g < p.G) *reinterpret_cast<float2*>(out + g * (D + 2)) = make_float2(m, sum);
#pragma unroll
            for (int i = 0; i < FB; ++i) {
                if (2 * t < p.G) {
                    out[2 * t * (D + 2) + 2 + 16 * i + g] = o[i][0] * a0;
                    out[2 * t * (D + 2) + 2 + 16 * i + 8 + g] = o[i][2] * a0;
                }
                if (2 * t + 1 < p.G) {
                    out[(2 * t + 1) * (D + 2) + 2 + 16 * i + g] = o[i][1] * a1;
                    out[(2 * t + 1) * (D + 2) + 2 + 16 * i + 8 + g] = o[i][3] * a1;
                }
                o[i][0] = 0.f; o[i][1] = 0.f; o[i][2] = 0.f; o[i][3] = 0.f;
            }
            m = mw = -INFINITY;
            sum = 0.f;
        }
        if (u + 1 < n_unit) {
            at.next(s_before, p.Hk);
            if (leaves) load_q();
        }
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
    const long long total = (long long)all * p.Hk, first = (long long)before * p.Hk + (long long)r * own;
    // warp of a unit: the one whose run holds it
    const long long runs = min(total, (long long)p.warps);
    const int w0 = own > 0 ? int(((first + 1) * runs - 1) / total) : 0, w1 = own > 0 ? int(((first + own) * runs - 1) / total) : -1;
    const int S = w1 - w0 + 1, n = S + (p.l > 0 ? 1 : 0);            // the last one is that of the depth pairs
    const size_t stride = size_t(p.G) * (D + 2), group = size_t(b) * p.Hk + r;
    const float* part = p.part + (size_t(w0) + group) * stride + g * (D + 2);
    const float* depth = p.part + (size_t(p.warps) + size_t(p.B) * p.Hk + group) * stride + g * (D + 2);
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
            const float f = fast_exp2(ml[u].x - base);               // 0 for a partial without keys, whose sums are 0 or NaN
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
