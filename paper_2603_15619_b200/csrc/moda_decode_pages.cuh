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

constexpr int kPagesMostBatch = 4096;                                // sequences of a call: their blocks are counted in shared memory
constexpr int kPagesMergeThreads = 128;
constexpr int kPagesDecodeWarps(int d) { return d == 64 ? 16 : 8; }  // of a CTA, one an SM
constexpr int kPagesPieces = 3;                                      // key or value halves of blocks that a warp has in shared memory or on the way
constexpr int kPagesWarpBytes(int d) { return kPagesPieces * kPageBlock * d + 2 * 8 * kPageBlock; }
constexpr int kPagesSplitSmem(int d, int B) { return kPagesDecodeWarps(d) * kPagesWarpBytes(d) + (B + 1) * 4; }
static_assert(kPagesSplitSmem(128, kPagesMostBatch) <= 226 * 1024 && kPagesSplitSmem(64, kPagesMostBatch) <= 226 * 1024, "shared memory");

__device__ __forceinline__ void mma_f16_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
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

template <int D>
__global__ void __launch_bounds__(kPagesDecodeWarps(D) * 32, 1)
pages_split_kernel(const PagesDecodeParams p) {
    constexpr int NW = kPagesDecodeWarps(D), NT = NW * 32;
    constexpr int KP = D / 64, FB = D / 16;                          // 64-feature parts of a key row; 16-feature rows of the value product
    constexpr int PIECE = kPageBlock * D, CH = D / 16;               // bytes of a block's key or value codes; 16-byte pieces of a key row
    extern __shared__ __align__(16) uint8_t split_smem[];
    int* s_before = reinterpret_cast<int*>(split_smem + NW * kPagesWarpBytes(D));   // [B + 1]
    __shared__ int s_sum[NW];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, t = lane & 3;
    if (p.index) grid_dependency_wait();                             // launched beside what comes before it in the stream
    // ---- blocks of the sequences before each ----
    {
        const int per = (p.B + NT - 1) / NT;
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
        __syncthreads();
        int at = incl - sum;
        for (int w = 0; w < warp; ++w) at += s_sum[w];
        for (int b = b0; b < b1; ++b) {
            s_before[b] = at;
            at += p.units(b);
        }
        if (b0 < b1 && b1 == p.B) s_before[p.B] = at;
        __syncthreads();
        if (blockIdx.x == 0)
            for (int b = tid; b <= p.B; b += NT) p.before[b] = s_before[b];
    }
    const long long total = (long long)s_before[p.B] * p.Hk, runs = min(total, (long long)p.warps);
    const int w = warp * gridDim.x + blockIdx.x;                     // neighbours in the order are on different SMs
    if (w >= runs) return;
    const int first = int(total * w / runs), n_unit = int(total * (w + 1) / runs) - first;

    // ---- the ring: pieces (keys of a unit, then its values) in order, the next two on their way while one is worked on ----
    const uint8_t* ring = split_smem + warp * kPagesWarpBytes(D);
    const uint32_t ring_u32 = smem_u32(ring);
    float* scales = reinterpret_cast<float*>(split_smem + warp * kPagesWarpBytes(D) + kPagesPieces * PIECE);   // [2][128], of even and odd units
    PagesWalk ahead;                                                 // the unit whose pieces are requested next
    ahead.begin(s_before, p.B, p.Hk, first);
    PagesWalk at = ahead;                                            // the one in work
    int left = n_unit;                                               // units not yet looked up
    // Block of a unit, and where it lies (null: nowhere).
    struct Place { const uint8_t* rec; int rows; };
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
    // 16-byte piece c of key row r lies at c ^ 4 (r % 2) where a row has 8, so that two adjacent rows of four lanes each are in different banks.
    auto request_k = [&](const uint8_t* rec, int piece, int unit) {
        if (rec) {
            const uint32_t dst = ring_u32 + (piece % kPagesPieces) * PIECE;
#pragma unroll
            for (int i = 0; i < PIECE / 512; ++i) {
                const int e = i * 32 + lane, r = e / CH, c = e % CH;
                cp_async_16(dst + r * D + 16 * (D == 128 ? c ^ ((r & 1) << 2) : c), rec + e * 16);
            }
            cp_async_16(smem_u32(scales) + (unit & 1) * 512 + lane * 16, rec + 2 * PIECE + lane * 16);
        }
        cp_async_commit();
    };
    auto request_v = [&](const uint8_t* rec, int piece) {
        if (rec) {
            const uint32_t dst = ring_u32 + (piece % kPagesPieces) * PIECE;
#pragma unroll
            for (int i = 0; i < PIECE / 512; ++i) cp_async_16(dst + (i * 32 + lane) * 16, rec + PIECE + (i * 32 + lane) * 16);
        }
        cp_async_commit();
    };
    Place here = look_up(block_of()), next = {nullptr, 0};
    request_k(here.rec, 0, 0);
    request_v(here.rec, 1);
    if (n_unit > 1) next = look_up(block_of());
    request_k(next.rec, 2, 1);

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
        const int rows = here.rows;
        const int ahead_blk = left > 0 ? block_of() : 0;             // of unit u + 2
        if (u + 1 == n_unit) grid_launch_dependents();               // all loads are on their way: the merge may come up
        cp_async_wait<2>();
        __syncwarp();
        const uint8_t* sk = ring + (2 * u % kPagesPieces) * PIECE;
        const uint8_t* sv = ring + ((2 * u + 1) % kPagesPieces) * PIECE;
        float* own = scales + (u & 1) * 128;
        uint32_t pw[8];                                              // weights of keys 16 t + 2 n, + 1
        if (rows > 0) {
            const float2 v = *reinterpret_cast<const float2*>(own + kPageBlock + 2 * lane);
            *reinterpret_cast<float2*>(own + kPageBlock + 2 * lane) = make_float2(__log2f(v.x), __log2f(v.y));
            float s[8][2];
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KP; ++i) {
                    const uint4 x = *reinterpret_cast<const uint4*>(sk + (16 * (g >> 1) + 2 * n + (g & 1)) * D + 16 * (D == 128 ? (4 * i + t) ^ ((g & 1) << 2) : t));
                    const uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t b0, b1;
                        e4m3x4_to_f16(word[k], b0, b1);
                        mma_f16_16x8x16(c, qf[i][2 * k], 0u, qf[i][2 * k + 1], 0u, b0, b1);
                    }
                }
                s[n][0] = c[0];
                s[n][1] = c[1];
            }
            __syncwarp();                                            // everyone has read the keys; the logarithms are there
            request_v(next.rec, 2 * u + 3);
            float x[8][2];                                           // log2 of the values' scales, then the weights' exponents
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 a = *reinterpret_cast<const float4*>(own + 16 * t + 4 * i);
                const float4 c = *reinterpret_cast<const float4*>(own + kPageBlock + 16 * t + 4 * i);
                s[2 * i][0] *= a.x * q_scale; s[2 * i][1] *= a.y * q_scale;
                s[2 * i + 1][0] *= a.z * q_scale; s[2 * i + 1][1] *= a.w * q_scale;
                x[2 * i][0] = c.x; x[2 * i][1] = c.y; x[2 * i + 1][0] = c.z; x[2 * i + 1][1] = c.w;
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
        } else {
            request_v(next.rec, 2 * u + 3);
        }
        const bool leaves = u + 1 < n_unit && at.j + 1 == at.n;
        const Place then = left > 0 ? look_up(ahead_blk) : Place{nullptr, 0};
        cp_async_wait<2>();
        __syncwarp();
        if (rows > 0) {
            if (rows < kPageBlock) {                                 // value codes past the last key: zero, their weights are 0
                for (int e = lane; e < D * 4; e += 32) {
                    uint4* c = reinterpret_cast<uint4*>(const_cast<uint8_t*>(sv)) + e;
                    uint32_t word[4] = {c->x, c->y, c->z, c->w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int some = min(max(rows - 16 * (e & 3) - 4 * k, 0), 4);
                        word[k] = some == 4 ? word[k] : word[k] & ((1u << (8 * some)) - 1u);
                    }
                    *c = make_uint4(word[0], word[1], word[2], word[3]);
                }
                __syncwarp();
            }
#pragma unroll
            for (int f = 0; f < FB; ++f) {
                const uint4 v0 = *reinterpret_cast<const uint4*>(sv + (16 * f + g) * kPageBlock + 16 * t);
                const uint4 v1 = *reinterpret_cast<const uint4*>(sv + (16 * f + 8 + g) * kPageBlock + 16 * t);
                const uint32_t x[4] = {v0.x, v0.y, v0.z, v0.w}, y[4] = {v1.x, v1.y, v1.z, v1.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t a0, a1, a2, a3;
                    e4m3x4_to_f16(x[k], a0, a2);
                    e4m3x4_to_f16(y[k], a1, a3);
                    mma_f16_16x8x16(o[f], a0, a1, a2, a3, pw[2 * k], pw[2 * k + 1]);
                }
            }
        }
        __syncwarp();                                                // everyone has read the values (and the scales)
        request_k(then.rec, 2 * u + 4, u);
        here = next;
        next = then;
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

// One CTA of four warps per (query head, sequence); lanes hold D / 32 adjacent features, a warp takes every fourth depth slot and every fourth partial.  A
// token without any key has O = 0 and LSE = -inf.
template <int D>
__global__ void __launch_bounds__(kPagesMergeThreads)
pages_merge_kernel(const PagesDecodeParams p) {
    constexpr int FPL = D / 32, NW = kPagesMergeThreads / 32, UN = 4;
    __shared__ float s_d[256], s_red[NW], s_sum[NW];                 // depth scores (log2 domain), then weights; l <= 256
    __shared__ int s_units[3];                                       // blocks before this sequence, its own, all
    __shared__ __align__(16) float s_acc[NW][D];
    const int h = blockIdx.x, b = blockIdx.y;
    const int r = h / p.G, g = h - r * p.G;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    auto load_row = [&](const __nv_bfloat16* row, float (&x)[FPL]) {
        if constexpr (FPL == 4) {
            const uint2 v = *reinterpret_cast<const uint2*>(row + lane * 4);
            x[0] = bf16_lo_to_f32(v.x); x[1] = bf16_hi_to_f32(v.x); x[2] = bf16_lo_to_f32(v.y); x[3] = bf16_hi_to_f32(v.y);
        } else {
            const uint32_t v = *reinterpret_cast<const uint32_t*>(row + lane * 2);
            x[0] = bf16_lo_to_f32(v); x[1] = bf16_hi_to_f32(v);
        }
    };
    float q[FPL];
    load_row(p.q + (size_t(b) * p.H + h) * D, q);
#pragma unroll
    for (int c = 0; c < FPL; ++c) q[c] *= p.scale_log2;
    const int heads = p.Hk / p.kv_rep;
    const size_t slot_stride = size_t(p.B) * heads * 2 * D;          // elements between depth slots
    const __nv_bfloat16* depth0 = p.depth + (size_t(b) * heads + r / p.kv_rep) * 2 * D;
    float mx = -INFINITY;
    for (int i0 = warp; i0 < p.l; i0 += NW * UN) {
        float kd[UN][FPL];
#pragma unroll
        for (int u = 0; u < UN; ++u) load_row(depth0 + size_t(min(i0 + u * NW, p.l - 1)) * slot_stride, kd[u]);
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            float a = 0.f;
#pragma unroll
            for (int c = 0; c < FPL; ++c) a = fmaf(q[c], kd[u][c], a);
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) a += __shfl_xor_sync(0xffffffffu, a, off);
            mx = fmaxf(mx, a);
            if (lane == 0 && i0 + u * NW < p.l) s_d[i0 + u * NW] = a;
        }
    }
    if (p.B <= kPagesMergeThreads) {                                 // a thread per sequence
        const int v = tid < p.B ? p.units(tid) : 0;
        const int all = __reduce_add_sync(0xffffffffu, v), below = __reduce_add_sync(0xffffffffu, tid < b ? v : 0);
        if (tid == b) s_units[1] = v;
        if (lane == 0) { s_acc[warp][0] = __int_as_float(all); s_acc[warp][1] = __int_as_float(below); }
        __syncthreads();
        if (tid == 0) {
            int x = 0, y = 0;
#pragma unroll
            for (int i = 0; i < NW; ++i) { x += __float_as_int(s_acc[i][0]); y += __float_as_int(s_acc[i][1]); }
            s_units[0] = y;
            s_units[2] = x;
        }
    }
    // ---- from here on: what the split kernel wrote ----
    grid_dependency_wait();
    if (p.B > kPagesMergeThreads && tid == 0) {
        s_units[0] = __ldcg(p.before + b);
        s_units[1] = __ldcg(p.before + b + 1) - s_units[0];
        s_units[2] = __ldcg(p.before + p.B);
    }
    __syncthreads();
    const int own = s_units[1];
    const long long total = (long long)s_units[2] * p.Hk, first = (long long)s_units[0] * p.Hk + (long long)r * own;
    // warp of a unit: the one whose run holds it
    const long long runs = min(total, (long long)p.warps);
    const int w0 = own > 0 ? int(((first + 1) * runs - 1) / total) : 0, w1 = own > 0 ? int(((first + own) * runs - 1) / total) : -1;
    const int S = w1 - w0 + 1;
    const float* part = p.part + (size_t(w0) + size_t(b) * p.Hk + r) * p.G * (D + 2) + g * (D + 2);
    const size_t stride = size_t(p.G) * (D + 2);
    // ---- an online softmax over the warp's partials, then over its depth slots ----
    float m = -INFINITY, lt = 0.f, acc[FPL];
#pragma unroll
    for (int c = 0; c < FPL; ++c) acc[c] = 0.f;
    for (int s0 = warp; s0 < S; s0 += NW * UN) {
        float2 ml[UN];
        float x[UN][FPL];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const float* src = part + size_t(min(s0 + u * NW, S - 1)) * stride;
            ml[u] = __ldcg(reinterpret_cast<const float2*>(src));
#pragma unroll
            for (int c = 0; c < FPL; c += 2) {
                const float2 v = __ldcg(reinterpret_cast<const float2*>(src + 2 + lane * FPL + c));
                x[u][c] = v.x; x[u][c + 1] = v.y;
            }
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            if (s0 + u * NW >= S) ml[u] = make_float2(-INFINITY, 0.f);
            top = fmaxf(top, ml[u].x);
        }
        const float base = top == -INFINITY ? 0.f : top, alpha = fast_exp2(m - base);
        m = top;
        lt *= alpha;
#pragma unroll
        for (int c = 0; c < FPL; ++c) acc[c] *= alpha;
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const float f = ml[u].x == -INFINITY && !(ml[u].y != ml[u].y) ? 0.f : fast_exp2(ml[u].x - base);
            if (s0 + u * NW < S) {
                lt = fmaf(f, ml[u].y, lt);
#pragma unroll
                for (int c = 0; c < FPL; ++c) acc[c] = fmaf(f, x[u][c], acc[c]);
            }
        }
    }
    {
        const float top = fmaxf(m, mx), base = top == -INFINITY ? 0.f : top, alpha = fast_exp2(m - base);
        m = top;
        lt *= alpha;
#pragma unroll
        for (int c = 0; c < FPL; ++c) acc[c] *= alpha;
        for (int i0 = warp; i0 < p.l; i0 += NW * UN) {
            float vd[UN][FPL];
#pragma unroll
            for (int u = 0; u < UN; ++u) load_row(depth0 + size_t(min(i0 + u * NW, p.l - 1)) * slot_stride + D, vd[u]);
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                if (i0 + u * NW >= p.l) continue;
                const float f = fast_exp2(s_d[i0 + u * NW] - base);   // of this warp's own slots
                lt += f;
#pragma unroll
                for (int c = 0; c < FPL; ++c) acc[c] = fmaf(f, vd[u][c], acc[c]);
            }
        }
    }
    // ---- the four warps ----
    if (lane == 0) { s_red[warp] = m; s_sum[warp] = lt; }
#pragma unroll
    for (int c = 0; c < FPL; ++c) s_acc[warp][lane * FPL + c] = acc[c];
    __syncthreads();
    float top = s_red[0];
#pragma unroll
    for (int i = 1; i < NW; ++i) top = fmaxf(top, s_red[i]);
    const float base = top == -INFINITY ? 0.f : top;
    float all = 0.f, a = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const float f = fast_exp2(s_red[i] - base);
        all = fmaf(f, s_sum[i], all);
        if (tid < D) a = fmaf(f, s_acc[i][tid], a);
    }
    if (tid < D) p.O[(size_t(b) * p.H + h) * D + tid] = __float2bfloat16(all == 0.f ? 0.f : a / all);
    if (tid == 0) p.LSE[size_t(b) * p.H + h] = all == 0.f ? -INFINITY : (top + log2f(all)) * 0.6931471805599453f;
}

}  // namespace moda
