// The paged sequence cache in 8 bits: its layout, the kernels that write and read it, and the selection of the blocks that a token attends to.
//
// A block is 64 positions; a page has page_size / 64 of them.  Of every (block, key/value head):
//
//   pages   [page][block of the page][Hk] { key codes [64][d], value codes [d][64], key scales [64] fp32, value scales [64] fp32 }
//   bounds  [page][block of the page][Hk] { largest [d] int8, smallest [d] int8, scale fp32, 12 bytes that nothing reads }
//
// Codes are e4m3 by the depth cache's rule (moda_cache.cuh): scale = max|x| / 448 of a row, 1 for a row of zeros, code = e4m3(x / scale).  Keys lie row by
// row and values feature by feature, so that a lane of the decode step (moda_decode_pages.cuh) has its operands of a matrix product in 16 adjacent bytes
// of either and nothing is turned on the way.  The bounds of a block are those of its first keys, up to the sequence's end at the last write: largest and
// smallest dequantised value of each feature, over scale = max / 127, rounded outwards.  A block with a key that is not finite has codes 0 and scale inf.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "launch_rules.h"
#include "moda_cache.cuh"
#include "moda_evict.cuh"
#include "sm100_ptx.cuh"

namespace moda {

constexpr int kPageBlock = 64;
__host__ __device__ constexpr size_t page_block_bytes(int d) { return size_t(2 * kPageBlock) * d + 8 * kPageBlock; }
__host__ __device__ constexpr size_t page_bounds_bytes(int d) { return 2 * size_t(d) + 16; }

// What all calls over the pages have in common.
struct PagesParams {
    const int* table;             // [B][max_blocks]: page of every page_size positions of a sequence
    int B, Hk, sub, num_pages, max_blocks;   // sub: blocks of a page
    // Number of block `blk` of a sequence, over all pages; -1 where the table has no page for it.
    __device__ __forceinline__ int tile(int b, int blk) const {
        const int at = sub == 1 ? blk : blk / sub;
        const int page = at < max_blocks ? table[size_t(b) * max_blocks + at] : -1;
        return unsigned(page) < unsigned(num_pages) ? page * sub + (blk - at * sub) : -1;
    }
};

// Codes of 4 bytes as two pairs of f16 (exact).
__device__ __forceinline__ void e4m3x4_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n"
        ".reg .b16 a, b;\n"
        "mov.b32 {a, b}, %2;\n"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n"
        "cvt.rn.f16x2.e4m3x2 %1, b;\n"
        "}\n"
        : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ float2 f16x2_to_f32(uint32_t h) {
    float2 f;
    asm("{\n"
        ".reg .b16 a, b;\n"
        "mov.b32 {a, b}, %2;\n"
        "cvt.f32.f16 %0, a;\n"
        "cvt.f32.f16 %1, b;\n"
        "}\n"
        : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}
// Four words of four bytes, turned: byte j of a word i becomes byte i of word j.
__device__ __forceinline__ void turn4x4(uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
    const uint32_t ab0 = __byte_perm(a, b, 0x5140), ab1 = __byte_perm(a, b, 0x7362), cd0 = __byte_perm(c, d, 0x5140), cd1 = __byte_perm(c, d, 0x7362);
    a = __byte_perm(ab0, cd0, 0x5410);
    b = __byte_perm(ab0, cd0, 0x7632);
    c = __byte_perm(ab1, cd1, 0x5410);
    d = __byte_perm(ab1, cd1, 0x7632);
}

// Instructions that take two fp32 numbers in a 64-bit register (pair_f32), or three, for the write kernel, whose time went with the instructions that it issues.
__device__ __forceinline__ void unpair_f32(uint64_t x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma_f32x2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {           // NaN if one of them is
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t times_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// 16 features of a row that LANES adjacent lanes hold: their codes and the row's scale.  The depth cache's rule and bytes (but for the sign of a NaN), in fewer
// instructions: quotients two at a time, q = RN(x r) with r = RN(1 / d) corrected by its exact remainder (Markstein's theorem, as div_rn in moda_cache.cuh; a scale's
// significand, m / 7 of 128 <= m < 256, is never all ones); no element has a branch, as rows of which it would need one are brought into range first (exactly, by a power of
// two; or by 0, which makes of a row with an infinite element what the division by infinity would), and signs come from the input's words.
template <int LANES>
__device__ __forceinline__ uint4 quantise_row16(const uint4& lo, const uint4& hi, float& scale) {
    uint32_t w8[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    uint32_t most2 = w8[0], sign[4];                                 // largest magnitude of either half; NaN counts for nothing
#pragma unroll
    for (int k = 1; k < 8; ++k) asm("max.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(most2) : "r"(w8[k]));
#pragma unroll
    for (int k = 0; k < 4; ++k) sign[k] = __byte_perm(w8[2 * k], w8[2 * k + 1], 0x7531);
    float am = fmaxf(fabsf(bf16_lo_to_f32(most2)), fabsf(bf16_hi_to_f32(most2)));
    am = fmaxf(am, 0.f);                                             // 0 where all are NaN
#pragma unroll
    for (int off = 1; off < LANES; off <<= 1) am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, off));
    const float q0 = am * (1.f / 448.f);
    scale = fmaf(fmaf(-q0, 448.f, am), 1.f / 448.f, q0);
    float d = scale;
    constexpr float kTiny = 8.271806125530277e-25f;                  // 2^-80
    if (__any_sync(0xffffffffu, !(am >= kTiny && am < INFINITY))) {
        uint32_t factor = 0x3f803f80u;                               // 1
        if (!(am >= kTiny && am < INFINITY)) {
            scale = am > 0.f ? __fdiv_rn(am, 448.f) : 1.f;
            d = am == INFINITY ? 1.f : am > 0.f ? scale * 7.922816251426434e28f : 1.f;        // 2^96
            factor = am == INFINITY ? 0u : am > 0.f ? 0x6f806f80u : factor;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) w8[k] = times_bf16x2(w8[k], factor);
    }
    const float r = __frcp_rn(d);
    const uint64_t r2 = pair_f32(r, r), d2 = pair_f32(-d, -d);
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        uint32_t half[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint64_t x = pair_f32(bf16_lo_to_f32(w8[2 * k + i]), bf16_hi_to_f32(w8[2 * k + i])), q = mul_f32x2(x, r2);
            float a, b;
            unpair_f32(fma_f32x2(fma_f32x2(q, d2, x), r2, q), a, b);
            asm("{\n.reg .b16 t;\ncvt.rn.satfinite.e4m3x2.f32 t, %1, %2;\nmov.b32 %0, {t, 0};\n}\n" : "=r"(half[i]) : "f"(b), "f"(a));
        }
        w[k] = (__byte_perm(half[0], half[1], 0x5410) & 0x7f7f7f7fu) | (sign[k] & 0x80808080u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct PagesRowsParams : PagesParams {
    uint8_t* pages;
    uint8_t* bounds;              // may be null (and is for a read)
    const uint4* K;               // [B][T][Hk][d] bf16: rows that are written, or read into
    const uint4* V;
    const int* start;             // [B] position of a sequence's row 0, or null: 0
    const int* count;             // write: [B] rows that a sequence brings (0 .. T), or null: T.  read: [B] lengths of the sequences
    int T;
};

// Rows of block `blk` (blockIdx.x blocks behind the first one touched) that a call has to do with: [r0, r1), row r at position 64 blk + r, which is
// row `base` + r of the tensor.  False: none.
struct PagesRows { int blk, r0, r1, base; };
template <bool READ>
__device__ __forceinline__ bool pages_rows(const PagesRowsParams& p, int b, PagesRows& w) {
    const int cap = p.max_blocks * p.sub * kPageBlock;               // (fits: the host has seen to it)
    const int start = p.start ? min(max(p.start[b], 0), cap) : 0;
    int end = start + min(p.T, cap - start);
    if (READ) end = min(end, max(p.count[b], 0));
    else if (p.count) end = min(end, start + min(max(p.count[b], 0), cap - start));
    const unsigned blk = unsigned(start) / kPageBlock + blockIdx.x, p0 = blk * kPageBlock;   // below 2^32
    if (p0 >= unsigned(end)) return false;                           // (also where the sequence has no rows)
    w.blk = int(blk);
    w.r0 = max(start - int(p0), 0);
    w.r1 = min(end - int(p0), kPageBlock);
    w.base = int(p0) - start;
    return w.r0 < w.r1;
}

constexpr int kPagesThreads = 256;

// grid (blocks that T rows can touch, Hk, B): a CTA quantises the rows of one block of one head, and where `bounds` is given reads what the block's earlier
// keys left and writes the bounds anew.  It is the only one that writes the block (a page belongs to one sequence).
// 65536 rows of 8 heads, d = 128: 82 us, 5.0 TB/s (63.4 at the copy rate).  129 with a branch per element, 90.5 without, 83 with packed products
// and three-operand extremes; now 71 % of the issue slots and 53 % of DRAM's peak (profiler): the CTAs of an SM load, compute and store in turn.  A token of 64 sequences: 6.9 us, a chain of loads, quantisation, extremes and three barriers.
template <int D>
__global__ void __launch_bounds__(kPagesThreads)
pages_write_kernel(const PagesRowsParams p) {
    constexpr int CH = D / 8, LPR = D / 16, RPP = kPagesThreads / LPR, PASSES = kPageBlock / RPP;   // lanes of a row, rows at a time
    constexpr int KW = D / 4 + 4;                                    // words of a row of codes in shared memory, padded by 16 bytes
    constexpr int SETS = kPagesThreads / (D / 4);                    // threads that share four features of the bounds
    __shared__ __align__(16) uint32_t s_k[kPageBlock][KW], s_v[kPageBlock][KW];
    __shared__ __align__(16) float s_scale[kPageBlock], s_ext[2][SETS][D];   // largest and smallest of a set of rows
    __shared__ uint32_t s_most[kPagesThreads / 32];
    const int b = blockIdx.z, hk = blockIdx.y, tid = threadIdx.x;
    grid_dependency_wait();
    PagesRows w;
    if (!pages_rows<false>(p, b, w)) return;
    const int tile = p.tile(b, w.blk);
    if (tile < 0) return;
    uint8_t* rec = p.pages + (size_t(tile) * p.Hk + hk) * page_block_bytes(D);
    float* scales = reinterpret_cast<float*>(rec + 2 * kPageBlock * D);
    const int c = tid % LPR, row0 = tid / LPR;                       // 16 features; first row
    // the block's earlier keys
    if (p.bounds) {
        for (int e = tid; e < w.r0 * LPR; e += kPagesThreads)
            *reinterpret_cast<uint4*>(&s_k[e / LPR][4 * (e % LPR)]) = *reinterpret_cast<const uint4*>(rec + size_t(e) * 16);
        if (tid < w.r0) s_scale[tid] = scales[tid];
    }
    uint4 in[PASSES][2][2];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int row = row0 + i * RPP;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            in[i][kv][0] = in[i][kv][1] = make_uint4(0u, 0u, 0u, 0u);
            if (row >= w.r0 && row < w.r1) {
                const uint4* src = (kv ? p.V : p.K) + ((size_t(b) * p.T + (w.base + row)) * p.Hk + hk) * CH + 2 * c;
                in[i][kv][0] = src[0];
                in[i][kv][1] = src[1];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int row = row0 + i * RPP;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            float scale;
            const uint4 codes = quantise_row16<LPR>(in[i][kv][0], in[i][kv][1], scale);
            if (row >= w.r0 && row < w.r1) {
                *reinterpret_cast<uint4*>(kv ? &s_v[row][4 * c] : &s_k[row][4 * c]) = codes;
                if (kv == 0) *reinterpret_cast<uint4*>(rec + size_t(row) * D + 16 * c) = codes;
                if (c == 0) {
                    scales[kv * kPageBlock + row] = scale;
                    if (kv == 0) s_scale[row] = scale;
                }
            }
        }
    }
    __syncthreads();
    // values feature by feature: a thread turns 4 features of 16 positions
    for (int e = tid; e < D; e += kPagesThreads) {
        const int k0 = 16 * (e & 3), f = e >> 2;                     // first position; features 4 f .. 4 f + 3
        if (k0 + 16 <= w.r0 || k0 >= w.r1) continue;
        uint32_t t[4][4];                                            // [feature][positions 4 i ..]
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) t[j][i] = s_v[k0 + 4 * i + j][f];
            turn4x4(t[0][i], t[1][i], t[2][i], t[3][i]);
        }
        uint8_t* to = rec + kPageBlock * D + size_t(4 * f) * kPageBlock + k0;
        if (k0 >= w.r0 && k0 + 16 <= w.r1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4*>(to + j * kPageBlock) = make_uint4(t[j][0], t[j][1], t[j][2], t[j][3]);
        } else {                                                     // beside positions that stay as they are
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (k0 + k >= w.r0 && k0 + k < w.r1) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[j * kPageBlock + k] = uint8_t(t[j][k >> 2] >> (8 * (k & 3)));
                }
        }
    }
    if (!p.bounds) return;
    const int f = tid % (D / 4), set = tid / (D / 4);
    float hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) { hi[j] = -INFINITY; lo[j] = INFINITY; }
    for (int row = 2 * set; row < w.r1; row += 2 * SETS) {           // two rows at a time: the last one twice where it is alone
        const int other = min(row + 1, w.r1 - 1);
        uint32_t a0, a1, b0, b1;
        e4m3x4_to_f16(s_k[row][f], a0, a1);
        e4m3x4_to_f16(s_k[other][f], b0, b1);
        const float sa = s_scale[row], sb = s_scale[other];
        const uint64_t sa2 = pair_f32(sa, sa), sb2 = pair_f32(sb, sb);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float2 x = f16x2_to_f32(j ? a1 : a0), y = f16x2_to_f32(j ? b1 : b0);
            float x0, x1, y0, y1;
            unpair_f32(mul_f32x2(pair_f32(x.x, x.y), sa2), x0, x1);
            unpair_f32(mul_f32x2(pair_f32(y.x, y.y), sb2), y0, y1);
            hi[2 * j] = max3_nan(hi[2 * j], x0, y0);
            hi[2 * j + 1] = max3_nan(hi[2 * j + 1], x1, y1);
            lo[2 * j] = min3(lo[2 * j], x0, y0);
            lo[2 * j + 1] = min3(lo[2 * j + 1], x1, y1);
        }
    }
    *reinterpret_cast<float4*>(&s_ext[0][set][4 * f]) = make_float4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<float4*>(&s_ext[1][set][4 * f]) = make_float4(lo[0], lo[1], lo[2], lo[3]);
    __syncthreads();
    // a thread per feature for the largest, and one for the smallest
    const bool low = tid >= D;
    float x = 0.f;
    if (tid < 2 * D) {
        const float* of = &s_ext[low][0][low ? tid - D : tid];
        x = of[0];
#pragma unroll
        for (int s = 1; s + 1 < SETS; s += 2) x = low ? min3(x, of[s * D], of[(s + 1) * D]) : max3_nan(x, of[s * D], of[(s + 1) * D]);
        x = low ? fminf(x, of[(SETS - 1) * D]) : max3_nan(x, of[(SETS - 1) * D], x);
    }
    // bits of magnitudes are in the order of the numbers, and those of NaN are the largest
    const uint32_t most = __reduce_max_sync(0xffffffffu, __float_as_uint(x) & 0x7fffffffu);
    if (tid % 32 == 0) s_most[tid / 32] = most;
    __syncthreads();
    if (tid < 2 * D) {
        uint32_t all = s_most[0];
#pragma unroll
        for (int i = 1; i < 2 * D / 32; ++i) all = max(all, s_most[i]);
        const bool bad = all >= 0x7f800000u;
        const float scale = bad ? INFINITY : __fdiv_rn(__uint_as_float(all), 127.f);
        uint8_t* to = p.bounds + (size_t(tile) * p.Hk + hk) * page_bounds_bytes(D);
        const float over = __fdiv_rn(x, scale);
        const int code = bad || !(scale > 0.f) ? 0 : int(low ? fmaxf(floorf(over), -127.f) : fminf(ceilf(over), 127.f));
        to[tid] = uint8_t(code);
        if (tid == 0) *reinterpret_cast<float*>(to + 2 * D) = scale;
    }
}

// grid (blocks that T rows can touch, Hk, B): rows of one block of one head, as bf16(scale * code).  65536 rows of 8 heads, d = 128: 77.5 us, 5.2 TB/s; two of three bytes
// are written, and a fill of the outputs alone takes 69 us.
template <int D>
__global__ void __launch_bounds__(kPagesThreads)
pages_read_kernel(const PagesRowsParams p) {
    constexpr int CH = D / 8, LPR = D / 16, RPP = kPagesThreads / LPR, PASSES = kPageBlock / RPP;
    constexpr int KW = D / 4 + 4;
    __shared__ __align__(16) uint32_t s_v[kPageBlock][KW];
    const int b = blockIdx.z, hk = blockIdx.y, tid = threadIdx.x;
    grid_dependency_wait();
    PagesRows w;
    if (!pages_rows<true>(p, b, w)) return;
    const int tile = p.tile(b, w.blk);
    const uint8_t* rec = p.pages + (size_t(max(tile, 0)) * p.Hk + hk) * page_block_bytes(D);
    const float* scales = reinterpret_cast<const float*>(rec + 2 * kPageBlock * D);
    const int c = tid % LPR, row0 = tid / LPR;
    uint4 codes[PASSES];
    float scale[PASSES][2];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int row = row0 + i * RPP;
        codes[i] = make_uint4(0u, 0u, 0u, 0u);
        scale[i][0] = scale[i][1] = 0.f;
        if (tile >= 0 && row >= w.r0 && row < w.r1) {
            codes[i] = *reinterpret_cast<const uint4*>(rec + size_t(row) * D + 16 * c);
            scale[i][0] = scales[row];
            scale[i][1] = scales[kPageBlock + row];
        }
    }
    for (int e = tid; e < D; e += kPagesThreads) {
        const int k0 = 16 * (e & 3), f = e >> 2;
        uint32_t t[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (tile >= 0) x = *reinterpret_cast<const uint4*>(rec + kPageBlock * D + size_t(4 * f + j) * kPageBlock + k0);
            t[j][0] = x.x; t[j][1] = x.y; t[j][2] = x.z; t[j][3] = x.w;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            turn4x4(t[0][i], t[1][i], t[2][i], t[3][i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) s_v[k0 + 4 * i + j][f] = t[j][i];
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int row = row0 + i * RPP;
        if (row < w.r0 || row >= w.r1) continue;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            const uint4 x = kv ? *reinterpret_cast<const uint4*>(&s_v[row][4 * c]) : codes[i];
            const uint32_t in[4] = {x.x, x.y, x.z, x.w};
            uint32_t out[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t a, e;
                e4m3x4_to_f16(in[k], a, e);
                const float2 u = f16x2_to_f32(a), v = f16x2_to_f32(e);
                out[2 * k] = pack_bf16x2(u.x * scale[i][kv], u.y * scale[i][kv]);
                out[2 * k + 1] = pack_bf16x2(v.x * scale[i][kv], v.y * scale[i][kv]);
            }
            uint4* to = const_cast<uint4*>(kv ? p.V : p.K) + ((size_t(b) * p.T + (w.base + row)) * p.Hk + hk) * CH + 2 * c;
            to[0] = make_uint4(out[0], out[1], out[2], out[3]);
            to[1] = make_uint4(out[4], out[5], out[6], out[7]);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Selection.  Of the n = ceil(len / 64) blocks of (sequence, key/value head) the kept = min(n_keep, n) stay: the last min(n_recent, kept), and of the
// others those of the highest rating (equal ratings: the lower block).  With q8 = rint(q * (127 / max|q|)), one maximum for the heads of a group,
//
//     rating = scale * max over the heads of  sum_f max(q8_f smallest_f, q8_f largest_f)
//
// which is what a key within the block's bounds could score at most.  The sums are of whole numbers (dp4a), so that a rating has one value whatever the order, and
// ties are ties.
//
//   pages_select_one_kernel  a cluster of up to 8 CTAs per (sequence, head): each rates a share of the blocks into the first one's shared memory, which selects.  For few
//                            rows: one launch.
//   pages_rate_kernel        for many: a CTA per (sequence, up to 8 heads, some of its blocks) rates.  32 x 131072 positions, 8 heads: 17 us, 11.1 of their bytes at the copy
//                            rate; half of the issue slots are taken, and what is left is the way to a block, page number by page number, at the start of a CTA.
//   pages_select_kernel      and a CTA per (sequence, head) selects: 24.4 us together.  (In one kernel 5 us more, as the CTAs that select hold the place of others that would rate.)
//
// The selection is a chain of short phases, some 4 us whatever the length is: the lowest rating that stays digit by digit (8 bits, from the highest bit in which any two
// differ, until all that are left stay), then the blocks in their order.  The second kernel may come up when the first one's CTAs have ended, not before: 24.9 against 29.6 us.
// ---------------------------------------------------------------------------------------------------------------------
struct PagesSelectParams : PagesParams {
    const __nv_bfloat16* q;       // [B][Hk * G][d]
    const uint8_t* bounds;
    const int* lens;              // [B]
    int* index;                   // [B][Hk][n_keep]
    uint32_t* rating;             // [B][Hk][most]: integers in the order of the ratings
    int G, max_len, n_keep, n_recent, most, rounds;   // most: blocks of a sequence; rounds: that a warp of pages_rate_kernel takes
};

constexpr int kSelectThreads = 256, kSelectWarps = kSelectThreads / 32;
constexpr int kSelectSets = 4;                                       // blocks that a group of lanes has on its way
__host__ __device__ constexpr int select_step(int d) { return 32 / (d / 16) * kSelectSets; }    // blocks of a warp's round

__host__ __device__ inline int pages_blocks(int len) { return len / kPageBlock + (len % kPageBlock != 0); }

// Of the blocks of a sequence: `old` that are rated, `want` of which stay, and the recent ones.
struct SelectParts {
    int old, want, recent;
    __device__ __forceinline__ SelectParts(const PagesSelectParams& p, int b) {
        const int n = pages_blocks(min(max(p.lens[b], 0), p.max_len)), kept = min(p.n_keep, n);
        recent = min(p.n_recent, kept);
        old = n - recent;
        want = kept - recent;
    }
    __device__ __forceinline__ bool some() const { return want > 0 && want < old; }      // not all and not none of the old ones
};

// The queries of a group in 8 bits by a warp: positive parts and negative parts, [2][G][D / 4] words of four features.
template <int D>
__device__ __forceinline__ void queries_in_8_bits(const PagesSelectParams& p, int b, int hk, uint32_t* to, int lane) {
    const int words = p.G * (D / 4);
    const uint2* q = reinterpret_cast<const uint2*>(p.q + (size_t(b) * p.Hk + hk) * p.G * D);
    float most = 0.f;
#pragma unroll 4
    for (int e = lane; e < words; e += 32) {
        const uint2 v = q[e];
        most = fmaxf(most, fmaxf(fmaxf(fabsf(bf16_lo_to_f32(v.x)), fabsf(bf16_hi_to_f32(v.x))), fmaxf(fabsf(bf16_lo_to_f32(v.y)), fabsf(bf16_hi_to_f32(v.y)))));
    }
    most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
    const float inv = most > 0.f ? __fdiv_rn(127.f, most) : 0.f;
#pragma unroll 4
    for (int e = lane; e < words; e += 32) {
        const uint2 v = q[e];
        const float x[4] = {bf16_lo_to_f32(v.x), bf16_hi_to_f32(v.x), bf16_lo_to_f32(v.y), bf16_hi_to_f32(v.y)};
        uint32_t pos = 0u, neg = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = min(max(__float2int_rn(x[j] * inv), -127), 127);
            pos |= uint32_t(max(i, 0)) << (8 * j);
            neg |= (uint32_t(min(i, 0)) & 0xffu) << (8 * j);
        }
        to[e] = pos;
        to[words + e] = neg;
    }
}

// Numbers of blocks i0 .. i0 + select_step(D) - 1 of a sequence (below `old`), one a lane.
template <int D>
__device__ __forceinline__ int tiles_of(const PagesSelectParams& p, int b, int i0, int old, int lane) {
    return lane < select_step(D) && i0 + lane < old ? p.tile(b, i0 + lane) : -1;
}

// Their ratings for a head by a warp, d / 16 lanes a block: put(block, integer in the order of the ratings).
template <int D, class Put>
__device__ __forceinline__ void rate_blocks(const PagesSelectParams& p, int tiles, int hk, int i0, int old, const uint32_t* s_qp, int lane, const Put& put) {
    constexpr int LPB = D / 16, GPW = 32 / LPB;                      // lanes of a block (16 features each), blocks at a time
    const uint32_t* s_qn = s_qp + p.G * (D / 4);
    const int grp = lane / LPB, sub = lane % LPB;
    const int mine = (LPB == 8 ? (sub >> 1) : sub);                  // which set this lane ends up with
    const uint8_t* head = p.bounds + size_t(hk) * page_bounds_bytes(D);
    const size_t stride = size_t(p.Hk) * page_bounds_bytes(D);
    uint4 hi[kSelectSets], lo[kSelectSets];
#pragma unroll
    for (int s = 0; s < kSelectSets; ++s) {
        const int tile = __shfl_sync(0xffffffffu, tiles, s * GPW + grp);
        hi[s] = lo[s] = make_uint4(0u, 0u, 0u, 0u);
        if (tile >= 0) {
            const uint8_t* rec = head + size_t(tile) * stride + 16 * sub;
            hi[s] = *reinterpret_cast<const uint4*>(rec);
            lo[s] = *reinterpret_cast<const uint4*>(rec + D);
        }
    }
    const int own = __shfl_sync(0xffffffffu, tiles, mine * GPW + grp);
    const float scale = own >= 0 ? *reinterpret_cast<const float*>(head + size_t(own) * stride + 2 * D) : 0.f;
    int best = INT_MIN;
    for (int h = 0; h < p.G; ++h) {
        const uint4 qp = *reinterpret_cast<const uint4*>(s_qp + h * (D / 4) + 4 * sub), qn = *reinterpret_cast<const uint4*>(s_qn + h * (D / 4) + 4 * sub);
        int a[kSelectSets];
#pragma unroll
        for (int s = 0; s < kSelectSets; ++s) {
            int v = __dp4a(int(qp.x), int(hi[s].x), 0);
            v = __dp4a(int(qp.y), int(hi[s].y), v);
            v = __dp4a(int(qp.z), int(hi[s].z), v);
            v = __dp4a(int(qp.w), int(hi[s].w), v);
            v = __dp4a(int(qn.x), int(lo[s].x), v);
            v = __dp4a(int(qn.y), int(lo[s].y), v);
            v = __dp4a(int(qn.z), int(lo[s].z), v);
            a[s] = __dp4a(int(qn.w), int(lo[s].w), v);
        }
        // sums over the lanes of a block; each lane keeps one of the four sets
        constexpr int O2 = LPB / 2, O1 = LPB / 4;
        const bool up2 = sub & O2, up1 = sub & O1;
        const int g0 = __shfl_xor_sync(0xffffffffu, up2 ? a[0] : a[2], O2), g1 = __shfl_xor_sync(0xffffffffu, up2 ? a[1] : a[3], O2);
        const int c0 = (up2 ? a[2] : a[0]) + g0, c1 = (up2 ? a[3] : a[1]) + g1;
        int v = (up1 ? c1 : c0) + __shfl_xor_sync(0xffffffffu, up1 ? c0 : c1, O1);
        if (LPB == 8) v += __shfl_xor_sync(0xffffffffu, v, 1);
        best = max(best, v);
    }
    const int blk = i0 + mine * GPW + grp;
    if ((LPB == 4 || (sub & 1) == 0) && blk < old)
        // a block without a page is the last to be taken, one with keys that are not finite the first
        put(blk, evict_key(own >= 0 ? (scale < INFINITY ? float(best) * scale : INFINITY) : -INFINITY));
}

struct SelectShared {
    __align__(16) uint32_t hist[4][256];          // all 0 at the start
    uint32_t gt[kSelectWarps], eq[kSelectWarps], mn[kSelectWarps], mx[kSelectWarps];
};

// The blocks that stay, by a CTA with their ratings in shared memory (mn, mx: least and largest that this thread has seen of them): those above the lowest that
// stays, and the first `ties` that equal it, in their order; then the recent ones, and -1.
__device__ __forceinline__ void select_blocks(const PagesSelectParams& p, const SelectParts& x, int* index, const uint32_t* s_key, uint32_t mn, uint32_t mx, SelectShared& s) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int old = x.old, want = x.want;
    const int run = ((old + kSelectThreads - 1) / kSelectThreads) | 1;   // ratings of a thread: adjacent ones, an odd number for the banks
    const int r0 = min(tid * run, old), r1 = min(r0 + run, old);
    uint32_t thr = 0u, ties = 0u;
    if (x.some()) {
        mn = __reduce_min_sync(0xffffffffu, mn);
        mx = __reduce_max_sync(0xffffffffu, mx);
        if (lane == 0) { s.mn[warp] = mn; s.mx[warp] = mx; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSelectWarps; ++i) { mn = min(mn, s.mn[i]); mx = max(mx, s.mx[i]); }
        int shift = mn == mx ? 0 : 32 - __clz(mn ^ mx);              // bits below `shift` are still to be found
        uint32_t left = uint32_t(want), count = uint32_t(old);       // still to take among those that agree so far, and how many agree
        thr = shift < 32 ? mx >> shift << shift : 0u;
        for (int pass = 0; shift > 0 && count > left; ++pass) {
            const int bits = min(shift, 8), agree = shift;
            shift -= bits;
            uint32_t* hist = s.hist[pass];
            for (int i = r0; i < r1; ++i) {
                const uint32_t k = s_key[i];
                if (agree == 32 || ((k ^ thr) >> agree) == 0u) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1u)], 1u);
            }
            __syncthreads();
            // every warp for itself: 8 bins a lane
            const uint4 u = *reinterpret_cast<const uint4*>(&hist[8 * lane]), v = *reinterpret_cast<const uint4*>(&hist[8 * lane + 4]);
            const uint32_t c[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
            uint32_t sum = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += c[j];
            uint32_t incl = sum;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const uint32_t up = __shfl_down_sync(0xffffffffu, incl, off);
                if (lane + off < 32) incl += up;
            }
            uint32_t over = incl - sum;                              // in bins above this lane's
            const int at = __ffs(__ballot_sync(0xffffffffu, over < left && incl >= left)) - 1;
            uint32_t bin = 8u * lane;
#pragma unroll
            for (int j = 7; j > 0; --j) {
                if (over + c[j] >= left) { bin += uint32_t(j); break; }
                over += c[j];
            }
            bin = __shfl_sync(0xffffffffu, bin, at);
            thr |= bin << shift;
            left -= __shfl_sync(0xffffffffu, over, at);
            count = hist[bin];
        }
        ties = left;
        if (shift > 0) {                                             // all that agree stay: rating >= thr, whose lower bits are 0
            ties = thr == 0u ? uint32_t(old) : 0u;
            thr = thr == 0u ? 0u : thr - 1u;
        }
    }
    uint32_t gt = 0, eq = 0;
    if (x.some()) {
        for (int i = r0; i < r1; ++i) { const uint32_t k = s_key[i]; gt += k > thr; eq += k == thr; }
    } else if (want > 0) {
        gt = uint32_t(r1 - r0);
    }
    uint32_t gt_incl = gt, eq_incl = eq;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t a = __shfl_up_sync(0xffffffffu, gt_incl, off), e = __shfl_up_sync(0xffffffffu, eq_incl, off);
        if (lane >= off) { gt_incl += a; eq_incl += e; }
    }
    if (lane == 31) { s.gt[warp] = gt_incl; s.eq[warp] = eq_incl; }
    __syncthreads();
    const uint32_t gt_before = __reduce_add_sync(0xffffffffu, lane < warp ? s.gt[lane] : 0u) + gt_incl - gt;
    uint32_t eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? s.eq[lane] : 0u) + eq_incl - eq;
    uint32_t at = gt_before + min(eq_before, ties);
    if (x.some()) {
        for (int i = r0; i < r1; ++i) {
            const uint32_t k = s_key[i];
            const bool tie = k == thr;
            if (k > thr || (tie && eq_before < ties)) index[at++] = i;
            eq_before += tie;
        }
    } else if (want > 0) {
        for (int i = r0; i < r1; ++i) index[at++] = i;
    }
    for (int i = tid; i < p.n_keep - want; i += kSelectThreads) index[want + i] = i < x.recent ? old + i : -1;
}

__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// grid (cluster, Hk, B)
template <int D>
__global__ void __launch_bounds__(kSelectThreads, 4)
pages_select_one_kernel(const PagesSelectParams p) {
    extern __shared__ __align__(16) uint32_t s_one[];                // [2][G][D / 4] queries, [most] ratings of the first CTA
    __shared__ SelectShared s;
    uint32_t* s_key = s_one + 2 * p.G * (D / 4);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int ranks = gridDim.x, rank = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
    grid_dependency_wait();
    const SelectParts x(p, b);
    uint32_t mn = 0xffffffffu, mx = 0u;
    if (x.some()) {
        if (ranks > 1) cluster_arrive();                             // this CTA has started
        constexpr int STEP = select_step(D);
        int i0 = (rank * kSelectWarps + warp) * STEP, tiles = tiles_of<D>(p, b, i0, x.old, lane);
        if (warp == 0) queries_in_8_bits<D>(p, b, hk, s_one, lane);
        else if (rank == 0)
            for (int i = tid - 32; i < 4 * 256; i += kSelectThreads - 32) s.hist[0][i] = 0u;
        __syncthreads();
        if (ranks > 1) cluster_wait();                               // and so has the first one
        const uint32_t keys = ranks > 1 ? cluster_map_shared(smem_u32(s_key), 0u) : smem_u32(s_key);
        while (i0 < x.old) {
            const int next = i0 + ranks * kSelectWarps * STEP, behind = tiles_of<D>(p, b, next, x.old, lane);
            rate_blocks<D>(p, tiles, hk, i0, x.old, s_one, lane, [&](int blk, uint32_t k) { st_cluster_u32(keys + 4u * uint32_t(blk), k); });
            i0 = next;
            tiles = behind;
        }
        if (ranks > 1) cluster_sync_all();
        else __syncthreads();
        if (rank == 0)
            for (int i = tid; i < x.old; i += kSelectThreads) { const uint32_t k = s_key[i]; mn = min(mn, k); mx = max(mx, k); }
    }
    if (rank == 0) select_blocks(p, x, p.index + (size_t(b) * p.Hk + hk) * p.n_keep, s_key, mn, mx, s);
}

// grid (parts of a sequence, eights of the key/value heads, B).  The warps of a CTA take adjacent heads, whose bounds are adjacent in memory.
template <int D>
__global__ void __launch_bounds__(kSelectThreads, 4)
pages_rate_kernel(const PagesSelectParams p) {
    constexpr int STEP = select_step(D);
    extern __shared__ __align__(16) uint32_t s_q[];                  // [heads][2][G][D / 4]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int hk0 = int(blockIdx.y) * kSelectWarps, heads = min(p.Hk - hk0, kSelectWarps), b = blockIdx.z;
    const int at_once = kSelectWarps / heads;                        // steps that the warps take side by side
    grid_dependency_wait();
    const SelectParts x(p, b);
    const int first = int(blockIdx.x) * at_once * p.rounds * STEP;
    if (!x.some() || first >= x.old) return;
    int i0 = first + warp / heads * STEP, tiles = tiles_of<D>(p, b, i0, x.old, lane);
    const uint32_t* queries = s_q + warp % heads * 2 * p.G * (D / 4);
    if (warp < heads) queries_in_8_bits<D>(p, b, hk0 + warp, s_q + warp * 2 * p.G * (D / 4), lane);
    __syncthreads();
    if (warp >= at_once * heads) return;
    const int hk = hk0 + warp % heads;
    uint32_t* rating = p.rating + (size_t(b) * p.Hk + hk) * p.most;
    for (int round = 0; round < p.rounds && i0 < x.old; ++round) {
        const int next = i0 + at_once * STEP, behind = tiles_of<D>(p, b, next, x.old, lane);
        rate_blocks<D>(p, tiles, hk, i0, x.old, queries, lane, [&](int blk, uint32_t k) { rating[blk] = k; });
        i0 = next;
        tiles = behind;
    }
}

// grid (Hk, B)
__global__ void __launch_bounds__(kSelectThreads)
pages_select_kernel(const PagesSelectParams p) {
    extern __shared__ __align__(16) uint32_t s_key[];                // [most]
    __shared__ SelectShared s;
    const int tid = threadIdx.x, hk = blockIdx.x, b = blockIdx.y;
    const SelectParts x(p, b);
    for (int i = tid; i < 4 * 256; i += kSelectThreads) s.hist[0][i] = 0u;
    grid_dependency_wait();                                          // the ratings
    uint32_t mn = 0xffffffffu, mx = 0u;
    if (x.some()) {
        const uint32_t* rating = p.rating + (size_t(b) * p.Hk + hk) * p.most;
#pragma unroll 4
        for (int i = tid; i < x.old; i += kSelectThreads) {
            const uint32_t k = __ldcg(rating + i);
            s_key[i] = k;
            mn = min(mn, k);
            mx = max(mx, k);
        }
    }
    select_blocks(p, x, p.index + (size_t(b) * p.Hk + hk) * p.n_keep, s_key, mn, mx, s);
}

}  // namespace moda
