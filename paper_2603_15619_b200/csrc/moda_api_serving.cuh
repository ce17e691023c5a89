// The entry points that measure, bound and share the sequence cache of a serving program (include/moda.h): argument checks and
// launches.  Part of moda_api.cu, whose helpers it uses.
#pragma once

namespace {

// ------------------------------------------------------------------------------------------ attention weight of the keys
constexpr int kKeyMassCtas = 148;                 // most runs of a call: partial sums of that many fit the workspace

inline int key_mass_positions(int G) { return 128 / G; }

// CTAs that take adjacent heads at the same time.
inline int key_mass_team(int H_kv, int n_units) {
    if (n_units > 4) return 1;
    int team = 8;
    while (H_kv % team != 0) --team;
    return team;
}

template <int D, bool FEW>
int launch_key_mass(const void* Q, const void* K, int B, const KeyMassParams& p, unsigned ctas, bool join, cudaStream_t stream) {
    using L = KeyMassSmem<D>;
    // query rows of a unit: P positions of the G heads, position after position
    CUtensorMap mQ, mK;
    if (!make_box_map(&mQ, Q, B, p.T_q, p.Hk * p.G, D, p.G, p.P) || !make_bthd_map(&mK, K, B, p.T_cap, p.Hk, D)) return MODA_ERR_CUDA;
    static thread_local int configured_dev = -1;
    int dev = 0;
    if (!cuda_ok(cudaGetDevice(&dev))) return MODA_ERR_CUDA;
    if (configured_dev != dev) {
        if (!set_smem_limit(key_mass_kernel<D, FEW>, L::kDynamic)) return MODA_ERR_CUDA;
        configured_dev = dev;
    }
    key_mass_kernel<D, FEW><<<ctas, kKmThreads, L::kDynamic, stream>>>(mQ, mK, p);
    if (!cuda_ok(cudaGetLastError())) return MODA_ERR_CUDA;
    if (!join) return MODA_OK;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas, 1, 1);
    cfg.blockDim = dim3(kKmTile, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cuda_ok(cudaLaunchKernelEx(&cfg, key_mass_join_kernel, p)) ? MODA_OK : MODA_ERR_CUDA;
}

// ------------------------------------------------------------------------------------------------------ shared prefix
// CTAs that take the same key tiles at the same time (moda_shared.cuh): the largest divisor up to 8 of the heads with one row tile, up to 16 of
// the pairs of row tiles with more.  us, one row tile, a head alone / teams of 2 / 4 / 8: B = 37, 24 heads on 8, d = 64, 131072 keys 85 / 67 / 67 /
// 58, 10007 keys 20.0 / 20.1 / 19.0 / 15.6; d = 128, 10007 keys 27.7 / 27.2 / 25.2 / 20.5.
inline int shared_team(int H_kv, int row_tiles, int pairs) {
    const int of = row_tiles > 1 ? pairs : H_kv;
    int team = row_tiles > 1 ? 16 : 8;
    while (of % team != 0) --team;
    return team;
}

constexpr long long kSharedMostTiles = 0x3fffffffll;

// How the prefix of a call is cut, for `ctas` CTAs.
SharedParams shared_plan(int B, int P, int H, int H_kv, int d, int ctas) {
    SharedParams p = {};
    p.B = B; p.P = P; p.H = H; p.Hk = H_kv; p.G = H / H_kv;
    if (P == 0) return p;
    p.S = 128 / p.G;
    p.row_tiles = (B + p.S - 1) / p.S;
    p.pairs = (p.row_tiles + 1) / 2;
    p.key_tiles = (P + 127) / 128;
    p.team = shared_team(H_kv, p.row_tiles, p.pairs);
    const long long total = (long long)(shared_group(p, H_kv - 1, p.pairs - 1) + 1) * p.key_tiles;
    p.total = int(std::min(total, kSharedMostTiles));
    const int teams = ctas / p.team;
    p.run = std::max((p.total + teams - 1) / teams, p.row_tiles > 1 ? 1 : 2);      // with one row tile: a key tile for each stream
    shared_slots(d, p.row_tiles > 1, p.k_slots, p.v_slots);
    p.pieces = ((p.key_tiles + p.run - 2) / p.run + 1) * (p.row_tiles > 1 ? 1 : 2);
    return p;
}
size_t shared_prefix_bytes(const SharedParams& p, int d) {
    return (size_t(p.pieces) * p.B * p.H * (size_t(d) * 4 + 8) + 15) / 16 * 16;
}

template <int D>
int launch_shared_prefix(const void* q, const void* Kp, const void* Vp, const SharedParams& p, cudaStream_t stream) {
    using L = SharedSmem<D>;
    CUtensorMap mQ, mK, mV;
    if (!make_box_map(&mQ, q, 1, p.B, p.H, D, p.G, p.S) || !make_bthd_map(&mK, Kp, 1, p.P, p.Hk, D) || !make_bthd_map(&mV, Vp, 1, p.P, p.Hk, D))
        return MODA_ERR_CUDA;
    static thread_local int configured_dev = -1;
    int dev = 0;
    if (!cuda_ok(cudaGetDevice(&dev))) return MODA_ERR_CUDA;
    if (configured_dev != dev) {
        if (!set_smem_limit(shared_prefix_kernel<D>, L::kDynamic)) return MODA_ERR_CUDA;
        configured_dev = dev;
    }
    shared_prefix_kernel<D><<<unsigned((p.total + p.run - 1) / p.run) * unsigned(p.team), kSpThreads, L::kDynamic, stream>>>(mQ, mK, mV, p);
    return cuda_ok(cudaGetLastError()) ? MODA_OK : MODA_ERR_CUDA;
}

template <int D>
int launch_own_cache(const DecodeParams& p, cudaStream_t stream) {
    switch (p.H / p.Hk) {
        case 1: return launch_decode_split<D, 1>(p, stream);
        case 2: return launch_decode_split<D, 2>(p, stream);
        case 3: return launch_decode_split<D, 3>(p, stream);
        case 4: return launch_decode_split<D, 4>(p, stream);
        case 5: return launch_decode_split<D, 5>(p, stream);
        case 6: return launch_decode_split<D, 6>(p, stream);
        case 7: return launch_decode_split<D, 7>(p, stream);
        case 8: return launch_decode_split<D, 8>(p, stream);
        default: return MODA_ERR_BAD_GROUP;
    }
}

// Warps that merge a row (sequence, query head): four while the SMs hold all rows so, one when they would take turns, as a warp alone waits for
// nobody.  us of the step without own caches, l = 24, four / two / one: 128 rows of d = 128 10.5 / 10.7 / 11.7, 256 (long prefix) 24.9 / 26.8 / 33.5, 512
// 13.9 / 12.6 / 13.2, 2048 27.7 / 24.9 / 27.5, 2400 27.9 / 24.5 / 22.0, 3200 32.8 / 27.1 / 26.0, 4096 64 / 57 / 47.
constexpr long long kMergeFourWarps = 400, kMergeTwoWarps = 2200;

// Own caches (longest x heads of a group, longest) that the merge reads itself: every head of a group reads their keys again, but no
// kernel runs for them, whose pieces of a few keys cost some 2 us each, one behind the other.  us, split kernel / here (B, shared keys, heads on kv
// heads, d, l; longest own cache): 128, 16384, 32 on 8, 128, 24: 32 keys 73.7 / 55.8, 96 73.3 / 71.1, 128 73.7 / 78.7; 64, 1000, 64 on 8, 64, 16: 32 24.9 / 20.1,
// 64 24.9 / 23.2, 96 25.2 / 26.5; 128, 2000, 40 on 40, 128, 12: 32 114 / 54, 128 122 / 93, 256 137 / 140.
constexpr int kMergeOwnWork = 384, kMergeOwnLen = 192;

// A short prefix (key tiles of a CTA, were it on all SMs) with own caches that are not large (elements of K): the prefix takes half of the SMs
// and the own caches the others, at the same time; a CTA of either fills its SM.  Otherwise one behind the other, each on all
// SMs.  us, one behind the other -> side by side, l = 24 (B, shared keys, longest own cache, heads, d): 37, 10007, 301, 24 on 8, 64: 28.4 -> 23.1; 16, 8192,
// 512, 32 on 8, 128: 29.9 -> 24.2; 16, 30000, 512: 43.9 -> 41.0; 64, 4096, 128: 42.7 -> 35.8; 64, 16384, 128: 54.2 -> 52.0; 8, 20000, 2000, 16 on 4: 26.1 -> 22.0;
// but 128, 4000, 200, 16 on 16, 64 (26 M elements): 56 -> 80.
constexpr int kSharedShortRun = 16;
constexpr long long kSharedShortOwn = 16ll << 20;

template <int D>
int launch_shared(const void* q, const void* Kp, const void* Vp, const SharedMergeParams& p, cudaStream_t stream) {
    if (p.pre.P > 0)
        if (int rc = launch_shared_prefix<D>(q, Kp, Vp, p.pre, stream)) return rc;
    if (p.dec.T_kv > 0 && !p.own_here)
        if (int rc = launch_own_cache<D>(p.dec, stream)) return rc;
    const long long rows = (long long)p.dec.H * p.dec.B;
    const int warps = rows <= kMergeFourWarps ? 4 : rows <= kMergeTwoWarps ? 2 : 1;
    const long long ctas = (rows * warps * 32 + kSharedMergeThreads - 1) / kSharedMergeThreads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(ctas), 1, 1);
    cfg.blockDim = dim3(kSharedMergeThreads, 1, 1);
    // as for the merge of a decode step, within the 48 KiB that a kernel may have without asking
    cfg.dynamicSmemBytes = warps == 1 ? 0 : std::min<size_t>(decode_merge_reserve(ctas, p.dec.team * p.dec.teams), 36000);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.pre.P > 0 || (p.dec.T_kv > 0 && !p.own_here) ? 1 : 0;
    const cudaError_t rc = warps == 4   ? cudaLaunchKernelEx(&cfg, shared_merge_kernel<D, 4>, p)
                           : warps == 2 ? cudaLaunchKernelEx(&cfg, shared_merge_kernel<D, 2>, p)
                                        : cudaLaunchKernelEx(&cfg, shared_merge_kernel<D, 1>, p);
    return cuda_ok(rc) ? MODA_OK : MODA_ERR_CUDA;
}

template <int RUN, int NT, int CTAS>
int launch_evict_select(const EvictParams& p, int ranks, cudaStream_t stream) {
    static thread_local int configured_dev = -1;
    int dev = 0;
    if (!cuda_ok(cudaGetDevice(&dev))) return MODA_ERR_CUDA;
    if (configured_dev != dev) {
        if (!set_smem_limit(evict_select_kernel<RUN, NT, CTAS>, evict_select_smem(RUN, NT)) ||
            !cuda_ok(cudaFuncSetAttribute(evict_select_kernel<RUN, NT, CTAS>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)))
            return MODA_ERR_CUDA;
        configured_dev = dev;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(ranks), unsigned(p.Hk), unsigned(p.B));
    cfg.blockDim = dim3(NT, 1, 1);
    cfg.dynamicSmemBytes = size_t(evict_select_smem(RUN > 0 ? evict_run(p.T, ranks, NT) : 0, NT));
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(ranks);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cuda_ok(cudaLaunchKernelEx(&cfg, evict_select_kernel<RUN, NT, CTAS>, p)) ? MODA_OK : MODA_ERR_CUDA;
}

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

size_t decode_mass_stride(int T_kv) { return (size_t(T_kv) + 7) / 8 * 8; }

}  // namespace

extern "C" {

size_t moda_key_mass_workspace_bytes(int B, int T_q, int T_kv, int H, int H_kv, int d) {
    if (B < 1 || T_q < 1 || T_kv < T_q || H < 1 || check_groups(H, H_kv) || (d != 64 && d != 128)) return 0;
    return size_t(kKeyMassCtas) * (2 * kKmTile * 4 + 2 * 8);
}

int moda_attn_key_mass(const void* Q, const void* K, const float* LSE, const float* mass_in,
                       int B, int T_q, int T_kv, int T_cap, int H, int H_kv, int d, float scale,
                       float* mass, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_shape(B, T_q, H, d)) return rc;
    if (T_kv < T_q || T_cap < T_kv) return MODA_ERR_BAD_SHAPE;
    if (int rc = check_scale(scale)) return rc;
    if (int rc = check_groups(H, H_kv)) return rc;
    if ((long long)B * T_cap > 0x7fffffffLL / H) return MODA_ERR_BAD_SHAPE;
    if (!Q || !K || !LSE || !mass) return MODA_ERR_NULL_POINTER;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(LSE) || !aligned16(mass) || !aligned16(mass_in)) return MODA_ERR_MISALIGNED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < moda_key_mass_workspace_bytes(B, T_q, T_kv, H, H_kv, d)) return MODA_ERR_WORKSPACE;
    KeyMassParams p = {};
    p.LSE = LSE; p.mass_in = mass_in; p.mass = mass; p.part = static_cast<float*>(workspace);
    p.T_q = T_q; p.T_kv = T_kv; p.T_cap = T_cap; p.Hk = H_kv; p.G = H / H_kv;
    p.P = key_mass_positions(p.G);
    p.n_units = (T_q + p.P - 1) / p.P;
    p.tiles = (T_kv + kKmTile - 1) / kKmTile;
    for (int j = 0; j < p.tiles; ++j) p.per_head += p.n_units - key_mass_first_unit(j, T_kv - T_q, p.P);
    if (p.per_head > 0x3fffffffLL) return MODA_ERR_BAD_SHAPE;
    if (int rc = check_device()) return rc;
    int sms = 0;
    if (int rc = device_sm_count(&sms)) return rc;
    const bool all_see_all = key_mass_first_unit(p.tiles - 1, T_kv - T_q, p.P) == 0;
    p.team = key_mass_team(H_kv, p.n_units);
    const long long teams = std::min(sms, kKeyMassCtas) / p.team;
    p.total = p.per_head * B * (H_kv / p.team);
    long long run = (p.total + teams - 1) / teams;
    // whole tiles where they cost little: nothing to join then
    if (all_see_all && (run + p.n_units - 1) / p.n_units * p.n_units <= run + run / 16) run = (run + p.n_units - 1) / p.n_units * p.n_units;
    const bool join = !(all_see_all && run % p.n_units == 0);
    if (run > 0x3fffffffLL || (long long)B * H_kv * p.tiles > 0x7fffffffLL) return MODA_ERR_BAD_SHAPE;
    p.run = int(run);
    p.scale_log2 = scale * kLog2e;
    p.inv_scale = 1.f / scale;
    p.least = -127.f / p.scale_log2;
    key_mass_slots(d, p.n_units, p.k_slots, p.q_slots);
    const bool few = p.n_units <= 4 && p.k_slots == 4;                  // (a slot of a half is that of even or of odd tiles)
    p.stay = p.q_slots % p.n_units == 0 && all_see_all;
    const unsigned ctas = unsigned((p.total + run - 1) / run) * unsigned(p.team);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (few) return d == 128 ? launch_key_mass<128, true>(Q, K, B, p, ctas, join, st) : launch_key_mass<64, true>(Q, K, B, p, ctas, join, st);
    return d == 128 ? launch_key_mass<128, false>(Q, K, B, p, ctas, join, st) : launch_key_mass<64, false>(Q, K, B, p, ctas, join, st);
}

size_t moda_decode_mass_workspace_bytes(int B, int T_kv, int H, int H_kv, int d) {
    if (B < 1 || T_kv < 1 || H < 1 || check_groups(H, H_kv) || (d != 64 && d != 128)) return 0;
    return decode_workspace_bytes(B, H, d) + size_t(B) * H * decode_mass_stride(T_kv) * 4;
}

int moda_attn_decode_mass(const void* q, const void* K, const void* V, const int* seq_lens,
                          const void* depth_kv_token, const float* mass_in,
                          int B, int T_kv, int T_cap, int H, int H_kv, int d, int l, float scale,
                          void* O, float* LSE, float* mass, void* workspace, size_t workspace_bytes, void* stream) {
    if (B < 1 || T_kv < 1 || H < 1 || T_cap < T_kv) return MODA_ERR_BAD_SHAPE;
    if (d != 64 && d != 128) return MODA_ERR_BAD_HEAD_DIM;
    if (int rc = check_scale(scale)) return rc;
    if ((long long)B * T_cap > 0x7fffffffLL / H) return MODA_ERR_BAD_SHAPE;
    if (int rc = check_groups(H, H_kv)) return rc;
    if ((long long)B * H * kDecodeMaxSplits > 0x7fffffffLL || B > 65535 || H_kv > 65535) return MODA_ERR_BAD_SHAPE;
    if (l < 0 || l > MODA_MAX_DEPTH) return MODA_ERR_BAD_DEPTH;
    if (!q || !K || !V || !O || !LSE || !mass || (l > 0 && !depth_kv_token)) return MODA_ERR_NULL_POINTER;
    if (!aligned4(seq_lens) || !aligned16(q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(LSE) || !aligned16(mass) ||
        !aligned16(mass_in) || (l > 0 && !aligned16(depth_kv_token)))
        return MODA_ERR_MISALIGNED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < moda_decode_mass_workspace_bytes(B, T_kv, H, H_kv, d)) return MODA_ERR_WORKSPACE;
    if (int rc = check_device()) return rc;
    int sms = 0;
    if (int rc = device_sm_count(&sms)) return rc;
    DecodeParams p = decode_params(q, K, V, seq_lens, nullptr, depth_kv_token, B, T_kv, T_cap, 0, 0, H, H_kv, d, l, scale, O, LSE, workspace, sms);
    p.scores = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + decode_workspace_bytes(B, H, d));
    p.score_stride = decode_mass_stride(T_kv);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (int rc = d == 128 ? launch_decode<128, kDecodeKeepScores>(p, st) : launch_decode<64, kDecodeKeepScores>(p, st)) return rc;
    DecodeKeyMassParams m = {};
    m.scores = p.scores; m.LSE = LSE; m.mass_in = mass_in; m.mass = mass; m.seq_lens = seq_lens;
    m.stride = p.score_stride; m.T_kv = T_kv; m.T_cap = T_cap; m.H = H; m.Hk = H_kv;
    const unsigned blocks = unsigned((T_kv + 4 * kDecodeMassThreads - 1) / (4 * kDecodeMassThreads));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks, unsigned(H_kv), unsigned(B));
    cfg.blockDim = dim3(kDecodeMassThreads, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cuda_ok(cudaLaunchKernelEx(&cfg, decode_key_mass_kernel, m)) ? MODA_OK : MODA_ERR_CUDA;
}

int moda_kv_evict(const void* K, const void* V, const float* mass, const int* seq_lens,
                  int B, int T, int T_cap, int H_kv, int d, int n_keep, int n_recent, int T_out,
                  void* K_out, void* V_out, float* mass_out, int* index, int* lens_out, void* stream) {
    if (B < 1 || T < 1 || H_kv < 1 || T_cap < T || n_keep < 1 || T_out < n_keep || n_recent < 0 || n_recent > n_keep) return MODA_ERR_BAD_SHAPE;
    if (d != 64 && d != 128) return MODA_ERR_BAD_HEAD_DIM;
    if ((long long)B * T_cap > 0x7fffffffLL / H_kv || (long long)B * T_out > 0x7fffffffLL / H_kv || B > 65535 || H_kv > 4096) return MODA_ERR_BAD_SHAPE;
    if (!K || !V || !mass || !K_out || !V_out || !index) return MODA_ERR_NULL_POINTER;
    if (!aligned16(K) || !aligned16(V) || !aligned16(K_out) || !aligned16(V_out) || !aligned4(mass) || !aligned4(mass_out) || !aligned4(index) ||
        !aligned4(seq_lens) || !aligned4(lens_out))
        return MODA_ERR_MISALIGNED;
    const size_t row = size_t(H_kv) * d * 2;
    auto apart = [&](const void* in, const void* out) {
        const auto a = reinterpret_cast<uintptr_t>(in), b = reinterpret_cast<uintptr_t>(out);
        return b >= a + size_t(B) * T_cap * row || a >= b + size_t(B) * T_out * row;
    };
    if (!apart(K, K_out) || !apart(V, V_out) || !apart(K, V_out) || !apart(V, K_out)) return MODA_ERR_BAD_SHAPE;
    if (mass_out) {
        const auto a = reinterpret_cast<uintptr_t>(mass), b = reinterpret_cast<uintptr_t>(mass_out);
        if (b < a + size_t(B) * H_kv * T_cap * 4 && a < b + size_t(B) * H_kv * T_out * 4) return MODA_ERR_BAD_SHAPE;
    }
    if (seq_lens && lens_out && lens_out != seq_lens) {              // in place, but not over another sequence's length
        const auto a = reinterpret_cast<uintptr_t>(seq_lens), b = reinterpret_cast<uintptr_t>(lens_out);
        if (b < a + size_t(B) * 4 && a < b + size_t(B) * 4) return MODA_ERR_BAD_SHAPE;
    }
    if (int rc = check_device()) return rc;
    EvictParams p = {};
    p.K = static_cast<const __nv_bfloat16*>(K); p.V = static_cast<const __nv_bfloat16*>(V); p.mass = mass; p.seq_lens = seq_lens;
    p.K_out = static_cast<__nv_bfloat16*>(K_out); p.V_out = static_cast<__nv_bfloat16*>(V_out); p.mass_out = mass_out; p.index = index;
    p.lens_out = lens_out;
    p.B = B; p.T = T; p.T_cap = T_cap; p.T_out = T_out; p.Hk = H_kv; p.n_keep = n_keep; p.n_recent = n_recent;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int sms = 0;
    if (int rc = device_sm_count(&sms)) return rc;
    const EvictForm f = evict_form(T, (long long)B * H_kv, sms);
    if (int rc = f.most == 5    ? launch_evict_select<5, 512, 2>(p, f.ranks, st)
                 : f.most == 9  ? launch_evict_select<9, 512, 2>(p, f.ranks, st)
                 : f.most == 17 ? launch_evict_select<17, 512, 2>(p, f.ranks, st)
                 : f.most == 0  ? launch_evict_select<0, 512, 1>(p, f.ranks, st)
                 : f.threads > 512 ? launch_evict_select<kEvictMostRun, kEvictMostThreads, 1>(p, f.ranks, st)
                 : f.ctas == 2  ? launch_evict_select<33, 512, 2>(p, f.ranks, st)
                                : launch_evict_select<33, 512, 1>(p, f.ranks, st))
        return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const int rows = std::max(1, kEvictGatherPieces / (H_kv * (d / 8)));
    const int longest = std::min(n_keep, T);
    cfg.gridDim = dim3(unsigned((longest + rows - 1) / rows), unsigned(B), 1);
    cfg.blockDim = dim3(kEvictGatherThreads, 1, 1);
    cfg.dynamicSmemBytes = size_t(rows) * H_kv * 4;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    const bool ok = d == 128 ? cuda_ok(cudaLaunchKernelEx(&cfg, evict_gather_kernel<128>, p, rows))
                             : cuda_ok(cudaLaunchKernelEx(&cfg, evict_gather_kernel<64>, p, rows));
    return ok ? MODA_OK : MODA_ERR_CUDA;
}

size_t moda_decode_shared_workspace_bytes(int B, int T_prefix, int H, int H_kv, int d) {
    if (B < 1 || T_prefix < 0 || H < 1 || check_groups(H, H_kv) || (d != 64 && d != 128)) return 0;
    return decode_workspace_bytes(B, H, d) + shared_prefix_bytes(shared_plan(B, T_prefix, H, H_kv, d, kSharedCtas), d);
}

int moda_attn_decode_shared(const void* q, const void* K_prefix, const void* V_prefix, const void* K, const void* V, const int* seq_lens,
                            const void* depth_kv_token,
                            int B, int T_prefix, int max_seq_len, int T_cap, int H, int H_kv, int d, int l, float scale,
                            void* O, float* LSE, void* workspace, size_t workspace_bytes, void* stream) {
    if (B < 1 || T_prefix < 0 || max_seq_len < 0 || H < 1 || T_cap < max_seq_len) return MODA_ERR_BAD_SHAPE;
    if (d != 64 && d != 128) return MODA_ERR_BAD_HEAD_DIM;
    if (int rc = check_scale(scale)) return rc;
    if ((long long)B * T_cap > 0x7fffffffLL / H || T_prefix > 0x7fffffffLL / H) return MODA_ERR_BAD_SHAPE;
    if (int rc = check_groups(H, H_kv)) return rc;
    if ((long long)B * H * kDecodeMaxSplits > 0x7fffffffLL || B > 65535) return MODA_ERR_BAD_SHAPE;
    if (l < 0 || l > MODA_MAX_DEPTH) return MODA_ERR_BAD_DEPTH;
    if (!q || !O || !LSE || (l > 0 && !depth_kv_token) || (T_prefix > 0 && (!K_prefix || !V_prefix)) || (max_seq_len > 0 && (!K || !V)))
        return MODA_ERR_NULL_POINTER;
    if (!aligned4(seq_lens) || !aligned16(q) || !aligned16(O) || !aligned16(LSE) || (l > 0 && !aligned16(depth_kv_token)) ||
        (T_prefix > 0 && (!aligned16(K_prefix) || !aligned16(V_prefix))) || (max_seq_len > 0 && (!aligned16(K) || !aligned16(V))))
        return MODA_ERR_MISALIGNED;
    if (shared_plan(B, T_prefix, H, H_kv, d, kSharedCtas).total >= kSharedMostTiles) return MODA_ERR_BAD_SHAPE;
    if (!workspace || !aligned16(workspace) || workspace_bytes < moda_decode_shared_workspace_bytes(B, T_prefix, H, H_kv, d)) return MODA_ERR_WORKSPACE;
    if (int rc = check_device()) return rc;
    int sms = 0;
    if (int rc = device_sm_count(&sms)) return rc;
    SharedMergeParams p = {};
    p.pre = shared_plan(B, T_prefix, H, H_kv, d, std::min(sms, kSharedCtas));
    p.own_here = max_seq_len <= kMergeOwnLen && max_seq_len * std::min(H / H_kv, 8) <= kMergeOwnWork;
    int own_sms = sms;
    if (T_prefix > 0 && !p.own_here && max_seq_len > 0 && p.pre.run <= kSharedShortRun && (long long)B * max_seq_len * H_kv * d <= kSharedShortOwn) {
        p.pre = shared_plan(B, T_prefix, H, H_kv, d, std::max(std::min(sms, kSharedCtas) / 2, p.pre.team));
        own_sms = std::max(sms - (p.pre.total + p.pre.run - 1) / p.pre.run * p.pre.team, sms / 2);
    }
    p.dec = decode_params(q, K, V, seq_lens, nullptr, depth_kv_token, B, std::max(max_seq_len, 1), T_cap, 0, 0, H, H_kv, d, l, scale, O, LSE,
                          workspace, own_sms);
    p.dec.T_kv = max_seq_len;
    p.dec.beside = T_prefix > 0;
    uint8_t* at = static_cast<uint8_t*>(workspace) + decode_workspace_bytes(B, H, d);
    p.pre.o = reinterpret_cast<float*>(at);
    p.pre.ml = reinterpret_cast<float2*>(at + size_t(p.pre.pieces) * B * H * d * 4);
    p.pre.scale_log2 = scale * kDecodeLog2e;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d == 128 ? launch_shared<128>(q, K_prefix, V_prefix, p, st) : launch_shared<64>(q, K_prefix, V_prefix, p, st);
}

}  // extern "C"
