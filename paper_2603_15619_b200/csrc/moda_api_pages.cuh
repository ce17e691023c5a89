// The entry points of the paged sequence cache in 8 bits (include/moda.h): argument checks and launches.  Part of moda_api.cu, whose helpers it uses.
#pragma once

namespace {

// What the calls over the pages check alike.
int check_pages(int B, int page_size, int num_pages, int max_blocks, int H_kv, int d) {
    if (B < 1 || H_kv < 1 || page_size < kPageBlock || page_size % kPageBlock != 0 || num_pages < 1 || max_blocks < 1) return MODA_ERR_BAD_SHAPE;
    if (d != 64 && d != 128) return MODA_ERR_BAD_HEAD_DIM;
    if (B > 65535 || H_kv > 65535) return MODA_ERR_BAD_SHAPE;
    if ((long long)num_pages * (page_size / kPageBlock) > 0x7fffffffLL || (long long)max_blocks * page_size > 0x7fffffffLL) return MODA_ERR_BAD_SHAPE;
    return MODA_OK;
}
void set_pages(PagesParams& p, const int* table, int B, int Hk, int page_size, int num_pages, int max_blocks) {
    p.table = table; p.B = B; p.Hk = Hk; p.sub = page_size / kPageBlock; p.num_pages = num_pages; p.max_blocks = max_blocks;
}

// Rows written or read: all blocks that T of them can touch.
int pages_rows_grid(int B, int T, int H_kv, dim3* grid) {
    if (T < 1 || (long long)B * T > 0x7fffffffLL / H_kv) return MODA_ERR_BAD_SHAPE;
    *grid = dim3(unsigned(((long long)T + kPageBlock - 2) / kPageBlock + 1), unsigned(H_kv), unsigned(B));
    return MODA_OK;
}

constexpr int kPagesMostCtas = 148;               // partial results of that many fit the workspace

inline int pages_split_warps(int d) { return d == 64 ? PagesSplit<64>::kWarps : PagesSplit<128>::kWarps; }
inline size_t pages_part_bytes(int B, int H, int G, int d) {
    return (size_t(kPagesMostCtas) * pages_split_warps(d) * G + size_t(2) * B * H) * (d + 2) * 4;
}
size_t pages_workspace_bytes(int B, int H, int H_kv, int d) {
    return (pages_part_bytes(B, H, std::min(H / H_kv, 8), d) + size_t(B + 1) * 4 + 15) / 16 * 16;
}

// Every kernel over the pages is launched beside the end of what comes before it in the stream, whatever that is, and every one of its CTAs waits for that before it
// writes, ends or lets a later kernel start, so that what waits for it may use what came before as well.  Calls in a loop, launched so and plainly: a token of 64 sequences written 7.2 and
// 8.8 us, selection for one sequence 7.5 and 10.4, its decode step 9.0 and 10.5, that of 32 ragged ones 60.0 and 62.2.
template <typename P>
int launch_pages(void (*kernel)(P), dim3 grid, int threads, size_t smem, const P& p, cudaStream_t stream, int ranks = 1) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(unsigned(threads), 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (ranks > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = unsigned(ranks);
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    return cuda_ok(cudaLaunchKernelEx(&cfg, kernel, p)) ? MODA_OK : MODA_ERR_CUDA;
}

// A kernel's limit of dynamic shared memory, raised to `most` on a thread's first call on a device that needs more than a kernel may have without asking.
template <typename Kernel>
int raise_smem(Kernel kernel, size_t need, int most, int* configured_dev) {
    if (need <= 40000) return MODA_OK;            // beside the static part
    int dev = 0;
    if (!cuda_ok(cudaGetDevice(&dev))) return MODA_ERR_CUDA;
    if (*configured_dev != dev) {
        if (!set_smem_limit(kernel, most)) return MODA_ERR_CUDA;
        *configured_dev = dev;
    }
    return MODA_OK;
}

template <int D>
int launch_select(PagesSelectParams& p, int sms, cudaStream_t stream) {
    static thread_local int rate_dev = -1, select_dev = -1;
    const long long rows = (long long)p.B * p.Hk;
    const size_t ratings = size_t(p.most) * 4, queries = size_t(2) * p.G * D;
    const int ranks = select_ranks(p.most, rows, sms);
    if (ranks > 0)                                // at most 4096 blocks: within what a kernel may have without asking
        return launch_pages(pages_select_one_kernel<D>, dim3(unsigned(ranks), unsigned(p.Hk), unsigned(p.B)), kSelectThreads, queries + ratings, p, stream, ranks);
    const int heads = std::min(p.Hk, kSelectWarps), eights = (p.Hk + kSelectWarps - 1) / kSelectWarps;
    const int step = kSelectWarps / heads * select_step(D);
    p.rounds = rate_rounds(p.most, step, (long long)p.B * eights, sms);
    const unsigned parts = unsigned((p.most + step * p.rounds - 1) / (step * p.rounds));
    if (int rc = raise_smem(pages_rate_kernel<D>, heads * queries, kSelectWarps * 2 * MODA_MAX_GROUP * D, &rate_dev)) return rc;
    if (int rc = launch_pages(pages_rate_kernel<D>, dim3(parts, unsigned(eights), unsigned(p.B)), kSelectThreads, heads * queries, p, stream)) return rc;
    if (int rc = raise_smem(pages_select_kernel, ratings, kSelectMostBlocks * 4, &select_dev)) return rc;
    return launch_pages(pages_select_kernel, dim3(unsigned(p.Hk), unsigned(p.B)), kSelectThreads, ratings, p, stream);
}

template <int D>
int launch_decode_pages(const PagesDecodeParams& p, cudaStream_t stream) {
    static thread_local int configured_dev = -1;
    int dev = 0;
    if (!cuda_ok(cudaGetDevice(&dev))) return MODA_ERR_CUDA;
    if (configured_dev != dev) {
        if (!set_smem_limit(pages_split_kernel<D>, PagesSplit<D>::smem(kPagesMostBatch))) return MODA_ERR_CUDA;
        configured_dev = dev;
    }
    if (int rc = launch_pages(pages_split_kernel<D>, dim3(unsigned(p.warps / PagesSplit<D>::kWarps)), PagesSplit<D>::kThreads, size_t(PagesSplit<D>::smem(p.B)), p, stream))
        return rc;
    const long long rows = (long long)p.B * p.H;
    // Four warps a row while the rows leave SMs idle and have more than two partial results each, else one.  In us, four and one: 16 rows 8.7 and 11.0, 512 25.2 and
    // 30.5, 1024 37.3 and 38.2, 1536 48.2 and 47.9, 2048 61.2 and 58.7; 1024 with one to two results each 60.4 and 58.6.
    const bool wide = rows <= 8 * kPagesMostCtas && 2ll * p.B * p.Hk <= p.warps;
    const long long per = kPagesMergeThreads / 32 / (wide ? 4 : 1);
    return launch_pages(wide ? pages_merge_kernel<D, 4> : pages_merge_kernel<D, 1>, dim3(unsigned((rows + per - 1) / per)), kPagesMergeThreads, 0, p, stream);
}

}  // namespace

extern "C" {

size_t moda_kv_page_e4m3_bytes(int page_size, int H_kv, int d) {
    if (check_pages(1, page_size, 1, 1, H_kv, d)) return 0;
    return size_t(page_size / kPageBlock) * H_kv * page_block_bytes(d);
}
size_t moda_kv_page_bounds_bytes(int page_size, int H_kv, int d) {
    if (check_pages(1, page_size, 1, 1, H_kv, d)) return 0;
    return size_t(page_size / kPageBlock) * H_kv * page_bounds_bytes(d);
}

int moda_kv_write_e4m3(void* pages, void* bounds, const void* K, const void* V, const int* block_table, const int* start, const int* n_new,
                       int B, int T, int page_size, int num_pages, int max_blocks_per_seq, int H_kv, int d, void* stream) {
    if (int rc = check_pages(B, page_size, num_pages, max_blocks_per_seq, H_kv, d)) return rc;
    dim3 grid;
    if (int rc = pages_rows_grid(B, T, H_kv, &grid)) return rc;
    if (!pages || !K || !V || !block_table) return MODA_ERR_NULL_POINTER;
    if (!aligned16(pages) || !aligned16(bounds) || !aligned16(K) || !aligned16(V) || !aligned4(block_table) || !aligned4(start) || !aligned4(n_new))
        return MODA_ERR_MISALIGNED;
    if (int rc = check_device()) return rc;
    PagesRowsParams p = {};
    set_pages(p, block_table, B, H_kv, page_size, num_pages, max_blocks_per_seq);
    p.pages = static_cast<uint8_t*>(pages); p.bounds = static_cast<uint8_t*>(bounds);
    p.K = static_cast<const uint4*>(K); p.V = static_cast<const uint4*>(V); p.start = start; p.count = n_new; p.T = T;
    return launch_pages(d == 128 ? pages_write_kernel<128> : pages_write_kernel<64>, grid, kPagesThreads, 0, p, static_cast<cudaStream_t>(stream));
}

int moda_kv_read_e4m3(const void* pages, const int* block_table, const int* seq_lens, const int* start,
                      int B, int T, int page_size, int num_pages, int max_blocks_per_seq, int H_kv, int d, void* K_out, void* V_out, void* stream) {
    if (int rc = check_pages(B, page_size, num_pages, max_blocks_per_seq, H_kv, d)) return rc;
    dim3 grid;
    if (int rc = pages_rows_grid(B, T, H_kv, &grid)) return rc;
    if (!pages || !block_table || !seq_lens || !K_out || !V_out) return MODA_ERR_NULL_POINTER;
    if (!aligned16(pages) || !aligned16(K_out) || !aligned16(V_out) || !aligned4(block_table) || !aligned4(start) || !aligned4(seq_lens))
        return MODA_ERR_MISALIGNED;
    if (int rc = check_device()) return rc;
    PagesRowsParams p = {};
    set_pages(p, block_table, B, H_kv, page_size, num_pages, max_blocks_per_seq);
    p.pages = static_cast<uint8_t*>(const_cast<void*>(pages));
    p.K = static_cast<const uint4*>(K_out); p.V = static_cast<const uint4*>(V_out); p.start = start; p.count = seq_lens; p.T = T;
    return launch_pages(d == 128 ? pages_read_kernel<128> : pages_read_kernel<64>, grid, kPagesThreads, 0, p, static_cast<cudaStream_t>(stream));
}

size_t moda_kv_select_workspace_bytes(int B, int max_seq_len, int H_kv) {
    if (B < 1 || H_kv < 1 || max_seq_len < 0 || pages_blocks(max_seq_len) > kSelectMostBlocks) return 0;
    return (size_t(B) * H_kv * std::max(pages_blocks(max_seq_len), 1) * 4 + 15) / 16 * 16;
}

int moda_kv_select_blocks(const void* q, const void* bounds, const int* block_table, const int* seq_lens,
                          int B, int max_seq_len, int page_size, int num_pages, int max_blocks_per_seq, int H, int H_kv, int d,
                          int n_blocks, int n_recent, int* index, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_pages(B, page_size, num_pages, max_blocks_per_seq, H_kv, d)) return rc;
    if (H < 1 || max_seq_len < 0 || max_seq_len > max_blocks_per_seq * page_size || pages_blocks(max_seq_len) > kSelectMostBlocks) return MODA_ERR_BAD_SHAPE;
    if (n_blocks < 1 || n_recent < 0 || n_recent > n_blocks || (long long)B * H_kv > 0x7fffffffLL / n_blocks) return MODA_ERR_BAD_SHAPE;
    if (int rc = check_groups(H, H_kv)) return rc;
    if (!q || !bounds || !block_table || !seq_lens || !index) return MODA_ERR_NULL_POINTER;
    if (!aligned16(q) || !aligned16(bounds) || !aligned4(block_table) || !aligned4(seq_lens) || !aligned4(index)) return MODA_ERR_MISALIGNED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < moda_kv_select_workspace_bytes(B, max_seq_len, H_kv)) return MODA_ERR_WORKSPACE;
    if (int rc = check_device()) return rc;
    int sms = 0;
    if (int rc = device_sm_count(&sms)) return rc;
    PagesSelectParams p = {};
    set_pages(p, block_table, B, H_kv, page_size, num_pages, max_blocks_per_seq);
    p.q = static_cast<const __nv_bfloat16*>(q); p.bounds = static_cast<const uint8_t*>(bounds); p.lens = seq_lens; p.index = index;
    p.rating = static_cast<uint32_t*>(workspace);
    p.G = H / H_kv; p.max_len = max_seq_len; p.n_keep = n_blocks; p.n_recent = n_recent;
    p.most = std::max(pages_blocks(max_seq_len), 1);                                    // a grid has a part, also where no sequence has a block
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d == 128 ? launch_select<128>(p, sms, st) : launch_select<64>(p, sms, st);
}

size_t moda_decode_e4m3_workspace_bytes(int B, int H, int H_kv, int d) {
    if (B < 1 || B > kPagesMostBatch || H < 1 || check_groups(H, H_kv) || (d != 64 && d != 128)) return 0;
    return pages_workspace_bytes(B, H, H_kv, d);
}

int moda_attn_decode_e4m3(const void* q, const void* pages, const int* block_table, const int* seq_lens, const int* index, int n_blocks,
                          const void* depth_kv_token,
                          int B, int max_seq_len, int page_size, int num_pages, int max_blocks_per_seq, int H, int H_kv, int d, int l, float scale,
                          void* O, float* LSE, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_pages(B, page_size, num_pages, max_blocks_per_seq, H_kv, d)) return rc;
    if (H < 1 || max_seq_len < 0 || max_seq_len > max_blocks_per_seq * page_size || B > kPagesMostBatch) return MODA_ERR_BAD_SHAPE;
    if (int rc = check_scale(scale)) return rc;
    if (int rc = check_groups(H, H_kv)) return rc;
    if (index && (n_blocks < 1 || (long long)B * H_kv > 0x7fffffffLL / n_blocks)) return MODA_ERR_BAD_SHAPE;
    if ((long long)B * H > 0x7fffffffLL / std::max(pages_blocks(max_seq_len), 1)) return MODA_ERR_BAD_SHAPE;
    if (l < 0 || l > MODA_MAX_DEPTH) return MODA_ERR_BAD_DEPTH;
    if (!q || !pages || !block_table || !seq_lens || !O || !LSE || (l > 0 && !depth_kv_token)) return MODA_ERR_NULL_POINTER;
    if (!aligned16(q) || !aligned16(pages) || !aligned16(O) || !aligned16(LSE) || !aligned4(block_table) || !aligned4(seq_lens) || !aligned4(index) ||
        (l > 0 && !aligned16(depth_kv_token)))
        return MODA_ERR_MISALIGNED;
    if (!workspace || !aligned16(workspace) || workspace_bytes < pages_workspace_bytes(B, H, H_kv, d)) return MODA_ERR_WORKSPACE;
    if (int rc = check_device()) return rc;
    int sms = 0;
    if (int rc = device_sm_count(&sms)) return rc;
    PagesDecodeParams p = {};
    p.kv_rep = H / H_kv > 8 ? H / H_kv / 8 : 1;
    set_pages(p, block_table, B, H_kv, page_size, num_pages, max_blocks_per_seq);
    p.q = static_cast<const __nv_bfloat16*>(q); p.pages = static_cast<const uint8_t*>(pages); p.lens = seq_lens; p.index = index;
    p.depth = static_cast<const __nv_bfloat16*>(depth_kv_token); p.O = static_cast<__nv_bfloat16*>(O); p.LSE = LSE;
    p.G = H / H_kv / p.kv_rep; p.H = H; p.l = l; p.max_len = max_seq_len; p.n_index = n_blocks;
    p.part = static_cast<float*>(workspace);
    p.before = reinterpret_cast<int*>(static_cast<uint8_t*>(workspace) + pages_part_bytes(B, H, p.G, d));
    p.warps = std::min(sms, kPagesMostCtas) * pages_split_warps(d);
    p.scale_log2 = scale * kDecodeLog2e;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d == 128 ? launch_decode_pages<128>(p, st) : launch_decode_pages<64>(p, st);
}

}  // extern "C"
