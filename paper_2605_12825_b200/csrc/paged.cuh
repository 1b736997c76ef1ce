// Declarations of the paged-cache calls: what their translation units share.
#pragma once
#include <cuda.h>
#include <atomic>
#include "common.cuh"

namespace orthrus {

struct PageTablesParams {
    int B, page_shift, n_pages, max_pages, max_new;
    const int32_t *cache_len, *n_new, *held_in;
    int32_t *held_out, *table, *free_list;
    const int32_t *n_free_in;
    int32_t *n_free_out, *granted;
    int64_t *slot_map;
    int32_t *status;
};
cudaError_t launch_page_tables(const PageTablesParams &p, cudaStream_t st);

cudaError_t launch_paged_kv_write(const orthrus_paged_layer_t &L, const int64_t *slot_map, const void *q, const void *k_blk,
                                  const void *v_blk, double theta, void *q_out, int32_t *status, cudaStream_t st);   // q null: no rotation

// Attention over pages.  A unit is (request, KV head, tile of query rows); rows of a request are ordered
// r = i * G + g as in AttnParams.
struct PagedParams {
    const void *q, *k_pages, *v_pages;
    const int32_t *table, *cache_len, *n_new;
    void *out;
    int32_t *status;
    int B, K, Hq, Hkv, G, d;
    int page_shift, max_pages;
    long long n_pages;
    int max_pos;            // max_pages * page_size
    int causal;
    float scale_log2;
    int early, quiescent;   // launch as a programmatic dependent; first tiles ahead of the preceding kernel
};
int small_rows_knob();                      // ORTHRUS_TC_SMALL_ROWS: 0, 1, or -1 where it is not set
bool simt_forced();                         // orthrus_set_path("simt")
void set_last_path(const char *name);       // what orthrus_last_path() answers on this thread; a literal
bool paged_simt_shape(const orthrus_paged_layer_t &L);       // its grid can be launched
size_t paged_simt_workspace_bytes(const orthrus_paged_layer_t &L);
cudaError_t launch_paged_attend_simt(const PagedParams &p, const orthrus_paged_layer_t &L, void *ws_body, cudaStream_t st);
bool paged_tc_shape(const orthrus_paged_layer_t &L);        // the tensor-core kernel serves this shape
size_t paged_tc_workspace_bytes(const orthrus_paged_layer_t &L);
cudaError_t launch_paged_attend_tc(const PagedParams &p, const orthrus_paged_layer_t &L, void *ws_body, cudaStream_t st);

int paged_keys_splits(const orthrus_paged_layer_t &L, int max_len);       // attend_keys.cu: few query rows, where latency counts
cudaError_t launch_paged_attend_keys(const PagedParams &p, int S, cudaStream_t st);
// a pool as [rows][d], boxes of `box` rows and 64 columns, 128-byte swizzle
bool page_map(const void *ptr, unsigned d, unsigned long long rows, unsigned box, CUtensorMap *out);

// Prefix length and rows of request b, clamped to what the layer can hold (`bad`: they had to be).  Read past L1, where a look ahead of
// the wait for the preceding kernel could have left what that kernel then changed.
__device__ inline void paged_request(const PagedParams &p, int b, int &P, int &n, bool &bad)
{
    P = __ldcg(p.cache_len + b);
    const int given = p.n_new ? __ldcg(p.n_new + b) : p.K;
    n = min(max(given, 0), min(p.K, p.max_pos));
    bad = n != given;
    bad |= P < 0 || P > p.max_pos - n;
    P = min(max(P, 0), p.max_pos - n);
}

// Query rows (G to a position, the first at position `pos0`) in front of the first that sees key `key` of a causal call; keys up to some 64
// positions behind pos0.  All rows see a key of the prefix; how far in front it lies, times G, need not fit 31 bits.
__host__ __device__ inline int rows_before_key(int key, int pos0, int G) { return key > pos0 ? (key - pos0) * G : 0; }

// Pieces that have arrived of a unit that is cut over CTAs.  The counts are in the workspace's header behind the status word, six of five bits in
// a word, because a workspace may serve calls of other shapes and kinds in between, which write anything to the rest of it.  They are zero
// between calls.
constexpr int kMostPieces = 31, kCounts = (kHeaderBytes / 4 - 1) * 6;
// One more of the n pieces (at most kMostPieces) of count i: is it the last?  By one thread; releases what a barrier before has gathered of its
// block's stores, acquires what the others have released.
__device__ inline bool last_piece(int32_t *header, int i, int n)
{
    int32_t *word = header + 1 + i / 6;
    const int shift = i % 6 * 5;
    uint32_t before;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], %2;" : "=r"(before) : "l"(word), "r"(1u << shift) : "memory");
    const bool last = (int)(before >> shift & 31) == n - 1;
    if (last) atomicSub(reinterpret_cast<uint32_t *>(word), (uint32_t)n << shift);
    return last;
}

cudaError_t launch_sample_tokens(const void *logits, int dtype, int rows, int vocab, long long stride, const float *temperature,
                                 const int32_t *top_k, const float *top_p, const float *min_p, const float *u, int32_t *token,
                                 float *logprob, cudaStream_t st);

// launch_kernel in clusters of C CTAs along x
template <class... Params, class... Args>
cudaError_t launch_clusters(bool early, int C, void (*kernel)(Params...), dim3 grid, unsigned threads, size_t smem,
                            cudaStream_t st, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = C; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = early && early_launch_allowed() ? 2 : 1;
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
}

// Attributes of a kernel, set once per device.  `done`: a static of the caller's, one bit per device.
template <class Kernel>
cudaError_t configure(Kernel *kernel, std::atomic<uint64_t> &done, int smem, bool wide_clusters)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1)) return cudaSuccess;
    if (smem > 48 * 1024 && (e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return e;
    if (wide_clusters && (e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1)) != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
    return cudaSuccess;
}

}  // namespace orthrus
